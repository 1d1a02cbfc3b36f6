"""Plain 64-bit forms of the operators on packed rows, with bounds on a kernel's error.

`attention` returns the exact results and, for each, how far a kernel may be that takes bf16
operands, sums in fp32, and rounds p, dS and the results to bf16 (each rounding at most
u = 2^-8 of the value).  With A = p |v|, elementwise:
  o      u A (p) + u |o|                                       <= 2 u A
  delta  sum |dO| err(o), since it is formed from the rounded o =: D
  dv     u p^T |dO| (p) + u |dv|
  dS     u |dS| + p D;  dq = scale dS k: scale err(dS) |k| + u |dq|;  dk likewise
F covers the fp32 part: a score's sum of at most 256 products, its scaling, the exponential and lse
are together less than 2^-10 relative in p for the scores that the tests make (|score| sums
below 2^5: (256 + 16) 2^-24 2^5 = 2^-10.9), and as much of |dP| and delta.
"""

import math

import numpy as np
import torch

U, F = 2.0 ** -8, 2.0 ** -10


def allowed(n, causal, window, device):
    i = torch.arange(n, device=device)
    d = i[:, None] - i[None, :]
    ok = torch.ones(n, n, dtype=torch.bool, device=device)
    if causal:
        ok &= d >= 0
    if window:
        ok &= d.abs() < window
    return ok


def attention(q, k, v, cu, H, Hkv, dh, causal, scale, window=0, dout=None):
    """Exact {name: rows} and {name: bound}; rows outside every sequence are 0 with bound 0."""
    T = q.shape[0]
    q, k, v = q[:, :H * dh].double(), k[:, :Hkv * dh].double(), v[:, :Hkv * dh].double()
    do = None if dout is None else dout[:, :H * dh].double()
    names = ["o"] + ([] if do is None else ["dq", "dk", "dv"])
    shape = dict(o=H, dq=H, dk=Hkv, dv=Hkv)
    out = {n: torch.zeros(T, shape[n] * dh, dtype=torch.float64, device=q.device) for n in names}
    err = {n: torch.zeros_like(t) for n, t in out.items()}
    out["lse"], err["lse"] = (torch.zeros(H, T, dtype=torch.float64, device=q.device) for _ in range(2))
    for a, b in zip(cu, cu[1:]):
        if b <= a:
            continue
        ok = allowed(b - a, causal, window, q.device)
        r = slice(a, b)
        for h in range(H):
            c, ck = slice(h * dh, (h + 1) * dh), slice(h // (H // Hkv) * dh, (h // (H // Hkv) + 1) * dh)
            Q, K, V = q[r, c], k[r, ck], v[r, ck]
            x = (Q @ K.T * scale).masked_fill(~ok, -math.inf)
            lse = torch.logsumexp(x, 1)
            p = torch.exp(x - lse[:, None])
            O = p @ V
            A = p @ V.abs()
            out["o"][r, c], err["o"][r, c] = O, (2 * U + F) * A
            out["lse"][h, r] = lse
            err["lse"][h, r] = 272 * 2.0 ** -24 * (1 + scale * (Q.abs() @ K.T.abs()).masked_fill(~ok, 0).amax(1))
            if do is None:
                continue
            G = do[r, c]
            dP, delta = G @ V.T, (G * O).sum(1, keepdim=True)
            dS = p * (dP - delta)
            D = (G.abs() * err["o"][r, c]).sum(1, keepdim=True)
            eS = U * dS.abs() + p * (D + F * (G.abs() @ V.T.abs() + (G * O).abs().sum(1, keepdim=True)))
            for n, val, e in (("dq", dS @ K * scale, eS @ K.abs() * scale), ("dk", dS.T @ Q * scale, eS.T @ Q.abs() * scale),
                              ("dv", p.T @ G, (U + F) * (p.T @ G.abs()))):
                cc = c if n == "dq" else ck
                out[n][r, cc] += val
                err[n][r, cc] += e
    for n in ("dq", "dk", "dv"):
        if n in out:
            err[n] += U * out[n].abs() * (1 + U) + 1e-30
    return out, err


def angles(pos, pairs, base, own_freqs):
    """[rows, sum(pairs)] in 64 bits."""
    pos = np.asarray(pos, np.float64)
    half = sum(pairs)
    cols, i = [], 0
    for a, n in enumerate(pairs):
        for j in range(n):
            cols.append(pos[:, a] * base ** (-(j / n if own_freqs else i / half)))
            i += 1
    return np.stack(cols, 1)


def rotary(x, pos, H, dh, pairs, base=10000.0, interleaved=True, own_freqs=False, inverse=False):
    x = np.array(x, np.float64)
    ang = angles(pos, pairs, base, own_freqs) * (-1 if inverse else 1)
    c, s = np.cos(ang), np.sin(ang)
    half = sum(pairs)
    for h in range(H):
        y = x[:, h * dh:h * dh + 2 * half].copy()
        u, w = (y[:, 0::2], y[:, 1::2]) if interleaved else (y[:, :half], y[:, half:])
        y2 = np.empty_like(y)
        if interleaved:
            y2[:, 0::2], y2[:, 1::2] = u * c - w * s, u * s + w * c
        else:
            y2[:, :half], y2[:, half:] = u * c - w * s, u * s + w * c
        x[:, h * dh:h * dh + 2 * half] = y2
    return x


def adamw(p, g, m, v, lr, b1, b2, eps, wd, t):
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return p * (1 - lr * wd) - lr / (1 - b1 ** t) * m / (np.sqrt(v) / math.sqrt(1 - b2 ** t) + eps), m, v


def decode(code, exp, mantissa):
    """Values of 8-bit magnitudes (code 0: zero) under the exponents of their 256-element blocks."""
    c = np.asarray(code, np.float64)
    e = np.repeat(np.asarray(exp, np.float64), 256)[:c.size]
    f = 2 ** mantissa
    return np.where(c > 0, (1 + c % f / f) * 2.0 ** (np.floor(c / f) - 15 + e - 127), 0.0)


def moments8(m, v, m_exp, v_exp):
    m = np.asarray(m)
    return np.where(m >= 128, -1.0, 1.0) * decode(m & 127, m_exp, 3), decode(v, v_exp, 4) ** 2
