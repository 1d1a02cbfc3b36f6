"""64-bit forms of the operators around a step's blocks (numpy, written from their definitions), with bounds on
the error that fp32 arithmetic in the kernels' order may make."""

import numpy as np

E = 2.0 ** -24  # half a step of fp32


# ---------------------------------------------------------------- dropout

def philox(counter, key):
    """Philox4x32-10: four arrays of 32-bit words (as uint64) of a counter's four and a key's two."""
    c = [np.asarray(x, np.uint64) for x in counter]
    k = [int(x) for x in key]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), q & low, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(rows, cols, p, seed, step=0, row0=0):
    """(mask [rows, cols], factor as fp32) of dropout."""
    t = int(np.rint(65536 * p))
    n = -(-cols // 8)
    q, r = np.meshgrid(np.arange(n, dtype=np.uint64), np.arange(row0, row0 + rows, dtype=np.uint64))
    w = philox([q, r, np.full_like(q, step & 0xFFFFFFFF), np.full_like(q, step >> 32)], [seed & 0xFFFFFFFF, seed >> 32])
    halves = np.stack([h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))], -1).reshape(rows, 8 * n)
    return halves[:, :cols] >= t, np.float32(65536 / (65536 - t) if t < 65536 else 0)


# ---------------------------------------------------------------- residual norm

def stats(a, kind, eps):
    mean = a.mean(1) if kind == "layer" else np.zeros(len(a))
    return mean, 1 / np.sqrt(((a - mean[:, None]) ** 2).mean(1) + eps)


def _or(x, v):
    return np.float64(v) if x is None else x


def factors(T, d, o):
    """beta m of dropout, and whether an element is kept."""
    if not o["p"]:
        return np.full((T, d), o["beta"]), np.ones((T, d), bool)
    keep, up = kept(T, d, o["p"], o["seed"], o["step"])
    return np.where(keep, o["beta"] * np.float64(up), 0.0), keep & (up > 0)


def _normed(a, st, kind, gain, shift):
    """The norm's outcome and a bound on its fp32 error: 31 additions at most lie between an element and a row's
    sum (8 in a thread, 6 in a wave, 16 waves, one more), so a mean is off by 31 E of the mean magnitude, a reciprocal
    deviation by half of 40 E and a step of two; an outcome takes six more roundings."""
    mean, rstd = st
    xh = (a - mean[:, None]) * rstd[:, None]
    size = np.abs(xh) + (np.abs(a).mean(1) * rstd)[:, None] * (kind == "layer") + np.abs(mean * rstd)[:, None]
    out = xh * _or(gain, 1) + _or(shift, 0)
    return out, 64 * E * (np.abs(_or(gain, 1)) * size + np.abs(_or(shift, 0)))


def residual_fwd(x, f, o):
    """(y, its bound, statistics of f)."""
    T, d = x.shape
    u, off, st = f, 0.0, None
    m, keep = factors(T, d, o)
    if o["post"]:
        st = stats(f, o["post"], o["eps"])
        u, off = _normed(f, st, o["post"], o["g_post"], o["b_post"])
    k = m * _or(o["gate"], 1)
    with np.errstate(invalid="ignore"):
        b = np.where(keep, k * u, 0.0)
    return o["alpha"] * x + b, 8 * E * (np.abs(o["alpha"] * x) + np.abs(b)) + np.abs(k) * off, st


def residual_next(y, o):
    """(h, its bound, statistics) of the stream as it is stored."""
    st = stats(y, o["pre"], o["eps"])
    return (*_normed(y, st, o["pre"], o["g_pre"], o["b_pre"]), st)


def _norm_back(g, off, a, st, kind, gain):
    """Gradient through a norm and its bound, from g and g's."""
    mean, rstd = st
    xh = (a - mean[:, None]) * rstd[:, None]
    oxh = 4 * E * (np.abs(xh) + np.abs(mean * rstd)[:, None])
    b = g * _or(gain, 1)
    ob = off * np.abs(_or(gain, 1)) + 2 * E * np.abs(b)
    m0 = b.mean(1, keepdims=True) if kind == "layer" else 0.0
    o0 = ob.mean(1, keepdims=True) + 34 * E * np.abs(b).mean(1, keepdims=True)
    m1 = (b * xh).mean(1, keepdims=True)
    o1 = (ob * np.abs(xh) + np.abs(b) * oxh).mean(1, keepdims=True) + 36 * E * np.abs(b * xh).mean(1, keepdims=True)
    r = rstd[:, None]
    out = r * (b - m0 - xh * m1)
    bound = r * (ob + o0 + np.abs(xh) * o1 + oxh * np.abs(m1) + 6 * E * (np.abs(b) + np.abs(m0) + np.abs(xh * m1)))
    return out, bound, xh, oxh


def residual_bwd(dy, dh, y, f, st, o, adds):
    """{name: (value, bound)} of the backward; st: [4, T]; adds: additions between a row's term and a sum over rows."""
    T, d = dy.shape
    out = {}
    t, ot = dy, np.zeros_like(dy)

    def total(name, terms, off):
        out[name] = (terms.sum(0), off.sum(0) + (adds + 2) * E * np.abs(terms).sum(0))

    if o["pre"]:
        g, og, yh, oyh = _norm_back(dh, 0.0, y, st[2:], o["pre"], o["g_pre"])
        t, ot = dy + g, og + E * np.abs(dy + g) + E * np.abs(g)
        total("dg_pre", dh * yh, np.abs(dh) * oyh + E * np.abs(dh * yh))
        total("db_pre", dh, np.zeros_like(dh))
    out["dx"] = (o["alpha"] * t, np.abs(o["alpha"]) * ot + 2 * E * np.abs(o["alpha"] * t))
    m, keep = factors(T, d, o)
    gate = _or(o["gate"], 1)
    tm = np.where(keep, t * m, 0.0)
    otm = np.abs(m) * ot + 4 * E * np.abs(tm)
    if o["post"]:
        xh0 = (f - st[0][:, None]) * st[1][:, None]
        u = xh0 * _or(o["g_post"], 1) + _or(o["b_post"], 0)
        ou = 8 * E * (np.abs(_or(o["g_post"], 1)) * (np.abs(xh0) + np.abs(st[0] * st[1])[:, None]) + np.abs(_or(o["b_post"], 0)))
    else:
        u, ou = f, np.zeros_like(f)
    with np.errstate(invalid="ignore"):
        total("dgate", np.where(keep, tm * u, 0.0), np.where(keep, otm * np.abs(u) + np.abs(tm) * ou + E * np.abs(tm * u), 0.0))
    du, odu = tm * gate, otm * np.abs(gate) + E * np.abs(tm * gate)
    if o["post"]:
        g, og, xh, oxh = _norm_back(du, odu, f, st[:2], o["post"], o["g_post"])
        total("dg_post", du * xh, odu * np.abs(xh) + np.abs(du) * oxh + E * np.abs(du * xh))
        total("db_post", du, odu)
        du, odu = g, og
    out["df"] = (du, odu)
    return out


# ---------------------------------------------------------------- head with cross entropy

def head(x, w, labels, bias=None, weight=None, grads=True):
    """{name: (value, bound)} of the linear head's cross entropy, torch tensors in 64 bits on any device (x, w, bias
    and weight 64-bit, labels int64; rows whose label is outside the vocabulary take no part).

    Bounds.  A logit is a sum of d products in fp32, at most d + 2 roundings of E each (twice that if they are not to
    the nearest).  exp2 of a product by log2 e: 2^-22 and 4 E |z - m|; a row's sum and its joining: at most 64 + 2
    in a lane pair, 32 + 16 pieces, the pieces' factors: 256 E in all.  The gradients' operand is rounded to bf16 twice
    (2^-8 each), the label's once; a product's sum of n terms is off by (n + 2) 2 E of their magnitudes."""
    import torch
    N, (V, d) = len(labels), w.shape
    live = (labels >= 0) & (labels < V)
    at = torch.where(live, labels, 0)[:, None]
    z = x @ w.T
    oz = 2 * E * (d + 2) * (x.abs() @ w.abs().T)
    if bias is not None:
        z = z + bias
        oz = oz + E * torch.where(bias.isinf(), 0.0, bias.abs()) + E * torch.where(z.isinf(), 0.0, z.abs())
    lse = torch.logsumexp(z, 1, keepdim=True)
    empty = lse.isinf()
    p = torch.where(empty, 0.0, torch.exp(z - torch.where(empty, 0.0, lse)))
    far = torch.where(z.isinf(), 0.0, (z - z.amax(1, keepdim=True)).abs())
    op = oz + 4 * E * far + 2.0 ** -22       # relative error of exp(z - m)
    ol = (p * op).sum(1, keepdim=True) + 256 * E  # of lse
    zl, ozl = z.gather(1, at), oz.gather(1, at)
    use = live & ~empty[:, 0]
    out = {}
    loss = torch.where(use, (lse - zl)[:, 0], 0.0)
    top = (z.amax(1, keepdim=True) - zl).abs()
    out["lse"] = (torch.where(live, lse[:, 0], 0.0), (ol + 4 * E * torch.where(empty, 0.0, lse.abs()))[:, 0])
    out["row_loss"] = (loss, torch.where(use, (ol + ozl + 4 * E * top)[:, 0], 0.0) + 4 * E * loss.abs())
    n = int(live.sum())
    out["inv_n"] = (torch.tensor([1 / max(n, 1)], dtype=torch.float64, device=x.device), torch.tensor([2 * E], device=x.device))
    if not grads:
        return out
    c = (torch.full((N,), 1 / max(n, 1), dtype=torch.float64, device=x.device) if weight is None else weight) * use
    hot = torch.zeros_like(p).scatter_(1, at, 1.0)
    dz = c[:, None] * (p - hot)
    soft = c.abs()[:, None] * p * (op + ol + 8 * E)  # of c p before roundings
    two = torch.where(hot > 0, 2.0 ** -8 * dz.abs(), 2.0 ** -7 * 1.01 * dz.abs())
    odz = (soft + 4 * E * (c.abs()[:, None] * hot)) * 1.01 + two
    tiny = 2.0 ** -126
    total = lambda a, b, oa, k: (a @ b, oa @ b.abs() + 2 * E * (k + 2) * (a.abs() @ b.abs()) + tiny)  # noqa: E731
    out["dx"] = total(dz, w, odz, V)
    out["dw"] = total(dz.T.contiguous(), x, odz.T.contiguous(), N)
    odb = soft * 1.01 + 4 * E * (c.abs()[:, None] * hot) + torch.where(hot > 0, 0.0, 2.0 ** -8 * 1.01 * dz.abs())
    out["db"] = (dz.sum(0), odb.sum(0) + E * (N + 2) * dz.abs().sum(0) + tiny)
    return out
