"""delta of the packed backward, whether its work is split among workgroups (with scratch) or not.

Heads of up to 128 dims: dK and dV take delta = sum P dP in fp32, and so does dQ where a query sees
no more than 128 keys of its block; nothing there goes by the bf16 o.  So the bound has no term for o's rounding:
  err(p)     E p,  E = (dh + 16) 2^-24 max(1, scale sum |q| |k|), the fp32 score, its exponential and lse
  err(dP)    E |dO| |v|;  err(delta) = sum over the keys of 2 E p |dO| |v|
  err(dS)    (u + 2 E) |dS| + 2 E p (|dO| |v| + sum p |dO| |v|),  u = 2^-8 for its rounding to bf16
  dk         scale err(dS)^T |q| + u |dk|;  dq likewise
Rows of v that differ by one step of bf16 make every dS small, and o lies between two
neighbours of bf16, so that an error of delta by o's rounding stands out."""

import ctypes as C

import pytest
import torch

from tests import packed_ref as R
from tests.gpu_util import flush
from tests.test_gpu_attention_packed import _make

pytestmark = pytest.mark.gpu


def _alike(s):
    """Rows of v one of two neighbours in bf16 in each sequence, dO = +- one of them, scores of about 1."""
    G = s["H"] // s["Hkv"]
    g = torch.Generator(device="cuda").manual_seed(9)
    s["q"].mul_(0.25)
    for a, b in zip(s["rows"], s["rows"][1:]):
        if b > a:
            one = s["v"][a:a + 1].clone()
            up = torch.randint(0, 2, (b - a, 1), device="cuda", generator=g, dtype=torch.int16)
            s["v"][a:b] = (one.view(torch.int16) + up).view(torch.bfloat16)
            v = one.reshape(1, s["Hkv"], 1, s["dh"]).expand(b - a, -1, G, -1)
            sign = torch.randint(0, 2, (b - a, s["H"], 1), device="cuda", generator=g) * 2 - 1
            s["dout"][a:b] = (v.reshape(b - a, s["H"], s["dh"]) * sign).reshape(b - a, -1)


def _bounds(s, causal, window, scale):
    """Exact dq, dk, dv and their bounds."""
    want, _ = R.attention(s["q"], s["k"], s["v"], s["rows"], s["H"], s["Hkv"], s["dh"], causal, scale, window, s["dout"])
    err = {n: torch.zeros_like(want[n]) for n in ("dq", "dk", "dv")}
    dh, G = s["dh"], s["H"] // s["Hkv"]
    for a, b in zip(s["rows"], s["rows"][1:]):
        if b <= a:
            continue
        ok = R.allowed(b - a, causal, window, "cuda")
        for h in range(s["H"]):
            c, ck = slice(h * dh, h * dh + dh), slice(h // G * dh, h // G * dh + dh)
            q, do = s["q"][a:b, c].double(), s["dout"][a:b, c].double()
            k, v = s["k"][a:b, ck].double(), s["v"][a:b, ck].double()
            size = (q.abs() @ k.abs().T * scale).masked_fill(~ok, 0).max()
            E = (dh + 16) * 2.0 ** -24 * max(1.0, float(size))
            p = torch.softmax((q @ k.T * scale).masked_fill(~ok, float("-inf")), 1)
            dP, A = do @ v.T, do.abs() @ v.abs().T
            dS = p * (dP - (p * dP).sum(1, keepdim=True))
            e = (R.U + 2 * E) * dS.abs() + 2 * E * p * (A + (p * A).sum(1, keepdim=True))
            err["dq"][a:b, c] += scale * e @ k.abs()
            err["dk"][a:b, ck] += scale * e.T @ q.abs()
            err["dv"][a:b, ck] += (R.U + E) * (p.T @ do.abs())
    for n in err:
        err[n] += R.U * want[n].abs() * (1 + R.U) + 1e-30
    return want, err


def _run(s, causal, window, scale, scratch):
    """Forward and backward; without scratch the backward gets no more than it needs."""
    from paper_2309_01226_amd import _lib, ops
    T, H, Hkv, dh = s["T"], s["H"], s["Hkv"], s["dh"]
    shape = dict(n_seq=len(s["rows"]) - 1, T=T, H=H, Hkv=Hkv, dh=dh, causal=causal, window=window)
    n = C.c_int64()
    _lib.call("sat_op_attention_packed_bwd_ws", _lib.sat_attn_packed_desc(**shape), n)
    least = (H * T + 3) // 4 * 4
    assert n.value > least, "a shape that is not split"
    ws = torch.empty(n.value if scratch else least, device="cuda")
    p = {x: s[x].data_ptr() for x in ("q", "k", "v", "o", "lse", "cu", "dout", "dq", "dk", "dv")}
    ld = {"ld" + x: s[x].stride(0) for x in ("q", "k", "v", "o", "dq", "dk", "dv")}
    d = _lib.sat_attn_packed_desc(**p, **ld, **shape, lddo=s["dout"].stride(0), scale=scale)
    _lib.call("sat_op_attention_packed_fwd", d, ops._stream())
    d.ws, d.ws_elems = ws.data_ptr(), ws.numel()
    _lib.call("sat_op_attention_packed_bwd", d, ops._stream())
    torch.cuda.synchronize()


SHAPES = [([3000], 2, 1, True, 0), ([2500, 70, 0, 130, 1], 2, 2, True, 0), ([2048], 1, 1, False, 0), ([3500], 2, 1, True, 1500)]


@pytest.mark.parametrize("scratch", [True, False])
@pytest.mark.parametrize("alike", [True, False])
@pytest.mark.parametrize("dh", [24, 32, 64, 80, 96, 128])
def test_delta_is_the_sum_of_p_dp(dh, alike, scratch):
    for lens, H, Hkv, causal, window in SHAPES:
        flush("packed delta", dh, alike, scratch, lens, H, Hkv, causal, window)
        s = _make(lens, H, Hkv, dh, seed=dh)
        if alike:
            _alike(s)
        scale = dh ** -0.5
        _run(s, causal, window, scale, scratch)
        want, err = _bounds(s, causal, window, scale)
        few = torch.zeros(s["T"], dtype=torch.bool, device="cuda")  # rows whose blocks see 128 keys at most
        for a, b in zip(s["rows"], s["rows"][1:]):
            few[a:min(a + 128, b) if causal or b - a <= 128 else a] = True
        for n in ("dk", "dv", "dq"):
            off = (s[n].double() - want[n]).abs() - err[n]
            if n == "dq":
                off = off[few]
            assert off.numel() == 0 or float(off.max()) <= 0, (n, lens, float(off.max()))


@pytest.mark.parametrize("dh", [64, 96, 128])
def test_short_sequences_of_a_split_call_keep_their_bits(dh):
    """Blocks whose keys fit two steps are not cut: the same dQ with scratch and without."""
    lens = [2500, 70, 128, 1]
    s, t = (_make(lens, 2, 2, dh, seed=1) for _ in range(2))
    _run(s, True, 0, 0.1, True)
    _run(t, True, 0, 0.1, False)
    assert torch.equal(s["dq"][2500:], t["dq"][2500:])
    assert torch.equal(s["dq"][:128], t["dq"][:128])
