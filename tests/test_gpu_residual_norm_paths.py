"""The boundary's kernels by how they reach their rows: as whole 16-byte pieces, ahead of their use (aligned rows), past the caches
as well (large calls), or by elements.  Every option meets every path, in place too, over more rows than a grid holds at
once; large calls' sums over the rows are held to 64-bit ones."""

import numpy as np
import pytest
import torch

from tests import block_ref as R
from tests import test_gpu_residual_norm as T
from tests.gpu_util import flush

BF, F4 = torch.bfloat16, torch.float32
E = R.E

# gain, shift, gate, alpha, beta, p
OPTIONS = [(True, True, True, 0.7, 1.0, 0.2), (False, False, False, 1.0, 1.0, 0.0), (True, False, True, 0.7, -0.5, 0.0),
           (False, True, False, 1.0, -0.5, 0.3)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF, F4])
@pytest.mark.parametrize("pre", [None, "layer", "rms"])
@pytest.mark.parametrize("post", [None, "layer", "rms"])
@pytest.mark.parametrize("d", [64, 264])  # rows on lanes, and on waves
def test_options(pre, post, dt, d):
    """Rows of an aligned buffer and of one that is not; in place and not, with and without a gradient along the stream."""
    for i, (gain, shift, gate, alpha, beta, p) in enumerate(OPTIONS):
        for width in (8 * (i % 3), 5):
            for inplace, nody in ((True, False), (False, True), (False, False)):
                T._case(21, d, dt, pre, post, gain, shift, gate, alpha, beta, p, width, inplace, nody)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF, F4])
@pytest.mark.parametrize("rows,d", [(33001, 64), (17000, 128), (9001, 256), (4500, 264), (1400, 1280), (530, 3584), (600, 4096), (300, 6152), (300, 8192)])
def test_more_rows_than_a_grid(rows, d, dt):
    """In place, where the next rows are read before a row is written."""
    for width in (8, 5):
        T._case(rows, d, dt, "layer", "rms", width=width, inplace=True)
        T._case(rows, d, dt, "rms", None, p=0.0, width=width, inplace=True, beta=0.5)


# ---------------------------------------------------------------- sums of large calls

def sums(dy, dh, y, f, st, o, adds):
    """{name: (value, bound)} of the five sums over rows, as block_ref.residual_bwd, on tensors of 64 bits and without dropout."""
    d = y.shape[1]
    out = {}

    def total(name, terms, off):
        out[name] = (terms.sum(0), off.sum(0) + (adds + 2) * E * terms.abs().sum(0))

    def back(g, off, a, mean, rstd, kind, gain):
        xh = (a - mean) * rstd
        oxh = 4 * E * (xh.abs() + (mean * rstd).abs())
        b, ob = g * gain, off * gain.abs() + 2 * E * (g * gain).abs()
        m0 = b.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(mean)
        o0 = ob.mean(1, keepdim=True) + 34 * E * b.abs().mean(1, keepdim=True)
        m1 = (b * xh).mean(1, keepdim=True)
        o1 = (ob * xh.abs() + b.abs() * oxh).mean(1, keepdim=True) + 36 * E * (b * xh).abs().mean(1, keepdim=True)
        value = rstd * (b - m0 - xh * m1)
        return value, rstd * (ob + o0 + xh.abs() * o1 + oxh * m1.abs() + 6 * E * (b.abs() + m0.abs() + (xh * m1).abs())), xh, oxh

    m0, r0, m1, r1 = (s[:, None] for s in st)
    one, none = torch.ones(d, dtype=y.dtype, device=y.device), torch.zeros(d, dtype=y.dtype, device=y.device)
    g, og, yh, oyh = back(dh, torch.zeros_like(dh), y, m1, r1, o["pre"], o["g_pre"])
    total("dg_pre", dh * yh, dh.abs() * oyh + E * (dh * yh).abs())
    total("db_pre", dh, torch.zeros_like(dh))
    t, ot = dy + g, og + E * (dy + g).abs() + E * g.abs()
    tm = o["beta"] * t
    otm = abs(o["beta"]) * ot + 4 * E * tm.abs()
    u, ou = f, torch.zeros_like(f)
    gain, shift = (o["g_post"], o["b_post"]) if o["post"] else (one, none)
    xh0 = (f - m0) * r0
    if o["post"]:
        u = xh0 * gain + shift
        ou = 8 * E * (gain.abs() * (xh0.abs() + (m0 * r0).abs()) + shift.abs())
    total("dgate", tm * u, otm * u.abs() + tm.abs() * ou + E * (tm * u).abs())
    if o["post"]:
        du = tm * o["gate"]
        odu = otm * o["gate"].abs() + E * du.abs()
        oxh = 4 * E * (xh0.abs() + (m0 * r0).abs())
        total("dg_post", du * xh0, odu * xh0.abs() + du.abs() * oxh + E * (du * xh0).abs())
        total("db_post", du, odu)
    return out


@pytest.mark.parametrize("pre,post", [("layer", "rms"), ("rms", "layer"), ("layer", None)])
def test_sums_are_the_reference(pre, post):
    rng = np.random.default_rng(5)
    rows, d = 40, 24
    o = dict(pre=pre, post=post, g_pre=rng.normal(size=d), b_pre=rng.normal(size=d), g_post=rng.normal(size=d) if post else None,
             b_post=rng.normal(size=d) if post else None, gate=rng.normal(size=d), alpha=0.5, beta=0.75, eps=1e-5, p=0.0, seed=0, step=0)
    y, f, dy, dh = (rng.normal(size=(rows, d)) + 0.5 for _ in range(4))
    st = np.zeros((4, rows))
    if post:
        st[:2] = R.stats(f, post, 1e-5)
    st[2:] = R.stats(y, pre, 1e-5)
    want = R.residual_bwd(dy, dh, y, f, st, o, 9)
    c = lambda v: torch.as_tensor(v) if isinstance(v, np.ndarray) else v  # noqa: E731
    for k, pair in sums(*(c(a) for a in (dy, dh, y, f, st)), {n: c(v) for n, v in o.items()}, 9).items():
        for a, b in zip(pair, want[k]):
            assert np.allclose(a.numpy(), b, rtol=1e-12, atol=1e-15), k


@pytest.mark.gpu
@pytest.mark.parametrize("dt,post,rows,d", [
    (BF, "rms", 20011, 1280), (BF, None, 22011, 1280), (F4, "layer", 14001, 1280), (BF, "layer", 6011, 4096), (F4, "rms", 4003, 4096),
    (F4, None, 5003, 4096), (BF, "layer", 2571, 8192), (F4, "rms", 2003, 8192), (BF, "rms", 80021, 264), (F4, "layer", 300007, 64)])
def test_sums_of_large_calls(dt, post, rows, d):
    """Past the size where rows go past the caches (narrow rows: a call as large), dx in place of dy: all five sums."""
    from paper_2309_01226_amd import ops
    flush("sums of large calls", dt, post, rows, d)
    wide = rows * d * (3 * (2 if dt is BF else 4) + 6)
    assert wide >= 240000000
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    y, dy = (2 * r(rows, d) + r(rows, 1)).to(dt), (r(rows, d) + 0.1).to(dt)
    f, dh = (r(rows, d) + 0.5 * r(rows, 1)).to(BF), (r(rows, d) + 0.1).to(BF)
    o = dict(pre="layer", post=post, gate=r(d), alpha=0.5, beta=0.75)
    names = ["g_pre", "b_pre"] + (["g_post", "b_post"] if post else [])
    o.update({n: (n[0] == "g") + 0.3 * r(d) for n in names})
    st = torch.zeros(4, rows, device="cuda")
    for i, (a, kind) in enumerate(((f, post), (y, "layer"))):
        if kind:
            a = a.double()
            mean = a.mean(1) if kind == "layer" else torch.zeros(rows, device="cuda", dtype=torch.float64)
            st[2 * i], st[2 * i + 1] = mean, 1 / ((a - mean[:, None]).square().mean(1) + 1e-5).sqrt()
    c = lambda t: t.double() if torch.is_tensor(t) else t  # noqa: E731
    want = {}
    for at in torch.arange(rows, device="cuda").split(4096):  # a few rows at a time
        part = sums(*(a[at].double() for a in (dy, dh, y, f)), st[:, at].double(), {k: c(v) for k, v in o.items()}, T._adds(rows, d))
        for k, v in part.items():
            want[k] = tuple(p + q for p, q in zip(want[k], v)) if k in want else v
    got = {k: torch.full((d,), 7.0, device="cuda") for k in want}
    ops.residual_norm_bwd(dy, dh, y, f, st, dy, torch.empty_like(f), d, **got, **o)
    torch.cuda.synchronize()
    assert set(got) == {"dg_pre", "db_pre", "dgate"} | ({"dg_post", "db_post"} if post else set())
    for k, (value, bound) in want.items():
        off = (got[k].double() - value).abs() / (bound + E * (value.abs() + bound))
        assert off.max().item() <= 1, (k, off.max().item(), int(off.argmax()))
