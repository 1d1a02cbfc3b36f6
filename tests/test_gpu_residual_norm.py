"""The boundary of two sublayers against its 64-bit form; block_ref derives the bounds."""

import math

import numpy as np
import pytest
import torch

from tests import block_ref as R
from tests.gpu_util import flush

pytestmark = pytest.mark.gpu
BF, F4 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F4: 2.0 ** -24}


def _dev(a, dt, width=None, fill=7.0):
    """[rows, columns] of a wider device buffer."""
    rows, d = a.shape
    buf = torch.full((rows, d + (width or 0)), fill, dtype=dt, device="cuda")
    buf[:, :d] = torch.as_tensor(a, dtype=F4).to(dt)
    return buf, buf[:, :d]


def _host(t):
    return t.double().cpu().numpy()


def _check(name, got, want, bound, dt):
    got = _host(got)
    bound = bound + HALF[dt] * (np.abs(want) + bound) + np.finfo(np.float32).tiny
    assert np.isfinite(got).all(), name
    off = np.abs(got - want) / bound
    assert off.max(initial=0) <= 1, (name, float(off.max()), np.unravel_index(off.argmax(), off.shape))


def _options(rng, d, pre, post, gain, shift, gate, alpha, beta, p):
    v = lambda on, a, b: (a + b * rng.normal(size=d)).astype(np.float32) if on else None  # noqa: E731
    return dict(pre=pre, post=post, g_pre=v(pre and gain, 1, 0.3), b_pre=v(pre and shift, 0, 0.3), g_post=v(post and gain, 1, 0.3),
                b_post=v(post and shift, 0, 0.3), gate=v(gate, 0, 0.7), alpha=alpha, beta=beta, eps=1e-5, p=p, seed=12345 << 20, step=3)


def _gpu_options(o):
    g = {k: torch.as_tensor(v).cuda() if isinstance(v, np.ndarray) else v for k, v in o.items()}
    g["step"] = torch.tensor([o["step"]], device="cuda")
    return g


def _wide(o):
    w = {k: v.astype(np.float64) if isinstance(v, np.ndarray) else v for k, v in o.items()}
    return {**w, "alpha": float(np.float32(o["alpha"])), "beta": float(np.float32(o["beta"])), "eps": float(np.float32(o["eps"]))}


def _adds(T, d):
    """Additions between a row's term and its sum over the rows: at least 256 workgroups share the rows where there are more
    than a workgroup holds at once, so a thread adds T / 256 + 1 of them at most; then the rows that a workgroup holds at
    once (12 waves of 8 rows at most), a sixteenth of at most 512 workgroups, and the 16 slices of those."""
    return T // 256 + 1 + 96 + 512 // 16 + 16


def _case(T, d, dt, pre, post, gain=True, shift=True, gate=True, alpha=1.0, beta=1.0, p=0.1, width=0, inplace=False, nody=False):
    from paper_2309_01226_amd import ops
    flush("residual_norm", T, d, dt, pre, post, gain, shift, gate, alpha, beta, p, width, inplace, nody)
    rng = np.random.default_rng((T, d, len(pre or "") * 8 + len(post or "")))
    o = _options(rng, d, pre, post, gain, shift, gate, alpha, beta, p)
    go, w = _gpu_options(o), _wide(o)
    scale = np.exp(0.5 * rng.normal(size=d))
    xb, x = _dev(3 * rng.normal(size=(T, d)) * scale + rng.normal(size=(T, 1)), dt, width)
    fb, f = _dev(rng.normal(size=(T, d)) + 0.5 * rng.normal(size=(T, 1)), BF, width)
    yb, y = (xb, x) if inplace else _dev(np.zeros((T, d)), dt, width)
    hb, h = _dev(np.zeros((T, d)), BF, width) if pre else (None, None)
    st = torch.full((4, T), 7.0, device="cuda")
    xh, fh = _host(x), _host(f)
    ops.residual_norm_fwd(x, f, y, h, st, d, **go)
    torch.cuda.synchronize()
    want, bound, fst = R.residual_fwd(xh, fh, w)
    _check("y", y, want, bound, dt)
    sth = _host(st)

    def stats_near(i, a, kind, ref):
        if not kind:
            assert (sth[2 * i:2 * i + 2] == 7).all()
            return
        assert (np.abs(sth[2 * i] - ref[0]) <= 32 * R.E * np.abs(a).mean(1) + 1e-30).all()
        # (mean's error)^2 joins the variance, far below 40 E of it unless the mean dwarfs it
        lost = 1 + (np.abs(a).mean(1) * ref[1]) ** 2 * 64 * R.E
        assert (np.abs(sth[2 * i + 1] - ref[1]) <= 40 * R.E * lost * ref[1]).all()

    stats_near(0, fh, post, fst)
    if pre:
        want, bound, yst = R.residual_next(_host(y), w)
        _check("h", h, want, bound, BF)
        stats_near(1, _host(y), pre, yst)
    else:
        assert (sth[2:] == 7).all()
    for b in (xb, fb, yb, hb):
        assert b is None or (b[:, d:] == 7).all()

    dyb, dy = _dev(rng.normal(size=(T, d)), dt, width)
    dhb, dh = _dev(rng.normal(size=(T, d)), BF, width) if pre else (None, None)
    dyh = np.zeros((T, d)) if nody else _host(dy)
    want = R.residual_bwd(dyh, None if dh is None else _host(dh), _host(y), fh, sth, w, _adds(T, d))
    dxb, dx = (dyb, dy) if inplace and not nody else _dev(np.zeros((T, d)), dt, width)
    dfb, df = _dev(np.zeros((T, d)), BF, width)
    names = [n for n, on in (("dg_pre", pre), ("db_pre", pre), ("dg_post", post), ("db_post", post), ("dgate", gate)) if on]
    sums = {n: torch.full((d,), 7.0, device="cuda") for n in names}
    run = lambda dx, df, sums: ops.residual_norm_bwd(None if nody else dy, dh, y, f, st, dx, df, d, **sums, **go)  # noqa: E731
    if not (inplace and not nody):  # the same bits on another call
        again = dx.clone(), df.clone(), {n: t.clone() for n, t in sums.items()}
        run(again[0], again[1], again[2])
    run(dx, df, sums)
    torch.cuda.synchronize()
    _check("dx", dx, *want["dx"], dt)
    _check("df", df, *want["df"], BF)
    for n in names:
        _check(n, sums[n], *want[n], F4)
    if not (inplace and not nody):
        assert torch.equal(again[0], dx) and torch.equal(again[1], df) and all(torch.equal(again[2][n], sums[n]) for n in names)
    for b in (dxb, dfb, dyb, dhb):
        assert b is None or (b[:, d:] == 7).all()


@pytest.mark.parametrize("dt", [BF, F4])
@pytest.mark.parametrize("T,d", [(1, 8), (3, 1), (2, 2), (5, 7), (257, 64), (300, 203), (9, 512), (7, 513), (100, 768), (64, 1021), (1031, 1280),
                                 (1, 4096), (515, 4096), (11, 4104), (6, 5000), (300, 8192), (2, 8191)])
def test_sizes(T, d, dt):
    _case(T, d, dt, "layer", "rms")
    _case(T, d, dt, "rms", "layer", alpha=0.9, beta=0.25, p=0.5)


@pytest.mark.parametrize("dt", [BF, F4])
@pytest.mark.parametrize("pre", [None, "layer", "rms"])
@pytest.mark.parametrize("post", [None, "layer", "rms"])
def test_combinations(pre, post, dt):
    for i, (gain, shift, gate, p) in enumerate([(True, True, True, 0.2), (False, False, False, 0.0), (True, False, True, 0.0),
                                                (False, True, False, 0.3)]):
        _case(21, 264, dt, pre, post, gain, shift, gate, 1.0 if i % 2 else 0.7, 1.0 if i < 2 else -0.5, p, width=5 * i, inplace=i == 2,
              nody=i == 3)


def test_same_dropout_as_the_operator():
    """Without norms, gate and scales the branch is dropout's outcome, bit for bit."""
    from paper_2309_01226_amd import ops
    f = torch.randn(77, 1000, device="cuda").to(BF)
    x, y = torch.zeros(77, 1000, device="cuda"), torch.empty(77, 1000, device="cuda")
    step = torch.tensor([9], device="cuda")
    ops.residual_norm_fwd(x, f, y, None, None, 1000, p=0.3, seed=5, step=step)
    assert torch.equal(y, ops.dropout(f.float(), 0.3, 5, step=step))


@pytest.mark.parametrize("post", [None, "rms"])
def test_dropped_branch_does_not_matter(post):
    """Infinities and NaN of a branch, where it is dropped and not normed, reach nothing."""
    from paper_2309_01226_amd import ops
    T, d = 16, 520
    drop = ~torch.as_tensor(R.kept(T, d, 0.5, 5)[0]).cuda()
    x, gate = torch.randn(T, d, device="cuda"), torch.randn(d, device="cuda")
    f = torch.randn(T, d, device="cuda").to(BF)
    if post is None:
        f = f.masked_fill(drop, float("nan"))
    else:
        f[3] = float("nan")  # spoils its own row, where it is kept
    st, y, h = torch.empty(4, T, device="cuda"), torch.empty_like(x), torch.empty_like(f)
    kw = dict(pre="layer", post=post, gate=gate, p=0.5, seed=5)
    ops.residual_norm_fwd(x, f, y, h, st, d, **kw)
    dx, df, dgate = torch.empty_like(x), torch.empty_like(f), torch.empty(d, device="cuda")
    ops.residual_norm_bwd(torch.randn_like(x), torch.randn_like(x).to(BF), y, f, st, dx, df, d, dgate=dgate, **kw)
    torch.cuda.synchronize()
    if post is None:
        assert all(torch.isfinite(t).all() for t in (y, h, dx, df, dgate))
    else:
        ok = torch.arange(T, device="cuda") != 3
        assert torch.equal(y[3][drop[3]], x[3][drop[3]])
        assert all(torch.isfinite(t[ok]).all() for t in (y, h, dx, df)) and torch.isnan(h[3]).all()


def test_far_means():
    """Rows whose mean dwarfs their deviation: formed from differences, so that the deviation stays."""
    from paper_2309_01226_amd import ops
    T, d = 9, 4096
    x = (1000 + torch.randn(T, d, dtype=torch.float64)).float().cuda()
    f = torch.zeros(T, d, dtype=BF, device="cuda")
    y, h, st = torch.empty_like(x), torch.empty_like(f), torch.empty(4, T, device="cuda")
    ops.residual_norm_fwd(x, f, y, h, st, d, pre="layer", eps=0.0)
    torch.cuda.synchronize()
    want = 1 / x.double().std(1, unbiased=False)
    # differences of x and a mean that is off by 31 E of 1000: 2e-3 at most, whose square joins the variance
    assert ((st[3].double() - want).abs() / want).max().item() <= 40 * R.E + (31 * R.E * 1000) ** 2
    assert math.isclose(h.double().mean().item(), 0.0, abs_tol=31 * R.E * 1000 + 2.0 ** -8)


def test_no_rows():
    from paper_2309_01226_amd import ops
    e = lambda dt: torch.empty(0, 64, dtype=dt, device="cuda")  # noqa: E731
    st = torch.empty(4, 0, device="cuda")
    ops.residual_norm_fwd(e(F4), e(BF), e(F4), e(BF), st, 64, pre="rms")
    s = {n: torch.full((64,), 7.0, device="cuda") for n in ("dg_pre", "dgate")}
    ops.residual_norm_bwd(e(F4), e(BF), e(F4), e(BF), st, e(F4), e(BF), 64, pre="rms", gate=torch.ones(64, device="cuda"), **s)
    assert not s["dg_pre"].any() and not s["dgate"].any()


def test_refusals():
    from paper_2309_01226_amd import _lib, ops
    x, f = torch.randn(8, 64, device="cuda"), torch.randn(8, 64, device="cuda").to(BF)
    y, h, st, g = torch.empty_like(x), torch.empty_like(f), torch.empty(4, 8, device="cuda"), torch.ones(64, device="cuda")
    fwd = lambda **k: ops.residual_norm_fwd(**{**dict(x=x, f=f, y=y, h=h, stats=st, d=64, pre="rms"), **k})  # noqa: E731
    fwd()
    for bad in (dict(pre="batch"), dict(f=x), dict(y=f), dict(h=x), dict(stats=st[:2]), dict(g_pre=g[:8]), dict(g_pre=g.double()),
                dict(x=x.T), dict(f=f[:7]), dict(d=72), dict(gate=torch.ones(64)), dict(step=torch.zeros(2, dtype=torch.int64, device="cuda"))):
        with pytest.raises((TypeError, ValueError)):
            fwd(**bad)
    for bad in (dict(h=None), dict(stats=None), dict(p=1.5), dict(eps=-1.0), dict(beta=math.inf), dict(g_post=g), dict(d=0)):
        with pytest.raises((_lib.SatError, ValueError)):
            fwd(**bad)
    bwd = lambda **k: ops.residual_norm_bwd(**{**dict(dy=x, dh=f, y=y, f=f, stats=st, dx=torch.empty_like(x), df=h, d=64, pre="rms"), **k})  # noqa: E731
    bwd()
    for bad in (dict(dg_post=g), dict(dgate=g), dict(dh=None), dict(y=None), dict(stats=None), dict(f=None, gate=g, dgate=g)):
        with pytest.raises((_lib.SatError, ValueError)):
            bwd(**bad)


def test_streams_and_graph():
    """Two streams at once, and captured with the step moving on: each replay is the eager call's bits."""
    from paper_2309_01226_amd import ops
    T, d = 300, 1280
    x, f = torch.randn(T, d, device="cuda").to(BF), torch.randn(T, d, device="cuda").to(BF)
    dy, dh, gate = torch.randn(T, d, device="cuda").to(BF), torch.randn(T, d, device="cuda").to(BF), torch.randn(d, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def buffers():
        e = lambda *s, dt=F4: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
        return dict(y=e(T, d, dt=BF), h=e(T, d, dt=BF), st=e(4, T), dx=e(T, d, dt=BF), df=e(T, d, dt=BF), dg=e(d), dgate=e(d))

    def go(b):
        kw = dict(pre="layer", post="rms", gate=gate, p=0.2, seed=4, step=step)
        ops.residual_norm_fwd(x, f, b["y"], b["h"], b["st"], d, **kw)
        ops.residual_norm_bwd(dy, dh, b["y"], f, b["st"], b["dx"], b["df"], d, dg_post=b["dg"], dgate=b["dgate"], **kw)

    same = lambda a, b: all(torch.equal(a[k], b[k]) for k in a)  # noqa: E731
    eager = buffers()
    go(eager)
    torch.cuda.synchronize()
    sides = [(torch.cuda.Stream(), buffers()) for _ in range(2)]
    for s, b in sides:
        with torch.cuda.stream(s):
            go(b)
    torch.cuda.synchronize()
    assert all(same(b, eager) for _, b in sides)
    graphs = []
    for _ in range(2):
        b, g = buffers(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            go(b)
        graphs.append((g, b))
    for i in range(3):
        step.fill_(i)
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        go(eager)
        torch.cuda.synchronize()
        assert all(same(b, eager) for _, b in graphs)


@pytest.mark.parametrize("dt,post,T,d", [(F4, "rms", 20011, 4096), (BF, "rms", 20011, 4096), (F4, None, 60001, 1280), (BF, None, 9000, 8192),
                                         (F4, "layer", 6000, 8192), (BF, "layer", 300007, 264), (F4, "layer", 300007, 256),
                                         (F4, "layer", 30001, 1280), (BF, None, 20011, 1280)])
def test_large_calls(dt, post, T, d):
    """Calls past the size where rows go past the caches: their first and last rows are those of small calls, bit for bit."""
    from paper_2309_01226_amd import ops
    flush("large", dt, post, T, d)
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    r = lambda rows, t: torch.randn(rows, d, device="cuda", generator=g, dtype=torch.float32).to(t)  # noqa: E731
    x, f, dy, dh = r(T, dt), r(T, BF), r(T, dt), r(T, BF)
    kw = dict(pre="layer", post=post, gate=torch.randn(d, device="cuda", generator=g), alpha=0.5)

    def go(at, p):
        a = [t[at] for t in (x, f, dy, dh)]
        y, h, st = torch.empty_like(a[0]), torch.empty_like(a[1]), torch.empty(4, len(a[0]), device="cuda")
        dx, df, dgate = torch.empty_like(a[2]), torch.empty_like(a[1]), torch.empty(d, device="cuda")
        ops.residual_norm_fwd(a[0], a[1], y, h, st, d, p=p, seed=3, **kw)
        ops.residual_norm_bwd(a[2], a[3], y, a[1], st, dx, df, d, dgate=dgate, p=p, seed=3, **kw)
        assert torch.isfinite(dgate).all()
        return y, h, dx, df

    for at, p in ((slice(0, 130), 0.25), (slice(T - 130, T), 0.0)):
        whole, part = go(slice(0, T), p), go(at, p)
        for name, a, b in zip(("y", "h", "dx", "df"), whole, part):
            assert torch.equal(a[at], b), (name, p)
        del whole
