"""AdamW over many tensors: 32-bit moments bitwise those of the single-tensor call, 8-bit moments within
a code's step of the 64-bit update, their rounding right on average."""

import numpy as np
import pytest
import torch

from tests import packed_ref as R
from tests.gpu_util import flush

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS = 1e-3, 0.9, 0.999, 1e-8
SIZES = [1, 3, 255, 256, 257, 0, 1000, 4095, 4096, 4097, 20003]


def _place(a, shift):
    """The array in a buffer that begins `shift` elements past an aligned place, guards around it."""
    buf = torch.full((a.numel() + 32 + shift,), 99, device="cuda").to(a.dtype)
    v = buf[16 + shift:16 + shift + a.numel()]
    v.copy_(a)
    return v, buf


class Set:
    def __init__(self, sizes, bits, grad, shift=0, shadows=True, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.bufs, self.sizes = [], sizes

        def place(a):
            v, b = _place(a, shift)
            self.bufs.append((b, 16 + shift, a.numel()))
            return v
        rnd = lambda n: torch.randn(n, device="cuda", generator=g)  # noqa: E731
        self.p = [place(rnd(n)) for n in sizes]
        size = [torch.exp(2 * rnd(n)) for n in sizes]
        self.g = [place((1e-2 * rnd(n) * s).to(torch.bfloat16 if grad == "bf16" else torch.float32)) for n, s in zip(sizes, size)]
        self.sh = [place(torch.zeros(n, device="cuda", dtype=torch.bfloat16)) for n in sizes] if shadows else None
        self.wd = [0.01 * (i % 3) for i in range(len(sizes))]
        kw = {}
        if bits == 32:
            self.m = [place(3e-3 * rnd(n) * s) for n, s in zip(sizes, size)]
            self.v = [place(1e-5 * s * s * torch.rand(n, device="cuda", generator=g)) for n, s in zip(sizes, size)]
        else:
            byte = lambda n, lo, hi: torch.randint(lo, hi, (n,), device="cuda", generator=g).to(torch.uint8)  # noqa: E731
            self.m, self.v = [place(byte(n, 0, 256)) for n in sizes], [place(byte(n, 0, 256)) for n in sizes]
            self.me, self.ve = ([place(byte(-(-n // 256), lo, lo + 6)) for n in sizes] for lo in (116, 118))
            kw = dict(m_exp=self.me, v_exp=self.ve)
        from paper_2309_01226_amd import ops
        self.table = ops.AdamWTensors(self.p, self.g, self.m, self.v, shadows=self.sh, weight_decay=self.wd, **kw)

    def guards(self):
        for b, o, n in self.bufs:
            assert (b[:o] == 99).all() and (b[o + n:] == 99).all()


@pytest.mark.parametrize("shift", [0, 1, 2, 4])
@pytest.mark.parametrize("shadows", [True, False])
def test_32_bits_as_the_single_call(shift, shadows):
    from paper_2309_01226_amd import ops
    flush("adamw multi 32", shift, shadows)
    s = Set(SIZES * 8, 32, "fp32", shift, shadows)  # more tensors than a launch takes
    one = [[t.clone() for t in x] for x in (s.p, s.m, s.v)]
    sh = [torch.zeros(n, device="cuda", dtype=torch.bfloat16) for n in s.sizes]
    for t in (1, 2, 7):
        ops.adamw_multi(s.table, LR, B1, B2, EPS, t)
        for i, n in enumerate(s.sizes):
            if n:
                ops.adamw(one[0][i], s.g[i].clone(), one[1][i], one[2][i], sh[i], n, LR, B1, B2, EPS, s.wd[i], t)
    torch.cuda.synchronize()
    for i in range(len(s.sizes)):
        assert torch.equal(s.p[i], one[0][i]) and torch.equal(s.m[i], one[1][i]) and torch.equal(s.v[i], one[2][i]), i
        if shadows:
            assert torch.equal(s.sh[i], sh[i])
    s.guards()


def _np(t):
    return t.double().cpu().numpy()


def _check_p(got, want, old, g, m0, v, t):
    # p - lr wd p and the step: a few roundings of p (2^-24 each), and a dozen of the step with each of the two terms of m
    terms = LR / (1 - B1 ** t) * (B1 * np.abs(m0) + (1 - B1) * np.abs(g)) / (np.sqrt(v) / (1 - B2 ** t) ** 0.5 + EPS)
    off = np.abs(got - want) - 4 * 2.0 ** -24 * np.abs(old) - 16 * 2.0 ** -24 * terms
    assert off.max() <= 1e-30, float(off.max())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["fp32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_against_64_bits(bits, grad, shift):
    from paper_2309_01226_amd import ops
    flush("adamw multi", bits, grad, shift)
    s = Set(SIZES, bits, grad, shift, seed=bits + shift)
    old = [_np(p) for p in s.p]
    before = [(_np(m), _np(v)) if bits == 32 else
              R.moments8(m.cpu().numpy(), v.cpu().numpy(), s.me[i].cpu().numpy(), s.ve[i].cpu().numpy())
              for i, (m, v) in enumerate(zip(s.m, s.v))]
    ops.adamw_multi(s.table, LR, B1, B2, EPS, 3, seed=11)
    torch.cuda.synchronize()
    s.guards()
    for i, n in enumerate(s.sizes):
        if n == 0:
            continue
        p, m, v = R.adamw(old[i], _np(s.g[i]), *before[i], LR, B1, B2, EPS, s.wd[i], 3)
        _check_p(_np(s.p[i]), p, old[i], _np(s.g[i]), before[i][0], v, 3)
        assert torch.equal(s.sh[i], s.p[i].to(torch.bfloat16))
        if bits == 32:
            # m, v: three roundings of terms no larger than |b m| + |(1 - b) g|
            assert (np.abs(_np(s.m[i]) - m) <= 3 * 2.0 ** -24 * (B1 * np.abs(before[i][0]) + 0.1 * np.abs(_np(s.g[i])))).all()
            assert (np.abs(_np(s.v[i]) - v) <= 4 * 2.0 ** -24 * v).all()
            continue
        me, ve = s.me[i].cpu().numpy(), s.ve[i].cpu().numpy()
        m8, v8 = R.moments8(s.m[i].cpu().numpy(), s.v[i].cpu().numpy(), me, ve)
        r, r8 = np.sqrt(v), np.sqrt(v8)
        top = lambda x: np.repeat([x[j:j + 256].max() for j in range(0, n, 256)], 256)[:n]  # noqa: E731
        # within one code's step of the value (1 / 8 and 1 / 16 of it), or under the least code; 1e-6 for the fp32 part
        least = 2.25 * 2.0 ** -15 * 2.0 / 1.75 * top(np.abs(m))
        assert (np.abs(m8 - m) <= np.maximum(np.abs(m) * (0.125 + 1e-6), least)).all()
        least = 2.125 * 2.0 ** -15 * 2.0 / 1.9 * top(r)
        assert (np.abs(r8 - r) <= np.maximum(r * (0.0625 + 1e-6), least)).all()
        assert (r8[r > 0] > 0).all() and ((m8 == 0) | (np.sign(m8) == np.sign(m))).all()
        # the largest of each block is within the codes: the block's power of two is the least that holds it
        for j in range(0, n, 256):
            big = np.abs(m[j:j + 256]).max()
            e = 2.0 ** (float(me[j // 256]) - 127)
            assert 0.9 * e <= big * (1 + 1e-6) and big <= 1.875 * e * (1 + 1e-6)


def test_8_bit_rounding_is_right_on_average_and_by_seed():
    """Equal elements: the mean of what is kept is the value, to 5 standard errors of a two-point choice."""
    from paper_2309_01226_amd import ops
    n = 1 << 20
    z8 = lambda k: torch.zeros(k, device="cuda", dtype=torch.uint8)  # noqa: E731
    g = torch.full((n,), 0.0123, device="cuda")
    g[0] = 0.05  # the block's largest
    kept = []
    for seed in (1, 1, 2):
        p, m, v, me, ve = torch.zeros(n, device="cuda"), z8(n), z8(n), z8(n // 256), z8(n // 256)
        t = ops.AdamWTensors([p], [g], [m], [v], m_exp=[me], v_exp=[ve])
        ops.adamw_multi(t, LR, B1, B2, EPS, 1, seed=seed)
        mo, vo = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        ops.adamw_multi_state(t, [mo], [vo])
        torch.cuda.synchronize()
        kept.append((m.clone(), v.clone()))
        for got, want in ((mo[256:], 0.1 * 0.0123), (vo[256:].sqrt(), (0.001 * 0.0123 ** 2) ** 0.5)):
            x = got.double()
            steps = x.unique()
            assert len(steps) == 2
            lo, hi = steps.tolist()
            assert lo <= want <= hi
            sd = (hi - lo) / 2 / (n - 256) ** 0.5
            assert abs(float(x.mean()) - want) <= 5 * sd
    assert torch.equal(kept[0][0], kept[1][0]) and torch.equal(kept[0][1], kept[1][1])
    assert not torch.equal(kept[0][0], kept[2][0])


def test_8_bit_averages_move_by_less_than_a_step():
    """v under gradients that stop falls by a thousandth a step, a sixtieth of a code's step."""
    from paper_2309_01226_amd import ops
    n = 1 << 16
    z8 = lambda k: torch.zeros(k, device="cuda", dtype=torch.uint8)  # noqa: E731
    p, m, v, me, ve = torch.zeros(n, device="cuda"), z8(n), z8(n), z8(n // 256), z8(n // 256)
    g = torch.randn(n, device="cuda")
    t = ops.AdamWTensors([p], [g], [m], [v], m_exp=[me], v_exp=[ve])
    ops.adamw_multi(t, 0.0, B1, B2, EPS, 1, seed=5)
    out = [torch.empty(n, device="cuda") for _ in range(2)]
    ops.adamw_multi_state(t, [out[0]], [out[1]])
    first = float(out[1].double().sqrt().mean())
    g.zero_()
    for k in range(2, 302):
        ops.adamw_multi(t, 0.0, B1, B2, EPS, k, seed=5)
    ops.adamw_multi_state(t, [out[0]], [out[1]])
    torch.cuda.synchronize()
    # the root falls by 0.999^(300 / 2) = 0.861; 300 roundings of at most a 16th, independent over 65536
    # elements: the mean of each walk's end is off by less than 300^0.5 / 32 / 65536^0.5 = 0.2 %, 5 of these
    assert abs(float(out[1].double().sqrt().mean()) / first - 0.999 ** 150) < 0.011
    assert float(out[0].abs().max()) < 1e-3  # 0.9^300 is gone


def test_8_bit_zeros_and_tiny_and_huge():
    from paper_2309_01226_amd import ops
    n = 1024
    z8 = lambda k: torch.zeros(k, device="cuda", dtype=torch.uint8)  # noqa: E731
    p = torch.randn(n, device="cuda")
    p0 = p.clone()
    m, v, me, ve = z8(n), z8(n), z8(4), z8(4)
    g = torch.zeros(n, device="cuda")
    g[256] = 1e-30       # squares to nothing: only m moves
    g[512:768] = 1e15
    g[600] = 0.0
    t = ops.AdamWTensors([p], [g], [m], [v], weight_decay=0.1, m_exp=[me], v_exp=[ve])
    ops.adamw_multi(t, LR, B1, B2, EPS, 1)
    out = [torch.empty(n, device="cuda") for _ in range(2)]
    ops.adamw_multi_state(t, [out[0]], [out[1]])
    torch.cuda.synchronize()
    still = torch.ones(n, dtype=torch.bool, device="cuda")
    still[256] = False
    still[512:768] = False
    still[600] = True
    assert (m[still] == 0).all() and (v[still] == 0).all() and not out[0][still].any() and not out[1][still].any()
    assert torch.allclose(p[still], p0[still] * (1 - LR * 0.1), rtol=1e-6, atol=0)
    assert 0.8e-31 < float(out[0][256]) < 1.2e-31 and float(out[1][256]) == 0
    moved = out[0][512:768][g[512:768] > 0]
    assert ((moved - 1e14).abs() <= 0.126e14).all()
    assert torch.isfinite(p).all()


def test_8_bit_gradient_that_is_not_finite_stays_in_its_block():
    from paper_2309_01226_amd import ops
    s = Set([1024], 8, "fp32")
    r = Set([1024], 8, "fp32")
    s.g[0][300] = float("nan")
    s.g[0][700] = float("inf")
    for x in (s, r):
        ops.adamw_multi(x.table, LR, B1, B2, EPS, 2, seed=3)
    torch.cuda.synchronize()
    for a in ("p", "m", "v"):
        x, y = getattr(s, a)[0], getattr(r, a)[0]
        assert torch.equal(x[:256], y[:256]) and torch.equal(x[768:], y[768:]), a
    assert not torch.isfinite(s.p[0][[300, 700]]).any()
    keep = torch.ones(1024, dtype=torch.bool)
    keep[[300, 700]] = False
    assert torch.equal(s.p[0][keep], r.p[0][keep])


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_state_values(dt, shift):
    from paper_2309_01226_amd import ops
    s = Set(SIZES, 8, "fp32", shift)
    outs = [[_place(torch.zeros(n, device="cuda", dtype=dt), shift) for n in SIZES] for _ in range(2)]
    ops.adamw_multi_state(s.table, *[[v for v, _ in o] for o in outs])
    torch.cuda.synchronize()
    for i in range(len(SIZES)):
        m, v = R.moments8(s.m[i].cpu().numpy(), s.v[i].cpu().numpy(), s.me[i].cpu().numpy(), s.ve[i].cpu().numpy())
        assert np.array_equal(_np(outs[0][i][0]), m)
        want = torch.as_tensor(v).float().to(dt)
        assert torch.equal(outs[1][i][0].cpu(), want)
    for o in outs:
        for v, b in o:
            assert (b[:16 + shift] == 99).all() and (b[16 + shift + v.numel():] == 99).all()


@pytest.mark.parametrize("bits", [8, 32])
def test_captured(bits):
    """Replays of a captured step, with eager steps of another set between them."""
    from paper_2309_01226_amd import ops
    a, b, other = (Set([5000, 17, 300], bits, "bf16", seed=1) for _ in range(3))
    ops.adamw_multi(other.table, LR, B1, B2, EPS, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.adamw_multi(a.table, LR, B1, B2, EPS, 4, seed=9)
    for k in range(3):
        graph.replay()
        ops.adamw_multi(b.table, LR, B1, B2, EPS, 4, seed=9)
        ops.adamw_multi(other.table, LR, B1, B2, EPS, k + 2)
        torch.cuda.synchronize()
        for x in ("p", "m", "v", "sh"):
            assert all(torch.equal(s, t) for s, t in zip(getattr(a, x), getattr(b, x))), (k, x)


def test_python_checks():
    from paper_2309_01226_amd import ops
    f = lambda n=300: torch.zeros(n, device="cuda")  # noqa: E731
    u = lambda n=300: torch.zeros(n, device="cuda", dtype=torch.uint8)  # noqa: E731
    p = f()
    ok = dict(params=[p], grads=[f()], m=[f()], v=[f()])
    ops.AdamWTensors(**ok)
    whole = f(600)
    bad = [dict(grads=[f(299)]), dict(m=[f().half()]), dict(v=[f().cpu()]), dict(grads=[]), dict(m=[p]), dict(m=[whole[:300]], v=[whole[299:599]]),
           dict(grads=[p]), dict(m=[u()], v=[u()]), dict(m=[u()], v=[u()], m_exp=[u(1)], v_exp=[u(2)]), dict(m_exp=[u(2)], v_exp=[u(2)]),
           dict(params=[f(600)[::2]]), dict(weight_decay=[0.1, 0.2]), dict(shadows=[f()])]
    for b in bad:
        with pytest.raises((TypeError, ValueError)):
            ops.AdamWTensors(**{**ok, **b})
    # gradients may be one tensor, parameters may not
    g = f()
    ops.AdamWTensors([f(), f()], [g, g], [f(), f()], [f(), f()])
    with pytest.raises(ValueError):
        ops.AdamWTensors([p, p], [f(), f()], [f(), f()], [f(), f()])
    t = ops.AdamWTensors(**ok)
    with pytest.raises(ValueError):
        ops.adamw_multi_state(t, [f()], [f()])
    from paper_2309_01226_amd._lib import SatError
    with pytest.raises(SatError):
        ops.adamw_multi(t, LR, B1, B2, EPS, 0)


@pytest.mark.parametrize("bits", [32, 8])
def test_more_than_2_31_elements(bits):
    """The last elements of a long tensor, and of one behind it, as a call on them alone: of the 8-bit form the
    parameters only, since its rounding goes by the element's number."""
    from paper_2309_01226_amd import ops
    flush("adamw multi long", bits)
    n, k = (1 << 31) + 5000, 4360  # the tail begins a block
    st = torch.float32 if bits == 32 else torch.uint8
    zeros = lambda c, dt: torch.zeros(c, device="cuda", dtype=dt)  # noqa: E731
    sizes = [n, 777]
    p, g, m, v = ([zeros(c, dt) for c in sizes] for dt in (torch.float32, torch.bfloat16, st, st))
    kw = {}
    if bits == 8:
        kw = dict(m_exp=[zeros(-(-c // 256), st) for c in sizes], v_exp=[zeros(-(-c // 256), st) for c in sizes])
    gen = torch.Generator(device="cuda").manual_seed(1)
    cut = (n - k) // 256 * 256
    tail = [p[0][cut:], p[1]]
    tg = [g[0][cut:], g[1]]
    for a, b in zip(tail, tg):
        a.normal_(generator=gen)
        b.normal_(generator=gen)
    small = [t.clone() for t in tail]
    sm, sv = ([zeros(t.numel(), st) for t in tail] for _ in range(2))
    skw = {x: [zeros(-(-t.numel() // 256), st) for t in tail] for x in kw}
    ops.adamw_multi(ops.AdamWTensors(small, tg, sm, sv, weight_decay=0.1, **skw), LR, B1, B2, EPS, 1)
    ops.adamw_multi(ops.AdamWTensors(p, g, m, v, weight_decay=0.1, **kw), LR, B1, B2, EPS, 1)
    for a, b in zip(tail, small):
        assert torch.equal(a, b)
    if bits == 32:
        assert torch.equal(m[0][cut:], sm[0]) and torch.equal(v[0][cut:], sv[0]) and torch.equal(m[1], sm[1])
    else:
        assert torch.equal(kw["m_exp"][0][cut // 256:], skw["m_exp"][0]) and bool(v[0][cut:].any())
    step = 1 << 28  # all before the tail stayed as it was
    for a in (p[0], m[0], v[0]):
        assert not any(bool(a[i:min(cut, i + step)].any()) for i in range(0, cut, step))
