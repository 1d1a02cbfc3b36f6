"""AdamW over many tensors: tables of more than 4.2 M elements, whose kernels take chunks of 4096 elements past the
caches, and outputs of the moments' values that lie next to each other, in any order."""

import numpy as np
import pytest
import torch

from tests import packed_ref as R
from tests.gpu_util import flush
from tests.test_gpu_adamw_multi import B1, B2, EPS, LR, SIZES, Set, _check_p, _np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_state_values_side_by_side(dt):
    from paper_2309_01226_amd import ops
    sizes = [257, 0, 1, 1000, 4096]
    s = Set(sizes, 8, "fp32")
    apart = [[torch.zeros(n, device="cuda", dtype=dt) for n in sizes] for _ in range(2)]
    ops.adamw_multi_state(s.table, *apart)
    whole = torch.zeros(2 * sum(sizes), device="cuda", dtype=dt)
    cuts = list(whole.split(sizes[::-1] + sizes[::-1]))[::-1]  # from the end on, nothing between them
    ops.adamw_multi_state(s.table, cuts[:len(sizes)], cuts[len(sizes):])
    torch.cuda.synchronize()
    for a, b in zip(apart[0] + apart[1], cuts):
        assert torch.equal(a, b)
    with pytest.raises(RuntimeError):
        ops.adamw_multi_state(s.table, apart[0], apart[0])


BIG, CUT = 5_000_003, 1 << 20  # a tensor that makes the table a large one; a whole number of blocks of it


def _pair(bits, grad, shift, seed):
    """More tensors than a launch takes and a long one behind them; the same with the long one cut short."""
    few = SIZES * 6
    a, b = Set(few + [BIG], bits, grad, shift, seed=seed), Set(few + [CUT], bits, grad, shift, seed=seed)
    assert sum(a.sizes) >= 1024 * 4096 > sum(b.sizes)
    for x in ("p", "g", "m", "v") + (("me", "ve") if bits == 8 else ()):
        for u, w in zip(getattr(a, x), getattr(b, x)):
            w.copy_(u[:w.numel()])
    return a, b


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["fp32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 2, 3, 4])
def test_large_table_as_a_small_one(bits, grad, shift):
    """Chunks of 4096 elements past the caches: the bits of the chunks of 1024 in them, codes and exponents too."""
    from paper_2309_01226_amd import ops
    flush("adamw multi large", bits, grad, shift)
    a, b = _pair(bits, grad, shift, seed=bits + shift)
    for t in (1, 4):
        for s in (a, b):
            ops.adamw_multi(s.table, LR, B1, B2, EPS, t, seed=11)
    torch.cuda.synchronize()
    a.guards()
    b.guards()
    for x in ("p", "m", "v", "sh") + (("me", "ve") if bits == 8 else ()):
        for i, (u, w) in enumerate(zip(getattr(a, x), getattr(b, x))):
            assert torch.equal(u[:w.numel()], w), (x, i)


@pytest.mark.parametrize("shift", [0, 1])
def test_large_table_of_32_bits_as_single_calls(shift):
    from paper_2309_01226_amd import ops
    s = Set(SIZES + [BIG], 32, "fp32", shift)
    one = [[t.clone() for t in x] for x in (s.p, s.m, s.v)]
    sh = [torch.zeros(n, device="cuda", dtype=torch.bfloat16) for n in s.sizes]
    for t in (1, 5):
        ops.adamw_multi(s.table, LR, B1, B2, EPS, t)
        for i, n in enumerate(s.sizes):
            if n:
                ops.adamw(one[0][i], s.g[i].clone(), one[1][i], one[2][i], sh[i], n, LR, B1, B2, EPS, s.wd[i], t)
    torch.cuda.synchronize()
    for i in range(len(s.sizes)):
        assert torch.equal(s.p[i], one[0][i]) and torch.equal(s.m[i], one[1][i]) and torch.equal(s.v[i], one[2][i]), i
        assert torch.equal(s.sh[i], sh[i])
    s.guards()


@pytest.mark.parametrize("grad", ["fp32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1])
def test_long_tensor_of_8_bits_against_64_bits(grad, shift):
    from paper_2309_01226_amd import ops
    s = Set([300, BIG], 8, grad, shift, seed=3)
    old, g = _np(s.p[1]), _np(s.g[1])
    m0, v0 = R.moments8(*(t[1].cpu().numpy() for t in (s.m, s.v, s.me, s.ve)))
    ops.adamw_multi(s.table, LR, B1, B2, EPS, 3, seed=11)
    torch.cuda.synchronize()
    s.guards()
    p, m, v = R.adamw(old, g, m0, v0, LR, B1, B2, EPS, s.wd[1], 3)
    _check_p(_np(s.p[1]), p, old, g, m0, v, 3)
    m8, v8 = R.moments8(*(t[1].cpu().numpy() for t in (s.m, s.v, s.me, s.ve)))
    r, r8 = np.sqrt(v), np.sqrt(v8)

    def top(x):
        y = np.zeros(-(-BIG // 256) * 256)
        y[:BIG] = x
        return np.repeat(y.reshape(-1, 256).max(1), 256)[:BIG]
    # within one code's step of the value (1 / 8 and 1 / 16 of it), or under the least code, which is 2^-15 of the
    # block's factor, itself under 2 / 1.75 and 2 / 1.9 of its largest; 1e-6 for the fp32 part
    assert (np.abs(m8 - m) <= np.maximum(np.abs(m) * (0.125 + 1e-6), 2.25 * 2.0 ** -15 * 2.0 / 1.75 * top(np.abs(m)))).all()
    assert (np.abs(r8 - r) <= np.maximum(r * (0.0625 + 1e-6), 2.125 * 2.0 ** -15 * 2.0 / 1.9 * top(r))).all()
    assert (r8[r > 0] > 0).all()


def test_second_moments_of_8_bits_at_the_end_of_the_range():
    """v of 2^-125.3 is kept and decays by 0.999; below 2^-126 it counts as 0, and p moves by m / eps alone."""
    from paper_2309_01226_amd import ops
    n = 512
    z8 = lambda k: torch.zeros(k, device="cuda", dtype=torch.uint8)  # noqa: E731
    p, g, m, v, me, ve = torch.zeros(n, device="cuda"), torch.full((n,), 1.25 * 2.0 ** -58, device="cuda"), z8(n), z8(n), z8(2), z8(2)
    g[256:] = 1.25 * 2.0 ** -59
    t = ops.AdamWTensors([p], [g], [m], [v], m_exp=[me], v_exp=[ve])
    ops.adamw_multi(t, LR, B1, B2, EPS, 1, seed=1)
    out = [torch.empty(n, device="cuda") for _ in range(2)]
    ops.adamw_multi_state(t, [out[0]], [out[1]])
    torch.cuda.synchronize()
    want = 0.001 * (1.25 * 2.0 ** -58) ** 2
    assert float((out[1][:256].double().sqrt() / want ** 0.5 - 1).abs().max()) <= 1 / 16 + 1e-5 and not v[256:].any()
    # root / (1 - b2) is 4e-18, nothing against eps
    step = LR * _np(g) / EPS
    assert (np.abs(_np(p) + step) <= 16 * 2.0 ** -24 * step).all()
