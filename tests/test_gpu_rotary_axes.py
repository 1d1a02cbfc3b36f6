"""Rotary positions with several axes against their 64-bit form.

fp32: two products and a sum, each off by 2^-24 of its magnitude, with cos and sin off by at most
2^-22 (two ulp of the function, the angle's part within half a turn kept to 24 bits: 2 pi 2^-25):
|err| <= (2^-22 + 2^-23) (|u| + |w|).  bf16: that, and one rounding of the result, 2^-8 of it."""

import numpy as np
import pytest
import torch

from tests import packed_ref as R
from tests.gpu_util import flush

pytestmark = pytest.mark.gpu


def _check(got, x, want, dt):
    size = np.abs(x).max(1, keepdims=True) * 2
    bound = 2.0 ** -21 * size + (2.0 ** -8 * np.abs(want) if dt == torch.bfloat16 else 2.0 ** -24 * np.abs(want))
    off = np.abs(got - want) - bound
    assert np.isfinite(got).all() and off.max() <= 0, float(off.max())


def _case(T, H, dh, pairs, dt, inter, own, inv, *, inplace=True, tail=8, offset=0, base=1e4, far=1 << 20, seed=0):
    from paper_2309_01226_amd import ops
    flush("rotary", T, H, dh, pairs, dt, inter, own, inv, inplace, tail, offset)
    rng = np.random.default_rng((T, H, dh, seed))
    x = torch.as_tensor(rng.normal(size=(T, H * dh + tail)), dtype=torch.float32).to(dt)
    pos = rng.integers(-5, far, size=(T, len(pairs))).astype(np.int32)
    buf = torch.zeros(x.numel() + 16, dtype=dt, device="cuda")
    xd = buf[offset:offset + x.numel()].view(x.shape)
    xd.copy_(x)
    out = None if inplace else torch.full((T, H * dh + tail + 4), 7.0, dtype=dt, device="cuda")
    got = ops.rotary_axes(xd, torch.as_tensor(pos).cuda(), H, dh, pairs, out=out, base=base, interleaved=inter, own_freqs=own,
                          inverse=inv)
    torch.cuda.synchronize()
    xh = x.double().numpy()
    want = R.rotary(xh, pos, H, dh, pairs, base, inter, own, inv)
    g = got.double().cpu().numpy()
    if inplace:
        assert got.data_ptr() == xd.data_ptr()
        assert np.array_equal(g[:, H * dh:], xh[:, H * dh:])
    else:
        assert torch.equal(xd.cpu(), x) and (g[:, H * dh:] == 7.0).all()
    half = sum(pairs)
    for h in range(H):  # dims behind the pairs: as they were
        assert np.array_equal(g[:, h * dh + 2 * half:(h + 1) * dh], xh[:, h * dh + 2 * half:(h + 1) * dh])
    _check(g[:, :H * dh], xh[:, :H * dh], want[:, :H * dh], dt)
    assert not buf[offset + x.numel():].any() and not buf[:offset].any()


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter,own,inv,inplace", [(True, True, False, True), (False, False, True, True), (True, False, True, False),
                                                   (False, True, False, False)])
@pytest.mark.parametrize("T,H,dh,pairs", [
    (1, 1, 2, (1,)), (257, 3, 80, (20, 20)), (33, 5, 64, (8, 12, 12)), (100, 2, 128, (16, 24, 24)), (17, 4, 256, (16, 16)),
    (9, 7, 10, (1, 2)), (31, 2, 36, (3, 0, 5, 7)), (64, 1, 16, (8,)), (50, 20, 128, (64,)), (12, 2, 512, (100, 28)),
    (5, 2, 80, (10, 10)), (40, 3, 72, (36,)),
])
def test_rotary(T, H, dh, pairs, inter, own, inv, inplace, dt):
    _case(T, H, dh, pairs, dt, inter, own, inv, inplace=inplace)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset,tail", [(1, 8), (2, 8), (4, 8), (8, 1), (8, 2), (8, 4), (3, 3)])
def test_alignment(offset, tail, dt):
    for inter in (True, False):
        _case(45, 3, 64, (16, 16), dt, inter, False, False, offset=offset, tail=tail)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_many_rows_and_heads(dt):
    _case(5000, 6, 64, (16, 8, 8), dt, False, True, False)
    _case(700, 130, 64, (32,), dt, True, False, True)   # more items in a row than a workgroup keeps in flight
    _case(3, 600, 8, (4,), dt, True, False, False)


def test_far_positions():
    """Positions up to 2^31: the angle's part within a turn keeps 32-bit accuracy."""
    from paper_2309_01226_amd import ops
    T = 64
    pos = np.linspace(1, 2 ** 31 - 1, T).astype(np.int64).astype(np.int32)[:, None]
    x = np.random.default_rng(0).normal(size=(T, 64)).astype(np.float32)
    got = ops.rotary_axes(torch.as_tensor(x).cuda(), torch.as_tensor(pos).cuda(), 1, 64, (32,)).double().cpu().numpy()
    # the 64-bit angle itself is off by 2^-53 of up to 2^31, twice (frequency and product)
    want = R.rotary(x, pos, 1, 64, (32,))
    bound = (2.0 ** -21 + 2.0 ** -21) * 2 * np.abs(x).max(1, keepdims=True)
    assert (np.abs(got - want) <= bound).all()


def test_inverse_is_the_transpose():
    """<R x, y> = <x, R^T y>, the gradient of the rotation."""
    from paper_2309_01226_amd import ops
    g = torch.Generator(device="cuda").manual_seed(0)
    x, y = (torch.randn(50, 2 * 48, device="cuda", generator=g) for _ in range(2))
    pos = torch.randint(0, 9999, (50, 2), device="cuda", dtype=torch.int32, generator=g)
    for inter in (True, False):
        a = ops.rotary_axes(x, pos, 2, 48, (10, 14), out=torch.empty_like(x), interleaved=inter)
        b = ops.rotary_axes(y, pos, 2, 48, (10, 14), out=torch.empty_like(y), interleaved=inter, inverse=True)
        l, r = (a.double() * y.double()).sum(), (x.double() * b.double()).sum()
        size = float((x.double().norm() * y.double().norm()))
        assert abs(float(l - r)) <= 2.0 ** -21 * size


def test_one_axis_as_the_batch_form():
    """One axis whose positions are t % S, interleaved: the kernel of equal rows, to one bf16 step."""
    from paper_2309_01226_amd import ops
    B, S, H, dh, rd = 2, 65, 3, 64, 32
    x = torch.randn(B * S, 2 * H * dh, device="cuda").to(torch.bfloat16)
    y = x.clone()
    ops.rotary(y, 2 * H * dh, B, S, H, dh, rd)
    pos = (torch.arange(B * S, device="cuda") % S).to(torch.int32)[:, None]
    ops.rotary_axes(x, pos, 2 * H, dh, (rd // 2,))
    torch.cuda.synchronize()
    assert float(((x.float() - y.float()).abs() - 2.0 ** -7 * y.float().abs()).max()) <= 2.0 ** -18


def test_shared_positions_and_views():
    """Positions as columns of a wider table; an empty call; one row."""
    from paper_2309_01226_amd import ops
    tab = torch.randint(0, 100, (20, 4), device="cuda", dtype=torch.int32)
    x = torch.randn(20, 64, device="cuda")
    a = ops.rotary_axes(x.clone(), tab[:, 1:3], 1, 64, (10, 22))
    b = ops.rotary_axes(x.clone(), tab[:, 1:3].contiguous(), 1, 64, (10, 22))
    assert torch.equal(a, b)
    ops.rotary_axes(torch.empty(0, 64, device="cuda"), tab[:0, :1], 1, 64, (32,))
    one = ops.rotary_axes(x[:1].clone(), tab[:1, 1:3], 1, 64, (10, 22))
    assert torch.equal(one, a[:1])


def test_captured():
    from paper_2309_01226_amd import ops
    x = torch.randn(70, 128, device="cuda").to(torch.bfloat16)
    y = torch.empty_like(x)
    pos = torch.zeros(70, 2, dtype=torch.int32, device="cuda")
    ops.rotary_axes(x, pos, 2, 64, (16, 16), out=y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.rotary_axes(x, pos, 2, 64, (16, 16), out=y)
    for k in range(3):
        pos.copy_(torch.randint(0, 1000, (70, 2), device="cuda", dtype=torch.int32))
        graph.replay()
        want = ops.rotary_axes(x, pos, 2, 64, (16, 16), out=torch.empty_like(x))
        torch.cuda.synchronize()
        assert torch.equal(y, want), k


def test_python_checks():
    from paper_2309_01226_amd import ops
    x = torch.randn(6, 128, device="cuda")
    pos = torch.zeros(6, 2, dtype=torch.int32, device="cuda")
    for args, kw in (((x.half(), pos, 2, 64, (32,)), {}), ((x, pos.long(), 2, 64, (32,)), {}), ((x, pos[:5], 2, 64, (32,)), {}),
                     ((x, pos, 3, 64, (32,)), {}), ((x, pos, 2, 64, (16, 16, 0)), {}), ((x.t(), pos, 1, 4, (2,)), {}),
                     ((x, pos, 2, 64, (32,)), dict(out=x.bfloat16()))):
        with pytest.raises((TypeError, ValueError)):
            ops.rotary_axes(*args, **kw)


def test_pair_counts_that_are_refused():
    from paper_2309_01226_amd import ops
    x, pos = torch.randn(6, 128, device="cuda"), torch.zeros(6, 1, dtype=torch.int32, device="cuda")
    for n in ((1 << 32) + 16, 129, 33, -1):
        with pytest.raises((ValueError, RuntimeError)):
            ops.rotary_axes(x, pos, 2, 64, (n,))


def test_widest_rows():
    """H dh^2 just under 2^32, one element at a time: the last heads' items are the largest numbers divided."""
    T, H, dh = 2, 4094, 1024
    g = torch.Generator().manual_seed(5)
    x = torch.randn(T, H * dh, generator=g).to(torch.bfloat16)
    pos = torch.tensor([[3], [-70000]], dtype=torch.int32)
    from paper_2309_01226_amd import ops
    buf = torch.zeros(T, H * dh + 1, device="cuda", dtype=torch.bfloat16)[:, 1:]  # 2-byte aligned
    ops.rotary_axes(x.cuda(), pos.cuda(), H, dh, (3,), out=buf, interleaved=False)
    want = torch.as_tensor(R.rotary(x.double().numpy(), pos.numpy(), H, dh, (3,), interleaved=False))
    got = buf.double().cpu()
    # (2^-22 + 2^-23) (|u| + |w|) as above, and one rounding of the result
    tol = 2.0 ** -8 * want.abs() + 2.0 ** -20 * x.double().abs().max()
    assert bool(((got - want).abs() <= tol).all())
    rest = got.view(T, H, dh)[:, :, 6:]
    assert torch.equal(rest, x.double().view(T, H, dh)[:, :, 6:])


@pytest.mark.parametrize("inplace", [True, False])
def test_offsets_past_32_bits(inplace):
    from paper_2309_01226_amd import ops
    flush("rotary far rows", inplace)
    ld, T, H, dh = (1 << 22) + 8, 1030, 2, 64
    big = torch.empty(T * ld, device="cuda", dtype=torch.bfloat16)
    x = big.as_strided((T, H * dh), (ld, 1))
    out = None if inplace else big.as_strided((T, H * dh), (ld, 1), 1 << 21)
    a = torch.randn(T, H * dh, device="cuda").to(torch.bfloat16)
    x.copy_(a)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")[:, None].contiguous()
    got = ops.rotary_axes(x, pos, H, dh, (32,), out=out)
    near = ops.rotary_axes(a.clone(), pos, H, dh, (32,))
    assert torch.equal(got, near)


@pytest.mark.parametrize("inter", [True, False])
@pytest.mark.parametrize("dt,T", [(torch.bfloat16, 11003), (torch.float32, 5503)])
@pytest.mark.parametrize("inplace", [True, False])
def test_large_calls_as_their_parts(inplace, dt, T, inter):
    """Past 80 MB the rows bypass the caches: the same bits as calls on fewer rows."""
    from paper_2309_01226_amd import ops
    flush("rotary large", inplace, dt, T, inter)
    H, dh = 30, 128
    x = torch.randn(T, H * dh, device="cuda").to(dt)
    pos = torch.randint(-99, 999, (T, 2), device="cuda", dtype=torch.int32)
    kw = dict(interleaved=inter, inverse=True)
    want = torch.cat([ops.rotary_axes(a.clone(), p, H, dh, (24, 40), **kw) for a, p in zip(x.split(1999), pos.split(1999))])
    got = ops.rotary_axes(x, pos, H, dh, (24, 40), out=None if inplace else torch.empty_like(x), **kw)
    assert torch.equal(got, want)
