"""Dropout against its definition: the numbers are whole, the product with the factor is one rounding of fp32 and
one of the type, so every element is the reference's bit for bit."""

import numpy as np
import pytest
import torch

from tests import block_ref as R
from tests.gpu_util import flush

pytestmark = pytest.mark.gpu
BF, F4 = torch.bfloat16, torch.float32


def _want(x, p, seed, step=0):
    keep, up = R.kept(*x.shape, p, seed, step)
    return torch.where(torch.as_tensor(keep), (x.float() * torch.tensor(up)).to(x.dtype), torch.zeros((), dtype=x.dtype))


def _same(a, b):
    bits = torch.int16 if a.dtype == BF else torch.int32
    return torch.equal(a.contiguous().view(bits), b.contiguous().view(bits))


def _randn(rows, width, dt, seed=0):
    return torch.as_tensor(np.random.default_rng((rows, width, seed)).normal(size=(rows, width)), dtype=F4).to(dt)


@pytest.mark.parametrize("dt", [BF, F4])
@pytest.mark.parametrize("rows,cols,spare,offset", [
    (1, 1, 0, 0), (1, 8, 0, 0), (3, 7, 1, 1), (257, 64, 0, 0), (100, 1021, 3, 5), (5, 8192, 8, 0), (2000, 9, 0, 3), (33, 255, 2, 1),
    (4097, 40, 0, 8), (2, 65536, 0, 0), (1, 1 << 18, 0, 0), (600, 16, 16, 2),
])
@pytest.mark.parametrize("p,seed,step", [(0.1, 1, None), (0.5, (1 << 64) - 1, (5 << 32) + 7)])
def test_dropout(rows, cols, spare, offset, p, seed, step, dt):
    from paper_2309_01226_amd import ops
    flush("dropout", rows, cols, spare, offset, p, dt)
    x = _randn(rows, cols + spare, dt)
    want = x.clone()
    want[:, :cols] = _want(x[:, :cols], p, seed, step or 0)
    st = None if step is None else torch.tensor([step], device="cuda")
    buf = torch.full((x.numel() + 32,), 3.0, dtype=dt, device="cuda")
    xd = buf[offset:offset + x.numel()].view(x.shape)
    xd.copy_(x)
    out = torch.full((rows, cols + spare + 1), 7.0, dtype=dt, device="cuda")
    ops.dropout(xd[:, :cols], p, seed, step=st, out=out[:, :cols])
    torch.cuda.synchronize()
    assert _same(out[:, :cols].cpu(), want[:, :cols]) and (out[:, cols:] == 7).all() and _same(xd.cpu(), x)
    got = ops.dropout(xd[:, :cols], p, seed, step=st)  # in place
    torch.cuda.synchronize()
    assert got.data_ptr() == xd.data_ptr() and _same(xd.cpu(), want)
    assert (buf[:offset] == 3).all() and (buf[offset + x.numel():] == 3).all()


@pytest.mark.parametrize("dt", [BF, F4])
def test_rates(dt):
    """p 0 copies, p 1 leaves zeros, the least p that 16 bits can say drops its share; the mean stays."""
    from paper_2309_01226_amd import ops
    x = _randn(512, 4096, dt).cuda()
    out = torch.empty_like(x)
    assert _same(ops.dropout(x, 0.0, 5, out=out), x)
    assert not ops.dropout(x, 1.0, 5, out=out).any()
    ones = torch.ones(2048, 8192, dtype=F4, device="cuda")
    n = ones.numel()
    for p in (2.0 ** -16, 0.01, 0.37, 0.9, 65535 / 65536):
        y = ops.dropout(ones, p, 77)
        share = (y == 0).double().mean().item()
        q = round(65536 * p) / 65536
        # five deviations of n independent draws
        assert abs(share - q) <= 5 * (q * (1 - q) / n) ** 0.5, (p, share)
        ones.fill_(1.0)


def test_dropped_values_do_not_matter():
    from paper_2309_01226_amd import ops
    keep, _ = R.kept(64, 200, 0.4, 9)
    drop = ~torch.as_tensor(keep).cuda()
    for dt in (BF, F4):
        for bad in (float("nan"), float("inf"), -torch.finfo(dt).max):
            x = torch.ones(64, 200, dtype=dt, device="cuda").masked_fill(drop, bad)
            y = ops.dropout(x, 0.4, 9)
            assert (y[drop] == 0).all() and torch.isfinite(y).all()
    x = torch.full((64, 200), float("nan"), device="cuda")  # kept ones stay what they are
    assert torch.isnan(ops.dropout(x, 0.4, 9)[~drop]).all()


def test_seeds_steps_and_rows_differ():
    """Other seeds (either half), steps (either half) and rows drop other elements: two masks of rate 1/2 agree on half."""
    from paper_2309_01226_amd import ops
    ones = lambda: torch.ones(256, 4096, device="cuda")  # noqa: E731
    st = lambda v: torch.tensor([v], device="cuda")  # noqa: E731
    masks = [ops.dropout(ones(), 0.5, s, step=None if t is None else st(t)) > 0
             for s, t in ((1, None), (2, None), (1 << 32, None), (1, 1), (1, 1 << 32))]
    assert torch.equal(masks[0], ops.dropout(ones(), 0.5, 1, step=st(0)) > 0)
    for i, a in enumerate(masks):
        for b in masks[:i]:
            assert abs((a == b).double().mean().item() - 0.5) < 5 * 0.5 / 1024
        assert abs((a[1:] == a[:-1]).double().mean().item() - 0.5) < 5 * 0.5 / 1024


def test_empty_and_strides():
    from paper_2309_01226_amd import ops
    assert ops.dropout(torch.empty(0, 16, device="cuda"), 0.5, 1).shape == (0, 16)
    assert ops.dropout(torch.empty(16, 0, device="cuda"), 0.5, 1).shape == (16, 0)
    x = _randn(64, 48, BF).cuda()
    with pytest.raises(ValueError):
        ops.dropout(x.T, 0.5, 1)
    with pytest.raises(ValueError):
        ops.dropout(x, 0.5, 1, out=torch.empty(64, 47, dtype=BF, device="cuda"))
    with pytest.raises(ValueError):
        ops.dropout(x[0], 0.5, 1)
    with pytest.raises(TypeError):
        ops.dropout(x.half(), 0.5, 1)
    with pytest.raises(TypeError):
        ops.dropout(x, 0.5, 1, step=torch.zeros(1, device="cuda"))
    with pytest.raises(ValueError):
        ops.dropout(x, 0.5, 1 << 64)
    with pytest.raises(ValueError):
        ops.dropout(x, 0.5, -1)


def test_captured_step_moves_on():
    """A captured call takes the step of the replay; backward and forward agree."""
    from paper_2309_01226_amd import ops
    x, g = _randn(33, 264, BF).cuda(), _randn(33, 264, BF, 1).cuda()
    y, dx = torch.empty_like(x), torch.empty_like(x)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ops.dropout(x, 0.3, 11, step=step, out=y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        ops.dropout(x, 0.3, 11, step=step, out=y)
        ops.dropout(g, 0.3, 11, step=step, out=dx)
    for i in range(1, 4):
        graph.replay()
        torch.cuda.synchronize()
        assert _same(y.cpu(), _want(x.cpu(), 0.3, 11, i)) and _same(dx.cpu(), _want(g.cpu(), 0.3, 11, i))


def test_more_elements_than_32_bits():
    """Elements and bytes past 2^32, checked at the borders and at the end."""
    from paper_2309_01226_amd import ops
    rows, cols = 70000, 65536
    x = torch.ones(rows, cols, dtype=BF, device="cuda")
    ops.dropout(x, 0.25, 3)
    for r in (0, 16383, 16384, 32767, 32768, 65535, 65536, rows - 1):
        keep, up = R.kept(1, cols, 0.25, 3, row0=r)
        want = torch.where(torch.as_tensor(keep), torch.tensor(up).to(BF), torch.zeros((), dtype=BF))
        assert _same(x[r:r + 1].cpu(), want), r
