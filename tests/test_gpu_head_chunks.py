"""The head's calls in several chunks of tokens: by a chunk's statistics, by its 16-bit numbers, by its most rows."""

import pytest
import torch

from tests import test_gpu_linear_xent as T
from tests import test_head_operand as O
from tests.gpu_util import flush
from tests.test_head_workspace import LOOSE, P, _ws

pytestmark = pytest.mark.gpu
BF, F4 = torch.bfloat16, torch.float32


def test_scores_in_chunks():
    """More rows than the statistics of the widest vocabulary allow in one chunk."""
    N, V, d = 9000, 1 << 20, 64
    flush("scores in chunks", N, V, d)
    shared = lambda n: _ws(N=n, V=V, d=d) - (2 * d + 16) * n  # noqa: E731
    assert abs(shared(N) - shared(4608)) < LOOSE  # two chunks: half the rows, in whole tiles
    i = T._inputs(N, V, d, 0.1, "plain")
    o = T._outputs(i, grads="")
    T._call(i, o)
    torch.cuda.synchronize()
    live = (i["labels"] >= 0) & (i["labels"] < V)
    assert o["inv_n"].item() == pytest.approx(1 / int(live.sum()), rel=2.0 ** -23)
    for at in torch.arange(N, device="cuda").split(1000):
        rows = {k: i[k][at] for k in ("x", "labels")}
        want = T._want({**i, **rows}, False)
        T._check({k: o[k][at] for k in ("row_loss", "lse")}, want)


def _several(N, V, d):
    """Several chunks: then bf16 gradients have fp32 sums beside them."""
    a = dict(N=N, V=V, d=d, dx=P, dw=P, db=P, bias=P)
    return _ws(**a) - _ws(**a, grad_f32=1) >= 4 * V * d


@pytest.mark.parametrize("dt", [BF, F4])
def test_chunks_of_a_wide_vocabulary(dt):
    """More rows than there are 16-bit numbers for in 1 GiB: dw and db summed over two chunks."""
    N, V, d = 11000, 50257, 64
    flush("chunks of a wide vocabulary", N, V, d, dt)
    assert _several(N, V, d) and not _several(10496, V, d)
    i = T._inputs(N, V, d, 0.05, "plain", True)
    o = T._outputs(i, dt)
    T._call(i, o)
    torch.cuda.synchronize()
    T._check(o, T._want(i))


@pytest.mark.parametrize("dt,accumulate", [(BF, False), (F4, False), (F4, True)])
@pytest.mark.parametrize("more", [1, 100, 256, 257])
def test_last_chunk_of_few_rows(more, dt, accumulate):
    """A full chunk of rows that take part and a few: those have dz in two parts, and slices chosen on the device."""
    N, V, d, full = 17000, 300, 64, 8704  # two chunks, of 8500 in whole tiles
    flush("last chunk of few rows", more, dt, accumulate)
    assert _several(N, V, d)
    g = torch.Generator().manual_seed(more)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    labels = torch.full((N,), -1, dtype=torch.int32)
    rows = torch.randperm(N, generator=g)[:full + more].sort().values
    labels[rows] = torch.randint(0, V, (full + more,), generator=g, dtype=torch.int32)
    # few entries for the last rows, which then are all that these entries' dw has (but for other rows' softmax, which
    # the bias keeps small)
    labels[rows[:full]] %= V - 20
    labels[rows[full:]] = labels[rows[full:]] % 20 + V - 20
    bias = r(V)
    bias[-20:] -= 14
    i = O.on_device(dict(x=(1.5 * r(N, d)).to(BF), w=(r(V, d) / 8).to(BF), labels=labels, bias=bias, weight=torch.rand(N, generator=g) + 0.1))
    few = torch.zeros(N, dtype=torch.bool)
    few[rows[full:]] = more <= O.FEW
    want = O.gradients(i, few.cuda())
    o = T._outputs(i, dt)
    add = {}
    if accumulate:
        for k in ("dw", "db"):
            add[k] = r(*o[k].shape).cuda() * 1e-3
            o[k].copy_(add[k])
    T._call(i, o, accumulate=accumulate)
    torch.cuda.synchronize()
    T._check({k: o[k] for k in want}, want, {k: t.double() for k, t in add.items()})
    T._check({k: o[k] for k in ("row_loss", "lse", "inv_n")}, T._want(i, False))


@pytest.mark.parametrize("N,V,d,ignored", [(1, 2, 8, 0.0), (33, 257, 1024, 0.3), (333, 1501, 256, 0.3), (300, 9001, 768, 0.1), (700, 2050, 320, 0.5),
                                           (17000, 300, 64, 0.45), (2000, 20011, 256, 0.9)])
def test_workspace_contents(N, V, d, ignored):
    """What a workspace holds before a call (zeros, NaN) reaches no output, nor do outputs' own earlier values."""
    from paper_2309_01226_amd import _lib as L
    flush("workspace contents", N, V, d, ignored)
    i = T._inputs(N, V, d, ignored, "plain", True)
    for dt, grads in ((BF, "dx dw db"), (F4, "dx dw db"), (BF, "dx"), (F4, "dw"), (BF, "db"), (BF, "")):
        seen = []
        for fill in (0, 255):
            o = T._outputs(i, dt, grads=grads)
            for t in o.values():
                t.view(torch.uint8).fill_(fill)
            at = lambda k: o[k].data_ptr() if k in o else None  # noqa: E731
            sizes = dict(N=N, V=V, d=d, dx=at("dx"), dw=at("dw"), db=at("db"), bias=i["bias"].data_ptr(), grad_f32=dt == F4)
            ws = torch.full((_ws(**sizes),), fill, dtype=torch.uint8, device="cuda")
            L.call("sat_op_linear_xent", L.sat_linear_xent_desc(
                x=i["x"].data_ptr(), ldx=d, w=i["w"].data_ptr(), ldw=d, labels=i["labels"].data_ptr(), row_weight=i["weight"].data_ptr(),
                row_loss=at("row_loss"), lse=at("lse"), inv_n=at("inv_n"), lddx=d, lddw=d, ws=ws.data_ptr(), ws_bytes=ws.numel(), **sizes),
                torch.cuda.current_stream().cuda_stream)
            torch.cuda.synchronize()
            seen.append(o)
        assert all(torch.equal(seen[0][k], seen[1][k]) for k in o), (dt, grads)
