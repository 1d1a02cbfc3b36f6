"""Rows and entries whose offsets pass 32 bits: the same as the same rows in small buffers."""

import pytest
import torch

from tests import test_head_operand as O
from tests.gpu_util import flush

pytestmark = pytest.mark.gpu
BF, F4 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


def _far(rows, pitch, d, dt):
    """[rows, d] of a buffer whose rows are far apart (what lies between is not set)."""
    return torch.empty(rows, pitch, dtype=dt, device="cuda")[:, :d]


@pytest.mark.parametrize("dt", [BF, F4])
def test_dropout(dt):
    from paper_2309_01226_amd import ops
    rows, cols, pitch = 70001, 41, 65536
    flush("far dropout", dt)
    near = torch.randn(rows, cols, device="cuda").to(dt)
    far = _far(rows, pitch, cols, dt)
    assert rows * pitch > 1 << 32
    far.copy_(near)
    want = ops.dropout(near, 0.3, 9, out=torch.empty_like(near))
    assert torch.equal(ops.dropout(far, 0.3, 9, out=torch.empty_like(near)), want)  # far reads
    assert torch.equal(ops.dropout(far, 0.3, 9), want)  # and writes


@pytest.mark.parametrize("pitch,small", [((1 << 21) - 8, 264), ((1 << 21) + 8, 265)])  # whole 16-byte pieces, and by elements
def test_boundary(pitch, small):
    from paper_2309_01226_amd import ops
    T, d = 2100, 264
    flush("far boundary", pitch)
    assert T * pitch > 1 << 32
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x, f, dy, dh = (torch.randn(T, d, device="cuda", generator=g).to(BF) for _ in range(4))
    kw = dict(pre="layer", post="rms", gate=torch.randn(d, device="cuda", generator=g), p=0.2, seed=3)

    def go(width):
        m = lambda t=None: _far(T, width, d, BF) if t is None else _far(T, width, d, BF).copy_(t)  # noqa: E731
        st, dgate = torch.empty(4, T, device="cuda"), torch.empty(d, device="cuda")
        a, b, h = m(x), m(f), m()
        ops.residual_norm_fwd(a, b, a, h, st, d, **kw)
        y, next_in = a.clone(), h.clone()
        c, e = m(dy), h.copy_(dh)
        df = m()
        ops.residual_norm_bwd(c, e, a, b, st, c, df, d, dgate=dgate, **kw)
        return y, next_in, st, c, df, dgate

    for name, p, q in zip(("y", "h", "stats", "dx", "df", "dgate"), go(pitch), go(small)):
        assert torch.equal(p, q), name


def test_head():
    """w and dw of more than 2^31 elements, x and dx with rows far apart."""
    from paper_2309_01226_amd import ops
    N, V, d, pitch = 1100, 1 << 20, 2056, (1 << 21) - 8
    flush("far head")
    assert V * d > 1 << 31 and N * pitch > 1 << 31
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    w = torch.empty(V, d, dtype=BF, device="cuda")
    for part in w.split(1 << 16):
        part.copy_(torch.randn(part.shape, device="cuda", generator=g) / 45)
    labels = torch.randint(0, V, (N,), device="cuda", generator=g, dtype=torch.int32)
    labels[::3] = V - 1 - labels[::3] % 50
    x, dx = _far(N, pitch, d, BF), _far(N, pitch, d, BF)
    x.copy_(torch.randn(N, d, device="cuda", generator=g) + 8 * w[labels.long()].float())
    dw = torch.full((V, d), 7.0, dtype=BF, device="cuda")
    loss, lse, inv = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty(1, device="cuda")
    ops.linear_cross_entropy(x, w, labels, loss, lse, inv, dx=dx, dw=dw)
    torch.cuda.synchronize()
    # some rows, over all entries; and some entries, over all rows, whose lse is the kernel's (held by the first check)
    at = torch.tensor([0, 1, 2, N // 2, N - 3, N - 2, N - 1], device="cuda")
    xs = x[at].double()
    z = torch.cat([xs @ part.double().T for part in w.split(1 << 16)], 1)
    ref = torch.logsumexp(z, 1)
    # of a logit: a sum of d products, whose magnitudes add up to |x| |w| at most
    long = max(part.float().norm(dim=1).max().item() for part in w.split(1 << 16)) * x.float().norm(dim=1).max().item()
    bound = 2 * O.E * (d + 2) * long + 300 * O.E
    assert ((lse[at].double() - ref).abs() <= bound).all()
    dz = torch.exp(z - ref[:, None])
    dz[torch.arange(len(at)), labels[at].long()] -= 1
    want = sum(a.double() @ b.double() for a, b in zip(dz.split(1 << 16, 1), w.split(1 << 16))) / N
    # dz is off by 2^-8 and 2^-11.5 of itself, dx by its own rounding; sums of V terms: 2 E (V + 2) of their magnitudes
    size = sum(a.abs() @ b.double().abs() for a, b in zip(dz.split(1 << 16, 1), w.split(1 << 16))) / N
    assert ((dx[at].double() - want).abs() <= (2.0 ** -8 * 1.1 + 2.0 ** -11.5 + bound * 2) * size + 2.0 ** -8 * want.abs() + 2 * O.E * (V + 2) * size).all()
    entries = torch.cat([labels[:40].long().unique(), torch.tensor([0, 1, V // 2, V - 60, V - 1], device="cuda")]).unique()
    ze = x.double() @ w[entries].double().T
    de = torch.exp(ze - lse.double()[:, None]) - (labels.long()[:, None] == entries[None]).double()
    want, size = de.T @ x.double() / N, de.abs().T @ x.double().abs() / N
    assert ((dw[entries].double() - want).abs() <= (2.0 ** -8 * 1.1 + 2.0 ** -11.5 + bound * 2) * size + 2.0 ** -8 * want.abs()
            + 2 * O.E * (N + 2) * size).all()
    assert not (dw == 7).any()


@pytest.mark.parametrize("rows,cols", [((1 << 32) + 5, 1), (1 << 31, 1)])
def test_too_many_rows(rows, cols):
    """More rows than 32 bits hold are refused, not cut to what they hold."""
    from paper_2309_01226_amd import _lib, ops
    flush("too many rows", rows)
    x = torch.empty(rows, cols, dtype=BF, device="cuda")
    x[:8] = 1
    with pytest.raises((ValueError, _lib.SatError)):
        ops.dropout(x, 0.5, 1)
    assert (x[:8] == 1).all()


def test_too_many_rows_to_turn():
    from paper_2309_01226_amd import ops
    flush("too many rows to turn")
    rows = (1 << 32) + 3
    x, pos = torch.empty(rows, 2, dtype=BF, device="cuda"), torch.empty(rows, 1, dtype=torch.int32, device="cuda")
    x[:8], pos[:8] = 1, 1
    with pytest.raises(ValueError):
        ops.rotary_axes(x, pos, 1, 2, [1])
    assert (x[:8] == 1).all()
