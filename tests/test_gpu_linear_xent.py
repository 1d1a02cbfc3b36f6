"""The head with its cross entropy against its 64-bit form; block_ref derives the bounds."""

import math

import pytest
import torch

from tests import block_ref as R
from tests.gpu_util import flush

pytestmark = pytest.mark.gpu
BF, F4, F8 = torch.bfloat16, torch.float32, torch.float64
HALF = {BF: 2.0 ** -8, F4: 2.0 ** -24}


def _inputs(N, V, d, ignored=0.0, bias=None, weights=False, spare=0, seed=0):
    """Logits of a few units, some rows near sure of their label; labels < 0 and >= V among the ignored."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 * N + 10 * V + d + seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    w = (r(V, d + spare) / math.sqrt(d)).to(BF)[:, :d]
    labels = torch.randint(0, V, (N,), device="cuda", generator=g)
    x = 1.5 * r(N, d + spare)
    x[:, :d] += w[labels].float() * 16 * torch.rand(N, 1, device="cuda", generator=g) ** 2
    out = torch.rand(N, device="cuda", generator=g) < ignored
    odd = torch.tensor([-1, -100, V, 2 ** 31 - 1, -2 ** 31], device="cuda")
    labels = torch.where(out, odd[torch.arange(N, device="cuda") % 5], labels)
    b = None
    if bias:
        b = 0.5 * r(V)
        if bias == "masked" and V > 4:
            keep = torch.zeros(V, dtype=torch.bool, device="cuda")
            keep[labels[(labels >= 0) & (labels < V)]] = True
            b[(torch.rand(V, device="cuda", generator=g) < 0.4) & ~keep] = -math.inf
    return dict(x=x.to(BF)[:, :d], w=w, labels=labels.to(torch.int32), bias=b,
                weight=torch.rand(N, device="cuda", generator=g) - 0.3 if weights else None)


def _outputs(i, dt=BF, spare=0, grads="dx dw db"):
    (N, d), V = i["x"].shape, len(i["w"])
    o = dict(row_loss=torch.full((N,), 7.0, device="cuda"), lse=torch.full((N,), 7.0, device="cuda"), inv_n=torch.full((1,), 7.0, device="cuda"))
    full = lambda r, t: torch.full((r, d + spare), 7.0, device="cuda", dtype=t)[:, :d]  # noqa: E731
    if "dx" in grads:
        o["dx"] = full(N, BF)
    if "dw" in grads:
        o["dw"] = full(V, dt)
    if "db" in grads and i["bias"] is not None:
        o["db"] = torch.full((V,), 7.0, device="cuda", dtype=dt)
    return o


def _call(i, o, **kw):
    from paper_2309_01226_amd import ops
    ops.linear_cross_entropy(i["x"], i["w"], i["labels"], o["row_loss"], o["lse"], o["inv_n"], bias=i["bias"], row_weight=i["weight"],
                             **{k: o[k] for k in ("dx", "dw", "db") if k in o}, **kw)


def _want(i, grads=True):
    c = lambda t: None if t is None else t.double()  # noqa: E731
    return R.head(c(i["x"]), c(i["w"]), i["labels"].long(), c(i["bias"]), c(i["weight"]), grads)


def _check(o, want, add=None):
    for k, got in o.items():
        value, bound = want[k]
        got = got.double()
        if add and k in add:
            value, bound = value + add[k], bound + R.E * (value + add[k]).abs() + R.E * add[k].abs()
        assert got.shape == value.shape, k
        same = got == value  # infinities
        bound = bound + HALF[o[k].dtype] * (value.abs() + bound)
        off = torch.where(same, 0.0, (got - value).abs() / bound.clamp(min=1e-300))
        assert not off.isnan().any() and (off.numel() == 0 or off.max().item() <= 1), (k, off.max().item(), int(off.argmax()))


@pytest.mark.parametrize("N,V,d", [
    (1, 1, 8), (1, 2, 8), (3, 7, 16), (64, 512, 64), (5, 129, 72), (256, 256, 128), (257, 255, 136), (300, 1000, 64), (17, 5001, 200),
    (511, 640, 512), (700, 2050, 320), (33, 257, 1024), (1, 4099, 768),
])
@pytest.mark.parametrize("ignored,bias,weights,dt", [(0.0, None, False, BF), (0.4, "masked", True, F4), (0.9, "plain", False, BF)])
def test_sizes(N, V, d, ignored, bias, weights, dt):
    flush("linear_xent", N, V, d, ignored, bias, weights, dt)
    i = _inputs(N, V, d, ignored, bias, weights, spare=8 if weights else 0)
    o = _outputs(i, dt, spare=16 if weights else 0)
    _call(i, o)
    torch.cuda.synchronize()
    want = _want(i)
    _check(o, want)
    out = (i["labels"] < 0) | (i["labels"] >= V)
    assert not o["dx"][out].any() and not o["row_loss"][out].any() and not o["lse"][out].any()
    if weights:  # columns behind d stay as they are
        for k in ("dx", "dw"):
            wide = o[k].as_strided((o[k].shape[0], 16), o[k].stride(), d)
            assert (wide == 7).all(), k
    again = _outputs(i, dt)
    _call(i, again)
    assert all(torch.equal(again[k], o[k]) for k in o)


def test_scores_alone():
    """Without gradients: the same losses, bit for bit; each gradient alone is the one of the full call."""
    i = _inputs(333, 1500, 256, 0.3, "masked", True)
    full = _outputs(i)
    _call(i, full)
    for grads in ("", "dx", "dw", "db", "dx db"):
        o = _outputs(i, grads=grads)
        _call(i, o)
        assert all(torch.equal(o[k], full[k]) for k in o), grads


@pytest.mark.parametrize("rows", [1, 2, 8, 16, 17, 40, 64, 65])
def test_few_rows(rows):
    """The next tokens of a few sequences, scored, over a vocabulary of many tiles."""
    flush("few rows", rows)
    i = _inputs(rows, 20011, 512)
    o = _outputs(i, grads="")
    _call(i, o)
    torch.cuda.synchronize()
    _check(o, _want(i, False))


@pytest.mark.parametrize("rows,V,ignored", [(1, 300, 1.0), (7, 50, 0.5), (128, 700, 0.3), (129, 700, 0.3), (90, 1000, 1.0)])
def test_few_rows_without_labels(rows, V, ignored):
    """Few rows scored, some or all of which take no part, whatever they hold."""
    flush("few rows without labels", rows, V, ignored)
    i = _inputs(rows, V, 136, ignored, "plain", spare=8)
    out = (i["labels"] < 0) | (i["labels"] >= V)
    i["x"][out] = math.nan
    o = _outputs(i, grads="")
    _call(i, o)
    torch.cuda.synchronize()
    assert not o["row_loss"][out].any() and not o["lse"][out].any()
    i["x"][out] = 0.0
    _check(o, _want(i, False))


@pytest.mark.parametrize("N,V,d,ignored,dt", [
    (17000, 300, 64, 0.0, BF), (17000, 300, 64, 0.45, F4), (6000, 50257, 64, 0.0, BF), (40000, 70, 32, 0.7, BF),
    (12000, 66, 96, 0.3, BF), (12001, 66, 96, 0.3, F4)])
def test_chunks(N, V, d, ignored, dt):
    """More rows than a chunk holds (with many ignored, the last chunks are empty), or than one kernel numbers."""
    flush("chunks", N, V, d, ignored, dt)
    i = _inputs(N, V, d, ignored, "plain", True)
    o = _outputs(i, dt)
    _call(i, o)
    torch.cuda.synchronize()
    _check(o, _want(i))


@pytest.mark.parametrize("N,V,d", [(4000, 1000, 1280), (2048, 130, 2048), (300, 9000, 768), (1500, 20000, 256)])
def test_split_products(N, V, d):
    """Products whose K is split: few tiles of a long sum."""
    flush("split", N, V, d)
    i = _inputs(N, V, d, 0.2)
    o = _outputs(i)
    _call(i, o)
    torch.cuda.synchronize()
    _check(o, _want(i))


@pytest.mark.parametrize("N,V,d,dt", [(33, 40000, 200, BF), (300, 34001, 520, F4), (1, 50001, 1024, BF), (2000, 8000, 800, F4)])
def test_many_tiles(N, V, d, dt):
    """Products of more small tiles than there are compute units, with and without gradients, the same on each call."""
    flush("many tiles", N, V, d, dt)
    i = _inputs(N, V, d, 0.2 if N > 1 else 0.0, "masked", True, spare=8)
    o, again, scored = _outputs(i, dt, spare=16), _outputs(i, dt), _outputs(i, grads="")
    for each in (o, again, scored):
        _call(i, each)
    torch.cuda.synchronize()
    _check(o, _want(i))
    assert all(torch.equal(again[k], o[k]) for k in o) and all(torch.equal(scored[k], o[k]) for k in scored)


def test_accumulate():
    for N, V in ((200, 700), (17000, 64)):  # one chunk and two
        i = _inputs(N, V, 128, 0.3, "plain")
        o = _outputs(i, F4)
        g = torch.Generator(device="cuda")
        g.manual_seed(5)
        add = {k: torch.randn(o[k].shape, device="cuda", generator=g) * 1e-3 for k in ("dw", "db")}
        for k in add:
            o[k].copy_(add[k])
        _call(i, o, accumulate=True)
        torch.cuda.synchronize()
        _check(o, _want(i), {k: v.double() for k, v in add.items()})


@pytest.mark.parametrize("N", [0, 5])
def test_no_row_takes_part(N):
    i = _inputs(N, 300, 64, 1.1, "plain")
    for dt in (BF, F4):
        o = _outputs(i, dt)
        _call(i, o)
        torch.cuda.synchronize()
        assert o["inv_n"].item() == 1 and not any(o[k].any() for k in o if k != "inv_n")
    o["dw"].fill_(3.0)
    o["db"].fill_(3.0)
    _call(i, o, accumulate=True)
    assert (o["dw"] == 3).all() and (o["db"] == 3).all()


def test_masked_vocabulary():
    """Every entry of a piece, of all but one, of all pieces at -inf."""
    i = _inputs(70, 900, 64, 0.0, "plain")
    i["labels"] = i["labels"] % 100 + 400
    i["bias"][:384] = -math.inf
    i["bias"][512:] = -math.inf
    o = _outputs(i)
    _call(i, o)
    torch.cuda.synchronize()
    _check(o, _want(i))
    assert not o["dw"][:384].any() and not o["dw"][512:].any() and not o["db"][512:].any()
    i["bias"].fill_(-math.inf)
    i["bias"][450] = 0.0
    i["labels"].fill_(450)
    _call(i, o)  # one entry: sure
    assert (o["row_loss"] == 0).all() and not o["dx"].any() and not o["dw"].any()
    i["labels"][3] = 451  # an entry that is out: infinite loss, finite gradients
    _call(i, o)
    assert o["row_loss"][3] == math.inf and all(torch.isfinite(o[k]).all() for k in ("dx", "dw", "db"))
    i["bias"].fill_(-math.inf)
    _call(i, o)
    assert not o["row_loss"].any() and (o["lse"] == -math.inf).all() and not any(o[k].any() for k in ("dx", "dw", "db"))


def test_large_logits():
    """Logits of +-1000: no overflow, the running maximum carries them."""
    i = _inputs(90, 600, 64, 0.0, "plain")
    i["bias"] = torch.linspace(-1000, 1000, 600, device="cuda")
    o = _outputs(i)
    _call(i, o)
    torch.cuda.synchronize()
    _check(o, _want(i))


def test_spoiled_rows():
    """NaN in an ignored row reaches nothing; in another row its own loss and dx."""
    i = _inputs(64, 300, 64, 0.3)
    out = i["labels"] < 0
    i["x"][out] = float("nan")
    o = _outputs(i)
    _call(i, o)
    torch.cuda.synchronize()
    assert all(torch.isfinite(o[k]).all() for k in o)
    row = int((i["labels"] >= 0).nonzero()[0])
    i["x"][row] = float("nan")
    _call(i, o)
    ok = torch.arange(64, device="cuda") != row
    assert torch.isnan(o["row_loss"][row]) and torch.isfinite(o["row_loss"][ok]).all() and torch.isfinite(o["dx"][ok]).all()


def test_as_the_kept_logits():
    """The losses of the framework's cross entropy on kept logits, and its gradient's products."""
    from paper_2309_01226_amd import ops
    i = _inputs(128, 1000, 256, 0.25)
    N, V, d = 128, 1000, 256
    i["labels"] = torch.where(i["labels"] < V, i["labels"].clamp(min=-1), -1).to(torch.int32)
    o = _outputs(i, F4)
    _call(i, o)
    z, dz = torch.empty(N, V, device="cuda"), torch.empty(N, V, dtype=BF, device="cuda")
    loss, inv = torch.empty(N, device="cuda"), torch.empty(1, device="cuda")
    ops.gemm(i["x"], i["w"], N, V, d, z, lda=d, ldb=d)
    ops.cross_entropy(z, i["labels"], loss, dz, inv, N, V)
    dw = torch.empty(V, d, device="cuda")
    ops.gemm(dz, i["x"], V, d, N, dw, lda=V, ldb=d, a_layout=ops.LAY_MN, b_layout=ops.LAY_MN)
    want = _want(i)
    _check({k: o[k] for k in ("row_loss", "dw")}, want)
    _check({"row_loss": loss, "inv_n": inv}, want)
    value, bound = want["dw"]
    assert ((dw.double() - value).abs() <= bound).all() and torch.equal(inv, o["inv_n"])


def test_refusals():
    from paper_2309_01226_amd import _lib
    i = _inputs(8, 40, 64, 0.0, "plain", True)
    o = _outputs(i)
    _call(i, o)
    for k, bad in (("x", i["x"].float()), ("x", i["x"][:7]), ("x", i["x"][:, :56]), ("w", i["w"].T), ("labels", i["labels"].long()),
                   ("bias", i["bias"][:39]), ("weight", i["weight"].double()), ("x", i["x"].cpu())):
        with pytest.raises((TypeError, ValueError)):
            _call({**i, k: bad}, o)
    for k, bad in (("row_loss", o["row_loss"][:7]), ("lse", o["lse"].double()), ("dx", o["dx"].float()), ("dw", o["dw"][:39]),
                   ("db", o["db"].float()), ("inv_n", o["row_loss"])):
        with pytest.raises((TypeError, ValueError)):
            _call(i, {**o, k: bad})
    with pytest.raises(_lib.SatError):
        _call(i, o, accumulate=True)  # bf16 sums are not added to
    with pytest.raises(_lib.SatError):
        _call({**i, "bias": None}, o)  # db of no bias
    with pytest.raises(_lib.SatError):
        odd = torch.empty(8, 65, dtype=BF, device="cuda")[:, :64]
        _call({**i, "x": odd}, o)


def test_streams_and_graph():
    """Two streams at once; two graphs, replayed with other labels and inputs: the eager call's bits."""
    i = _inputs(300, 1111, 128, 0.3, "plain")
    eager, same = _outputs(i), lambda a, b: all(torch.equal(a[k], b[k]) for k in a)
    _call(i, eager)
    torch.cuda.synchronize()
    sides = [(torch.cuda.Stream(), _outputs(i)) for _ in range(2)]
    for s, o in sides:
        with torch.cuda.stream(s):
            _call(i, o)
    torch.cuda.synchronize()
    assert all(same(o, eager) for _, o in sides)
    graphs = []
    for _ in range(2):
        o, g = _outputs(i), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _call(i, o)
        graphs.append((g, o))
    for k in range(4):
        j = _inputs(300, 1111, 128, (0.0, 0.9, 1.1, 0.3)[k], "plain", seed=k)
        for n in ("x", "labels"):
            i[n].copy_(j[n])
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        _call(i, eager)
        torch.cuda.synchronize()
        assert all(same(o, eager) for _, o in graphs), k
