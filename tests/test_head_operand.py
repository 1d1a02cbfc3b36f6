"""How exact the head's gradients are: the operand dz of their products, seen by itself and in random products, against
bounds of the scheme that saturn_ops.h states.  That the bounds tell this scheme from coarser ones is shown on the CPU."""

import math

import pytest
import torch

from tests import block_ref as R
from tests.gpu_util import flush

BF, F4 = torch.bfloat16, torch.float32
E = R.E
HALF = {BF: 2.0 ** -8, F4: 2.0 ** -24}
FEW = 256  # rows of a chunk up to which dz is kept in two parts


# ---------------------------------------------------------------- the bounds

def operand(i, few):
    """(dz, its bound, c p's part of it) in 64 bits.  few [N]: whether the row's chunk keeps dz in two parts.

    block_ref.head derives the relative error of exp(z - lse) before it is kept: op + ol + 8 E.  It is kept as 16
    bits of log2: half a step of 2^-10, ln 2 / 2^11 < 2^-11.5 of the value, where it is within 2^-32 of the largest of its
    piece (and so wherever it is within 2^-32 of the row's largest), four times that below; a value below 2^-159 of it
    may be 0.  The label's entry is not kept but formed from its fp32 logit.  Then one rounding to bf16, 2^-8; of two
    parts the second rounds what the first lost: 2^-16.  db sums dz before that rounding."""
    x, w, labels = i["x"].double(), i["w"].double(), i["labels"].long()
    N, V, d = len(labels), len(w), x.shape[1]
    live = (labels >= 0) & (labels < V)
    at = torch.where(live, labels, 0)[:, None]
    z, oz = x @ w.T, 2 * E * (d + 2) * (x.abs() @ w.abs().T)
    if i["bias"] is not None:
        b = i["bias"].double()
        z, oz = z + b, oz + E * b.abs() + E * (z + b).abs()
    lse, top = torch.logsumexp(z, 1, keepdim=True), z.amax(1, keepdim=True)
    p, far = torch.exp(z - lse), top - z
    op = oz + 4 * E * far + 2.0 ** -22
    ol = (p * op).sum(1, keepdim=True) + 256 * E
    n = max(1, int(live.sum()))
    c = (torch.full((N,), 1 / n, dtype=torch.float64, device=x.device) if i["weight"] is None else i["weight"].double()) * live
    c = c[:, None]
    hot = torch.zeros_like(p).scatter_(1, at, 1.0)
    dz = c * (p - hot)
    kept = torch.where(far * math.log2(math.e) < 31.9, 2.0 ** -11.5, 2.0 ** -9.5) * (1 - hot)
    before = (c.abs() * p * (op + ol + 8 * E + kept) + 4 * E * c.abs() * hot + c.abs() * 2.0 ** -159) * 1.001
    last = torch.where(few, 2.0 ** -16, 2.0 ** -8)[:, None]
    return dz, before + 1.01 * last * dz.abs(), before


def gradients(i, few):
    """{name: (value, bound)}: the products' sums of n terms, twice as many in two parts, as in block_ref.head; 1 / n or
    its product takes four roundings more."""
    dz, odz, before = operand(i, few)
    x, w, N, V = i["x"].double(), i["w"].double(), len(dz), dz.shape[1]
    total = lambda a, oa, b, k: (a @ b, oa @ b.abs() + 2 * E * (2 * k + 4) * (a.abs() @ b.abs()) + 2.0 ** -120)  # noqa: E731
    out = dict(dx=total(dz, odz, w, V), dw=total(dz.T.contiguous(), odz.T.contiguous(), x, N))
    out["db"] = dz.sum(0), before.sum(0) + E * (N + 4) * dz.abs().sum(0) + 2.0 ** -120
    return out


def worst(got, want, dt):
    value, bound = want
    bound = bound + HALF[dt] * (value.abs() + bound)
    return ((got.double() - value).abs() / bound).max().item()


# ---------------------------------------------------------------- inputs

def _labels(g, N, V):
    return torch.randint(0, V, (N,), generator=g, dtype=torch.int32)


def shown_by_dw(N, V=300, weights=False):
    """Rows that are 4 times a unit vector each: dw[v, t] is 4 dz[t, v]."""
    g = torch.Generator().manual_seed(N)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return dict(x=(4 * torch.eye(N)).to(BF), w=r(V, N).to(BF), labels=_labels(g, N, V), bias=r(V),
                weight=torch.rand(N, generator=g) + 0.1 if weights else None)


def shown_by_dx(N, V=256, weights=False):
    """Entries that are 167 / 128 times a unit vector: dx[t, v] is as much of dz[t, v] (which rounds again)."""
    g = torch.Generator().manual_seed(N + 1)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return dict(x=(3 * r(N, V)).to(BF), w=(167 / 128 * torch.eye(V)).to(BF), labels=_labels(g, N, V), bias=r(V),
                weight=torch.rand(N, generator=g) + 0.1 if weights else None)


def random_rows(N, V, d, weights=False):
    g = torch.Generator().manual_seed(7 * N + V + d)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    w = (r(V, d) / math.sqrt(d)).to(BF)
    labels = _labels(g, N, V)
    x = 1.5 * r(N, d) + w[labels.long()].float() * 16 * torch.rand(N, 1, generator=g) ** 2
    return dict(x=x.to(BF), w=w, labels=labels, bias=0.5 * r(V), weight=torch.rand(N, generator=g) - 0.3 if weights else None)


SHOWN = [(n, weights) for n in (64, 256, 264, 512) for weights in (False, True)]
SIZES = [(64, 512, 64), (256, 256, 128), (33, 257, 1024), (3, 7, 16), (1, 2, 8), (17, 500, 200), (257, 255, 136), (300, 1000, 64), (511, 640, 512)]


def few_rows(i):
    return torch.full((len(i["labels"]),), len(i["labels"]) <= FEW, device=i["labels"].device)


# ---------------------------------------------------------------- what the bounds tell apart

def coarser(i, exponentials=False):
    """{name: gradient} in 64 bits from dz that is rounded to bf16 once, after bf16 exponentials (of z - the row's maximum) or not."""
    dz = operand(i, few_rows(i))[0]
    n = i["labels"].shape[0]
    unit = dz * n if i["weight"] is None else dz  # the common factor stays out of the operand
    if exponentials:
        z = i["x"].double() @ i["w"].double().T + i["bias"].double()
        e = torch.exp(z - z.amax(1, keepdim=True))
        c = 1.0 if i["weight"] is None else i["weight"].double()[:, None]
        rounded = c * e.to(BF).double() / e.sum(1, keepdim=True)
        unit = torch.where(torch.arange(dz.shape[1]) == i["labels"].long()[:, None], unit, rounded)
    unit = unit.to(BF).double()
    dz = unit / n if i["weight"] is None else unit
    return dict(dx=dz @ i["w"].double(), dw=dz.T @ i["x"].double())


@pytest.mark.parametrize("weights", [False, True])
def test_bounds_tell_one_part_from_two(weights):
    """A single bf16 operand breaks the bound of few rows, in each product."""
    for N in (64, 256):
        i = shown_by_dw(N, weights=weights)
        assert worst(coarser(i)["dw"].float(), gradients(i, few_rows(i))["dw"], F4) > 2
        i = shown_by_dx(N, weights=weights)
        assert worst(coarser(i)["dx"].to(BF), gradients(i, few_rows(i))["dx"], BF) > 1.2
    for size in SIZES[:4]:
        i = random_rows(*size, weights)
        want, got = gradients(i, few_rows(i)), coarser(i)
        assert worst(got["dw"].float(), want["dw"], F4) > 2, size
        if size[2] < 1024:  # (there each element of dx has a sum of 257 terms of like size, and its own rounding hides them)
            assert worst(got["dx"].to(BF), want["dx"], BF) > 1.2, size


@pytest.mark.parametrize("weights", [False, True])
def test_bounds_tell_rounded_exponentials(weights):
    """bf16 exponentials before the bf16 operand break the bound of many rows."""
    i = shown_by_dw(512, weights=weights)
    want = gradients(i, few_rows(i))["dw"]
    assert worst(coarser(i)["dw"].float(), want, F4) <= 1
    assert worst(coarser(i, True)["dw"].float(), want, F4) > 1.2


def test_values_are_the_reference():
    for size in SIZES:
        i = random_rows(*size, True)
        want = R.head(*(i[k].double() for k in ("x", "w")), i["labels"].long(), i["bias"].double(), i["weight"].double())
        for k, (value, bound) in gradients(i, few_rows(i)).items():
            assert torch.allclose(value, want[k][0], rtol=1e-12, atol=1e-15) and (bound < 2 * want[k][1] + 1e-30).all(), (size, k)


# ---------------------------------------------------------------- the kernels

def call(i, dt, grads="dx dw db"):
    from paper_2309_01226_amd import ops
    e = lambda s, t: torch.full(s, 7.0, device="cuda", dtype=t)  # noqa: E731
    (N, d), V = i["x"].shape, len(i["w"])
    o = {k: t for k, t in (("dx", e((N, d), BF)), ("dw", e((V, d), dt)), ("db", e((V,), dt))) if k in grads}
    ops.linear_cross_entropy(i["x"], i["w"], i["labels"], e((N,), F4), e((N,), F4), e((1,), F4), bias=i["bias"], row_weight=i["weight"], **o)
    torch.cuda.synchronize()
    return o


def on_device(i):
    return {k: None if t is None else t.cuda() for k, t in i.items()}


@pytest.mark.gpu
@pytest.mark.parametrize("N,weights", SHOWN)
def test_operand_of_dw(N, weights):
    flush("operand of dw", N, weights)
    i = on_device(shown_by_dw(N, weights=weights))
    assert worst(call(i, F4)["dw"], gradients(i, few_rows(i))["dw"], F4) <= 1


@pytest.mark.gpu
@pytest.mark.parametrize("N,weights", SHOWN)
def test_operand_of_dx(N, weights):
    flush("operand of dx", N, weights)
    i = on_device(shown_by_dx(N, weights=weights))
    assert worst(call(i, F4)["dx"], gradients(i, few_rows(i))["dx"], BF) <= 1


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF, F4])
@pytest.mark.parametrize("N,V,d", SIZES)
def test_products(N, V, d, dt):
    for weights in (False, True):
        flush("products", N, V, d, dt, weights)
        i = on_device(random_rows(N, V, d, weights))
        o, want = call(i, dt), gradients(i, few_rows(i))
        for k in o:
            assert worst(o[k], want[k], o[k].dtype) <= 1, k
