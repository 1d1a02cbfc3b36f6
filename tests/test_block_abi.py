"""Host-side checks of the operators around a step's blocks that need no GPU: refusals of the C entry points before
any launch, workspace sizes, the references against published numbers and differences."""

import ctypes as C
import math

import numpy as np
import pytest

from tests import block_ref as R

P = 1 << 20  # stands for a device address: no call here gets as far as reading it


def _L():
    from paper_2309_01226_amd import _lib
    return _lib


def _refused(fn, *args, word):
    L = _L()
    assert getattr(L.lib(), fn)(*args) == L.SAT_EINVAL
    assert word in L.last_error()


# ---------------------------------------------------------------- dropout

@pytest.mark.parametrize("bad", [
    dict(x=None), dict(y=None), dict(x=P + 1), dict(y=P + 2, f32=1), dict(rows=-1), dict(cols=-1), dict(cols=(1 << 18) + 1, ldx=1 << 19, ldy=1 << 19),
    dict(rows=1 << 30, cols=72), dict(p=-0.1), dict(p=1.01), dict(p=math.nan), dict(ldx=63), dict(ldy=63), dict(ldx=1 << 40),
    dict(y=P, ldy=72), dict(step=P + 4),
    dict(rows=1 << 28, cols=64), dict(rows=1 << 16, cols=1 << 18, ldx=1 << 18, ldy=1 << 18),
])
def test_dropout_refusals(bad):
    a = dict(x=P, ldx=64, y=2 * P, ldy=64, f32=0, rows=9, cols=64, p=0.5, seed=1, step=None)
    a.update(bad)
    _refused("sat_op_dropout", *a.values(), None, word="dropout")


def test_dropout_of_nothing():
    L = _L()
    for rows, cols in ((0, 64), (9, 0)):
        assert L.lib().sat_op_dropout(None, 64, None, 64, 0, rows, cols, 0.5, 1, None, None) == L.SAT_OK


def test_philox_known_answers():
    """The published vectors of Philox4x32-10 (Random123's known answers)."""
    for ctr, key, want in [
            ([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
            ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
            ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0], [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])]:
        assert [int(x) for x in R.philox(ctr, key)] == want


# ---------------------------------------------------------------- residual norm

def _boundary(**kw):
    d = dict(x=P, ldx=64, f=2 * P, ldf=64, y=3 * P, ldy=64, h=4 * P, ldh=64, stats=5 * P, g_pre=6 * P, b_pre=None, g_post=6 * P, b_post=None,
             gate=7 * P, T=9, d=64, stream_f32=1, pre=1, post=2, alpha=1.0, beta=1.0, eps=1e-5, p=0.1, seed=1, step=None, dy=8 * P, lddy=64,
             dh=9 * P, lddh=64, dx=10 * P, lddx=64, df=11 * P, lddf=64, dg_pre=12 * P, dgate=13 * P, ws=14 * P, ws_elems=1 << 40)
    d.update(kw)
    return _L().sat_residual_norm_desc(**d)


SHARED = [dict(T=-1), dict(T=1 << 30), dict(d=0), dict(d=8193), dict(pre=3), dict(post=-1), dict(pre=0), dict(post=0), dict(alpha=math.inf),
          dict(beta=math.nan), dict(eps=-1e-5), dict(eps=math.nan), dict(p=-0.5), dict(p=1.5), dict(p=math.nan), dict(stats=None),
          dict(stats=P + 2), dict(gate=P + 1), dict(b_pre=P + 2), dict(step=P + 4)]


@pytest.mark.parametrize("bad", SHARED + [
    dict(x=None), dict(f=None), dict(y=None), dict(h=None), dict(x=P + 2), dict(f=P + 1), dict(h=P + 1), dict(ldx=63), dict(ldf=63),
    dict(ldy=63), dict(ldh=1 << 40), dict(y=P, ldy=72),
])
def test_residual_norm_refusals(bad):
    _refused("sat_op_residual_norm_fwd", C.byref(_boundary(**bad)), None, word="residual_norm_fwd")


@pytest.mark.parametrize("bad", SHARED + [
    dict(dh=None), dict(y=None), dict(f=None), dict(dx=None), dict(df=None), dict(dy=P + 2), dict(dx=P + 2), dict(df=P + 1), dict(lddx=63),
    dict(lddf=63), dict(lddh=63), dict(lddy=63), dict(dx=8 * P, lddx=72), dict(gate=None), dict(ws=None), dict(ws_elems=127),  # one workgroup's two sums of 64
    dict(dgate=P + 2), dict(db_post=P + 1), dict(post=0, g_post=None, db_post=P),
])
def test_residual_norm_backward_refusals(bad):
    _refused("sat_op_residual_norm_bwd", C.byref(_boundary(**bad)), None, word="residual_norm_bwd")


def test_residual_norm_null_and_ws():
    L = _L()
    n = C.c_int64()
    _refused("sat_op_residual_norm_fwd", None, None, word="null")
    _refused("sat_op_residual_norm_bwd", None, None, word="null")
    _refused("sat_op_residual_norm_bwd_ws", None, C.byref(n), word="null")
    _refused("sat_op_residual_norm_bwd_ws", C.byref(_boundary()), None, word="null")
    _refused("sat_op_residual_norm_bwd_ws", C.byref(_boundary(d=8193)), C.byref(n), word="sizes")
    # sizes and which sums are wanted are read; no sums, no workspace
    for kw, least in ((dict(T=9, d=64), 0), (dict(T=9, d=64, dgate=P), 64), (dict(T=1 << 20, d=8192, dgate=P, dg_pre=P), 2 * 8192 * 256)):
        assert L.lib().sat_op_residual_norm_bwd_ws(C.byref(L.sat_residual_norm_desc(**kw)), C.byref(n)) == 0
        assert n.value >= least and (least or n.value == 0)
    assert L.lib().sat_op_residual_norm_fwd(C.byref(_boundary(T=0, x=None, f=None, y=None, h=None, stats=None)), None) == L.SAT_OK


@pytest.mark.parametrize("pre,post", [("layer", "rms"), ("rms", "layer"), ("layer", None), (None, "layer"), (None, None)])
def test_residual_norm_gradients(pre, post):
    """The reference's gradients are those of its own forward, by central differences of a weighted sum."""
    rng = np.random.default_rng(3)
    T, d = 4, 11
    o = dict(pre=pre, post=post, g_pre=rng.normal(size=d) if pre else None, b_pre=rng.normal(size=d) if pre else None,
             g_post=rng.normal(size=d) if post else None, b_post=rng.normal(size=d) if post else None, gate=rng.normal(size=d),
             alpha=0.8, beta=1.3, eps=1e-3, p=0.25, seed=77, step=2)
    x, f, dy, dh = (rng.normal(size=(T, d)) for _ in range(4))

    def value(x, f, o):
        y = R.residual_fwd(x, f, o)[0]
        return (y * dy).sum() + ((R.residual_next(y, o)[0] * dh).sum() if pre else 0.0)

    y = R.residual_fwd(x, f, o)[0]
    st = np.zeros((4, T))
    if post:
        st[:2] = R.stats(f, post, o["eps"])
    if pre:
        st[2:] = R.stats(y, pre, o["eps"])
    got = R.residual_bwd(dy, dh, y, f, st, o, 0)
    e = 1e-5

    def near(name, change):
        """change(i, step): the value with element i moved; a difference is off by O(e^2) and rounding / e."""
        g = got[name][0]
        num = np.array([(change(i, e) - change(i, -e)) / (2 * e) for i in range(g.size)]).reshape(g.shape)
        assert np.abs(num - g).max() < 1e-7 * max(1.0, np.abs(g).max()), name

    def moved(a, i, s):
        b = a.copy()
        b.flat[i] += s
        return b

    near("dx", lambda i, s: value(moved(x, i, s), f, o))
    near("df", lambda i, s: value(x, moved(f, i, s), o))
    for name in ("gate", "g_pre", "b_pre", "g_post", "b_post"):
        if o[name] is not None:
            near("d" + name, lambda i, s: value(x, f, {**o, name: moved(o[name], i, s)}))


# ---------------------------------------------------------------- head with cross entropy

def _head(**kw):
    d = dict(x=P, ldx=64, w=2 * P, ldw=64, labels=3 * P, bias=4 * P, row_weight=None, row_loss=5 * P, lse=6 * P, inv_n=7 * P, dx=8 * P, lddx=64,
             dw=9 * P, lddw=64, db=10 * P, N=9, V=100, d=64, grad_f32=0, accumulate=0, ws=11 * P, ws_bytes=1 << 40)
    d.update(kw)
    return _L().sat_linear_xent_desc(**d)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(w=None), dict(labels=None), dict(row_loss=None), dict(lse=None), dict(inv_n=None), dict(ws=None), dict(ws_bytes=1000),
    dict(ws=11 * P + 16), dict(N=-1), dict(N=1 << 30), dict(V=0), dict(V=(1 << 20) + 1), dict(d=0), dict(d=60, ldx=64), dict(d=(1 << 16) + 8),
    dict(ldx=56), dict(ldw=56), dict(ldx=68), dict(ldw=1 << 21), dict(x=P + 8), dict(w=P + 2), dict(lddx=56), dict(lddx=68), dict(dx=P + 8),
    dict(lddw=56), dict(lddw=68), dict(dw=P + 8), dict(grad_f32=1, lddw=66), dict(accumulate=1), dict(bias=None), dict(bias=P + 2),
    dict(labels=P + 1), dict(row_weight=P + 2), dict(lse=P + 1), dict(db=P + 1), dict(db=P + 2, grad_f32=1), dict(inv_n=P + 3),
    dict(N=(1 << 25) + 1), dict(dx=P), dict(dw=2 * P),
])
def test_head_refusals(bad):
    _refused("sat_op_linear_xent", C.byref(_head(**bad)), None, word="linear_xent")


def test_head_null_and_ws():
    L = _L()
    n = C.c_int64()
    _refused("sat_op_linear_xent", None, None, word="null")
    _refused("sat_op_linear_xent_ws", None, C.byref(n), word="null")
    _refused("sat_op_linear_xent_ws", C.byref(_head()), None, word="null")

    def ws(**kw):
        assert L.lib().sat_op_linear_xent_ws(C.byref(L.sat_linear_xent_desc(**kw)), C.byref(n)) == 0
        return n.value

    # scoring keeps nothing of the size of the logits; the gradients what the header says
    score = ws(N=4096, V=50400, d=4096)
    assert score < 2 * 4096 * 4096 + (1 << 24)
    for N in (4096, 16384, 100000):
        x = 2 * N * 4096
        small = 400 * 8 * 16384 + 24 * N + (N // 512 + 2) * 4 * 50400 + (1 << 20)
        assert ws(N=N, V=50400, d=4096, dx=P, dw=P, bias=P, db=P) <= (1 << 30) + x + (1 << 27) + 4 * 50400 * 4096 + small
        assert ws(N=N, V=50400, d=4096, dx=P, dw=P, grad_f32=1) <= (1 << 30) + x + (1 << 27) + small
    assert ws(N=0, V=100, d=64, dw=P) > 0


def test_head_gradients():
    """The reference's gradients are those of its own loss, by central differences."""
    import torch
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x, w, b, c = r(6, 5), r(9, 5), r(9), r(6)
    labels = torch.tensor([0, 8, -1, 3, 9, 3])
    got = R.head(x, w, labels, b, c)
    value = lambda: (c * R.head(x, w, labels, b, c, False)["row_loss"][0]).sum().item()  # noqa: E731
    for t, k in ((x, "dx"), (w, "dw"), (b, "db")):
        for i in range(t.numel()):
            old, e = t.view(-1)[i].item(), 1e-5
            t.view(-1)[i] = old + e
            up = value()
            t.view(-1)[i] = old - e
            down = value()
            t.view(-1)[i] = old
            assert abs((up - down) / (2 * e) - got[k][0].reshape(-1)[i].item()) < 1e-8, (k, i)
    assert not got["dx"][0][2].any() and not got["dx"][0][4].any() and got["row_loss"][0][2] == 0
