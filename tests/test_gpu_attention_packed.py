"""Attention inside packed sequences against its 64-bit form: lengths from 0 and 1 to long ones,
head widths, shared K / V heads, windows, strided rows, rows outside every sequence, captured calls.
The bounds come from packed_ref.attention, element by element."""

import math

import numpy as np
import pytest
import torch

from tests import packed_ref as R
from tests.gpu_util import flush

pytestmark = pytest.mark.gpu

SENTINEL = 123.0


def _cu(lens, first=0):
    return np.concatenate([[first], first + np.cumsum(lens)]).tolist() if lens else [first]


def _make(lens, H, Hkv, dh, *, seed=0, before=0, after=0, gap=0, fused=True):
    """q, k, v, dout whose rows outside the sequences are NaN, outputs filled with a sentinel; gap:
    columns behind the heads."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    cu = _cu(lens, before)
    T = cu[-1] + after
    widths = [H * dh, Hkv * dh, Hkv * dh]

    def three(fill):
        if fused:
            buf = fill(T, sum(widths) + gap)
            return list(buf.split(widths + [gap], 1))[:3]
        return [fill(T, w + gap)[:, :w] for w in widths]

    def rand(r, c):
        x = torch.randn(r, c, device="cuda", generator=g).to(torch.bfloat16)
        x[:before] = float("nan")
        x[cu[-1]:] = float("nan")
        return x

    def mark(r, c, dt=torch.bfloat16):
        return torch.full((r, c), SENTINEL, device="cuda", dtype=dt)

    q, k, v = three(rand)
    dq, dk, dv = three(mark)
    return dict(q=q, k=k, v=v, o=mark(T, H * dh), lse=mark(H, T, torch.float32), dout=rand(T, H * dh), dq=dq, dk=dk, dv=dv,
                cu=torch.tensor(cu, dtype=torch.int32, device="cuda"), rows=cu, H=H, Hkv=Hkv, dh=dh, T=T)


def _run(s, causal, window, scale, train=True):
    from paper_2309_01226_amd import ops
    a = [s["q"], s["k"], s["v"], s["o"], s["lse"], s["cu"]]
    ops.attention_packed_fwd(*a, s["H"], s["Hkv"], s["dh"], causal, scale, window=window)
    if train:
        ops.attention_packed_bwd(*a, s["dout"], s["dq"], s["dk"], s["dv"], s["H"], s["Hkv"], s["dh"], causal, scale,
                                 window=window)


def _check(s, causal, window, scale, names=("o", "lse", "dq", "dk", "dv")):
    clean = [torch.nan_to_num(s[n]) for n in ("q", "k", "v", "dout")]
    want, err = R.attention(*clean[:3], s["rows"], s["H"], s["Hkv"], s["dh"], causal, scale, window, clean[3])
    inside = torch.zeros(s["T"], dtype=torch.bool, device="cuda")
    inside[s["rows"][0]:s["rows"][-1]] = True
    for n in names:
        got = s[n].double()
        rows = inside if n != "lse" else inside[None, :].expand_as(got)
        assert (got[~rows] == SENTINEL).all(), f"{n}: a row outside the sequences was written"
        off = ((got - want[n]).abs() - err[n])[rows]
        assert torch.isfinite(got[rows]).all(), n
        assert off.numel() == 0 or float(off.max()) <= 0, (n, float(off.max()), float((got - want[n])[rows].abs().max()))


def _case(lens, H, Hkv, dh, causal, window=0, **kw):
    flush("packed attention", lens[:8], len(lens), H, Hkv, dh, causal, window, kw)
    s = _make(lens, H, Hkv, dh, seed=len(lens) + dh, **kw)
    scale = 1 / math.sqrt(dh)
    _run(s, causal, window, scale)
    torch.cuda.synchronize()
    _check(s, causal, window, scale)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dh", [8, 16, 40, 64, 72, 80, 96, 120, 128, 136, 200, 256])
def test_head_widths(dh, causal):
    _case([5, 0, 70, 1, 129], 2, 1, dh, causal, before=3, after=5)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dh", [64, 80, 128, 256])
def test_lengths(dh, causal):
    _case([1, 2, 31, 32, 33, 0, 63, 64, 65, 0, 0, 127, 128, 129, 255, 256, 257, 321], 2, 2, dh, causal, after=1)


@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 1), (6, 2), (8, 8), (8, 2), (16, 1), (9, 3), (20, 10)])
@pytest.mark.parametrize("dh", [64, 256])
def test_shared_heads(H, Hkv, dh):
    _case([97, 160, 3], H, Hkv, dh, True)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [1, 2, 31, 64, 65, 100, 300, 100000, 2 ** 31 - 1])
@pytest.mark.parametrize("dh", [64, 80, 128, 256])
def test_windows(dh, window, causal):
    _case([1, 40, 0, 300, 129], 4, 2, dh, causal, window, before=2, after=2)


@pytest.mark.parametrize("dh", [48, 64, 80, 128, 256])
def test_long_sequences(dh):
    _case([2500, 64, 1333], 2, 1, dh, True, after=9)
    _case([1900], 1, 1, dh, False)
    _case([2200, 10], 2, 2, dh, True, 500)


@pytest.mark.parametrize("dh", [24, 64, 80, 128])
def test_few_blocks_are_split(dh):
    """Too few blocks for the chip: their work is split and joined (and, without scratch, is not)."""
    import ctypes as C

    from paper_2309_01226_amd import _lib, ops
    for lens, H, Hkv, causal, window in (([4000], 1, 1, True, 0), ([3000, 0, 70], 8, 1, True, 0), ([2100], 2, 2, False, 0),
                                         ([3500], 2, 1, True, 1500), ([1024, 1030], 8, 1, False, 600)):
        _case(lens, H, Hkv, dh, causal, window, before=1, after=3)
    s = _make([3000], 2, 1, dh)
    d = _lib.sat_attn_packed_desc(n_seq=1, T=3000, H=2, Hkv=1, dh=dh, causal=1)
    n = C.c_int64()
    for name, least in (("fwd", 0), ("bwd", 2 * 3000)):
        _lib.call(f"sat_op_attention_packed_{name}_ws", d, n)
        assert n.value > least
    _run(s, True, 0, 0.1)
    torch.cuda.synchronize()
    split = {x: s[x].clone() for x in ("o", "lse", "dq", "dk", "dv")}
    p = {x: s[x].data_ptr() for x in ("q", "k", "v", "o", "lse", "cu", "dout", "dq", "dk", "dv")}
    ld = {"ld" + x: s[x].stride(0) for x in ("q", "k", "v", "o", "dq", "dk", "dv")}
    ws = torch.empty(6000, device="cuda")
    d = _lib.sat_attn_packed_desc(**p, **ld, lddo=s["dout"].stride(0), n_seq=1, T=3000, H=2, Hkv=1, dh=dh, causal=1, scale=0.1)
    _lib.call("sat_op_attention_packed_fwd", d, ops._stream())
    d.ws, d.ws_elems = ws.data_ptr(), 6000
    _lib.call("sat_op_attention_packed_bwd", d, ops._stream())
    torch.cuda.synchronize()
    _check(s, True, 0, 0.1)
    assert any(not torch.equal(s[x], split[x]) for x in split)  # another order of sums


@pytest.mark.parametrize("dh", [64, 256])
@pytest.mark.parametrize("n", [64, 65, 700, 4200])
def test_many_sequences(n, dh):
    """More sequences than one, two rounds of the search; a third of them empty."""
    lens = [(i * 7) % 6 // 2 * (1 + i % 3) for i in range(n)]
    lens[n // 2] = 150
    if n > 1000:
        lens = [min(x, 1) if i != n // 2 else x for i, x in enumerate(lens)]
    _case(lens, 2, 1, dh, True, before=1, after=1)


@pytest.mark.parametrize("dh", [64, 80, 128, 256])
def test_separate_wide_buffers(dh):
    _case([33, 100], 4, 2, dh, True, fused=False, gap=24)
    _case([33, 100], 4, 2, dh, False, gap=40)


def test_many_blocks():
    """Enough blocks that every XCD takes several units."""
    _case([1000, 30, 2000, 700, 3000, 129, 1], 8, 4, 64, True)


def test_nothing_to_do():
    from paper_2309_01226_amd import ops
    s = _make([0, 0], 2, 1, 64, after=4)
    _run(s, True, 0, 0.125)
    e = _make([], 2, 1, 64, after=4)
    _run(e, True, 0, 0.125)
    torch.cuda.synchronize()
    for x in (s, e):
        for n in ("o", "lse", "dq", "dk", "dv"):
            assert (x[n] == SENTINEL).all()
    t = [torch.empty(0, 64, device="cuda", dtype=torch.bfloat16) for _ in range(4)]
    ops.attention_packed_fwd(*t, torch.empty(1, 0, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), 1, 1, 64,
                             True, 0.125)
    ops.attention_packed_bwd(*t, torch.empty(1, 0, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), *t, 1, 1, 64,
                             True, 0.125)


@pytest.mark.parametrize("dh", [64, 128, 256])
def test_offsets_past_32_bits(dh):
    """Rows whose element offsets pass 2^32: a leading dimension of nearly 2^22."""
    flush("packed attention far rows", dh)
    ld, T, at = (1 << 22) - 8, 1290, 1040
    big = torch.empty(T * ld, device="cuda", dtype=torch.bfloat16)
    s = _make([T - at], 1, 1, dh, before=at)
    q = big.as_strided((T, dh), (ld, 1))
    dq = big.as_strided((T, dh), (ld, 1), 1024)
    q.copy_(s["q"])
    dq.fill_(SENTINEL)
    s.update(q=q, dq=dq)
    _run(s, True, 0, 0.1)
    torch.cuda.synchronize()
    _check(s, True, 0, 0.1)


def test_large_scores_and_equal_scores():
    """Scores far apart (all weight on one key) and all equal (weights 1 / keys, exact means)."""
    flush("packed attention extreme scores")
    s = _make([200], 2, 2, 64)
    s["q"].mul_(40)
    _run(s, True, 0, 1.0, train=False)
    torch.cuda.synchronize()
    want, err = R.attention(s["q"], s["k"], s["v"], s["rows"], 2, 2, 64, True, 1.0)
    # scores reach 40 * 64: their fp32 sums, and so p, are off by more than F; what the largest weight takes is not
    p_off = 272 * 2.0 ** -24 * 40 * 64 * 4
    assert float(((s["o"].double() - want["o"]).abs() - err["o"] - 2 * p_off * s["v"].abs().max()).max()) <= 0
    assert float(((s["lse"].double() - want["lse"]).abs() - err["lse"]).max()) <= 0
    s["k"].zero_()
    _run(s, False, 0, 1.0)
    torch.cuda.synchronize()
    _check(s, False, 0, 1.0)
    assert float((s["lse"] - math.log(200)).abs().max()) < 1e-5


def test_bad_rows_of_one_sequence_stay_in_it():
    for dh in (64, 80, 128, 256):
        s = _make([70, 50, 90], 2, 1, dh)
        ref = _make([70, 50, 90], 2, 1, dh)
        for n in ("q", "k", "v", "dout"):
            s[n][70:120] = float("nan")
            s[n][75:80] = float("inf")
        _run(s, True, 0, 0.1)
        _run(ref, True, 0, 0.1)
        torch.cuda.synchronize()
        for n in ("o", "dq", "dk", "dv"):
            assert torch.equal(s[n][:70], ref[n][:70]) and torch.equal(s[n][120:], ref[n][120:]), (dh, n)


def test_row_numbers_out_of_range_touch_nothing_else():
    """cu below 0 and past T is taken as 0 and T; a decreasing pair is an empty sequence."""
    s = _make([60, 68], 2, 1, 64)
    ref = _make([60, 68], 2, 1, 64)
    s["cu"] = torch.tensor([-500, 60, 1 << 30], dtype=torch.int32, device="cuda")
    _run(s, True, 0, 0.1)
    _run(ref, True, 0, 0.1)
    torch.cuda.synchronize()
    for n in ("o", "lse", "dq", "dk", "dv"):
        assert torch.equal(s[n], ref[n]), n


@pytest.mark.parametrize("dh,H,Hkv", [(64, 4, 4), (80, 2, 2), (128, 8, 2), (256, 4, 2)])
def test_same_bits_again_and_on_another_stream(dh, H, Hkv):
    s = _make([300, 5, 77], H, Hkv, dh)
    _run(s, True, 0, 0.1)
    torch.cuda.synchronize()
    first = {n: s[n].clone() for n in ("o", "lse", "dq", "dk", "dv")}
    for n in first:
        s[n].fill_(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _run(s, True, 0, 0.1)
    torch.cuda.current_stream().wait_stream(side)
    for n, x in first.items():
        assert torch.equal(s[n], x), n


@pytest.mark.parametrize("dh", [64, 256])
def test_captured_call_takes_the_lengths_of_the_replay(dh):
    flush("packed attention captured", dh)
    s = _make([100, 28], 4, 2, dh)
    _run(s, True, 0, 0.1)  # warm-up
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _run(s, True, 0, 0.1)
    for lens in ([100, 28], [1, 127], [64, 64], [128, 0]):
        e = _make(lens, 4, 2, dh)
        for n in ("q", "k", "v", "dout"):
            e[n].copy_(s[n])
        _run(e, True, 0, 0.1)
        s["cu"].copy_(e["cu"])
        for n in ("o", "lse", "dq", "dk", "dv"):
            s[n].fill_(SENTINEL)
        graph.replay()
        torch.cuda.synchronize()
        for n in ("o", "lse", "dq", "dk", "dv"):
            assert torch.equal(s[n], e[n]), (lens, n)


def test_gradients_against_differences():
    """The kernel's gradients along a direction, against differences of the 64-bit forward."""
    for dh, window in ((64, 0), (80, 20), (256, 0)):
        s = _make([40, 1, 65], 4, 2, dh, seed=7)
        _run(s, True, window, 0.1)
        g = torch.Generator(device="cuda").manual_seed(1)
        _, err = R.attention(s["q"], s["k"], s["v"], s["rows"], 4, 2, dh, True, 0.1, window, s["dout"])
        for n in ("q", "k", "v"):
            d = torch.randn(s[n].shape, device="cuda", generator=g, dtype=torch.float64)
            f = []
            for step in (1e-4, -1e-4):
                a = {x: s[x].double() for x in ("q", "k", "v")}
                a[n] = a[n] + step * d
                o = R.attention(a["q"], a["k"], a["v"], s["rows"], 4, 2, dh, True, 0.1, window)[0]["o"]
                f.append(float((o * s["dout"].double()).sum()))
            want = (f[0] - f[1]) / 2e-4
            # at most the elements' bounds along |d|, and the difference's own error
            room = float((err["d" + n] * d.abs()).sum()) + 1e-4 * abs(want) + 1e-3
            assert abs(float((s["d" + n].double() * d).sum()) - want) <= room, (dh, n)


def test_python_checks():
    from paper_2309_01226_amd import ops
    s = _make([10], 2, 1, 64)

    def fwd(**kw):
        a = dict(s, **kw)
        ops.attention_packed_fwd(a["q"], a["k"], a["v"], a["o"], a["lse"], a["cu"], 2, 1, 64, True, 0.1)
    fwd()
    bad = [dict(q=s["q"].float()), dict(k=s["k"][:9]), dict(v=s["v"][:, :32]), dict(o=s["o"].t()), dict(lse=s["lse"][:1]),
           dict(lse=s["lse"].t().contiguous().t()), dict(cu=s["cu"].long()), dict(cu=s["cu"][:0]), dict(cu=s["cu"].cpu())]
    for b in bad:
        with pytest.raises((TypeError, ValueError)):
            fwd(**b)


@pytest.mark.parametrize("window", [-1, 1 << 31, (1 << 32) + 5])
def test_windows_that_are_refused(window):
    from paper_2309_01226_amd import ops
    s = _make([10], 2, 1, 64)
    with pytest.raises(ValueError):
        ops.attention_packed_fwd(s["q"], s["k"], s["v"], s["o"], s["lse"], s["cu"], 2, 1, 64, True, 0.1, window=window)


@pytest.mark.parametrize("dh,H,Hkv", [(64, 4, 1), (128, 4, 1), (256, 2, 1)])
def test_two_streams_at_once(dh, H, Hkv):
    """Calls that overlap have scratch of their own; long sequences of few heads are the ones that use it."""
    sets = [_make([2500 + i, 33], H, Hkv, dh, seed=i) for i in range(2)]
    for s in sets:
        _run(s, True, 0, 0.1)
    torch.cuda.synchronize()
    names = ("o", "lse", "dq", "dk", "dv")
    alone = [{n: s[n].clone() for n in names} for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(4):
        for s in sets:
            for n in names:
                s[n].fill_(0)
        torch.cuda.synchronize()
        for s, side in zip(sets, streams):
            with torch.cuda.stream(side):
                for _ in range(2):
                    _run(s, True, 0, 0.1)
        torch.cuda.synchronize()
        for s, want in zip(sets, alone):
            for n in names:
                assert torch.equal(s[n], want[n]), n


def test_two_captured_graphs_at_once():
    sets = [_make([2500 + i, 33], 4, 1, 64, seed=i) for i in range(2)]
    for s in sets:
        _run(s, True, 0, 0.1)
    torch.cuda.synchronize()
    names = ("o", "lse", "dq", "dk", "dv")
    alone = [{n: s[n].clone() for n in names} for s in sets]
    graphs = [torch.cuda.CUDAGraph() for _ in sets]
    for s, g in zip(sets, graphs):
        with torch.cuda.graph(g):
            _run(s, True, 0, 0.1)
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        for s in sets:
            for n in names:
                s[n].fill_(0)
        torch.cuda.synchronize()
        for g, side in zip(graphs, streams):
            with torch.cuda.stream(side):
                g.replay()
        torch.cuda.synchronize()
        for s, want in zip(sets, alone):
            for n in names:
                assert torch.equal(s[n], want[n]), n


@pytest.mark.parametrize("dh", [136, 200, 256])
def test_few_blocks_of_wide_heads_are_split(dh):
    """Heads of more than 128 dims: few blocks split and joined, parts without a block, and no scratch."""
    import ctypes as C

    from paper_2309_01226_amd import _lib, ops
    for lens, H, Hkv, causal, window in (([4000], 1, 1, True, 0), ([3000, 0, 70], 4, 1, True, 0), ([2100], 2, 2, False, 0),
                                         ([3500], 2, 1, True, 1500), ([1024, 1030], 4, 1, False, 600), ([2000, 1, 130], 1, 1, True, 0)):
        _case(lens, H, Hkv, dh, causal, window, before=1, after=3)
    s = _make([3000], 2, 1, dh)
    d = _lib.sat_attn_packed_desc(n_seq=1, T=3000, H=2, Hkv=1, dh=dh, causal=1)
    n = C.c_int64()
    for name, least in (("fwd", 0), ("bwd", 2 * 3000)):
        _lib.call(f"sat_op_attention_packed_{name}_ws", d, n)
        assert n.value > least
    _run(s, True, 0, 0.1)
    torch.cuda.synchronize()
    split = {x: s[x].clone() for x in ("o", "lse", "dq", "dk", "dv")}
    p = {x: s[x].data_ptr() for x in ("q", "k", "v", "o", "lse", "cu", "dout", "dq", "dk", "dv")}
    ld = {"ld" + x: s[x].stride(0) for x in ("q", "k", "v", "o", "dq", "dk", "dv")}
    ws = torch.empty(6000, device="cuda")
    d = _lib.sat_attn_packed_desc(**p, **ld, lddo=s["dout"].stride(0), n_seq=1, T=3000, H=2, Hkv=1, dh=dh, causal=1, scale=0.1)
    _lib.call("sat_op_attention_packed_fwd", d, ops._stream())
    d.ws, d.ws_elems = ws.data_ptr(), 6000
    _lib.call("sat_op_attention_packed_bwd", d, ops._stream())
    torch.cuda.synchronize()
    _check(s, True, 0, 0.1)
    assert any(not torch.equal(s[x], split[x]) for x in split)  # another order of sums
