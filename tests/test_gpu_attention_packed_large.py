"""The kernels that large calls of packed attention run (four waves a workgroup, nothing split) against the 64-bit
form, K and V beyond the last-level cache, and row numbers that decrease."""

import ctypes as C
import math

import pytest
import torch

from tests import packed_ref as R
from tests.gpu_util import flush
from tests.test_gpu_attention_packed import SENTINEL, _case, _check, _make, _run

pytestmark = pytest.mark.gpu


def _scratch(s, causal, window):
    """fp32 elements of scratch beyond delta of the forward and the backward."""
    from paper_2309_01226_amd import _lib
    d = _lib.sat_attn_packed_desc(n_seq=len(s["rows"]) - 1, T=s["T"], H=s["H"], Hkv=s["Hkv"], dh=s["dh"], causal=causal,
                                  window=window)
    n = C.c_int64()
    _lib.call("sat_op_attention_packed_fwd_ws", d, n)
    fwd = n.value
    _lib.call("sat_op_attention_packed_bwd_ws", d, n)
    return fwd + n.value - (s["H"] * s["T"] + 3) // 4 * 4


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 100), (False, 200)])
@pytest.mark.parametrize("H,Hkv", [(16, 16), (32, 16), (16, 4)])
@pytest.mark.parametrize("dh", [24, 64, 72, 80, 96, 120, 128])
def test_whole_blocks_of_four_waves(dh, H, Hkv, causal, window):
    """(T / 128 + 1) Hkv >= 192 workgroups of sequences of 160 rows and more on average: four waves in every pass, and with
    16 K / V heads nothing split."""
    flush("packed attention, four waves", dh, H, Hkv, causal, window)
    lens = [160 + (i * 137) % 441 for i in range(16)] + [1, 0, 127, 128, 129, 640]
    s = _make(lens, H, Hkv, dh, seed=dh, before=1, after=2)
    assert (s["T"] // 128 + 1) * Hkv >= 192 and s["T"] // len(lens) >= 160
    assert Hkv < 16 or _scratch(s, causal, window) == 0
    scale = 1 / math.sqrt(dh)
    _run(s, causal, window, scale)
    torch.cuda.synchronize()
    _check(s, causal, window, scale)


@pytest.mark.parametrize("dh", [32, 96])
def test_few_blocks_are_split_in_kernels_of_their_width(dh):
    for lens, H, Hkv, causal, window in (([4000], 1, 1, True, 0), ([3000, 0, 70], 8, 1, True, 0), ([2100], 2, 2, False, 0),
                                         ([3500], 2, 1, True, 1500), ([1024, 1030], 8, 1, False, 600)):
        _case(lens, H, Hkv, dh, causal, window, before=1, after=3)


@pytest.mark.parametrize("dh,H", [(64, 32), (128, 16), (256, 8)])
def test_beyond_the_last_level_cache_as_two_calls(dh, H):
    """K and V of more than 2^28 bytes: blocks in another order, the same bits as calls on half of the sequences."""
    flush("packed attention beyond the cache", dh, H)
    lens = [1000 + 13 * i for i in range(34)]
    s = _make(lens, H, H, dh)
    assert 4 * s["T"] * H * dh > 1 << 28 and _scratch(s, True, 0) == 0
    _run(s, True, 0, 0.1)
    for first in (0, 17):
        rows = s["rows"][first:first + 18]
        at = slice(rows[0], rows[-1])
        part = dict(s, rows=[r - rows[0] for r in rows], T=rows[-1] - rows[0])
        part["cu"] = s["cu"][first:first + 18] - rows[0]
        assert 4 * part["T"] * H * dh <= 1 << 28 and _scratch(part, True, 0) == 0
        for n in ("q", "k", "v", "dout"):
            part[n] = s[n][at]
        for n in ("o", "dq", "dk", "dv"):
            part[n] = torch.full_like(s[n][at], SENTINEL, memory_format=torch.contiguous_format)
        part["lse"] = torch.full((H, part["T"]), SENTINEL, device="cuda")
        _run(part, True, 0, 0.1)
        torch.cuda.synchronize()
        for n in ("o", "dq", "dk", "dv"):
            assert torch.equal(part[n], s[n][at]), (n, first)
        assert torch.equal(part["lse"], s["lse"][:, at]), first
    # and a few heads of one sequence against the 64-bit form
    a, b = s["rows"][20], s["rows"][21]
    c = slice((H - 1) * dh, H * dh)
    want, err = R.attention(*(s[n][a:b, c] for n in ("q", "k", "v")), [0, b - a], 1, 1, dh, True, 0.1, 0, s["dout"][a:b, c])
    for n in ("o", "dq", "dk", "dv"):
        assert float(((s[n][a:b, c].double() - want[n]).abs() - err[n]).max()) <= 0, n


@pytest.mark.parametrize("empty", [0, 70])
def test_a_decreasing_pair_of_rows_is_an_empty_sequence(empty):
    """Up to 256 sequences, where no sequence of the rest shares rows with another."""
    s = _make([60, 68], 2, 1, 64)
    ref = _make([60, 68], 2, 1, 64)
    rows = [60, 0, 60, 60, 128] + [128] * empty
    s["cu"] = torch.tensor(rows, dtype=torch.int32, device="cuda")
    _run(s, True, 0, 0.1)
    _run(ref, True, 0, 0.1)
    torch.cuda.synchronize()
    for n in ("o", "lse", "dq", "dk", "dv"):
        assert torch.equal(s[n], ref[n]), n


@pytest.mark.parametrize("dh", [64, 256])
@pytest.mark.parametrize("n", [20, 200, 400])
def test_decreasing_rows_stay_within_their_range(n, dh):
    """What rows that several sequences claim hold is not defined; no other row is written."""
    s = _make([100], 2, 1, dh, before=10, after=10)
    g = torch.Generator().manual_seed(n)
    s["cu"] = torch.randint(10, 111, (n + 1,), generator=g, dtype=torch.int32).cuda()
    _run(s, True, 0, 0.1)
    torch.cuda.synchronize()
    for x in ("o", "dq", "dk", "dv"):
        assert (s[x][:10] == SENTINEL).all() and (s[x][110:] == SENTINEL).all(), x
    assert (s["lse"][:, :10] == SENTINEL).all() and (s["lse"][:, 110:] == SENTINEL).all()
