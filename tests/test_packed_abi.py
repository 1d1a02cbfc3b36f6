"""Host-side checks of the operators on packed rows that need no GPU: refusals of the C entry
points before any launch, workspace sizes, the reference's gradients against differences."""

import ctypes as C
import math

import numpy as np
import pytest
import torch

from tests import packed_ref as R


def _L():
    from paper_2309_01226_amd import _lib
    return _lib


def _desc(**kw):
    d = dict(q=1 << 20, k=1 << 20, v=1 << 20, ldq=512, ldk=256, ldv=256, o=1 << 20, ldo=512, lse=1 << 20, cu=1 << 20,
             n_seq=3, T=100, H=8, Hkv=4, dh=64, causal=1, window=0, scale=0.125, dout=1 << 20, lddo=512, dq=1 << 20,
             dk=1 << 20, dv=1 << 20, lddq=512, lddk=256, lddv=256, ws=1 << 20, ws_elems=1 << 40)
    d.update(kw)
    return _L().sat_attn_packed_desc(**d)


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(lse=None), dict(cu=None),
    dict(q=(1 << 20) + 8), dict(v=(1 << 20) + 2), dict(o=(1 << 20) + 8), dict(lse=(1 << 20) + 2), dict(cu=(1 << 20) + 1),
    dict(ldq=504), dict(ldk=248), dict(ldv=260), dict(ldo=516), dict(ldq=1 << 22),
    dict(T=-1), dict(T=(1 << 29) + 1), dict(n_seq=-1), dict(H=6), dict(Hkv=0), dict(H=0), dict(Hkv=-4),
    dict(dh=0), dict(dh=60), dict(dh=264), dict(window=-1), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=math.nan), dict(scale=math.inf), dict(T=1 << 29, H=1 << 16, Hkv=1 << 16, dh=8, ldq=1 << 20),
])
def test_attention_refusals(bad):
    L = _L()
    d = _desc(**bad)
    for f in (L.lib().sat_op_attention_packed_fwd, L.lib().sat_op_attention_packed_bwd):
        assert f(C.byref(d), None) == L.SAT_EINVAL
        assert "attention_packed" in L.last_error()


@pytest.mark.parametrize("bad", [
    dict(dout=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(ws=None), dict(ws_elems=799), dict(lddo=504),
    dict(lddo=516), dict(dout=(1 << 20) + 8), dict(dq=(1 << 20) + 4), dict(lddq=508), dict(lddk=255), dict(lddv=252),
    dict(ws=(1 << 20) + 2), dict(lddo=1 << 22),
])
def test_attention_backward_refusals(bad):
    L = _L()
    d = _desc(**bad)
    assert L.lib().sat_op_attention_packed_bwd(C.byref(d), None) == L.SAT_EINVAL
    assert L.last_error()


def test_attention_null_descriptor_and_ws():
    L = _L()
    assert L.lib().sat_op_attention_packed_fwd(None, None) == L.SAT_EINVAL
    assert L.lib().sat_op_attention_packed_bwd(None, None) == L.SAT_EINVAL
    n = C.c_int64()
    assert L.lib().sat_op_attention_packed_bwd_ws(None, C.byref(n)) == L.SAT_EINVAL
    assert L.lib().sat_op_attention_packed_bwd_ws(C.byref(_desc()), None) == L.SAT_EINVAL
    # sizes alone are read
    d = L.sat_attn_packed_desc(n_seq=3, T=100, H=8, Hkv=4, dh=64)
    assert L.lib().sat_op_attention_packed_bwd_ws(C.byref(d), C.byref(n)) == 0 and n.value >= 800


def _rotary(**kw):
    a = dict(x=1 << 20, ldx=320, y=1 << 20, ldy=320, f32=0, pos=1 << 20, ldp=2, n_axes=2, pairs=(16, 16), T=9, H=4, dh=80,
             base=1e4, interleaved=1, own_freqs=0, inverse=0)
    a.update(kw)
    p = a["pairs"]
    a["pairs"] = None if p is None else (C.c_int32 * max(1, len(p)))(*p)
    return _L().lib().sat_op_rotary_axes(*a.values(), None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(y=None), dict(pos=None), dict(pairs=None), dict(n_axes=0), dict(n_axes=5, pairs=(1,) * 5, ldp=5),
    dict(pairs=(41, 0)), dict(pairs=(0, 0)), dict(pairs=(-1, 9)), dict(pairs=(20, 21)), dict(T=-1), dict(H=0), dict(dh=81, ldx=400, ldy=400),
    dict(ldx=319), dict(ldy=319, y=1 << 24), dict(ldp=1), dict(ldy=328), dict(x=(1 << 20) + 1), dict(f32=1, x=(1 << 20) + 2),
    dict(pos=(1 << 20) + 2), dict(base=0.0), dict(base=-1.0), dict(base=math.inf), dict(base=math.nan),
    dict(pairs=(129, 0), dh=512, ldx=2048, ldy=2048),
])
def test_rotary_refusals(bad):
    assert _rotary(**bad) == _L().SAT_EINVAL
    assert "rotary_axes" in _L().last_error()


def _adamw(bits=32, bf=0, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, t=1, count=None, **kw):
    L = _L()
    e = dict(p=1 << 20, g=1 << 20, m=1 << 20, v=1 << 20, m_exp=1 << 20, v_exp=1 << 20, shadow=None, n=10, weight_decay=0.0)
    e.update(kw)
    tab = (L.sat_adamw_tensor * 1)(L.sat_adamw_tensor(**e))
    return L.lib().sat_op_adamw_multi(tab, 1 if count is None else count, bits, bf, lr, b1, b2, eps, t, 0, None)


@pytest.mark.parametrize("bad", [
    dict(bits=16), dict(t=0), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=math.nan), dict(eps=-1.0), dict(lr=math.inf),
    dict(count=-1), dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(bits=8, m_exp=None), dict(bits=8, v_exp=None),
    dict(n=-1), dict(n=(1 << 42) + 1), dict(p=(1 << 20) + 2), dict(g=(1 << 20) + 2), dict(bf=1, g=(1 << 20) + 1),
    dict(m=(1 << 20) + 1), dict(v=(1 << 20) + 2), dict(shadow=(1 << 20) + 1),
])
def test_adamw_refusals(bad):
    assert _adamw(**bad) == _L().SAT_EINVAL
    assert "adamw_multi" in _L().last_error()


def test_adamw_empty_tables():
    L = _L()
    assert L.lib().sat_op_adamw_multi(None, 0, 32, 0, 1e-3, 0.9, 0.999, 1e-8, 1, 0, None) == 0
    assert L.lib().sat_op_adamw_multi(None, 1, 32, 0, 1e-3, 0.9, 0.999, 1e-8, 1, 0, None) == L.SAT_EINVAL
    assert _adamw(n=0, p=None, g=None) == 0  # an empty tensor needs nothing
    one = (C.c_void_p * 1)(None)
    tab = (L.sat_adamw_tensor * 1)(L.sat_adamw_tensor(m=1 << 20, v=1 << 20, m_exp=1 << 20, v_exp=1 << 20, n=4))
    assert L.lib().sat_op_adamw_multi_state(tab, 1, one, one, 0, None) == L.SAT_EINVAL
    assert L.lib().sat_op_adamw_multi_state(tab, 1, None, one, 0, None) == L.SAT_EINVAL
    odd = (C.c_void_p * 1)((1 << 20) + 1)
    assert L.lib().sat_op_adamw_multi_state(tab, 1, odd, odd, 1, None) == L.SAT_EINVAL
    assert L.lib().sat_op_adamw_multi_state(None, 0, None, None, 0, None) == 0


def test_python_entry_points_refuse_host_tensors():
    from paper_2309_01226_amd import ops
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        ops.rotary_axes(x, torch.zeros(4, 1, dtype=torch.int32), 1, 64, (32,))
    with pytest.raises(TypeError):
        ops.attention_packed_fwd(x, x, x, x, torch.zeros(1, 4), torch.zeros(2, dtype=torch.int32), 1, 1, 64, True, 0.125)
    p = [torch.zeros(8)]
    with pytest.raises(TypeError):
        ops.AdamWTensors(p, p, p, p)
    with pytest.raises(ValueError):
        ops.AdamWTensors(p, p, [torch.zeros(8, dtype=torch.uint8)], [torch.zeros(8, dtype=torch.uint8)])


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 3), (False, 2)])
def test_reference_gradients_against_differences(causal, window):
    """The formulas that the kernels are held to, against central differences of the forward."""
    g = torch.Generator().manual_seed(3)
    H, Hkv, dh, cu = 4, 2, 8, [1, 1, 6, 7, 12]
    q, k, v, do = (torch.randn(13, n * dh, generator=g, dtype=torch.float64) for n in (H, Hkv, Hkv, H))
    out, _ = R.attention(q, k, v, cu, H, Hkv, dh, causal, 0.3, window, do)
    step = 1e-5
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        d = torch.randn(x.shape, generator=g, dtype=torch.float64)
        f = []
        for s in (step, -step):
            a = dict(q=q, k=k, v=v)
            a[name[1]] = x + s * d
            f.append(float((R.attention(**a, cu=cu, H=H, Hkv=Hkv, dh=dh, causal=causal, scale=0.3, window=window)[0]["o"] * do).sum()))
        want = float((out[name] * d).sum())
        # the difference is off by step^2 times a third derivative, and by rounding / step: 1e-8 at most here
        assert abs((f[0] - f[1]) / (2 * step) - want) < 1e-7 * max(1.0, abs(want))


def test_reference_rotary_is_orthogonal_and_inverse():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(7, 40))
    pos = rng.integers(-50, 1 << 20, size=(7, 3))
    for inter in (True, False):
        for own in (True, False):
            y = R.rotary(x, pos, 2, 20, (3, 0, 5), interleaved=inter, own_freqs=own)
            assert np.allclose(np.linalg.norm(y, axis=1), np.linalg.norm(x, axis=1))
            back = R.rotary(y, pos, 2, 20, (3, 0, 5), interleaved=inter, own_freqs=own, inverse=True)
            assert np.allclose(back, x)
            assert np.array_equal(y[:, 16:20], x[:, 16:20])


@pytest.mark.parametrize("bad", [dict(H=64, Hkv=64, n_seq=1 << 18, ldq=4096), dict(T=1 << 26, H=32, Hkv=32, dh=8)])
def test_attention_refuses_more_threads_than_a_launch_has(bad):
    d = _desc(**{**bad, "ldk": 4096, "ldv": 4096, "ldo": 4096, "lddo": 4096, "lddq": 4096, "lddk": 4096, "lddv": 4096})
    L = _L()
    for f in (L.lib().sat_op_attention_packed_fwd, L.lib().sat_op_attention_packed_bwd):
        assert f(C.byref(d), None) == L.SAT_EINVAL
        assert "too many" in L.last_error()


@pytest.mark.parametrize("bad", [
    dict(T=1 << 24), dict(H=257, dh=4096, ldx=1 << 21, ldy=1 << 21), dict(H=1 << 16, dh=256, ldx=1 << 24, ldy=1 << 24),
])
def test_rotary_refuses_rows_that_its_division_does_not_hold(bad):
    assert _rotary(**bad) == _L().SAT_EINVAL
    assert "rotary_axes" in _L().last_error()


def test_rotary_division_is_exact_within_the_limits():
    """The kernel's x / d by a product with 2^32 / d + 1: items of one row, d of them to a head, H d^2 < 2^32."""
    for d in [2, 3, 7, 31, 40, 127, 255, 1000, 2999, 4095, 4096]:
        heads = min(1 << 16, ((1 << 32) - 1) // (d * d))
        inv = (1 << 32) // d + 1
        x = np.unique(np.concatenate([np.arange(0, heads * d, max(1, heads * d // 100003)), d * np.arange(1, heads) - 1,
                                      d * np.arange(heads), [heads * d - 1]])).astype(np.uint64)
        assert np.array_equal((x * np.uint64(inv)) >> np.uint64(32), x // np.uint64(d)), d


def test_adamw_refuses_more_than_a_launch_takes():
    assert _adamw(n=(1 << 35) + 1) == _L().SAT_EINVAL


def test_scratch_follows_the_chip_and_not_the_number_of_sequences():
    """Parts only fill the CUs: at most four rounds of the workgroups that these hold, each with fp32 dk and dv of its rows.
    256 CUs x 128 rows x workgroups on a CU x dims are at most 32768 x 256; rows of up to twice as many block
    numbers as there are blocks (T / R + n_seq against the larger of the two)."""
    L = _L()
    n = C.c_int64()
    for T in (64, 1000, 4096, 16384, 32768, 131072):
        for n_seq in (1, 4, 64, 1024, 4096, 16384):
            for H, Hkv in ((1, 1), (8, 8), (16, 4), (8, 1), (64, 1)):
                for dh in (8, 64, 80, 128, 136, 256):
                    for causal, window in ((1, 0), (0, 0), (1, 512)):
                        d = L.sat_attn_packed_desc(n_seq=n_seq, T=T, H=H, Hkv=Hkv, dh=dh, causal=causal, window=window)
                        for name, delta in (("fwd", 0), ("bwd", (H * T + 3) // 4 * 4)):
                            f = getattr(L.lib(), f"sat_op_attention_packed_{name}_ws")
                            assert f(C.byref(d), C.byref(n)) == 0
                            assert 0 <= n.value - delta <= 4 * 2 * 32768 * 256 * 2, (T, n_seq, H, Hkv, dh, causal, window, name)


def test_adamw_table_keeps_the_memory_that_it_points_to(monkeypatch):
    """Neither the caller's lists nor the tensors' own storage may be swapped under the pointers."""
    from paper_2309_01226_amd import ops
    monkeypatch.setattr(ops, "_device", lambda t, name: -1)  # of host tensors: nothing is launched here
    lists = {k: [torch.zeros(300) for _ in range(2)] for k in ("params", "grads", "m", "v")}
    sh = [torch.zeros(300, dtype=torch.bfloat16) for _ in range(2)]
    t = ops.AdamWTensors(**lists, shadows=sh)
    fields = dict(params="p", grads="g", m="m", v="v", shadows="shadow")
    for name, ts in dict(lists, shadows=sh).items():
        ts[0] = torch.ones(300)                   # another gradient, say
        ts[1].data = torch.ones_like(ts[1].data)  # a parameter that moved
        for i in range(2):
            assert t.tensors[name][i].data_ptr() == getattr(t.table[i], fields[name]), (name, i)


@pytest.mark.parametrize("m_out,v_out", [
    ((4096, 8192), (4096, 16384)), ((4096, 5292), (8192, 16384)), ((4096, 8192), (16384, 7000)),  # outputs over outputs
    ((1 << 20, 8192), (4096, 16384)), ((4096, 8192), (12288, (1 << 21) - 1196)),                   # over codes
    ((4096, (1 << 22) - 1196), (8192, 16384)), ((4096, 8192), (12288, (1 << 23))),                # over exponents
])
def test_state_refuses_outputs_that_overlap(m_out, v_out):
    """Two tensors of 300 values, fp32 outputs of 1200 bytes."""
    L = _L()
    tab = (L.sat_adamw_tensor * 2)(L.sat_adamw_tensor(m=1 << 20, v=1 << 21, m_exp=1 << 22, v_exp=(1 << 22) + 64, n=300),
                                   L.sat_adamw_tensor(m=(1 << 20) + 300, v=(1 << 21) + 300, m_exp=(1 << 23) - 1, v_exp=(1 << 23) + 1, n=300))
    mo, vo = ((C.c_void_p * 2)(*x) for x in (m_out, v_out))
    assert L.lib().sat_op_adamw_multi_state(tab, 2, mo, vo, 0, None) == L.SAT_EINVAL
    assert "overlap" in L.last_error()


@pytest.mark.parametrize("H,dh,pairs", [
    (1, 64, (16 - (1 << 32),)), (1, 64, ((1 << 32) + 16,)), (1, 64, (-1,)), (1, 64, (20, -4)),
    (1 - (1 << 32), 64, (16,)), (1, 64 - (1 << 32), (16,)), (0, 64, (16,)),
])
def test_rotary_sizes_that_32_bits_would_cut_are_refused(H, dh, pairs):
    from paper_2309_01226_amd import ops
    with pytest.raises(ValueError):
        ops.rotary_axes(torch.zeros(4, 64), torch.zeros(4, 2, dtype=torch.int32), H, dh, pairs)
