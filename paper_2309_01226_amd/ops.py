"""Kernel-level entry points on torch device tensors (marshalling only).

Each function checks shapes on the host, then calls one sat_op_* entry point
of libsaturn.so on the current torch stream.  torch provides device memory and
the stream; every element of every output is computed by the HIP kernels.
"""

import ctypes as C
import functools
import struct
from array import array

import torch

from . import _lib

LAY_K, LAY_MN = 0, 1
EPI_F32, EPI_RESID_F32, EPI_BF16, EPI_DGELU_BF16 = 0, 1, 2, 3


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(dev=None):
    """The current stream's handle on the current device `dev` (without the torch.cuda.Stream object, which takes
    3 us to make)."""
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if dev is None else dev)


def _need(t, dtype, name):
    if t is None:
        return
    if not t.is_cuda or t.dtype != dtype:
        raise TypeError(f"{name}: expected a CUDA tensor of {dtype}, got {t.device} {t.dtype}")


def _gemm_desc(A, B, M, N, K, out, lda, ldb, a_layout, b_layout, epilogue, ldo, bias, bias_col0,
               resid, ldr, out2, ldo2, gelu_col0, aux, ldaux, gelu_erf, splitk_ws):
    _need(A, torch.bfloat16, "A")
    _need(B, torch.bfloat16, "B")
    _need(bias, torch.float32, "bias")
    _need(resid, torch.float32, "resid")
    _need(aux, torch.bfloat16, "aux")
    _need(splitk_ws, torch.float32, "splitk_ws")
    need_a = (M - 1) * lda + K if a_layout == LAY_K else (K - 1) * lda + M
    need_b = (N - 1) * ldb + K if b_layout == LAY_K else (K - 1) * ldb + N
    if A.numel() < need_a or B.numel() < need_b:
        raise ValueError("gemm: operand smaller than its sizes imply")
    ldo = N if ldo is None else ldo
    if out.numel() < (M - 1) * ldo + N:
        raise ValueError("gemm: out too small")
    return _lib.sat_gemm_desc(
        A=A.data_ptr(), B=B.data_ptr(), M=M, N=N, K=K, lda=lda, ldb=ldb,
        a_layout=a_layout, b_layout=b_layout, epilogue=epilogue,
        out=out.data_ptr(), ldo=ldo,
        bias=None if bias is None else bias.data_ptr(), bias_col0=bias_col0,
        resid=None if resid is None else resid.data_ptr(), ldr=ldo if ldr is None else ldr,
        out2=None if out2 is None else out2.data_ptr(), ldo2=ldo2, gelu_col0=gelu_col0,
        aux=None if aux is None else aux.data_ptr(), ldaux=ldaux, gelu_erf=gelu_erf,
        splitk_ws=None if splitk_ws is None else splitk_ws.data_ptr(),
        splitk_ws_elems=0 if splitk_ws is None else splitk_ws.numel())


def gemm(A, B, M, N, K, out, *, lda, ldb, a_layout=LAY_K, b_layout=LAY_K, epilogue=EPI_F32,
         ldo=None, bias=None, bias_col0=0, resid=None, ldr=None, out2=None, ldo2=0, gelu_col0=0,
         aux=None, ldaux=0, gelu_erf=0, splitk_ws=None):
    """C[m, n] = sum_k A(m, k) B(n, k) with the chosen epilogue (see saturn_ops.h);
    splitk_ws: optional fp32 scratch that lets a small fp32-output product of either layout run
    split-K; calls that may overlap on different streams need one each."""
    d = _gemm_desc(A, B, M, N, K, out, lda, ldb, a_layout, b_layout, epilogue, ldo, bias, bias_col0,
                   resid, ldr, out2, ldo2, gelu_col0, aux, ldaux, gelu_erf, splitk_ws)
    _lib.call("sat_op_gemm_splitk", C.byref(d), _stream())
    return out


def gemm_noalloc(A, B, M, N, K, out, *, lda, ldb, a_layout=LAY_K, b_layout=LAY_K, epilogue=EPI_F32,
                 ldo=None, bias=None, bias_col0=0, resid=None, ldr=None, out2=None, ldo2=0,
                 gelu_col0=0, aux=None, ldaux=0, gelu_erf=0):
    """The same product through sat_op_gemm_noalloc: split-K partials go to the
    library's own per-device scratch, and the call allocates nothing."""
    d = _gemm_desc(A, B, M, N, K, out, lda, ldb, a_layout, b_layout, epilogue, ldo, bias, bias_col0,
                   resid, ldr, out2, ldo2, gelu_col0, aux, ldaux, gelu_erf, None)
    _lib.call("sat_op_gemm_noalloc", C.byref(d), _stream())
    return out


def _p(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def layernorm_fwd(x, g, b, y, mean, rstd, rows, d, eps, *, ldx=None, row_stride=1, ldy=None):
    _need(x, torch.float32, "x")
    _need(y, torch.bfloat16, "y")
    _lib.call("sat_op_layernorm_fwd", _p(x), ldx or d, row_stride, _p(g), _p(b), _p(y), ldy or d,
              _p(mean), _p(rstd), rows, d, C.c_float(eps), _stream())


def layernorm_bwd(dy, x, g, mean, rstd, dres, dg, db, rows, d, *, lddy=None, ldx=None, row_stride=1,
                  ldres=None):
    n_part = min(rows, 1024)
    work = torch.empty(2 * n_part * d, device=dy.device, dtype=torch.float32)
    _lib.call("sat_op_layernorm_bwd", _p(dy), lddy or d, _p(x), ldx or d, row_stride, _p(g),
              _p(mean), _p(rstd), _p(dres), ldres or d, _p(dg), _p(db), _p(work), rows, d, _stream())
    return work


def attention_fwd(q, k, v, o, lse, B, H, S, dh, causal, scale, *, ldq, ldk, ldv, ldo):
    for n, t in (("q", q), ("k", k), ("v", v), ("o", o)):
        _need(t, torch.bfloat16, n)
    _need(lse, torch.float32, "lse")
    if lse.numel() < B * H * S:
        raise ValueError("lse too small")
    _lib.call("sat_op_attention_fwd", _p(q), _p(k), _p(v), ldq, ldk, ldv, _p(o), ldo, _p(lse),
              B, H, S, dh, int(causal), C.c_float(scale), _stream())


def attention_bwd(q, k, v, o, lse, dout, dq, dk, dv, B, H, S, dh, causal, scale, *, ldq, ldk, ldv,
                  ldo, lddo, lddq, lddk, lddv):
    delta = torch.empty(B * H * S, device=q.device, dtype=torch.float32)
    _lib.call("sat_op_attention_bwd", _p(q), _p(k), _p(v), ldq, ldk, ldv, _p(o), ldo, _p(lse),
              _p(dout), lddo, _p(delta), _p(dq), _p(dk), _p(dv), lddq, lddk, lddv, B, H, S, dh,
              int(causal), C.c_float(scale), _stream())
    return delta


def rotary(qk, ld, B, S, H, dh, rd, inverse=False):
    _need(qk, torch.bfloat16, "qk")
    _lib.call("sat_op_rotary", _p(qk), ld, B, S, H, dh, rd, int(inverse), _stream())


def cross_entropy(z, labels, row_loss, dz, inv_n, N, V, *, ldz=None, lddz=None):
    _need(z, torch.float32, "z")
    _need(dz, torch.bfloat16, "dz")
    _need(labels, torch.int32, "labels")
    _lib.call("sat_op_cross_entropy", _p(z), ldz or V, _p(labels), N, V, _p(row_loss), _p(dz),
              lddz or V, _p(inv_n), _stream())


def adamw(p, g, m, v, shadow, n, lr, beta1, beta2, eps, wd, t):
    for name, t_ in (("p", p), ("g", g), ("m", m), ("v", v)):
        _need(t_, torch.float32, name)
    _need(shadow, torch.bfloat16, "shadow")
    _lib.call("sat_op_adamw", _p(p), _p(g), _p(m), _p(v), _p(shadow), n, float(lr), float(beta1),
              float(beta2), float(eps), float(wd), t, _stream())


def embed_fwd(tok, wte, wpe, h, T, S, d, V):
    _need(tok, torch.int32, "tok")
    _lib.call("sat_op_embed_fwd", _p(tok), _p(wte), _p(wpe), _p(h), T, S, d, V, _stream())


def embed_bwd(tok, dh, dwte, T, d, V):
    work = torch.empty(max(min(T, 16384), 1), device=dh.device, dtype=torch.int32)
    _lib.call("sat_op_embed_bwd", _p(tok), _p(dh), _p(dwte), T, d, V, _p(work), _stream())


def colsum(X, out, rows, cols, ldx=None):
    work = torch.empty(min(rows, 256) * max(cols, 1), device=X.device, dtype=torch.float32)
    _lib.call("sat_op_colsum", _p(X), ldx or cols, rows, cols, _p(out), _p(work), _stream())


def transpose_bf16(src, dst, rows, cols, *, lds=None, ldd=None):
    """dst[c, r] = src[r, c] (bf16, rows and cols multiples of 8)."""
    _need(src, torch.bfloat16, "src")
    _need(dst, torch.bfloat16, "dst")
    _lib.call("sat_op_transpose_bf16", _p(src), lds or cols, _p(dst), ldd or rows, rows, cols,
              _stream())


# ---------------------------------------------------------------- ResNet kernels

def _hw(H, k, stride, pad):
    return (H + 2 * pad - k) // stride + 1


def im2col(x, N, H, W, C, k, stride, pad):
    """x bf16 [N*H*W, C] -> col bf16 [N*Ho*Wo, k*k*C]."""
    _need(x, torch.bfloat16, "x")
    Ho, Wo = _hw(H, k, stride, pad), _hw(W, k, stride, pad)
    if x.numel() < N * H * W * C:
        raise ValueError("im2col: x too small")
    col = torch.empty(N * Ho * Wo, k * k * C, device=x.device, dtype=torch.bfloat16)
    _lib.call("sat_op_im2col", _p(x), _p(col), N, H, W, C, k, stride, pad, _stream())
    return col


def im2col_t(x, N, H, W, C, k, stride, pad):
    """x bf16 [N*H*W, C] -> colT bf16 [k*k*C, N*Ho*Wo] (im2col transposed)."""
    _need(x, torch.bfloat16, "x")
    Ho, Wo = _hw(H, k, stride, pad), _hw(W, k, stride, pad)
    if x.numel() < N * H * W * C:
        raise ValueError("im2col_t: x too small")
    P = N * Ho * Wo
    colT = torch.empty(k * k * C, P, device=x.device, dtype=torch.bfloat16)
    _lib.call("sat_op_im2col_t", _p(x), _p(colT), P, N, H, W, C, k, stride, pad, _stream())
    return colT


def col2im(dcol, N, H, W, C, k, stride, pad, dx=None):
    """dcol fp32 [N*Ho*Wo, k*k*C] -> dx fp32 [N*H*W, C] (accumulated into dx when given)."""
    _need(dcol, torch.float32, "dcol")
    Ho, Wo = _hw(H, k, stride, pad), _hw(W, k, stride, pad)
    if dcol.numel() < N * Ho * Wo * k * k * C:
        raise ValueError("col2im: dcol too small")
    acc = dx is not None
    if dx is None:
        dx = torch.empty(N * H * W, C, device=dcol.device, dtype=torch.float32)
    _lib.call("sat_op_col2im", _p(dcol), _p(dx), N, H, W, C, k, stride, pad, int(acc), _stream())
    return dx


def batchnorm_fwd(x, g, b, eps, relu=False):
    """Training-mode batch norm of x fp32 [P, C]: (y bf16, yf fp32, mean, rstd)."""
    _need(x, torch.float32, "x")
    P, Cc = x.shape
    part = torch.empty(2 * 1024 * Cc, device=x.device, dtype=torch.float32)
    mean = torch.empty(Cc, device=x.device, dtype=torch.float32)
    rstd = torch.empty_like(mean)
    y = torch.empty(P, Cc, device=x.device, dtype=torch.bfloat16)
    yf = torch.empty(P, Cc, device=x.device, dtype=torch.float32)
    _lib.call("sat_op_batchnorm_fwd", _p(x), P, Cc, _p(g), _p(b), C.c_float(eps), int(relu), _p(part),
              _p(mean), _p(rstd), _p(y), _p(yf), _stream())
    return y, yf, mean, rstd


def batchnorm_bwd(dy, x, mean, rstd, g, mask=None):
    """Backward of batchnorm_fwd (through a ReLU whose output is `mask`, bf16 or
    fp32, when given): (dx bf16, dg, db)."""
    _need(dy, torch.float32, "dy")
    P, Cc = dy.shape
    kind = 0 if mask is None else (1 if mask.dtype == torch.bfloat16 else 2)
    part = torch.empty(2 * 1024 * Cc, device=dy.device, dtype=torch.float32)
    dg = torch.empty(Cc, device=dy.device, dtype=torch.float32)
    db = torch.empty_like(dg)
    dx = torch.empty(P, Cc, device=dy.device, dtype=torch.bfloat16)
    _lib.call("sat_op_batchnorm_bwd", _p(dy), kind, _p(mask), _p(x), _p(mean), _p(rstd), _p(g), P, Cc,
              _p(part), _p(dg), _p(db), _p(dx), _stream())
    return dx, dg, db


def maxpool_fwd(x, N, H, W, C):
    """3 x 3 / 2 max pool (padding 1) of x fp32 [N*H*W, C]: (y fp32, y bf16, arg uint8)."""
    _need(x, torch.float32, "x")
    Ho, Wo = _hw(H, 3, 2, 1), _hw(W, 3, 2, 1)
    y = torch.empty(N * Ho * Wo, C, device=x.device, dtype=torch.float32)
    yb = torch.empty(N * Ho * Wo, C, device=x.device, dtype=torch.bfloat16)
    arg = torch.empty(N * Ho * Wo, C, device=x.device, dtype=torch.uint8)
    _lib.call("sat_op_maxpool_fwd", _p(x), N, H, W, C, _p(y), _p(yb), _p(arg), _stream())
    return y, yb, arg


def maxpool_bwd(dy, arg, N, H, W, C):
    _need(dy, torch.float32, "dy")
    dx = torch.empty(N * H * W, C, device=dy.device, dtype=torch.float32)
    _lib.call("sat_op_maxpool_bwd", _p(dy), _p(arg), N, H, W, C, _p(dx), _stream())
    return dx


# ---------------------------------------------------------------- packed rows

def _here(t, dtype, name, dev):
    """t: a tensor of `dtype` on the current device `dev` (the calls run on its current stream)."""
    if t.dtype is not dtype or t.get_device() != dev:
        _need(t, dtype, name)
        raise ValueError(f"{name}: on {t.device}, but the current device is cuda:{dev}")


def _device(t, name):
    """The current device, for a call on `t`, which has to be on some GPU."""
    if not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA tensor, got {t.device}")
    return torch.cuda.current_device()


def _rows_of(t, dtype, name, rows, cols, dev):
    """Leading dimension of a matrix of at least `rows` rows and `cols` columns, columns contiguous."""
    if t.dtype is not dtype or t.get_device() != dev:
        _here(t, dtype, name, dev)
    shape = t.shape
    if len(shape) == 2:
        r, c = shape
        ld, one = t.stride()
        if r >= rows and c >= cols and (one == 1 or c < 2):
            return ld if r > 1 else max(ld, c)
    raise ValueError(f"{name}: expected [{rows}, >= {cols}] with contiguous rows, got {tuple(shape)} strides {t.stride()}")


# sat_attn_packed_desc's fields (packing them takes a third of the time that ctypes takes to set them)
_PACKED = struct.Struct("3P3qPqPP7if" + "Pq3P3q" + "Pq")
assert _PACKED.size == C.sizeof(_lib.sat_attn_packed_desc)


def _packed_desc(q, k, v, o, lse, cu, H, Hkv, dh, causal, scale, window, dev, more=(0,) * 10):
    T = q.shape[0]
    bf, wq, wk = torch.bfloat16, H * dh, Hkv * dh
    _here(lse, torch.float32, "lse", dev)
    _here(cu, torch.int32, "cu", dev)
    n = cu.numel()
    if cu.dim() != 1 or n < 1 or not cu.is_contiguous():
        raise ValueError("cu: expected a contiguous vector of n_seq + 1 row numbers")
    if not 0 <= window < 1 << 31:  # ctypes would cut it
        raise ValueError(f"window: {window}")
    if lse.shape != (H, T) or not lse.is_contiguous():
        raise ValueError(f"lse: expected a contiguous [{H}, {T}], got {tuple(lse.shape)}")
    return _lib.sat_attn_packed_desc.from_buffer_copy(_PACKED.pack(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), _rows_of(q, bf, "q", T, wq, dev), _rows_of(k, bf, "k", T, wk, dev),
        _rows_of(v, bf, "v", T, wk, dev), o.data_ptr(), _rows_of(o, bf, "o", T, wq, dev), lse.data_ptr(), cu.data_ptr(),
        n - 1, T, H, Hkv, dh, bool(causal), window, scale, *more))


@functools.lru_cache(maxsize=256)
def _packed_ws(call, n_seq, T, H, Hkv, dh, causal, window):
    """fp32 elements of scratch of the forward ("fwd") or the backward ("bwd") for these sizes."""
    d = _lib.sat_attn_packed_desc(n_seq=n_seq, T=T, H=H, Hkv=Hkv, dh=dh, causal=causal, window=window)
    need = C.c_int64()
    _lib.call(f"sat_op_attention_packed_{call}_ws", d, need)
    return need.value


def attention_packed_fwd(q, k, v, o, lse, cu, H, Hkv, dh, causal, scale, *, window=0):
    """Attention inside packed sequences: rows cu[s] .. cu[s + 1] - 1 of q, o [T, >= H dh] and k, v
    [T, >= Hkv dh] (bf16, views of a wider buffer allowed) are sequence s; lse fp32 [H, T].  See
    saturn_ops.h for the masks.  Workspaces come from torch's allocator, on the current stream."""
    dev = _device(q, "q")
    d = _packed_desc(q, k, v, o, lse, cu, H, Hkv, dh, causal, scale, window, dev)
    need = _packed_ws("fwd", cu.numel() - 1, q.shape[0], H, Hkv, dh, bool(causal), window)
    if need:
        ws = torch.empty(need, device=q.device, dtype=torch.float32)
        d.ws, d.ws_elems = ws.data_ptr(), need
    _lib.call("sat_op_attention_packed_fwd", d, _stream(dev))


def attention_packed_bwd(q, k, v, o, lse, cu, dout, dq, dk, dv, H, Hkv, dh, causal, scale, *, window=0):
    """Its backward from dout [T, >= H dh] and the forward's o and lse; writes dq, dk, dv."""
    dev, T, bf, wq, wk = _device(q, "q"), q.shape[0], torch.bfloat16, H * dh, Hkv * dh
    need = _packed_ws("bwd", cu.numel() - 1, T, H, Hkv, dh, bool(causal), window)
    ws = torch.empty(max(1, need), device=q.device, dtype=torch.float32)
    d = _packed_desc(q, k, v, o, lse, cu, H, Hkv, dh, causal, scale, window, dev, (
        dout.data_ptr(), _rows_of(dout, bf, "dout", T, wq, dev), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
        _rows_of(dq, bf, "dq", T, wq, dev), _rows_of(dk, bf, "dk", T, wk, dev), _rows_of(dv, bf, "dv", T, wk, dev),
        ws.data_ptr(), need))
    _lib.call("sat_op_attention_packed_bwd", d, _stream(dev))


_PAIRS = frozenset(range(129))  # that one axis may turn


def rotary_axes(x, pos, H, dh, pairs, *, out=None, base=10000.0, interleaved=True, own_freqs=False, inverse=False):
    """Rotary positions with len(pairs) axes on the H heads of x [T, >= H dh] (bf16 or fp32), axis a
    turning pairs[a] pairs of every head by pos[:, a] (int32 [T, axes]); in place, or into `out`.
    See saturn_ops.h.  Returns the rotated tensor."""
    if H < 1 or dh < 1 or not _PAIRS.issuperset(pairs):  # ctypes would cut what 32 bits do not hold
        raise ValueError(f"H={H}, dh={dh}, pairs: {pairs}")
    f32 = x.dtype == torch.float32
    dt = torch.float32 if f32 else torch.bfloat16
    T, A, dev = x.shape[0], len(pairs), _device(x, "x")
    y = x if out is None else out
    ldx = _rows_of(x, dt, "x", T, H * dh, dev)
    ldy = ldx if out is None else _rows_of(out, dt, "out", T, H * dh, dev)
    ldp = _rows_of(pos, torch.int32, "pos", T, A, dev)
    _lib.call("sat_op_rotary_axes", x.data_ptr(), ldx, y.data_ptr(), ldy, f32, pos.data_ptr(), ldp, A,
              (C.c_int32 * A)(*pairs), T, H, dh, base, interleaved, own_freqs, inverse, _stream(dev))
    return y


class AdamWTensors:
    """The tensors of adamw_multi: parameters (fp32), gradients (all fp32 or all bf16), moments
    (all fp32, or all uint8 with m_exp and v_exp, one uint8 for each 256 elements of a tensor), bf16
    shadows (optional) and weight decay (a number, or one per tensor).  Holds the tensors' memory as it is now:
    a step reads and writes there even if a caller's list or tensor gets another storage later, so gradients
    are to be written into the same tensors in every step (or the table is built again)."""

    def __init__(self, params, grads, m, v, *, shadows=None, weight_decay=0.0, m_exp=None, v_exp=None):
        n = len(params)
        if any(len(x) != n for x in (grads, m, v)):
            raise ValueError("one of everything for each parameter")
        self.bits = 8 if n and m[0].dtype == torch.uint8 else 32
        self.grad_bf16 = bool(n) and grads[0].dtype == torch.bfloat16
        st = torch.uint8 if self.bits == 8 else torch.float32
        decay = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(w) for w in weight_decay]
        lists = dict(params=params, grads=grads, m=m, v=v)
        if shadows is not None:
            lists["shadows"] = shadows
        if self.bits == 8:
            if m_exp is None or v_exp is None:
                raise ValueError("8-bit moments need m_exp and v_exp")
            lists.update(m_exp=m_exp, v_exp=v_exp)
        elif m_exp is not None or v_exp is not None:
            raise ValueError("m_exp and v_exp belong to 8-bit moments")
        if any(len(x) != n for x in lists.values()) or len(decay) != n:
            raise ValueError("one of everything for each parameter")
        dtypes = dict(params=torch.float32, grads=torch.bfloat16 if self.grad_bf16 else torch.float32, m=st, v=st,
                      shadows=torch.bfloat16, m_exp=torch.uint8, v_exp=torch.uint8)
        dev = _device(params[0], "params[0]") if n else None
        sizes = [t.numel() for t in params]
        eighth = [-(-k // 256) for k in sizes]
        spans, ptrs = [], {}
        for name, ts in lists.items():
            dtype, written, want = dtypes[name], name != "grads", eighth if name.endswith("_exp") else sizes
            ptrs[name] = [t.data_ptr() for t in ts]
            for i, t in enumerate(ts):
                if t.dtype is not dtype or t.get_device() != dev:
                    _here(t, dtype, f"{name}[{i}]", dev)
                if not t.is_contiguous() or t.numel() != want[i]:
                    raise ValueError(f"{name}[{i}]: expected {want[i]} contiguous elements, got {tuple(t.shape)}")
            size = dtype.itemsize
            spans += [(p, p + k * size, written, name, i) for i, (p, k) in enumerate(zip(ptrs[name], want)) if k]
        end, last = 0, None
        for span in sorted(spans):
            if span[0] < end and (span[2] or last[2]):
                raise ValueError("{}[{}] overlaps {}[{}]".format(*span[3:], *last[3:]))
            if span[1] > end:
                end, last = span[1], span
        # aliases: the memory stays while the table does, whatever becomes of the caller's lists and tensors
        self.tensors = {name: list(map(torch.Tensor.detach, ts)) for name, ts in lists.items()}
        self.sizes, self.device = sizes, dev
        self.table = (_lib.sat_adamw_tensor * n)()
        none = [None] * n
        columns = [ptrs.get(x, none) for x in ("params", "grads", "m", "v", "m_exp", "v_exp", "shadows")]
        for i, row in enumerate(zip(*columns, sizes, decay)):
            self.table[i] = row


def adamw_multi(tensors, lr, beta1, beta2, eps, t, *, seed=0):
    """One AdamW step t (>= 1) on all of `tensors` (AdamWTensors); seed: of the rounding of 8-bit moments."""
    _on_device(tensors)
    _lib.call("sat_op_adamw_multi", tensors.table, len(tensors.table), tensors.bits, tensors.grad_bf16, lr, beta1, beta2,
              eps, t, seed & 0xFFFFFFFFFFFFFFFF, _stream())


def adamw_multi_state(tensors, m_out, v_out):
    """The values of 8-bit moments, to one contiguous tensor per parameter in each list (all fp32 or all bf16)."""
    _on_device(tensors)
    if tensors.bits != 8:
        raise ValueError("adamw_multi_state: the moments are fp32 already")
    n = len(tensors.table)
    if len(m_out) != n or len(v_out) != n:
        raise ValueError("adamw_multi_state: one output of each kind for each parameter")
    dt = torch.bfloat16 if n and m_out[0].dtype == torch.bfloat16 else torch.float32
    T, dev = torch.Tensor, tensors.device
    for name, ts in (("m_out", m_out), ("v_out", v_out)):
        # all at once first: a look at every tensor takes longer than the launches
        if (list(map(T.numel, ts)) == tensors.sizes and all(map(T.is_contiguous, ts)) and set(map(T.get_device, ts)) <= {dev}
                and {t.dtype for t in ts} <= {dt}):
            continue
        for i, (t, k) in enumerate(zip(ts, tensors.sizes)):
            _here(t, dt, f"{name}[{i}]", dev)
            if not t.is_contiguous() or t.numel() != k:
                raise ValueError(f"{name}[{i}]: expected {k} contiguous elements, got {tuple(t.shape)}")
    ms, vs = ((C.c_void_p * n).from_buffer(array("Q", map(T.data_ptr, ts))) for ts in (m_out, v_out))
    _lib.call("sat_op_adamw_multi_state", tensors.table, n, ms, vs, dt == torch.bfloat16, _stream())


def _on_device(tensors):
    if tensors.device not in (None, torch.cuda.current_device()):
        raise ValueError(f"params: on cuda:{tensors.device}, but the current device is cuda:{torch.cuda.current_device()}")
