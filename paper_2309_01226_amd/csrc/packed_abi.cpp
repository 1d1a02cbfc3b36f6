// Kernel-level C ABI (include/saturn_ops.h) of the operators on packed rows: attention inside
// packed sequences, rotary positions with several axes, AdamW over many tensors.  Argument
// checks, then the launches; nothing is allocated on the device.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <memory>
#include <new>
#include <utility>

#include "../../include/saturn_ops.h"
#include "abi_common.h"
#include "kernels.h"

static inline hipStream_t S(void* s) { return reinterpret_cast<hipStream_t>(s); }
static bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

static constexpr int64_t kMaxGroups = 1 << 24;  // of 256 threads: a launch has fewer than 2^32

// ---------------------------------------------------------------- attention

static constexpr int64_t kMaxLd = 1 << 22;  // a block's rows stay within 32-bit buffer offsets

static sat_status packed_sizes(const sat_attn_packed_desc* d, const char* fn) {
  SAT_CHECK_ARG(d != nullptr, "%s: null descriptor", fn);
  SAT_CHECK_ARG(d->T >= 0 && d->T <= (1 << 29) && d->n_seq >= 0 && d->n_seq <= (1 << 28),
                "%s: bad sizes T=%d n_seq=%d", fn, d->T, d->n_seq);
  SAT_CHECK_ARG(d->Hkv > 0 && d->H > 0 && d->H <= (1 << 16) && d->H % d->Hkv == 0,
                "%s: H=%d must be a positive multiple of Hkv=%d", fn, d->H, d->Hkv);
  SAT_CHECK_ARG(d->dh >= 8 && d->dh <= 256 && d->dh % 8 == 0,
                "%s: head dim %d must be a multiple of 8 up to 256", fn, d->dh);
  // workgroups, a whole number of them for each of up to 8 parts: blocks of 64 rows have 128 threads, of
  // 128 rows up to 512, and a launch fewer than 2^32 threads
  SAT_CHECK_ARG(((int64_t)d->T / 64 + 2 * ((int64_t)d->n_seq + 8)) * d->H < (1LL << 24), "%s: too many rows x heads", fn);
  return SAT_OK;
}

static sat_status packed_args(const sat_attn_packed_desc* d, AttnPackedArgs* out, const char* fn) {
  sat_status st = packed_sizes(d, fn);
  if (st != SAT_OK) return st;
  SAT_CHECK_ARG(d->T == 0 || (d->q && d->k && d->v && d->o && d->lse && d->cu), "%s: null pointer", fn);
  const int64_t wq = (int64_t)d->H * d->dh, wk = (int64_t)d->Hkv * d->dh;
  SAT_CHECK_ARG(d->ldq >= wq && d->ldo >= wq && d->ldk >= wk && d->ldv >= wk && d->ldq < kMaxLd &&
                    d->ldk < kMaxLd && d->ldv < kMaxLd && d->ldo < kMaxLd,
                "%s: leading dimensions must cover the heads and be below 2^22", fn);
  SAT_CHECK_ARG(d->ldq % 8 == 0 && d->ldk % 8 == 0 && d->ldv % 8 == 0 && d->ldo % 8 == 0 && aligned(d->q, 16) &&
                    aligned(d->k, 16) && aligned(d->v, 16) && aligned(d->o, 16),
                "%s: q, k, v, o must be 16-byte aligned with leading dimensions %% 8 == 0", fn);
  SAT_CHECK_ARG(aligned(d->lse, 4) && aligned(d->cu, 4), "%s: lse and cu must be aligned to their elements", fn);
  SAT_CHECK_ARG(d->window >= 0, "%s: negative window", fn);
  SAT_CHECK_ARG(d->scale > 0.f && isfinite(d->scale), "%s: scale must be positive and finite", fn);
  AttnPackedArgs& a = *out;
  a.q = (const bf16*)d->q; a.k = (const bf16*)d->k; a.v = (const bf16*)d->v;
  a.ldq = d->ldq; a.ldk = d->ldk; a.ldv = d->ldv;
  a.o = (bf16*)d->o; a.ldo = d->ldo; a.lse = d->lse; a.cu = d->cu;
  a.n_seq = d->n_seq; a.T = d->T; a.H = d->H; a.Hkv = d->Hkv; a.dh = d->dh;
  a.causal = d->causal != 0;
  a.window = d->window == 0 || d->window > (1 << 30) ? 1 << 30 : d->window;
  a.scale = d->scale;
  a.ws = nullptr;
  a.ws_elems = 0;
  a.ntile = a.parts = a.split = a.by_place = 0;
  return SAT_OK;
}

extern "C" sat_status sat_op_attention_packed_fwd(const sat_attn_packed_desc* d, void* stream) {
  AttnPackedArgs a;
  sat_status st = packed_args(d, &a, "attention_packed_fwd");
  if (st != SAT_OK) return st;
  SAT_CHECK_ARG(d->ws_elems >= 0 && aligned(d->ws, 16), "attention_packed_fwd: ws must be 16-byte aligned");
  a.ws = d->ws;
  a.ws_elems = d->ws ? d->ws_elems : 0;
  SAT_HIP(launch_attn_packed_fwd(a, S(stream)));
  return SAT_OK;
}

// The part of the arguments that the workspaces depend on.
static AttnPackedArgs shape_of(const sat_attn_packed_desc* d) {
  AttnPackedArgs a;
  memset(&a, 0, sizeof a);
  a.n_seq = d->n_seq; a.T = d->T; a.H = d->H; a.Hkv = d->Hkv; a.dh = d->dh;
  a.causal = d->causal != 0;
  a.window = d->window <= 0 || d->window > (1 << 30) ? 1 << 30 : d->window;
  return a;
}

extern "C" sat_status sat_op_attention_packed_fwd_ws(const sat_attn_packed_desc* d, int64_t* elems) {
  SAT_CHECK_ARG(elems != nullptr, "attention_packed_fwd_ws: null pointer");
  sat_status st = packed_sizes(d, "attention_packed_fwd_ws");
  if (st != SAT_OK) return st;
  *elems = attn_packed_ws(shape_of(d), false);
  return SAT_OK;
}

// delta, rounded up so that what follows is aligned.
static int64_t delta_elems(const sat_attn_packed_desc* d) { return ((int64_t)d->H * d->T + 3) / 4 * 4; }

extern "C" sat_status sat_op_attention_packed_bwd_ws(const sat_attn_packed_desc* d, int64_t* elems) {
  SAT_CHECK_ARG(elems != nullptr, "attention_packed_bwd_ws: null pointer");
  sat_status st = packed_sizes(d, "attention_packed_bwd_ws");
  if (st != SAT_OK) return st;
  *elems = delta_elems(d) + attn_packed_ws(shape_of(d), true);
  return SAT_OK;
}

extern "C" sat_status sat_op_attention_packed_bwd(const sat_attn_packed_desc* d, void* stream) {
  const char* fn = "attention_packed_bwd";
  AttnPackedBwdArgs a;
  sat_status st = packed_args(d, &a.f, fn);
  if (st != SAT_OK) return st;
  SAT_CHECK_ARG(d->T == 0 || (d->dout && d->dq && d->dk && d->dv && d->ws), "%s: null pointer", fn);
  const int64_t wq = (int64_t)d->H * d->dh, wk = (int64_t)d->Hkv * d->dh;
  SAT_CHECK_ARG(d->lddo >= wq && d->lddq >= wq && d->lddk >= wk && d->lddv >= wk && d->lddo < kMaxLd,
                "%s: leading dimensions must cover the heads, dout's be below 2^22", fn);
  SAT_CHECK_ARG(d->lddo % 8 == 0 && aligned(d->dout, 16), "%s: dout must be 16-byte aligned with lddo %% 8 == 0", fn);
  SAT_CHECK_ARG(d->lddq % 4 == 0 && d->lddk % 4 == 0 && d->lddv % 4 == 0 && aligned(d->dq, 8) && aligned(d->dk, 8) &&
                    aligned(d->dv, 8),
                "%s: dq, dk, dv must be 8-byte aligned with leading dimensions %% 4 == 0", fn);
  const int64_t need = delta_elems(d);
  SAT_CHECK_ARG(d->ws_elems >= need && aligned(d->ws, 16),
                "%s: ws of %ld elements, at least %ld needed, 16-byte aligned", fn, (long)d->ws_elems, (long)need);
  a.dout = (const bf16*)d->dout; a.lddo = d->lddo;
  a.delta = d->ws;
  a.f.ws = d->ws + need;
  a.f.ws_elems = d->ws_elems - need;
  a.dq = (bf16*)d->dq; a.dk = (bf16*)d->dk; a.dv = (bf16*)d->dv;
  a.lddq = d->lddq; a.lddk = d->lddk; a.lddv = d->lddv;
  SAT_HIP(launch_attn_packed_bwd(a, S(stream)));
  return SAT_OK;
}

// ---------------------------------------------------------------- rotary

extern "C" sat_status sat_op_rotary_axes(const void* x, int64_t ldx, void* y, int64_t ldy, int32_t f32,
                                         const int32_t* pos, int64_t ldp, int32_t n_axes, const int32_t* pairs,
                                         int32_t T, int32_t H, int32_t dh, double base, int32_t interleaved,
                                         int32_t own_freqs, int32_t inverse, void* stream) {
  const char* fn = "rotary_axes";
  SAT_CHECK_ARG(pairs && (T == 0 || (x && y && pos)), "%s: null pointer", fn);
  SAT_CHECK_ARG(n_axes >= 1 && n_axes <= 4, "%s: %d axes, 1 to 4 are possible", fn, n_axes);
  SAT_CHECK_ARG(T >= 0 && T < kMaxGroups && H >= 1 && H <= (1 << 16) && dh >= 2 && dh % 2 == 0 && dh <= (1 << 12),
                "%s: bad sizes T=%d H=%d dh=%d (dh must be even)", fn, T, H, dh);
  SAT_CHECK_ARG((int64_t)H * dh * dh < (1LL << 32), "%s: %d heads of %d dims are too wide", fn, H, dh);
  int half = 0;
  for (int a = 0; a < n_axes; ++a) {
    SAT_CHECK_ARG(pairs[a] >= 0 && pairs[a] <= 128, "%s: axis %d has %d pairs", fn, a, pairs[a]);
    half += pairs[a];
  }
  SAT_CHECK_ARG(half >= 1 && half <= 128 && 2 * half <= dh, "%s: %d pairs must be 1 to 128 and fit head dim %d", fn,
                half, dh);
  SAT_CHECK_ARG(ldx >= (int64_t)H * dh && ldy >= (int64_t)H * dh && ldp >= n_axes,
                "%s: leading dimensions must cover the heads and the axes", fn);
  SAT_CHECK_ARG(x != y || !x || ldx == ldy, "%s: in place, ldx and ldy must agree", fn);
  SAT_CHECK_ARG(aligned(x, f32 ? 4 : 2) && aligned(y, f32 ? 4 : 2) && aligned(pos, 4),
                "%s: x, y and pos must be aligned to their elements", fn);
  SAT_CHECK_ARG(base > 0 && isfinite(base), "%s: base must be positive and finite", fn);
  RotaryAxes a;
  memset(&a, 0, sizeof a);
  a.x = x; a.y = y; a.pos = pos;
  a.ldx = ldx; a.ldy = ldy; a.ldp = ldp;
  a.T = T; a.H = H; a.dh = dh; a.half = half; a.inverse = inverse != 0;
  // turns per position of pair j of n: base^(-j / n) / (2 pi), as the product of two powers (a power
  // for each pair would take longer than the launch)
  const double turn = 6.283185307179586476925286766559;
  double fine[8], coarse[16];
  auto powers = [&](int n) {
    for (int k = 0; k < 8 && k < n; ++k) fine[k] = pow(base, -(double)k / n);
    for (int k = 0; 8 * k < n; ++k) coarse[k] = pow(base, -8.0 * k / n) / turn;
  };
  if (!own_freqs) powers(half);
  for (int ax = 0, i = 0; ax < n_axes; ++ax) {
    if (own_freqs && pairs[ax]) powers(pairs[ax]);
    for (int j = 0; j < pairs[ax]; ++j, ++i) {
      const int k = own_freqs ? j : i;
      a.axis[i] = (uint8_t)ax;
      a.freq[i] = fine[k & 7] * coarse[k >> 3];
    }
  }
  SAT_HIP(launch_rotary_axes(a, f32 != 0, interleaved != 0, S(stream)));
  return SAT_OK;
}

// ---------------------------------------------------------------- AdamW

// 32 bits that stand for step t of tensor j: a 64-bit mix of the three.
static uint32_t dither_key(uint64_t seed, int64_t t, int j) {
  uint64_t z = seed ^ ((uint64_t)t * 0x9E3779B97F4A7C15ull);
  z += (uint64_t)j * 0xD1B54A32D192ED03ull;
  z ^= z >> 32;
  z *= 0xD6E8FEB86659FD93ull;
  return (uint32_t)(z ^ z >> 32);
}

// Fills launches of up to kAdamWEntries tensors and hands each to `go` (chunks, arguments).
template <class Fill, class Go>
static hipError_t over_tensors(const sat_adamw_tensor* t, int32_t count, int chunk, const AdamWConsts& c, Fill fill,
                               Go go) {
  AdamWMulti a;
  a.c = c;
  a.count = 0;
  int64_t chunks = 0;
  for (int k = 0; k < count; ++k) {
    if (t[k].n == 0) continue;
    const int64_t more = (t[k].n + chunk - 1) / chunk;
    if (a.count == kAdamWEntries || chunks + more >= kMaxGroups) {
      const hipError_t e = go(a, (int)chunks);
      if (e != hipSuccess) return e;
      a.count = 0;
      chunks = 0;
    }
    a.first[a.count] = (int)chunks;
    fill(k, a.t[a.count]);
    chunks += more;
    ++a.count;
  }
  return a.count ? go(a, (int)chunks) : hipSuccess;
}

static constexpr int64_t kMaxN = 1LL << 35;  // one tensor's chunks fit a launch

extern "C" sat_status sat_op_adamw_multi(const sat_adamw_tensor* t, int32_t count, int32_t state_bits,
                                         int32_t grad_bf16, double lr, double beta1, double beta2, double eps,
                                         int64_t step, uint64_t seed, void* stream) {
  const char* fn = "adamw_multi";
  SAT_CHECK_ARG(count >= 0 && (t != nullptr || count == 0), "%s: no table of %d tensors", fn, count);
  SAT_CHECK_ARG(state_bits == 8 || state_bits == 32, "%s: state_bits must be 8 or 32", fn);
  SAT_CHECK_ARG(step >= 1, "%s: t >= 1 required", fn);
  SAT_CHECK_ARG(beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1 && eps >= 0 && isfinite(lr),
                "%s: betas must be in [0, 1), eps >= 0 and lr finite", fn);
  const uintptr_t ga = grad_bf16 ? 2 : 4, sa = state_bits == 8 ? 1 : 4;
  int64_t total = 0;
  for (int k = 0; k < count; ++k) {
    const sat_adamw_tensor& e = t[k];
    SAT_CHECK_ARG(e.n >= 0 && e.n <= kMaxN, "%s: tensor %d has n=%ld", fn, k, (long)e.n);
    if (e.n == 0) continue;
    total += e.n;
    SAT_CHECK_ARG(e.p && e.g && e.m && e.v && (state_bits == 32 || (e.m_exp && e.v_exp)), "%s: tensor %d: null pointer",
                  fn, k);
    SAT_CHECK_ARG(aligned(e.p, 4) && aligned(e.g, ga) && aligned(e.m, sa) && aligned(e.v, sa) && aligned(e.shadow, 2),
                  "%s: tensor %d: arrays must be aligned to their elements", fn, k);
  }
  const AdamWConsts c = adamw_consts(lr, beta1, beta2, eps, 0.0, step);
  const int chunk = total < 1024LL * kAdamWMultiChunk ? kAdamWMultiSmall : kAdamWMultiChunk;
  SAT_HIP(over_tensors(
      t, count, chunk, c,
      [&](int k, AdamWEntry& o) {
        const sat_adamw_tensor& e = t[k];
        o.p = e.p; o.g = e.g; o.m = e.m; o.v = e.v; o.m_exp = e.m_exp; o.v_exp = e.v_exp;
        o.shadow = (bf16*)e.shadow;
        o.n = e.n;
        o.lr_wd = (float)(lr * e.weight_decay);
        o.key = dither_key(seed, step, k);
        o.vec = aligned(e.p, 16) && aligned(e.g, 4 * ga) && aligned(e.m, 4 * sa) && aligned(e.v, 4 * sa) &&
                aligned(e.shadow, 8);
      },
      [&](const AdamWMulti& a, int chunks) {
        return launch_adamw_multi(a, chunks, chunk, state_bits, grad_bf16 != 0, S(stream));
      }));
  return SAT_OK;
}

// Whether outputs of adamw_multi_state, elements of `size` bytes, overlap each other or what it reads.
static sat_status state_outputs(const sat_adamw_tensor* t, int32_t count, void* const* m_out, void* const* v_out,
                                uintptr_t size, const char* fn) {
  struct Span {
    uintptr_t at, end;
  };
  const std::unique_ptr<Span[]> out(new (std::nothrow) Span[2 * (size_t)count + 1]);
  if (!out) {
    sat_set_error("%s: no host memory for %d tensors", fn, count);
    return SAT_ENOMEM;
  }
  size_t n = 0;
  for (void* const* list : {m_out, v_out})
    for (int k = 0; k < count; ++k) {
      if (t[k].n == 0) continue;
      const uintptr_t at = reinterpret_cast<uintptr_t>(list[k]);
      out[n++] = Span{at, at + (uintptr_t)t[k].n * size};
    }
  Span* const end = out.get() + n;
  const auto before = [](const Span& a, const Span& b) { return a.at < b.at; };
  if (!std::is_sorted(out.get(), end, before)) std::sort(out.get(), end, before);
  for (size_t i = 1; i < n; ++i) SAT_CHECK_ARG(out[i].at >= out[i - 1].end, "%s: outputs overlap each other", fn);
  for (int k = 0; k < count; ++k) {
    if (t[k].n == 0) continue;
    const uintptr_t blocks = (uintptr_t)(t[k].n + 255) / 256;
    const std::pair<const void*, uintptr_t> reads[] = {
        {t[k].m, (uintptr_t)t[k].n}, {t[k].v, (uintptr_t)t[k].n}, {t[k].m_exp, blocks}, {t[k].v_exp, blocks}};
    for (const auto& r : reads) {
      const uintptr_t at = reinterpret_cast<uintptr_t>(r.first);
      // the last output that begins before the end of what is read ends before its beginning
      const Span* o = std::lower_bound(out.get(), end, Span{at + r.second, 0}, before);
      SAT_CHECK_ARG(o == out.get() || o[-1].end <= at, "%s: tensor %d: an output overlaps its moments", fn, k);
    }
  }
  return SAT_OK;
}

extern "C" sat_status sat_op_adamw_multi_state(const sat_adamw_tensor* t, int32_t count, void* const* m_out,
                                               void* const* v_out, int32_t out_bf16, void* stream) {
  const char* fn = "adamw_multi_state";
  SAT_CHECK_ARG(count >= 0 && ((t && m_out && v_out) || count == 0), "%s: no tables of %d tensors", fn, count);
  const uintptr_t oa = out_bf16 ? 2 : 4;
  for (int k = 0; k < count; ++k) {
    const sat_adamw_tensor& e = t[k];
    SAT_CHECK_ARG(e.n >= 0 && e.n <= kMaxN, "%s: tensor %d has n=%ld", fn, k, (long)e.n);
    if (e.n == 0) continue;
    SAT_CHECK_ARG(e.m && e.v && e.m_exp && e.v_exp && m_out[k] && v_out[k], "%s: tensor %d: null pointer", fn, k);
    SAT_CHECK_ARG(aligned(m_out[k], oa) && aligned(v_out[k], oa), "%s: tensor %d: outputs must be aligned to their elements",
                  fn, k);
  }
  if (count > 0) {
    const sat_status st = state_outputs(t, count, m_out, v_out, oa, fn);
    if (st != SAT_OK) return st;
  }
  AdamWConsts none;
  memset(&none, 0, sizeof none);
  SAT_HIP(over_tensors(
      t, count, kAdamWMultiChunk, none,
      [&](int k, AdamWEntry& o) {
        const sat_adamw_tensor& e = t[k];
        memset(&o, 0, sizeof o);
        o.m = e.m; o.v = e.v; o.m_exp = e.m_exp; o.v_exp = e.v_exp;
        o.m_out = m_out[k]; o.v_out = v_out[k];
        o.n = e.n;
        o.vec = aligned(e.m, 16 / oa) && aligned(e.v, 16 / oa) && aligned(m_out[k], 16) && aligned(v_out[k], 16);
      },
      [&](const AdamWMulti& a, int chunks) { return launch_adamw_state(a, chunks, out_bf16 != 0, S(stream)); }));
  return SAT_OK;
}
