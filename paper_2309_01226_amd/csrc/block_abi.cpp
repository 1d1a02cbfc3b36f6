// Kernel-level C ABI (include/saturn_ops.h) of the operators around a step's blocks: dropout, the
// boundary of two sublayers, the head with its cross entropy.  Argument checks, then the launches; nothing is
// allocated on the device.
#include <math.h>
#include <string.h>

#include "../../include/saturn_ops.h"
#include "abi_common.h"
#include "kernels.h"

static inline hipStream_t S(void* s) { return reinterpret_cast<hipStream_t>(s); }
static bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

static constexpr int64_t kMaxLd = 1LL << 40;  // rows x ld stays within 64 bits

// ---------------------------------------------------------------- dropout

struct DropRate {
  uint32_t limit;
  float up;
};
static DropRate drop_rate(double p) {
  const uint32_t limit = (uint32_t)nearbyint(65536.0 * p);
  return DropRate{limit, limit < 65536 ? (float)(65536.0 / (65536 - limit)) : 0.f};
}

extern "C" sat_status sat_op_dropout(const void* x, int64_t ldx, void* y, int64_t ldy, int32_t f32, int32_t rows,
                                     int32_t cols, double p, uint64_t seed, const int64_t* step, void* stream) {
  const char* fn = "dropout";
  SAT_CHECK_ARG(rows >= 0 && cols >= 0 && cols <= (1 << 18), "%s: bad sizes rows=%d cols=%d (up to 2^18)", fn, rows, cols);
  SAT_CHECK_ARG((int64_t)rows * ((cols + 7) / 8) < (1LL << 31), "%s: %d rows of %d columns are too many", fn, rows, cols);
  SAT_CHECK_ARG(rows == 0 || cols == 0 || (x && y), "%s: null pointer", fn);
  SAT_CHECK_ARG(p >= 0 && p <= 1, "%s: p=%g must be in [0, 1]", fn, p);
  SAT_CHECK_ARG(ldx >= cols && ldy >= cols && ldx < kMaxLd && ldy < kMaxLd, "%s: leading dimensions must cover the columns", fn);
  SAT_CHECK_ARG(x != y || !x || ldx == ldy, "%s: in place, ldx and ldy must agree", fn);
  const uintptr_t size = f32 ? 4 : 2;
  SAT_CHECK_ARG(aligned(x, size) && aligned(y, size) && aligned(step, 8), "%s: x, y and step must be aligned to their elements", fn);
  const DropRate r = drop_rate(p);
  DropoutArgs a;
  memset(&a, 0, sizeof a);
  a.x = x; a.y = y; a.ldx = ldx; a.ldy = ldy; a.rows = rows; a.cols = cols;
  a.seed = seed; a.limit = r.limit; a.up = r.up; a.step = (const uint64_t*)step;
  SAT_HIP(launch_dropout(a, f32 != 0, S(stream)));
  return SAT_OK;
}

// ---------------------------------------------------------------- residual norm

// Checks what forward and backward share and fills their arguments.
static sat_status residual_norm_args(const sat_residual_norm_desc* d, ResidualNormArgs* out, const char* fn) {
  SAT_CHECK_ARG(d != nullptr, "%s: null descriptor", fn);
  SAT_CHECK_ARG(d->T >= 0 && d->T < (1 << 30) && d->d >= 1 && d->d <= kResidualNormMaxD, "%s: bad sizes T=%d d=%d (1 to %d)",
                fn, d->T, d->d, kResidualNormMaxD);
  SAT_CHECK_ARG(d->pre >= 0 && d->pre <= 2 && d->post >= 0 && d->post <= 2, "%s: norms must be 0, 1 or 2, got %d and %d", fn,
                d->pre, d->post);
  SAT_CHECK_ARG((d->pre || (!d->g_pre && !d->b_pre)) && (d->post || (!d->g_post && !d->b_post)),
                "%s: a gain or shift of a norm that is not there", fn);
  SAT_CHECK_ARG(isfinite(d->alpha) && isfinite(d->beta), "%s: alpha and beta must be finite", fn);
  SAT_CHECK_ARG(d->eps >= 0 && isfinite(d->eps), "%s: eps must be finite and not negative", fn);
  SAT_CHECK_ARG(d->p >= 0 && d->p <= 1, "%s: p=%g must be in [0, 1]", fn, d->p);
  SAT_CHECK_ARG(d->T == 0 || (!d->pre && !d->post) || d->stats, "%s: null pointer", fn);
  SAT_CHECK_ARG(aligned(d->stats, 4) && aligned(d->g_pre, 4) && aligned(d->b_pre, 4) && aligned(d->g_post, 4) &&
                    aligned(d->b_post, 4) && aligned(d->gate, 4) && aligned(d->step, 8),
                "%s: vectors must be aligned to their elements", fn);
  const DropRate r = drop_rate(d->p);
  ResidualNormArgs& a = *out;
  memset(&a, 0, sizeof a);
  a.x = d->x; a.y = d->y; a.f = (const bf16*)d->f; a.h = (bf16*)d->h; a.stats = d->stats;
  a.g_pre = d->g_pre; a.b_pre = d->b_pre; a.g_post = d->g_post; a.b_post = d->b_post; a.gate = d->gate;
  a.ldx = d->ldx; a.ldy = d->ldy; a.ldf = d->ldf; a.ldh = d->ldh;
  a.T = d->T; a.d = d->d; a.pre = d->pre; a.post = d->post;
  a.alpha = d->alpha; a.beta = d->beta; a.eps = d->eps;
  a.seed = d->seed; a.limit = r.limit; a.up = r.up; a.step = (const uint64_t*)d->step;
  return SAT_OK;
}

// Rows of `size`-byte elements at p that the call needs.
static bool rows_ok(const void* p, int64_t ld, uintptr_t size, const sat_residual_norm_desc* d) {
  return (d->T == 0 || p) && ld >= d->d && ld < kMaxLd && aligned(p, size);
}

extern "C" sat_status sat_op_residual_norm_fwd(const sat_residual_norm_desc* d, void* stream) {
  const char* fn = "residual_norm_fwd";
  ResidualNormArgs a;
  const sat_status st = residual_norm_args(d, &a, fn);
  if (st != SAT_OK) return st;
  const uintptr_t size = d->stream_f32 ? 4 : 2;
  SAT_CHECK_ARG(rows_ok(d->x, d->ldx, size, d) && rows_ok(d->y, d->ldy, size, d) && rows_ok(d->f, d->ldf, 2, d) &&
                    (!d->pre || rows_ok(d->h, d->ldh, 2, d)),
                "%s: x, f, y and, with a norm, h: null, not aligned to their elements, or rows shorter than d", fn);
  SAT_CHECK_ARG(d->x != d->y || !d->x || d->ldx == d->ldy, "%s: in place, ldx and ldy must agree", fn);
  SAT_HIP(launch_residual_norm_fwd(a, d->stream_f32 != 0, S(stream)));
  return SAT_OK;
}

static int sums_of(const sat_residual_norm_desc* d) {
  return !!d->dg_pre + !!d->db_pre + !!d->dg_post + !!d->db_post + !!d->dgate;
}

extern "C" sat_status sat_op_residual_norm_bwd_ws(const sat_residual_norm_desc* d, int64_t* elems) {
  SAT_CHECK_ARG(d && elems, "residual_norm_bwd_ws: null pointer");
  SAT_CHECK_ARG(d->T >= 0 && d->T < (1 << 30) && d->d >= 1 && d->d <= kResidualNormMaxD,
                "residual_norm_bwd_ws: bad sizes T=%d d=%d", d->T, d->d);
  *elems = residual_norm_ws(d->T, d->d, sums_of(d));
  return SAT_OK;
}

extern "C" sat_status sat_op_residual_norm_bwd(const sat_residual_norm_desc* d, void* stream) {
  const char* fn = "residual_norm_bwd";
  ResidualNormArgs a;
  const sat_status st = residual_norm_args(d, &a, fn);
  if (st != SAT_OK) return st;
  const uintptr_t size = d->stream_f32 ? 4 : 2;
  SAT_CHECK_ARG((!d->dy || rows_ok(d->dy, d->lddy, size, d)) && rows_ok(d->dx, d->lddx, size, d) &&
                    rows_ok(d->df, d->lddf, 2, d) &&
                    (!d->pre || (rows_ok(d->y, d->ldy, size, d) && rows_ok(d->dh, d->lddh, 2, d))) &&
                    ((!d->post && !d->dgate) || rows_ok(d->f, d->ldf, 2, d)),
                "%s: dx, df and what the norms and the gate need of dy, dh, y and f: null, not aligned to their elements, "
                "or rows shorter than d",
                fn);
  SAT_CHECK_ARG(d->dx != d->dy || !d->dx || d->lddx == d->lddy, "%s: in place, lddx and lddy must agree", fn);
  SAT_CHECK_ARG((d->pre || (!d->dg_pre && !d->db_pre)) && (d->post || (!d->dg_post && !d->db_post)) && (d->gate || !d->dgate),
                "%s: a gradient of something that is not there", fn);
  SAT_CHECK_ARG(aligned(d->dg_pre, 4) && aligned(d->db_pre, 4) && aligned(d->dg_post, 4) && aligned(d->db_post, 4) &&
                    aligned(d->dgate, 4) && aligned(d->ws, 4),
                "%s: vectors must be aligned to their elements", fn);
  const int64_t need = residual_norm_ws(d->T, d->d, sums_of(d));
  SAT_CHECK_ARG(need == 0 || (d->ws && d->ws_elems >= need), "%s: ws of %ld elements, %ld needed", fn, (long)d->ws_elems,
                (long)need);
  a.dy = d->dy; a.dh = (const bf16*)d->dh; a.dx = d->dx; a.df = (bf16*)d->df;
  a.lddy = d->lddy; a.lddh = d->lddh; a.lddx = d->lddx; a.lddf = d->lddf;
  a.dg_pre = d->dg_pre; a.db_pre = d->db_pre; a.dg_post = d->dg_post; a.db_post = d->db_post; a.dgate = d->dgate;
  a.ws = d->ws;
  SAT_HIP(launch_residual_norm_bwd(a, d->stream_f32 != 0, S(stream)));
  return SAT_OK;
}

// ---------------------------------------------------------------- head with cross entropy

static constexpr int64_t kMaxHeadLd = 1 << 21;  // a tile's rows stay within 32-bit buffer offsets

static sat_status linear_xent_sizes(const sat_linear_xent_desc* d, LinearXentArgs* out, const char* fn) {
  SAT_CHECK_ARG(d != nullptr, "%s: null descriptor", fn);
  SAT_CHECK_ARG(d->N >= 0 && d->N <= (1 << 25) && d->V >= 1 && d->V <= (1 << 20),
                "%s: bad sizes N=%d V=%d (up to 2^25 and 2^20)", fn, d->N, d->V);
  SAT_CHECK_ARG(d->d >= 8 && d->d <= (1 << 16) && d->d % 8 == 0, "%s: d=%d must be a multiple of 8 up to 2^16", fn, d->d);
  SAT_CHECK_ARG(!d->accumulate || d->grad_f32, "%s: only fp32 gradients are added to", fn);
  SAT_CHECK_ARG(!d->db || d->bias, "%s: a gradient of a bias that is not there", fn);
  LinearXentArgs& a = *out;
  memset(&a, 0, sizeof a);
  a.dx = (bf16*)d->dx; a.dw = d->dw; a.db = d->db;
  a.N = d->N; a.V = d->V; a.d = d->d;
  a.dw_f32 = d->grad_f32 != 0;
  a.accumulate = d->accumulate != 0;
  return SAT_OK;
}

extern "C" sat_status sat_op_linear_xent_ws(const sat_linear_xent_desc* d, int64_t* bytes) {
  SAT_CHECK_ARG(bytes != nullptr, "linear_xent_ws: null pointer");
  LinearXentArgs a;
  const sat_status st = linear_xent_sizes(d, &a, "linear_xent_ws");
  if (st != SAT_OK) return st;
  *bytes = linear_xent_ws(a);
  return SAT_OK;
}

extern "C" sat_status sat_op_linear_xent(const sat_linear_xent_desc* d, void* stream) {
  const char* fn = "linear_xent";
  LinearXentArgs a;
  const sat_status st = linear_xent_sizes(d, &a, fn);
  if (st != SAT_OK) return st;
  SAT_CHECK_ARG(d->N == 0 || (d->x && d->labels && d->row_loss && d->lse), "%s: null pointer", fn);
  SAT_CHECK_ARG(d->w && d->inv_n && d->ws, "%s: null pointer", fn);
  SAT_CHECK_ARG(d->ldx >= d->d && d->ldw >= d->d && d->ldx < kMaxHeadLd && d->ldw < kMaxHeadLd && d->ldx % 8 == 0 &&
                    d->ldw % 8 == 0 && aligned(d->x, 16) && aligned(d->w, 16),
                "%s: x and w must be 16-byte aligned with leading dimensions %% 8 == 0, at least d and below 2^21", fn);
  SAT_CHECK_ARG(!d->dx || (d->lddx >= d->d && d->lddx < kMaxLd && d->lddx % 8 == 0 && aligned(d->dx, 16)),
                "%s: dx must be 16-byte aligned with lddx %% 8 == 0, at least d", fn);
  SAT_CHECK_ARG(!d->dw || (d->lddw >= d->d && d->lddw < kMaxLd && d->lddw % (d->grad_f32 ? 4 : 8) == 0 && aligned(d->dw, 16)),
                "%s: dw must be 16-byte aligned with 16-byte aligned rows of at least d", fn);
  SAT_CHECK_ARG((!d->dx || d->dx != d->x) && (!d->dw || d->dw != d->w), "%s: gradients are not written over x or w", fn);
  SAT_CHECK_ARG(aligned(d->labels, 4) && aligned(d->bias, 4) && aligned(d->row_weight, 4) && aligned(d->row_loss, 4) &&
                    aligned(d->lse, 4) && aligned(d->inv_n, 4) && aligned(d->db, d->grad_f32 ? 4 : 2),
                "%s: vectors must be aligned to their elements", fn);
  const int64_t need = linear_xent_ws(a);
  SAT_CHECK_ARG(d->ws_bytes >= need && aligned(d->ws, 256), "%s: ws of %ld bytes, %ld needed, 256-byte aligned", fn,
                (long)d->ws_bytes, (long)need);
  a.x = (const bf16*)d->x; a.w = (const bf16*)d->w; a.labels = d->labels; a.bias = d->bias; a.row_weight = d->row_weight;
  a.row_loss = d->row_loss; a.lse = d->lse; a.inv_n = d->inv_n;
  a.ldx = d->ldx; a.ldw = d->ldw; a.lddx = d->lddx; a.lddw = d->lddw;
  SAT_HIP(launch_linear_xent(a, d->ws, S(stream)));
  return SAT_OK;
}
