// C ABI of the individual kernels: argument checks and marshalling only.
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <new>
#include <utility>
#include <vector>

#include "../../include/bamboo_debug.h"
#include "../../include/bamboo_kernels.h"
#include "../../include/bamboo_stage.h"
#include "common.h"

using namespace bamboo;

namespace {
int finish(hipError_t e) {
  if (e == hipSuccess) return BAMBOO_OK;
  if (getenv("BAMBOO_DEBUG")) fprintf(stderr, "[bamboo] HIP error %d: %s\n", (int)e, hipGetErrorString(e));
  (void)hipGetLastError();
  return e == hipErrorNotSupported ? BAMBOO_E_STATE : BAMBOO_E_HIP;
}
int run_gemm(int dtype, int impl, GemmDesc& d, void* stream) {
  (void)hipGetLastError();  // an earlier, unrelated failure in this thread must not be blamed on this launch
  if (dtype != 0 && dtype != 1) return BAMBOO_E_ARG;
  if (d.M <= 0 || d.N <= 0 || d.K <= 0 || !d.A || !d.B || !d.C) return BAMBOO_E_ARG;
  hipStream_t s = (hipStream_t)stream;
  if (impl == 1) return finish(launch_gemm_simple(s, dtype, d));
  d.tiled_only = impl == 2;
  // the forced kernel takes whole groups of 8 in every dimension; the automatic choice has no such limit on rows
  if (impl == 2) return dtype == 1 && d.M % 8 == 0 && d.K % 8 == 0 ? finish(launch_gemm_mfma(s, d)) : BAMBOO_E_STATE;
  if (impl != 0) return BAMBOO_E_ARG;
  return finish(launch_gemm(s, dtype, d));
}
}  // namespace

extern "C" {

int bk_linear_fwd(int dtype, int impl, int T, int N, int K, const void* X, const void* W, const void* bias,
                  const void* res, void* Y, void* gelu_out, void* stream) {
  if (!bias || (res && gelu_out)) return BAMBOO_E_ARG;   // with gelu_out: Y = GELU'(h), gelu_out = GELU(h)
  GemmDesc d;
  memset(&d, 0, sizeof(d));
  d.A = X; d.B = W; d.C = Y; d.M = T; d.N = N; d.K = K;
  d.a_sm = K; d.a_sk = 1; d.b_sk = N; d.b_sn = 1;
  d.bias = bias; d.res = res; d.aux_out = gelu_out;
  d.epi = gelu_out ? EPI_BIAS_GELU : (res ? EPI_BIAS_RES : EPI_BIAS);
  return run_gemm(dtype, impl, d, stream);
}

int bk_linear_bwd_input(int dtype, int impl, int T, int K, int N, const void* dY, const void* W, const void* res,
                        const void* mul, void* dX, void* stream) {
  if (mul && res) return BAMBOO_E_ARG;
  GemmDesc d;
  memset(&d, 0, sizeof(d));
  d.A = dY; d.B = W; d.C = dX; d.M = T; d.N = K; d.K = N;
  d.a_sm = N; d.a_sk = 1; d.b_sk = 1; d.b_sn = N;
  d.res = res; d.aux_in = mul;
  d.epi = mul ? EPI_MUL : (res ? EPI_RES : EPI_STORE);
  return run_gemm(dtype, impl, d, stream);
}

int bk_linear_bwd_weight(int dtype, int impl, int T, int K, int N, const void* X, const void* dY, float* dW,
                         float* db, float* partial, void* stream) {
  if (db != nullptr && partial == nullptr) return BAMBOO_E_ARG;
  GemmDesc d;
  memset(&d, 0, sizeof(d));
  d.A = X; d.B = dY; d.C = dW; d.M = K; d.N = N; d.K = T;
  d.a_sm = 1; d.a_sk = K; d.b_sk = N; d.b_sn = 1;
  d.epi = EPI_ACC_F32;
  d.colsum_out = db; d.colsum_partial = partial;
  if (impl != 0 && db != nullptr) {   // a forced kernel bypasses launch_gemm: the column sum is launched here
    (void)hipGetLastError();
    const int rc = finish(launch_colsum_acc((hipStream_t)stream, dtype, T, N, dY, db, partial));
    if (rc != BAMBOO_OK) return rc;
    d.colsum_out = nullptr;
  }
  return run_gemm(dtype, impl, d, stream);
}

int bk_linear_bwd_weight_group(int dtype, int n, const int* T, const int* K, const int* N, const void* const* X,
                               const void* const* dY, float* const* dW, void* stream) {
  if ((dtype != 0 && dtype != 1) || n < 1 || n > GemmGroup::MAX || !T || !K || !N || !X || !dY || !dW) return BAMBOO_E_ARG;
  GemmDesc d[GemmGroup::MAX];
  memset(d, 0, sizeof(d));
  for (int i = 0; i < n; ++i) {
    if (T[i] <= 0 || K[i] <= 0 || N[i] <= 0 || !X[i] || !dY[i] || !dW[i]) return BAMBOO_E_ARG;
    d[i].A = X[i]; d[i].B = dY[i]; d[i].C = dW[i]; d[i].M = K[i]; d[i].N = N[i]; d[i].K = T[i];
    d[i].a_sm = 1; d[i].a_sk = K[i]; d[i].b_sk = N[i]; d[i].b_sn = 1; d[i].epi = EPI_ACC_F32;
  }
  (void)hipGetLastError();
  return finish(launch_gemm_group((hipStream_t)stream, dtype, d, n));
}

int bk_colsum_acc(int dtype, int T, int N, const void* A, float* out, float* partial, void* stream) {
  if ((dtype != 0 && dtype != 1) || T <= 0 || N <= 0 || N % 2 || !A || !out || !partial) return BAMBOO_E_ARG;
  (void)hipGetLastError();
  return finish(launch_colsum_acc((hipStream_t)stream, dtype, T, N, A, out, partial));
}
uint64_t bk_colsum_scratch_floats(int N) { return colsum_partial_floats(N); }

static int attn_desc(AttnDesc& a, int dtype, int batch, int seq, int heads, int d, int causal) {
  if ((dtype != 0 && dtype != 1) || batch <= 0 || seq <= 0 || heads <= 0 || d <= 0 || d > 128) return BAMBOO_E_ARG;
  memset(&a, 0, sizeof(a));
  a.B = batch; a.S = seq; a.heads = heads; a.d = d; a.causal = causal != 0;
  return BAMBOO_OK;
}

int bk_attention_fwd(int dtype, int impl, int batch, int seq, int heads, int d, int causal, const void* qkv, void* ctx,
                     float* lse, void* stream) {
  AttnDesc a;
  if (attn_desc(a, dtype, batch, seq, heads, d, causal) != BAMBOO_OK || !qkv || !ctx || !lse) return BAMBOO_E_ARG;
  a.qkv = qkv; a.ctx = ctx; a.lse = lse;
  hipStream_t s = (hipStream_t)stream;
  (void)hipGetLastError();
  if (impl == 1) return finish(launch_attention_fwd_simple(s, dtype, a));
  if (impl == 2) return dtype == 1 ? finish(launch_attention_fwd_mfma(s, a)) : BAMBOO_E_STATE;
  if (impl != 0) return BAMBOO_E_ARG;
  return finish(launch_attention_fwd(s, dtype, a));
}

int bk_attention_bwd(int dtype, int impl, int batch, int seq, int heads, int d, int causal, const void* qkv,
                     const void* ctx, const float* lse, const void* dctx, void* dqkv, float* delta, void* stream) {
  AttnDesc a;
  if (attn_desc(a, dtype, batch, seq, heads, d, causal) != BAMBOO_OK || !qkv || !ctx || !lse || !dctx || !dqkv ||
      !delta)
    return BAMBOO_E_ARG;
  a.qkv = qkv; a.ctx = (void*)ctx; a.lse = (float*)lse; a.dctx = dctx; a.dqkv = dqkv; a.delta = delta;
  hipStream_t s = (hipStream_t)stream;
  (void)hipGetLastError();
  if (impl == 1) return finish(launch_attention_bwd_simple(s, dtype, a));
  if (impl == 2) return dtype == 1 ? finish(launch_attention_bwd_mfma(s, a)) : BAMBOO_E_STATE;
  if (impl != 0) return BAMBOO_E_ARG;
  return finish(launch_attention_bwd(s, dtype, a));
}

int bk_layernorm_fwd(int dtype, int T, int H, float eps, const void* r, const void* gamma, const void* beta, void* y,
                     float* stats, void* stream) {
  if ((dtype != 0 && dtype != 1) || T <= 0 || H <= 0 || H % 8 || !r || !gamma || !beta || !y || !stats)
    return BAMBOO_E_ARG;
  (void)hipGetLastError();
  return finish(launch_layernorm_fwd((hipStream_t)stream, dtype, T, H, eps, r, gamma, beta, y, stats));
}

int bk_layernorm_bwd(int dtype, int T, int H, const void* dout, const void* r, const float* stats, const void* gamma,
                     const void* add, void* dr, float* dgamma, float* dbeta, float* partial, void* stream) {
  if ((dtype != 0 && dtype != 1) || T <= 0 || H <= 0 || H % 8 || !dout || !r || !stats || !gamma || !dr || !dgamma ||
      !dbeta || !partial)
    return BAMBOO_E_ARG;
  (void)hipGetLastError();
  return finish(launch_layernorm_bwd((hipStream_t)stream, dtype, T, H, dout, r, stats, gamma, add, dr, dgamma, dbeta,
                                     partial));
}
int bk_layernorm_bwd_bias(int dtype, int T, int H, const void* dout, const void* r, const float* stats, const void* gamma,
                          const void* add, void* dr, float* dgamma, float* dbeta, float* dbias, float* partial, void* stream) {
  if ((dtype != 0 && dtype != 1) || T <= 0 || H <= 0 || H % 8 || !dout || !r || !stats || !gamma || !dr || !dgamma ||
      !dbeta || !dbias || !partial)
    return BAMBOO_E_ARG;
  (void)hipGetLastError();
  const size_t rows = ln_bwd_partial_floats(H) / 2;
  float *pg = partial, *pb = pg + rows, *pc = pb + rows;
  int parts = 0;
  hipError_t e = launch_layernorm_bwd_partials((hipStream_t)stream, dtype, T, H, dout, r, stats, gamma, add, dr, pg, pb, pc,
                                               &parts);
  GradReduceBatch sums;
  sums.n = 0;
  if (e == hipSuccess && !(grad_reduce_add(&sums, H, parts, pg, dgamma, pb, dbeta) &&
                           grad_reduce_add(&sums, H, parts, pc, dbias, nullptr, nullptr)))
    return BAMBOO_E_STATE;
  if (e == hipSuccess) e = launch_grad_reduce((hipStream_t)stream, sums);
  return finish(e);
}
uint64_t bk_layernorm_bwd_scratch_floats(int H) { return ln_bwd_partial_floats(H); }

int bk_copy(const void* src, void* dst, uint64_t bytes, void* stream) {
  if (!src || !dst || bytes % 16 || ((uintptr_t)src & 15) || ((uintptr_t)dst & 15)) return BAMBOO_E_ARG;
  (void)hipGetLastError();
  return finish(launch_calibration_copy((hipStream_t)stream, src, dst, (size_t)bytes));
}

int bk_adam(int dtype, int64_t n, const float* g, float* master, float* m, float* v, void* w, float lr, float beta1,
            float beta2, float eps, int step, void* stream) {
  if (dtype != 0 && dtype != 1) return BAMBOO_E_ARG;
  if (n <= 0 || n % 4 || step < 1 || !g || !master || !m || !v || !w) return BAMBOO_E_ARG;
  const void* ptrs[] = {g, master, m, v, w};
  for (const void* p : ptrs)
    if (((uintptr_t)p) & 15) return BAMBOO_E_ARG;
  (void)hipGetLastError();
  return finish(launch_adam((hipStream_t)stream, dtype, (long)n, g, master, m, v, w, lr, beta1, beta2, eps, step));
}

int bk_embedding_fwd(int dtype, int T, int seq, int H, int V, const int32_t* ids, const void* E_tok, const void* E_pos,
                     void* out, void* stream) {
  if ((dtype != 0 && dtype != 1) || T <= 0 || seq <= 0 || H <= 0 || H % 8 || V <= 0) return BAMBOO_E_ARG;
  if (!ids || !E_tok || !E_pos || !out) return BAMBOO_E_ARG;
  if (((uintptr_t)E_tok | (uintptr_t)E_pos | (uintptr_t)out) & 31) return BAMBOO_E_ARG;
  (void)hipGetLastError();
  return finish(launch_embed_fwd((hipStream_t)stream, dtype, T, seq, H, V, ids, E_tok, E_pos, out));
}

int bk_embedding_bwd(int dtype, int T, int seq, int H, int V, const int32_t* ids, const void* g, float* dE_tok,
                     float* dE_pos, void* stream) {
  if ((dtype != 0 && dtype != 1) || T <= 0 || seq <= 0 || T % seq || H <= 0 || V <= 0) return BAMBOO_E_ARG;
  if (!ids || !g || !dE_tok || !dE_pos) return BAMBOO_E_ARG;
  (void)hipGetLastError();
  return finish(launch_embed_bwd((hipStream_t)stream, dtype, T, seq, H, V, ids, g, dE_tok, dE_pos));
}

int bk_softmax_xent_fwd(int dtype, int T, int V, const void* logits, const int32_t* labels, float* lse,
                        float* loss_tok, void* stream) {
  if ((dtype != 0 && dtype != 1) || T <= 0 || V <= 0 || V % 8) return BAMBOO_E_ARG;
  if (!logits || !labels || !lse || !loss_tok || ((uintptr_t)logits & 31)) return BAMBOO_E_ARG;
  (void)hipGetLastError();
  return finish(launch_xent_fwd((hipStream_t)stream, dtype, T, V, logits, labels, lse, loss_tok));
}

int bk_softmax_xent_bwd(int dtype, int T, int V, const void* logits, const int32_t* labels, const float* lse,
                        float scale, void* dlogits, void* stream) {
  if ((dtype != 0 && dtype != 1) || T <= 0 || V <= 0 || V % 8) return BAMBOO_E_ARG;
  if (!logits || !labels || !lse || !dlogits || (((uintptr_t)logits | (uintptr_t)dlogits) & 31)) return BAMBOO_E_ARG;
  (void)hipGetLastError();
  return finish(launch_xent_bwd((hipStream_t)stream, dtype, T, V, logits, labels, lse, scale, dlogits));
}

int bk_ordered_sum(int64_t n, const float* in, float scale, float* out, void* stream) {
  if (n <= 0 || !in || !out) return BAMBOO_E_ARG;
  (void)hipGetLastError();
  return finish(launch_ordered_sum((hipStream_t)stream, (long)n, in, scale, out));
}

// ---- operators around the stage ----------------------------------------------

// A matrix in memory: rows of `cols` elements of `es` bytes, ld elements apart.
struct Matrix {
  const void* p;
  int64_t rows, ld, cols;
  int es;
  uintptr_t first() const { return (uintptr_t)p; }
  uintptr_t last() const { return (uintptr_t)p + (uintptr_t)(((rows - 1) * ld + cols) * es); }
};
// Whether two matrices share an element; columns of one matrix beside each other do not, nor does a matrix with itself, row
// on row, where `itself` says that it may be there.
static bool overlap(const Matrix& a, const Matrix& b, bool itself = false) {
  if (a.first() >= b.last() || b.first() >= a.last()) return false;
  const int64_t away = (int64_t)(b.first() - a.first());
  const int64_t ld = a.rows == 1 ? b.ld : a.ld;                  // the distance between the rows of a single one says nothing
  if ((ld != b.ld && b.rows > 1) || a.es != b.es || away % a.es) return true;
  if (away == 0) return !itself;
  const int64_t off = ((away / a.es) % ld + ld) % ld;            // columns that b's rows begin behind a's
  return !(off >= a.cols && ld - off >= b.cols);
}
constexpr int kMaxVocab = 1 << 27;      // offsets inside a row, and a grid's second dimension
static int element_size(int dtype) { return dtype == 1 ? 2 : 4; }
static bool element_aligned(int dtype, const void* p) { return ((uintptr_t)p & (element_size(dtype) - 1)) == 0; }

int bk_rotary(int dtype, int T, int seq, int heads, int d, int rot, int interleaved, int inverse, const void* x,
              int64_t ldx, const int32_t* pos, const double* freq, float amplitude, void* y, int64_t ldy, void* stream) {
  if ((dtype != 0 && dtype != 1) || T <= 0 || heads <= 0 || d < 2 || d > 512 || rot < 2 || rot > d || rot % 2) return BAMBOO_E_ARG;
  if (!x || !y || !freq || (!pos && seq <= 0)) return BAMBOO_E_ARG;
  const int64_t cols = (int64_t)heads * d;
  if (cols > 0x7fffffff / 8 || ldx < cols || ldy < cols || !element_aligned(dtype, x) || !element_aligned(dtype, y)) return BAMBOO_E_ARG;
  const int es = element_size(dtype);
  if (overlap({x, T, ldx, cols, es}, {y, T, ldy, cols, es}, true)) return BAMBOO_E_ARG;
  RotaryDesc a;
  memset(&a, 0, sizeof(a));
  a.x = x; a.y = y; a.ldx = ldx; a.ldy = ldy; a.T = T; a.seq = seq; a.heads = heads; a.d = d; a.rot = rot;
  a.neighbours = interleaved != 0; a.inverse = inverse != 0; a.copy = x != y; a.pos = pos; a.freq = freq; a.amplitude = amplitude;
  (void)hipGetLastError();
  return finish(launch_rotary((hipStream_t)stream, dtype, a));
}

int bk_rotary_frequencies(int rot, double base, int scaling, double factor, int length, double* freq, float* amplitude) {
  if (rot < 2 || rot % 2 || !(base > 1.) || scaling < 0 || scaling > 3 || !freq) return BAMBOO_E_ARG;
  if (!(base < INFINITY) || (scaling != 0 && !(factor >= 1. && factor < INFINITY)) || (scaling == 3 && length <= 0)) return BAMBOO_E_ARG;
  if (scaling == 2 && rot > 2) base *= pow(factor, (double)rot / (rot - 2));
  for (int i = 0; i < rot / 2; ++i) {
    double f = pow(base, -2. * i / rot);
    if (scaling == 1) f /= factor;
    if (scaling == 3) {
      const double turns = length * f / 6.283185307179586477, kept = fmin(1., fmax(0., (turns - 1.) / 31.));
      f *= kept + (1. - kept) / factor;
    }
    freq[i] = f;
  }
  if (amplitude) *amplitude = scaling == 3 ? (float)(0.1 * log(factor) + 1.) : 1.f;
  return BAMBOO_OK;
}

static bool cross_sizes(int batch, int sq, int sk, int heads, int kv_heads, int d) {
  if (batch <= 0 || sq <= 0 || sk <= 0 || heads <= 0 || kv_heads <= 0 || heads % kv_heads || d <= 0 || d > 128) return false;
  // row numbers and workgroups are 32-bit
  const int64_t group = heads / kv_heads, rows = sq * group, pairs = (int64_t)batch * kv_heads;
  const int64_t most = rows > sk ? rows : sk;
  return rows <= 0x7fffff00 && rows * group <= 0xffffffffLL && sk <= 0x7fffff00 && pairs <= 0x7fffffff &&
         (most + 1024) * pairs <= 0x7fffffff && pairs * most * 2 * d / 256 + 1 <= 0x7fffffff;
}
static int cross_desc(CrossDesc& a, int dtype, int impl, int batch, int sq, int sk, int heads, int kv_heads, int d, const void* q,
                      int64_t ldq, const void* k, const void* v, int64_t ldkv, const int32_t* kv_len, const void* ctx, int64_t ldc,
                      const float* lse, float* scratch) {
  if ((dtype != 0 && dtype != 1) || impl < 0 || impl > 2 || !cross_sizes(batch, sq, sk, heads, kv_heads, d)) return BAMBOO_E_ARG;
  if (!q || !k || !v || !ctx || !lse) return BAMBOO_E_ARG;
  for (const void* p : {q, k, v, ctx})
    if (!element_aligned(dtype, p)) return BAMBOO_E_ARG;
  if (ldq < (int64_t)heads * d || ldkv < (int64_t)kv_heads * d || ldc < (int64_t)heads * d) return BAMBOO_E_ARG;
  if ((!scratch && bk_cross_attention_scratch_floats(batch, sq, sk, heads, kv_heads, d) > 0) || ((uintptr_t)scratch & 15)) return BAMBOO_E_ARG;
  memset(&a, 0, sizeof(a));
  a.B = batch; a.sq = sq; a.sk = sk; a.heads = heads; a.kv_heads = kv_heads; a.d = d;
  a.q = q; a.k = k; a.v = v; a.ldq = ldq; a.ldkv = ldkv; a.kv_len = kv_len;
  a.ctx = (void*)ctx; a.ldc = ldc; a.lse = (float*)lse; a.scratch = scratch;
  return BAMBOO_OK;
}
static Matrix query_rows(const CrossDesc& a, int dtype, const void* p, int64_t ld) {
  return {p, (int64_t)a.B * a.sq, ld, (int64_t)a.heads * a.d, element_size(dtype)};
}
static Matrix key_rows(const CrossDesc& a, int dtype, const void* p, int64_t ld) {
  return {p, (int64_t)a.B * a.sk, ld, (int64_t)a.kv_heads * a.d, element_size(dtype)};
}

uint64_t bk_cross_attention_scratch_floats(int batch, int sq, int sk, int heads, int kv_heads, int d) {
  if (!cross_sizes(batch, sq, sk, heads, kv_heads, d)) return 0;
  return cross_attention_scratch_floats(batch, sq, sk, heads, kv_heads, d);
}

int bk_cross_attention_fwd(int dtype, int impl, int batch, int sq, int sk, int heads, int kv_heads, int d, const void* q,
                           int64_t ldq, const void* k, const void* v, int64_t ldkv, const int32_t* kv_len, void* ctx,
                           int64_t ldc, float* lse, float* scratch, void* stream) {
  CrossDesc a;
  const int rc = cross_desc(a, dtype, impl, batch, sq, sk, heads, kv_heads, d, q, ldq, k, v, ldkv, kv_len, ctx, ldc, lse, scratch);
  if (rc != BAMBOO_OK) return rc;
  const Matrix out = query_rows(a, dtype, ctx, ldc);
  if (overlap(query_rows(a, dtype, q, ldq), out) || overlap(key_rows(a, dtype, k, ldkv), out) || overlap(key_rows(a, dtype, v, ldkv), out))
    return BAMBOO_E_ARG;
  (void)hipGetLastError();
  return finish(launch_cross_attention_fwd((hipStream_t)stream, dtype, impl, a));
}

int bk_cross_attention_bwd(int dtype, int impl, int batch, int sq, int sk, int heads, int kv_heads, int d, const void* q,
                           int64_t ldq, const void* k, const void* v, int64_t ldkv, const int32_t* kv_len,
                           const void* ctx, int64_t ldc, const float* lse, const void* dctx, int64_t lddc, void* dq,
                           int64_t lddq, void* dk, void* dv, int64_t lddkv, float* scratch, void* stream) {
  CrossDesc a;
  const int rc = cross_desc(a, dtype, impl, batch, sq, sk, heads, kv_heads, d, q, ldq, k, v, ldkv, kv_len, ctx, ldc, lse, scratch);
  if (rc != BAMBOO_OK) return rc;
  if (!dctx || !dq || !dk || !dv || lddc < (int64_t)heads * d || lddq < (int64_t)heads * d || lddkv < (int64_t)kv_heads * d)
    return BAMBOO_E_ARG;
  for (const void* p : {dctx, (const void*)dq, (const void*)dk, (const void*)dv})
    if (!element_aligned(dtype, p)) return BAMBOO_E_ARG;
  const Matrix in[] = {query_rows(a, dtype, q, ldq), query_rows(a, dtype, ctx, ldc), query_rows(a, dtype, dctx, lddc),
                       key_rows(a, dtype, k, ldkv), key_rows(a, dtype, v, ldkv)};
  const Matrix out[] = {query_rows(a, dtype, dq, lddq), key_rows(a, dtype, dk, lddkv), key_rows(a, dtype, dv, lddkv)};
  for (const Matrix& o : out)
    for (const Matrix& i : in)
      if (overlap(i, o)) return BAMBOO_E_ARG;
  if (overlap(out[0], out[1]) || overlap(out[0], out[2]) || overlap(out[1], out[2])) return BAMBOO_E_ARG;
  a.dctx = dctx; a.lddc = lddc; a.dq = dq; a.lddq = lddq; a.dk = dk; a.dv = dv; a.lddkv = lddkv;
  (void)hipGetLastError();
  return finish(launch_cross_attention_bwd((hipStream_t)stream, dtype, impl, a));
}

// the gradient's buffer: whole elements, and either the logits' own rows or none of them
static bool bad_gradient(int dtype, int64_t rows, int V, const void* logits, int64_t ldl, const void* dlogits, int64_t ldd) {
  const int es = element_size(dtype);
  return ldd < V || !element_aligned(dtype, dlogits) || overlap({logits, rows, ldl, V, es}, {dlogits, rows, ldd, V, es}, true);
}

int bk_policy_loss(int dtype, int T, int V, const void* logits, int64_t ldl, const int32_t* labels, const uint8_t* mask,
                   const float* old_logp, const float* ref_logp, const float* adv, float clip_low, float clip_high,
                   float kl_coef, float ent_coef, float scale, float* logp, float* loss_tok, float* kl_tok,
                   float* entropy, void* dlogits, int64_t ldd, void* stream) {
  if ((dtype != 0 && dtype != 1) || T <= 0 || T > kMaxWorkgroups || V <= 0 || V > kMaxVocab || ldl < V) return BAMBOO_E_ARG;
  if (!logits || !labels || !old_logp || !adv || !logp || !loss_tok || !element_aligned(dtype, logits)) return BAMBOO_E_ARG;
  if (!(clip_low >= 0.f && clip_low <= 1.f && clip_high >= 0.f)) return BAMBOO_E_ARG;
  if (dlogits && bad_gradient(dtype, T, V, logits, ldl, dlogits, ldd)) return BAMBOO_E_ARG;
  PolicyDesc a;
  memset(&a, 0, sizeof(a));
  a.logits = logits; a.ldl = ldl; a.T = T; a.V = V; a.labels = labels; a.mask = mask; a.old_logp = old_logp; a.ref_logp = ref_logp;
  a.adv = adv; a.clip_low = clip_low; a.clip_high = clip_high; a.kl_coef = kl_coef; a.ent_coef = ent_coef; a.scale = scale;
  a.logp = logp; a.loss_tok = loss_tok; a.kl_tok = kl_tok; a.entropy = entropy; a.dlogits = dlogits; a.ldd = ldd;
  (void)hipGetLastError();
  return finish(launch_policy_loss((hipStream_t)stream, dtype, a));
}

static int preference_desc(PreferenceDesc& a, int dtype, int pairs, int seq, int V, const void* logits, int64_t ldl,
                           const int32_t* labels, const uint8_t* mask, float beta, float smoothing) {
  if ((dtype != 0 && dtype != 1) || pairs <= 0 || seq <= 0 || V <= 0 || V > kMaxVocab || ldl < V) return BAMBOO_E_ARG;
  if ((int64_t)2 * pairs * seq > kMaxWorkgroups || !logits || !labels || !element_aligned(dtype, logits)) return BAMBOO_E_ARG;
  if (!(smoothing >= 0.f && smoothing <= 1.f)) return BAMBOO_E_ARG;
  memset(&a, 0, sizeof(a));
  a.logits = logits; a.ldl = ldl; a.pairs = pairs; a.seq = seq; a.V = V; a.labels = labels; a.mask = mask; a.beta = beta;
  a.smoothing = smoothing;
  return BAMBOO_OK;
}

int bk_preference_loss_fwd(int dtype, int pairs, int seq, int V, const void* logits, int64_t ldl, const int32_t* labels,
                           const uint8_t* mask, const float* ref_logp, float beta, float smoothing, float* lse,
                           float* logp, float* logp_seq, float* margin, float* loss, double* scratch, void* stream) {
  PreferenceDesc a;
  const int rc = preference_desc(a, dtype, pairs, seq, V, logits, ldl, labels, mask, beta, smoothing);
  if (rc != BAMBOO_OK) return rc;
  if (!ref_logp || !lse || !logp || !logp_seq || !margin || !loss || !scratch || ((uintptr_t)scratch & 7)) return BAMBOO_E_ARG;
  a.ref_logp = ref_logp; a.lse = lse; a.logp = logp; a.logp_seq = logp_seq; a.margin = margin; a.loss = loss; a.scratch = scratch;
  (void)hipGetLastError();
  return finish(launch_preference_fwd((hipStream_t)stream, dtype, a));
}

int bk_preference_loss_bwd(int dtype, int pairs, int seq, int V, const void* logits, int64_t ldl, const int32_t* labels,
                           const uint8_t* mask, const float* lse, const float* margin, float beta, float smoothing,
                           float scale, void* dlogits, int64_t ldd, void* stream) {
  PreferenceDesc a;
  const int rc = preference_desc(a, dtype, pairs, seq, V, logits, ldl, labels, mask, beta, smoothing);
  if (rc != BAMBOO_OK) return rc;
  if (!lse || !margin || !dlogits || bad_gradient(dtype, (int64_t)2 * pairs * seq, V, logits, ldl, dlogits, ldd)) return BAMBOO_E_ARG;
  a.lse = (float*)lse; a.margin = (float*)margin; a.scale = scale; a.dlogits = dlogits; a.ldd = ldd;
  (void)hipGetLastError();
  return finish(launch_preference_bwd((hipStream_t)stream, dtype, a));
}

int bk_adamw_group(int dtype, int moment_bits, int n, const int64_t* numel, const float* const* g, float* const* master,
                   void* const* m, void* const* v, float* const* m_scale, float* const* v_scale, void* const* w,
                   const double* decay, double lr, double beta1, double beta2, double eps, int step, uint32_t seed,
                   void* stream) {
  if ((dtype != 0 && dtype != 1) || (moment_bits != 32 && moment_bits != 8) || n < 1 || step < 1) return BAMBOO_E_ARG;
  if (!numel || !g || !master || !m || !v || !w || !decay || (moment_bits == 8) != (m_scale && v_scale)) return BAMBOO_E_ARG;
  if ((moment_bits == 32 && (m_scale || v_scale)) || !(beta1 >= 0. && beta1 < 1.) || !(beta2 >= 0. && beta2 < 1.) || !(eps >= 0.))
    return BAMBOO_E_ARG;
  try {
    std::vector<AdamwTensor> t((size_t)n);
    std::vector<std::pair<uintptr_t, uintptr_t>> held;
    held.reserve((size_t)n);
    for (int i = 0; i < n; ++i) {
      AdamwTensor& p = t[i];
      memset(&p, 0, sizeof(p));
      p.numel = numel[i];
      if (p.numel < 0 || p.numel > kAdamwMost) return BAMBOO_E_ARG;
      if (p.numel == 0) continue;
      p.g = g[i]; p.master = master[i]; p.m = m[i]; p.v = v[i]; p.w = w[i];
      if (!p.g || !p.master || !p.m || !p.v || !p.w || !element_aligned(dtype, p.w)) return BAMBOO_E_ARG;
      uintptr_t words = (uintptr_t)p.g | (uintptr_t)p.master;
      if (moment_bits == 8) {
        p.m_scale = m_scale[i]; p.v_scale = v_scale[i];
        if (!p.m_scale || !p.v_scale) return BAMBOO_E_ARG;
        words |= (uintptr_t)p.m_scale | (uintptr_t)p.v_scale;
      } else {
        words |= (uintptr_t)p.m | (uintptr_t)p.v;
      }
      if (words & 3) return BAMBOO_E_ARG;
      held.emplace_back((uintptr_t)p.master, (uintptr_t)(p.master + p.numel));
    }
    // the same weights twice would be two steps at once on one tensor
    std::sort(held.begin(), held.end());
    for (size_t i = 1; i < held.size(); ++i)
      if (held[i].first < held[i - 1].second) return BAMBOO_E_ARG;
    AdamwHyper h = {lr, beta1, beta2, eps, step};
    (void)hipGetLastError();
    return finish(launch_adamw((hipStream_t)stream, dtype, moment_bits, h, n, t.data(), decay, seed));
  } catch (const std::bad_alloc&) {
    return BAMBOO_E_NOMEM;
  }
}

int bk_gemm_tile(int code) {
  if (!gemm_tile_code_valid(code)) return BAMBOO_E_ARG;
  return set_gemm_tile(code);
}

int bk_gemm_stages(int n) {
  if (n != 0 && (n < 2 || n > 4)) return BAMBOO_E_ARG;
  return set_gemm_stages(n);
}

}  // extern "C"
