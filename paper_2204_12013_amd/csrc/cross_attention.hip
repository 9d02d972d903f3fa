// Attention over an encoder's states: which kernels run, how many parts the streamed side is cut into, and the launch that
// joins the parts.
#include <math.h>

#include "cross_rows.h"

namespace bamboo {

namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNone = -1.0e30f;     // maximum of no scores

// Row of `rows` per pair: out = sum of the parts, weighted to their common maximum.  One wavefront a row.
template <typename T>
__global__ __launch_bounds__(256) void cross_join_fwd_kernel(CrossDesc a) {
  const int lane = threadIdx.x & 63;
  const long n = (long)a.B * a.kv_heads * a.rows, i = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= n) return;
  const int pair = (int)(i / a.rows), b = pair / a.kv_heads;
  const CrossRow at = cross_row(a, pair % a.kv_heads, (int)(i % a.rows));
  // 64 parts at a time, one a lane: their maxima and sums, then their weights; the rows of eight parts are requested together
  float m = kNone, l = 0.f, o0 = 0.f, o1 = 0.f;
  const int c0 = min(lane, a.d - 1), c1 = min(lane + 64, a.d - 1);
  for (int s0 = 0; s0 < a.splits; s0 += 64) {
    const int k = min(64, a.splits - s0);
    const long p = (long)(s0 + min(lane, k - 1)) * n + i;
    float ms = a.part_stats[2 * p], ls = a.part_stats[2 * p + 1];
    if (lane >= k || ls == 0.f) {                 // no part, or one without keys
      ms = kNone;
      ls = 0.f;
    }
    const float to = fmaxf(m, wave_max(ms)), old = __builtin_amdgcn_exp2f(m - to);
    const float w = ls == 0.f ? 0.f : __builtin_amdgcn_exp2f(ms - to);
    l = l * old + wave_sum_of_products(w, ls);
    o0 *= old;
    o1 *= old;
    m = to;
    const float* row = a.part + ((long)s0 * n + i) * a.d;
    for (int s = 0; s < k; s += 8) {
      float x0[8], x1[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float* at_row = row + (long)min(s + q, k - 1) * n * a.d;
        x0[q] = at_row[c0];
        x1[q] = at_row[c1];
      }
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float wq = s + q < k ? of_lane(w, min(s + q, k - 1)) : 0.f;
        o0 = wq > 0.f ? fmaf(wq, x0[q], o0) : o0;
        o1 = wq > 0.f ? fmaf(wq, x1[q], o1) : o1;
      }
    }
  }
  l = of_lane(l, 0);
  const float inv = l > 0.f ? 1.f / l : l;
  T* out = (T*)a.ctx + ((long)b * a.sq + at.query) * a.ldc + (long)at.head * a.d;
  if (lane < a.d) out[lane] = from_f32<T>(o0 * inv);
  if (lane + 64 < a.d) out[lane + 64] = from_f32<T>(o1 * inv);
  if (lane == 0) a.lse[cross_stat(a, b, at)] = cross_len(a, b) > 0 ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// Gradients: sums of the parts in order.  A thread takes four elements and has eight parts in flight (one element and part at a
// time: 32 parts of 256 keys x 128 took 61 us); the parts are `stride` floats apart, a multiple of 4.  KEYS: dk and dv,
// otherwise dq.
template <typename T, bool KEYS>
__global__ __launch_bounds__(256) void cross_join_bwd_kernel(CrossDesc a, long n, long stride) {
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  const int per = KEYS ? a.sk : a.rows, cols = KEYS ? 2 * a.d : a.d;
  const long i = ((long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= n) return;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < a.splits; s += 8) {
    f32x4 p[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) p[q] = *(const f32x4*)(a.part + min(s + q, a.splits - 1) * stride + i);
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (s + q < a.splits) x += p[q];
  }
  const float scale = rsqrtf((float)a.d);
  long row = i / cols;
  int c = (int)(i % cols);
#pragma unroll
  for (int j = 0; j < 4; ++j, ++c) {
    if (i + j >= n) break;
    if (c == cols) {
      c = 0;
      ++row;
    }
    const int pair = (int)(row / per), r = (int)(row % per), b = pair / a.kv_heads, kvh = pair % a.kv_heads;
    if (KEYS) {
      const long out = ((long)b * a.sk + r) * a.lddkv + (long)kvh * a.d;
      if (c < a.d) ((T*)a.dk)[out + c] = from_f32<T>(x[j] * scale);
      else ((T*)a.dv)[out + c - a.d] = from_f32<T>(x[j]);
    } else {
      const CrossRow at = cross_row(a, kvh, r);
      ((T*)a.dq)[((long)b * a.sq + at.query) * a.lddq + (long)at.head * a.d + c] = from_f32<T>(x[j] * scale);
    }
  }
}
template <bool KEYS>
hipError_t join_bwd(hipStream_t s, int dtype, const CrossDesc& a) {
  const long n = (long)a.B * a.kv_heads * (KEYS ? 2L * a.sk : (long)a.rows) * a.d;
  const dim3 grid((unsigned)((n + 1023) / 1024));
  if (dtype == 1) hipLaunchKernelGGL((cross_join_bwd_kernel<bf16_t, KEYS>), grid, dim3(256), 0, s, a, n, a.part_stride);
  else hipLaunchKernelGGL((cross_join_bwd_kernel<float, KEYS>), grid, dim3(256), 0, s, a, n, a.part_stride);
  return hipGetLastError();
}

long up4(long n) { return (n + 3) / 4 * 4; }

// Parts of the streamed side (`streamed` rows) for `owned` rows of each of `pairs` problems: the number, of `least` tiles each
// at least, with the smallest time by this account.  The busiest CU gets `k` workgroups.  In bf16 two of them at a time take
// 1.6 times as long as one, each hiding the other's waits; in fp32 the four wavefronts of one keep the matrix cores busy and
// the time is k times one's.  A tile of 64 rows takes a workgroup `tile_us`.  Joining is a launch, and a part's results
// (`floats`) are written and read again at 5 TB/s.  Measured: dK and dV of 1 x 2048 x 4096, 96 heads over 8 of 128 (256
// workgroups), 1018 us as one part, 830 + 28 as two; of 8 x 512 x 333, 16 heads of 64 (384), 26 us as one, 35 + 20 as two; in
// fp32, 13 x 502 x 514, 32 heads over 4 of 128 (260, four more than CUs), 2231 us as one, 1351 + 57 as nine.
int parts(long owned, long streamed, long pairs, long floats, float tile_us, bool mfma, int least) {
  const long wgs = (owned + 127) / 128 * pairs, tiles = (streamed + 63) / 64;
  const long room = kMaxWorkgroups / wgs < 64 ? kMaxWorkgroups / wgs : 64;
  const int most = (int)(tiles / least < room ? tiles / least : room);
  int best = 1;
  float best_us = 0.f;
  for (int n = 1; n <= most || n == 1; ++n) {
    const long per = (tiles + n - 1) / n;
    if (n > 1 && (tiles + per - 1) / per != n) continue;      // the last part would be empty
    const long k = (wgs * n + 255) / 256;
    const float units = mfma ? 1.6f * (k / 2) + (k & 1) : (float)k;
    const float us = units * per * tile_us + (n > 1 ? 4.f + n * floats * 1.6e-6f : 0.f);
    if (n == 1 || us < best_us) {
      best = n;
      best_us = us;
    }
  }
  return best;
}

struct Plan {
  int fwd, dq, dkv;                       // parts
  long fwd_floats, delta, dq_floats, dkv_floats;
};
Plan plan(bool mfma, int B, int sq, int sk, int heads, int kv_heads, int d) {
  const long pairs = (long)B * kv_heads, rows = (long)sq * (heads / kv_heads);
  const long row_floats = pairs * rows * d, key_floats = 2 * pairs * (long)sk * d;
  const bool padded = d != 64 && d != 128;          // tiles through registers
  const float tile_us = mfma ? (0.4f + 0.008f * d) * (padded ? 1.6f : 1.f) : 0.5f + 0.05f * d;
  const int least = mfma ? 2 : 1;
  Plan p;
  p.fwd = parts(rows, sk, pairs, row_floats, tile_us, mfma, least);
  p.dq = parts(rows, sk, pairs, row_floats, 1.5f * tile_us, mfma, least);
  p.dkv = parts(sk, rows, pairs, key_floats, 2.f * tile_us, mfma, least);
  p.fwd_floats = p.fwd > 1 ? up4(p.fwd * row_floats) + up4(p.fwd * pairs * rows * 2) : 0;
  p.delta = up4(pairs * rows);
  p.dq_floats = p.dq > 1 ? p.dq * up4(row_floats) : 0;
  p.dkv_floats = p.dkv > 1 ? p.dkv * up4(key_floats) : 0;
  return p;
}
long floats_of(const Plan& p) {
  // the parts of one pass after the other in the same place, behind delta
  const long bwd = p.delta + (p.dq_floats > p.dkv_floats ? p.dq_floats : p.dkv_floats);
  return p.fwd_floats > bwd ? p.fwd_floats : bwd;
}
void shared_fields(CrossDesc& a) {
  a.group = a.heads / a.kv_heads;
  a.group_inv = a.group == 1 ? 0 : (unsigned)(((1ull << 32) + a.group - 1) / a.group);
  a.rows = a.sq * a.group;
}

}  // namespace

uint64_t cross_attention_scratch_floats(int B, int sq, int sk, int heads, int kv_heads, int d) {
  const long x = floats_of(plan(true, B, sq, sk, heads, kv_heads, d)), y = floats_of(plan(false, B, sq, sk, heads, kv_heads, d));
  return (uint64_t)(x > y ? x : y);
}

hipError_t launch_cross_attention_fwd(hipStream_t s, int dtype, int impl, const CrossDesc& d) {
  CrossDesc a = d;
  shared_fields(a);
  const bool mfma = impl != 1 && dtype == 1;
  if (impl == 2 && !mfma) return hipErrorNotSupported;
  const Plan p = plan(mfma, a.B, a.sq, a.sk, a.heads, a.kv_heads, a.d);
  a.splits = p.fwd;
  a.part = a.scratch;
  a.part_stats = a.scratch + up4(p.fwd * (long)a.B * a.kv_heads * a.rows * a.d);
  hipError_t e = mfma ? launch_cross_fwd_mfma(s, a) : launch_cross_fwd_f32(s, dtype, a);
  if (e != hipSuccess || a.splits == 1) return e;
  const dim3 grid((unsigned)(((long)a.B * a.kv_heads * a.rows + 3) / 4));
  if (dtype == 1) hipLaunchKernelGGL(cross_join_fwd_kernel<bf16_t>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(cross_join_fwd_kernel<float>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_cross_attention_bwd(hipStream_t s, int dtype, int impl, const CrossDesc& d) {
  CrossDesc a = d;
  shared_fields(a);
  const bool mfma = impl != 1 && dtype == 1;
  if (impl == 2 && !mfma) return hipErrorNotSupported;
  const Plan p = plan(mfma, a.B, a.sq, a.sk, a.heads, a.kv_heads, a.d);
  a.delta = a.scratch;
  a.part = a.scratch + p.delta;
  a.splits = p.dq;
  a.part_stride = p.dq_floats / p.dq;
  hipError_t e = mfma ? launch_cross_dq_mfma(s, a) : launch_cross_dq_f32(s, dtype, a);
  if (e == hipSuccess && a.splits > 1) e = join_bwd<false>(s, dtype, a);
  if (e != hipSuccess) return e;
  a.splits = p.dkv;
  a.part_stride = p.dkv_floats / p.dkv;
  e = mfma ? launch_cross_dkv_mfma(s, a) : launch_cross_dkv_f32(s, dtype, a);
  if (e == hipSuccess && a.splits > 1) e = join_bwd<true>(s, dtype, a);
  return e;
}

}  // namespace bamboo
