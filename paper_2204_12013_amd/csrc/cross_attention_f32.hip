// Attention over an encoder's states in fp32 arithmetic on the matrix cores: fp32 tensors, and bf16 ones where a caller asks
// for it; any head size up to 128, any alignment.
//
// Four wavefronts own 32 rows each and share tiles of 32 streamed rows, held in LDS in fp32 with the head size padded
// by zeros to DP.  The score tile is computed transposed (streamed rows along a lane's registers, owned rows along the
// lanes), as in the bf16 kernels; v_mfma_f32_32x32x2 takes one value a lane of each operand, so register r of the
// accumulator is at once the operand of the second product: the streamed rows of its two halves are 8 (r / 4) + r % 4 and
// that plus 4, and the other operand is read for just these.  The contraction over the head size runs over feature i of
// the lower and DP / 2 + i of the upper half in step i, so that a lane's values are neighbours in LDS.
// Bound by the matrix instruction: 64 clocks for 2048 multiply-adds, a sixteenth of the bf16 one's rate (a large library
// product reaches 154 TFLOP/s).  13 x 502 x 514, 32 heads over 4 of 128: forward 518 us (106 TFLOP/s), dQ 850 us (97), dK and dV
// 1351 us (81), one wavefront a SIMD in the backward; what is missing are the steps' own chains: barrier, scores, exponentials.
#include <math.h>

#include "cross_rows.h"

namespace bamboo {

namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kMasked = -1.0e30f;
constexpr int TR = 32;     // rows of a streamed tile

__device__ __forceinline__ int acc_row(int r) { return 8 * (r >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (r & 3); }

// features c .. c+3 of a row, zero from d on; VEC: d is a multiple of 4 and the row is aligned to 4 elements
template <typename T, bool VEC>
__device__ __forceinline__ f32x4 row4(const T* row, int c, int d) {
  typedef T vec __attribute__((ext_vector_type(4)));
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if constexpr (VEC) {
    if (c < d) {
      const vec t = *(const vec*)(row + c);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = to_f32<T>(t[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + j < d) o[j] = to_f32<T>(row[c + j]);
  }
  return o;
}
// The lane's half of a row: features g * DP/2 + i, as it enters the contraction
template <typename T, int DP, bool VEC>
__device__ __forceinline__ void row_half(float (&f)[DP / 2], const T* row, bool live, int d) {
  const int g = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int i = 0; i < DP / 2; i += 4) {
    const f32x4 t = live ? row4<T, VEC>(row, g * (DP / 2) + i, d) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) f[i + j] = t[j];
  }
}
// Two tiles of 32 rows on their way to LDS: requested ahead of a step, stored behind it.
template <typename T, int DP, bool VEC>
struct TilePair {
  static constexpr int LD = DP + 4, N = DP / 32;
  f32x4 v0[N], v1[N];
  // row(i): the two rows' addresses of row i of the tile, both valid
  template <typename ROW> __device__ __forceinline__ void fetch(ROW row, int d) {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int i = threadIdx.x + u * 256, r = i / (DP / 4), c = (i % (DP / 4)) * 4;
      const T *p0, *p1;
      row(r, &p0, &p1);
      v0[u] = row4<T, VEC>(p0, c, d);
      v1[u] = row4<T, VEC>(p1, c, d);
    }
  }
  __device__ __forceinline__ void stash(float* s0, float* s1) const {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int i = threadIdx.x + u * 256, r = i / (DP / 4), c = (i % (DP / 4)) * 4;
      *(f32x4*)(s0 + r * LD + c) = v0[u];
      *(f32x4*)(s1 + r * LD + c) = v1[u];
    }
  }
};
// X Y^T of the 32 rows in LDS and the lanes' rows
template <int DP>
__device__ __forceinline__ f32x16 rows_times(const float* tile, const float (&f)[DP / 2], f32x16 acc) {
  const float* p = tile + (threadIdx.x & 31) * (DP + 4) + ((threadIdx.x & 63) >> 5) * (DP / 2);
#pragma unroll
  for (int i = 0; i < DP / 2; i += 4) {
    const f32x4 a = *(const f32x4*)(p + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], f[i + j], acc, 0, 0, 0);
  }
  return acc;
}
// out^T += X^T P: X the 32 rows in LDS, P the accumulator tile
template <int DP>
__device__ __forceinline__ void add_product(f32x16 (&out)[DP / 32], const float* tile, const f32x16& p) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const float* x = tile + acc_row(r) * (DP + 4) + (threadIdx.x & 31);
#pragma unroll
    for (int dt = 0; dt < DP / 32; ++dt) out[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[dt * 32], p[r], out[dt], 0, 0, 0);
  }
}
template <int N> __device__ __forceinline__ void clear(f32x16 (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) x[i][r] = 0.f;
}
// the lane's row of a transposed result, scaled
template <typename T, int DP, bool VEC>
__device__ __forceinline__ void store_row(T* row, const f32x16 (&x)[DP / 32], float mul, int d) {
  typedef T vec __attribute__((ext_vector_type(4)));
  const int g = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const int c = dt * 32 + 8 * a + 4 * g;
      if constexpr (VEC) {
        if (c < d) {
          vec t;
#pragma unroll
          for (int j = 0; j < 4; ++j) t[j] = from_f32<T>(x[dt][4 * a + j] * mul);
          *(vec*)(row + c) = t;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c + j < d) row[c + j] = from_f32<T>(x[dt][4 * a + j] * mul);
      }
    }
}

// -------------------------------------------------------------------------------------------- forward
template <typename T, int DP, bool VEC>
__global__ __launch_bounds__(256) void cross_fwd_f32_kernel(CrossDesc a) {
  __shared__ __attribute__((aligned(16))) float Ks[TR * (DP + 4)], Vs[TR * (DP + 4)];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 5, d = a.d;
  const CrossBlock w = cross_block(a);
  const int len = cross_len(a, w.b);
  int t0, t1;
  cross_part(len, a.splits, w.split, &t0, &t1);
  const int k_end = min(len, t1 * 64), row = w.blk * 128 + wave * 32 + (lane & 31);
  const bool live = row < a.rows;
  const CrossRow at = cross_row(a, w.kvh, live ? row : a.rows - 1);
  float q[DP / 2];
  row_half<T, DP, VEC>(q, (const T*)a.q + ((long)w.b * a.sq + at.query) * a.ldq + (long)at.head * d, live, d);
  const T* kb = (const T*)a.k + (long)w.b * a.sk * a.ldkv + (long)w.kvh * d;
  const T* vb = (const T*)a.v + (long)w.b * a.sk * a.ldkv + (long)w.kvh * d;
  const float c = rsqrtf((float)d) * kLog2e;
  f32x16 o[DP / 32];
  clear(o);
  float m = kMasked, l = 0.f;
  TilePair<T, DP, VEC> next;
  auto fetch = [&](int k0) {
    next.fetch([&](int r, const T** p0, const T** p1) {
      const long at_row = (long)min(k0 + r, len - 1) * a.ldkv;
      *p0 = kb + at_row;
      *p1 = vb + at_row;
    }, d);
  };
  if (t0 * 64 < k_end) fetch(t0 * 64);
  for (int k0 = t0 * 64; k0 < k_end; k0 += TR) {
    __syncthreads();
    next.stash(Ks, Vs);
    __syncthreads();
    if (k0 + TR < k_end) fetch(k0 + TR);
    if (w.blk * 128 + wave * 32 >= a.rows) continue;                // uniform over the wavefront
    f32x16 s = {};
    s = rows_times<DP>(Ks, q, s);
    float mx = kMasked;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = k0 + acc_row(r) < len ? s[r] : kMasked;
      mx = fmaxf(mx, s[r]);
    }
    mx = fmaxf(mx, lane_across(mx)) * c;
    if (__builtin_amdgcn_ballot_w64(mx > m) != 0) {
      const float to = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - to);
      l *= alpha;
      m = to;
#pragma unroll
      for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -m));
      l += s[r];
    }
    add_product<DP>(o, Vs, s);
  }
  l += lane_across(l);
  if (!live) return;
  if (a.splits > 1) {
    const long i = ((long)w.split * a.B * a.kv_heads + w.pair) * a.rows + row;
    store_row<float, DP, VEC>(a.part + i * d, o, 1.f, d);
    if (g == 0) {
      a.part_stats[2 * i] = m;
      a.part_stats[2 * i + 1] = l;
    }
    return;
  }
  store_row<T, DP, VEC>((T*)a.ctx + ((long)w.b * a.sq + at.query) * a.ldc + (long)at.head * d, o, l > 0.f ? 1.f / l : l, d);
  if (g == 0) a.lse[cross_stat(a, w.b, at)] = len > 0 ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// ------------------------------------------------------------------------------------------- backward
template <typename T, int DP, bool VEC>
__global__ __launch_bounds__(256, 1) void cross_dq_f32_kernel(CrossDesc a) {
  __shared__ __attribute__((aligned(16))) float Ks[TR * (DP + 4)], Vs[TR * (DP + 4)];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 5, d = a.d;
  const CrossBlock w = cross_block(a);
  const int len = cross_len(a, w.b);
  int t0, t1;
  cross_part(len, a.splits, w.split, &t0, &t1);
  const int k_end = min(len, t1 * 64), row = w.blk * 128 + wave * 32 + (lane & 31);
  const bool live = row < a.rows;
  const CrossRow at = cross_row(a, w.kvh, live ? row : a.rows - 1);
  const long tok = (long)w.b * a.sq + at.query, stat = cross_stat(a, w.b, at);
  float q[DP / 2], go[DP / 2];
  row_half<T, DP, VEC>(q, (const T*)a.q + tok * a.ldq + (long)at.head * d, live, d);
  row_half<T, DP, VEC>(go, (const T*)a.dctx + tok * a.lddc + (long)at.head * d, live, d);
  float delta = 0.f;
  {
    float of[DP / 2];
    row_half<T, DP, VEC>(of, (const T*)a.ctx + tok * a.ldc + (long)at.head * d, live, d);
#pragma unroll
    for (int i = 0; i < DP / 2; ++i) delta = fmaf(of[i], go[i], delta);
    delta += lane_across(delta);
  }
  if (live && g == 0 && w.split == 0) a.delta[stat] = delta;
  const float lse2 = a.lse[stat] * kLog2e;
  const T* kb = (const T*)a.k + (long)w.b * a.sk * a.ldkv + (long)w.kvh * d;
  const T* vb = (const T*)a.v + (long)w.b * a.sk * a.ldkv + (long)w.kvh * d;
  const float scale = rsqrtf((float)d), c = scale * kLog2e;
  f32x16 dq[DP / 32];
  clear(dq);
  TilePair<T, DP, VEC> next;
  auto fetch = [&](int k0) {
    next.fetch([&](int r, const T** p0, const T** p1) {
      const long at_row = (long)min(k0 + r, len - 1) * a.ldkv;
      *p0 = kb + at_row;
      *p1 = vb + at_row;
    }, d);
  };
  if (t0 * 64 < k_end) fetch(t0 * 64);
  for (int k0 = t0 * 64; k0 < k_end; k0 += TR) {
    __syncthreads();
    next.stash(Ks, Vs);
    __syncthreads();
    if (k0 + TR < k_end) fetch(k0 + TR);
    if (w.blk * 128 + wave * 32 >= a.rows) continue;
    f32x16 s = {}, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) dp[r] = -delta;
    s = rows_times<DP>(Ks, q, s);
    dp = rows_times<DP>(Vs, go, dp);
#pragma unroll
    for (int r = 0; r < 16; ++r)
      s[r] = k0 + acc_row(r) < len ? __builtin_amdgcn_exp2f(fmaf(s[r], c, -lse2)) * dp[r] : 0.f;
    add_product<DP>(dq, Ks, s);
  }
  if (!live) return;
  if (a.splits > 1) {
    store_row<float, DP, VEC>(a.part + w.split * a.part_stride + ((long)w.pair * a.rows + row) * d, dq, 1.f, d);
    return;
  }
  store_row<T, DP, VEC>((T*)a.dq + tok * a.lddq + (long)at.head * d, dq, scale, d);
}

// Owns keys, streams rows.
template <typename T, int DP, bool VEC>
__global__ __launch_bounds__(256, 1) void cross_dkv_f32_kernel(CrossDesc a) {
  __shared__ __attribute__((aligned(16))) float Qs[TR * (DP + 4)], Gs[TR * (DP + 4)], lse_s[TR], del_s[TR];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, d = a.d;
  const CrossBlock w = cross_block(a);
  const int len = cross_len(a, w.b);
  int t0, t1;
  cross_part(a.rows, a.splits, w.split, &t0, &t1);
  const int key0 = w.blk * 128, key = key0 + wave * 32 + (lane & 31);
  const int r_end = key0 < len ? min(a.rows, t1 * 64) : t0 * 64;    // no rows where none of the keys counts
  const bool counts = key < len;
  const long at_key = ((long)w.b * a.sk + min(key, a.sk - 1)) * a.ldkv + (long)w.kvh * d;
  float kf[DP / 2], vf[DP / 2];
  row_half<T, DP, VEC>(kf, (const T*)a.k + at_key, counts, d);
  row_half<T, DP, VEC>(vf, (const T*)a.v + at_key, counts, d);
  const float scale = rsqrtf((float)d), c = scale * kLog2e;
  f32x16 dk[DP / 32], dv[DP / 32];
  clear(dk);
  clear(dv);
  TilePair<T, DP, VEC> next;
  float lse_r = 0.f, del_r = 0.f;
  auto fetch = [&](int r0) {
    next.fetch([&](int r, const T** p0, const T** p1) {
      const CrossRow at = cross_row(a, w.kvh, min(r0 + r, a.rows - 1));
      const long tok = (long)w.b * a.sq + at.query;
      *p0 = (const T*)a.q + tok * a.ldq + (long)at.head * d;
      *p1 = (const T*)a.dctx + tok * a.lddc + (long)at.head * d;
    }, d);
    if (threadIdx.x < TR) {
      const long stat = cross_stat(a, w.b, cross_row(a, w.kvh, min(r0 + (int)threadIdx.x, a.rows - 1)));
      lse_r = a.lse[stat] * kLog2e;
      del_r = -a.delta[stat];
    }
  };
  if (t0 * 64 < r_end) fetch(t0 * 64);
  for (int r0 = t0 * 64; r0 < r_end; r0 += TR) {
    __syncthreads();
    next.stash(Qs, Gs);
    if (threadIdx.x < TR) {
      lse_s[threadIdx.x] = lse_r;
      del_s[threadIdx.x] = del_r;
    }
    __syncthreads();
    if (r0 + TR < r_end) fetch(r0 + TR);
    if (key0 + wave * 32 >= len) continue;
    f32x16 s = {}, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) dp[r] = del_s[acc_row(r)];
    s = rows_times<DP>(Qs, kf, s);
    dp = rows_times<DP>(Gs, vf, dp);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float p = __builtin_amdgcn_exp2f(fmaf(s[r], c, -lse_s[acc_row(r)]));
      s[r] = counts && r0 + acc_row(r) < a.rows ? p : 0.f;
      dp[r] = s[r] > 0.f ? dp[r] * s[r] : s[r];
    }
    add_product<DP>(dv, Gs, s);
    add_product<DP>(dk, Qs, dp);
  }
  if (key >= a.sk) return;
  if (!counts) {                                  // their probabilities are 0, but 0 times a row that is not finite is NaN
    clear(dk);
    clear(dv);
  }
  if (a.splits > 1) {
    float* out = a.part + w.split * a.part_stride + ((long)w.pair * a.sk + key) * (2 * d);
    store_row<float, DP, VEC>(out, dk, 1.f, d);
    store_row<float, DP, VEC>(out + d, dv, 1.f, d);
    return;
  }
  const long out = ((long)w.b * a.sk + key) * a.lddkv + (long)w.kvh * d;
  store_row<T, DP, VEC>((T*)a.dk + out, dk, scale, d);
  store_row<T, DP, VEC>((T*)a.dv + out, dv, 1.f, d);
}

// every row, head and buffer at a multiple of four elements
template <typename T> bool vectors(const CrossDesc& a) {
  uintptr_t bits = 0;
  for (const void* p : {a.q, a.k, a.v, (const void*)a.ctx, a.dctx, (const void*)a.dq, (const void*)a.dk, (const void*)a.dv})
    bits |= (uintptr_t)p;
  const long lds = a.ldq | a.ldkv | a.ldc | a.lddc | a.lddq | a.lddkv;
  return a.d % 4 == 0 && lds % 4 == 0 && bits % (4 * sizeof(T)) == 0;
}
enum { FWD, DQ, DKV };
template <typename T, int DP, bool VEC>
hipError_t launch(hipStream_t s, int pass, const CrossDesc& a) {
  const unsigned grid = (unsigned)(((pass == DKV ? a.sk : a.rows) + 127) / 128) * a.splits * a.B * a.kv_heads;
  const auto kern = pass == FWD ? cross_fwd_f32_kernel<T, DP, VEC>
                                : (pass == DQ ? cross_dq_f32_kernel<T, DP, VEC> : cross_dkv_f32_kernel<T, DP, VEC>);
  hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename T>
hipError_t by_size(hipStream_t s, int pass, const CrossDesc& a) {
  const bool vec = vectors<T>(a);
  if (a.d <= 32) return vec ? launch<T, 32, true>(s, pass, a) : launch<T, 32, false>(s, pass, a);
  if (a.d <= 64) return vec ? launch<T, 64, true>(s, pass, a) : launch<T, 64, false>(s, pass, a);
  if (a.d <= 96) return vec ? launch<T, 96, true>(s, pass, a) : launch<T, 96, false>(s, pass, a);
  return vec ? launch<T, 128, true>(s, pass, a) : launch<T, 128, false>(s, pass, a);
}
hipError_t by_type(hipStream_t s, int dtype, int pass, const CrossDesc& a) {
  return dtype == 1 ? by_size<bf16_t>(s, pass, a) : by_size<float>(s, pass, a);
}

}  // namespace

hipError_t launch_cross_fwd_f32(hipStream_t s, int dtype, const CrossDesc& a) { return by_type(s, dtype, FWD, a); }
hipError_t launch_cross_dq_f32(hipStream_t s, int dtype, const CrossDesc& a) { return by_type(s, dtype, DQ, a); }
hipError_t launch_cross_dkv_f32(hipStream_t s, int dtype, const CrossDesc& a) { return by_type(s, dtype, DKV, a); }

}  // namespace bamboo
