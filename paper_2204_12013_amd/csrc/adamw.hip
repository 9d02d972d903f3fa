// AdamW on many tensors at once, moments in 32 or in 8 bits:
//   m <- b1 m + (1-b1) g,  v <- b2 v + (1-b2) g^2,
//   w <- w (1 - lr decay) - lr (m / (1-b1^t)) / (sqrt(v / (1-b2^t)) + eps)
// on fp32 master weights, with the storage copy of the new weights rewritten in the same pass.
//
// HBM-bound: per parameter 28 bytes of gradient, master weight and moments and the storage copy, or 16 + 1/16 with
// moments in 8 bits.  One launch takes up to kAdamwTensors tensors, whose descriptors travel in the kernel's arguments
// (nothing on the device has to outlive the call, and a captured graph holds its own copy); a workgroup finds its tensor
// with one load per lane and a ballot.  75.6 M parameters in 72 tensors: 382 us, 5.9 TB/s (two groups of 256 a wavefront 427 us,
// storage weights kept in the caches 402 us); 184 M with moments in 8 bits: 556 to 632 us, 5.3 to 6.0 TB/s (codes made by comparisons and shifts
// 658 us: the arithmetic was as long as the traffic).
//
// 8 bits: blocks of 256 elements share a scale (largest / 448) and each element is an e4m3 code, value = code * scale.
// The second moment is held as its root: the codes span a factor of 2^17.8, so its own range is squared.  A wavefront owns
// a block, four elements a lane.  The second moment moves by a thousandth of its way a step, less than half the distance
// to the next code (1/16 to 1/32 of the value), so rounding to the nearest would keep it where it is for good; both
// go up or down with the probability that keeps the mean, by 16 bits of a hash of (seed, step, tensor, element): the
// same bits wherever the step runs.  A root that is not zero never becomes zero, which would make the next step huge.
// The step itself uses the moments before they are rounded.
#include <math.h>

#include "common.h"

namespace bamboo {

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;

constexpr int kGroups = 1;                        // groups of 256 elements a wavefront takes
constexpr int kPerWg = 4 * kGroups * 256;
static_assert(kAdamwMost == kMaxWorkgroups * kPerWg, "a tensor is one launch's at most");

template <bool STREAM> __device__ __forceinline__ f32x4 load4(const float* p) {
  return STREAM ? __builtin_nontemporal_load((const f32x4*)p) : *(const f32x4*)p;
}
template <bool STREAM> __device__ __forceinline__ void store4(float* p, const f32x4& v) {
  if (STREAM) __builtin_nontemporal_store(v, (f32x4*)p);
  else *(f32x4*)p = v;
}

// A group's 256 elements: element j of a lane is at 4 lane + j where they are moved as vectors, at 64 j + lane where the
// tensor is not aligned or ends inside the group.
template <bool STREAM> __device__ __forceinline__ f32x4 get4(const float* p, bool vec, int lane, int left) {
  if (vec) return load4<STREAM>(p + 4 * lane);
  f32x4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = 64 * j + lane < left ? p[64 * j + lane] : 0.f;
  return v;
}
template <bool STREAM> __device__ __forceinline__ void put4(float* p, const f32x4& v, bool vec, int lane, int left) {
  if (vec) return store4<STREAM>(p + 4 * lane, v);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (64 * j + lane < left) p[64 * j + lane] = v[j];
}
template <bool STREAM> __device__ __forceinline__ void put_storage(float* p, const f32x4& v, bool vec, int lane, int left) {
  put4<STREAM>(p, v, vec, lane, left);
}
template <bool STREAM> __device__ __forceinline__ void put_storage(bf16_t* p, const f32x4& v, bool vec, int lane, int left) {
  if (vec) {
    bf16x4 t;
#pragma unroll
    for (int j = 0; j < 4; ++j) t[j] = (bf16_t)v[j];
    if (STREAM) __builtin_nontemporal_store(t, (bf16x4*)(p + 4 * lane));
    else *(bf16x4*)(p + 4 * lane) = t;
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (64 * j + lane < left) p[64 * j + lane] = (bf16_t)v[j];
}

__device__ __forceinline__ unsigned get_codes(const unsigned char* p, bool vec, int lane, int left) {
  if (vec) return *(const unsigned*)(p + 4 * lane);
  unsigned c = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (64 * j + lane < left) c |= (unsigned)p[64 * j + lane] << (8 * j);
  return c;
}
__device__ __forceinline__ void put_codes(unsigned char* p, unsigned c, bool vec, int lane, int left) {
  if (vec) {
    *(unsigned*)(p + 4 * lane) = c;
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (64 * j + lane < left) p[64 * j + lane] = (unsigned char)(c >> (8 * j));
}
__device__ __forceinline__ f32x4 decode(unsigned c, float scale) {
  f32x4 v;
  v[0] = __builtin_amdgcn_cvt_f32_fp8((int)c, 0) * scale;
  v[1] = __builtin_amdgcn_cvt_f32_fp8((int)c, 1) * scale;
  v[2] = __builtin_amdgcn_cvt_f32_fp8((int)c, 2) * scale;
  v[3] = __builtin_amdgcn_cvt_f32_fp8((int)c, 3) * scale;
  return v;
}
// An integer hash of 32 bits: shifts and multipliers are a published set, found by a search for the least bias between input and
// output bits (C. Wellons, "Prospecting for Hash Functions", 2018).
__host__ __device__ __forceinline__ unsigned mix(unsigned x) {
  x ^= x >> 16;
  x *= 0x7feb352du;
  x ^= x >> 15;
  x *= 0x846ca68bu;
  return x ^ (x >> 16);
}

// |x| inv, at most 448, moved to one of the two codes around it: up where the part beyond the lower one and `up` / 65536 (plus
// half of that unit) make a whole step, codes being 2^(e-3) apart in [2^e, 2^(e+1)) and 2^-9 below 2^-6.  The conversion
// adds 20 bits behind the code's last, of which these are the first 17; NaN stays NaN, and so does an infinite x, whose block's
// inv is 0.
__device__ __forceinline__ float scaled(float x, float inv) {
  const float q = x * inv;
  return q == q ? fminf(fmaxf(q, -448.f), 448.f) : q;
}
// a block whose largest is infinite has NaN for its scale: every code of it is worth NaN, the smallest root's too
__device__ __forceinline__ float scale_of(float top) { return top < INFINITY ? top * (1.f / 448.f) : NAN; }
template <int J> __device__ __forceinline__ int put_code(float q, unsigned up, int c) {
  return __builtin_amdgcn_cvt_sr_fp8_f32(q, (int)(up << 16 | 0x8000u), c, J);
}

template <typename T, int BITS, bool STREAM>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwBatch a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // this workgroup's tensor: the last whose first workgroup is not behind it
  const bool here = lane < a.n && a.first_wg[min(lane, kAdamwTensors - 1)] <= (int)blockIdx.x;
  const int k = __popcll(__ballot(here)) - 1;
  const AdamwTensor& p = a.t[k];
  const long start = (long)((int)blockIdx.x - a.first_wg[k]) * kPerWg + wave * (kGroups * 256);
  const long n = p.numel;
  f32x4 g[kGroups], w[kGroups], m[kGroups], v[kGroups];
  bool vec[kGroups];
  int left[kGroups];
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    const long at = start + u * 256;
    left[u] = (int)min(256L, n - at);
    if (left[u] <= 0) continue;
    vec[u] = p.aligned && left[u] == 256;
    g[u] = get4<STREAM>(p.g + at, vec[u], lane, left[u]);
    if (BITS == 32) {
      m[u] = get4<STREAM>((const float*)p.m + at, vec[u], lane, left[u]);
      v[u] = get4<STREAM>((const float*)p.v + at, vec[u], lane, left[u]);
    } else {
      m[u] = decode(get_codes((const unsigned char*)p.m + at, vec[u], lane, left[u]), p.m_scale[at >> 8]);
      v[u] = decode(get_codes((const unsigned char*)p.v + at, vec[u], lane, left[u]), p.v_scale[at >> 8]);
      v[u] *= v[u];
    }
    w[u] = get4<STREAM>(p.master + at, vec[u], lane, left[u]);
  }
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    const long at = start + u * 256;
    if (left[u] <= 0) continue;
    f32x4 root;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[u][j] = a.beta1 * m[u][j] + a.not_beta1 * g[u][j];
      v[u][j] = a.beta2 * v[u][j] + a.not_beta2 * g[u][j] * g[u][j];
      root[j] = sqrtf(v[u][j]);
      // all that is taken off first: 1 - lr decay in 32 bits would be off by up to 2^-25, part of a decay of 10^-6
      w[u][j] -= fmaf(w[u][j], p.lr_decay, a.lr_c1 * m[u][j] / fmaf(root[j], a.root_c2, a.eps));
    }
    put4<STREAM>(p.master + at, w[u], vec[u], lane, left[u]);
    put_storage<STREAM>((T*)p.w + at, w[u], vec[u], lane, left[u]);
    if (BITS == 32) {
      put4<STREAM>((float*)p.m + at, m[u], vec[u], lane, left[u]);
      put4<STREAM>((float*)p.v + at, v[u], vec[u], lane, left[u]);
      continue;
    }
    float top_m = 0.f, top_v = 0.f;                                    // elements behind the end are 0
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      top_m = fmaxf(top_m, fabsf(m[u][j]));
      top_v = fmaxf(top_v, root[j]);
    }
    top_m = wave_max(top_m);
    top_v = wave_max(top_v);
    // a block with nothing above 1e-30 becomes zeros: 448 / top would leave the range
    const float inv_m = top_m > 1e-30f ? 448.f / top_m : 0.f, inv_v = top_v > 1e-30f ? 448.f / top_v : 0.f;
    unsigned h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned i = (unsigned)at + (vec[u] ? 4 * lane + j : 64 * j + lane);
      h[j] = mix(i ^ p.key);
      m[u][j] = scaled(m[u][j], inv_m);
      root[j] = scaled(root[j], inv_v);
    }
    int cm = put_code<0>(m[u][0], h[0], 0), cv = put_code<0>(root[0], h[0] >> 16, 0);
    cm = put_code<1>(m[u][1], h[1], cm), cv = put_code<1>(root[1], h[1] >> 16, cv);
    cm = put_code<2>(m[u][2], h[2], cm), cv = put_code<2>(root[2], h[2] >> 16, cv);
    cm = put_code<3>(m[u][3], h[3], cm), cv = put_code<3>(root[3], h[3] >> 16, cv);
    // a root that is not zero has the smallest code at least; it is a code's last bit
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (v[u][j] > 0.f && ((unsigned)cv >> (8 * j) & 0xffu) == 0) cv |= 1 << (8 * j);
    put_codes((unsigned char*)p.m + at, (unsigned)cm, vec[u], lane, left[u]);
    put_codes((unsigned char*)p.v + at, (unsigned)cv, vec[u], lane, left[u]);
    if (lane == 0) {
      p.m_scale[at >> 8] = scale_of(top_m);
      p.v_scale[at >> 8] = scale_of(top_v);
    }
  }
}

template <typename T, int BITS>
hipError_t adamw_launch(hipStream_t s, const AdamwBatch& b, int wgs, bool stream) {
  const auto kern = stream ? adamw_kernel<T, BITS, true> : adamw_kernel<T, BITS, false>;
  hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(256), 0, s, b);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_adamw(hipStream_t s, int dtype, int bits, const AdamwHyper& h, int n, const AdamwTensor* t, const double* decay,
                        uint32_t seed) {
  AdamwBatch b;
  b.beta1 = (float)h.beta1;
  b.beta2 = (float)h.beta2;
  b.not_beta1 = (float)(1. - h.beta1);
  b.not_beta2 = (float)(1. - h.beta2);
  b.eps = (float)h.eps;
  b.lr_c1 = (float)(h.lr / (1. - pow(h.beta1, (double)h.step)));
  b.root_c2 = (float)sqrt(1. / (1. - pow(h.beta2, (double)h.step)));
  long total = 0;
  for (int i = 0; i < n; ++i) total += t[i].numel;
  const bool stream = streams_past_cache(total * ((bits == 32 ? 28 : 16) + (dtype == 1 ? 2 : 4)));
  const unsigned run = mix(seed + (unsigned)h.step * 0x9e3779b9u);
  int i = 0;
  while (i < n) {
    b.n = 0;
    long wgs = 0;
    for (; i < n && b.n < kAdamwTensors; ++i) {
      if (t[i].numel == 0) continue;
      const long need = (t[i].numel + kPerWg - 1) / kPerWg;
      if (b.n > 0 && wgs + need > kMaxWorkgroups) break;
      AdamwTensor& p = b.t[b.n++];
      p = t[i];
      b.first_wg[b.n - 1] = (int)wgs;
      p.lr_decay = (float)(h.lr * decay[i]);
      p.key = mix(run + (unsigned)i * 0x85ebca6bu);
      uintptr_t at = (uintptr_t)p.g | (uintptr_t)p.master;
      at |= bits == 32 ? (uintptr_t)p.m | (uintptr_t)p.v : ((uintptr_t)p.m | (uintptr_t)p.v) << 2;
      at |= dtype == 1 ? (uintptr_t)p.w << 1 : (uintptr_t)p.w;
      p.aligned = (at & 15) == 0;
      wgs += need;
    }
    if (b.n == 0) break;
    const hipError_t e = dtype == 1 ? (bits == 32 ? adamw_launch<bf16_t, 32>(s, b, (int)wgs, stream)
                                                  : adamw_launch<bf16_t, 8>(s, b, (int)wgs, stream))
                                    : (bits == 32 ? adamw_launch<float, 32>(s, b, (int)wgs, stream)
                                                  : adamw_launch<float, 8>(s, b, (int)wgs, stream));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace bamboo
