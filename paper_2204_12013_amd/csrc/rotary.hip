// Rotary positions: in every head, pair i of the first `rot` features is turned by the angle position * f_i,
//   (a, b) -> amplitude * (a cos - b sin, b cos + a sin),
// pairs being (i, i + rot/2) or neighbours (2i, 2i + 1).  The backward turns the other way (the map is a rotation
// times a number, so its transpose is the inverse rotation times that number).
//
// HBM-bound: every rotated element is read and written once (2048 tokens, 192 heads of 128, half of each rotated and half
// passed on, 201 MB: 44 us, 4.6 TB/s, as with other numbers of items in flight, heads to a workgroup and loops; with stores that
// bypass the caches 42 us, but the next call reads what is stored here).  A workgroup takes a few tokens and a range of heads;
// the angles' cosines and sines are formed once per token and pair, into LDS, and shared by all heads.
// Angles are products in 64 bits, reduced to one turn there: at position 10^6 a 32-bit product would be off by up to
// 0.03 rad.  The reduced angle, at most pi, is then exact to 2^-24 * pi in 32 bits.
#include <math.h>

#include "common.h"

namespace bamboo {

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotTokens = 16;      // tokens a workgroup takes at most

// K elements of storage type T, aligned to themselves
template <typename T, int K> struct Pack {
  typedef T type __attribute__((ext_vector_type(K)));
};
template <typename T> struct Pack<T, 1> { typedef T type; };
template <typename T, int K> __device__ __forceinline__ float get(const typename Pack<T, K>::type& v, int j) {
  if constexpr (K == 1) return to_f32<T>(v);
  else return to_f32<T>(v[j]);
}
template <typename T, int K> __device__ __forceinline__ void set(typename Pack<T, K>::type& v, int j, float x) {
  if constexpr (K == 1) v = from_f32<T>(x);
  else v[j] = from_f32<T>(x);
}

// An item is K pairs of one head (two vectors of K elements), or K of the elements behind `rot` that are passed on.
// FLIGHT items of a thread are requested together.
template <typename T, int K, bool NEIGHBOURS>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryDesc a) {
  typedef typename Pack<T, K>::type vec;
  constexpr int FLIGHT = 4;
  extern __shared__ __attribute__((aligned(16))) float2 turn[];     // [tokens][rot / 2]
  const int half = a.rot / 2;
  const int t0 = blockIdx.x * a.tokens, nt = min(a.tokens, a.T - t0);
  for (int i = threadIdx.x; i < nt * half; i += kRotThreads) {
    const int t = t0 + i / half;
    const int pos = a.pos != nullptr ? a.pos[t] : t % a.seq;
    const double angle = (double)pos * a.freq[i % half];
    const double r = fma(-rint(angle * 0.15915494309189533577), 6.283185307179586477, angle);
    float s, c;
    sincosf((float)r, &s, &c);
    turn[i] = make_float2(c * a.amplitude, (a.inverse ? -s : s) * a.amplitude);
  }
  __syncthreads();
  const int pairs = half / K;                                       // rotated items of a head
  const int per = pairs + (a.copy ? (a.d - a.rot) / K : 0);         // items of a head
  const int h0 = blockIdx.y * a.heads_per_wg, nh = min(a.heads_per_wg, a.heads - h0);
  const int per_token = per * nh, total = per_token * nt;
  // this thread's item as (token, head, place), moved on by kRotThreads without a division
  int tok = threadIdx.x / per_token, rest = threadIdx.x % per_token, head = rest / per, it = rest % per;
  const int dt = kRotThreads / per_token, drest = kRotThreads % per_token, dh = drest / per, di = drest % per;
  const T* x0 = (const T*)a.x + (long)t0 * a.ldx + (long)h0 * a.d;
  T* y0 = (T*)a.y + (long)t0 * a.ldy + (long)h0 * a.d;
  for (int first = threadIdx.x; first < total; first += FLIGHT * kRotThreads) {
    vec v[FLIGHT][2];
    int at[FLIGHT], token[FLIGHT], place[FLIGHT];
#pragma unroll
    for (int u = 0; u < FLIGHT; ++u) {
      token[u] = tok;
      place[u] = it;
      at[u] = head * a.d + (it < pairs ? it * K * (NEIGHBOURS ? 2 : 1) : a.rot + (it - pairs) * K);
      if (first + u * kRotThreads < total) {
        const T* p = x0 + (long)tok * a.ldx + at[u];
        v[u][0] = *(const vec*)p;
        if (it < pairs) v[u][1] = *(const vec*)(p + (NEIGHBOURS ? K : half));
      }
      it += di;
      head += dh;
      tok += dt;
      if (it >= per) { it -= per; ++head; }
      if (head >= nh) { head -= nh; ++tok; }
    }
#pragma unroll
    for (int u = 0; u < FLIGHT; ++u) {
      if (first + u * kRotThreads >= total) break;
      T* p = y0 + (long)token[u] * a.ldy + at[u];
      if (place[u] < pairs) {
        const float2* cs = turn + token[u] * half + place[u] * K;
        vec o0, o1;
#pragma unroll
        for (int j = 0; j < K; ++j) {
          const float2 w = cs[j];
          // neighbours: elements 2j, 2j + 1 of the 2K in a row
          const int p0 = NEIGHBOURS ? (2 * j) % K : j, p1 = NEIGHBOURS ? (2 * j + 1) % K : j;
          const int w0 = NEIGHBOURS ? (2 * j) / K : 0, w1 = NEIGHBOURS ? (2 * j + 1) / K : 1;
          const float e = get<T, K>(v[u][w0], p0), f = get<T, K>(v[u][w1], p1);
          set<T, K>(w0 ? o1 : o0, p0, e * w.x - f * w.y);
          set<T, K>(w1 ? o1 : o0, p1, f * w.x + e * w.y);
        }
        *(vec*)p = o0;
        *(vec*)(p + (NEIGHBOURS ? K : half)) = o1;
      } else {
        *(vec*)p = v[u][0];
      }
    }
  }
}

template <typename T, int K>
hipError_t rotary_launch(hipStream_t s, RotaryDesc a) {
  const int per = a.rot / 2 / K + (a.copy ? (a.d - a.rot) / K : 0);
  // about four items in flight for every thread; wide rows of few tokens are split over their heads
  const long row = (long)a.heads * per;
  a.tokens = (int)(row >= 1024 ? 1 : (1024 + row - 1) / row);
  if (a.tokens > kRotTokens) a.tokens = kRotTokens;
  while (a.tokens > 1 && (a.T + a.tokens - 1) / a.tokens < 512) a.tokens /= 2;
  while (a.tokens < kRotTokens && (a.T + (long)a.tokens - 1) / a.tokens > kMaxWorkgroups) ++a.tokens;
  const int blocks = (a.T + a.tokens - 1) / a.tokens;
  int parts = 1;
  while (blocks * parts < 512 && row / (parts * 2) >= kRotThreads) parts *= 2;
  if (parts > a.heads) parts = a.heads;
  a.heads_per_wg = (a.heads + parts - 1) / parts;
  const dim3 grid(blocks, (a.heads + a.heads_per_wg - 1) / a.heads_per_wg);
  const size_t lds = (size_t)a.tokens * (a.rot / 2) * sizeof(float2);
  const auto kern = a.neighbours ? rotary_kernel<T, K, true> : rotary_kernel<T, K, false>;
  hipLaunchKernelGGL(kern, grid, dim3(kRotThreads), lds, s, a);
  return hipGetLastError();
}

template <typename T, int MAXK>
hipError_t rotary_choose(hipStream_t s, const RotaryDesc& a) {
  // vectors of 16 bytes where every row, head and half starts at one; pairs of 2 elements or single ones otherwise
  auto fits = [&](int k) {
    const long m = (long)k * sizeof(T);
    auto at = [&](const void* p) { return (uintptr_t)p % m == 0; };
    return (a.rot / 2) % k == 0 && a.d % k == 0 && a.ldx % k == 0 && a.ldy % k == 0 && at(a.x) && at(a.y);
  };
  if (fits(MAXK)) return rotary_launch<T, MAXK>(s, a);
  if (fits(2)) return rotary_launch<T, 2>(s, a);
  return rotary_launch<T, 1>(s, a);
}

}  // namespace

hipError_t launch_rotary(hipStream_t s, int dtype, const RotaryDesc& a) {
  return dtype == 1 ? rotary_choose<bf16_t, 8>(s, a) : rotary_choose<float, 4>(s, a);
}

}  // namespace bamboo
