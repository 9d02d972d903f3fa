// Losses on the log-probability of given tokens, from the logits [T, V] of the head: a clipped policy loss with a KL
// and an entropy term, its gradient in the same pass, and a preference loss over pairs of sequences.
//
// With z a row of logits, s = sum_v exp(z_v - max), p_v = exp(z_v - max) / s:
//   logp = (z_y - max) - log s,   H = -sum_v p_v log p_v = log s - (sum_v exp(z_v - max) (z_v - max)) / s
// A loss L(logp, H) = F(logp) - e H has the gradient  dL/dz_v = c ([v = y] - p_v) + e p_v (log p_v + H),  c = F'(logp).
//
// Bound by the traffic of the logits: the policy loss reads them once and writes the gradient once, which takes the row
// on chip.  It is held in registers, in the storage type: a workgroup of 256 to 1024 threads requests its whole row at
// once (up to 16 vectors of 16 bytes a thread), which also is what keeps enough loads in flight.  Rows beyond that are
// read again.  All sums are in 32 bits, in a fixed order.
#include <math.h>

#include <type_traits>

#include "common.h"

namespace bamboo {

namespace {

// exp(t) for t <= 0: the product with log2 e in two parts, whose rounding would otherwise shift every term the same way
constexpr float kL2e = 1.4426950408889634f, kL2eRest = 1.9259629911266175e-8f;
__device__ __forceinline__ float exp_of(float t) { return __builtin_amdgcn_exp2f(fmaf(t, kL2eRest, t * kL2e)); }

// 16 bytes of a row, at any alignment of an element (the rows of a vocabulary that divides by nothing start anywhere)
template <typename T> struct Chunk;
template <> struct Chunk<bf16_t> {
  static constexpr int N = 8;
  typedef bf16_t type __attribute__((ext_vector_type(8)));
  typedef bf16_t loose __attribute__((ext_vector_type(8), aligned(2)));
};
template <> struct Chunk<float> {
  static constexpr int N = 4;
  typedef float type __attribute__((ext_vector_type(4)));
  typedef float loose __attribute__((ext_vector_type(4), aligned(4)));
};
template <typename T> __device__ __forceinline__ typename Chunk<T>::type load_chunk(const T* row, int v, int V) {
  if (v + Chunk<T>::N <= V) return *(const typename Chunk<T>::loose*)(row + v);
  typename Chunk<T>::type x;
#pragma unroll
  for (int j = 0; j < Chunk<T>::N; ++j) x[j] = v + j < V ? row[v + j] : (T)(-INFINITY);    // adds nothing
  return x;
}
template <typename T> __device__ __forceinline__ void store_chunk(T* row, int v, int V, typename Chunk<T>::type x) {
  if (v + Chunk<T>::N <= V) {
    *(typename Chunk<T>::loose*)(row + v) = x;
    return;
  }
#pragma unroll
  for (int j = 0; j < Chunk<T>::N; ++j)
    if (v + j < V) row[v + j] = x[j];
}

template <int NT> __device__ __forceinline__ float block_max(float v, float* red) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) v = fmaxf(v, red[w]);
  return v;
}
template <int NT> __device__ __forceinline__ void block_sum2(float* a, float* b, float* red) {
  const float x = wave_sum(*a), y = wave_sum(*b);
  if ((threadIdx.x & 63) == 0) {
    red[threadIdx.x >> 6] = x;
    red[NT / 64 + (threadIdx.x >> 6)] = y;
  }
  __syncthreads();
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    s += red[w];
    t += red[NT / 64 + w];
  }
  *a = s;
  *b = t;
}
__device__ __forceinline__ int clamp_label(int id, int V) { return id < 0 ? 0 : (id >= V ? V - 1 : id); }

// What a row's pass leaves: its maximum (0 in the place of -inf), the sum and its log, logp of the label, entropy.
struct RowStats { float top, sum, log_s, at_label, logp, entropy; };

// NC > 0: the row lies in registers, NC chunks a thread.  NC = 0: it is read as often as it is needed.
// A NaN or +inf in a row, or a row of -inf alone, makes its results NaN; other -inf add nothing.
template <typename T, int NT, int NC, bool ENT>
struct RowPass {
  typedef typename Chunk<T>::type vec;
  static constexpr int E = Chunk<T>::N, HELD = NC > 0 ? NC : 1;
  vec x[HELD];
  __device__ __forceinline__ static int place(int c) { return (c * NT + (int)threadIdx.x) * E; }
  __device__ __forceinline__ RowStats run(const T* row, int V, int label, float* red) {
    const float at_label = to_f32<T>(row[label]);
    float m = -INFINITY, s = 0.f, w = 0.f;
    bool bad = false;
    if constexpr (NC > 0) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (place(c) < V) x[c] = load_chunk<T>(row, place(c), V);
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (place(c) < V)
#pragma unroll
          for (int j = 0; j < E; ++j) m = fmaxf(m, to_f32<T>(x[c][j]));
      m = block_max<NT>(m, red);
      const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (place(c) < V) add(x[c], from, &s, &w);
      block_sum2<NT>(&s, &w, red + NT / 64);
      m = from;
    } else {
      for (int c0 = 0; place(c0) < V; c0 += 4) {
        vec y[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (place(c0 + q) < V) y[q] = load_chunk<T>(row, place(c0 + q), V);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (place(c0 + q) >= V) break;
          float top = m;
#pragma unroll
          for (int j = 0; j < E; ++j) top = fmaxf(top, to_f32<T>(y[q][j]));
          if (top > m) {
            const float away = m - top, by = exp_of(away);
            if (ENT) w = by > 0.f ? by * (w + away * s) : 0.f;    // 0 * -inf is 0 here; a NaN is in s too
            s *= by;
            m = top;
          }
          add(y[q], m == -INFINITY ? 0.f : m, &s, &w);
        }
      }
      const float top = block_max<NT>(m, red);
      const float from = top == -INFINITY ? 0.f : top;
      const float away = m - from, by = exp_of(away);
      if (m == -INFINITY) {
        bad = s != 0.f;                                           // NaN among -inf
        s = w = bad ? NAN : 0.f;
      } else {
        if (ENT) w = by > 0.f ? by * (w + away * s) : 0.f;
        s *= by;
      }
      block_sum2<NT>(&s, &w, red + NT / 64);
      m = from;
    }
    RowStats r;
    r.top = m;
    r.sum = s;
    r.at_label = at_label;
    r.log_s = s > 0.f ? logf(s) : NAN;                            // a row of -inf alone, or a NaN in it
    r.logp = (at_label - m) - r.log_s;
    r.entropy = ENT ? r.log_s - w / s : 0.f;
    return r;
  }
  // sums of exp(z - from) and, for the entropy, of exp(z - from) (z - from)
  __device__ __forceinline__ static void add(const vec& v, float from, float* s, float* w) {
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const float t = to_f32<T>(v[j]) - from, e = exp_of(t);
      *s += e;
      if (ENT) *w += e > 0.f ? e * t : 0.f;                       // 0 * -inf is 0 here
    }
  }
};

// d = scale * (coef * [v = label] + p_v * (ent * (log p_v + H) - coef))
template <typename T, int NT, int NC, bool ENT>
__device__ __forceinline__ void write_gradient(RowPass<T, NT, NC, ENT>& pass, const T* row, T* out, int V, int label,
                                               const RowStats& r, float coef, float ent, float scale) {
  typedef typename Chunk<T>::type vec;
  constexpr int E = Chunk<T>::N;
  auto one = [&](int v, const vec& x) {
    vec o;
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const float lp = (to_f32<T>(x[j]) - r.top) - r.log_s;
      const float p = exp_of(lp);
      float k = -coef;
      if (ENT) k = p > 0.f ? fmaf(ent, lp + r.entropy, -coef) : -coef;
      const float hit = v + j == label ? coef : 0.f;
      o[j] = from_f32<T>(fmaf(p, k, hit) * scale);
    }
    store_chunk<T>(out, v, V, o);
  };
  if constexpr (NC > 0) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int v = pass.place(c);
      if (v < V) one(v, pass.x[c]);
    }
  } else {
    for (int v = threadIdx.x * E; v < V; v += NT * E) one(v, load_chunk<T>(row, v, V));
  }
}

template <typename T, int NT>
__device__ __forceinline__ void write_zeros(T* out, int V) {
  typename Chunk<T>::type o;
#pragma unroll
  for (int j = 0; j < Chunk<T>::N; ++j) o[j] = (T)0.f;
  for (int v = threadIdx.x * Chunk<T>::N; v < V; v += NT * Chunk<T>::N) store_chunk<T>(out, v, V, o);
}

// One workgroup per token.
template <typename T, int NT, int NC, bool ENT>
__global__ __launch_bounds__(NT) void policy_loss_kernel(PolicyDesc a) {
  __shared__ float red[3 * NT / 64];
  const long t = blockIdx.x;
  T* out = a.dlogits != nullptr ? (T*)a.dlogits + t * a.ldd : nullptr;
  if (a.mask != nullptr && a.mask[t] == 0) {          // uniform over the workgroup: nothing of the row is read
    if (out != nullptr) write_zeros<T, NT>(out, a.V);
    if (threadIdx.x == 0) {
      a.logp[t] = 0.f;
      a.loss_tok[t] = 0.f;
      if (a.kl_tok != nullptr) a.kl_tok[t] = 0.f;
      if (a.entropy != nullptr) a.entropy[t] = 0.f;
    }
    return;
  }
  const T* row = (const T*)a.logits + t * a.ldl;
  const int label = clamp_label(a.labels[t], a.V);
  const float old = a.old_logp[t], adv = a.adv[t], ref = a.ref_logp != nullptr ? a.ref_logp[t] : 0.f;
  RowPass<T, NT, NC, ENT> pass;
  const RowStats r = pass.run(row, a.V, label, red);
  const float ratio = expf(r.logp - old);
  const float free = ratio * adv, held = fminf(fmaxf(ratio, 1.f - a.clip_low), 1.f + a.clip_high) * adv;
  // the smaller of the two counts; a ratio or advantage that is NaN stays one
  const bool counts = !(free > held);
  float loss = -(counts ? free : held), coef = counts ? -free : 0.f, kl = 0.f;
  if (a.ref_logp != nullptr) {
    const float away = ref - r.logp, grown = expm1f(away);
    kl = grown - away;
    loss = fmaf(a.kl_coef, kl, loss);
    coef = fmaf(-a.kl_coef, grown, coef);
  }
  if (ENT) loss = fmaf(-a.ent_coef, r.entropy, loss);
  if (threadIdx.x == 0) {
    a.logp[t] = r.logp;
    a.loss_tok[t] = loss;
    if (a.kl_tok != nullptr) a.kl_tok[t] = kl;
    if (ENT && a.entropy != nullptr) a.entropy[t] = r.entropy;
  }
  if (out != nullptr) write_gradient<T, NT, NC, ENT>(pass, row, out, a.V, label, r, coef, a.ent_coef, a.scale);
}

// lse and the label's log-probability of every token that counts (0 for the others).  The latter in 64 bits too: the margin
// is a small difference of two sums over sequences, and roundings of each term, a few 10^-7, would be most of its error.
template <typename T, int NT, int NC>
__global__ __launch_bounds__(NT) void token_logp_kernel(PreferenceDesc a) {
  __shared__ float red[3 * NT / 64];
  const long t = blockIdx.x;
  if (a.mask != nullptr && a.mask[t] == 0) {
    if (threadIdx.x == 0) {
      a.lse[t] = a.logp[t] = 0.f;
      a.scratch[t] = 0.;
    }
    return;
  }
  RowPass<T, NT, NC, false> pass;
  const RowStats r = pass.run((const T*)a.logits + t * a.ldl, a.V, clamp_label(a.labels[t], a.V), red);
  if (threadIdx.x == 0) {
    a.lse[t] = r.top + r.log_s;
    a.logp[t] = r.logp;
    a.scratch[t] = ((double)r.at_label - r.top) - (r.sum > 0.f ? log((double)r.sum) : NAN);
  }
}

// log(1 + exp(x)) without overflow
__device__ __forceinline__ double softplus(double x) { return x > 0 ? x + log1p(exp(-x)) : log1p(exp(x)); }

// Per pair: sums of both sequences' log-probabilities (64 bits, fixed order), margin and loss.
__global__ __launch_bounds__(256) void pair_loss_kernel(PreferenceDesc a) {
  __shared__ double red[2][256];
  const int i = blockIdx.x;
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const double* lp = a.scratch + ((long)side * a.pairs + i) * a.seq;
    double s = 0.;
    for (int t = threadIdx.x; t < a.seq; t += 256) s += lp[t];
    red[side][threadIdx.x] = s;
  }
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o)
#pragma unroll
      for (int side = 0; side < 2; ++side) red[side][threadIdx.x] += red[side][threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    const double c = red[0][0], r = red[1][0];
    const double margin = (double)a.beta * ((c - a.ref_logp[i]) - (r - a.ref_logp[a.pairs + i]));
    a.logp_seq[i] = (float)c;
    a.logp_seq[a.pairs + i] = (float)r;
    a.margin[i] = (float)margin;
    a.loss[i] = (float)((1. - (double)a.smoothing) * softplus(-margin) + (double)a.smoothing * softplus(margin));
  }
}

// dlogits = scale * dL/dlogp_seq * ([v = label] - p), dL/dlogp_seq = +-beta (sigmoid(margin) - (1 - smoothing))
template <typename T>
__global__ __launch_bounds__(256) void preference_bwd_kernel(PreferenceDesc a) {
  typedef typename Chunk<T>::type vec;
  constexpr int E = Chunk<T>::N, AHEAD = 4;
  const long t = blockIdx.x;
  T* out = (T*)a.dlogits + t * a.ldd;
  if (a.mask != nullptr && a.mask[t] == 0) {
    write_zeros<T, 256>(out, a.V);
    return;
  }
  const T* row = (const T*)a.logits + t * a.ldl;
  const int label = clamp_label(a.labels[t], a.V);
  const int seq = (int)(t / a.seq), pair = seq < a.pairs ? seq : seq - a.pairs;
  const double g = 1. / (1. + exp(-(double)a.margin[pair])) - (1. - (double)a.smoothing);
  const float coef = (float)((seq < a.pairs ? g : -g) * (double)a.beta * (double)a.scale);
  const float lse = a.lse[t];
  for (int v0 = threadIdx.x * E; v0 < a.V; v0 += AHEAD * 256 * E) {
    vec x[AHEAD];
#pragma unroll
    for (int q = 0; q < AHEAD; ++q)
      if (v0 + q * 256 * E < a.V) x[q] = load_chunk<T>(row, v0 + q * 256 * E, a.V);
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      const int v = v0 + q * 256 * E;
      if (v >= a.V) break;
      vec o;
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const float p = exp_of(to_f32<T>(x[q][j]) - lse);
        o[j] = from_f32<T>(coef * ((v + j == label ? 1.f : 0.f) - p));
      }
      store_chunk<T>(out, v, a.V, o);
    }
  }
}

// Calls go(threads, chunks) with the smallest workgroup and number of chunks a thread that hold V elements of T.
template <typename T, typename GO>
hipError_t by_row_length(int V, GO go) {
  const int chunks = (V + Chunk<T>::N - 1) / Chunk<T>::N;
  if (chunks <= 256) return go(std::integral_constant<int, 256>(), std::integral_constant<int, 1>());
  if (chunks <= 512) return go(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
  if (chunks <= 1024) return go(std::integral_constant<int, 256>(), std::integral_constant<int, 4>());
  if (chunks <= 2048) return go(std::integral_constant<int, 256>(), std::integral_constant<int, 8>());
  if (chunks <= 4096) return go(std::integral_constant<int, 512>(), std::integral_constant<int, 8>());
  if (chunks <= 8192) return go(std::integral_constant<int, 1024>(), std::integral_constant<int, 8>());
  if (chunks <= 16384) return go(std::integral_constant<int, 1024>(), std::integral_constant<int, 16>());
  return go(std::integral_constant<int, 1024>(), std::integral_constant<int, 0>());
}

template <typename T>
hipError_t policy_launch(hipStream_t s, const PolicyDesc& a) {
  return by_row_length<T>(a.V, [&](auto nt, auto nc) {
    constexpr int NT = decltype(nt)::value, NC = decltype(nc)::value;
    const auto kern = a.entropy != nullptr || a.ent_coef != 0.f ? policy_loss_kernel<T, NT, NC, true>
                                                                : policy_loss_kernel<T, NT, NC, false>;
    hipLaunchKernelGGL(kern, dim3((unsigned)a.T), dim3(NT), 0, s, a);
    return hipGetLastError();
  });
}
template <typename T>
hipError_t token_logp_launch(hipStream_t s, const PreferenceDesc& a, unsigned rows) {
  return by_row_length<T>(a.V, [&](auto nt, auto nc) {
    constexpr int NT = decltype(nt)::value, NC = decltype(nc)::value;
    hipLaunchKernelGGL((token_logp_kernel<T, NT, NC>), dim3(rows), dim3(NT), 0, s, a);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_policy_loss(hipStream_t s, int dtype, const PolicyDesc& a) {
  return dtype == 1 ? policy_launch<bf16_t>(s, a) : policy_launch<float>(s, a);
}

hipError_t launch_preference_fwd(hipStream_t s, int dtype, const PreferenceDesc& a) {
  const unsigned rows = 2u * (unsigned)a.pairs * (unsigned)a.seq;
  const hipError_t e = dtype == 1 ? token_logp_launch<bf16_t>(s, a, rows) : token_logp_launch<float>(s, a, rows);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pair_loss_kernel, dim3(a.pairs), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_preference_bwd(hipStream_t s, int dtype, const PreferenceDesc& a) {
  const unsigned rows = 2u * (unsigned)a.pairs * (unsigned)a.seq;
  if (dtype == 1) hipLaunchKernelGGL(preference_bwd_kernel<bf16_t>, dim3(rows), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(preference_bwd_kernel<float>, dim3(rows), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace bamboo
