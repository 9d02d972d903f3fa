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
// read again.  All sums are in 32 bits, in a fixed order; those over a sequence in 64.
// 4096 x 50304 bf16 with KL and entropy, a quarter of the tokens left out (721 MB): 139 us, 5.2 TB/s (191 us with three
// operations to an exponent, comparisons with the label, and 1024 threads a row, of which a CU holds one workgroup).  Preference
// loss 4096 x 30528 bf16, half of the tokens left out: log-probabilities 25 us, gradient 51 us.
#include <math.h>

#include <type_traits>

#include "common.h"

namespace bamboo {

namespace {

// exp(t) for t <= 0: the product with log2 e in two parts, whose rounding would otherwise shift every term the same way
constexpr float kL2e = 1.4426950408889634f, kL2eRest = 1.9259629911266175e-8f, kLn2 = 0.6931471805599453f;
constexpr float kFar = -300.f;      // an exponent of 2 whose power is 0
constexpr float kWide = 1 << 20;    // maxima from here on are taken off the logits before anything else
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
  for (int j = 0; j < Chunk<T>::N; ++j) x[j] = v + j < V ? row[v + j] : (T)(-INFINITY);    // no maximum, and adds nothing
  return x;
}
// STREAM: not to be kept in the caches.  Gradients that do not fit there any more would only push out the logits that are still
// to be read (4096 x 30528, of which half count: log-probabilities 40 us behind gradients that are kept, 23 behind streamed
// ones; the gradients 53 and 51 us; policy loss of 4096 x 50304 144 and 138 us).
template <typename T, bool STREAM>
__device__ __forceinline__ void store_chunk(T* row, int v, int V, typename Chunk<T>::type x) {
  if (v + Chunk<T>::N <= V) {
    auto* p = (typename Chunk<T>::loose*)(row + v);
    if (STREAM) __builtin_nontemporal_store((typename Chunk<T>::loose)x, p);
    else *p = x;
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

// What a row's pass leaves.  e_v below is 2^(z_v log2 e - m2) with m2 = round(max log2 e), one multiply-add and the
// exponential: what m2 is off by shifts all e_v and their sum alike, so that p_v = e_v / sum is free of it; from the sum's
// logarithm it is taken back (`slip`).  (What log2 e is off by, 1e-8 of the distance to the maximum, stays.)  From a maximum of
// 2^20 on `slip` would grow beyond a sixteenth, and m2 out of the range of 32 bits in the end (a row that a mask has set to -1e30 or the
// type's lowest value): there z_v - base with base = max stands in for z_v, in the storage type too: it is exact where z_v is
// within a factor of two of the maximum, and so far away otherwise that e_v is 0.
struct RowStats {
  float top, base, m2;     // maximum (0 in the place of -inf); the maximum from kWide on, otherwise 0; see above
  float sum, log_s, slip;  // of e_v; log of the sum of exp(z_v - top), = log(sum) - slip
  float at_label, logp, entropy;
  bool far;                // logits so far below the maximum that the distance is -inf
};

// NC > 0: the row lies in registers, NC chunks a thread; in fp32 the e_v take the logits' place.  NC = 0: it is read as
// often as it is needed.  A NaN or +inf in a row, or a row of -inf alone, makes its results NaN; other -inf add nothing.
template <typename T, int NT, int NC, bool ENT>
struct RowPass {
  typedef typename Chunk<T>::type vec;
  static constexpr int E = Chunk<T>::N, HELD = NC > 0 ? NC : 1;
  static constexpr bool KEEPS_EXP = NC > 0 && sizeof(T) == 4;
  vec x[HELD];
  __device__ __forceinline__ static int place(int c) { return (c * NT + (int)threadIdx.x) * E; }
  __device__ __forceinline__ RowStats run(const T* row, int V, int label, float* red) {
    RowStats r;
    r.at_label = to_f32<T>(row[label]);
    float m = -INFINITY, s = 0.f, w = 0.f;
    if constexpr (NC > 0) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (place(c) < V) x[c] = load_chunk<T>(row, place(c), V);
      centre(&r, block_max<NT>(own_max(V), red));
      if (r.base != 0.f) {                                        // the same for the whole workgroup
#pragma unroll
        for (int c = 0; c < NC; ++c)
          if (place(c) < V)
#pragma unroll
            for (int j = 0; j < E; ++j) x[c][j] = from_f32<T>(to_f32<T>(x[c][j]) - r.base);
      }
      if constexpr (ENT) close(V);
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (place(c) < V)
#pragma unroll
          for (int j = 0; j < E; ++j) {
            const float t = fmaf(to_f32<T>(x[c][j]), kL2e, -r.m2), e = __builtin_amdgcn_exp2f(t);
            s += e;
            if (ENT) w = fmaf(e, t, w);
            if constexpr (KEEPS_EXP) x[c][j] = e;
          }
      block_sum2<NT>(&s, &w, red + NT / 64);
      r.far = ENT && w != w && s == s;                            // 0 * -inf somewhere: the same for the whole workgroup
      if (r.far) {
        w = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
          if (place(c) < V)
#pragma unroll
            for (int j = 0; j < E; ++j) {
              float t, e;
              term(x[c], j, r, &t, &e);
              w = fmaf(e, fmaxf(t, kFar), w);
            }
        float none = 0.f;
        __syncthreads();
        block_sum2<NT>(&w, &none, red + NT / 64);
      }
    } else {
      r.far = true;
      // a thread's sums are of exp(z - m) and of that times (z - m), for its own running maximum m
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
          const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
          for (int j = 0; j < E; ++j) {
            const float t = to_f32<T>(y[q][j]) - from, e = exp_of(t);
            s += e;
            if (ENT) w = fmaf(e, fmaxf(t, kFar), w);
          }
        }
      }
      centre(&r, block_max<NT>(m, red));
      if (m == -INFINITY) {                                       // nothing above -inf here: 0, or NaN
        w = s;
      } else {
        const float away = m - r.top, by = exp_of(away);
        if (ENT) w = by > 0.f ? by * (w + away * s) : 0.f;
        s *= by;
      }
      block_sum2<NT>(&s, &w, red + NT / 64);
      // in the units of the other form
      const float shift = __builtin_amdgcn_exp2f(r.slip * kL2e);
      if (ENT) w = (w * kL2e + r.slip * kL2e * s) * shift;
      s *= shift;
    }
    r.sum = s;
    const float l = s > 0.f ? logf(s) : NAN;                      // a row of -inf alone, or a NaN in it
    r.log_s = l - r.slip;
    r.logp = (r.at_label - r.top) - r.log_s;
    r.entropy = ENT ? l - kLn2 * w / s : 0.f;
    return r;
  }
  // of element j of a chunk: the exponent, and e_v.  Where e_v is what is held, an exponent below -126 has left 0: any finite one
  // will do in its place, and the logarithm's -inf would not, 0 * -inf being NaN
  __device__ __forceinline__ static void term(const vec& v, int j, const RowStats& r, float* t, float* e) {
    if constexpr (KEEPS_EXP) {
      *e = v[j];
      *t = fmaxf(__builtin_amdgcn_logf(*e), kFar);
    } else {
      *t = fmaf(NC > 0 ? to_f32<T>(v[j]) : to_f32<T>(v[j]) - r.base, kL2e, -r.m2);
      *e = __builtin_amdgcn_exp2f(*t);
    }
  }
  // Maximum of the thread's part of the row.  bf16: as integers of 16 bits, two at a time, numbers from 0 up are in order and
  // above all negative ones, so the largest is found there unless there are none but negative ones.
  __device__ __forceinline__ float own_max(int V) const {
    if constexpr (sizeof(T) == 2) {
      typedef short short2_t __attribute__((ext_vector_type(2)));
      short2_t top = {(short)-32768, (short)-32768};
#pragma unroll
      for (int c = 0; c < HELD; ++c)
        if (place(c) < V) {
          union { vec v; short2_t p[4]; } u;
          u.v = x[c];
#pragma unroll
          for (int j = 0; j < 4; ++j) top = __builtin_elementwise_max(top, u.p[j]);
        }
      const short most = top[0] > top[1] ? top[0] : top[1];
      if (most >= 0) return __builtin_bit_cast(float, (unsigned)(unsigned short)most << 16);
    }
    float m = -INFINITY;
#pragma unroll
    for (int c = 0; c < HELD; ++c)
      if (place(c) < V)
#pragma unroll
        for (int j = 0; j < E; ++j) m = fmaxf(m, to_f32<T>(x[c][j]));
    return m;
  }
  // What fills the last vector behind the row's end has been -inf for the maximum; from here on it is far below it but finite, so
  // that e * t is 0 there and `far` speaks of the row's own logits alone.
  __device__ __forceinline__ void close(int V) {
    const int chunk = V / E;                                      // the partial one, of thread chunk % NT
    if (V % E == 0) return;
#pragma unroll
    for (int c = 0; c < HELD; ++c)
      if (c == chunk / NT && (int)threadIdx.x == chunk % NT)
#pragma unroll
        for (int j = 0; j < E; ++j)
          if (j >= V % E) x[c][j] = from_f32<T>(-1e30f);
  }
  __device__ __forceinline__ static void centre(RowStats* r, float top) {
    r->top = top == -INFINITY ? 0.f : top;
    r->base = fabsf(r->top) >= kWide ? r->top : 0.f;
    const float near = r->top - r->base;                          // NaN for +inf
    r->m2 = near * kL2e;
    r->slip = (fmaf(near, kL2e, -r->m2) + near * kL2eRest) * kLn2;
  }
};

// d = scale * (coef * [v = label] + p_v * (ent * (log p_v + H) - coef))
template <typename T, int NT, int NC, bool ENT, bool STREAM>
__device__ __forceinline__ void write_gradient(const RowPass<T, NT, NC, ENT>& pass, const T* row, T* out, int V, int label,
                                               const RowStats& r, float coef, float ent, float scale) {
  typedef typename Chunk<T>::type vec;
  constexpr int E = Chunk<T>::N;
  const float per = scale / r.sum, hit = coef * scale;
  const float k1 = ent * per * kLn2, k0 = (ent * (r.entropy - (r.log_s + r.slip)) - coef) * per;      // of t, and without it
  auto write = [&](auto with_log, auto far) {
    auto one = [&](int v, const vec& x) {
      float d[E];
#pragma unroll
      for (int j = 0; j < E; ++j) {
        float t, e;
        RowPass<T, NT, NC, ENT>::term(x, j, r, &t, &e);
        d[j] = e * (with_log ? fmaf(k1, far ? fmaxf(t, kFar) : t, k0) : k0);
      }
      if ((unsigned)(label - v) < (unsigned)E) {                  // one chunk of the row
#pragma unroll
        for (int j = 0; j < E; ++j) d[j] += v + j == label ? hit : 0.f;
      }
      vec o;
#pragma unroll
      for (int j = 0; j < E; ++j) o[j] = from_f32<T>(d[j]);
      store_chunk<T, STREAM>(out, v, V, o);
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
  };
  if (!ENT || ent == 0.f) write(std::false_type(), std::false_type());
  else if (r.far) write(std::true_type(), std::true_type());
  else write(std::true_type(), std::false_type());
}

template <typename T, int NT, bool STREAM>
__device__ __forceinline__ void write_zeros(T* out, int V) {
  typename Chunk<T>::type o;
#pragma unroll
  for (int j = 0; j < Chunk<T>::N; ++j) o[j] = (T)0.f;
  for (int v = threadIdx.x * Chunk<T>::N; v < V; v += NT * Chunk<T>::N) store_chunk<T, STREAM>(out, v, V, o);
}

// One workgroup per token.
template <typename T, int NT, int NC, bool ENT, bool STREAM>
__global__ __launch_bounds__(NT) void policy_loss_kernel(PolicyDesc a) {
  __shared__ float red[3 * NT / 64];
  const long t = blockIdx.x;
  T* out = a.dlogits != nullptr ? (T*)a.dlogits + t * a.ldd : nullptr;
  if (a.mask != nullptr && a.mask[t] == 0) {          // uniform over the workgroup: nothing of the row is read
    if (out != nullptr) write_zeros<T, NT, STREAM>(out, a.V);
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
  // differences to logp from its parts: logp itself is rounded to a few 10^-7, which a small KL term would not forgive
  const float below = r.at_label - r.top, ratio = expf((below - old) - r.log_s);
  const float free = ratio * adv, held = fminf(fmaxf(ratio, 1.f - a.clip_low), 1.f + a.clip_high) * adv;
  // the smaller of the two counts; a ratio or advantage that is NaN stays one
  const bool counts = !(free > held);
  float loss = -(counts ? free : held), coef = counts ? -free : 0.f, kl = 0.f;
  if (a.ref_logp != nullptr) {
    const float away = (ref - below) + r.log_s, grown = expm1f(away);
    kl = grown < INFINITY ? grown - away : grown;               // exp(u) - u - 1 grows without bound with u
    if (a.kl_coef != 0.f) {                                     // an infinite term without weight adds nothing
      loss = fmaf(a.kl_coef, kl, loss);
      coef = fmaf(-a.kl_coef, grown, coef);
    }
  }
  if (ENT) loss = fmaf(-a.ent_coef, r.entropy, loss);
  if (threadIdx.x == 0) {
    a.logp[t] = r.logp;
    a.loss_tok[t] = loss;
    if (a.kl_tok != nullptr) a.kl_tok[t] = kl;
    if (ENT && a.entropy != nullptr) a.entropy[t] = r.entropy;
  }
  if (out != nullptr) write_gradient<T, NT, NC, ENT, STREAM>(pass, row, out, a.V, label, r, coef, a.ent_coef, a.scale);
}

// lse and the label's log-probability of every token that counts (0 for the others).  The latter in 64 bits too: the margin
// is a small difference of two sums over sequences, and roundings of each term, a few 10^-7, would be most of its error.
template <typename T, int NT>
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
  RowPass<T, NT, 0, false> pass;
  const RowStats r = pass.run((const T*)a.logits + t * a.ldl, a.V, clamp_label(a.labels[t], a.V), red);
  if (threadIdx.x == 0) {
    a.lse[t] = r.top + r.log_s;
    a.logp[t] = r.logp;
    a.scratch[t] = ((double)r.at_label - r.top) - (r.sum > 0.f ? log((double)r.sum) - r.slip : NAN);
  }
}

// log(1 + exp(x)) without overflow
__device__ __forceinline__ double softplus(double x) { return x > 0 ? x + log1p(exp(-x)) : log1p(exp(x)); }

// Per pair: sums of both sequences' log-probabilities (64 bits, fixed order), margin and loss.
__global__ __launch_bounds__(256) void pair_loss_kernel(PreferenceDesc a) {
  __shared__ double red[2][4];
  const int i = blockIdx.x;
  const double *lc = a.scratch + (long)i * a.seq, *lr = lc + (long)a.pairs * a.seq;
  double sc = 0., sr = 0.;
  for (int t = threadIdx.x; t < a.seq; t += 1024) {
    double x[4], y[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      x[q] = t + 256 * q < a.seq ? lc[t + 256 * q] : 0.;
      y[q] = t + 256 * q < a.seq ? lr[t + 256 * q] : 0.;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      sc += x[q];
      sr += y[q];
    }
  }
  for (int o = 32; o > 0; o >>= 1) {
    sc += __shfl_xor(sc, o, 64);
    sr += __shfl_xor(sr, o, 64);
  }
  if ((threadIdx.x & 63) == 0) {
    red[0][threadIdx.x >> 6] = sc;
    red[1][threadIdx.x >> 6] = sr;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const double c = (red[0][0] + red[0][1]) + (red[0][2] + red[0][3]), r = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
    const double margin = (double)a.beta * ((c - a.ref_logp[i]) - (r - a.ref_logp[a.pairs + i]));
    a.logp_seq[i] = (float)c;
    a.logp_seq[a.pairs + i] = (float)r;
    a.margin[i] = (float)margin;
    // a side without weight adds nothing, infinite or not
    const double yes = 1. - (double)a.smoothing, no = (double)a.smoothing;
    a.loss[i] = (float)((yes > 0. ? yes * softplus(-margin) : 0.) + (no > 0. ? no * softplus(margin) : 0.));
  }
}

// dlogits = scale * dL/dlogp_seq * ([v = label] - p), dL/dlogp_seq = +-beta (sigmoid(margin) - (1 - smoothing)), here as
// smoothing sigmoid(margin) - (1 - smoothing) sigmoid(-margin): of pairs that are told apart well sigmoid(margin) is 1 to the last
// bit, and the difference to 1 is all there is.
// A workgroup takes four chunks a thread of a row: no thread needs another's, and the rows of a short batch fill the chip.
constexpr int kAhead = 4;
template <typename T, bool STREAM>
__global__ __launch_bounds__(256) void preference_bwd_kernel(PreferenceDesc a) {
  typedef typename Chunk<T>::type vec;
  constexpr int E = Chunk<T>::N;
  const long t = blockIdx.x;
  const int v0 = (int)(blockIdx.y * kAhead * 256 + threadIdx.x) * E;
  T* out = (T*)a.dlogits + t * a.ldd;
  if (a.mask != nullptr && a.mask[t] == 0) {
    vec o;
#pragma unroll
    for (int j = 0; j < E; ++j) o[j] = (T)0.f;
#pragma unroll
    for (int q = 0; q < kAhead; ++q)
      if (v0 + q * 256 * E < a.V) store_chunk<T, STREAM>(out, v0 + q * 256 * E, a.V, o);
    return;
  }
  const T* row = (const T*)a.logits + t * a.ldl;
  vec x[kAhead];
#pragma unroll
  for (int q = 0; q < kAhead; ++q)
    if (v0 + q * 256 * E < a.V) x[q] = load_chunk<T>(row, v0 + q * 256 * E, a.V);
  const int label = clamp_label(a.labels[t], a.V);
  const int seq = (int)(t / a.seq), pair = seq < a.pairs ? seq : seq - a.pairs;
  const float lse = a.lse[t];
  const double m = a.margin[pair], e = exp(-fabs(m)), most = 1. / (1. + e), least = e * most;
  const double g = (double)a.smoothing * (m >= 0. ? most : least) - (1. - (double)a.smoothing) * (m >= 0. ? least : most);
  const float coef = (float)((seq < a.pairs ? g : -g) * (double)a.beta * (double)a.scale);
#pragma unroll
  for (int q = 0; q < kAhead; ++q) {
    const int v = v0 + q * 256 * E;
    if (v >= a.V) break;
    float d[E];
#pragma unroll
    for (int j = 0; j < E; ++j) d[j] = -coef * exp_of(to_f32<T>(x[q][j]) - lse);
    if ((unsigned)(label - v) < (unsigned)E) {
#pragma unroll
      for (int j = 0; j < E; ++j) d[j] += v + j == label ? coef : 0.f;
    }
    vec o;
#pragma unroll
    for (int j = 0; j < E; ++j) o[j] = from_f32<T>(d[j]);
    store_chunk<T, STREAM>(out, v, a.V, o);
  }
}

// Calls go(threads, chunks) with the smallest workgroup and number of chunks a thread that hold V elements of T; where the
// rows do not fill the chip, with more threads: a row's time is then its own chain of arithmetic and trips to memory.  With 1024
// threads always and never, us (8 to 256 rows: a workgroup a CU at most):
//                    8 rows       48         128        256        320        512        1024       2048
//   bf16  17000    8.8 /  9.4   8.9 /  9.6   9.4 / 10.0  11.2 / 11.5  14.3 / 13.7  15.8 / 15.7  23.4 / 21.8   39 /  38
//   bf16  30528    9.9 / 11.3  10.3 / 11.9  11.9 / 13.3  14.5 / 15.5  19.0 / 20.2  19.8 / 21.2  33.7 / 33.9   57 /  58
//   bf16  50304   12.3 / 12.6  12.9 / 13.3  15.4 / 15.9  19.5 / 19.7  25.3 / 24.6  35.1 / 31.9  59.1 / 51.8  101 /  86
//   fp32   8300    7.7 /  9.1   7.9 /  9.3   8.6 /  9.7  10.1 / 11.1  12.1 / 12.3  13.5 / 13.9  21.0 / 17.8   36 /  36
//   fp32  16000    8.6 / 11.6   9.3 / 12.2  10.5 / 13.1  13.0 / 15.3  15.2 / 16.7  17.0 / 20.5  33.2 / 29.9   57 /  64
//   fp32  32003   11.0 / 12.5  12.2 / 13.8  14.8 / 16.3  18.6 / 19.5  30.3 / 28.2  36.4 / 31.8  67.8 / 61.5  112 / 112
// Up to 256 rows more threads never lose; beyond, which of the two wins changes with the length, and the most they win is 17 %.
template <typename T, typename GO>
hipError_t by_row_length(int rows, int V, GO go) {
  const int chunks = (V + Chunk<T>::N - 1) / Chunk<T>::N;
#define BAMBOO_ROW(NT, NC) \
  if (chunks <= NT * NC) return go(std::integral_constant<int, NT>(), std::integral_constant<int, NC>())
  if (rows <= 256 && chunks > 2048) {
    BAMBOO_ROW(1024, 4);
    BAMBOO_ROW(1024, 8);
  }
  BAMBOO_ROW(256, 1);
  BAMBOO_ROW(256, 2);
  BAMBOO_ROW(256, 4);
  BAMBOO_ROW(256, 6);
  BAMBOO_ROW(256, 8);
  BAMBOO_ROW(256, 12);
  BAMBOO_ROW(256, 16);
  BAMBOO_ROW(512, 10);
  BAMBOO_ROW(512, 13);
  BAMBOO_ROW(512, 16);
  BAMBOO_ROW(1024, 12);
  BAMBOO_ROW(1024, 16);
#undef BAMBOO_ROW
  return go(std::integral_constant<int, 1024>(), std::integral_constant<int, 0>());
}

template <typename T>
hipError_t policy_launch(hipStream_t s, const PolicyDesc& a) {
  const bool stream = streams_past_cache(2L * a.T * a.V * (long)sizeof(T));
  return by_row_length<T>(a.T, a.V, [&](auto nt, auto nc) {
    constexpr int NT = decltype(nt)::value, NC = decltype(nc)::value;
    const bool ent = a.entropy != nullptr || a.ent_coef != 0.f;
    const auto kern = ent ? (stream ? policy_loss_kernel<T, NT, NC, true, true> : policy_loss_kernel<T, NT, NC, true, false>)
                          : (stream ? policy_loss_kernel<T, NT, NC, false, true> : policy_loss_kernel<T, NT, NC, false, false>);
    hipLaunchKernelGGL(kern, dim3((unsigned)a.T), dim3(NT), 0, s, a);
    return hipGetLastError();
  });
}
// Read once, so nothing is held.  Few rows: their time is a chain of trips to memory, fewer with more threads (held in
// registers, for the cheaper exponents, 96 rows of 50257 took 7.6 us in the place of 7.2).  With 256 and with 1024 threads, us, the
// launch that sums the sequences included:
//                  48 rows      128        256        384        512        768        1024       2048
//   bf16   1000   5.8 /  5.9   5.9 /  6.1   5.8 /  6.1   6.2 /  6.7   6.1 /  6.7   6.4 /  7.8   6.9 /  8.6   7.5 / 12.1
//   bf16   8000   6.4 /  6.4   6.5 /  6.5   6.7 /  6.8   7.4 /  7.9   7.8 /  8.1   9.2 /  9.5   9.9 / 10.9  12.4 / 16.2
//   bf16  30528   8.6 /  7.7   9.4 /  8.2  10.4 /  9.8  11.5 / 12.2  12.5 / 12.4  14.9 / 15.1  16.4 / 17.5  31.2 / 31.5
//   bf16  50257  11.8 /  9.6  13.7 / 10.6  14.2 / 11.3  15.8 / 14.8  17.0 / 15.7  25.1 / 25.1  32.9 / 31.2  54.3 / 53.1
//   fp32  32003  11.7 /  8.7  12.4 /  9.3  13.5 / 11.0  14.7 / 14.2  16.4 / 16.6  24.9 / 24.3  31.9 / 30.8  54.1 / 52.1
// 1024 threads win up to 24 % for long rows below 512 of them and lose up to 10 % for short ones, whose whole call is 6 us; from 512
// rows on they win 8 % at most and lose up to 38 %.
template <typename T>
hipError_t token_logp_launch(hipStream_t s, const PreferenceDesc& a, unsigned rows) {
  if (rows >= 512) hipLaunchKernelGGL((token_logp_kernel<T, 256>), dim3(rows), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((token_logp_kernel<T, 1024>), dim3(rows), dim3(1024), 0, s, a);
  return hipGetLastError();
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
  const bool stream = streams_past_cache(2L * rows * a.V * (dtype == 1 ? 2 : 4));
  const int per = kAhead * 256 * (dtype == 1 ? Chunk<bf16_t>::N : Chunk<float>::N);
  const dim3 grid(rows, (unsigned)((a.V + (long)per - 1) / per));
  const auto kern = dtype == 1 ? (stream ? preference_bwd_kernel<bf16_t, true> : preference_bwd_kernel<bf16_t, false>)
                               : (stream ? preference_bwd_kernel<float, true> : preference_bwd_kernel<float, false>);
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace bamboo
