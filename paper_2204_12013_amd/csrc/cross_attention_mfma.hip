// Attention over an encoder's states on the matrix cores (bf16 in, fp32 softmax and accumulation), head size up to 128.
//
// The tiles, their placement in LDS and the operand fragments are those of the self-attention; here the two sides have
// lengths of their own, keys end at each sample's length, query heads that share a key head are rows of one problem
// (cross_rows.h), and where the owned rows fill too few workgroups the streamed side is cut into parts whose results are
// joined by a second launch (the softmax's running maximum and sum make the parts of the forward independent; the
// gradients are sums).  No atomics: results are bitwise reproducible.
//
// Probabilities and dS are rounded to bf16 as operands of the second products: dQ of 8 x 512 x 333 is 0.0025 of its norm off, 0.0017
// of that the rounding of the result itself.
// Large problems are bound by the matrix instructions (1 x 2048 x 4096, 96 heads over 8 of 128: forward 419 us, 980 TFLOP/s; dQ
// 523 us, 1180; dK and dV 843 us, 980; a large library product 1210), those of few tiles by a wavefront's own chain of vector
// and matrix instructions at two to three wavefronts a SIMD (8 x 512 x 333, 16 heads of 64: 13.2, 17.0 and 21.9 us; 1.25 us a
// tile of 64 keys in the forward) and by what a launch takes to start and end.
#include "attention_tiles.h"
#include "cross_rows.h"

namespace bamboo {

namespace {

// PAD: head sizes other than 64 and 128, and rows that are not aligned to 16 bytes.  Tiles pass through registers, where
// features behind the head's last become zeros; they add nothing to any product, and are not stored.  Vectors are loaded and
// stored at any alignment of an element.
typedef bf16_t loose8 __attribute__((ext_vector_type(8), aligned(2)));
template <bool PAD> __device__ __forceinline__ bf16x8 load8(const bf16_t* p, int left) {       // left: features from p on
  if (!PAD) return *(const bf16x8*)p;
  if (left >= 8) return *(const loose8*)p;
  bf16x8 t = {};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < left) t[j] = p[j];
  return t;
}
template <bool PAD> __device__ __forceinline__ void store8(bf16_t* p, const bf16x8& x, int left) {
  if (!PAD) {
    *(bf16x8*)p = x;
  } else if (left >= 8) {
    *(loose8*)p = x;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[j] = x[j];
  }
}

// The lane's operand fragments of one row: elements 16 ks + 8 (l / 32) .. + 7, zero where it is not live.
template <int D, bool PAD>
__device__ __forceinline__ void lane_row(bf16x8 (&f)[D / 16], const bf16_t* row, bool live, int d) {
  const int l = threadIdx.x & 63;
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) {
    const int c = ks * 16 + (l >> 5) * 8;
    bf16x8 t = {};
    if (live) t = load8<PAD>(row + c, d - c);
    f[ks] = t;
  }
}
// A wavefront's transposed result (lane = row) through its private LDS area to rows wherever `at` says they are.
template <int D, bool PAD, typename AT>
__device__ __forceinline__ void put_rows(const f32x16 (&acc)[D / 32], float mul, bf16_t* stage, int row0, int row_lim, int d, AT at) {
  constexpr int LD = D + 8;
  const int l = threadIdx.x & 63;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      bf16x4 o;
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] = (bf16_t)(acc[dt][4 * a + c] * mul);
      *(bf16x4*)(stage + (l & 31) * LD + dt * 32 + 8 * a + 4 * (l >> 5)) = o;
    }
  __builtin_amdgcn_s_waitcnt(0xc07f);
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int it = 0; it < 32 * (D / 8) / 64; ++it) {
    const int idx = l + it * 64;
    const int row = idx / (D / 8), ch = (idx % (D / 8)) * 8;
    const bf16x8 t = *(const bf16x8*)(stage + row * LD + ch);
    if (row0 + row < row_lim) store8<PAD>(at(row0 + row) + ch, t, d - ch);
  }
  __builtin_amdgcn_s_waitcnt(0xc07f);
  __builtin_amdgcn_wave_barrier();
}
// the lane's row of a part's result, unscaled
template <int D, bool PAD>
__device__ __forceinline__ void put_part(const f32x16 (&acc)[D / 32], float* row, int d) {
  const int g = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const int f = dt * 32 + 8 * a + 4 * g;
      if (PAD) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (f + c < d) row[f + c] = acc[dt][4 * a + c];
      } else {
        f32x4 t;
#pragma unroll
        for (int c = 0; c < 4; ++c) t[c] = acc[dt][4 * a + c];
        *(f32x4*)(row + f) = t;
      }
    }
}
// PAD: the same rows of two tensors, 64 to a tile, requested (fetch) ahead of a step and put into LDS (stash) behind it.
// rows(i, &p, &q): where row i of both is; i may lie behind the last.
template <int D>
struct PadTiles {
  static constexpr int N = TileCopy<D>::N, STEP = 256 / (D / 8);
  bf16x8 x[N], y[N];
  template <typename ROWS> __device__ __forceinline__ void fetch(ROWS rows, int tile, int d) {
    const int row = threadIdx.x / (D / 8), col = ((threadIdx.x % (D / 8)) ^ swz<D>(row)) * 8;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bf16_t *p, *q;
      rows(tile * TILE + row + i * STEP, &p, &q);
      x[i] = load8<true>(p + col, d - col);
      y[i] = load8<true>(q + col, d - col);
    }
  }
  __device__ __forceinline__ void stash(unsigned lds0, unsigned lds1) const {
    typedef __attribute__((address_space(3))) bf16x8* lds_ptr;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      *(lds_ptr)(lds0 + threadIdx.x * 16 + i * 4096) = x[i];
      *(lds_ptr)(lds1 + threadIdx.x * 16 + i * 4096) = y[i];
    }
  }
};
template <int N> __device__ __forceinline__ void clear(f32x16 (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) x[i][r] = 0.f;
}

// -------------------------------------------------------------------------------------------- forward
template <int D, bool PAD>
__global__ __launch_bounds__(256, D == 64 && !PAD ? 3 : 2) void cross_fwd_mfma_kernel(CrossDesc a) {
  constexpr unsigned TB = TileCopy<D>::BYTES;
  extern __shared__ __attribute__((aligned(256))) unsigned char smem_raw[];
  const unsigned ring = lds_address(smem_raw);    // [2][keys, values]
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 5, d = PAD ? a.d : D;
  const CrossBlock w = cross_block(a);
  const int len = __builtin_amdgcn_readfirstlane(cross_len(a, w.b));
  int t0, t1;
  cross_part(len, a.splits, w.split, &t0, &t1);
  const int nt = t1 - t0;
  const int qw0 = w.blk * 128 + wave * 32, row = qw0 + (lane & 31);
  const bool live = row < a.rows, busy = qw0 < a.rows;
  const CrossRow at = cross_row(a, w.kvh, min(row, a.rows - 1));
  const bf16_t* kb = (const bf16_t*)a.k + (long)w.b * a.sk * a.ldkv + w.kvh * d;
  const bf16_t* vb = (const bf16_t*)a.v + (long)w.b * a.sk * a.ldkv + w.kvh * d;
  const float c = rsqrtf((float)d) * kLog2e;

  bf16x8 qf[D / 16];
  lane_row<D, PAD>(qf, (const bf16_t*)a.q + ((long)w.b * a.sq + at.query) * a.ldq + at.head * d, live, d);
  f32x16 o[D / 32];
  clear(o);
  float m_i = kMasked, l_i = 0.f;
  TileCopy<D> copy;
  copy.init(a.ldkv, max(len, 1));
  FragAddr<D, true> fr;
  fr.init(ring);
  PadTiles<D> pad;
  const auto keys = [&](int r, const bf16_t** p, const bf16_t** q) {
    const long at_row = (long)min(r, len - 1) * a.ldkv;
    *p = kb + at_row;
    *q = vb + at_row;
  };
  if (nt > 0) {
    if constexpr (PAD) {
      pad.fetch(keys, t0, d);
      pad.stash(ring, ring + TB);
    } else {
      copy.issue(kb, t0, ring);
      copy.issue(vb, t0, ring + TB);
    }
  }
  for_each_tile(nt, [&](int t, int slot) __attribute__((always_inline)) {
    const unsigned buf = slot * 2 * TB;
    if constexpr (!PAD) wait_tiles<0>();
    __syncthreads();                              // tile t is there, and tile t - 1 has been read everywhere
    if constexpr (PAD) {
      if (t + 1 < nt) pad.fetch(keys, t0 + t + 1, d);
    } else if (t + 1 < nt) {
      const unsigned ring = lds_address(smem_raw);
      copy.issue(kb, t0 + t + 1, ring + (slot ^ 1) * 2 * TB);
      copy.issue(vb, t0 + t + 1, ring + (slot ^ 1) * 2 * TB + TB);
    }
    if (busy) {                                   // uniform over the wavefront
      const int k0 = (t0 + t) * TILE;
      f32x16 s[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[u][r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr.frag_k(buf, 0, u * 32, ks), qf[ks], s[u], 0, 0, 0);
      // Online softmax in the log2 domain.  The running maximum is raised only where some row's has grown by more than 8
      // (a factor of 256, harmless in fp32 and bf16): the output is rescaled on a few tiles instead of on every one.
      if (k0 + TILE > len) {                      // the last tile: keys behind the length
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[u][r] = k0 + u * 32 + acc_row(r) < len ? s[u][r] : kMasked;
      }
      float mx = kMasked;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[u][r]);
      mx *= c;
      mx = fmaxf(mx, other_half(mx));
      const bool grow = mx > m_i + 8.f;
      if (__builtin_amdgcn_ballot_w64(grow) != 0) {
        const float m_new = grow ? mx : m_i;
        const float alpha = __builtin_amdgcn_exp2f(m_i - m_new);
        l_i *= alpha;
        m_i = m_new;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[u][r] = __builtin_amdgcn_exp2f(fmaf(s[u][r], c, -m_i));
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bf16x8 pb = pack8(s[u >> 1], u & 1);
#pragma unroll
        for (int j = 0; j < 8; ++j) l_i += s[u >> 1][8 * (u & 1) + j];
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr.frag_tr(buf, TB, dt, 16 * u), pb, o[dt], 0, 0, 0);
      }
    }
    if constexpr (PAD)
      if (t + 1 < nt) pad.stash(ring + (slot ^ 1) * 2 * TB, ring + (slot ^ 1) * 2 * TB + TB);
  });
  __syncthreads();                                // the tiles' place takes the results
  const float l_tot = l_i + other_half(l_i);
  if (a.splits > 1) {
    if (!live) return;
    const long i = ((long)w.split * a.B * a.kv_heads + w.pair) * a.rows + row;
    put_part<D, PAD>(o, a.part + i * d, d);
    if (g == 0) {
      a.part_stats[2 * i] = m_i;
      a.part_stats[2 * i + 1] = l_tot;
    }
    return;
  }
  bf16_t* stage = (bf16_t*)smem_raw + wave * 32 * (D + 8);
  put_rows<D, PAD>(o, l_tot > 0.f ? 1.f / l_tot : l_tot, stage, qw0, a.rows, d, [&](int r) {
    const CrossRow p = cross_row(a, w.kvh, r);
    return (bf16_t*)a.ctx + ((long)w.b * a.sq + p.query) * a.ldc + p.head * d;
  });
  if (g == 0 && live) a.lse[cross_stat(a, w.b, at)] = len > 0 ? (m_i + __builtin_amdgcn_logf(l_tot)) * kLn2 : -INFINITY;
}

// ------------------------------------------------------------------------------------------- backward
// Owns rows, streams keys, 32 at a time (64: 552 us in the place of 530).
template <int D, bool PAD>
__global__ __launch_bounds__(256, PAD && D == 128 ? 1 : 2) void cross_dq_mfma_kernel(CrossDesc a) {
  constexpr unsigned TB = TileCopy<D>::BYTES;
  extern __shared__ __attribute__((aligned(256))) unsigned char smem_raw[];
  const unsigned ring = lds_address(smem_raw);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, d = PAD ? a.d : D;
  const CrossBlock w = cross_block(a);
  const int len = __builtin_amdgcn_readfirstlane(cross_len(a, w.b));
  int t0, t1;
  cross_part(len, a.splits, w.split, &t0, &t1);
  const int nt = t1 - t0;
  const int qw0 = w.blk * 128 + wave * 32, row = qw0 + (lane & 31);
  const bool live = row < a.rows, busy = qw0 < a.rows;
  const CrossRow at = cross_row(a, w.kvh, min(row, a.rows - 1));
  const long tok = (long)w.b * a.sq + at.query, stat = cross_stat(a, w.b, at);
  const bf16_t* kb = (const bf16_t*)a.k + (long)w.b * a.sk * a.ldkv + w.kvh * d;
  const bf16_t* vb = (const bf16_t*)a.v + (long)w.b * a.sk * a.ldkv + w.kvh * d;
  const float scale = rsqrtf((float)d), c = scale * kLog2e;

  bf16x8 qf[D / 16], dof[D / 16];
  lane_row<D, PAD>(qf, (const bf16_t*)a.q + tok * a.ldq + at.head * d, live, d);
  lane_row<D, PAD>(dof, (const bf16_t*)a.dctx + tok * a.lddc + at.head * d, live, d);
  const float lse2 = a.lse[stat] * kLog2e;
  float delta = 0.f;                              // rowsum(ctx * dctx)
  {
    bf16x8 of[D / 16];
    lane_row<D, PAD>(of, (const bf16_t*)a.ctx + tok * a.ldc + at.head * d, live, d);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int j = 0; j < 8; ++j) delta += (float)of[ks][j] * (float)dof[ks][j];
    delta += other_half(delta);
  }
  f32x16 dq[D / 32];
  clear(dq);
  FragAddr<D, false> fr;
  fr.init(0);
  TileCopy<D> copy;
  copy.init(a.ldkv, max(len, 1));
  PadTiles<D> pad;
  const auto keys = [&](int r, const bf16_t** p, const bf16_t** q) {
    const long at_row = (long)min(r, len - 1) * a.ldkv;
    *p = kb + at_row;
    *q = vb + at_row;
  };
  // tile t of this part (-t0: the sample's first) to `slot`, at once
  const auto bring = [&](int t, int slot) {
    if constexpr (PAD) {
      pad.fetch(keys, t0 + t, d);
      pad.stash(ring + slot * 2 * TB, ring + slot * 2 * TB + TB);
    } else {
      copy.issue(kb, t0 + t, ring + slot * 2 * TB);
      copy.issue(vb, t0 + t, ring + slot * 2 * TB + TB);
    }
  };
  const int all = (len + TILE - 1) / TILE;
  const bool few = nt > 0 && all <= 2;
  if (nt > 0) bring(few ? -t0 : 0, 0);
  const f32x16 zero16 = {};
  if (few) {
    // Few keys: both tiles of the sample fit the ring, and delta is the sum of p dP as the scores give it.  ctx has been rounded to
    // bf16, and what that is off by does not average out over few keys (error of dQ: 3 keys 0.0043 of its norm, 0.0024 this way; at
    // 333 keys the roundings of dS and dQ themselves are 0.0024 and those of delta 0.0007).  Where the two are of different parts,
    // each part forms delta from both.
    if (all == 2) bring(1 - t0, 1);
    wait_tiles<0>();
    __syncthreads();
    delta = 0.f;
    if (busy)
      for (int t = 0; t < all; ++t) {
        const unsigned buf = ring + t * 2 * TB;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          f32x16 s = zero16, dp = zero16;
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr.frag_k(buf, 0, u * 32, ks), qf[ks], s, 0, 0, 0);
            dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr.frag_k(buf, TB, u * 32, ks), dof[ks], dp, 0, 0, 0);
          }
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (t * TILE + u * 32 + acc_row(r) < len) delta = fmaf(__builtin_amdgcn_exp2f(fmaf(s[r], c, -lse2)), dp[r], delta);
        }
      }
    delta += other_half(delta);
    if (t0 > 0) {                                 // the part of the second tile alone
      __syncthreads();
      bring(0, 0);
    }
  }
  if (lane < 32 && live && w.split == 0) a.delta[stat] = delta;
  f32x16 neg_delta, neg_lse;                      // the products start from these: dP less delta, scores less the log-sum-exp
  const float lse_s = -a.lse[stat] * sqrtf((float)d);
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    neg_delta[r] = -delta;
    neg_lse[r] = lse_s;
  }
  wait_tiles<0>();
  __syncthreads();
  for (int t = 0; t < nt; ++t) {
    const int slot = t & 1;
    const unsigned buf = ring + slot * 2 * TB;
    const int k0 = (t0 + t) * TILE;
    if constexpr (PAD) {
      if (t + 1 < nt) pad.fetch(keys, t0 + t + 1, d);
    } else {
      if (t + 1 < nt) bring(t + 1, slot ^ 1);
    }
    if (busy) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x16 s, dp;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr.frag_k(buf, 0, u * 32, ks), qf[ks], ks == 0 ? neg_lse : s, 0, 0, 0);
          dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr.frag_k(buf, TB, u * 32, ks), dof[ks], ks == 0 ? neg_delta : dp, 0, 0, 0);
        }
        if (k0 + u * 32 + 32 > len) {               // the last keys
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = k0 + u * 32 + acc_row(r) < len ? s[r] : kMasked;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(s[r] * c) * dp[r];       // dS^T
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bf16x8 dsb = pack8(s, h);
#pragma unroll
          for (int dt = 0; dt < D / 32; ++dt)
            dq[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr.frag_tr(buf, 0, dt, 32 * u + 16 * h), dsb, dq[dt], 0, 0, 0);
        }
      }
    }
    if constexpr (PAD)
      if (t + 1 < nt) pad.stash(ring + (slot ^ 1) * 2 * TB, ring + (slot ^ 1) * 2 * TB + TB);
    wait_tiles<0>();
    __syncthreads();
  }
  if (a.splits > 1) {
    if (live) put_part<D, PAD>(dq, a.part + w.split * a.part_stride + ((long)w.pair * a.rows + row) * d, d);
    return;
  }
  bf16_t* stage = (bf16_t*)smem_raw + wave * 32 * (D + 8);
  put_rows<D, PAD>(dq, scale, stage, qw0, a.rows, d, [&](int r) {
    const CrossRow p = cross_row(a, w.kvh, r);
    return (bf16_t*)a.dq + ((long)w.b * a.sq + p.query) * a.lddq + p.head * d;
  });
}

// Rows of the pair, 64 to a tile, from wherever their query and head are.  Offsets in 32 bits: see straight().
template <int D>
struct RowCopy {
  static constexpr int N = TileCopy<D>::N, STEP = 256 / (D / 8);     // rows between a thread's chunks: their places are alike
  static_assert(STEP % 16 == 0, "swz repeats after 16 rows");
  unsigned col, wave_lds;
  __device__ __forceinline__ void init() {
    const int r = threadIdx.x / (D / 8);
    col = (unsigned)(((threadIdx.x % (D / 8)) ^ swz<D>(r)) * 8) * 2u;
    wave_lds = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 1024;
  }
  // the same rows of two tensors
  __device__ __forceinline__ void issue(const CrossDesc& a, const bf16_t* g0, long ld0, unsigned lds0, const bf16_t* g1, long ld1,
                                        unsigned lds1, int tile) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = min(tile * TILE + (int)threadIdx.x / (D / 8) + i * STEP, a.rows - 1);
      const CrossRow p = cross_row(a, 0, r);
      const unsigned in_row = (unsigned)p.head * (D * 2) + col;
      asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                   :
                   : "v"((unsigned)p.query * (unsigned)(ld0 * 2) + in_row), "s"(g0), "s"(lds0 + wave_lds + i * 4096)
                   : "memory", "m0");
      asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                   :
                   : "v"((unsigned)p.query * (unsigned)(ld1 * 2) + in_row), "s"(g1), "s"(lds1 + wave_lds + i * 4096)
                   : "memory", "m0");
    }
  }
};

// Owns keys, streams rows.  The streamed rows are worked on 32 at a time, and the score products start from the negated
// log-sum-exp as those of dP do from -delta: at head size 128 that is what lets two wavefronts share a SIMD (256 registers, 8 spilled
// outside the products; 64 rows at a time and one wavefront: 1366 us in the place of 830).  Rows behind the last one and keys
// that do not count get exponents far below all others: no element is compared with a length.
template <int D, bool PAD>
__global__ __launch_bounds__(256, PAD && D == 128 ? 1 : 2) void cross_dkv_mfma_kernel(CrossDesc a) {
  constexpr unsigned TB = TileCopy<D>::BYTES;
  extern __shared__ __attribute__((aligned(256))) unsigned char smem_raw[];
  const unsigned ring = lds_address(smem_raw);    // [2][queries, gradients]
  float* lse_s = (float*)(smem_raw + 4 * TB);     // [2][64], behind the tiles
  float* del_s = lse_s + 2 * TILE;                // [2][64]
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 5, d = PAD ? a.d : D;
  const CrossBlock w = cross_block(a);
  const int len = __builtin_amdgcn_readfirstlane(cross_len(a, w.b));
  const int kw0 = w.blk * 128 + wave * 32, key = kw0 + (lane & 31);
  int t0, t1;
  cross_part(a.rows, a.splits, w.split, &t0, &t1);
  const int nt = w.blk * 128 < len ? t1 - t0 : 0;
  const bool busy = kw0 < len;
  const bf16_t* qb = (const bf16_t*)a.q + (long)w.b * a.sq * a.ldq + w.kvh * a.group * d;
  const bf16_t* gb = (const bf16_t*)a.dctx + (long)w.b * a.sq * a.lddc + w.kvh * a.group * d;
  const float scale = rsqrtf((float)d), rscale = sqrtf((float)d), c = scale * kLog2e;

  bf16x8 kf[D / 16], vf[D / 16];
  const long at_key = ((long)w.b * a.sk + min(key, a.sk - 1)) * a.ldkv + w.kvh * d;
  lane_row<D, PAD>(kf, (const bf16_t*)a.k + at_key, key < len, d);
  lane_row<D, PAD>(vf, (const bf16_t*)a.v + at_key, key < len, d);
  const float shut = key < len ? 0.f : kMasked;   // keys that do not count: exponents of their probabilities
  f32x16 dk[D / 32], dv[D / 32];
  clear(dk);
  clear(dv);
  float lse_r = 0.f, del_r = 0.f;
  auto fetch_stats = [&](int r0) {
    if (threadIdx.x < TILE) {
      const int r = r0 + threadIdx.x;
      const long stat = cross_stat(a, w.b, cross_row(a, w.kvh, min(r, a.rows - 1)));
      // the accumulators start from these: scores come out less the log-sum-exp, dP less delta
      lse_r = r < a.rows ? -a.lse[stat] * rscale : kMasked;    // behind the last row: probabilities of 0
      del_r = -a.delta[stat];
    }
  };
  auto stash_stats = [&](int buf) {
    if (threadIdx.x < TILE) {
      lse_s[buf * TILE + threadIdx.x] = lse_r;
      del_s[buf * TILE + threadIdx.x] = del_r;
    }
  };
  FragAddr<D, false> fr;
  fr.init(0);
  RowCopy<D> copy;
  copy.init();
  PadTiles<D> pad;
  const auto rows = [&](int r, const bf16_t** p, const bf16_t** q) {
    const CrossRow at = cross_row(a, 0, min(r, a.rows - 1));
    *p = qb + (long)at.query * a.ldq + at.head * d;
    *q = gb + (long)at.query * a.lddc + at.head * d;
  };
  if (nt > 0) {
    if constexpr (PAD) {
      pad.fetch(rows, t0, d);
      pad.stash(ring, ring + TB);
    } else {
      copy.issue(a, qb, a.ldq, ring, gb, a.lddc, ring + TB, t0);
    }
    fetch_stats(t0 * TILE);
    stash_stats(0);
  }
  wait_tiles<0>();
  __syncthreads();
  for (int t = 0; t < nt; ++t) {
    const int slot = t & 1;
    const unsigned buf = ring + slot * 2 * TB;
    if (t + 1 < nt) {
      fetch_stats((t0 + t + 1) * TILE);
      if constexpr (PAD) pad.fetch(rows, t0 + t + 1, d);
      else copy.issue(a, qb, a.ldq, ring + (slot ^ 1) * 2 * TB, gb, a.lddc, ring + (slot ^ 1) * 2 * TB + TB, t0 + t + 1);
    }
    if (busy) {
      // 32 rows at a time: the second half's scores would be 32 registers more
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x16 s, dp;
#pragma unroll
        for (int a4 = 0; a4 < 4; ++a4) {
          const f32x4 l4 = *(const f32x4*)(lse_s + slot * TILE + u * 32 + 8 * a4 + 4 * g);
          const f32x4 d4 = *(const f32x4*)(del_s + slot * TILE + u * 32 + 8 * a4 + 4 * g);
#pragma unroll
          for (int cc = 0; cc < 4; ++cc) {
            s[4 * a4 + cc] = l4[cc];
            dp[4 * a4 + cc] = d4[cc];
          }
        }
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr.frag_k(buf, 0, u * 32, ks), kf[ks], s, 0, 0, 0);
          dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr.frag_k(buf, TB, u * 32, ks), vf[ks], dp, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, shut));
          dp[r] *= s[r];                               // dS
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bf16x8 pb = pack8(s, h), dsb = pack8(dp, h);
#pragma unroll
          for (int dt = 0; dt < D / 32; ++dt) {
            dv[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr.frag_tr(buf, TB, dt, 32 * u + 16 * h), pb, dv[dt], 0, 0, 0);
            dk[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr.frag_tr(buf, 0, dt, 32 * u + 16 * h), dsb, dk[dt], 0, 0, 0);
          }
        }
        if (D == 128) __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (t + 1 < nt) {
      stash_stats(slot ^ 1);
      if constexpr (PAD) pad.stash(ring + (slot ^ 1) * 2 * TB, ring + (slot ^ 1) * 2 * TB + TB);
    }
    wait_tiles<0>();
    __syncthreads();
  }
  if (key >= len) {                               // a NaN in a row must not reach them either
    clear(dk);
    clear(dv);
  }
  if (a.splits > 1) {
    if (key < a.sk) {
      float* out = a.part + w.split * a.part_stride + ((long)w.pair * a.sk + key) * (2 * d);
      put_part<D, PAD>(dk, out, d);
      put_part<D, PAD>(dv, out + d, d);
    }
    return;
  }
  bf16_t* stage = (bf16_t*)smem_raw + wave * 32 * (D + 8);
  const long out = (long)w.b * a.sk * a.lddkv + w.kvh * d;
  put_rows<D, PAD>(dk, scale, stage, kw0, a.sk, d, [&](int r) { return (bf16_t*)a.dk + out + (long)r * a.lddkv; });
  put_rows<D, PAD>(dv, 1.f, stage, kw0, a.sk, d, [&](int r) { return (bf16_t*)a.dv + out + (long)r * a.lddkv; });
}

enum { FWD, DQ, DKV };
template <int D, bool PAD, int PASS>
hipError_t launch(hipStream_t s, const CrossDesc& a) {
  constexpr int BYTES = 4 * TileCopy<D>::BYTES + (PASS == DKV ? 4 * TILE * 4 : 0);
  static_assert(BYTES >= 4 * 32 * (D + 8) * 2, "the four staging areas");
  constexpr auto kern = PASS == FWD ? cross_fwd_mfma_kernel<D, PAD>
                                    : (PASS == DQ ? cross_dq_mfma_kernel<D, PAD> : cross_dkv_mfma_kernel<D, PAD>);
  const hipError_t e = ensure_lds_attribute<kern, BYTES>();
  if (e != hipSuccess) return e;
  const unsigned grid = (unsigned)(((PASS == DKV ? a.sk : a.rows) + 127) / 128) * a.splits * a.B * a.kv_heads;
  hipLaunchKernelGGL(kern, dim3(grid), dim3(256), BYTES, s, a);
  return hipGetLastError();
}
// Straight to LDS where the head size and every row's alignment allow it, and byte offsets inside one sample are 32-bit, those
// of the rows of a last, partial tile included (they are clamped after the add).
bool straight(const CrossDesc& a) {
  if (a.d != 64 && a.d != 128) return false;
  uintptr_t bits = 0;
  for (const void* p : {a.q, a.k, a.v, (const void*)a.ctx, a.dctx, (const void*)a.dq, (const void*)a.dk, (const void*)a.dv})
    bits |= (uintptr_t)p;
  const long lds = a.ldq | a.ldkv | a.ldc | a.lddc | a.lddq | a.lddkv, widest = 1L << 32;
  if (lds % 8 || bits & 15) return false;
  return ((long)a.sk + TILE) * a.ldkv * 2 < widest && (long)a.sq * a.ldq * 2 < widest && (long)a.sq * a.lddc * 2 < widest;
}
template <int PASS> hipError_t by_size(hipStream_t s, const CrossDesc& a) {
  if (straight(a)) return a.d == 64 ? launch<64, false, PASS>(s, a) : launch<128, false, PASS>(s, a);
  return a.d <= 64 ? launch<64, true, PASS>(s, a) : launch<128, true, PASS>(s, a);
}

}  // namespace

hipError_t launch_cross_fwd_mfma(hipStream_t s, const CrossDesc& a) { return by_size<FWD>(s, a); }
hipError_t launch_cross_dq_mfma(hipStream_t s, const CrossDesc& a) { return by_size<DQ>(s, a); }
hipError_t launch_cross_dkv_mfma(hipStream_t s, const CrossDesc& a) { return by_size<DKV>(s, a); }

}  // namespace bamboo
