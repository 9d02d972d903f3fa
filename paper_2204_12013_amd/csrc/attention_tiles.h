// What the bf16 attention kernels on the matrix cores share: the copy of 64-row tiles to LDS, the placement
// of their 16-byte chunks there, and the operand fragments that are read from it.
#pragma once
#include "common.h"

namespace bamboo {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) short short4_t;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kMasked = -1.0e30f;
constexpr int TILE = 64;   // rows streamed through LDS per step

// ---- cooperative copy of 64 rows x D (bf16) global -> LDS ---------------------------
// The tiles go straight to LDS (global_load_lds_dwordx4: 16 bytes per lane to consecutive addresses behind a
// wavefront-uniform base), so nothing waits in registers and no LDS store is issued.  Rows are not padded; the 16-byte
// chunk ch of row r sits at position ch ^ swz(r) of its row, which every lane applies to the chunk that it FETCHES.  The
// placement serves both ways a tile is read: 16 consecutive rows of one chunk (frag_k) and 4 rows x 64 bytes (frag_tr)
// each cover the 64 banks once.  With the rows padded to D + 8 (D + 16 for the values of the forward pass) and staged
// through registers the second kind, half of the backward's reads, met its own banks twice.  Backward in us, before and now
// (samples x tokens x heads x size; the forward: see fwd_launch in attention_mfma.hip):
//   8 x 512 x 16 x 64   45.0 / 42.6     4 x 1024 x 25 x 64 causal   81.3 / 79.8     1 x 2048 x 96 x 128 causal  613 / 512
//   4 x 512 x 16 x 64   23.7 / 22.8     2 x 2048 x 25 x 64 causal  129.9 / 129.2    2 x 512 x 24 x 128        52.9 / 50.1
//   3 x 333 x 16 x 64   17.3 / 16.7     1 x 8192 x 16 x 64 causal  517 / 492        1 x 1500 x 20 x 128 causal 136.5 / 124.6
// What bounds both passes is still a wavefront's own chain of matrix and vector instructions, at two wavefronts per SIMD.
// Rows at or beyond row_lim are read from row row_lim - 1 (finite values that the consumers' masks turn
// into exact zeros), so no load sits behind a branch.  A thread's byte offsets inside a tile and their
// upper limits (the same chunk in the last valid row) are computed once; per tile and chunk an add and a
// min remain.  Offsets are 32-bit: the launcher checks that a sequence stays below 4 GiB.
// The loads are inline assembly, which the compiler's wait counts do not see: wait_tiles() before the barrier that
// publishes a tile.
template <int D>
__device__ __forceinline__ int swz(int r) {
  return D == 64 ? ((r & 2) << 1) | ((r >> 2) & 3)       // rows of 128 bytes: two to a line of the 64 banks
                 : ((r & 3) << 2) | ((r >> 2) & 3);      // rows of 256 bytes
}
typedef __attribute__((address_space(3))) void* lds_void_ptr;
__device__ __forceinline__ unsigned lds_address(const void* p) { return (unsigned)(uintptr_t)(lds_void_ptr)p; }
template <int D>
struct TileCopy {
  static constexpr int N = TILE * D / 8 / 256;   // 16-byte chunks per thread
  static constexpr int BYTES = TILE * D * 2;
  unsigned ofs[N], last[N];
  unsigned tile_bytes;                           // 64 rows
  unsigned wave_lds;
  __device__ __forceinline__ void init(long row_stride, int row_lim) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = threadIdx.x + i * 256, r = c / (D / 8);
      const unsigned col = (unsigned)(((c % (D / 8)) ^ swz<D>(r)) * 8) * 2u;
      ofs[i] = (unsigned)r * (unsigned)row_stride * 2u + col;
      last[i] = (unsigned)(row_lim - 1) * (unsigned)row_stride * 2u + col;
    }
    tile_bytes = (unsigned)TILE * (unsigned)row_stride * 2u;
    wave_lds = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 1024;
  }
  // tile: index of the 64-row tile counted from g; lds: where it goes (all uniform)
  __device__ __forceinline__ void issue(const bf16_t* g, int tile, unsigned lds) const {
    const unsigned t0 = (unsigned)tile * tile_bytes;
#pragma unroll
    for (int i = 0; i < N; ++i)
      asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                   :
                   : "v"(min(t0 + ofs[i], last[i])), "s"(g), "s"(lds + wave_lds + i * 4096)
                   : "memory", "m0");
  }
};
// at most the N youngest of this wavefront's loads are still on their way
template <int N>
__device__ __forceinline__ void wait_tiles() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// The same placement through registers: requested (fetch) ahead of a step, put into LDS (stash) behind it.
template <int D>
struct RegCopy {
  static constexpr int N = TileCopy<D>::N;
  bf16x8 v[N];
  __device__ __forceinline__ void fetch(const TileCopy<D>& c, const bf16_t* g, int tile) {
    const unsigned t0 = (unsigned)tile * c.tile_bytes;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = *(const bf16x8*)((const char*)g + min(t0 + c.ofs[i], c.last[i]));
  }
  __device__ __forceinline__ void stash(unsigned lds) const {
    typedef __attribute__((address_space(3))) bf16x8* lds_ptr;
#pragma unroll
    for (int i = 0; i < N; ++i) *(lds_ptr)(lds + i * 4096) = v[i];
  }
};

// Addresses of the operand fragments.  Tiles are 256-byte aligned and the placement moves bits 4 to 7 only, so a fragment's
// address is the slot's + (row 0, this lane's chunk ^ chunk) + an immediate offset for the tile in the slot and the row.
// HELD: one register per chunk, and with slots that are constants (for_each_tile) no address arithmetic in a step: the
// forward 0.94 to 0.98 of the time with addresses formed in each.  The backward passes, where registers are short, form
// them from chunk 0, once for both tiles of a slot (held there: 1.02 to 1.08 of the time, from other schedules and spills).
template <int D, bool HELD>
struct FragAddr {
  unsigned k[HELD ? D / 16 : 1];       // frag_k at row 0
  unsigned tr[HELD ? D / 32 : 1][2];   // frag_tr at row 0: its two halves
  __device__ __forceinline__ void init(unsigned ring) {
    const int l = threadIdx.x & 63, i = l & 15, q = 4 * (l >> 5) + (i >> 2);
    const int ch = ((l >> 4) & 1) * 2 + ((i & 3) >> 1);
#pragma unroll
    for (int ks = 0; ks < (HELD ? D / 16 : 1); ++ks)
      k[ks] = ring + (l & 31) * D * 2 + ((((l >> 5) ^ swz<D>(l & 31)) ^ (2 * ks)) << 4);
#pragma unroll
    for (int dt = 0; dt < (HELD ? D / 32 : 1); ++dt)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        tr[dt][h] = ring + (q + 8 * h) * D * 2 + (((ch ^ swz<D>(q + 8 * h)) ^ (4 * dt)) << 4) + (i & 1) * 8;
  }
  // Operand fragment with the contraction index contiguous in LDS: lane l holds
  // row row_base + l%32, contraction elements 16*ks + 8*(l/32) .. +7.
  __device__ __forceinline__ bf16x8 frag_k(unsigned slot, unsigned tile, int row_base, int ks) const {
    typedef __attribute__((address_space(3))) const bf16x8* lds_ptr;
    const unsigned at = HELD ? k[HELD ? ks : 0] + slot : (k[0] + slot) ^ (ks << 5);
    return *(lds_ptr)(at + (tile + row_base * D * 2));
  }
  // Operand fragment with the contraction index running over LDS rows (transposing
  // load): lane l holds column 32*dt + l%32; its 8 contraction slots are rows
  // kbase + 4*(l/32) + {0..3} and kbase + 8 + 4*(l/32) + {0..3} -- the order in
  // which a 32x32 accumulator tile hands 8 of a lane's 16 values to the next MFMA.
  __device__ __forceinline__ bf16x8 frag_tr(unsigned slot, unsigned tile, int dt, int kbase) const {
    typedef __attribute__((address_space(3))) short4_t* lds_ptr;
    union { short4_t s4[2]; bf16x8 b; } u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const unsigned at = HELD ? tr[HELD ? dt : 0][h] + slot : (tr[0][h] + slot) ^ (dt << 6);
      u.s4[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + (tile + kbase * D * 2)));
    }
    return u.b;
  }
};
// step(t, slot) for t = 0 .. nt - 1, slot = t mod 2 as a constant
template <typename STEP>
__device__ __forceinline__ void for_each_tile(int nt, STEP step) {
  for (int t = 0; t < nt; t += 2) {
    step(t, 0);
    if (t + 1 < nt) step(t + 1, 1);
  }
}
// registers 8*half .. 8*half+7 of an accumulator tile as a bf16 operand fragment
__device__ __forceinline__ bf16x8 pack8(const f32x16& t, int half) {
  bf16x8 o;
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = (bf16_t)t[8 * half + j];
  return o;
}
// the value the lane 32 places away holds (v_permlane32_swap: no trip through LDS)
__device__ __forceinline__ float other_half(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  // r[0]: lanes 0..31 keep theirs, lanes 32..63 receive the lower half's; r[1]: the other way round
  const unsigned lo = r[0], hi = r[1];
  return __builtin_bit_cast(float, (threadIdx.x & 32) ? lo : hi);
}
// row index inside a 32x32 accumulator tile of register r for this lane
__device__ __forceinline__ int acc_row(int r) { return 8 * (r >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (r & 3); }

}  // namespace bamboo
