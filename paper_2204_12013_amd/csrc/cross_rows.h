// What the kernels of the attention over an encoder's states share: which rows and keys a workgroup works on.
//
// The query heads that share a key head are rows of one problem: row r of the pair (sample, key head) is query
// r / group, head key_head * group + r % group, so that a tile of keys is fetched once for all of them and their gradients
// are summed where they arise.  Keys behind a sample's length are never read: tiles end at the last one that counts.
#pragma once
#include "common.h"

namespace bamboo {

struct CrossRow { int query, head; };
__device__ __forceinline__ CrossRow cross_row(const CrossDesc& a, int kvh, int r) {
  CrossRow o;
  o.query = a.group == 1 ? r : (int)__umulhi((unsigned)r, a.group_inv);     // r * group < 2^32
  o.head = kvh * a.group + (r - o.query * a.group);
  return o;
}
// index into lse and delta, both [sample, head, query]
__device__ __forceinline__ long cross_stat(const CrossDesc& a, int b, const CrossRow& r) {
  return ((long)b * a.heads + r.head) * a.sq + r.query;
}
__device__ __forceinline__ int cross_len(const CrossDesc& a, int b) {
  return a.kv_len == nullptr ? a.sk : min(max(a.kv_len[b], 0), a.sk);
}
// Workgroup -> (block of owned rows, part of the streamed side, pair); the pairs of a block and part are consecutive.
struct CrossBlock { int blk, split, pair, b, kvh; };
__device__ __forceinline__ CrossBlock cross_block(const CrossDesc& a) {
  const int pairs = a.B * a.kv_heads;
  CrossBlock o;
  o.pair = (int)blockIdx.x % pairs;
  const int rest = (int)blockIdx.x / pairs;
  o.split = rest % a.splits;
  o.blk = rest / a.splits;
  o.b = o.pair / a.kv_heads;
  o.kvh = o.pair % a.kv_heads;
  return o;
}
// the part's range of 64-row tiles of n streamed rows
__device__ __forceinline__ void cross_part(int n, int splits, int split, int* first, int* last) {
  const int tiles = (n + 63) / 64, per = (tiles + splits - 1) / splits;
  *first = min(tiles, split * per);
  *last = min(tiles, *first + per);
}

}  // namespace bamboo
