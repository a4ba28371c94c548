// attention_items.h -- which rows and keys a workgroup of the attention kernels takes:
// the device's division of a batch into items, from lengths that only the GPU knows.
#ifndef EB_ATTENTION_ITEMS_H
#define EB_ATTENTION_ITEMS_H

#include <hip/hip_runtime.h>

#include "attention.h"

namespace eb {
namespace {

struct Item {
  int32_t b = -1;         // sequence, -1: none
  int32_t split = 0, splits = 1;
  int32_t q0 = 0, n = 0;  // first row of q, new tokens to compute
  int32_t p0 = 0;         // place of the first new token
  int32_t kv = 0;
  int32_t rows = 0;       // of the tile
  uint32_t tiles = 0;     // of the sequence
  int32_t tok0 = 0, head0 = 0;  // of the tile's first row
};

struct Seq {
  int32_t q0, n, p0, kv, tiles, units;
};

__device__ inline Seq seq_of(const AttnArgs &a, int32_t b) {
  const eb_attention_op &o = a.o;
  Seq s;
  const int32_t r0 = min(max(o.q_start[b], 0), o.rows), r1 = min(max(o.q_start[b + 1], r0), o.rows);
  s.kv = min(max(o.kv_len[b], 0), a.kv_max);
  s.q0 = r0;
  s.p0 = s.kv - (r1 - r0);
  s.n = min(r1 - r0, o.max_new);
  s.tiles = (s.n * a.group + a.tile_rows - 1) / a.tile_rows;
  // units of keys that a tile may see
  int32_t see = s.kv;
  if (o.window > 0 && o.window < see && o.mask != EB_MASK_FULL && !o.prefix)
    see = min(see, o.window + a.tile_rows);
  s.units = (see + a.unit - 1) / a.unit;
  return s;
}

// Units of a split, of `units` units in all tiles of several sequences, `longest` of
// them in one: so that the splits of all together are about a.target, and none where
// the tiles are so alike that the GPU is busy to their end.
__device__ inline uint32_t units_per_split(const AttnArgs &a, float units, int32_t longest) {
  // exact below 2^24
  const uint32_t per = units < 16777216.f ? ((uint32_t)units + a.target - 1) / a.target
                                          : (uint32_t)(units / a.target) + 2;
  return max(max(per, (uint32_t)a.min_units), (float)longest <= a.even * units ? (uint32_t)longest : 0u);
}

// Item number `at` of a key/value head.  A sequence's items are the tiles of its first
// split, those of its second and so on, so that neighbours read the same keys.  JOIN: item
// `at` of the tiles with several splits, *base the item of its first split.  One sequence is
// split as often as fits a.target items; of several, each into splits of
// units_per_split units, so that a longer one gets more.  Every wave of every
// workgroup finds the same numbers from the lengths; of more than kScanBatch
// sequences attn_items_kernel has found them.
template <bool JOIN>
__device__ inline Item find_item(const AttnArgs &a, uint32_t at, uint32_t *base = nullptr) {
  const eb_attention_op &o = a.o;
  const int lane = threadIdx.x & 63;
  auto uni = [](int32_t v) { return __builtin_amdgcn_readfirstlane(v); };
  Item it;
  Seq s{};
  uint32_t rest = at, first = 0, splits = 1;
  if (o.batch == 1) {
    s = seq_of(a, 0);
    if (a.target > 0) {
      const int32_t most = min(a.target / max(s.tiles, 1), s.units / a.min_units);
      if (most > 1) {
        const int32_t per = (s.units + most - 1) / most;
        splits = (s.units + per - 1) / per;
      }
    }
    if (at >= s.tiles * (JOIN ? 1 : splits) || (JOIN && splits == 1)) return it;
    it.b = 0;
    it.splits = uni(splits);
  } else if (o.batch > kScanBatch) {
    const int4 e = (JOIN ? a.tile_table : a.item_table)[at];
    it.b = uni(e.x);
    if (it.b < 0) return it;
    s = seq_of(a, it.b);
    it.splits = max(uni(e.w), 1);
    rest = JOIN ? e.y : e.z * s.tiles + e.y;
    first = JOIN ? e.z : 0;
  } else {
    uint32_t per = 1;
    if (a.target > 0) {
      float units = 0.f;
      int32_t longest = 0;
      if (lane < o.batch) {
        s = seq_of(a, lane);
        units = (float)s.tiles * (float)s.units;
        longest = s.tiles > 0 ? s.units : 0;
      }
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) {
        units += __shfl_xor(units, d);
        longest = max(longest, __shfl_xor(longest, d));
      }
      per = units_per_split(a, units, longest);
    }
    uint32_t items = 0, tiles = 0;
    if (lane < o.batch) {
      if (a.target <= 0) s = seq_of(a, lane);  // (else it is here already)
      splits = a.target > 0 && s.units > 0 ? (s.units + per - 1) / per : 1;
      items = s.tiles * splits;
      tiles = splits > 1 ? s.tiles : 0;
    }
    uint32_t sum = items, count = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t u = __shfl_up(sum, d), v = JOIN ? __shfl_up(count, d) : 0;
      if (lane >= d) sum += u, count += v;
    }
    const uint64_t past = __ballot((JOIN ? count : sum) > rest);
    if (!past) return it;
    const int src = __builtin_ctzll(past);
    auto from = [&](int32_t v) { return __builtin_amdgcn_readlane(v, src); };
    if (JOIN) first += from(sum - items);
    rest -= from(JOIN ? count - tiles : sum - items);
    s.q0 = from(s.q0);
    s.n = from(s.n);
    s.p0 = from(s.p0);
    s.kv = from(s.kv);
    s.tiles = from(s.tiles);
    it.splits = from(splits);
    it.b = src;
  }
  const uint32_t tiles = uni(s.tiles), r = uni(rest), split = JOIN ? 0 : r / max(tiles, 1u);
  const uint32_t tile = r - split * tiles;
  it.split = (int32_t)split;
  it.tiles = tiles;
  if (JOIN) *base = first;
  it.q0 = uni(s.q0);
  it.n = uni(s.n);
  it.p0 = uni(s.p0);
  it.kv = uni(s.kv);
  // Under a causal mask the last tile of one sequence sees most keys and begins first
  // (4096 x 4096, 24 heads: 157 -> 134 us; in ragged batches it cost 2 us of 18).
  if (tile >= tiles || it.split >= it.splits) {  // (offsets that are none: sequences that overlap without end)
    it.b = -1;
    return it;
  }
  if (JOIN) *base += tile;
  const uint32_t row0 = (o.batch > 1 || o.mask == EB_MASK_FULL ? tile : tiles - 1 - tile) * a.tile_rows;
  it.rows = min(a.tile_rows, (int32_t)(it.n * a.group - row0));
  it.tok0 = uni(row0 / a.group);
  it.head0 = uni(row0 - it.tok0 * a.group);
  return it;
}

}  // namespace
}  // namespace eb

#endif  // EB_ATTENTION_ITEMS_H
