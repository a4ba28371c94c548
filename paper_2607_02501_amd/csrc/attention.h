// attention.h -- declarations shared by the translation units of the steps
// between a layer's QKV and O projections (include/eb_attention.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/eb_attention.h"

namespace eb {

constexpr int kMaxBatch = 4096;
constexpr int kMaxSplits = 1024;  // of a row tile
constexpr int kScanBatch = 64;    // sequences that every wave looks over itself (attn_items_kernel)

hipError_t launch_kv_extend(const eb_kv_extend_op &o, hipStream_t s);
hipError_t launch_rope_append(const eb_rope_append_op &o, hipStream_t s);
size_t attention_ws_bytes(const eb_attention_op &o);
void attention_plan(const eb_attention_op &o, int32_t *tile_rows, int32_t *splits);
hipError_t launch_attention(const eb_attention_op &o, void *ws, hipStream_t s);

// Splits of a tile up to which the join takes whole rows (attn_join_kernel): 7 splits of 50
// tokens, 12.1 us so and 14.2 by workgroups; 63 splits of one token, 21.4 and 16.1.
constexpr int kJoinRows = 16;

// What the attention kernels take beside the op itself.
struct AttnArgs {
  eb_attention_op o;
  float *ws;           // sums of splits
  int4 *item_table;    // batch > kScanBatch: items' (sequence or -1, tile, split, splits)
  int4 *tile_table;    // and split tiles' (sequence or -1, tile, first item, splits)
  int64_t head_rows;   // cache rows of a page: heads * page
  int32_t page_shift;
  int32_t kv_max;      // keys of a table row
  int32_t group;       // query heads per key/value head
  int32_t tile_rows;   // 128: the tile kernel, 32: the stream kernel
  int32_t unit;        // keys that splits are counted in
  int32_t min_units;   // of a split
  int32_t target;      // items of a key/value head that splits may add; 0: no splits
  int32_t part_rows;   // rows of a tile that a split may have sums of
  int32_t join_tiles;  // row tiles of a key/value head that may be split: at most target
  int32_t join_splits; // of one of them, at most about
  float even;          // a batch whose longest tile is at most this part of all is not split
  uint32_t tiles;      // row tiles of all sequences, at most
  uint32_t items;      // of a key/value head, at most: tiles + target
  uint32_t grid;       // items of all heads
  uint32_t grid_wgs;   // workgroups: grid rounded up to the XCDs
  bool spread;         // one row tile a sequence: workgroups in order of item
  uint32_t flip;       // sign bits of a pair of queries where the scale is negative
  float scale2;        // 2^(scale2 s) without a cap; 2^(scale2 s) = e^(2 scale s / cap) with one
  float cap2;          // cap * log2 e, 0 without a cap
};

// The kernels of one cache type (attention_bf16.hip, attention_f16.hip).
template <int T>
hipError_t attn_launch(const AttnArgs &a, hipStream_t s);

}  // namespace eb
