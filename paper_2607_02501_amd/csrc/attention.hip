// attention.hip -- how attention over a paged cache is launched: the kernel, its
// tiles and the split of keys (include/eb_attention.h, attention_tile.h).
#include <hip/hip_runtime.h>

#include "attention.h"
#include "attention_items.h"
#include "eb_internal.h"

namespace eb {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// The tables of a batch of more than kScanBatch sequences.  As in eb_kv_extend, each
// workgroup sums over the whole batch itself and then fills its part: a wave of the
// attention kernels would take 0.4 us for every 64 sequences (4000 of them: 25 us each).
constexpr int kItemThreads = 512;
__global__ void __launch_bounds__(kItemThreads) attn_items_kernel(AttnArgs a) {
  __shared__ uint32_t items[kMaxBatch + 1], tiles[kMaxBatch + 1];
  __shared__ uint32_t red[2][kItemThreads / 64];
  __shared__ float unit_red[kItemThreads / 64];
  const int32_t batch = a.o.batch, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  uint32_t per = 1;
  if (a.target > 0) {
    float units = 0.f;
    for (int32_t b = threadIdx.x; b < batch; b += kItemThreads) {
      const Seq s = seq_of(a, b);
      units += (float)s.tiles * (float)s.units;
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) units += __shfl_xor(units, d);
    if (lane == 0) unit_red[wv] = units;
    __syncthreads();
    units = 0.f;
    for (int w = 0; w < kItemThreads / 64; ++w) units += unit_red[w];
    per = units_per_split(a, units);
  }
  // (sums stop at 2^30: offsets that overlap without end may ask for more)
  auto most = [](uint32_t x, uint32_t y) { return min(x + y, 1u << 30); };
  uint32_t item0 = 0, tile0 = 0;
  for (int32_t b0 = 0; b0 < batch; b0 += kItemThreads) {
    const int32_t b = b0 + (int32_t)threadIdx.x;
    uint32_t n = 0, t = 0;
    if (b < batch) {
      const Seq s = seq_of(a, b);
      t = s.tiles;
      n = min(t * (a.target > 0 && s.units > 0 ? (s.units + per - 1) / per : 1), 1u << 30);
    }
    uint32_t sn = n, st = t;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t u = __shfl_up(sn, d), v = __shfl_up(st, d);
      if (lane >= d) sn = most(sn, u), st = most(st, v);
    }
    __syncthreads();
    if (lane == 63) red[0][wv] = sn, red[1][wv] = st;
    __syncthreads();
    uint32_t bn = item0, bt = tile0;
    for (int w = 0; w < kItemThreads / 64; ++w) {
      if (w < wv) bn = most(bn, red[0][w]), bt = most(bt, red[1][w]);
      item0 = most(item0, red[0][w]), tile0 = most(tile0, red[1][w]);
    }
    if (b < batch) items[b] = most(bn, sn - n), tiles[b] = most(bt, st - t);
  }
  if (threadIdx.x == 0) items[batch] = item0, tiles[batch] = tile0;
  __syncthreads();
  auto find = [&](const uint32_t *sums, uint32_t v) {  // the last b with sums[b] <= v
    int32_t lo = 0, hi = batch;
    while (hi - lo > 1) {
      const int32_t mid = (lo + hi) >> 1;
      if (sums[mid] <= v)
        lo = mid;
      else
        hi = mid;
    }
    return lo;
  };
  const uint32_t step = gridDim.x * kItemThreads, at0 = blockIdx.x * kItemThreads + threadIdx.x;
  for (uint32_t at = at0; at < a.items; at += step) {
    int4 e = make_int4(-1, 0, 0, 1);
    if (at < item0) {
      const int32_t b = find(items, at);
      const uint32_t t = tiles[b + 1] - tiles[b], splits = (items[b + 1] - items[b]) / max(t, 1u);
      const uint32_t r = at - items[b];
      e = make_int4(b, r / max(splits, 1u), r % max(splits, 1u), splits);
    }
    a.item_table[at] = e;
  }
  for (uint32_t at = at0; at < a.tiles; at += step) {
    int4 e = make_int4(-1, 0, 0, 1);
    if (at < tile0) {
      const int32_t b = find(tiles, at);
      const uint32_t t = tiles[b + 1] - tiles[b], splits = (items[b + 1] - items[b]) / max(t, 1u);
      const uint32_t r = at - tiles[b];
      e = make_int4(b, r, items[b] + r * splits, splits);
    }
    a.tile_table[at] = e;
  }
}

AttnArgs plan(const eb_attention_op &o) {
  AttnArgs a{};
  a.o = o;
  a.page_shift = __builtin_ctz((unsigned)o.cache.page);
  a.head_rows = (int64_t)o.cache.heads << a.page_shift;
  a.kv_max = o.table_stride << a.page_shift;
  a.group = o.q_heads / o.cache.heads;
  if (o.softcap > 0.f) {
    a.scale2 = 2.f * kLog2e * o.scale / o.softcap;
    a.cap2 = o.softcap * kLog2e;
  } else {
    // a negative scale is a sign on the queries; with a scale of 0 every score
    // becomes 0 times a number that a hidden key's -infinity outweighs
    a.flip = o.scale < 0.f ? 0x80008000u : 0u;
    a.scale2 = o.scale == 0.f ? 1e-30f : (o.scale < 0.f ? -o.scale : o.scale) * kLog2e;
  }
  const int64_t max_new = o.max_new < o.rows ? o.max_new : o.rows;
  const int64_t rows = max_new * a.group;  // of a sequence and key/value head
  const int64_t heads = o.cache.heads, cus = device_cu_count();
  // row tiles of all sequences, at most
  auto tiles_of = [&](int64_t tile_rows) {
    const int64_t each = o.batch * ((rows + tile_rows - 1) / tile_rows);
    const int64_t packed = (int64_t)o.rows * a.group / tile_rows + o.batch;
    return o.batch > 1 && packed < each ? packed : each;
  };
  a.tile_rows = rows <= 32 || tiles_of(128) * heads < cus ? 32 : 128;
  const int64_t tiles = tiles_of(a.tile_rows);
  a.part_rows = (int32_t)(rows < a.tile_rows ? rows : a.tile_rows);
  // Splits of the keys: where the tiles alone leave workgroup slots idle, or one
  // sequence of a batch may be far longer than the others.
  // (workgroups on a CU: see kStreamWgs and the tile kernel's launch bounds)
  const int64_t slots = cus * (o.cache.dim == 256 ? 1 : o.cache.dim == 64 && a.tile_rows == 32 ? 3 : 2);
  a.unit = a.tile_rows == 32 ? 128 : 64;
  a.min_units = a.tile_rows == 32 ? 1 : 16;
  int64_t see = o.max_kv;
  if (o.window > 0 && o.mask != EB_MASK_FULL && !o.prefix && see > (int64_t)o.window + a.tile_rows)
    see = (int64_t)o.window + a.tile_rows;
  const int64_t units = (see + a.unit - 1) / a.unit;
  if (tiles * heads * 2 <= slots ? units > a.min_units : o.batch > 1 && units > 16) {
    const int64_t target = (slots + heads - 1) / heads;
    a.target = (int32_t)(target < kMaxSplits ? target : kMaxSplits);
  }
  a.tiles = (uint32_t)tiles;
  a.spread = rows <= a.tile_rows;
  a.items = (uint32_t)(tiles + a.target);
  const int64_t grid = (int64_t)a.items * heads;
  a.grid = (uint32_t)grid;
  a.grid_wgs = (uint32_t)((grid + 7) / 8 * 8);
  return a;
}

}  // namespace

// The workspace: sums of splits, then the tables of a large batch.
static size_t sums_bytes(const AttnArgs &a) {
  if (a.target <= 0) return 0;
  const size_t bytes = (size_t)a.grid * (size_t)a.part_rows * (size_t)(a.o.cache.dim + 2) * 4;
  return (bytes + 255) / 256 * 256;
}

static size_t table_bytes(const AttnArgs &a) {
  return a.o.batch > kScanBatch ? ((size_t)a.items + a.tiles + 15) / 16 * 16 * sizeof(int4) : 0;
}

size_t attention_ws_bytes(const eb_attention_op &o) {
  const AttnArgs a = plan(o);
  return sums_bytes(a) + table_bytes(a);
}

hipError_t launch_attention(const eb_attention_op &o, void *ws, hipStream_t s) {
  AttnArgs a = plan(o);
  a.ws = static_cast<float *>(ws);
  if (o.batch > kScanBatch) {
    a.item_table = reinterpret_cast<int4 *>(static_cast<uint8_t *>(ws) + sums_bytes(a));
    a.tile_table = a.item_table + a.items;
    const uint32_t wgs = (a.items + kItemThreads - 1) / kItemThreads;
    attn_items_kernel<<<wgs < 64 ? wgs : 64, kItemThreads, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return o.cache.type == EB_F16 ? attn_launch<EB_F16>(a, s) : attn_launch<EB_BF16>(a, s);
}

}  // namespace eb
