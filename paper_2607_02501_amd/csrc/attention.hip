// attention.hip -- how attention over a paged cache is launched: the kernel, its
// tiles and the split of keys (include/eb_attention.h, attention_tile.h).
#include <hip/hip_runtime.h>

#include "attention.h"
#include "eb_internal.h"

namespace eb {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

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

size_t attention_ws_bytes(const eb_attention_op &o) {
  const AttnArgs a = plan(o);
  if (a.target <= 0) return 0;
  const size_t bytes = (size_t)a.grid * (size_t)a.part_rows * (size_t)(o.cache.dim + 2) * 4;
  return (bytes + 255) / 256 * 256;
}

hipError_t launch_attention(const eb_attention_op &o, void *ws, hipStream_t s) {
  AttnArgs a = plan(o);
  a.ws = static_cast<float *>(ws);
  return o.cache.type == EB_F16 ? attn_launch<EB_F16>(a, s) : attn_launch<EB_BF16>(a, s);
}

}  // namespace eb
