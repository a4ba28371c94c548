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
// attention kernels would take 0.4 us for every 64 sequences (single tokens of 1000
// sequences: 127 us, 206 if every wave looks them over; of 4000, 352 and 1590).  Up to
// kScanBatch = 64 a wave looks them over in one step, which is less than another launch
// (500 keys each, 2 sequences: 11.0 us, with tables 13.2; 64 sequences: 28.7, 32.5).
constexpr int kItemThreads = 512;
__global__ void __launch_bounds__(kItemThreads) attn_items_kernel(AttnArgs a) {
  __shared__ uint32_t items[kMaxBatch + 1], tiles[kMaxBatch + 1];
  __shared__ uint32_t red[2][kItemThreads / 64];
  __shared__ float unit_red[kItemThreads / 64];
  __shared__ int32_t long_red[kItemThreads / 64];
  const int32_t batch = a.o.batch, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  uint32_t per = 1;
  if (a.target > 0) {
    float units = 0.f;
    int32_t longest = 0;
    for (int32_t b = threadIdx.x; b < batch; b += kItemThreads) {
      const Seq s = seq_of(a, b);
      units += (float)s.tiles * (float)s.units;
      longest = max(longest, s.tiles > 0 ? s.units : 0);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
      units += __shfl_xor(units, d);
      longest = max(longest, __shfl_xor(longest, d));
    }
    if (lane == 0) unit_red[wv] = units, long_red[wv] = longest;
    __syncthreads();
    units = 0.f;
    for (int w = 0; w < kItemThreads / 64; ++w) units += unit_red[w], longest = max(longest, long_red[w]);
    per = units_per_split(a, units, longest);
  }
  // (sums stop at 2^30: offsets that overlap without end may ask for more)
  auto splits_of = [&](const Seq &s) { return a.target > 0 && s.units > 0 ? (s.units + per - 1) / per : 1u; };
  auto most = [](uint32_t x, uint32_t y) { return min(x + y, 1u << 30); };
  uint32_t item0 = 0, tile0 = 0;
  for (int32_t b0 = 0; b0 < batch; b0 += kItemThreads) {
    const int32_t b = b0 + (int32_t)threadIdx.x;
    uint32_t n = 0, t = 0;
    if (b < batch) {
      const Seq s = seq_of(a, b);
      const uint32_t splits = splits_of(s);
      n = min(s.tiles * splits, 1u << 30);
      t = splits > 1 ? s.tiles : 0;
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
      const Seq s = seq_of(a, b);
      const uint32_t r = at - items[b], n = max(s.tiles, 1);
      e = make_int4(b, r % n, r / n, splits_of(s));
    }
    a.item_table[at] = e;
  }
  for (uint32_t at = at0; at < (uint32_t)a.join_tiles; at += step) {
    int4 e = make_int4(-1, 0, 0, 1);
    if (at < tile0) {
      const int32_t b = find(tiles, at);
      e = make_int4(b, at - tiles[b], items[b], splits_of(seq_of(a, b)));
    }
    a.tile_table[at] = e;
  }
}

// What a unit of keys (128 of the stream kernel, 64 of the tile kernel) takes a workgroup
// that has its CU to itself, and a CU whose slots are full, in us: from chunks of 16 to
// 1024 tokens after 1500 to 16000 keys, unsplit on few CUs and on all, causal and without a
// cap.  A split's sums are written and read at kSumBytesPerUs, its join takes kJoinUs beside.
// Outside that range they are extrapolated: 816 capped rows of 8 heads of 256 behind a
// prefix, 8.7 us by these paces, take 19.  The factors in plan (half the bound of a batch's
// lengths, 0.75 of a full CU's pace for tiles that share it, half the longest tile after the
// rest) and `even` below are set by the cases named there and the ones in the table.
struct Pace {
  float alone, full;
};
constexpr Pace kPace[2][3] = {{{0.71f, 0.48f}, {0.95f, 0.85f}, {1.24f, 1.24f}},   // 32 rows; dim 64, 128, 256
                              {{0.82f, 0.64f}, {1.09f, 1.07f}, {1.99f, 2.10f}}};  // 128 rows
constexpr double kBytesPerUs = 5.2e6, kSumBytesPerUs = 1.2e6, kJoinUs = 4.;

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
    // a negative scale is a sign on the queries; in place of a scale of 0, which would make
    // NaN of a hidden key's -infinity, the least above it: no finite score times it is over
    // 2^-21
    a.flip = o.scale < 0.f ? 0x80008000u : 0u;
    a.scale2 = o.scale == 0.f ? 0x1p-149f : (o.scale < 0.f ? -o.scale : o.scale) * kLog2e;
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
  // Kernel and splits: the least time by the paces above, of the two kernels, each
  // without splits and with the number of pieces whose sums cost least.  Tiles of 32 rows
  // are shorter and more, those of 128 read keys from L2 and LDS a quarter as often, and
  // splits pay where tiles are few and keys many.  Measured, causal, 8 key/value and 32
  // query heads of 128, us (32 rows whole, in pieces; 128 rows whole, in pieces):
  //   256 tokens, no others      9.3   19    12.0    -        chosen: 9.3
  //   2048 tokens, no others     69    81    53      65       52.7
  //   1 token, 8000 keys         60    15.8   -      -        15.8
  //   64 tokens, 1500 keys       18.0  15.6  33.3    20.2     15.6
  //   256 tokens, 16000 keys     137   104   273     85       88
  //   1024 tokens, 16000 keys    337   337   285     261      290 (the estimate has it shorter)
  double best = 0.;
  for (int32_t tile_rows = 32; tile_rows <= (rows <= 32 ? 32 : 128); tile_rows += 96) {
    const Pace pace = kPace[tile_rows == 128][o.cache.dim / 128];
    const int64_t tiles = tiles_of(tile_rows), unit = tile_rows == 32 ? 128 : 64;
    const int32_t part_rows = (int32_t)(rows < tile_rows ? rows : tile_rows);
    int64_t see = o.max_kv > 0 ? o.max_kv : 1;
    double mean = (double)see - (o.mask == EB_MASK_FULL || o.prefix ? 0. : 0.5 * max_new);  // keys of a row
    if (o.window > 0 && o.mask != EB_MASK_FULL && !o.prefix && see > (int64_t)o.window + tile_rows)
      see = (int64_t)o.window + tile_rows;
    if (mean > see) mean = (double)see;
    if (mean < 1.) mean = 1.;
    if (o.batch > 1) mean *= 0.5;  // (lengths are known to the GPU alone)
    const double slots = (double)(cus * (o.cache.dim == 256 ? 1 : o.cache.dim == 64 && tile_rows == 32 ? 3 : 2));
    const double wgs = (tiles - 0.5 * (o.batch - 1)) * heads, units = (double)((see + unit - 1) / unit);
    // of the CUs together, and of the longest tile
    const double compute = wgs * mean / unit * pace.full / cus;
    const double memory = (double)o.batch * heads * mean * o.cache.dim * 4. / kBytesPerUs;
    const double work = compute > memory ? compute : memory;
    const double shared = 0.75 * pace.full * (wgs < slots ? wgs : slots) / cus;
    const double longest = units * (shared > pace.alone ? shared : pace.alone);
    // (several sequences: the longest may begin when others have ended.  Single tokens of
    // 64 sequences of 30 to 16000 keys: 272 us whole, 152 in pieces; of 4000 keys each: 185,
    // 191 with a join that finds nothing to do.)
    const double whole = o.batch > 1 ? work + 0.5 * longest : work > longest ? work : longest;
    // With splits: pieces of all tiles, each of which writes its sums once.
    const double sums = part_rows * (o.cache.dim + 2) * 4. / kSumBytesPerUs;
    const double all = (o.batch > 1 ? wgs * mean / unit : wgs * units) * pace.alone;
    double pieces = slots;
    if (pieces * pieces * sums > all) pieces = __builtin_sqrt(all / sums);
    // (one workgroup a CU reaches the copy rate: 131071 keys of one head of 256, 256 pieces
    // 35 us, 97 of them 43; of 128, 256 pieces 21.9 us, 512 of them 24.7)
    if (o.batch == 1 && memory > compute && pieces > cus) pieces = (double)cus;
    int64_t target = (int64_t)(pieces / heads);
    if (target > kMaxSplits) target = kMaxSplits;
    if (tile_rows == 128 && target > tiles * kJoinRows) target = tiles * kJoinRows;
    if (o.batch == 1) target = target / tiles * tiles;  // the same number of splits for all
    double split = whole + 1.;
    if (target > (o.batch > 1 ? 0 : tiles)) {
      const double piece = all / (target * heads);
      split = (work > piece ? work : piece) + kJoinUs + target * heads * sums;
    }
    const double time = split < whole ? split : whole;
    if (tile_rows > 32 && time >= best) break;
    best = time;
    a.tile_rows = tile_rows;
    a.unit = (int32_t)unit;
    a.min_units = tile_rows == 32 ? 1 : 4;  // (16 tokens, 1500 keys: with 16 units 34 us, 14.4)
    a.part_rows = part_rows;
    a.tiles = (uint32_t)tiles;
    a.target = split < whole ? (int32_t)target : 0;
    a.join_splits = (int32_t)(o.batch > 1 ? target : target / tiles);
  }
  // (half of what a CU gets on average: single tokens of 128 sequences of 30 to 4000 keys,
  // 99 us, with 1.25 of it 104; to 1500 keys, 56 and 54)
  a.even = 0.6f * (float)heads / (float)cus;
  a.join_tiles = a.target < (int64_t)a.tiles ? a.target : (int32_t)a.tiles;
  a.items = o.batch > 1 ? a.tiles + (uint32_t)a.target : a.target > 0 ? (uint32_t)a.target : a.tiles;
  // In order over the XCDs, or a run of neighbours to each: single tiles share no keys;
  // under a causal mask or of ragged sequences, runs are of unequal work unless each XCD
  // gets whole heads (causal, 4096 tokens, one head of 256: 126 us spread, 185 in runs;
  // 8 heads of 128: 148 either way).
  a.spread = rows <= a.tile_rows ||
             (heads % 8 != 0 && (o.batch > 1 || (a.target == 0 && o.mask != EB_MASK_FULL && !o.prefix)));
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
  return a.o.batch > kScanBatch ? ((size_t)a.items + a.join_tiles + 15) / 16 * 16 * sizeof(int4) : 0;
}

size_t attention_ws_bytes(const eb_attention_op &o) {
  const AttnArgs a = plan(o);
  return sums_bytes(a) + table_bytes(a);
}

void attention_plan(const eb_attention_op &o, int32_t *tile_rows, int32_t *splits) {
  const AttnArgs a = plan(o);
  *tile_rows = a.tile_rows;
  *splits = a.target;
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
