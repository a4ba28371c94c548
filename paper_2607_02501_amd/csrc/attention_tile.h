// attention_tile.h -- attention of new tokens over a paged cache on the matrix
// cores: the kernels behind eb_attention (include/eb_attention.h), instantiated
// for each cache type in its own translation unit.
//
// Rows.  The query heads of one key/value head and the new tokens of a sequence
// form its rows: row R is token R / group, head R % group of the group.  A
// workgroup of four waves takes a tile of rows of one sequence and key/value head
// and a range of its keys; a wave takes 32 rows.
//
// Products.  S^T = K Q^T, so that a lane holds the scores of one row (column
// lane % 32 of the 32 x 32 result) and softmax statistics need no more than one
// exchange with lane ^ 32; then O^T += V^T P^T, whose P^T operand is the scores'
// own registers: result register i of lane half h is key 8 (i / 4) + 4 h + i % 4,
// and the order of the 16 keys of a product's contraction is free, so V^T is
// read in that order (transposing LDS reads, 4 keys of one element per lane) and
// no score changes lanes.
//
// Softmax.  One pass, with a running maximum m and sum l per row in fp32; p =
// 2^((s - m) c + lift).  m is raised, and O and l rescaled, only when a row's
// maximum has grown by more than a factor 2^late in p: p then stays below
// 2^(late + lift), and most tiles skip the rescale.  p enters the product rounded to
// the cache's type, since the matrix cores take two 16-bit operands (its sum l takes p
// itself).  bfloat16 has fp32's exponents: late 8, lift 0.  binary16 ends at 2^16 and
// has fewer bits below 2^-14: late 4, lift 11, so that a weight of 2^-25 of the
// row's largest is still a normal number, where without a lift one of 2^-14 was the
// last and one of 2^-26 was 0.  The lift is in O, l and the maximum that goes
// with them, so it cancels.
//
// Masks.  The keys a row sees are one interval; a tile that lies inside every
// row's interval skips the comparisons.  Keys past the sequence's end and on
// missing pages are read as zeros (buffer bounds), so what the cache holds there
// cannot reach a sum.  A key that only some rows of the tile see enters the
// product of the others with p = 0, which hides any value but infinities and
// NaN: a row whose result is not finite is computed again, key by key
// (row_again).
#ifndef EB_ATTENTION_TILE_H
#define EB_ATTENTION_TILE_H

#include <hip/hip_runtime.h>

#include "attention.h"
#include "attention_items.h"
#include "epilogue.h"
#include "mfma_common.h"

namespace eb {
namespace {

typedef short s16x4_t __attribute__((ext_vector_type(4)));

// The keys lo <= j < hi that the token at place p sees.
__device__ inline void interval(const AttnArgs &a, int32_t p, int32_t kv, int32_t prefix, int32_t &lo,
                                int32_t &hi) {
  hi = a.o.mask == EB_MASK_FULL ? kv : min(kv, max(p + 1, prefix));
  lo = a.o.window > 0 && p >= a.o.window ? p - a.o.window + 1 : 0;
}

// ---------------------------------------------------------------------------
// pages and copies to LDS
// ---------------------------------------------------------------------------

// Page numbers of 64 consecutive table entries, one per lane, and of the 64
// after them, requested while these are used: at least 1024 keys of each.
struct Pages {
  const int32_t *table;  // of the sequence
  int32_t count;         // entries that hold its keys
  int32_t pages;         // valid page numbers are below
  int32_t first;         // entry of lane 0
  int32_t now, next;
  bool holes;            // a page of `now` is missing

  __device__ int32_t load(int32_t at) const {
    const int32_t i = at + (int32_t)(threadIdx.x & 63);
    const int32_t id = i < count ? table[i] : 0;
    return id >= 0 && id < pages ? id : -1;
  }
  __device__ void begin(int32_t at) {
    first = at;
    now = load(at);
    next = load(at + 64);
    holes = __ballot(now < 0) != 0;
  }
  // Makes entry `at` (which never decreases) one of `now`'s.
  __device__ void reach(int32_t at) {
    while (at - first >= 64) {
      first += 64;
      now = next;
      next = load(first + 64);
      holes = __ballot(now < 0) != 0;
    }
  }
  __device__ int32_t id(int32_t at) const { return __builtin_amdgcn_readlane(now, at - first); }
};

// Where 16 keys (a multiple of 16 first) lie in the cache, and how many are there:
// none of a missing page, and none past the end.
struct Block {
  int64_t at;    // bytes into k or v
  int32_t rows;
};

template <int D>
__device__ inline Block block_of(const AttnArgs &a, const Pages &pg, int32_t kh, int32_t key, int32_t kv) {
  const int32_t id = pg.id(key >> a.page_shift);
  const int32_t in_page = key & (a.o.cache.page - 1);
  Block b;
  b.rows = id < 0 ? 0 : min(max(kv - key, 0), 16);
  b.at = ((int64_t)max(id, 0) * a.head_rows + ((int64_t)kh << a.page_shift) + in_page) * (D * 2);
  return b;
}

// Copies of a wave: 16 keys of D elements go to 16 LDS rows of D / 8 chunks of 16
// bytes, 1 KiB at a time; rows that are not there are zeros.  Chunk c of row r is
// stored at c ^ swizzle: for keys (read as 8 rows by one chunk) r % 8, for values
// (read as 4 rows by 2 chunks) 2 (r % 8), or 2 (r % 4) in rows of 8 chunks, so that
// a read's lanes fall on different banks.  The swizzle repeats every 8 rows, so
// D / 64 lane offsets serve all copies; one buffer descriptor serves the 16 keys
// (built for each copy, its 30 scalar instructions took 140 ns of a lone wave, four
// times what the copy does).
template <int D>
__device__ inline uint32_t k_swizzle(uint32_t r) { return r & 7; }
template <int D>
__device__ inline uint32_t v_swizzle(uint32_t r) { return (r & (D == 64 ? 3 : 7)) << 1; }

template <int D, bool V>
struct Copy {
  static constexpr int kRows = 512 / D;      // of one copy
  static constexpr int kCopies = D / 32;     // of 16 keys
  static constexpr int kOffsets = D / 64;    // copies of 8 rows
  uint32_t off[kOffsets];

  __device__ void begin() {
    const uint32_t lane = threadIdx.x & 63, lr = lane / (D / 8), lc = lane % (D / 8);
#pragma unroll
    for (int i = 0; i < kOffsets; ++i) {
      const uint32_t r = i * kRows + lr;
      off[i] = r * (D * 2) + (lc ^ (V ? v_swizzle<D>(r) : k_swizzle<D>(r))) * 16;
    }
  }
  __device__ void issue(const void *cache, const Block &b, uint32_t lds) const {
    i32x4_t r4 = rsrc4(static_cast<const uint8_t *>(cache) + b.at, (uint32_t)b.rows * (D * 2));
#pragma unroll
    for (int i = 0; i < 3; ++i) r4[i] = __builtin_amdgcn_readfirstlane(r4[i]);
#pragma unroll
    for (int c = 0; c < kCopies; ++c)
      copy_lds(r4, off[c % kOffsets] + (c / kOffsets) * (8 * D * 2), lds + c * 1024);
  }
};

template <int N>
__device__ inline void wait_vm() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// This wave's reads of LDS have been answered.
__device__ inline void wait_lds() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

__device__ inline uint32_t lds_addr(const void *p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}

// ---------------------------------------------------------------------------
// one wave's 32 rows
// ---------------------------------------------------------------------------

// Transposing LDS read: with 8 bytes at p from each lane, lane l of 16 gets element
// l % 4 of the four lanes 4 j + l / 4, j = 0 .. 3.
__device__ inline uint2 read_tr(const uint8_t *p) {
  return __builtin_bit_cast(
      uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)p));
}

template <int T, int D, int BK, bool CAP>
struct Wave {
  static constexpr int kSteps = D / 16;   // of a score's contraction
  static constexpr int kBlocks = D / 32;  // of output elements
  static constexpr int kTiles = BK / 32;  // of scores

  uint4 q[kSteps];
  f32x16_t o[kBlocks];
  float m, l;
  int32_t lo, hi;        // keys that this lane's row sees (a lane without a row: all)
  int32_t all_lo, all_hi;  // keys that every row of the wave sees
  int32_t any_lo, any_hi;  // and that some row sees
  bool masked;           // a tile was compared

  static constexpr float kLift = T == EB_F16 ? 11.f : 0.f, kLate = T == EB_F16 ? 4.f : 8.f;

  __device__ void begin() {
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) o[b] = f32x16_t(0.f);
    m = -INFINITY;
    l = 0.f;
    masked = false;
  }

  // A row's value in lane l and in lane l ^ 32, in both lanes.  The exchange swaps
  // halves of two registers; of one register, given twice, it makes nothing useful,
  // and the compiler would give one where both are the same value.
  __device__ static float2 both(float v) {
    uint32_t x = __builtin_bit_cast(uint32_t, v), y = x;
    asm("" : "+v"(y));
    const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    return make_float2(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
  }
  __device__ static float row_max(float v) {
    const float2 r = both(v);
    return fmaxf(r.x, r.y);
  }
  __device__ static float row_sum(float v) {
    const float2 r = both(v);
    return r.x + r.y;
  }

  // Operands from LDS: of product i of the scores (tile i % kTiles, elements 16 c ..,
  // c = i / kTiles) and of the values (block i % kBlocks, keys 16 c .., c = i / kBlocks).
  struct Operands {
    const uint8_t *k, *v;
    uint32_t kx, vx;

    __device__ Operands(const uint8_t *keys, const uint8_t *values) {
      const uint32_t lane = threadIdx.x & 63, half = lane >> 5;
      k = keys + (lane & 31) * (D * 2);
      kx = half ^ k_swizzle<D>(lane & 31);
      const uint32_t row = 4 * half + (lane & 15) / 4, quad = lane & 3;
      v = values + row * (D * 2) + (quad & 1) * 8;
      vx = (2 * ((lane >> 4) & 1) + quad / 2) ^ v_swizzle<D>(row);
    }
    __device__ uint4 key(int i) const {
      const int c = i / kTiles, t = i % kTiles;
      return *reinterpret_cast<const uint4 *>(k + ((((2 * c) & 7) ^ kx) << 4) + t * (32 * D * 2) +
                                              (((2 * c) & ~7) << 4));
    }
    __device__ uint4 value(int i) const {
      const int c = i / kBlocks, b = i % kBlocks;
      const uint8_t *const at = v + ((((4 * b) & 15) ^ vx) << 4) + (16 * c) * (D * 2) + (((4 * b) & ~15) << 4);
      const uint2 x = read_tr(at), y = read_tr(at + 8 * (D * 2));
      return make_uint4(x.x, x.y, y.x, y.y);
    }
  };
  static constexpr int kScoreProducts = kSteps * kTiles, kValueProducts = 2 * kTiles * kBlocks;
  static constexpr int kAhead = 3;  // products that operands are read ahead of theirs

  // Scores of BK keys in LDS.  A single tile's long sums are taken in two halves: a
  // product that waits for the one before takes twice as long (dim 256: 22.8 -> 20.4 us
  // for the 816-row prefill; of 4 products the halves' sum costs what it saves).
  __device__ void scores(f32x16_t (&s)[kTiles], const uint8_t *k) const {
    const Operands from(k, k);
    constexpr int kSums = kTiles == 2 || kSteps >= 8 ? 2 : 1;
    f32x16_t sum[kSums];
#pragma unroll
    for (int i = 0; i < kSums; ++i) sum[i] = f32x16_t(0.f);
    uint4 f[kScoreProducts];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) f[i] = from.key(i);
#pragma unroll
    for (int i = 0; i < kScoreProducts; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      sum[i % kSums] = mfma32<T>(f[i], q[i / kTiles], sum[i % kSums]);
      if (i + kAhead < kScoreProducts) f[i + kAhead] = from.key(i + kAhead);
    }
    s[0] = sum[0];
    if (kTiles == 2)
      s[kTiles - 1] = sum[kSums - 1];
    else if (kSums == 2)
      s[0] += sum[kSums - 1];
  }

  // Capped: in units of log2 e, as the exponent takes them.
  __device__ static float capped(const AttnArgs &a, float s) {
    const float e = __builtin_amdgcn_exp2f(s * a.scale2);
    return __builtin_fmaf(-2.f * a.cap2, __builtin_amdgcn_rcpf(1.f + e), a.cap2);
  }

  // Scores of keys from k0 on that a row does not see become -infinity, and its
  // maximum is raised where they call for it
  // (top: the maximum of the scores as they are).
  __device__ static float top_of(const f32x16_t (&s)[kTiles]) {
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[t][i]);
    return top;
  }
  __device__ void settle(const AttnArgs &a, f32x16_t (&s)[kTiles], float top, int32_t k0, uint32_t missing) {
    const int half = (threadIdx.x & 63) >> 5;
    const float c = CAP ? 1.f : a.scale2;
    if (k0 < all_lo || k0 + BK > all_hi || missing) {
      masked = true;
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int32_t key = k0 + 32 * t + 8 * (i / 4) + 4 * half + i % 4;
          const bool see = key >= lo && key < hi && !(missing >> (2 * t + i / 8) & 1);
          s[t][i] = see ? s[t][i] : -INFINITY;
        }
      top = top_of(s);
    }
    top = row_max(top);
    if (__ballot((top - m) * c > kLate)) {
      const float to = fmaxf(m, top);
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - to) * c);
      m = to;
      l *= f;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) o[b] *= f;  // whole vectors: by element, the loop would copy them
    }
  }

  // What settled scores' exponents start from, and a pair's weights.
  __device__ float base_of(const AttnArgs &a) const { return m == -INFINITY ? 0.f : -top_exponent(a); }
  // O and l are sums of 2^(t - this), t being a score times c.
  __device__ float top_exponent(const AttnArgs &a) const { return __builtin_fmaf(m, CAP ? 1.f : a.scale2, -kLift); }
  __device__ uint32_t pair(const AttnArgs &a, float base, float x, float y) {
    const float c = CAP ? 1.f : a.scale2;
    const float u = __builtin_amdgcn_exp2f(__builtin_fmaf(x, c, base));
    const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(y, c, base));
    l += u + v;
    return pack2<T>(u, v);
  }

  // From scores to p, with the maximum and sum of each row; p in pairs.
  __device__ void softmax(const AttnArgs &a, f32x16_t (&s)[kTiles], uint32_t (&p)[kTiles][8], int32_t k0,
                          uint32_t missing) {
    if (CAP) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = capped(a, s[t][i]);
    }
    settle(a, s, top_of(s), k0, missing);
    const float base = base_of(a);
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 8; ++i) p[t][i] = pair(a, base, s[t][2 * i], s[t][2 * i + 1]);
  }

  // The scores of the next tile beside the weights of this one, then this one's
  // values beside the cap and the maximum of the next one's scores: a lone wave's
  // vector instructions issue while its matrix instructions, which do not wait for
  // them, execute.  Left to itself the compiler issues the matrix instructions in
  // runs, so the order is written out: operands are read kAhead products ahead, and
  // nothing moves from one product's group to another's.  Returns the maximum.
  __device__ float step(const AttnArgs &a, const f32x16_t (&s)[kTiles], f32x16_t (&next)[kTiles],
                        const uint8_t *k, const uint8_t *v) {
    constexpr int QK = kScoreProducts, PV = kValueProducts, kPairs = 8 * kTiles;
    const Operands from(k, v);
    uint4 f[QK + PV];
    auto read = [&](int i) __attribute__((always_inline)) {
      if (i < QK)
        f[i] = from.key(i);
      else if (i < QK + PV)
        f[i] = from.value(i - QK);
    };
    uint32_t p[kPairs];
    const float base = base_of(a);
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) next[t] = f32x16_t(0.f);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) read(i);
#pragma unroll
    for (int i = 0; i < QK + PV; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      if (i < QK) {
        next[i % kTiles] = mfma32<T>(f[i], q[i / kTiles], next[i % kTiles]);
      } else {
        const int c = (i - QK) / kBlocks, b = (i - QK) % kBlocks;
        o[b] = mfma32<T>(f[i], make_uint4(p[4 * c], p[4 * c + 1], p[4 * c + 2], p[4 * c + 3]), o[b]);
      }
      read(i + kAhead);
      // pairs of weights: spread over the products up to the middle of the values'
#pragma unroll
      for (int n = kPairs * i / (QK + PV / 2); n < kPairs * (i + 1) / (QK + PV / 2); ++n)
        if (n < kPairs) p[n] = pair(a, base, s[n / 8][2 * (n % 8)], s[n / 8][2 * (n % 8) + 1]);
      if (i >= QK) {
#pragma unroll
        for (int n = 16 * kTiles * (i - QK) / PV; n < 16 * kTiles * (i - QK + 1) / PV; ++n) {
          if (CAP) next[n / 16][n % 16] = capped(a, next[n / 16][n % 16]);
          top = fmaxf(top, next[n / 16][n % 16]);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    return top;
  }

  // O^T += V^T P^T over BK keys in LDS.
  __device__ void values(const uint32_t (&p)[kTiles][8], const uint8_t *v) {
    const Operands from(v, v);
    uint4 f[kValueProducts];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) f[i] = from.value(i);
#pragma unroll
    for (int i = 0; i < kValueProducts; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      const int c = i / kBlocks, b = i % kBlocks;
      const uint32_t *w = &p[c / 2][4 * (c % 2)];
      o[b] = mfma32<T>(f[i], make_uint4(w[0], w[1], w[2], w[3]), o[b]);
      if (i + kAhead < kValueProducts) f[i + kAhead] = from.value(i + kAhead);
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  __device__ bool finite() const {
    float z = l * 0.f;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) z = __builtin_fmaf(o[b][i], 0.f, z);
    return z == 0.f;
  }
};

// Loads the queries of a lane's row as the operand of scores(): elements 16 c +
// 8 half .. + 7 of step c; with a negative scale, negated (exactly).
template <int D>
__device__ inline void load_query(uint4 (&q)[D / 16], const uint16_t *row, uint32_t flip) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int c = 0; c < D / 16; ++c) {
    q[c] = row ? *reinterpret_cast<const uint4 *>(row + 16 * c + 8 * half) : make_uint4(0, 0, 0, 0);
    q[c].x ^= flip;
    q[c].y ^= flip;
    q[c].z ^= flip;
    q[c].w ^= flip;
  }
}

// ---------------------------------------------------------------------------
// one row by one wave, key by key: exact about what the row does not see
// ---------------------------------------------------------------------------

template <int T, int D>
struct Row {
  static constexpr int kElems = D / 64;  // of a lane: lane * kElems + e
  float m, l, acc[kElems];
};

template <int T, int D, bool CAP>
__device__ inline void row_again(const AttnArgs &a, const uint16_t *qrow, int64_t head,
                                                    const int32_t *table, int32_t count, int32_t lo,
                                                    int32_t hi, Row<T, D> *out) {
  constexpr int E = D / 64;
  const eb_attention_op &o = a.o;
  const int lane = threadIdx.x & 63;
  float qe[E], acc[E] = {};
#pragma unroll
  for (int e = 0; e < E; ++e) qe[e] = from_y16(qrow[lane * E + e] ^ (uint16_t)a.flip, T);
  float m = -INFINITY, l = 0.f;
  const float c = CAP ? 1.f : a.scale2;
  for (int32_t j0 = lo; j0 < hi; j0 += 64) {
    const int32_t j = j0 + lane, at = j >> a.page_shift;
    int32_t id = j < hi && at < count ? table[at] : -1;
    if (id >= o.cache.pages) id = -1;
    const int64_t row = (max(id, 0) * a.head_rows + head + (j & (o.cache.page - 1))) * D;
    float t = -INFINITY;
    {
      const uint4 *k = reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(o.cache.k) + row);
      float s = 0.f;
      for (int ch = 0; ch < D / 8; ++ch) {
        uint32_t w[4] = {0, 0, 0, 0};
        if (id >= 0) {
          const uint4 u = k[ch];
          w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int e = 8 * ch + i;
          const float x = __shfl(qe[i % E], e / E);
          s = __builtin_fmaf(from_y16((uint16_t)(w[i / 2] >> (16 * (i & 1))), T), x, s);
        }
      }
      if (CAP) {
        const float e = __builtin_amdgcn_exp2f(s * a.scale2);
        s = __builtin_fmaf(-2.f * a.cap2, __builtin_amdgcn_rcpf(1.f + e), a.cap2);
      }
      if (id >= 0) t = s;
    }
    float top = t;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float to = fmaxf(m, top), base = to == -INFINITY ? 0.f : to;
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - base) * c);
    const float w = id >= 0 ? __builtin_amdgcn_exp2f((t - base) * c) : 0.f;
    m = to;
    float sum = w;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
    l = l * f + sum;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] *= f;
    for (uint64_t left = __ballot(id >= 0); left; left &= left - 1) {
      const int src = __builtin_ctzll(left);
      const float wk = __shfl(w, src);
      const uint16_t *v = static_cast<const uint16_t *>(o.cache.v) + __shfl(row, src) + lane * E;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = __builtin_fmaf(wk, from_y16(v[e], T), acc[e]);
    }
  }
  out->m = m;
  out->l = l;
#pragma unroll
  for (int e = 0; e < E; ++e) out->acc[e] = acc[e];
}

// ---------------------------------------------------------------------------
// kernels
// ---------------------------------------------------------------------------

// Sums of a split: D values of each row of the tile, the exponent that they are above
// (Wave::top_exponent; of row_again's, its maximum times c) and their sum.
__device__ inline float *part_o(const AttnArgs &a, int64_t item, int32_t row, int d) {
  return a.ws + (item * a.part_rows + row) * d;
}
__device__ inline float2 *part_ml(const AttnArgs &a, int64_t item, int32_t row, int d) {
  return reinterpret_cast<float2 *>(a.ws + (int64_t)a.grid * a.part_rows * d) + item * a.part_rows + row;
}

// This workgroup's item and key/value head.  Neighbouring workgroups go to the 8
// XCDs in turn; each XCD gets a contiguous run of (head, item) so that tiles of
// one sequence and head, which read the same keys, share its L2.
__device__ inline void locate(const AttnArgs &a, int32_t &head, uint32_t &at) {
  // Single tiles share nothing: in order, the items that exist (the grid is an
  // upper bound) fall to the XCDs evenly.
  const uint32_t per = (a.grid + kXcds - 1) / kXcds;
  const uint32_t id = a.spread ? blockIdx.x : (blockIdx.x % kXcds) * per + blockIdx.x / kXcds;
  head = (int32_t)(a.spread ? id % a.o.cache.heads : id / a.items);
  at = a.spread ? id / a.o.cache.heads : id % a.items;
}

// The row of q / out that row `r` of an item's tile is, or -1.
__device__ inline int64_t row_of(const AttnArgs &a, const Item &it, int32_t r, int32_t kh, int32_t &tok,
                                 int32_t &head) {
  const uint32_t at = it.head0 + r, t = at / (uint32_t)a.group;
  tok = it.tok0 + (int32_t)t;
  head = kh * a.group + (int32_t)(at - t * a.group);
  return r < it.rows ? (int64_t)it.q0 + tok : -1;
}

// Intervals of a wave's rows r0 .. r0 + 31 of the tile: each lane's own, and
// bounds over the lanes, which the first and the last row give (a later token's
// interval neither begins nor ends before an earlier one's).
template <class W>
__device__ inline void intervals(const AttnArgs &a, const Item &it, int32_t r0, int32_t tok, bool live, W &w) {
  const int32_t prefix = a.o.prefix ? a.o.prefix[it.b] : 0;
  interval(a, it.p0 + tok, it.kv, prefix, w.lo, w.hi);
  if (!live) w.lo = 0, w.hi = 0x7fffffff;
  int32_t first, last, head;
  row_of(a, it, r0, 0, first, head);
  row_of(a, it, min(r0 + 31, it.rows - 1), 0, last, head);
  int32_t fl, fh, ll, lh;
  interval(a, it.p0 + first, it.kv, prefix, fl, fh);
  interval(a, it.p0 + last, it.kv, prefix, ll, lh);
  const bool some = r0 < it.rows;
  w.any_lo = __builtin_amdgcn_readfirstlane(some ? fl : 0x7fffffff);
  w.any_hi = __builtin_amdgcn_readfirstlane(some ? lh : 0);
  w.all_lo = __builtin_amdgcn_readfirstlane(ll);
  w.all_hi = __builtin_amdgcn_readfirstlane(fh);
}

// Tiles of BK keys [t0, t1) of a split of [lo, hi).
template <int BK>
__device__ inline void split_range(const Item &it, int32_t lo, int32_t hi, int32_t &t0, int32_t &t1) {
  const int32_t a = lo / BK, b = hi > lo ? (hi + BK - 1) / BK : a;
  // (told to be the same in all lanes, or the loop over them would run on lane masks)
  t0 = __builtin_amdgcn_readfirstlane(a + (int32_t)((int64_t)(b - a) * it.split / it.splits));
  t1 = __builtin_amdgcn_readfirstlane(a + (int32_t)((int64_t)(b - a) * (it.split + 1) / it.splits));
}

// Bit s is set where the 16 keys from k0 + 16 s on are on a missing page.
template <int BK>
__device__ inline uint32_t missing_of(const Pages &pg, int32_t k0, int32_t kv, int page_shift) {
  if (!pg.holes) return 0;
  uint32_t bits = 0;
#pragma unroll
  for (int s = 0; s < BK / 16; ++s)
    if (k0 + 16 * s < kv && pg.id((k0 + 16 * s) >> page_shift) < 0) bits |= 1u << s;
  return bits;
}

// Many rows: 128 of a tile, 32 to each wave, all waves over the same keys, which
// are copied to LDS ahead of their use (one barrier a tile).  Bound by the matrix
// cores: 4096 tokens that all see each other, 24 heads of 128, bf16: 200 to 212 us, 0.97
// to 1.03 PFLOP/s, where a plain 8192^3 product of the same type reaches 1.19; 45% of
// cycles issue MFMA, LDS is as busy, the rest is softmax beside them.  Heads of 256 (tiles
// of 32 keys, one wave a SIMD) 950 TFLOP/s, of 64 (twice the softmax a product) 830.
// Causal: 134 us, half the work at 0.77 of the rate.  Half-masked key blocks are 3% of
// it; the rest is uneven CUs: each XCD gets three heads of 32 tiles, each longest first,
// so the first 64 items put the longest tiles of two heads on one CU, 128 units of 64 keys
// where the mean CU has 99 (at 1.07 us a unit that is 137 us, and 106 if all had the mean).
template <int T, int D, int BK, bool CAP>
__global__ void __launch_bounds__(256, D == 256 ? 1 : 2) attn_tile_kernel(AttnArgs a) {
  constexpr int kTile = BK * D * 2;  // bytes of a tile of keys or values
  __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * kTile];
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  int32_t kh;
  uint32_t at;
  locate(a, kh, at);
  if (kh >= a.o.cache.heads || at >= a.items) return;
  const Item it = find_item<false>(a, at);
  if (it.b < 0) return;

  Wave<T, D, BK, CAP> w;
  int32_t tok, head;
  const int64_t row = row_of(a, it, 32 * wv + (lane & 31), kh, tok, head);
  const bool live = row >= 0;
  const uint16_t *qrow =
      live ? static_cast<const uint16_t *>(a.o.q) + row * a.o.q_stride + (int64_t)head * D : nullptr;
  load_query<D>(w.q, qrow, a.flip);
  intervals(a, it, 32 * wv, tok, live, w);
  w.begin();

  // keys that any row of the workgroup sees: its first and last token bound them
  int32_t lo, hi, t0, t1;
  {
    int32_t first, last, h;
    row_of(a, it, 0, 0, first, h);
    row_of(a, it, it.rows - 1, 0, last, h);
    const int32_t prefix = a.o.prefix ? a.o.prefix[it.b] : 0;
    int32_t x;
    interval(a, it.p0 + first, it.kv, prefix, lo, x);
    interval(a, it.p0 + last, it.kv, prefix, x, hi);
  }
  split_range<BK>(it, lo, hi, t0, t1);
  Pages pg;
  pg.table = a.o.table + (int64_t)it.b * a.o.table_stride;
  pg.count = (it.kv + a.o.cache.page - 1) >> a.page_shift;
  pg.pages = a.o.cache.pages;
  const int64_t ho = (int64_t)kh << a.page_shift;
  const uint32_t base = lds_addr(lds);
  Copy<D, false> kc;
  Copy<D, true> vc;
  kc.begin();
  vc.begin();
  // Keys are copied two tiles ahead and values one: 16 keys and 16 values to each
  // wave, or (tiles of 32 keys) 16 keys to the first two waves, 16 values to the others.
  const int part = wv % (BK / 16);
  Block there{0, 0};       // of the tile whose keys were requested last
  uint32_t gone = 0, gone1 = 0;  // missing pages of that tile, and of the one before
  auto keys = [&](int32_t t) {
    const int32_t k0 = t * BK;
    pg.reach(k0 >> a.page_shift);
    there = block_of<D>(a, pg, kh, k0 + 16 * part, it.kv);
    if (BK == 64 || wv < 2) kc.issue(a.o.cache.k, there, base + (t & 1) * kTile + part * (16 * D * 2));
    gone1 = gone;
    gone = missing_of<BK>(pg, k0, it.kv, a.page_shift);
  };
  auto values = [&](int32_t t) {
    if (BK == 64 || wv >= 2) vc.issue(a.o.cache.v, there, base + (2 + (t & 1)) * kTile + part * (16 * D * 2));
  };
  if (t0 < t1) {
    pg.begin((t0 * BK) >> a.page_shift);
    keys(t0);
    wait_vm_barrier<0>();
    values(t0);
    if (t0 + 1 < t1) keys(t0 + 1);
  }
  // The keys of tile t + 1 and the values of tile t are in LDS, and every wave has
  // done with the keys of t and the values of t - 1, whose room is filled next.
  auto arrive = [&](int32_t t) {
    wait_vm_barrier<0>();
    if (t + 1 < t1) values(t + 1);
    if (t + 2 < t1) keys(t + 2);
  };
  // This wave's tiles, c0 .. c1 - 1, between those that only others need (sums that a
  // branch in the loop may or may not change would be copied, 64 registers a tile).
  // Each step takes the scores of the tile after its own; the last one's are not used.
  const int32_t c0 = min(max(w.any_lo / BK, t0), t1), c1 = max(min((w.any_hi + BK - 1) / BK, t1), c0);
  int32_t t = t0;
  f32x16_t s0[BK / 32], s1[BK / 32];
  auto first = [&](int32_t at) {
    w.scores(s0, lds + (at & 1) * kTile);
    if (CAP) {
#pragma unroll
      for (int u = 0; u < BK / 32; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) s0[u][i] = w.capped(a, s0[u][i]);
    }
    w.settle(a, s0, w.top_of(s0), at * BK, at + 1 < t1 ? gone1 : gone);
  };
  auto step = [&](const f32x16_t (&s)[BK / 32], f32x16_t (&n)[BK / 32]) {
    arrive(t);
    const float top = w.step(a, s, n, lds + ((t + 1) & 1) * kTile, lds + (2 + (t & 1)) * kTile);
    if (t + 1 < c1) w.settle(a, n, top, (t + 1) * BK, t + 2 < t1 ? gone1 : gone);
    return ++t < c1;
  };
  if (c0 < c1) {
    for (; t < c0; ++t) arrive(t);
    first(c0);
    while (step(s0, s1) && step(s1, s0)) {
    }
  }
  for (; t < t1; ++t) arrive(t);

  w.l = Wave<T, D, BK, CAP>::row_sum(w.l);
  const bool split = it.splits > 1;
  const float c = CAP ? 1.f : a.scale2;
  const int64_t item = (int64_t)kh * a.items + at;
  const int half = lane >> 5;
  if (live) {
    if (split) {
      float *dst = part_o(a, item, 32 * wv + (lane & 31), D);
#pragma unroll
      for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<float4 *>(dst + 32 * b + 8 * (i / 4) + 4 * half) =
              make_float4(w.o[b][i], w.o[b][i + 1], w.o[b][i + 2], w.o[b][i + 3]);
      if (half == 0) *part_ml(a, item, 32 * wv + (lane & 31), D) = make_float2(w.top_exponent(a), w.l);
    } else {
      uint16_t *dst = static_cast<uint16_t *>(a.o.out) + row * a.o.out_stride + (int64_t)head * D;
      const float inv = w.l != 0.f ? 1.f / w.l : 0.f;
#pragma unroll
      for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<uint2 *>(dst + 32 * b + 8 * (i / 4) + 4 * half) =
              make_uint2(pack2<T>(w.o[b][i] * inv, w.o[b][i + 1] * inv),
                         pack2<T>(w.o[b][i + 2] * inv, w.o[b][i + 3] * inv));
    }
  }
  // rows whose sums took up an infinity or NaN where some key was hidden
  uint64_t again = __ballot(live && w.masked && !w.finite());
  again = (again | again >> 32) & 0xffffffffu;
  if (again) wait_vm<0>();  // what is written again has been written
  while (again) {
    const int src = __builtin_ctzll(again);
    again &= again - 1;
    const int32_t klo = max(__builtin_amdgcn_readlane(w.lo, src), t0 * BK);
    const int32_t khi = min(__builtin_amdgcn_readlane(w.hi, src), t1 * BK);
    int32_t tk, hd;
    const int64_t rw = row_of(a, it, 32 * wv + src, kh, tk, hd);
    Row<T, D> r;
    row_again<T, D, CAP>(a, static_cast<const uint16_t *>(a.o.q) + rw * a.o.q_stride + (int64_t)hd * D, ho,
                         pg.table, pg.count, klo, khi, &r);
    constexpr int E = D / 64;
    if (split) {
      float *dst = part_o(a, item, 32 * wv + src, D);
#pragma unroll
      for (int e = 0; e < E; ++e) dst[lane * E + e] = r.acc[e];
      if (lane == 0) *part_ml(a, item, 32 * wv + src, D) = make_float2(r.m * c, r.l);
    } else {
      uint16_t *dst = static_cast<uint16_t *>(a.o.out) + rw * a.o.out_stride + (int64_t)hd * D;
      const float inv = r.l != 0.f ? 1.f / r.l : 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) dst[lane * E + e] = to_y16(r.acc[e] * inv, T);
    }
  }
}

// Workgroups of the stream kernel on a CU: what its registers (D = 64) or its part of
// LDS allow.
template <int D>
constexpr int kStreamWgs = D == 64 ? 3 : 256 / D;

// Few rows: up to 32, the same for all waves, which take the tiles of 32 keys in
// turn.  A wave copies its own tiles to its own part of LDS, keys while it works
// on values and values while it works on keys, and waits for no other wave; the
// four waves' sums are joined in LDS at the end.  Of one tile or few a wave the
// kernel is a chain of latencies, and fetching code that has not run yet is one of
// them: the sums are joined in chunks of 16 bytes, a quarter of the code.
// Measured, means of 40 launches: single tokens of 48 sequences, 456 MB of keys and values,
// 91 us (5.0 TB/s, a large copy 5.14); one token after 131071 keys of 256, 134 MB, 25.4 us
// (5.3 TB/s); after 900 of 32 heads, 6.8 us, of which 1.4 wait for lengths, 0.4 for the page
// table, 1.3 for keys, 0.5 for values and 1 goes into the join in LDS.  Chunks are bound by the copies
// to LDS, which each wave makes for its 32 rows alone: 128 keys of 128 take 0.95 us on a
// CU by itself, 65 KB which is 69 GB/s; a CU reads 126 from L2.
template <int T, int D, bool CAP>
__global__ void __launch_bounds__(256, kStreamWgs<D>) attn_stream_kernel(AttnArgs a) {
  constexpr int BK = 32, kTile = BK * D * 2;
  constexpr int kCopies = 2 * Copy<D, false>::kCopies;  // of a wave's tile of keys, or of values
  static_assert(2 * kTile == 32 * D * 4, "a wave's tiles and its sums take the same room");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * 2 * kTile];
  __shared__ float2 ml[4][32];
  __shared__ float4 factor[32];  // of the waves' sums of a row
  __shared__ float2 total[32];   // a row's maximum and sum; or 1 / sum twice
  __shared__ int64_t place[32];  // a row's first element in `out`
  __shared__ uint32_t again;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  int32_t kh;
  uint32_t at;
  locate(a, kh, at);
  if (kh >= a.o.cache.heads || at >= a.items) return;
  const Item it = find_item<false>(a, at);
  if (it.b < 0) return;

  Wave<T, D, BK, CAP> w;
  int32_t tok, head;
  const int64_t row = row_of(a, it, lane & 31, kh, tok, head);
  const bool live = row >= 0;
  Pages pg;
  pg.table = a.o.table + (int64_t)it.b * a.o.table_stride;
  pg.count = (it.kv + a.o.cache.page - 1) >> a.page_shift;
  pg.pages = a.o.cache.pages;
  intervals(a, it, 0, tok, live, w);
  int32_t t0, t1;
  split_range<BK>(it, w.any_lo, w.any_hi, t0, t1);
  const int64_t ho = (int64_t)kh << a.page_shift;
  uint8_t *const mine = lds + wv * (2 * kTile);
  const uint32_t to = lds_addr(mine);
  Copy<D, false> kc;
  Copy<D, true> vc;
  kc.begin();
  vc.begin();
  Block b0, b1;  // the tile whose keys were requested last
  auto keys = [&](int32_t t) {
    pg.reach((t * BK) >> a.page_shift);
    b0 = block_of<D>(a, pg, kh, t * BK, it.kv);
    b1 = block_of<D>(a, pg, kh, t * BK + 16, it.kv);
    kc.issue(a.o.cache.k, b0, to);
    kc.issue(a.o.cache.k, b1, to + kTile / 2);
  };
  auto values = [&] {
    vc.issue(a.o.cache.v, b0, to + kTile);
    vc.issue(a.o.cache.v, b1, to + kTile + kTile / 2);
  };
  const int32_t begin = t0 + wv;
  if (begin < t1) {
    pg.begin((begin * BK) >> a.page_shift);
    keys(begin);
    values();
  }
  load_query<D>(w.q, live ? static_cast<const uint16_t *>(a.o.q) + row * a.o.q_stride + (int64_t)head * D
                          : nullptr, a.flip);
  w.begin();
  for (int32_t t = begin; t < t1; t += 4) {
    const int32_t k0 = t * BK;
    const uint32_t missing = missing_of<BK>(pg, k0, it.kv, a.page_shift);
    f32x16_t s[1];
    uint32_t p[1][8];
    wait_vm<kCopies>();  // the keys are here
    w.scores(s, mine);
    const bool more = t + 4 < t1;
    if (more) {
      wait_lds();  // and read: their room is free
      keys(t + 4);
    }
    w.softmax(a, s, p, k0, missing);
    if (more)
      wait_vm<kCopies>();
    else
      wait_vm<0>();
    w.values(p, mine + kTile);
    if (more) {
      wait_lds();
      values();
    }
  }
  w.l = Wave<T, D, BK, CAP>::row_sum(w.l);

  // The waves' sums, brought to one maximum and added in the waves' order.  Elements
  // 4 c .. 4 c + 3 of row r of a wave are chunk c ^ (r % 8) of row r of its part.
  const float c = CAP ? 1.f : a.scale2;
  const int r = lane & 31, half = lane >> 5;
  if (half == 0) ml[wv][r] = make_float2(w.top_exponent(a), w.l);
  if (threadIdx.x == 0) again = 0;
  float4 *const sums = reinterpret_cast<float4 *>(mine) + r * (D / 4);
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      sums[(8 * b + i / 2 + half) ^ (r & 7)] = make_float4(w.o[b][i], w.o[b][i + 1], w.o[b][i + 2], w.o[b][i + 3]);
  __syncthreads();
  const bool split = it.splits > 1;
  const int64_t item = (int64_t)kh * a.items + at;
  if (threadIdx.x < 32) {
    // what a row's elements share, once a row (by each thread for itself, a chunk took 0.5
    // us longer with D = 128, 1 us with 256)
    float mx = -INFINITY, l = 0.f, f[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) mx = fmaxf(mx, ml[u][threadIdx.x].x);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float2 x = ml[u][threadIdx.x];
      // (a wave that saw nothing has sums of 0, or NaN, which stays)
      f[u] = x.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.x - mx);
      l = __builtin_fmaf(x.y, f[u], l);
    }
    factor[threadIdx.x] = make_float4(f[0], f[1], f[2], f[3]);
    const float inv = l != 0.f ? 1.f / l : 0.f;
    total[threadIdx.x] = split ? make_float2(mx, l) : make_float2(inv, inv);
    if (live && !(l * 0.f == 0.f)) atomicOr(&again, 1u << threadIdx.x);
    place[threadIdx.x] = row * a.o.out_stride + (int64_t)head * D;
  }
  __syncthreads();
  const float4 *all = reinterpret_cast<const float4 *>(lds);
#pragma unroll 2
  for (int32_t e = threadIdx.x; e < it.rows * (D / 4); e += 256) {
    const int32_t rr = e / (D / 4), ch = e % (D / 4);
    const float4 f = factor[rr];
    const float2 t = total[rr];
    const float4 *const part = all + rr * (D / 4) + (ch ^ (rr & 7));
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](int u, float w) __attribute__((always_inline)) {
      const float4 y = part[u * (8 * D)];
      v.x = __builtin_fmaf(y.x, w, v.x);
      v.y = __builtin_fmaf(y.y, w, v.y);
      v.z = __builtin_fmaf(y.z, w, v.z);
      v.w = __builtin_fmaf(y.w, w, v.w);
    };
    add(0, f.x);
    add(1, f.y);
    add(2, f.z);
    add(3, f.w);
    if (!((v.x + v.y + v.z + v.w) * 0.f == 0.f)) atomicOr(&again, 1u << rr);
    if (split) {
      *reinterpret_cast<float4 *>(part_o(a, item, rr, D) + 4 * ch) = v;
      if (ch == 0) *part_ml(a, item, rr, D) = t;
    } else {
      *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.o.out) + place[rr] + 4 * ch) =
          make_uint2(pack2<T>(v.x * t.x, v.y * t.x), pack2<T>(v.z * t.x, v.w * t.x));
    }
  }
  __syncthreads();
  uint32_t todo = again;
  if (todo) {  // what is written again has been written
    wait_vm<0>();
    __syncthreads();
  }
  for (; todo; todo &= todo - 1) {
    const int src = __builtin_ctz(todo);
    if (src % 4 != wv) continue;
    const int32_t klo = max(__builtin_amdgcn_readlane(w.lo, src), t0 * BK);
    const int32_t khi = min(__builtin_amdgcn_readlane(w.hi, src), t1 * BK);
    int32_t tk, hd;
    const int64_t rw = row_of(a, it, src, kh, tk, hd);
    Row<T, D> x;
    row_again<T, D, CAP>(a, static_cast<const uint16_t *>(a.o.q) + rw * a.o.q_stride + (int64_t)hd * D, ho,
                         pg.table, pg.count, klo, khi, &x);
    constexpr int E = D / 64;
    if (split) {
      float *dst = part_o(a, item, src, D);
#pragma unroll
      for (int e = 0; e < E; ++e) dst[lane * E + e] = x.acc[e];
      if (lane == 0) *part_ml(a, item, src, D) = make_float2(x.m * c, x.l);
    } else {
      uint16_t *dst = static_cast<uint16_t *>(a.o.out) + rw * a.o.out_stride + (int64_t)hd * D;
      const float inv = x.l != 0.f ? 1.f / x.l : 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) dst[lane * E + e] = to_y16(x.acc[e] * inv, T);
    }
  }
}

// Joins the splits of a tile's rows, in an order that the number of splits decides.
// Up to 16: D / 4 lanes take a row, 8 splits at a time.  More: a workgroup takes 64
// elements of a row, 16 lanes reading a split's and 16 groups of lanes every 16th
// split, whose sums meet in LDS.  Either way as many requests at once as registers
// hold, since what other XCDs wrote comes from behind this one's L2.  A launch, the lengths and
// one round of requests: 3 us (8 splits of 32 rows) to 6 us (256 splits of 8).
template <int T, int D>
__global__ void __launch_bounds__(256) attn_join_kernel(AttnArgs a) {
  constexpr int kLanes = D / 4, kPlaces = 256 / kLanes, kParts = D / 64;
  __shared__ float weight[kMaxSplits];
  __shared__ float red[8];
  __shared__ float4 part[256];
  const int32_t kh = (int32_t)(blockIdx.x / a.join_tiles);
  uint32_t first;
  const Item it = find_item<true>(a, blockIdx.x % a.join_tiles, &first);
  if (it.b < 0 || it.splits <= 1 || it.splits > kMaxSplits) return;
  const int64_t step = it.tiles;  // from a split's item to the next one's
  if (first + (it.splits - 1) * step >= a.items) return;
  const int64_t base = (int64_t)kh * a.items + first;
  auto store = [&](int32_t r, int d0, float4 v, float l) {
    int32_t tok, head;
    const int64_t row = row_of(a, it, r, kh, tok, head);
    const float inv = l != 0.f ? 1.f / l : 0.f;
    *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.o.out) + row * a.o.out_stride + (int64_t)head * D + d0) =
        make_uint2(pack2<T>(v.x * inv, v.y * inv), pack2<T>(v.z * inv, v.w * inv));
  };
  auto add = [](float4 &v, const float4 &x, float f) {
    v.x = __builtin_fmaf(x.x, f, v.x);
    v.y = __builtin_fmaf(x.y, f, v.y);
    v.z = __builtin_fmaf(x.z, f, v.z);
    v.w = __builtin_fmaf(x.w, f, v.w);
  };
  if (it.splits <= kJoinRows) {
    const int place = threadIdx.x / kLanes, d0 = 4 * (threadIdx.x % kLanes);
    for (int32_t r = blockIdx.y * kPlaces + place; r < it.rows; r += gridDim.y * kPlaces) {
      float m = -INFINITY, l = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int32_t s0 = 0; s0 < it.splits; s0 += 8) {
        // (those past the last split repeat it and are left out)
        float2 ml[8];
        float4 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int64_t item = base + min(s0 + i, it.splits - 1) * step;
          ml[i] = *part_ml(a, item, r, D);
          x[i] = *reinterpret_cast<const float4 *>(part_o(a, item, r, D) + d0);
        }
        float to = m;
#pragma unroll
        for (int i = 0; i < 8; ++i) to = fmaxf(to, ml[i].x);
        const float f0 = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - to);
        m = to;
        l *= f0;
        v = make_float4(v.x * f0, v.y * f0, v.z * f0, v.w * f0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (s0 + i >= it.splits) continue;
          const float f = ml[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[i].x - m);
          l = __builtin_fmaf(ml[i].y, f, l);
          add(v, x[i], f);
        }
      }
      store(r, d0, v, l);
    }
    return;
  }
  const int wv = threadIdx.x >> 6, place = threadIdx.x >> 4;
  for (int32_t u = blockIdx.y; u < it.rows * kParts; u += gridDim.y) {
    const int32_t r = u / kParts;
    const int d0 = 64 * (u % kParts) + 4 * (threadIdx.x & 15);
    float m = -INFINITY, l = 0.f;
    for (int32_t s = threadIdx.x; s < it.splits; s += 256) m = fmaxf(m, part_ml(a, base + s * step, r, D)->x);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if ((threadIdx.x & 63) == 0) red[wv] = m;
    __syncthreads();
    m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    for (int32_t s = threadIdx.x; s < it.splits; s += 256) {
      const float2 ml = *part_ml(a, base + s * step, r, D);
      const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
      weight[s] = f;
      l = __builtin_fmaf(ml.y, f, l);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) l += __shfl_xor(l, d);
    if ((threadIdx.x & 63) == 0) red[4 + wv] = l;
    __syncthreads();
    l = (red[4] + red[5]) + (red[6] + red[7]);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int32_t s0 = place; s0 < it.splits; s0 += 16 * 8) {
      float4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int32_t s = min(s0 + 16 * i, it.splits - 1);
        x[i] = *reinterpret_cast<const float4 *>(part_o(a, base + s * step, r, D) + d0);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (s0 + 16 * i < it.splits) add(v, x[i], weight[s0 + 16 * i]);
    }
    part[threadIdx.x] = v;
    __syncthreads();
    if (place == 0) {
#pragma unroll
      for (int q = 1; q < 16; ++q) add(v, part[q * 16 + threadIdx.x], 1.f);
      store(r, d0, v, l);
    }
    __syncthreads();
  }
}

template <int T, int D>
hipError_t attn_launch_d(const AttnArgs &a, hipStream_t s) {
  constexpr int BK = D == 256 ? 32 : 64;
  const dim3 grid(a.grid_wgs);
  const bool cap = a.cap2 != 0.f;
  if (a.tile_rows == 128) {
    if (cap)
      attn_tile_kernel<T, D, BK, true><<<grid, 256, 0, s>>>(a);
    else
      attn_tile_kernel<T, D, BK, false><<<grid, 256, 0, s>>>(a);
  } else {
    if (cap)
      attn_stream_kernel<T, D, true><<<grid, 256, 0, s>>>(a);
    else
      attn_stream_kernel<T, D, false><<<grid, 256, 0, s>>>(a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.target <= 0) return e;
  // one workgroup for each 1024 / D rows, or, of many splits, for each 64 elements of a
  // row, while that is not far more than run at once (one token, 131071 keys: one
  // workgroup 91 us, its 32 parts 36; 32 tokens of 2000 keys each, where nothing is split:
  // 56.0 us with 1024, 57.7 with 2048; 256 tokens, 4000 keys: 39 with 2048, 48 with 8192)
  const uint32_t tiles = (uint32_t)(a.join_tiles * a.o.cache.heads), rows = (uint32_t)a.part_rows;
  const uint32_t parts = a.join_splits <= kJoinRows ? (rows * D + 1023) / 1024 : rows * (D / 64);
  const uint32_t most = (1024 + tiles - 1) / tiles;
  attn_join_kernel<T, D><<<dim3(tiles, parts < most ? parts : most), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

template <int T>
hipError_t attn_launch(const AttnArgs &a, hipStream_t s) {
  switch (a.o.cache.dim) {
    case 64: return attn_launch_d<T, 64>(a, s);
    case 128: return attn_launch_d<T, 128>(a, s);
    default: return attn_launch_d<T, 256>(a, s);
  }
}

}  // namespace eb

#endif  // EB_ATTENTION_TILE_H
