// rope.hip -- head norms, rotation and the cache write in one pass over a QKV
// projection's output (include/eb_attention.h, eb_rope_append).
//
// Per head x of d elements: y = x g / sqrt(eps + sum x^2 / d), then pairs
// (a, b) -> (a cos t - b sin t, b cos t + a sin t), t = position * freq; values
// are only copied.  Bound by bytes: QKV read once, queries, keys and values
// written once.  4096 rows of 24 + 48 heads of 128, bf16, 151 MB: 29.3 us, 5.15 TB/s (a large
// copy 5.14; means of 40 launches); 820 rows of 10 heads of 256, fp32 in, 12 MB: 5.7 us; one
// row: 3.5 us, a launch and three dependent reads.
//
// A lane holds 8 elements of a head: 4 rotated pairs, or 8 elements behind the
// rotated part, so both halves of every pair are in one lane for either pair
// style; d / 8 lanes make a head (their sums of squares meet in shuffles) and a
// wave takes 512 elements of a row at a time.  The sines and cosines of a
// lane's pairs serve all heads of the row: a wave computes them once and walks
// over heads.  Rows of few waves are shared out by heads, so that one token
// still fills several waves.
//
// The angle in turns, position * freq / 2 pi, is taken in fp64 and only its
// fraction goes on in fp32: at position 2^20 an fp32 product would be off by
// 0.06 radians.
#include <hip/hip_runtime.h>

#include "attention.h"
#include "epilogue.h"

namespace eb {
namespace {

constexpr int kThreads = 256;
constexpr double kInvTwoPi = 0.15915494309189533577;

// Eight elements of a lane as they lie in memory: 4 from e0 on and 4 from e1 on, or
// (JOINED) 8 from e0 on.
template <int IT, bool JOINED>
struct Raw {
  static constexpr int kWords = IT == EB_F32 ? 8 : 4;
  uint32_t w[kWords];

  __device__ void load(const char *p, int e0, int e1) {
    constexpr int kSize = IT == EB_F32 ? 4 : 2;
    if (IT == EB_F32) {
      *reinterpret_cast<uint4 *>(w) = *reinterpret_cast<const uint4 *>(p + e0 * kSize);
      *reinterpret_cast<uint4 *>(w + 4 % kWords) =
          *reinterpret_cast<const uint4 *>(p + (JOINED ? e0 + 4 : e1) * kSize);
    } else if (JOINED) {
      *reinterpret_cast<uint4 *>(w) = *reinterpret_cast<const uint4 *>(p + e0 * kSize);
    } else {
      *reinterpret_cast<uint2 *>(w) = *reinterpret_cast<const uint2 *>(p + e0 * kSize);
      *reinterpret_cast<uint2 *>(w + 2) = *reinterpret_cast<const uint2 *>(p + e1 * kSize);
    }
  }
  __device__ float at(int i) const {
    if (IT == EB_F32) return __builtin_bit_cast(float, w[i % kWords]);
    return from_y16((uint16_t)(w[i / 2 % kWords] >> (16 * (i & 1))), IT);
  }
};

template <int CT, bool JOINED>
__device__ inline void store8(uint16_t *p, int e0, int e1, const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = (uint32_t)to_y16(v[2 * i], CT) | (uint32_t)to_y16(v[2 * i + 1], CT) << 16;
  if (JOINED) {
    *reinterpret_cast<uint4 *>(p + e0) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    *reinterpret_cast<uint2 *>(p + e0) = make_uint2(w[0], w[1]);
    *reinterpret_cast<uint2 *>(p + e1) = make_uint2(w[2], w[3]);
  }
}

// ADJ: adjacent pairs, or nothing rotated: a lane's 8 elements lie together.
template <int IT, int CT, int D, bool ADJ>
__global__ void __launch_bounds__(kThreads)
    rope_append_kernel(eb_rope_append_op o, int page_shift, int parts) {
  constexpr int kLanes = D / 8;         // of a head
  constexpr int kHeads = 64 / kLanes;   // of a wave at a time
  const int lane = threadIdx.x & 63, sub = lane % kLanes;
  const uint32_t wave = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int64_t row = __builtin_amdgcn_readfirstlane(wave / (uint32_t)parts);
  const int part = __builtin_amdgcn_readfirstlane(wave % (uint32_t)parts);
  if (row >= o.rows) return;
  const int32_t slot = o.slots[row];
  const char *const src = static_cast<const char *>(o.qkv) + row * o.qkv_stride * (IT == EB_F32 ? 4 : 2);
  const int heads = o.q_heads + 2 * o.cache.heads;

  // elements of this lane: 4 from e0 on and 4 from e1 on
  const int half = o.rot / 2, pair = 4 * sub;
  const bool rotated = pair < half, split = !ADJ && rotated;
  const int e0 = split ? pair : 2 * pair;
  const int e1 = split ? half + pair : 2 * pair + 4;
  // one step ahead of its use: the next heads' elements
  const int step = parts * kHeads;
  int h = part * kHeads + lane / kLanes;
  Raw<IT, ADJ> next;
  next.load(src, min(h, heads - 1) * D + e0, min(h, heads - 1) * D + e1);

  float cs[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
  if (rotated) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = pair + j;
      const int axis = p < o.sections[0] ? 0 : (o.n_axes < 3 || p < o.sections[0] + o.sections[1] ? 1 : 2);
      const double turn = (double)o.positions[axis * o.pos_stride + row] * (double)o.freqs[p] * kInvTwoPi;
      // the nearest whole turn off: |fraction| <= 1/2
      sincospif(2.0f * (float)(turn - __builtin_rint(turn)), &sn[j], &cs[j]);
    }
  }
  float gq[8], gk[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) gq[j] = gk[j] = 1.f;
  if (o.q_norm) {
    *reinterpret_cast<float4 *>(gq) = *reinterpret_cast<const float4 *>(o.q_norm + e0);
    *reinterpret_cast<float4 *>(gq + 4) = *reinterpret_cast<const float4 *>(o.q_norm + e1);
  }
  if (o.k_norm) {
    *reinterpret_cast<float4 *>(gk) = *reinterpret_cast<const float4 *>(o.k_norm + e0);
    *reinterpret_cast<float4 *>(gk + 4) = *reinterpret_cast<const float4 *>(o.k_norm + e1);
  }
  const int32_t at = slot >> page_shift;
  if (slot < 0 || at >= o.cache.pages) return;
  uint16_t *const q_out = static_cast<uint16_t *>(o.q_out) + row * o.q_stride;
  const int64_t cell = (((int64_t)at * o.cache.heads) << page_shift) + (slot & (o.cache.page - 1));

  for (int h0 = part * kHeads; h0 < heads; h0 += step, h += step) {
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = next.at(j);
    if (h0 + step < heads)
      next.load(src, min(h + step, heads - 1) * D + e0, min(h + step, heads - 1) * D + e1);
    const bool is_q = h < o.q_heads, is_v = h >= o.q_heads + o.cache.heads;
    if (is_q ? o.q_norm != nullptr : (!is_v && o.k_norm != nullptr)) {
      float ss = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = __builtin_fmaf(x[j], x[j], ss);
      // (a head's lanes take this branch together)
#pragma unroll
      for (int d = kLanes / 2; d >= 1; d >>= 1) ss += __shfl_xor(ss, d);
      // 1 / sqrt to one step of fp32; its argument kept out of the subnormals
      const float ms = __builtin_fmaf(ss, 1.0f / D, o.norm_eps);
      const float r = __builtin_amdgcn_rsqf(ms < 1.17549435e-38f ? 1.17549435e-38f : ms);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = x[j] * r * (is_q ? gq[j] : gk[j]);
    }
    if (rotated && !is_v) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float &a = x[ADJ ? 2 * j : j], &b = x[ADJ ? 2 * j + 1 : 4 + j];
        const float u = a * cs[j] - b * sn[j], v = b * cs[j] + a * sn[j];
        a = u;
        b = v;
      }
    }
    if (h >= heads) continue;
    uint16_t *dst;
    if (is_q) {
      dst = q_out + h * D;
    } else {
      const int kh = h - o.q_heads - (is_v ? o.cache.heads : 0);
      dst = static_cast<uint16_t *>(is_v ? o.cache.v : o.cache.k) + (cell + ((int64_t)kh << page_shift)) * D;
    }
    store8<CT, ADJ>(dst, e0, e1, x);
  }
}

template <int IT, int CT, int D>
hipError_t launch_style(const eb_rope_append_op &o, int shift, int parts, unsigned grid, hipStream_t s) {
  if (o.style == EB_ROT_ADJACENT || o.rot == 0)
    rope_append_kernel<IT, CT, D, true><<<grid, kThreads, 0, s>>>(o, shift, parts);
  else
    rope_append_kernel<IT, CT, D, false><<<grid, kThreads, 0, s>>>(o, shift, parts);
  return hipGetLastError();
}

template <int IT, int CT>
hipError_t launch_d(const eb_rope_append_op &o, hipStream_t s) {
  const int shift = __builtin_ctz((unsigned)o.cache.page);
  const int64_t heads = (int64_t)o.q_heads + 2 * o.cache.heads;
  const int64_t steps = (heads * o.cache.dim + 511) / 512;  // of a wave over a row
  // A wave's sines and cosines serve all heads it takes, so a row is shared out only
  // until there are 4096 waves (820 rows of 48 heads of 128: 8.3 us, with 1024 waves 9.2,
  // with 16384 9.9; 4096 rows: 22.9 us, 32 if shared out; one row: 4.1, 9.2 if not).
  int64_t parts = (4096 + o.rows - 1) / o.rows;
  parts = parts < steps ? parts : steps;
  const int64_t waves = o.rows * parts;
  const unsigned grid = (unsigned)((waves + kThreads / 64 - 1) / (kThreads / 64));
  switch (o.cache.dim) {
    case 64: return launch_style<IT, CT, 64>(o, shift, (int)parts, grid, s);
    case 128: return launch_style<IT, CT, 128>(o, shift, (int)parts, grid, s);
    default: return launch_style<IT, CT, 256>(o, shift, (int)parts, grid, s);
  }
}

}  // namespace

hipError_t launch_rope_append(const eb_rope_append_op &o, hipStream_t s) {
  const bool f16 = o.cache.type == EB_F16;
  switch (o.qkv_type) {
    case EB_F32: return f16 ? launch_d<EB_F32, EB_F16>(o, s) : launch_d<EB_F32, EB_BF16>(o, s);
    case EB_F16: return f16 ? launch_d<EB_F16, EB_F16>(o, s) : launch_d<EB_F16, EB_BF16>(o, s);
    default: return f16 ? launch_d<EB_BF16, EB_F16>(o, s) : launch_d<EB_BF16, EB_BF16>(o, s);
  }
}

}  // namespace eb
