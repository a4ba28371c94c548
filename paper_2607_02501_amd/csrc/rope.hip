// rope.hip -- head norms, rotation and the cache write in one pass over a QKV
// projection's output (include/eb_attention.h, eb_rope_append).
//
// Per head x of d elements: y = x g / sqrt(eps + sum x^2 / d), then pairs
// (a, b) -> (a cos t - b sin t, b cos t + a sin t), t = position * freq; values
// are only copied.  Bound by bytes: QKV read once, queries, keys and values
// written once.
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

// Four elements from e on, as fp32.
template <int IT>
__device__ inline float4 load4(const void *p, int64_t e) {
  if (IT == EB_F32) return *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + e);
  const ushort4 u = *reinterpret_cast<const ushort4 *>(static_cast<const uint16_t *>(p) + e);
  return make_float4(from_y16(u.x, IT), from_y16(u.y, IT), from_y16(u.z, IT), from_y16(u.w, IT));
}

template <int CT>
__device__ inline void store4(uint16_t *p, const float (&v)[4]) {
  ushort4 u;
  u.x = to_y16(v[0], CT);
  u.y = to_y16(v[1], CT);
  u.z = to_y16(v[2], CT);
  u.w = to_y16(v[3], CT);
  *reinterpret_cast<ushort4 *>(p) = u;
}

template <int IT, int CT, int D>
__global__ void __launch_bounds__(kThreads)
    rope_append_kernel(eb_rope_append_op o, int page_shift, int parts) {
  constexpr int kLanes = D / 8;         // of a head
  constexpr int kHeads = 64 / kLanes;   // of a wave at a time
  const int lane = threadIdx.x & 63, sub = lane % kLanes;
  const int64_t wave = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int64_t row = wave / parts;
  const int part = (int)(wave - row * parts);
  if (row >= o.rows) return;
  const int32_t slot = o.slots[row];
  const int32_t at = slot >> page_shift;
  if (slot < 0 || at >= o.cache.pages) return;

  // elements of this lane: 4 from e0 on and 4 from e1 on
  const int half = o.rot / 2, pair = 4 * sub;
  const bool rotated = pair < half, split = rotated && o.style == EB_ROT_HALF;
  const int e0 = split ? pair : 2 * pair;
  const int e1 = split ? half + pair : 2 * pair + 4;
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
  const char *src = static_cast<const char *>(o.qkv) + row * o.qkv_stride * (IT == EB_F32 ? 4 : 2);
  const int heads = o.q_heads + 2 * o.cache.heads;
  const int64_t in_page = slot & (o.cache.page - 1);
  const float4 one = make_float4(1.f, 1.f, 1.f, 1.f);
  float4 gq0 = one, gq1 = one, gk0 = one, gk1 = one;
  if (o.q_norm) {
    gq0 = *reinterpret_cast<const float4 *>(o.q_norm + e0);
    gq1 = *reinterpret_cast<const float4 *>(o.q_norm + e1);
  }
  if (o.k_norm) {
    gk0 = *reinterpret_cast<const float4 *>(o.k_norm + e0);
    gk1 = *reinterpret_cast<const float4 *>(o.k_norm + e1);
  }
#pragma unroll 2
  for (int h0 = part * kHeads; h0 < heads; h0 += parts * kHeads) {
    const int h = h0 + lane / kLanes;
    const bool ok = h < heads;
    const int64_t in = (int64_t)(ok ? h : heads - 1) * D;
    const float4 a = load4<IT>(src, in + e0), b = load4<IT>(src, in + e1);
    const bool is_q = h < o.q_heads, is_v = h >= o.q_heads + o.cache.heads;
    float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) ss = __builtin_fmaf(x[j], x[j], ss);
#pragma unroll
    for (int d = kLanes / 2; d >= 1; d >>= 1) ss += __shfl_xor(ss, d);
    if (is_q ? o.q_norm != nullptr : (!is_v && o.k_norm != nullptr)) {
      const float r = 1.0f / __builtin_sqrtf(ss * (1.0f / D) + o.norm_eps);
      const float4 g0 = is_q ? gq0 : gk0, g1 = is_q ? gq1 : gk1;
      const float g[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = x[j] * r * g[j];
    }
    if (rotated && !is_v) {
      float y[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // halves: x[j] and x[4 + j]; adjacent: x[2 j] and x[2 j + 1]
        const float p = split ? x[j] : x[2 * j], q = split ? x[4 + j] : x[2 * j + 1];
        const float u = p * cs[j] - q * sn[j], v = q * cs[j] + p * sn[j];
        y[j] = u;
        y[4 + j] = v;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[j] = split ? y[j] : (j & 1 ? y[4 + j / 2] : y[j / 2]);
        x[4 + j] = split ? y[4 + j] : (j & 1 ? y[6 + j / 2] : y[2 + j / 2]);
      }
    }
    if (!ok) continue;
    uint16_t *dst;
    if (is_q) {
      dst = static_cast<uint16_t *>(o.q_out) + row * o.q_stride + (int64_t)h * D;
    } else {
      const int kh = h - o.q_heads - (is_v ? o.cache.heads : 0);
      dst = static_cast<uint16_t *>(is_v ? o.cache.v : o.cache.k) +
            ((((int64_t)at * o.cache.heads + kh) << page_shift) + in_page) * D;
    }
    const float lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
    store4<CT>(dst + e0, lo);
    store4<CT>(dst + e1, hi);
  }
}

template <int IT, int CT>
hipError_t launch_d(const eb_rope_append_op &o, hipStream_t s) {
  const int shift = __builtin_ctz((unsigned)o.cache.page);
  const int64_t heads = (int64_t)o.q_heads + 2 * o.cache.heads;
  const int64_t steps = (heads * o.cache.dim + 511) / 512;  // of a wave over a row
  int64_t parts = (8192 + o.rows - 1) / o.rows;
  parts = parts < steps ? parts : steps;
  const int64_t waves = o.rows * parts;
  const unsigned grid = (unsigned)((waves + kThreads / 64 - 1) / (kThreads / 64));
  if (o.cache.dim == 64)
    rope_append_kernel<IT, CT, 64><<<grid, kThreads, 0, s>>>(o, shift, (int)parts);
  else if (o.cache.dim == 128)
    rope_append_kernel<IT, CT, 128><<<grid, kThreads, 0, s>>>(o, shift, (int)parts);
  else
    rope_append_kernel<IT, CT, 256><<<grid, kThreads, 0, s>>>(o, shift, (int)parts);
  return hipGetLastError();
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
