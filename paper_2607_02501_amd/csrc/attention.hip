// attention.hip -- attention of new tokens over a paged cache
// (include/eb_attention.h, eb_attention).
//
// The keys a token sees are one interval lo <= j < hi (of its sequence's keys:
// a causal mask or a prefix bounds it above, a window below).  One wave per
// token and query head: 64 keys at a time, a lane taking the dot product of
// one key, then the lanes taking the elements of the head while the wave walks
// over the 64 values, with the running maximum and sum of the softmax.
#include <hip/hip_runtime.h>

#include "attention.h"
#include "epilogue.h"

namespace eb {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

struct Attn {
  eb_attention_op o;
  int page_shift;
  int32_t kv_max;  // keys of a table row
  int32_t group;   // query heads per key/value head
  float scale2;    // scale * log2 e without a cap, scale / cap with one
  float cap2;      // cap * log2 e, 0 without a cap
};

// The scores enter 2^t: t = scale log2e q.k, or cap log2e tanh(scale q.k / cap).
__device__ inline float score2(float s, const Attn &a) {
  s *= a.scale2;
  if (a.cap2 != 0.f) s = a.cap2 * (1.f - 2.f / (1.f + __builtin_amdgcn_exp2f(2.f * kLog2e * s)));
  return s;
}

// The sequence of row r: the last b with q_start[b] <= r.
__device__ inline int32_t find_sequence(const int32_t *q_start, int32_t batch, int32_t r) {
  int32_t lo = 0, hi = batch;
  while (hi - lo > 1) {
    const int32_t mid = (lo + hi) >> 1;
    if (q_start[mid] <= r)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

template <int T, int D>
__global__ void __launch_bounds__(kThreads) attn_row_kernel(Attn a) {
  constexpr int E = D / 64;  // elements of a lane
  __shared__ float qs[kThreads / 64][D];
  const eb_attention_op &o = a.o;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int64_t wave = (int64_t)blockIdx.x * (kThreads / 64) + wv;
  const int32_t row = (int32_t)(wave / o.q_heads), head = (int32_t)(wave % o.q_heads);
  const int32_t b = row < o.rows ? find_sequence(o.q_start, o.batch, row) : 0;
  const int32_t q0 = o.q_start[b], q1 = min(o.q_start[b + 1], o.rows);
  if (row >= o.rows || row < q0 || row >= q1 || row - q0 >= o.max_new) return;
  const int32_t kv = min(max(o.kv_len[b], 0), a.kv_max);
  const int32_t p = kv - (q1 - q0) + (row - q0);
  int32_t lo = 0, hi = kv;
  if (o.mask != EB_MASK_FULL) hi = min(kv, max(p + 1, o.prefix ? o.prefix[b] : 0));
  if (o.window > 0) lo = max(0, p - o.window + 1);
  const uint16_t *q = static_cast<const uint16_t *>(o.q) + row * o.q_stride + (int64_t)head * D;
  for (int e = lane; e < D; e += 64) qs[wv][e] = from_y16(q[e], T);
  __builtin_amdgcn_wave_barrier();
  const int32_t kh = head / a.group;
  const int32_t *table = o.table + (int64_t)b * o.table_stride;
  float m = -INFINITY, l = 0.f, acc[E] = {};
  for (int32_t j0 = lo; j0 < hi; j0 += 64) {
    const int32_t j = j0 + lane;
    int32_t id = j < hi ? table[j >> a.page_shift] : -1;
    if (id >= o.cache.pages) id = -1;
    const int64_t at =
        ((((int64_t)max(id, 0) * o.cache.heads + kh) << a.page_shift) + (j & (o.cache.page - 1))) * D;
    float t = -INFINITY;
    if (id >= 0) {
      const uint4 *k = reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(o.cache.k) + at);
      float s = 0.f;
      for (int c = 0; c < D / 8; ++c) {
        const uint4 u = k[c];
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s = __builtin_fmaf(from_y16(w[i] & 0xffff, T), qs[wv][8 * c + 2 * i], s);
          s = __builtin_fmaf(from_y16(w[i] >> 16, T), qs[wv][8 * c + 2 * i + 1], s);
        }
      }
      t = score2(s, a);
    }
    float mx = t;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
    const float mn = fmaxf(m, mx), base = mn == -INFINITY ? 0.f : mn;
    const float w = id >= 0 ? __builtin_amdgcn_exp2f(t - base) : 0.f, r = __builtin_amdgcn_exp2f(m - base);
    m = mn;
    float ws = w;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) ws += __shfl_xor(ws, d);
    l = l * r + ws;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] *= r;
    for (uint64_t left = __ballot(id >= 0); left; left &= left - 1) {
      const int src = __builtin_ctzll(left);
      const float wk = __shfl(w, src);
      const int64_t av = __shfl(at, src);
      const uint16_t *v = static_cast<const uint16_t *>(o.cache.v) + av + lane * E;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = __builtin_fmaf(wk, from_y16(v[e], T), acc[e]);
    }
  }
  uint16_t *dst = static_cast<uint16_t *>(o.out) + row * o.out_stride + (int64_t)head * D + lane * E;
  const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) dst[e] = to_y16(acc[e] * inv, T);
}

Attn attn_of(const eb_attention_op &o) {
  Attn a;
  a.o = o;
  a.page_shift = __builtin_ctz((unsigned)o.cache.page);
  a.kv_max = o.table_stride << a.page_shift;
  a.group = o.q_heads / o.cache.heads;
  a.scale2 = o.softcap > 0.f ? o.scale / o.softcap : o.scale * kLog2e;
  a.cap2 = o.softcap > 0.f ? o.softcap * kLog2e : 0.f;
  return a;
}

template <int T>
hipError_t launch_t(const Attn &a, hipStream_t s) {
  const int64_t waves = (int64_t)a.o.rows * a.o.q_heads;
  const unsigned grid = (unsigned)((waves + 3) / 4);
  if (a.o.cache.dim == 64)
    attn_row_kernel<T, 64><<<grid, kThreads, 0, s>>>(a);
  else if (a.o.cache.dim == 128)
    attn_row_kernel<T, 128><<<grid, kThreads, 0, s>>>(a);
  else
    attn_row_kernel<T, 256><<<grid, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t attention_ws_bytes(const eb_attention_op &) { return 0; }

hipError_t launch_attention(const eb_attention_op &o, void *, hipStream_t s) {
  const Attn a = attn_of(o);
  return o.cache.type == EB_F16 ? launch_t<EB_F16>(a, s) : launch_t<EB_BF16>(a, s);
}

}  // namespace eb
