// attention_api.cpp -- the C entry points of include/eb_attention.h (and eb_attention_plan
// of include/eb_tuning.h): host-side
// validation (before any HIP call, so that every error path runs without a GPU)
// and the launchers' calls.
#include <hip/hip_runtime.h>

#include <cmath>

#include "../../include/eb_tuning.h"
#include "attention.h"

namespace eb {
namespace {

constexpr int64_t kMaxRows = int64_t(1) << 24;
constexpr int64_t kMaxInt = 0x7fffffff;
constexpr int64_t kMaxKeys = int64_t(1) << 30;  // of a sequence: keys count in 32 bits

bool aligned(const void *p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

bool pow2_page(int32_t page) { return page >= 16 && page <= 65536 && (page & (page - 1)) == 0; }

// Buffers of a call: no output may overlap an input or another output.
struct Spans {
  struct One {
    uintptr_t a, b;
    bool out;
  };
  One v[20];
  int n = 0;
  void add(const void *p, int64_t bytes, bool out) {
    if (!p || bytes <= 0) return;
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    v[n++] = One{a, a + (uintptr_t)bytes, out};
  }
  bool clash() const {
    for (int i = 0; i < n; ++i)
      for (int j = i + 1; j < n; ++j)
        if ((v[i].out || v[j].out) && v[i].a < v[j].b && v[j].a < v[i].b) return true;
    return false;
  }
};

int64_t cache_bytes(const eb_kv_cache &c) { return (int64_t)c.pages * c.heads * c.page * c.dim * 2; }

eb_status check_cache(const eb_kv_cache &c) {
  if (c.reserved != 0 || c.heads < 1 || c.heads > 1024 || !pow2_page(c.page) || c.pages < 1 ||
      (int64_t)c.pages * c.page > kMaxInt)
    return EB_ERR_INVALID;
  if (c.type != EB_F16 && c.type != EB_BF16) return c.type == EB_F32 ? EB_ERR_UNSUPPORTED : EB_ERR_INVALID;
  if (c.dim != 64 && c.dim != 128 && c.dim != 256) return EB_ERR_UNSUPPORTED;
  if (!c.k || !c.v) return EB_ERR_INVALID;
  if (!aligned(c.k, 16) || !aligned(c.v, 16)) return EB_ERR_ALIGN;
  return EB_OK;
}

// Bytes that `rows` rows of `width` elements span at a stride.
int64_t row_bytes(int64_t rows, int64_t stride, int64_t width, int64_t size) {
  return rows > 0 ? ((rows - 1) * stride + width) * size : 0;
}

eb_status check_extend(const eb_kv_extend_op &o) {
  if (o.batch < 1 || o.batch > kMaxBatch || o.rows < 0 || o.rows > kMaxRows || !pow2_page(o.page) ||
      o.pages < 1 || (int64_t)o.pages * o.page > kMaxInt || o.table_stride < 1 ||
      (int64_t)o.table_stride * o.page > kMaxKeys || o.free_capacity < 0 || o.free_capacity > 1 << 27)
    return EB_ERR_INVALID;
  if (!o.cached || !o.added || !o.table || !o.n_free || !o.n_free_out || !o.q_start || !o.kv_len ||
      !o.short_rows || (o.free_capacity > 0 && !o.free_pages) || (o.rows > 0 && (!o.slots || !o.positions)))
    return EB_ERR_INVALID;
  const void *all[] = {o.cached, o.added, o.table, o.free_pages, o.n_free, o.n_free_out,
                       o.q_start, o.kv_len, o.slots, o.positions, o.short_rows};
  for (const void *p : all)
    if (!aligned(p, 4)) return EB_ERR_ALIGN;
  Spans s;
  s.add(o.cached, 4ll * o.batch, false);
  s.add(o.added, 4ll * o.batch, false);
  s.add(o.free_pages, 4ll * o.free_capacity, false);
  s.add(o.n_free, 4, false);
  s.add(o.table, 4ll * o.batch * o.table_stride, true);
  s.add(o.n_free_out, 4, true);
  s.add(o.q_start, 4ll * (o.batch + 1), true);
  s.add(o.kv_len, 4ll * o.batch, true);
  s.add(o.slots, 4ll * o.rows, true);
  s.add(o.positions, 4ll * o.rows, true);
  s.add(o.short_rows, 4, true);
  return s.clash() ? EB_ERR_INVALID : EB_OK;
}

eb_status check_rope(const eb_rope_append_op &o) {
  eb_status st = check_cache(o.cache);
  if (st != EB_OK) return st;
  const int64_t dim = o.cache.dim, width = ((int64_t)o.q_heads + 2 * o.cache.heads) * dim;
  if (o.q_heads < 1 || o.q_heads > 4096 || o.rows < 0 || o.rows > kMaxRows || o.qkv_stride < width ||
      o.q_stride < o.q_heads * dim || o.qkv_stride > kMaxInt || o.q_stride > kMaxInt)
    return EB_ERR_INVALID;
  if (o.qkv_type != EB_F32 && o.qkv_type != EB_F16 && o.qkv_type != EB_BF16) return EB_ERR_INVALID;
  if (o.rot < 0 || o.rot > dim || o.rot % 8 != 0 || o.n_axes < 1 || o.n_axes > 3 ||
      (o.style != EB_ROT_HALF && o.style != EB_ROT_ADJACENT))
    return EB_ERR_INVALID;
  int64_t pairs = 0;
  for (int a = 0; a < o.n_axes; ++a) {
    if (o.sections[a] < 0) return EB_ERR_INVALID;
    pairs += o.sections[a];
  }
  if (pairs != o.rot / 2) return EB_ERR_INVALID;
  if (!(std::isfinite(o.norm_eps) && o.norm_eps >= 0.0f)) return EB_ERR_INVALID;
  if (o.rot > 0 && o.pos_stride < o.rows) return EB_ERR_INVALID;
  if (o.pos_stride < 0 || o.pos_stride > kMaxInt) return EB_ERR_INVALID;
  if (o.rows == 0) return EB_OK;
  if (!o.qkv || !o.q_out || !o.slots || (o.rot > 0 && (!o.positions || !o.freqs))) return EB_ERR_INVALID;
  if (o.qkv_stride % 8 != 0 || o.q_stride % 8 != 0 || !aligned(o.qkv, 16) || !aligned(o.q_out, 16) ||
      !aligned(o.slots, 4) || !aligned(o.positions, 4) || !aligned(o.freqs, 4) || !aligned(o.q_norm, 16) ||
      !aligned(o.k_norm, 16))
    return EB_ERR_ALIGN;
  Spans s;
  s.add(o.qkv, row_bytes(o.rows, o.qkv_stride, width, o.qkv_type == EB_F32 ? 4 : 2), false);
  s.add(o.slots, 4ll * o.rows, false);
  if (o.rot > 0) s.add(o.positions, 4ll * ((o.n_axes - 1) * o.pos_stride + o.rows), false);
  if (o.rot > 0) s.add(o.freqs, 2ll * o.rot, false);
  s.add(o.q_norm, 4 * dim, false);
  s.add(o.k_norm, 4 * dim, false);
  s.add(o.q_out, row_bytes(o.rows, o.q_stride, o.q_heads * dim, 2), true);
  s.add(o.cache.k, cache_bytes(o.cache), true);
  s.add(o.cache.v, cache_bytes(o.cache), true);
  return s.clash() ? EB_ERR_INVALID : EB_OK;
}

eb_status check_attention(const eb_attention_op &o) {
  eb_status st = check_cache(o.cache);
  if (st != EB_OK) return st;
  const int64_t width = (int64_t)o.q_heads * o.cache.dim;
  if (o.rows < 0 || o.rows > kMaxRows || o.batch < 1 || o.batch > kMaxBatch || o.q_heads < 1 ||
      o.q_heads > 4096 || o.q_heads % o.cache.heads != 0 ||
      (int64_t)o.rows * (o.q_heads / o.cache.heads) > kMaxKeys || o.q_stride < width || o.out_stride < width ||
      o.q_stride > kMaxInt || o.out_stride > kMaxInt || o.table_stride < 1 ||
      (int64_t)o.table_stride * o.cache.page > kMaxKeys || o.max_new < 1 || o.max_kv < 1 || o.window < 0 ||
      (o.mask != EB_MASK_CAUSAL && o.mask != EB_MASK_FULL))
    return EB_ERR_INVALID;
  if (!(std::fabs(o.scale) <= 65536.0f) || !(std::isfinite(o.softcap) && o.softcap >= 0.0f)) return EB_ERR_INVALID;
  if (o.softcap > 0.0f && (o.softcap < 0x1p-10f || o.softcap > 0x1p10f)) return EB_ERR_UNSUPPORTED;
  if (o.rows == 0) return EB_OK;
  if (!o.q || !o.out || !o.table || !o.q_start || !o.kv_len) return EB_ERR_INVALID;
  if (o.q_stride % 8 != 0 || o.out_stride % 8 != 0 || !aligned(o.q, 16) || !aligned(o.out, 16) ||
      !aligned(o.table, 4) || !aligned(o.q_start, 4) || !aligned(o.kv_len, 4) || !aligned(o.prefix, 4))
    return EB_ERR_ALIGN;
  return EB_OK;
}

eb_status check_attention_buffers(const eb_attention_op &o, const void *ws, size_t wsb) {
  if (!ws && wsb != 0) return EB_ERR_INVALID;
  if (ws && !aligned(ws, 256)) return EB_ERR_ALIGN;
  const int64_t width = (int64_t)o.q_heads * o.cache.dim;
  Spans s;
  s.add(o.cache.k, cache_bytes(o.cache), false);
  s.add(o.cache.v, cache_bytes(o.cache), false);
  s.add(o.q, row_bytes(o.rows, o.q_stride, width, 2), false);
  s.add(o.table, 4ll * o.batch * o.table_stride, false);
  s.add(o.q_start, 4ll * (o.batch + 1), false);
  s.add(o.kv_len, 4ll * o.batch, false);
  s.add(o.prefix, 4ll * o.batch, false);
  s.add(o.out, row_bytes(o.rows, o.out_stride, width, 2), true);
  s.add(ws, (int64_t)wsb, true);
  return s.clash() ? EB_ERR_INVALID : EB_OK;
}

}  // namespace
}  // namespace eb

using namespace eb;

extern "C" {

eb_status eb_kv_extend(const eb_kv_extend_op *op, hipStream_t stream) {
  if (!op) return EB_ERR_INVALID;
  const eb_status st = check_extend(*op);
  if (st != EB_OK) return st;
  return launch_kv_extend(*op, stream) == hipSuccess ? EB_OK : EB_ERR_HIP;
}

eb_status eb_rope_append(const eb_rope_append_op *op, hipStream_t stream) {
  if (!op) return EB_ERR_INVALID;
  const eb_status st = check_rope(*op);
  if (st != EB_OK || op->rows == 0) return st;
  return launch_rope_append(*op, stream) == hipSuccess ? EB_OK : EB_ERR_HIP;
}

size_t eb_attention_workspace_bytes(const eb_attention_op *op) {
  if (!op || check_attention(*op) != EB_OK || op->rows == 0) return 0;
  return attention_ws_bytes(*op);
}

eb_status eb_attention_plan(const eb_attention_op *op, int32_t *tile_rows, int32_t *splits) {
  if (!op || !tile_rows || !splits) return EB_ERR_INVALID;
  const eb_status st = check_attention(*op);
  if (st != EB_OK) return st;
  if (op->rows == 0) return EB_ERR_INVALID;
  attention_plan(*op, tile_rows, splits);
  return EB_OK;
}

eb_status eb_attention(const eb_attention_op *op, void *workspace, size_t workspace_bytes,
                       hipStream_t stream) {
  if (!op) return EB_ERR_INVALID;
  eb_status st = check_attention(*op);
  if (st != EB_OK || op->rows == 0) return st;
  st = check_attention_buffers(*op, workspace, workspace_bytes);
  if (st != EB_OK) return st;
  if (attention_ws_bytes(*op) > workspace_bytes) return EB_ERR_INVALID;
  return launch_attention(*op, workspace, stream) == hipSuccess ? EB_OK : EB_ERR_HIP;
}

}  // extern "C"
