// attention.h -- declarations shared by the translation units of the steps
// between a layer's QKV and O projections (include/eb_attention.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/eb_attention.h"

namespace eb {

constexpr int kMaxBatch = 4096;

hipError_t launch_kv_extend(const eb_kv_extend_op &o, hipStream_t s);
hipError_t launch_rope_append(const eb_rope_append_op &o, hipStream_t s);
size_t attention_ws_bytes(const eb_attention_op &o);
hipError_t launch_attention(const eb_attention_op &o, void *ws, hipStream_t s);

}  // namespace eb
