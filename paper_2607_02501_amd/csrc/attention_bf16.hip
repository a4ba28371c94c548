// attention_bf16.hip -- attention kernels for caches of EB_BF16.
#include "attention_tile.h"

namespace eb {
template hipError_t attn_launch<EB_BF16>(const AttnArgs &a, hipStream_t s);
}  // namespace eb
