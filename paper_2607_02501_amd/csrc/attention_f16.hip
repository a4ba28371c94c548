// attention_f16.hip -- attention kernels for caches of EB_F16.
#include "attention_tile.h"

namespace eb {
template hipError_t attn_launch<EB_F16>(const AttnArgs &a, hipStream_t s);
}  // namespace eb
