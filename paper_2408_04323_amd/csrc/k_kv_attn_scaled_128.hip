// Attention over the block cache with scales of blocks and heads, for heads of 128 dimensions.
#include "kv_attn.h"

SCOOT_KV_ATTN_SCALED_DIM(128)
