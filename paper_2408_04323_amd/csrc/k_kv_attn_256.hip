// Attention over the block cache for heads of 256 dimensions.
#include "kv_attn.h"

SCOOT_KV_ATTN_DIM(256)
