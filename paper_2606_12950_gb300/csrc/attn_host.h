// attn_host.h -- host helpers of the attention calls shared by their files
// (not part of the ABI).
#pragma once

#include "kvpool.h"

// The argument checks common to all attention calls; *G_out = Hq / Hkv.
int kvp_attn_shape(const kv_pool *p, int layout, int S, int Hq, int max_blocks, int *G_out);
// The layout's tensor map of the pool, encoded on first use.
int kvp_ensure_tmap(kv_pool *p, int layout);
