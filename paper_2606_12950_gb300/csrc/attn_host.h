// attn_host.h -- host helpers of the attention calls shared by their files
// (not part of the ABI).
#pragma once

#include <cstdint>

#include <cuda.h>

#include "kvpool.h"

// The argument checks common to all attention calls; *G_out = Hq / Hkv.
int kvp_attn_shape(const kv_pool *p, int layout, int S, int Hq, int max_blocks, int *G_out);
// The layout's tensor map of the pool, encoded on first use.
int kvp_ensure_tmap(kv_pool *p, int layout);
// Tensor map of a contiguous array [d2][d1][d0] of bf16 (elem 2) or fp32 (elem
// 4), boxes of [b2][b1][b0] with the 128-byte swizzle.
int kvp_tmap_3d(CUtensorMap *map, const void *base, int elem, int64_t d0, int64_t d1, int64_t d2, int b0, int b1,
                int b2);
