// pages_internal.h -- page copies on the device and table entries changed by
// them (not part of the ABI).
#pragma once

#include <cstddef>
#include <cstdint>

#include "kvpool.h"

// Copy the first tokens[i] rows (null: all) of block src[i] to block dst[i] on
// `stream`, side by side: no destination is another pair's block.  The ids are
// the caller's to check.
int kvp_copy_pages(const kv_pool *p, int layout, int n, const int32_t *src, const int32_t *dst, const int32_t *tokens,
                   void *stream);

// Set entry i of slot s and mark it changed for the next sync (seqtab.cpp;
// does not throw).
void kvp_seqtab_set_entry(kv_seqtab *t, int s, int i, int32_t v);
