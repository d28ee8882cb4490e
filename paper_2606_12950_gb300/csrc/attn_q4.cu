// attn_q4.cu -- the calls of the 4-bit decode attention: argument checks,
// workspace and launch (the kernel is in attn_q4_impl.cuh).
#include <cmath>

#include "attn_host.h"
#include "attn_q4_impl.cuh"
#include "pool_internal.h"

namespace {

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

// the run table (an int2 per run, padded to 256 bytes), then the records
size_t q4_ws_layout(int S, int Hkv, int G, int D, int P, size_t *part_off)
{
    *part_off = ((size_t)S * Hkv * sizeof(int2) + 255) / 256 * 256;
    return *part_off + ((size_t)S * Hkv + (size_t)P) * (size_t)kvp::q4_record_floats(D, G) * 4;
}

int q4_shape(const kv_pool *p, int q4_layout, int S, int Hq, int max_blocks, int *G, int *D)
{
    if (!p || q4_layout < 0 || q4_layout >= p->desc.num_layouts) return KV_ERR_INVALID_ARG;
    if (S < 0 || max_blocks < 1 || Hq < 1) return KV_ERR_INVALID_ARG;
    const kv_layout &L = p->desc.layouts[q4_layout];
    if (!kvp_is_q4(L)) return KV_ERR_UNSUPPORTED;
    if (Hq % L.num_kv_heads) return KV_ERR_INVALID_ARG;
    *G = Hq / L.num_kv_heads;
    *D = kvp_head_dim(L);
    if (!(*G == 1 || *G == 2 || *G == 4 || *G == 5 || *G == 8)) return KV_ERR_UNSUPPORTED;
    // token and run numbers, and a sequence's cost, are 32-bit on the device
    if ((int64_t)max_blocks * p->desc.block_size >= INT32_MAX - kQ4Tile) return KV_ERR_INVALID_ARG;
    const int64_t tiles = ((int64_t)max_blocks * p->desc.block_size + kQ4Tile - 1) / kQ4Tile;
    if (tiles * L.num_kv_heads * kvp::kBf16Cost >= INT32_MAX) return KV_ERR_INVALID_ARG;
    if (S * tiles * L.num_kv_heads >= INT32_MAX) return KV_ERR_INVALID_ARG;  // (a CTA's share of the cost, too)
    return KV_OK;
}

int run(int D, int G, const kvp::Q4Args *a, int sms, cudaStream_t st, bool launch, int *P)
{
    return D == 64 ? kvp_q4_attn_d64(G, a, sms, st, launch, P) : kvp_q4_attn_d128(G, a, sms, st, launch, P);
}

}  // namespace

extern "C" {

int kv_q4_workspace_bytes(const kv_pool *p, int q4_layout, int S, int Hq, int max_blocks, size_t *out_bytes)
{
    int G, D, P;
    if (!out_bytes) return KV_ERR_INVALID_ARG;
    int rc = q4_shape(p, q4_layout, S, Hq, max_blocks, &G, &D);
    if (rc) return rc;
    if (p->sm_count <= 0) return KV_ERR_CUDA;
    rc = run(D, G, nullptr, p->sm_count, nullptr, false, &P);
    if (rc) return rc;
    size_t off;
    *out_bytes = q4_ws_layout(S, p->desc.layouts[q4_layout].num_kv_heads, G, D, P, &off);
    return KV_OK;
}

int paged_decode_attn_q4(kv_pool *p, int layout, int q4_layout, const uint16_t *q, const uint16_t *k_new,
                         const uint16_t *v_new, uint16_t *out, const int32_t *dev_table, const int32_t *dev_ctx_lens,
                         int max_blocks, const int32_t *dev_table4, const int32_t *dev_packed_lens, int max_blocks4,
                         int S, int Hq, float scale, void *workspace, size_t ws_bytes, void *stream)
{
    int G, D, P;
    if (!p || layout < 0 || layout >= p->desc.num_layouts || !std::isfinite(scale)) return KV_ERR_INVALID_ARG;
    if (kvp_is_q4(p->desc.layouts[layout])) return KV_ERR_UNSUPPORTED;
    int rc = q4_shape(p, q4_layout, S, Hq, max_blocks, &G, &D);
    if (!rc) rc = q4_shape(p, q4_layout, S, Hq, max_blocks4, &G, &D);
    if (rc) return rc;
    const kv_layout &L = p->desc.layouts[layout];
    if (L.num_kv_heads != p->desc.layouts[q4_layout].num_kv_heads || L.head_dim != D) return KV_ERR_INVALID_ARG;
    if (S == 0) return KV_OK;
    if (!q || !out || !dev_table || !dev_ctx_lens || !dev_table4 || !dev_packed_lens) return KV_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(out)) return KV_ERR_INVALID_ARG;
    if ((k_new || v_new) && (!k_new || !v_new || !aligned16(k_new) || !aligned16(v_new))) return KV_ERR_INVALID_ARG;
    if (p->sm_count <= 0) return KV_ERR_CUDA;
    if (!kvp_on_device(p)) return KV_ERR_INVALID_ARG;
    rc = run(D, G, nullptr, p->sm_count, nullptr, false, &P);
    if (rc) return rc;
    size_t part_off;
    if (!workspace || ws_bytes < q4_ws_layout(S, L.num_kv_heads, G, D, P, &part_off) || ((uintptr_t)workspace & 255u))
        return KV_ERR_WORKSPACE;
    kvp::Q4Args a{};
    a.q = q;
    a.out = out;
    a.k_new = k_new;
    a.v_new = v_new;
    a.pool = reinterpret_cast<uint8_t *>(p->desc.device_base);
    a.table = dev_table;
    a.lens = dev_ctx_lens;
    a.table4 = dev_table4;
    a.packed = dev_packed_lens;
    a.err = p->desc.device_error;
    a.ws_run = reinterpret_cast<int2 *>(workspace);
    a.ws_part = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(workspace) + part_off);
    a.page_bytes = (int64_t)p->page_bytes;
    a.pool_pages = p->n_pages;
    a.pages_per_block = p->pages_per_block[layout];
    a.pages_per_block4 = p->pages_per_block[q4_layout];
    a.max_blocks = max_blocks;
    a.max_blocks4 = max_blocks4;
    a.S = S;
    a.Hkv = L.num_kv_heads;
    a.G = G;
    a.bs = p->desc.block_size;
    a.qk_scale = scale * 1.4426950408889634f;
    return run(D, G, &a, p->sm_count, (cudaStream_t)stream, true, &P);
}

}  // extern "C"
