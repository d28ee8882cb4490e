// prompt.cu -- causal attention of prompt chunks over the paged pool
// (paged_prompt_attn): argument checks, the split of the key range, launches.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>

#include <cuda_runtime.h>

#include "attn_host.h"
#include "device_flags.h"
#include "pool_internal.h"
#include "prompt_impl.cuh"
#include "stream_order.h"

namespace {

// Row tiles the grid needs at most (the chunks' lengths are on the device).
int64_t row_tiles(int S, int T, int max_q, int TT)
{
    return std::min((int64_t)S * ((max_q + TT - 1) / TT), (int64_t)T / TT + S);
}

// Key splits: CTAs for every SM where the rows are few, each with at least
// kLeastTiles key tiles.  us with 1, 2, 4, 8 and up to 16 splits (32 q / 8 KV
// heads of 128): 16 tokens on a context of 16000 158, 87, 51, 32, 26; 64 on 8000
// 86, 52, 34, 25, 26; 256 on 8000 (4 by this rule) 90, 56, 38; 64 on 2000 (4) 30,
// 24, 20; 4 x 100, window 1024 (2) 28, 25.
// The lengths are on the device, so the rule takes the table's width for them: in
// a table much wider than its sequences a call pays for splits without keys and
// for a merge.  us in a table as wide as the context and in one of 32768 tokens
// (splits): 33 tokens, 4 q / 2 KV heads of 64, 6.4 (1) and 9.2 (16); 100 tokens,
// 32 / 8 of 128, 8.4 (1) and 13.6 (9); chunks of 60, 90 and 100 tokens, window
// 1024, 12.6 (1) and 15.2 (2); 16 tokens on 1000 13.4 (2) and 12.4 (16); 128 on
// 4000 20.7 (8) and 21.1 (9).
constexpr int kLeastTiles = 4;
int key_splits(int64_t ctas, int sm_count, int64_t reach, int TT, int window, int sinks)
{
    int64_t keys = reach;
    if (window > 0) keys = std::min(keys, (int64_t)window + TT + sinks);
    const int64_t tiles = (keys + kvp::kPrKeys - 1) / kvp::kPrKeys;
    const int64_t want = std::min((int64_t)sm_count / std::max<int64_t>(1, ctas), tiles / kLeastTiles);
    return (int)std::max<int64_t>(1, std::min<int64_t>(want, kvp::kPrMaxSplits));
}

struct Shape {
    int G, D, Hkv, TT, KS;
    int64_t tiles;
    size_t ws_bytes;
};

int prompt_shape(const kv_pool *p, int layout, int S, int Hq, int T, int max_q, int max_blocks, int window, int sinks,
                 Shape *s)
{
    const int rc = kvp_attn_shape(p, layout, S, Hq, max_blocks, &s->G);
    if (rc) return rc;
    if (T < 0 || max_q < 0 || max_q > T || window < 0 || sinks < 0) return KV_ERR_INVALID_ARG;
    if (T > 0 && (S == 0 || max_q == 0)) return KV_ERR_INVALID_ARG;
    // (positions of whole key tiles and boxes past the last token stay in 32 bits)
    if ((int64_t)max_blocks * p->desc.block_size > INT32_MAX - 4 * kvp::kPrKeys) return KV_ERR_INVALID_ARG;
    const kv_layout &L = p->desc.layouts[layout];
    s->D = L.head_dim;
    s->Hkv = L.num_kv_heads;
    s->TT = kvp::kPrTiles * (kvp::kPrRows / s->G);
    s->tiles = row_tiles(S, T, max_q, s->TT);
    if (p->sm_count <= 0) return KV_ERR_CUDA;
    s->KS = key_splits(s->tiles * s->Hkv, p->sm_count, (int64_t)max_blocks * p->desc.block_size, s->TT, window, sinks);
    if (s->tiles * s->Hkv * s->KS > INT32_MAX) return KV_ERR_INVALID_ARG;
    if ((int64_t)s->KS * T > INT32_MAX) return KV_ERR_INVALID_ARG;
    s->ws_bytes = s->KS > 1 ? (size_t)s->KS * T * Hq * (s->D + 2) * sizeof(float) : 0;
    return KV_OK;
}

template <int D>
int prompt_run(const CUtensorMap *tmap, const CUtensorMap &qmap, const CUtensorMap &omap, const kvp::PromptArgs &a,
               int sm_count, cudaStream_t st)
{
    static kvp::DeviceFlags attr_set;
    const size_t smem = kvp::prompt_smem_bytes<D>();
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return KV_ERR_CUDA;
    if (!attr_set.has(dev)) {
        if (cudaFuncSetAttribute(kvp::prompt_attn_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) !=
            cudaSuccess)
            return KV_ERR_CUDA;
        // the warpgroups' register shares wait for what the launch holds: no
        // launch without it
        cudaFuncAttributes at;
        if (cudaFuncGetAttributes(&at, kvp::prompt_attn_kernel<D>) != cudaSuccess || at.numRegs != kvp::kPrRegsLaunch)
            return KV_ERR_CUDA;
        attr_set.set(dev);
    }
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)std::min(a.n_items, sm_count));  // a CTA an SM: its TMEM
    cfg.blockDim = dim3(kvp::kPrThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kvp::prompt_attn_kernel<D>, *tmap, qmap, omap, a) != cudaSuccess) return KV_ERR_CUDA;
    kvp_note_stream(st, false);
    if (a.KS == 1) return KV_OK;
    const int64_t rows = (int64_t)a.T * a.Hkv * a.G;
    cfg.gridDim = dim3((unsigned)((rows + 7) / 8));
    cfg.blockDim = dim3(256);
    cfg.dynamicSmemBytes = 0;
    if (cudaLaunchKernelEx(&cfg, kvp::prompt_merge_kernel<D>, (const float *)a.ws, a.out, rows, (int)a.KS) !=
        cudaSuccess)
        return KV_ERR_CUDA;
    return KV_OK;
}

}  // namespace

extern "C" {

int kv_prompt_workspace_bytes(const kv_pool *p, int layout, int S, int Hq, int T, int max_q, int max_blocks, int window,
                              int sinks, size_t *out_bytes)
{
    if (!out_bytes) return KV_ERR_INVALID_ARG;
    Shape s{};
    const int rc = prompt_shape(p, layout, S, Hq, T, max_q, max_blocks, window, sinks, &s);
    if (rc) return rc;
    *out_bytes = s.ws_bytes;
    return KV_OK;
}

int paged_prompt_attn(kv_pool *p, int layout, const uint16_t *q, uint16_t *out, const int32_t *dev_q_starts, int T,
                      int max_q, const int32_t *dev_table, const int32_t *dev_ctx_lens, int max_blocks, int S, int Hq,
                      float scale, int window, int sinks, void *workspace, size_t ws_bytes, void *stream)
{
    if (!std::isfinite(scale)) return KV_ERR_INVALID_ARG;
    Shape s{};
    int rc = prompt_shape(p, layout, S, Hq, T, max_q, max_blocks, window, sinks, &s);
    if (rc) return rc;
    if (T == 0) return KV_OK;
    if (!q || !out || !dev_q_starts || !dev_table || !dev_ctx_lens) return KV_ERR_INVALID_ARG;
    if (((uintptr_t)q & 15u) || ((uintptr_t)out & 15u)) return KV_ERR_INVALID_ARG;
    if (s.ws_bytes && (!workspace || ws_bytes < s.ws_bytes || ((uintptr_t)workspace & 255u))) return KV_ERR_WORKSPACE;
    rc = kvp_ensure_tmap(p, layout);
    if (rc) return rc;
    kvp::PromptArgs a{};
    a.q = q;
    a.out = out;
    a.pool = reinterpret_cast<const uint16_t *>(p->desc.device_base);
    a.starts = dev_q_starts;
    a.table = dev_table;
    a.ctx_lens = dev_ctx_lens;
    a.err = p->desc.device_error;
    a.ws = reinterpret_cast<float *>(workspace);
    a.rows_per_page = (int64_t)(p->page_bytes / (2ull * s.D));
    a.pool_pages = p->n_pages;
    a.pages_per_block = p->pages_per_block[layout];
    a.max_blocks = max_blocks;
    a.S = S;
    a.Hkv = s.Hkv;
    a.G = s.G;
    a.bs = p->desc.block_size;
    a.T = T;
    a.max_q = max_q;
    a.KS = s.KS;
    const int32_t reach = max_blocks * a.bs;
    a.window = window < reach ? window : 0;  // one that no context outgrows is the whole context
    a.sinks = a.window > 0 ? std::min(sinks, reach) : 0;
    a.n_items = (int32_t)(s.tiles * s.Hkv * s.KS);
    a.sign = scale > 0.f ? 1.f : scale < 0.f ? -1.f : 0.f;
    a.qk_scale = scale == 0.f ? 1.f : std::fabs(scale) * 1.4426950408889634f;
    const cudaStream_t st = (cudaStream_t)stream;
    // q and out as [T][Hq][d], or the splits' records as [KS T][Hq][d]: boxes of
    // 128 bytes of G heads, a Q tile's tokens of q, a warp's rows of the other
    CUtensorMap qmap, omap;
    rc = kvp_tmap_3d(&qmap, q, 2, s.D, Hq, T, 64, s.G, kvp::kPrRows / s.G);
    if (rc == KV_OK && s.KS == 1) rc = kvp_tmap_3d(&omap, out, 2, s.D, Hq, T, 64, s.G, 32 / s.G);
    if (rc == KV_OK && s.KS > 1) rc = kvp_tmap_3d(&omap, workspace, 4, s.D, Hq, (int64_t)s.KS * T, 32, s.G, 32 / s.G);
    if (rc) return rc;
    return s.D == 64 ? prompt_run<64>(&p->tmap[layout], qmap, omap, a, p->sm_count, st)
                     : prompt_run<128>(&p->tmap[layout], qmap, omap, a, p->sm_count, st);
}

}  // extern "C"
