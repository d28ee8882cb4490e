// attn_q4_launch.cuh -- host-side launch of the 4-bit decode attention and its
// combine.
#pragma once

#include "attn_launch.cuh"
#include "attn_q4_impl.cuh"

namespace kvp {

template <int D, int G>
int q4_combine(const Q4Args &a, int sm_count, const cudaLaunchConfig_t &cfg)
{
    const CombineArgs c{a.out, a.ws_run, a.ws_part, a.S, a.Hkv, nullptr, nullptr, 0};
    const double per_run = (double)a.P / std::max(1, a.S * a.Hkv) + 1.0;
    if (a.by_part)
        return combine_launch<D, G, 1, 1, kRecCtasByPart>(c, combine_groups<D, G, 1>(per_run), cfg, a.P);
    return combine_run<D, G, kRecCtas>(c, per_run, sm_count, cfg);
}

template <int D>
int q4_attn_run(int G, const Q4Args *args, int sm_count, cudaStream_t st, bool launch, int *P_out)
{
    auto fn = q4_attn_kernel<D>;
    const size_t smem = q4_smem_bytes<D>(G);
    static DeviceFlags attr_set;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return KV_ERR_CUDA;
    if (!attr_set.has(dev)) {
        if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)q4_smem_bytes<D>(8)) != cudaSuccess)
            return KV_ERR_CUDA;
        attr_set.set(dev);
    }
    int occ = 0;
    static OccCache occ_cache;
    if (cached_occupancy(fn, kQ4Threads, smem, &occ, occ_cache) != KV_OK) return KV_ERR_CUDA;
    *P_out = std::max(1, occ) * std::max(1, sm_count);
    if (!launch) return KV_OK;
    Q4Args a = *args;
    a.P = *P_out;
    // with several waves of runs, a combine CTA per part (as in attn_launch.cuh)
    const int64_t runs = (int64_t)a.S * a.Hkv;
    a.by_part = runs >= 8 * (int64_t)a.P && 4 * runs > (int64_t)kSlicedCtas * sm_count;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.P);
    cfg.blockDim = dim3(kQ4Threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, fn, a) != cudaSuccess) return KV_ERR_CUDA;
    kvp_note_stream(st, false);
    switch (G) {
    case 1: return q4_combine<D, 1>(a, sm_count, cfg);
    case 2: return q4_combine<D, 2>(a, sm_count, cfg);
    case 4: return q4_combine<D, 4>(a, sm_count, cfg);
    case 5: return q4_combine<D, 5>(a, sm_count, cfg);
    case 8: return q4_combine<D, 8>(a, sm_count, cfg);
    default: return KV_ERR_UNSUPPORTED;
    }
}

}  // namespace kvp
