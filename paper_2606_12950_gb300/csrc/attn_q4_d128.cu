// attn_q4_d128.cu -- 4-bit decode attention, head dim 128.
#include "attn_q4_launch.cuh"

int kvp_q4_attn_d128(int G, const kvp::Q4Args *a, int sm_count, cudaStream_t st, bool launch, int *P_out)
{
    return kvp::q4_attn_run<128>(G, a, sm_count, st, launch, P_out);
}
