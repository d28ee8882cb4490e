// attn_win_d64.cu -- instantiations of the paged decode attention kernel with a
// sliding window and sinks for head dim 64.
#include "attn_launch.cuh"

int kvp_attn_win_d64(int G, const CUtensorMap *tmap, const kvp::AttnArgs *a, int P_req, int sm_count, cudaStream_t st,
                     int what, int *P_out)
{
    using namespace kvp;
#define KVP_CASE(GG) \
    case GG: return attn_run<64, GG, MmaCompute<64, GG, true>>(tmap, *a, P_req, sm_count, st, what, P_out);
    switch (G) {
        KVP_CASE(1)
        KVP_CASE(2)
        KVP_CASE(4)
        KVP_CASE(5)
        KVP_CASE(8)
    default:
        return KV_ERR_UNSUPPORTED;
    }
#undef KVP_CASE
}
