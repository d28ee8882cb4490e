// rotary_impl.cuh -- what the rotary kernels share: a token's sequence, bf16 pairs,
// a pair's turn.
#pragma once

#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "kvpool.h"
#include "ptx.cuh"

namespace kvp {

// largest s with starts[s] <= t (starts ascending, starts[0] <= t): N probes a
// round trip by the N lanes that share t; the whole warp, converged
template <int N>
__device__ __forceinline__ int seq_of_token(const int32_t *starts, int S, int t, int lane)
{
    const int own = lane & (N - 1);
    int lo = 0, n = S;  // the answer is in [lo, lo + n)
    while (__any_sync(0xffffffffu, n > 1)) {
        const int step = (n + N - 1) / N;
        const int i = lo + own * step;
        const unsigned le = __ballot_sync(0xffffffffu, own * step < n && starts[i] <= t) >> (lane - own);
        const int k = 31 - __clz((int)((N < 32 ? le & ((1u << (N & 31)) - 1u) : le) | 1u));
        n = min(step, n - k * step);
        lo += k * step;
    }
    return lo;
}

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&v);
}

__device__ __forceinline__ float2 unpack2(uint32_t w) { return make_float2(lo_f(w), hi_f(w)); }

// Two pairs of the half layout, (u, v) each, at once (c, s: their cos and sin).
__device__ __forceinline__ void turn2(float2 &u, float2 &v, float2 c, float2 s)
{
    const float2 p = __ffma2_rn(u, c, __fmul2_rn(v, make_float2(-s.x, -s.y)));
    v = __ffma2_rn(v, c, __fmul2_rn(u, s));
    u = p;
}
// an adjacent pair (c, s: its cos and sin)
__device__ __forceinline__ void turn(float &x, float &y, float c, float s)
{
    const float p = __fmaf_rn(x, c, -__fmul_rn(y, s));
    y = __fmaf_rn(y, c, __fmul_rn(x, s));
    x = p;
}

// the cos and sin of position `by` at a frequency of `step` turns a position, in
// units of 2^-64: the fraction of a turn is exact
__device__ __forceinline__ void turn_of(int32_t by, uint64_t step, float &sn, float &cn)
{
    const uint64_t turn = (uint64_t)(int64_t)by * step + (1ull << 31);
    sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &sn, &cn);
}

inline bool rotary_aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

// a row stride that holds the row and keeps 16-byte chunks aligned
inline bool rotary_stride_ok(int64_t stride, int64_t row) { return stride >= row && stride % 8 == 0; }

}  // namespace kvp

// The argument checks of the rotary appends; *go: there are rows.
int kvp_rotary_check(const kv_pool *p, int layout, const kv_rotary *rot, const uint16_t *q, int64_t q_stride,
                     const uint16_t *q_out, const uint16_t *k, int64_t k_stride, const uint16_t *v, int64_t v_stride,
                     const int32_t *dev_q_starts, int T, const int32_t *dev_table, const int32_t *dev_ctx_lens,
                     int max_blocks, int S, int Hq, bool *go);
