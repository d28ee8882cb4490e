// rotary_norm.cu -- the rotary append of models whose query and key heads are
// normed: each head x of q and k becomes
//     R(p) (x / sqrt(mean(x^2) + eps) * (weight + offset))
// (RMSNorm; Zhang and Sennrich, 2019) with R(p) its turn to position p (rotary.cu),
// v is copied, k and v go to the paged pool.
//
// Bound by HBM for prompts (each row read and written once) and by latency for a
// decode step.  A head's columns lie with 4 to 32 lanes of a warp (its items, as in
// rotary.cu: pairs of chunks that turn together, chunks that turn, chunks that only
// are normed), which sum its squares by shuffles, so a warp needs no other and no
// barrier: it takes a range of (token, batch of rows) units, the same number as every
// other, computes each token's angles among its lanes, and keeps its columns'
// frequencies from token to token; the weights lie in shared memory in fp32.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>

#include "pool_internal.h"
#include "rotary_impl.cuh"
#include "stream_order.h"

namespace {

using namespace kvp;

constexpr int kNormThreads = 128;
constexpr int kNormResident = 6;   // CTAs an SM
constexpr int kMaxNormDim = 256;   // a head's lanes are of one warp

struct NormArgs {
    const uint16_t *q, *k, *v;  // rows of token t at t * stride
    uint16_t *q_out;            // [T][Hq][d]
    int64_t q_stride, k_stride, v_stride;
    uint8_t *pool;
    const uint64_t *steps;      // [rot / 2] turns per position, in units of 2^-64
    const int32_t *positions;   // [T] or null
    const int32_t *starts;      // [S + 1] first token of each sequence, or null: token t is sequence t's
    const int32_t *table;
    const int32_t *ctx_lens;
    int32_t *err;
    const uint16_t *q_weight, *k_weight;  // [D], or null: not normed
    int64_t page_bytes, n_pages;
    int64_t warps, per_warp, longer;  // with units; a warp's units, the first `longer` warps have one more
    float magnitude, eps, offset, inv_d;
    int32_t pages_per_block, max_blocks;
    int32_t S, Hq, Hkv, D, bs, rot;
    int32_t items, batches;     // of a row; units of a token
};

// rows of a warp in a unit, times the lanes of a row
template <bool INTERLEAVED>
constexpr int kNormBatch = INTERLEAVED ? 4 : 2;

template <bool INTERLEAVED, int LANES>
__global__ void __launch_bounds__(kNormThreads, kNormResident) rotary_norm_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int RPW = 32 / LANES;             // rows side by side in a warp
    constexpr int NP = INTERLEAVED ? 4 : 8;     // pairs of an item
    constexpr int OWN = (NP + RPW - 1) / RPW;   // of which a lane computes
    constexpr int BATCH = kNormBatch<INTERLEAVED>;
    constexpr unsigned ALL = 0xffffffffu;
    // weights with the offset, of q and of k: a chunk's first four columns, then its others
    __shared__ __align__(16) float4 weights[2][2][kMaxNormDim / 8];
    const int lane = threadIdx.x & 31, item = lane % LANES, grp = lane / LANES;
    const int turned = INTERLEAVED ? a.rot / 8 : a.rot / 16;
    const bool holds = item < a.items, turns = item < turned, pair = !INTERLEAVED && turns;
    const int at = turns ? item : item + a.rot / 8 - turned;  // the item's (first) chunk
    const int far = a.rot / 16;                               // chunks to a pair's other one
    grid_dependency_wait();
    grid_launch_dependents();
    for (int i = threadIdx.x; i < a.D / 4; i += kNormThreads)  // (of q, then of k: four columns at a time)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const uint16_t *src = w ? a.k_weight : a.q_weight;
            float4 f = make_float4(1.f, 1.f, 1.f, 1.f);
            if (src) {
                const uint2 v = *reinterpret_cast<const uint2 *>(src + 4 * i);
                f = make_float4(lo_f(v.x) + a.offset, hi_f(v.x) + a.offset, lo_f(v.y) + a.offset, hi_f(v.y) + a.offset);
            }
            weights[w][i & 1][i >> 1] = f;
        }
    uint64_t step[OWN];  // of the pairs whose angles this lane computes
#pragma unroll
    for (int e = 0; e < OWN; ++e) {
        const int p = e * RPW + grp;
        step[e] = turns && p < NP ? a.steps[item * NP + p] : 0;
    }
    __syncthreads();

    const int64_t warp = (int64_t)blockIdx.x * (kNormThreads / 32) + (threadIdx.x >> 5);
    int64_t unit = warp * a.per_warp + min(warp, a.longer);
    const int64_t unit_end = unit + a.per_warp + (warp < a.longer);
    if (warp >= a.warps) return;
    int t = (int)(unit / a.batches);
    int first = (int)(unit - (int64_t)t * a.batches) * BATCH * RPW;  // the unit's first row
    const int q_rows = a.q ? a.Hq : 0, kv = a.k ? a.Hkv : 0, rows = q_rows + 2 * kv;
    const int64_t head_bytes = (int64_t)a.bs * a.D * 2;  // of one KV head in a block
    int32_t n = 0, end = INT32_MIN, s = 0;               // the token's sequence, its context, the token past it
    float2 c[NP / 2], sn[NP / 2];                        // of the item's pairs
    uint8_t *slot = nullptr;
    int now = -1;                                        // the token whose c, sn and slot these are
    for (; unit < unit_end; ++unit) {
        uint4 x[BATCH], y[BATCH];
        // the rows' addresses need the token alone: they are on their way before its
        // position, angles and slot, four dependent loads away, are known
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int r = first + b * RPW + grp, g = r - q_rows;
            if (holds && r < rows) {
                const uint16_t *src = g < 0    ? a.q + t * a.q_stride + r * a.D
                                      : g < kv ? a.k + t * a.k_stride + g * a.D
                                               : a.v + t * a.v_stride + (g - kv) * a.D;
                x[b] = *reinterpret_cast<const uint4 *>(src + at * 8);
                if (pair) y[b] = *reinterpret_cast<const uint4 *>(src + (at + far) * 8);
            }
        }
        if (t != now) {
            now = t;
            if (t >= end) {
                s = a.starts ? seq_of_token<32>(a.starts, a.S, t, lane) : t;
                n = a.ctx_lens[s];
                end = a.starts ? a.starts[s + 1] : t + 1;
            }
            const int32_t pos = n - (end - t);
            // a sequence without a context (n <= 0) keeps its pages as they are; a position
            // outside the table or a page outside the pool is reported (as is t >= end: a
            // bad array)
            slot = nullptr;
            if (kv && n > 0) {
                bool ok = t < end && pos >= 0 && pos < a.max_blocks * a.bs;
                if (ok) {
                    const int32_t b = pos / a.bs, phys = a.table[(int64_t)s * a.max_blocks + b];
                    ok = phys >= 0 && (int64_t)phys + a.pages_per_block <= a.n_pages;
                    if (ok) slot = a.pool + (int64_t)phys * a.page_bytes + (int64_t)(pos - b * a.bs) * a.D * 2 + at * 16;
                }
                if (!ok && lane == 0) atomicCAS(a.err, 0, KV_ERR_DEVICE_BOUNDS);
            }
            const int32_t by = a.positions ? a.positions[t] : pos;
            float own_c[OWN], own_s[OWN];
#pragma unroll
            for (int e = 0; e < OWN; ++e) {
                turn_of(by, step[e], own_s[e], own_c[e]);
                own_c[e] *= a.magnitude;
                own_s[e] *= a.magnitude;
            }
#pragma unroll
            for (int e = 0; e < NP; ++e) {
                const float ce = __shfl_sync(ALL, own_c[e / RPW], (e % RPW) * LANES + item);
                const float se = __shfl_sync(ALL, own_s[e / RPW], (e % RPW) * LANES + item);
                if (e & 1)
                    c[e / 2].y = ce, sn[e / 2].y = se;
                else
                    c[e / 2].x = ce, sn[e / 2].x = se;
            }
        }
        uint8_t *q_dst = reinterpret_cast<uint8_t *>(a.q_out + (int64_t)t * a.Hq * a.D) + at * 16;
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int r = first + b * RPW + grp, g = r - q_rows;
            const bool mine = holds && r < rows;
            if (first + b * RPW < q_rows + kv) {  // (the warp's rows of v alone need no more than a copy)
                float2 u[4], v[4];
                const uint32_t *xw = reinterpret_cast<const uint32_t *>(&x[b]), *yw = reinterpret_cast<const uint32_t *>(&y[b]);
                float2 sum2 = make_float2(0.f, 0.f);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    u[e] = mine ? unpack2(xw[e]) : make_float2(0.f, 0.f);
                    sum2 = __ffma2_rn(u[e], u[e], sum2);
                    if (!INTERLEAVED) {
                        v[e] = mine && pair ? unpack2(yw[e]) : make_float2(0.f, 0.f);
                        sum2 = __ffma2_rn(v[e], v[e], sum2);
                    }
                }
                float sum = sum2.x + sum2.y;
#pragma unroll
                for (int off = 1; off < LANES; off <<= 1) sum += __shfl_xor_sync(ALL, sum, off);
                if (g < kv) {
                    const bool of_k = g >= 0;
                    const float by = (of_k ? a.k_weight : a.q_weight) ? rsqrtf(fmaf(sum, a.inv_d, a.eps)) : 1.f;
                    const float2 by2 = make_float2(by, by);
                    auto scale = [&](float2 (&z)[4], int chunk) {
                        const float4 w0 = weights[of_k][0][chunk], w1 = weights[of_k][1][chunk];
                        z[0] = __fmul2_rn(__fmul2_rn(z[0], by2), make_float2(w0.x, w0.y));
                        z[1] = __fmul2_rn(__fmul2_rn(z[1], by2), make_float2(w0.z, w0.w));
                        z[2] = __fmul2_rn(__fmul2_rn(z[2], by2), make_float2(w1.x, w1.y));
                        z[3] = __fmul2_rn(__fmul2_rn(z[3], by2), make_float2(w1.z, w1.w));
                    };
                    if (holds) scale(u, at);
                    if (!INTERLEAVED && pair) scale(v, at + far);
                    if (turns) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if constexpr (INTERLEAVED)
                                turn1(u[e], e & 1 ? c[e / 2].y : c[e / 2].x, e & 1 ? sn[e / 2].y : sn[e / 2].x);
                            else
                                turn2(u[e], v[e], c[e], sn[e]);
                        }
                    }
                    x[b] = make_uint4(pack2(u[0].x, u[0].y), pack2(u[1].x, u[1].y), pack2(u[2].x, u[2].y), pack2(u[3].x, u[3].y));
                    if (!INTERLEAVED && pair)
                        y[b] = make_uint4(pack2(v[0].x, v[0].y), pack2(v[1].x, v[1].y), pack2(v[2].x, v[2].y), pack2(v[3].x, v[3].y));
                }
            }
            if (mine && (g < 0 || slot)) {
                uint8_t *dst = g < 0 ? q_dst + r * a.D * 2 : slot + g * head_bytes;  // v's heads follow k's
                *reinterpret_cast<uint4 *>(dst) = x[b];
                if (pair) *reinterpret_cast<uint4 *>(dst + far * 16) = y[b];
            }
        }
        first += BATCH * RPW;
        if (first >= rows) {
            first = 0;
            ++t;
        }
    }
}

template <bool INTERLEAVED>
void (*norm_variant(int lanes))(NormArgs)
{
    switch (lanes) {
    case 4: return rotary_norm_kernel<INTERLEAVED, 4>;
    case 8: return rotary_norm_kernel<INTERLEAVED, 8>;
    case 16: return rotary_norm_kernel<INTERLEAVED, 16>;
    default: return rotary_norm_kernel<INTERLEAVED, 32>;
    }
}

}  // namespace

extern "C" int kv_append_rotary_norm(kv_pool *p, int layout, const kv_rotary *rot, const kv_head_norm *norm, const uint16_t *q,
                                     int64_t q_stride, uint16_t *q_out, const uint16_t *k, int64_t k_stride,
                                     const uint16_t *v, int64_t v_stride, const int32_t *positions,
                                     const int32_t *dev_q_starts, int T, const int32_t *dev_table,
                                     const int32_t *dev_ctx_lens, int max_blocks, int S, int Hq, void *stream)
{
    if (!norm) return KV_ERR_INVALID_ARG;
    bool go;
    const int rc = kvp_rotary_check(p, layout, rot, q, q_stride, q_out, k, k_stride, v, v_stride, dev_q_starts, T, dev_table,
                                    dev_ctx_lens, max_blocks, S, Hq, &go);
    if (rc) return rc;
    if (!(norm->eps >= 0.f) || !std::isfinite(norm->eps) || !std::isfinite(norm->offset)) return KV_ERR_INVALID_ARG;
    if (!rotary_aligned16(norm->q_weight) || !rotary_aligned16(norm->k_weight)) return KV_ERR_INVALID_ARG;
    const kv_layout &L = p->desc.layouts[layout];
    if (L.head_dim > kMaxNormDim) return KV_ERR_UNSUPPORTED;
    if (!go) return KV_OK;
    NormArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_out = q_out;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.pool = reinterpret_cast<uint8_t *>(p->desc.device_base);
    a.steps = rot->steps;
    a.positions = positions;
    a.starts = dev_q_starts;
    a.table = dev_table;
    a.ctx_lens = dev_ctx_lens;
    a.err = p->desc.device_error;
    a.q_weight = norm->q_weight;
    a.k_weight = norm->k_weight;
    a.page_bytes = (int64_t)p->page_bytes;
    a.n_pages = p->n_pages;
    a.magnitude = rot->magnitude;
    a.eps = norm->eps;
    a.offset = norm->offset;
    a.inv_d = 1.f / (float)L.head_dim;
    a.pages_per_block = p->pages_per_block[layout];
    a.max_blocks = max_blocks;
    a.S = S;
    a.Hq = Hq;
    a.Hkv = L.num_kv_heads;
    a.D = L.head_dim;
    a.bs = p->desc.block_size;
    a.rot = rot->rot_dim;
    a.items = (rot->interleaved ? a.rot / 8 : a.rot / 16) + (a.D - a.rot) / 8;
    int lanes = 4;
    while (lanes < a.items) lanes *= 2;
    const int batch = (rot->interleaved ? kNormBatch<true> : kNormBatch<false>) * (32 / lanes);
    const int rows = (q ? Hq : 0) + (k ? 2 * a.Hkv : 0);
    a.batches = (rows + batch - 1) / batch;
    const int64_t units = (int64_t)T * a.batches;
    a.warps = std::min((int64_t)kNormResident * std::max(1, p->sm_count) * (kNormThreads / 32), units);
    a.per_warp = units / a.warps;
    a.longer = units % a.warps;
    void (*kernel)(NormArgs) = rot->interleaved ? norm_variant<true>(lanes) : norm_variant<false>(lanes);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.warps + kNormThreads / 32 - 1) / (kNormThreads / 32)));
    cfg.blockDim = dim3(kNormThreads);
    cfg.stream = (cudaStream_t)stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, a) != cudaSuccess) return KV_ERR_CUDA;
    kvp_note_stream(stream, false);
    return KV_OK;
}
