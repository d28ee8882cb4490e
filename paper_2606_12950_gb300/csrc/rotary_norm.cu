// rotary_norm.cu -- the rotary append of models whose query and key heads are
// normed: each head x of q and k becomes
//     R(p) (x / sqrt(mean(x^2) + eps) * (weight + offset))
// (RMSNorm; Zhang and Sennrich, 2019) with R(p) its turn to position p (rotary.cu),
// v is copied, k and v go to the paged pool.
//
// Bound by HBM for prompts (each row read and written once) and by latency for a
// decode step.  A head's columns lie with 4 to 16 lanes of a warp, 16 columns with each
// (two chunks; of the half layout, where it turns, those that turn together), which
// sum its squares by shuffles, so a warp needs no other and no barrier: it takes a range of (token, batch of rows of q, k or v) units, as many as
// every other, computes each token's angles among its lanes, and keeps its columns'
// frequencies from token to token; the weights lie in shared memory in fp32.
// 16000 tokens of 40 q and 8 KV heads of 128 (460 MB): 79.3 us, 5.80 TB/s (0.85 of the
// measured copy; the rotary append, without norms, 74.7), whatever part of a head turns
// and in which layout.  The rotary kernel with norms in it, a CTA a token: 143 (29
// instructions a value: addresses and the choice between q, k and v for every row);
// warps over ranges, rows of q, k and v mixed in a unit: 90.6; one chunk a lane: 79.8,
// and 133 for the half layout with half of a head turned.  Two rows a lane in flight
// and five CTAs an SM: three or four rows 86 and 83 (8 KV heads fill no unit of 12
// or 16 rows), the next unit's rows on their way before this one's products 78.7.
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
constexpr int kNormResident = 5;   // CTAs an SM
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
    int32_t items;                       // of a row
    int32_t units, q_units, kv_units;    // of a token: q_units + 2 kv_units
};

constexpr int kNormBatch = 2;  // rows of a lane in a unit

template <bool INTERLEAVED, int LANES>
__global__ void __launch_bounds__(kNormThreads, kNormResident) rotary_norm_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int RPW = 32 / LANES;             // rows side by side in a warp
    constexpr int NP = 8;                       // pairs of an item that turns
    constexpr int OWN = (NP + RPW - 1) / RPW;   // of which a lane computes
    constexpr int BATCH = kNormBatch;
    constexpr unsigned ALL = 0xffffffffu;
    // weights with the offset, of q and of k: a chunk's first four columns, then its others
    __shared__ __align__(16) float4 weights[2][2][kMaxNormDim / 8];
    const int lane = threadIdx.x & 31, item = lane % LANES, grp = lane / LANES;
    // An item is two chunks of eight columns: of the half layout two that turn together
    // or two that do not turn; of adjacent pairs a chunk of either half of the head.
    const int chunks = a.D / 8, turned = a.rot / 8;  // chunks; those that turn
    const int near = INTERLEAVED || item < turned / 2 ? item : item + turned / 2;
    const int apart = INTERLEAVED ? (chunks + 1) / 2 : item < turned / 2 ? turned / 2 : (chunks - turned + 1) / 2;
    const bool holds = item < a.items, pair = holds && near + apart < (INTERLEAVED || item >= turned / 2 ? chunks : turned);
    const bool turns0 = holds && near < turned, turns1 = INTERLEAVED ? pair && near + apart < turned : turns0;
    // (a lane without columns, or with one chunk, takes any chunk along)
    const int chunk0 = holds ? near : 0, chunk1 = pair ? near + apart : chunk0, hops = (chunk1 - chunk0) * 8;
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
        const int p = e * RPW + grp;  // of adjacent pairs: four of either chunk
        const bool any = p < NP && (INTERLEAVED && p >= 4 ? turns1 : turns0);
        step[e] = any ? a.steps[!INTERLEAVED ? chunk0 * 8 + p : p < 4 ? chunk0 * 4 + p : chunk1 * 4 + p - 4] : 0;
    }
    __syncthreads();

    const int64_t warp = (int64_t)blockIdx.x * (kNormThreads / 32) + (threadIdx.x >> 5);
    int64_t unit = warp * a.per_warp + min(warp, a.longer);
    const int64_t unit_end = unit + a.per_warp + (warp < a.longer);
    if (warp >= a.warps) return;
    int t = (int)(unit / a.units);
    int batch = (int)(unit - (int64_t)t * a.units);      // of the token's
    const int64_t head_bytes = (int64_t)a.bs * a.D * 2;  // of one KV head in a block
    int32_t n = 0, end = INT32_MIN, s = 0;               // the token's sequence, its context, the token past it
    float c[NP], sn[NP];                                 // of the item's pairs
    uint8_t *slot = nullptr;
    int now = -1;                                        // the token whose these are
    for (; unit < unit_end; ++unit) {
        // the unit's rows: of q, k or v alone
        const int of = batch < a.q_units ? 0 : batch < a.q_units + a.kv_units ? 1 : 2;
        const int first = (batch - (of == 0 ? 0 : of == 1 ? a.q_units : a.q_units + a.kv_units)) * BATCH * RPW + grp;
        const int rows = of == 0 ? a.Hq : a.Hkv;
        const uint16_t *src = (of == 0 ? a.q + t * a.q_stride : of == 1 ? a.k + t * a.k_stride : a.v + t * a.v_stride) + chunk0 * 8;
        uint4 x[BATCH], y[BATCH];
        // the rows' addresses need the token alone: they are on their way before its
        // position, angles and slot, four dependent loads away, are known.  (A thread
        // without a row, or without columns, loads others': no branch.)
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const uint16_t *row = src + min(first + b * RPW, rows - 1) * a.D;
            x[b] = *reinterpret_cast<const uint4 *>(row);
            y[b] = *reinterpret_cast<const uint4 *>(row + hops);
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
            if (a.kv_units && n > 0) {
                bool ok = t < end && pos >= 0 && pos < a.max_blocks * a.bs;
                if (ok) {
                    const int32_t b = pos / a.bs, phys = a.table[(int64_t)s * a.max_blocks + b];
                    ok = phys >= 0 && (int64_t)phys + a.pages_per_block <= a.n_pages;
                    if (ok) slot = a.pool + (int64_t)phys * a.page_bytes + (int64_t)(pos - b * a.bs) * a.D * 2;
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
                c[e] = __shfl_sync(ALL, own_c[e / RPW], (e % RPW) * LANES + item);
                sn[e] = __shfl_sync(ALL, own_s[e / RPW], (e % RPW) * LANES + item);
            }
        }
        if (of < 2) {
            const bool normed = (of ? a.k_weight : a.q_weight) != nullptr;
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                float2 u[4], v[4];
                const uint32_t *xw = reinterpret_cast<const uint32_t *>(&x[b]), *yw = reinterpret_cast<const uint32_t *>(&y[b]);
                float2 sum2 = make_float2(0.f, 0.f), far2 = make_float2(0.f, 0.f);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    u[e] = unpack2(xw[e]);
                    sum2 = __ffma2_rn(u[e], u[e], sum2);
                    v[e] = unpack2(yw[e]);
                    far2 = __ffma2_rn(v[e], v[e], far2);
                }
                float sum = (holds ? sum2.x + sum2.y : 0.f) + (pair ? far2.x + far2.y : 0.f);
#pragma unroll
                for (int off = 1; off < LANES; off <<= 1) sum += __shfl_xor_sync(ALL, sum, off);
                const float by = normed ? rsqrtf(fmaf(sum, a.inv_d, a.eps)) : 1.f;
                const float2 by2 = make_float2(by, by);
                auto scale = [&](float2 (&z)[4], int chunk) {
                    const float4 w0 = weights[of][0][chunk], w1 = weights[of][1][chunk];
                    z[0] = __fmul2_rn(__fmul2_rn(z[0], by2), make_float2(w0.x, w0.y));
                    z[1] = __fmul2_rn(__fmul2_rn(z[1], by2), make_float2(w0.z, w0.w));
                    z[2] = __fmul2_rn(__fmul2_rn(z[2], by2), make_float2(w1.x, w1.y));
                    z[3] = __fmul2_rn(__fmul2_rn(z[3], by2), make_float2(w1.z, w1.w));
                };
                scale(u, chunk0);
                scale(v, chunk1);
                if constexpr (INTERLEAVED) {
                    if (turns0) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) turn(u[e].x, u[e].y, c[e], sn[e]);
                    }
                    if (turns1) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) turn(v[e].x, v[e].y, c[4 + e], sn[4 + e]);
                    }
                } else if (turns0) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        turn2(u[e], v[e], make_float2(c[2 * e], c[2 * e + 1]), make_float2(sn[2 * e], sn[2 * e + 1]));
                }
                x[b] = make_uint4(pack2(u[0].x, u[0].y), pack2(u[1].x, u[1].y), pack2(u[2].x, u[2].y), pack2(u[3].x, u[3].y));
                y[b] = make_uint4(pack2(v[0].x, v[0].y), pack2(v[1].x, v[1].y), pack2(v[2].x, v[2].y), pack2(v[3].x, v[3].y));
            }
        }
        uint8_t *dst = of == 0   ? reinterpret_cast<uint8_t *>(a.q_out + (int64_t)t * a.Hq * a.D)
                       : of == 1 ? slot
                                 : slot + a.Hkv * head_bytes;
        const int64_t row_bytes = of == 0 ? a.D * 2 : head_bytes;
        if (holds && (of == 0 || slot)) {
            dst += chunk0 * 16;
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int r = first + b * RPW;
                if (r < rows) {
                    *reinterpret_cast<uint4 *>(dst + r * row_bytes) = x[b];
                    if (pair) *reinterpret_cast<uint4 *>(dst + r * row_bytes + hops * 2) = y[b];
                }
            }
        }
        if (++batch == a.units) {
            batch = 0;
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
    default: return rotary_norm_kernel<INTERLEAVED, 16>;  // (256 columns, and no more)
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
    if (!kvp_on_device(p)) return KV_ERR_INVALID_ARG;
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
    a.items = rot->interleaved ? (a.D / 8 + 1) / 2 : a.rot / 16 + ((a.D - a.rot) / 8 + 1) / 2;
    int lanes = 4;
    while (lanes < a.items) lanes *= 2;
    const int batch = kNormBatch * (32 / lanes);
    a.q_units = q ? (Hq + batch - 1) / batch : 0;
    a.kv_units = k ? (a.Hkv + batch - 1) / batch : 0;
    a.units = a.q_units + 2 * a.kv_units;
    const int64_t units = (int64_t)T * a.units;
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
