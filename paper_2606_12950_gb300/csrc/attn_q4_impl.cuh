// attn_q4_impl.cuh -- decode attention over a context whose first tokens are
// held in 4 bits (KV_Q4 blocks, q4_format.h) and whose last ones are in bf16.
//
// With K_j = s c_j + z (a scale and a least value per token and group of 64
// columns, codes c in 0..15), the scores are
//     q . K_j = sum over groups v of  s_jv (q_v . c_jv) + z_jv sum(q_v)
// and with weights p_j the output's columns of group v are
//     sum_j (p_j s_jv) c_jv + sum_j p_j z_jv.
// So the products take the codes alone, and s and z meet 16 scores and weights a
// token pair instead of 64 columns.  A code pair is an operand after one AND: a
// word masked with 0x000f000f holds two fp16 subnormals, c 2^-24 (16 c 2^-24 with
// 0x00f000f0), exact in the tensor cores' fp16 products.  The factors 2^-24 and
// 1/16 are powers of two that q, the scores' factor and the end of a run undo.
//
// Ranges.  q is scaled by a power of two (its largest column in [2^14, 2^15)),
// so that fp16 holds all bits of its bf16 columns down to 2^-28 of the largest.
// A weight meets V's scale before it is rounded to fp16: the running maximum M is
// that of score + L, L the power of two above the unit's largest V scale, so
// p s <= 2^15 (M moves only when it would be passed, by 2^8 at once).  The sums of
// p and p z are fp32 and need no such range, and records (M, l, o) merge as those
// of the bf16 kernel do.
//
// Work split: a tile is 16 tokens of a (sequence, KV head) run; it costs 9 where
// it is in 4 bits and 32 in bf16 (its bytes).  The batch's tiles, in order, are cut
// into parts of equal cost, one a warp.  A part's pieces of runs leave an output
// (a whole run) or a record for the combine.  Each warp streams its 4-bit tiles
// through its own ring of shared-memory stages (a bulk copy a tile) and reads its
// bf16 tiles straight into registers.
#pragma once

#include <cuda_fp16.h>

#include "attn_impl.cuh"
#include "q4_format.h"

namespace kvp {

constexpr int kQ4Warps = 8;
constexpr int kQ4Threads = kQ4Warps * 32;
constexpr int kQ4Stages = 3;
template <int D>
constexpr int kQ4Unit = D == 64 ? 4 : 2;  // tiles of a stage: 4608 bytes either way
constexpr int kQ4Cost = 9, kBf16Cost = 32;
constexpr int kQ4MinPart = 36;            // a part's least cost: more than any tile's, so that each has one

struct Q4Args {
    const uint16_t *q;
    uint16_t *out;
    const uint16_t *k_new;   // [S][Hkv][d] or null
    const uint16_t *v_new;
    uint8_t *pool;
    const int32_t *table;    // bf16 blocks [S][max_blocks]
    const int32_t *lens;
    const int32_t *table4;   // 4-bit blocks [S][max_blocks4]
    const int32_t *packed;   // tokens held there
    int32_t *err;
    float *ws_part;          // records (combine_kernel)
    int2 *ws_run;            // per run: the parts of its records, [x, y)
    int64_t page_bytes, pool_pages;
    int32_t pages_per_block, pages_per_block4;
    int32_t max_blocks, max_blocks4;
    int32_t S, Hkv, G, bs;
    int32_t P;               // CTAs
    float qk_scale;          // scale * log2(e)
};

template <int D>
inline size_t q4_smem_bytes()
{
    return 128 + (size_t)kQ4Warps * kQ4Stages * (kQ4Unit<D> * kQ4TileBytes<D> + 8) + (kQ4Threads + 1) * sizeof(int64_t);
}

// A sequence's lengths, clamped to what the tables can hold.
struct Q4Seq {
    int32_t n, p;    // tokens; of them in 4 bits
    bool append;     // a new row can be appended
    __device__ int32_t tiles4() const { return p >> 4; }
    __device__ int32_t tiles() const { return (p >> 4) + ((n - p + 15) >> 4); }
    __device__ int32_t cost() const { return kQ4Cost * (p >> 4) + kBf16Cost * ((n - p + 15) >> 4); }
};

__device__ __forceinline__ Q4Seq q4_seq(const Q4Args &a, int s)
{
    const int32_t n = a.lens[s], p = a.packed[s];
    const int32_t cap = a.max_blocks * a.bs, cap4 = a.max_blocks4 * a.bs;
    Q4Seq q;
    q.n = min(max(n, 0), cap);
    q.p = min(min(max(p, 0), q.n), cap4) & ~15;
    q.append = n == q.n && n > q.p;
    return q;
}

// the tile of a run at cost position x or the first one after it
__device__ __forceinline__ int32_t q4_tile_at(const Q4Seq &q, int32_t x)
{
    const int32_t c4 = kQ4Cost * q.tiles4();
    return x <= c4 ? (int32_t)((uint32_t)(x + kQ4Cost - 1) / (uint32_t)kQ4Cost)
                   : q.tiles4() + (x - c4 + kBf16Cost - 1) / kBf16Cost;
}

// D(16x8, f32) += A(16x16, f16, row) * B(16x8, f16, col)
__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                              uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t f16_pair(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// `bytes` from global to shared memory, completing on `bar`
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar, uint64_t policy)
{
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(
            dst),
        "l"(src), "r"(bytes), "r"(bar), "l"(policy)
        : "memory");
}

// One run's state in a warp.  lane = 4 g + t; tokens of a tile are rows g and g +
// 8 of the scores, query heads 2 t and 2 t + 1 their columns.
template <int D>
struct Q4State {
    static constexpr int NG = D / kQ4Group, NW = D / 32, NM = D / 16;
    uint32_t qh[NW][4];     // q, head g: words of 8 columns as the K words pair them, fp16
    float qsum[NG][2];      // 2^-24 times the scaled q's sums over groups, heads 2 t and 2 t + 1
    float factor[2];        // of the scores, to base-2 exponents
    float m[2], l[2];
    float z[NG][2];         // sums of p z over this lane's tokens
    float acc[NM][4];       // sums of p s c: row pairs (e, e + 1), odd columns times 16, all times 2^-24

    // qrow: q rows of the run's G heads
    __device__ __forceinline__ void begin(const uint16_t *qrow, int G, float qk_scale, int lane)
    {
        const int gid = lane >> 2, tig = lane & 3;
        uint4 w[NW];
        float mx = 0.f;
#pragma unroll
        for (int j = 0; j < NW; ++j) {
            w[j] = gid < G ? *reinterpret_cast<const uint4 *>(qrow + gid * D + 64 * (j >> 1) + 32 * (j & 1) + 8 * tig)
                           : make_uint4(0u, 0u, 0u, 0u);
            const uint32_t *x = reinterpret_cast<const uint32_t *>(&w[j]);
#pragma unroll
            for (int e = 0; e < 4; ++e) mx = fmaxf(mx, fmaxf(fabsf(bf_lo(x[e])), fabsf(bf_hi(x[e]))));
        }
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        // 2^e: the largest column to [2^14, 2^15)
        int e = 14 + 127 - (int)(__float_as_uint(mx) >> 23);
        e = mx > 0.f ? min(max(e, -90), 120) : 0;
        const float up = __uint_as_float((uint32_t)(e + 127) << 23);
        float sums[NG];
#pragma unroll
        for (int c = 0; c < NG; ++c) sums[c] = 0.f;
#pragma unroll
        for (int j = 0; j < NW; ++j) {
            const uint32_t *x = reinterpret_cast<const uint32_t *>(&w[j]);
            float f[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f[2 * i] = bf_lo(x[i]) * up;
                f[2 * i + 1] = bf_hi(x[i]) * up;
            }
            qh[j][0] = f16_pair(f[0], f[4]);
            qh[j][1] = f16_pair(f[1] * 0.0625f, f[5] * 0.0625f);
            qh[j][2] = f16_pair(f[2], f[6]);
            qh[j][3] = f16_pair(f[3] * 0.0625f, f[7] * 0.0625f);
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[j >> 1] += f[i];
        }
#pragma unroll
        for (int c = 0; c < NG; ++c) {
            sums[c] += __shfl_xor_sync(0xffffffffu, sums[c], 1);
            sums[c] += __shfl_xor_sync(0xffffffffu, sums[c], 2);
            qsum[c][0] = __shfl_sync(0xffffffffu, sums[c], 8 * tig) * 0x1p-24f;
            qsum[c][1] = __shfl_sync(0xffffffffu, sums[c], 8 * tig + 4) * 0x1p-24f;
            z[c][0] = z[c][1] = 0.f;
        }
        const int e0 = __shfl_sync(0xffffffffu, e, 8 * tig), e1 = __shfl_sync(0xffffffffu, e, 8 * tig + 4);
        factor[0] = qk_scale * __uint_as_float((uint32_t)(24 - e0 + 127) << 23);
        factor[1] = qk_scale * __uint_as_float((uint32_t)(24 - e1 + 127) << 23);
        m[0] = m[1] = kMaxStart;
        l[0] = l[1] = 0.f;
#pragma unroll
        for (int i = 0; i < NM; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[i][k] = 0.f;
    }

    // The maximum's new place where a score passes it: y0, y1 the lane's largest
    // scores plus L.
    __device__ __forceinline__ void raise(float y0, float y1)
    {
        if (!__any_sync(0xffffffffu, y0 > m[0] + 15.f || y1 > m[1] + 15.f)) return;
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) {
            y0 = fmaxf(y0, __shfl_xor_sync(0xffffffffu, y0, off));
            y1 = fmaxf(y1, __shfl_xor_sync(0xffffffffu, y1, off));
        }
        const float m0 = y0 > m[0] + 15.f ? y0 - 7.f : m[0], m1 = y1 > m[1] + 15.f ? y1 - 7.f : m[1];
        const float f0 = fast_exp2(m[0] - m0), f1 = fast_exp2(m[1] - m1);
        m[0] = m0;
        m[1] = m1;
        l[0] *= f0;
        l[1] *= f1;
#pragma unroll
        for (int c = 0; c < NG; ++c) {
            z[c][0] *= f0;
            z[c][1] *= f1;
        }
#pragma unroll
        for (int i = 0; i < NM; ++i) {
            acc[i][0] *= f0;
            acc[i][1] *= f1;
            acc[i][2] *= f0;
            acc[i][3] *= f1;
        }
    }

    // a unit of `tiles` tiles in 4 bits
    __device__ __forceinline__ void unit4(const uint8_t *stage, int tiles, int lane)
    {
        constexpr int U = kQ4Unit<D>, TILE = kQ4TileBytes<D>;
        const int gid = lane >> 2, tig = lane & 3;
        float y[U][4];
        uint32_t vp[U][2][NG];
        float y0 = -INFINITY, y1 = -INFINITY;
        uint32_t top = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u < tiles) {
                const uint8_t *tile = stage + u * TILE;
                uint32_t ka[NW], kb[NW];
                const uint8_t *ra = tile + gid * (D / 2) + tig * (D / 8), *rb = ra + 8 * (D / 2);
                if constexpr (NW == 4) {
                    const uint4 x = *reinterpret_cast<const uint4 *>(ra), w = *reinterpret_cast<const uint4 *>(rb);
                    ka[0] = x.x, ka[1] = x.y, ka[2] = x.z, ka[3] = x.w;
                    kb[0] = w.x, kb[1] = w.y, kb[2] = w.z, kb[3] = w.w;
                } else {
                    const uint2 x = *reinterpret_cast<const uint2 *>(ra), w = *reinterpret_cast<const uint2 *>(rb);
                    ka[0] = x.x, ka[1] = x.y;
                    kb[0] = w.x, kb[1] = w.y;
                }
                const uint32_t *kpar = reinterpret_cast<const uint32_t *>(tile + 16 * D);
                const uint32_t *vpar = kpar + 16 * NG;
                uint32_t kp[2][NG];
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int c = 0; c < NG; ++c) {
                        kp[r][c] = kpar[(gid + 8 * r) * NG + c];
                        vp[u][r][c] = vpar[(gid + 8 * r) * NG + c];
                        top = max(top, vp[u][r][c] << 16);
                    }
                float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < NG; ++c) {
                    float dot[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = 2 * c; j < 2 * c + 2; ++j) {
                        mma_f16_16816(dot, ka[j] & 0x000f000fu, kb[j] & 0x000f000fu, ka[j] & 0x00f000f0u,
                                      kb[j] & 0x00f000f0u, qh[j][0], qh[j][1]);
                        const uint32_t wa = ka[j] >> 8, wb = kb[j] >> 8;
                        mma_f16_16816(dot, wa & 0x000f000fu, wb & 0x000f000fu, wa & 0x00f000f0u, wb & 0x00f000f0u,
                                      qh[j][2], qh[j][3]);
                    }
                    const float sa = bf_lo(kp[0][c]), za = bf_hi(kp[0][c]), sb = bf_lo(kp[1][c]), zb = bf_hi(kp[1][c]);
                    x[0] = fmaf(dot[0], sa, fmaf(qsum[c][0], za, x[0]));
                    x[1] = fmaf(dot[1], sa, fmaf(qsum[c][1], za, x[1]));
                    x[2] = fmaf(dot[2], sb, fmaf(qsum[c][0], zb, x[2]));
                    x[3] = fmaf(dot[3], sb, fmaf(qsum[c][1], zb, x[3]));
                }
                y[u][0] = x[0] * factor[0];
                y[u][1] = x[1] * factor[1];
                y[u][2] = x[2] * factor[0];
                y[u][3] = x[3] * factor[1];
                y0 = fmaxf(y0, fmaxf(y[u][0], y[u][2]));
                y1 = fmaxf(y1, fmaxf(y[u][1], y[u][3]));
            }
        }
        // L: a power of two above every V scale of the unit, from 2^-40 to 2^80
        top = __reduce_max_sync(0xffffffffu, top);
        const float L = (float)min(max((int)(top >> 23) - 126, -40), 80);
        raise(y0 + L, y1 + L);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u < tiles) {
                const uint8_t *tile = stage + u * TILE;
                const float p0 = fast_exp2(y[u][0] - m[0]), p1 = fast_exp2(y[u][1] - m[1]);
                const float p2 = fast_exp2(y[u][2] - m[0]), p3 = fast_exp2(y[u][3] - m[1]);
                l[0] += p0 + p2;
                l[1] += p1 + p3;
#pragma unroll
                for (int c = 0; c < NG; ++c) {
                    const float sa = bf_lo(vp[u][0][c]), za = bf_hi(vp[u][0][c]);
                    const float sb = bf_lo(vp[u][1][c]), zb = bf_hi(vp[u][1][c]);
                    z[c][0] = fmaf(p0, za, fmaf(p2, zb, z[c][0]));
                    z[c][1] = fmaf(p1, za, fmaf(p3, zb, z[c][1]));
                    const uint32_t b0 = movmatrix_trans(f16_pair(p0 * sa, p1 * sa));
                    const uint32_t b1 = movmatrix_trans(f16_pair(p2 * sb, p3 * sb));
                    const uint4 v = *reinterpret_cast<const uint4 *>(tile + 8 * D + 512 * c + 16 * lane);
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t h = w[i] >> 8;
                        mma_f16_16816(acc[4 * c + i], w[i] & 0x000f000fu, w[i] & 0x00f000f0u, h & 0x000f000fu,
                                      h & 0x00f000f0u, b0, b1);
                    }
                }
            }
        }
    }

    // a tile of `valid` tokens in bf16: rows k[r], r = g and g + 8, and v[r], r = 2 t,
    // 2 t + 1, 2 t + 8, 2 t + 9 (null: none); qrow as in begin
    __device__ __forceinline__ void tile16(const uint16_t *const (&k)[2], const uint16_t *const (&v)[4],
                                           const uint16_t *qrow, int G, float qk_scale, int lane)
    {
        const int gid = lane >> 2, tig = lane & 3;
        uint4 kw[2][NW], vw[4][NG];
        const uint4 none = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int j = 0; j < NW; ++j)
#pragma unroll
            for (int r = 0; r < 2; ++r)
                kw[r][j] = k[r] ? *reinterpret_cast<const uint4 *>(k[r] + 64 * (j >> 1) + 32 * (j & 1) + 8 * tig) : none;
#pragma unroll
        for (int c = 0; c < NG; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                vw[r][c] = v[r] ? *reinterpret_cast<const uint4 *>(v[r] + 64 * c + 8 * gid) : none;
        float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NW; ++j) {
            const uint4 q = gid < G ? *reinterpret_cast<const uint4 *>(qrow + gid * D + 64 * (j >> 1) + 32 * (j & 1) + 8 * tig)
                                    : none;
            mma_bf16_16816(x, kw[0][j].x, kw[1][j].x, kw[0][j].y, kw[1][j].y, q.x, q.y);
            mma_bf16_16816(x, kw[0][j].z, kw[1][j].z, kw[0][j].w, kw[1][j].w, q.z, q.w);
        }
        const float no = -INFINITY;
        const float ya = k[0] ? x[0] * qk_scale : no, yb = k[0] ? x[1] * qk_scale : no;
        const float yc = k[1] ? x[2] * qk_scale : no, yd = k[1] ? x[3] * qk_scale : no;
        raise(fmaxf(ya, yc), fmaxf(yb, yd));
        const float p0 = fast_exp2(ya - m[0]), p1 = fast_exp2(yb - m[1]);
        const float p2 = fast_exp2(yc - m[0]), p3 = fast_exp2(yd - m[1]);
        l[0] += p0 + p2;
        l[1] += p1 + p3;
        // the accumulators' units: weights times 2^-24, odd columns times 16
        const float down = 0x1p-24f;
        const uint32_t b0 = movmatrix_trans(bf16_pair(p0 * down, p1 * down));
        const uint32_t b1 = movmatrix_trans(bf16_pair(p2 * down, p3 * down));
        const __nv_bfloat162 up = __float2bfloat162_rn(16.f);
#pragma unroll
        for (int c = 0; c < NG; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t a[4];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t w0 = reinterpret_cast<const uint32_t *>(&vw[2 * r][c])[i];
                    const uint32_t w1 = reinterpret_cast<const uint32_t *>(&vw[2 * r + 1][c])[i];
                    a[2 * r] = __byte_perm(w0, w1, 0x5410);
                    const uint32_t odd = __byte_perm(w0, w1, 0x7632);
                    const __nv_bfloat162 o = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&odd), up);
                    a[2 * r + 1] = *reinterpret_cast<const uint32_t *>(&o);
                }
                mma_bf16_16816(acc[4 * c + i], a[0], a[1], a[2], a[3], b0, b1);
            }
    }

    // end of a piece: the run's bf16 outputs, or its record (see attn_impl.cuh)
    __device__ __forceinline__ void store(uint16_t *orow, float *slot, bool split, int G, int lane)
    {
        const int gid = lane >> 2, tig = lane & 3;
#pragma unroll
        for (int off = 4; off < 32; off <<= 1)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                l[h] += __shfl_xor_sync(0xffffffffu, l[h], off);
#pragma unroll
                for (int c = 0; c < NG; ++c) z[c][h] += __shfl_xor_sync(0xffffffffu, z[c][h], off);
            }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int head = 2 * tig + h;
            if (head >= G) continue;
#pragma unroll
            for (int c = 0; c < NG; ++c) {
                float o[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    o[2 * i] = fmaf(acc[4 * c + i][h], 0x1p24f, z[c][h]);
                    o[2 * i + 1] = fmaf(acc[4 * c + i][2 + h], 0x1p20f, z[c][h]);
                }
                const int at = head * D + 64 * c + 8 * gid;
                if (split) {
                    *reinterpret_cast<float4 *>(slot + at) = make_float4(o[0], o[1], o[2], o[3]);
                    *reinterpret_cast<float4 *>(slot + at + 4) = make_float4(o[4], o[5], o[6], o[7]);
                } else {
                    uint4 w;
                    w.x = bf16_pair(o[0] / l[h], o[1] / l[h]);
                    w.y = bf16_pair(o[2] / l[h], o[3] / l[h]);
                    w.z = bf16_pair(o[4] / l[h], o[5] / l[h]);
                    w.w = bf16_pair(o[6] / l[h], o[7] / l[h]);
                    *reinterpret_cast<uint4 *>(orow + at) = w;
                }
            }
            if (split && gid == 0) {
                slot[G * D + head] = m[h];
                slot[G * D + G + head] = l[h];
            }
        }
    }
};

template <int D>
__global__ void __launch_bounds__(kQ4Threads, 2) q4_attn_kernel(const __grid_constant__ Q4Args a)
{
    constexpr int TILE = kQ4TileBytes<D>, U = kQ4Unit<D>, STAGE = U * TILE;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((128u - (smem_u32(smem_raw) & 127u)) & 127u);
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + (size_t)kQ4Warps * kQ4Stages * STAGE);
    int64_t *base = reinterpret_cast<int64_t *>(bars + kQ4Warps * kQ4Stages);  // [threads + 1] costs before a thread's sequences
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const int bid = blockIdx.x, S = a.S;
    if (tid == 0) {
        for (int i = 0; i < kQ4Warps * kQ4Stages; ++i) mbar_init(smem_u32(&bars[i]), 1);
        fence_mbar_init();
    }
    grid_launch_dependents();
    grid_dependency_wait();

    // ---- the cost before each thread's sequences ----
    const int per = (S + kQ4Threads - 1) / kQ4Threads;
    {
        const int lo = min(S, tid * per), hi = min(S, lo + per);
        int64_t sum = 0;
        for (int s = lo; s < hi; ++s) {
            const Q4Seq q = q4_seq(a, s);
            sum += (int64_t)q.cost() * a.Hkv;
            if (s % a.P == bid) {
                const int32_t n = a.lens[s], p = a.packed[s];
                if (n != q.n || p != q.p || (a.k_new && n > 0 && !q.append)) report(a.err, KV_ERR_DEVICE_BOUNDS);
                if (q.n == 0) {  // no softmax: zeros
                    for (int i = 0; i < a.Hkv * a.G * D; ++i) a.out[(int64_t)s * a.Hkv * a.G * D + i] = 0;
                    for (int g = 0; g < a.Hkv; ++g) a.ws_run[(int64_t)s * a.Hkv + g] = make_int2(0, 0);
                }
            }
        }
        int64_t incl = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int64_t v = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += v;
        }
        __shared__ int64_t tops[kQ4Warps];
        if (lane == 31) tops[warp] = incl;
        __syncthreads();
        int64_t before = 0;
        for (int w = 0; w < warp; ++w) before += tops[w];
        base[tid] = before + incl - sum;
        if (tid == kQ4Threads - 1) base[kQ4Threads] = before + incl;
        __syncthreads();
    }
    const int64_t W = base[kQ4Threads];
    const int64_t NP = min((int64_t)a.P * kQ4Warps, max((int64_t)1, W / kQ4MinPart));  // parts
    const int part = warp * a.P + bid;
    if (part >= NP || W == 0) return;  // (no barrier of the CTA below)
    const int64_t w0 = part * (W / NP) + part * (W % NP) / NP;
    const int64_t w1 = (part + 1) * (W / NP) + (part + 1) * (W % NP) / NP;

    // ---- the run at the part's start ----
    struct Run {
        Q4Seq q;
        int32_t s, g;
        int64_t begin;       // cost before it
        int32_t i0, i1;      // this part's tiles of it
    };
    auto tiles_of = [&](Run &r) {
        const int64_t x0 = w0 - r.begin, x1 = w1 - r.begin;
        r.i0 = x0 <= 0 ? 0 : q4_tile_at(r.q, (int32_t)x0);
        r.i1 = x1 >= r.q.cost() ? r.q.tiles() : q4_tile_at(r.q, (int32_t)x1);
    };
    // the run after r that has tiles in this part; false if there is none
    auto next = [&](Run &r) {
        r.begin += r.q.cost();
        if (++r.g == a.Hkv) {
            r.g = 0;
            do {
                if (r.begin >= w1 || ++r.s >= S) return false;
                r.q = q4_seq(a, r.s);
            } while (r.q.n == 0);
        }
        if (r.begin >= w1) return false;
        tiles_of(r);
        return r.i1 > r.i0;
    };
    Run run;
    {
        int lo = 0, hi = kQ4Threads;  // the last thread whose sequences start at or before w0, with any cost
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (base[mid] <= w0) lo = mid; else hi = mid;
        }
        run.begin = base[lo];
        run.s = lo * per;
        run.q = q4_seq(a, run.s);
        while (run.begin + (int64_t)run.q.cost() * a.Hkv <= w0) {
            run.begin += (int64_t)run.q.cost() * a.Hkv;
            run.q = q4_seq(a, ++run.s);
        }
        run.g = (int32_t)((w0 - run.begin) / run.q.cost());
        run.begin += (int64_t)run.g * run.q.cost();
        tiles_of(run);
        // (the part may start past this run's last tile)
        if (run.i0 >= run.i1 && !next(run)) return;
    }

    // ---- the ring: this warp's 4-bit tiles, piece after piece ----
    uint8_t *ring = smem + (size_t)warp * kQ4Stages * STAGE;
    const uint64_t policy = l2_policy_evict_first();
    Run ahead = run;
    bool more = true;       // `ahead` is a run of this part
    int32_t at = run.i0;    // its next tile to ask for
    int32_t ids = 0, ids_at = -32;  // table entries of tiles ids_at + lane
    uint32_t issued = 0;
    auto issue = [&]() {    // the next unit, if there is one
        while (more && at >= min(ahead.i1, ahead.q.tiles4())) {
            more = next(ahead);
            at = ahead.i0;
            ids_at = -32;
        }
        if (!more) return;
        const int32_t end = min(ahead.i1, ahead.q.tiles4());
        const int st = issued % kQ4Stages;
        const uint32_t bar = smem_u32(&bars[warp * kQ4Stages + st]);
        if (ids_at < 0 || at + U > ids_at + 32) {
            ids_at = at;
            const int32_t i = at + lane;
            ids = i < end ? a.table4[(int64_t)ahead.s * a.max_blocks4 + i * 16 / a.bs] : -1;
        }
        const int32_t i = at + lane;
        const bool mine = lane < U && i < end;
        const int32_t id = __shfl_sync(0xffffffffu, ids, (at - ids_at + lane) & 31);
        const bool good = mine && id >= 0 && (int64_t)id + a.pages_per_block4 <= a.pool_pages;
        if (mine && !good) report(a.err, KV_ERR_DEVICE_BOUNDS);
        const uint32_t n = __popc(__ballot_sync(0xffffffffu, good));
        if (lane == 0) mbar_arrive_expect_tx(bar, n * TILE);
        __syncwarp();
        if (good) {
            const int32_t t = i % (a.bs / 16);
            const uint8_t *src = a.pool + (int64_t)id * a.page_bytes + ((int64_t)ahead.g * (a.bs / 16) + t) * TILE;
            bulk_load(smem_u32(ring + st * STAGE + lane * TILE), src, TILE, bar, policy);
        }
        __syncwarp();
        at = min(at + U, end);
        ++issued;
    };
    for (int st = 0; st < kQ4Stages; ++st) issue();

    bool dead = false;
    uint32_t used = 0;
    for (bool go = true; go; go = next(run)) {
        const Q4Seq q = run.q;
        const int32_t r = run.s * a.Hkv + run.g;
        const uint16_t *qrow = a.q + (int64_t)r * a.G * D;
        Q4State<D> st;
        st.begin(qrow, a.G, a.qk_scale, lane);
        const int32_t end4 = min(run.i1, q.tiles4());
        for (int32_t i = run.i0; i < end4; i += U) {
            const int k = used % kQ4Stages;
            wait_phase(smem_u32(&bars[warp * kQ4Stages + k]), (used / kQ4Stages) & 1u, a.err, dead);
            st.unit4(ring + k * STAGE, min(U, end4 - i), lane);
            ++used;
            // the stage is refilled by bulk copies next: after this warp's reads
            fence_proxy_async_smem();
            __syncwarp();
            issue();
        }
        for (int32_t i = max(run.i0, q.tiles4()); i < run.i1; ++i) {
            const int32_t tok0 = q.p + (i - q.tiles4()) * 16;
            const int gid = lane >> 2, tig = lane & 3;
            auto row = [&](int rr, int kv) -> const uint16_t * {
                const int32_t j = tok0 + rr;
                if (j >= q.n) return nullptr;
                if (a.k_new && q.append && j == q.n - 1) return (kv ? a.v_new : a.k_new) + (int64_t)r * D;
                const int32_t id = a.table[(int64_t)run.s * a.max_blocks + j / a.bs];
                if (id < 0 || (int64_t)id + a.pages_per_block > a.pool_pages) {
                    report(a.err, KV_ERR_DEVICE_BOUNDS);
                    return nullptr;
                }
                return reinterpret_cast<const uint16_t *>(a.pool + (int64_t)id * a.page_bytes) +
                       ((int64_t)(kv * a.Hkv + run.g) * a.bs + j % a.bs) * D;
            };
            const uint16_t *const k[2] = {row(gid, 0), row(gid + 8, 0)};
            const uint16_t *const v[4] = {row(2 * tig, 1), row(2 * tig + 1, 1), row(2 * tig + 8, 1), row(2 * tig + 9, 1)};
            st.tile16(k, v, qrow, a.G, a.qk_scale, lane);
            if (a.k_new && q.append && tok0 + 16 >= q.n && lane < D / 4) {  // the new row's place
                const int32_t j = q.n - 1;
                const int32_t id = a.table[(int64_t)run.s * a.max_blocks + j / a.bs];
                if (id >= 0 && (int64_t)id + a.pages_per_block <= a.pool_pages) {
                    const int kv = lane / (D / 8), c = lane % (D / 8);
                    uint16_t *dst = reinterpret_cast<uint16_t *>(a.pool + (int64_t)id * a.page_bytes) +
                                    ((int64_t)(kv * a.Hkv + run.g) * a.bs + j % a.bs) * D;
                    *reinterpret_cast<uint4 *>(dst + c * 8) =
                        *reinterpret_cast<const uint4 *>((kv ? a.v_new : a.k_new) + (int64_t)r * D + c * 8);
                } else {
                    report(a.err, KV_ERR_DEVICE_BOUNDS);
                }
            }
        }
        // ---- end of a piece ----
        const bool first = run.i0 == 0, last = run.i1 == q.tiles();
        const bool split = !(first && last);
        st.store(a.out + (int64_t)r * a.G * D, a.ws_part + ((int64_t)r + part) * ((a.G * D + 2 * a.G + 3) / 4 * 4), split,
                 a.G, lane);
        if (lane == 0) {
            if (first) a.ws_run[r].x = part;
            if (last) a.ws_run[r].y = split ? part + 1 : part;
        }
    }
}

}  // namespace kvp

// one entry per head dim: the CTAs that are resident at once (launch false), or
// both kernels
int kvp_q4_attn_d64(int G, const kvp::Q4Args *a, int sm_count, cudaStream_t st, bool launch, int *P_out);
int kvp_q4_attn_d128(int G, const kvp::Q4Args *a, int sm_count, cudaStream_t st, bool launch, int *P_out);
