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
// into parts of equal cost, one a CTA, and those into equal ones, one a warp.  A
// run inside a CTA leaves its output, others a record a CTA for the combine (the
// warps' states merged in shared memory).  Each warp streams its 4-bit tiles
// through its own ring of shared-memory stages (a bulk copy a tile) and reads its
// bf16 tiles straight into registers.
#pragma once

#include <cuda_fp16.h>

#include "attn_impl.cuh"
#include "q4_format.h"

namespace kvp {

constexpr int kQ4Warps = 8;
constexpr int kQ4Threads = kQ4Warps * 32;
constexpr int kQ4Stages = 2;
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

__host__ __device__ constexpr int q4_record_floats(int D, int G) { return (G * D + 2 * G + 3) / 4 * 4; }

// shared memory of a CTA: per warp its stages and a record; barriers, costs
template <int D>
inline size_t q4_smem_bytes(int G)
{
    return 128 + (size_t)kQ4Warps * (kQ4Stages * (kQ4Unit<D> * kQ4TileBytes<D> + 8) + q4_record_floats(D, G) * 4 + 16) +
           (kQ4Threads + 1) * sizeof(int64_t);
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
// the same onto zeros
__device__ __forceinline__ void mma_f16_16816_0(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%10, %10, %10, %10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_bf16_16816_0(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                 uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%10, %10, %10, %10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
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
    uint32_t qsum[2];       // 2^-24 times the scaled q's sums over groups, head g, as the z's operand
    float factor[2];        // of the scores, to base-2 exponents; not negative
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
        // (a negative factor of the scores goes to q)
        const float up = __uint_as_float((uint32_t)(e + 127) << 23 | (__float_as_uint(qk_scale) & 0x80000000u));
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
        // each sum as three bf16 terms, which hold all its bits.  The operand's rows
        // k = 2 t and 2 t + 1 meet a group's (s, z) of a token: 0 for s, a term for z.
        uint32_t part[NG][3];
#pragma unroll
        for (int c = 0; c < NG; ++c) {
            sums[c] += __shfl_xor_sync(0xffffffffu, sums[c], 1);
            sums[c] += __shfl_xor_sync(0xffffffffu, sums[c], 2);
            float rest = sums[c] * 0x1p-24f;
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                const __nv_bfloat16 b = __float2bfloat16_rn(rest);
                rest -= __bfloat162float(b);
                part[c][i] = (uint32_t)__bfloat16_as_ushort(b) << 16;
            }
            z[c][0] = z[c][1] = 0.f;
        }
        if constexpr (NG == 2) {  // t: group t % 2, its first (t < 2) or second term; then the third
            qsum[0] = tig == 0 ? part[0][0] : tig == 1 ? part[1][0] : tig == 2 ? part[0][1] : part[1][1];
            qsum[1] = tig == 0 ? part[0][2] : tig == 1 ? part[1][2] : 0u;
        } else {                  // t: term t
            qsum[0] = tig == 0 ? part[0][0] : tig == 1 ? part[0][1] : tig == 2 ? part[0][2] : 0u;
            qsum[1] = 0u;
        }
        const int e0 = __shfl_sync(0xffffffffu, e, 8 * tig), e1 = __shfl_sync(0xffffffffu, e, 8 * tig + 4);
        factor[0] = fabsf(qk_scale) * __uint_as_float((uint32_t)(24 - e0 + 127) << 23);
        factor[1] = fabsf(qk_scale) * __uint_as_float((uint32_t)(24 - e1 + 127) << 23);
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

    // a unit of `tiles` tiles in 4 bits (FULL: of kQ4Unit)
    template <bool FULL>
    __device__ __forceinline__ void unit4(const uint8_t *stage, int tiles, int lane)
    {
        constexpr int U = kQ4Unit<D>, TILE = kQ4TileBytes<D>;
        const int gid = lane >> 2, tig = lane & 3;
        float x[U][4];
        uint32_t vp[U][2][NG];
        float x0 = -INFINITY, x1 = -INFINITY;
        uint32_t top = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (FULL || u < tiles) {
                const uint8_t *tile = stage + u * TILE;
                uint32_t ka[NW], kb[NW], kp[2][NG];
                const uint8_t *ra = tile + gid * (D / 2) + tig * (D / 8), *rb = ra + 8 * (D / 2);
                const uint8_t *pa = tile + 16 * D + gid * 8 * NG, *pb = pa + 64 * NG;
                if constexpr (NG == 2) {
                    const uint4 x = *reinterpret_cast<const uint4 *>(ra), w = *reinterpret_cast<const uint4 *>(rb);
                    ka[0] = x.x, ka[1] = x.y, ka[2] = x.z, ka[3] = x.w;
                    kb[0] = w.x, kb[1] = w.y, kb[2] = w.z, kb[3] = w.w;
                    const uint4 a = *reinterpret_cast<const uint4 *>(pa), b = *reinterpret_cast<const uint4 *>(pb);
                    kp[0][0] = a.x, kp[0][1] = a.y, vp[u][0][0] = a.z, vp[u][0][1] = a.w;
                    kp[1][0] = b.x, kp[1][1] = b.y, vp[u][1][0] = b.z, vp[u][1][1] = b.w;
                } else {
                    const uint2 x = *reinterpret_cast<const uint2 *>(ra), w = *reinterpret_cast<const uint2 *>(rb);
                    ka[0] = x.x, ka[1] = x.y;
                    kb[0] = w.x, kb[1] = w.y;
                    const uint2 a = *reinterpret_cast<const uint2 *>(pa), b = *reinterpret_cast<const uint2 *>(pb);
                    kp[0][0] = a.x, vp[u][0][0] = a.y;
                    kp[1][0] = b.x, vp[u][1][0] = b.y;
                }
                // z . q: the words (s, z) themselves are the operand
                float zq[4];
                const uint32_t wa = NG == 2 && (tig & 1) ? kp[0][NG - 1] : kp[0][0];
                const uint32_t wb = NG == 2 && (tig & 1) ? kp[1][NG - 1] : kp[1][0];
                mma_bf16_16816_0(zq, wa, wb, wa, wb, qsum[0], qsum[1]);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[u][i] = zq[i];
#pragma unroll
                for (int c = 0; c < NG; ++c) {
                    float dot[4];
#pragma unroll
                    for (int j = 2 * c; j < 2 * c + 2; ++j) {
                        if (j == 2 * c)
                            mma_f16_16816_0(dot, ka[j] & 0x000f000fu, kb[j] & 0x000f000fu, ka[j] & 0x00f000f0u,
                                            kb[j] & 0x00f000f0u, qh[j][0], qh[j][1]);
                        else
                            mma_f16_16816(dot, ka[j] & 0x000f000fu, kb[j] & 0x000f000fu, ka[j] & 0x00f000f0u,
                                          kb[j] & 0x00f000f0u, qh[j][0], qh[j][1]);
                        const uint32_t ha = ka[j] >> 8, hb = kb[j] >> 8;
                        mma_f16_16816(dot, ha & 0x000f000fu, hb & 0x000f000fu, ha & 0x00f000f0u, hb & 0x00f000f0u,
                                      qh[j][2], qh[j][3]);
                    }
                    const float sa = bf_lo(kp[0][c]), sb = bf_lo(kp[1][c]);
                    x[u][0] = fmaf(dot[0], sa, x[u][0]);
                    x[u][1] = fmaf(dot[1], sa, x[u][1]);
                    x[u][2] = fmaf(dot[2], sb, x[u][2]);
                    x[u][3] = fmaf(dot[3], sb, x[u][3]);
                    top = __vmaxu2(top, __vmaxu2(vp[u][0][c], vp[u][1][c]));
                }
                x0 = fmaxf(x0, fmaxf(x[u][0], x[u][2]));
                x1 = fmaxf(x1, fmaxf(x[u][1], x[u][3]));
            }
        }
        // L: a power of two above every V scale of the unit, from 2^-40 to 2^80
        top = __reduce_max_sync(0xffffffffu, top << 16);
        const float L = (float)min(max((int)(top >> 23) - 126, -40), 80);
        raise(fmaf(x0, factor[0], L), fmaf(x1, factor[1], L));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (FULL || u < tiles) {
                const uint8_t *tile = stage + u * TILE;
                const float p0 = fast_exp2(fmaf(x[u][0], factor[0], -m[0])), p1 = fast_exp2(fmaf(x[u][1], factor[1], -m[1]));
                const float p2 = fast_exp2(fmaf(x[u][2], factor[0], -m[0])), p3 = fast_exp2(fmaf(x[u][3], factor[1], -m[1]));
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
    const int G = a.G, MF = q4_record_floats(D, G);
    float *recs = reinterpret_cast<float *>(smem + (size_t)kQ4Warps * kQ4Stages * STAGE);  // [warps][MF]
    int4 *chains = reinterpret_cast<int4 *>(recs + kQ4Warps * MF);                          // [warps]
    uint64_t *bars = reinterpret_cast<uint64_t *>(chains + kQ4Warps);
    int64_t *base = reinterpret_cast<int64_t *>(bars + kQ4Warps * kQ4Stages);  // [threads + 1] costs before a thread's sequences
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const int bid = blockIdx.x, S = a.S;
    if (tid == 0) {
        for (int i = 0; i < kQ4Warps * kQ4Stages; ++i) mbar_init(smem_u32(&bars[i]), 1);
        fence_mbar_init();
    }
    if (lane == 0) chains[warp].x = -1;
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
                    for (int i = 0; i < a.Hkv * G * D; ++i) a.out[(int64_t)s * a.Hkv * G * D + i] = 0;
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
    // Equal shares of the cost: CTAs, and in a CTA its warps; a warp's is at least
    // kQ4MinPart.
    const int64_t W = base[kQ4Threads];
    const int NC = (int)min((int64_t)a.P, (W / kQ4MinPart + kQ4Warps - 1) / kQ4Warps + (W < kQ4MinPart));
    if (bid >= NC || W == 0) return;
    auto share = [](int64_t n, int i, int parts) { return i * (n / parts) + i * (n % parts) / parts; };
    const int64_t c0 = share(W, bid, NC);
    const int32_t cn = (int32_t)(share(W, bid + 1, NC) - c0);  // this CTA's
    const int nw = max(1, min(kQ4Warps, cn / kQ4MinPart));
    auto warp_begin = [&](int w) { return w * (cn / nw) + w * (cn % nw) / nw; };

    struct Run {
        Q4Seq q;
        int32_t s, g;
        int32_t begin;       // cost before it, from the CTA's start on
        int32_t i0, i1;      // this warp's tiles of it
    };
    if (warp < nw) {
        const int32_t w0 = warp_begin(warp), w1 = warp_begin(warp + 1);
        // a run's tiles from cost x on
        auto tile_from = [&](const Run &r, int32_t x) {
            x -= r.begin;
            return x <= 0 ? 0 : x >= r.q.cost() ? r.q.tiles() : min(r.q.tiles(), q4_tile_at(r.q, x));
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
            r.i0 = 0;
            r.i1 = tile_from(r, w1);
            return true;
        };
        // ---- the run at the part's start ----
        Run run;
        {
            int lo = 0, hi = kQ4Threads;  // the last thread whose sequences start at or before w0, with any cost
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (base[mid] <= c0 + w0) lo = mid; else hi = mid;
            }
            int64_t x = c0 + w0 - base[lo];  // cost from the sequence's start on
            run.s = lo * per;
            run.q = q4_seq(a, run.s);
            while (x >= (int64_t)run.q.cost() * a.Hkv) {
                x -= (int64_t)run.q.cost() * a.Hkv;
                run.q = q4_seq(a, ++run.s);
            }
            run.g = (int32_t)((uint32_t)x / (uint32_t)run.q.cost());
            run.begin = w0 - (int32_t)((uint32_t)x - (uint32_t)run.g * (uint32_t)run.q.cost());
            run.i0 = tile_from(run, w0);
            run.i1 = tile_from(run, w1);
        }
        // (the part may start past this run's last tile; it has one of the next then)
        bool go = run.i0 < run.i1 || next(run);

        // ---- the ring: this warp's 4-bit tiles, piece after piece ----
        uint8_t *ring = smem + (size_t)warp * kQ4Stages * STAGE;
        const uint32_t ring_addr = smem_u32(ring), bar0 = smem_u32(&bars[warp * kQ4Stages]);
        const uint64_t policy = l2_policy_evict_first();
        const int per_block = a.bs / kQ4Tile;
        Run ahead = run;
        bool more = go;          // `ahead` is a run of this part
        int32_t at = run.i0, end = 0;  // its next tile to ask for, and the tile past its last in 4 bits
        int32_t from = 0;        // tile of lane 0's address
        const uint8_t *src = nullptr;  // of tile from + lane
        uint32_t good = 0;       // lanes with one
        uint32_t issue_stage = 0;
        if (more) end = min(ahead.i1, ahead.q.tiles4());
        bool fresh = true;
        auto issue = [&]() {     // the next unit, if there is one
            while (at >= end) {
                if (!more) return;
                more = next(ahead);
                if (!more) return;
                at = 0;
                end = min(ahead.i1, ahead.q.tiles4());
                fresh = true;
            }
            if (fresh || at + U > from + 32) {  // the next 32 tiles' places
                fresh = false;
                from = at;
                const int32_t i = at + lane, b = (int32_t)((uint32_t)i / (uint32_t)per_block);
                const int32_t id = i < end ? a.table4[(int64_t)ahead.s * a.max_blocks4 + b] : -1;
                const bool ok = id >= 0 && (int64_t)id + a.pages_per_block4 <= a.pool_pages;
                if (i < end && !ok) report(a.err, KV_ERR_DEVICE_BOUNDS);
                src = a.pool + (int64_t)id * a.page_bytes + ((int64_t)ahead.g * per_block + (i - b * per_block)) * TILE;
                good = __ballot_sync(0xffffffffu, ok);
            }
            const int off = at - from;
            const uint32_t bar = bar0 + issue_stage * 8;
            if (lane == off) mbar_arrive_expect_tx(bar, __popc((good >> off) & ((1u << U) - 1u)) * TILE);
            __syncwarp();
            if ((uint32_t)(lane - off) < (uint32_t)U && ((good >> lane) & 1u))
                bulk_load(ring_addr + issue_stage * STAGE + (lane - off) * TILE, src, TILE, bar, policy);
            at += U;
            issue_stage = issue_stage + 1 == kQ4Stages ? 0 : issue_stage + 1;
        };
        for (int st = 0; st < kQ4Stages; ++st) issue();

        bool dead = false;
        uint32_t stage = 0, parity = 0;
        for (; go; go = next(run)) {
            const Q4Seq q = run.q;
            const int32_t r = run.s * a.Hkv + run.g;
            const uint16_t *qrow = a.q + (int64_t)r * G * D;
            Q4State<D> st;
            st.begin(qrow, G, a.qk_scale, lane);
            const int32_t end4 = min(run.i1, q.tiles4());
            for (int32_t i = run.i0; i < end4; i += U) {
                wait_phase(bar0 + stage * 8, parity, a.err, dead);
                if (i + U <= end4)
                    st.template unit4<true>(ring + stage * STAGE, U, lane);
                else
                    st.template unit4<false>(ring + stage * STAGE, end4 - i, lane);
                if (++stage == kQ4Stages) {
                    stage = 0;
                    parity ^= 1u;
                }
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
                st.tile16(k, v, qrow, G, a.qk_scale, lane);
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
            // ---- end of a piece: t0, t1 are the CTA's tiles of the run ----
            const int32_t t0 = tile_from(run, 0), t1 = tile_from(run, cn);
            const bool first = t0 == 0, last = t1 == q.tiles(), split = !(first && last);
            if (run.i0 == t0 && run.i1 == t1) {
                st.store(a.out + (int64_t)r * G * D, a.ws_part + ((int64_t)r + bid) * MF, split, G, lane);
                if (lane == 0) {
                    if (first) a.ws_run[r].x = bid;
                    if (last) a.ws_run[r].y = split ? bid + 1 : bid;
                }
            } else if (run.i0 != t0) {  // goes on from an earlier warp, which merges it
                st.store(nullptr, recs + warp * MF, true, G, lane);
            } else {  // goes on in the next warp: the last piece here, so the ring is free
                st.store(nullptr, reinterpret_cast<float *>(ring), true, G, lane);
                const int32_t last_tile = run.begin + min(t1 - 1, q.tiles4()) * kQ4Cost + max(0, t1 - 1 - q.tiles4()) * kBf16Cost;
                int e = warp;
                while (e + 1 < nw && warp_begin(e + 1) <= last_tile) ++e;
                if (lane == 0) chains[warp] = make_int4(r, e - warp, (first ? 1 : 0) | (last ? 2 : 0), split ? 1 : 0);
            }
        }
    }
    __syncthreads();
    // Chain w is the run whose share of this CTA starts in warp w and goes on
    // through warp w + chains[w].y: its states, merged in warp order, one thread per
    // four columns, give the output (a run inside this CTA) or one record.
    const int cols = G * D / 4;
    for (int i = tid; i < kQ4Warps * cols; i += kQ4Threads) {
        const int w = i / cols, c = i - w * cols, h = c * 4 / D;
        const int4 ch = chains[w];
        if (ch.x < 0) continue;
        float mv[kQ4Warps], lv[kQ4Warps];
        float4 ov[kQ4Warps];
#pragma unroll
        for (int k = 0; k < kQ4Warps; ++k) {
            mv[k] = -INFINITY;
            if (k <= ch.y) {
                const float *rec = k == 0 ? reinterpret_cast<const float *>(smem + (size_t)w * kQ4Stages * STAGE)
                                          : recs + (w + k) * MF;
                mv[k] = rec[G * D + h];
                lv[k] = rec[G * D + G + h];
                ov[k] = *reinterpret_cast<const float4 *>(rec + c * 4);
            }
        }
        float M, L;
        float4 O;
        merge_group(M, L, O, mv, lv, ov);
        if (ch.w == 0) {
            store_column(a.out + (int64_t)ch.x * (G * D) + c * 4, O, L);
        } else {
            float *slot = a.ws_part + ((int64_t)ch.x + bid) * MF;
            *reinterpret_cast<float4 *>(slot + c * 4) = O;
            if (c * 4 % D == 0) {
                slot[G * D + h] = M;
                slot[G * D + G + h] = L;
            }
        }
        if (c == 0 && (ch.z & 1)) a.ws_run[ch.x].x = bid;
        if (c == 0 && (ch.z & 2)) a.ws_run[ch.x].y = bid + ch.w;
    }
}

}  // namespace kvp

// one entry per head dim: the CTAs that are resident at once (launch false), or
// both kernels
int kvp_q4_attn_d64(int G, const kvp::Q4Args *a, int sm_count, cudaStream_t st, bool launch, int *P_out);
int kvp_q4_attn_d128(int G, const kvp::Q4Args *a, int sm_count, cudaStream_t st, bool launch, int *P_out);
