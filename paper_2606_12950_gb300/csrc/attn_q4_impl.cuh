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
// Weights p = 2^(score - M) are held under 2^-32 (M moves only when that would be
// passed, by 2^8 at once): the fp32 sums of p, p z and p v stay in range for any
// bf16 z and v.  A weight meets V's scale before it is rounded to fp16, and a power
// of two of its head and group, the gain, before that: the largest p s gain so far
// lies in [2^7, 2^16), and the gain moves only when 2^15 is passed.  So a group keeps
// its digits whatever the other's scales are, and whatever those of tokens of little
// weight.  Gains leave the sums where the tiles in 4 bits end; records (M, l, o) merge
// as those of the bf16 kernel do.  (One range for both groups, V's largest scale in M:
// 4 % faster, 10 % with short contexts, but a V group of scales 2^24 under the other's
// was lost, as was one beside a NaN.)
//
// Work split: a tile is 16 tokens of a (sequence, KV head) run; it costs 9 where
// it is in 4 bits and 32 in bf16 (its bytes), a run's first one kRunCost more (what
// starts and ends a run).  The batch's tiles, in order, are cut into parts of equal
// cost, one a CTA, and those into equal ones, one a warp.  A run inside a CTA leaves
// its output, others a record a CTA for the combine (the warps' states merged in
// shared memory).  Each warp streams its tiles through its own ring of two stages, a
// bulk copy a tile (or K or V, where they are in bf16).
//
// Bound by HBM in the long run, by its start and end in short ones.  Steady state (the
// slope from 240000 to 480000 tokens, 32 q / 8 KV heads of 128): 6.68 TB/s read, 0.99
// of the measured copy; 16 single heads of 64 6.35.  Around it a call spends about 13
// us: the lengths' round trip and the split 3, the table's and the first tiles' 3, warps
// that end apart 2, merges and the combine 4.  Calls (us; floor at 6.78 TB/s):
//   250 sequences, 40 q / 8 KV heads of 128, 700 MB    117.6 (103)
//   64 sequences, 32 / 8 of 128, 242 MB                 48.4 (35.7)
//   one of 100000 tokens, 32 / 8 of 128, 115 MB         30.2 (17.0)
//   40 sequences, 16 heads of 64, 140 MB                34.6 (20.7)
//   400 of 100 to 500 tokens, 32 / 8 of 128, 174 MB     45.3 (25.7)
//   1000 of 20 to 200 tokens, 32 / 8 of 128, 217 MB     60.2 (32.0)
//   8 of 600 to 3500 tokens, 32 / 8 of 128, 20 MB      14.4 (2.9)
// A tile of 128 columns takes 265 issue slots of the 396 that an SM quarter has while
// HBM brings it; half of them are masks and shifts of codes, which is why the masked
// words must be operands as they are.  (With a subtraction per pair, or codes as bf16,
// they would be twice as many.)  Short runs add what begins and ends them; there the
// kernel waits for instructions more than for data, and its size counts.
//
// Why this shape (64 / 250 sequences, us, with the rest of the code as it then was): a CTA
// of 16 warps an SM, not two of 8, of which the first ran 25% ahead and left the other
// half the SM: 54.0 / 123.9 to 48.2 / 117.4.  CTAs' records for the combine, not warps':
// 60.6 / 145.5 to 54.0 / 136.7.  bf16 tiles through the ring, not into registers: 54.0 /
// 136.7 to 51.0 / 123.9.  Runs' fields in shared memory, not registers, spilled in the
// loops (1000 short / 400): 92.4 / 58.3 to 66.4 / 48.8; one loop that asks for tiles and
// finds each run once: 64.8 / 48.2 to 55.5 / 41.2.
#pragma once

#include <cuda_fp16.h>

#include "attn_impl.cuh"
#include "q4_format.h"

namespace kvp {

constexpr int kQ4Warps = 16;
constexpr int kQ4Threads = kQ4Warps * 32;
constexpr int kQ4Stages = 2;
template <int D>
constexpr int kQ4Unit = D == 64 ? 4 : 2;  // tiles of a stage: 4608 bytes either way
constexpr int kQ4Rebalance = 32;          // tiles (see Q4State::rebalance)
constexpr float kWeightTop = -32.f;       // weights are below 2 to this,
constexpr float kWeightRest = 40.f;       // and the largest 2^-40 where M has moved
constexpr int kMostGain = 120;            // a scale of 2^-72 and a weight of 2^-40 make 2^8
constexpr int kQ4Cost = 9, kBf16Cost = 32;
template <int D>
constexpr int kRunCost = D == 64 ? 56 : 18;
constexpr int kQ4Spread = 4;              // warps of a CTA with parts, where there are few parts
// A part costs no less than any tile, so that each has one: this much before rounding.
template <int D>
constexpr int kQ4MinPart = kRunCost<D> + kBf16Cost + kQ4Warps;

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
    int2 *ws_run;            // as in AttnArgs (kRecCtas, or kRecCtasByPart)
    int64_t page_bytes, pool_pages;
    int32_t pages_per_block, pages_per_block4;
    int32_t max_blocks, max_blocks4;
    int32_t S, Hkv, G, bs;
    int32_t P;               // CTAs
    bool by_part;            // ws_run is per part
    float qk_scale;          // scale * log2(e)
};

__host__ __device__ constexpr int q4_record_floats(int D, int G) { return (G * D + 2 * G + 3) / 4 * 4; }

// shared memory of a CTA: per warp its stages and a record; barriers, costs
template <int D>
inline size_t q4_smem_bytes(int G)
{
    return 128 + (size_t)kQ4Warps * (kQ4Stages * (kQ4Unit<D> * kQ4TileBytes<D> + 8) + q4_record_floats(D, G) * 4 + 16) +
           (kQ4Threads + kQ4Warps) * sizeof(int64_t);
}

// A sequence's lengths, clamped to what the tables can hold.
template <int D>
struct Q4Seq {
    int32_t n, p;    // tokens; of them in 4 bits
    bool append;     // a new row can be appended
    __device__ int32_t tiles4() const { return p >> 4; }
    __device__ int32_t tiles() const { return (p >> 4) + ((n - p + 15) >> 4); }
    // of a run, and before its tile i
    __device__ int32_t cost() const { return n > 0 ? cost_to(tiles()) : 0; }
    __device__ int32_t cost_to(int32_t i) const
    {
        return i > 0 ? kRunCost<D> + kQ4Cost * min(i, p >> 4) + kBf16Cost * max(0, i - (p >> 4)) : 0;
    }
};

template <int D>
__device__ __forceinline__ Q4Seq<D> q4_seq(const Q4Args &a, int s)
{
    const int32_t n = a.lens[s], p = a.packed[s];
    const int32_t cap = a.max_blocks * a.bs, cap4 = a.max_blocks4 * a.bs;
    Q4Seq<D> q;
    q.n = min(max(n, 0), cap);
    q.p = min(min(max(p, 0), q.n), cap4) & ~15;
    q.append = n == q.n && n > q.p;
    return q;
}

// the first tile of a run with no less than cost x before it
template <int D>
__device__ __forceinline__ int32_t q4_tile_at(const Q4Seq<D> &q, int32_t x)
{
    if (x <= 0) return 0;
    if (x >= q.cost()) return q.tiles();
    x -= kRunCost<D>;
    const int32_t c4 = kQ4Cost * q.tiles4();
    const int32_t i = x <= c4 ? (int32_t)((uint32_t)(max(x, 0) + kQ4Cost - 1) / (uint32_t)kQ4Cost)
                              : q.tiles4() + (x - c4 + kBf16Cost - 1) / kBf16Cost;
    return max(1, i);
}

__device__ __forceinline__ void prefetch_l2(const void *p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// A run as a warp works on it, in units of its CTA's costs.
template <int D>
struct Q4Run {
    Q4Seq<D> q;
    int32_t s, g;
    int32_t begin;       // cost before it, from the CTA's start on
    int32_t i0, i1;      // this warp's tiles of it
    int32_t stop;        // the cost at the end of the warp's part
};

// Runs wait in shared memory while tiles are worked on (every lane stores and loads the
// same): the registers are needed there, and what is spilled is spilled in the loops.
template <int D>
__device__ __forceinline__ void put_run(uint32_t at, const Q4Run<D> &r)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(r.q.n), "r"(r.q.append ? ~r.q.p : r.q.p),
                 "r"(r.s), "r"(r.g));
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + 16), "r"(r.begin), "r"(r.i0), "r"(r.i1),
                 "r"(r.stop));
}
template <int D>
__device__ __forceinline__ Q4Run<D> get_run(uint32_t at)
{
    Q4Run<D> r;
    int32_t p;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.q.n), "=r"(p), "=r"(r.s), "=r"(r.g) : "r"(at));
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r.begin), "=r"(r.i0), "=r"(r.i1), "=r"(r.stop)
                 : "r"(at + 16));
    r.q.append = p < 0;
    r.q.p = p < 0 ? ~p : p;
    return r;
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

// 2^e, e from -126 to 127, and 0 below
__device__ __forceinline__ float pow2_of(int e) { return __uint_as_float((uint32_t)max(e + 127, 0) << 23); }
// the exponent of a power of two, or of the one below x
__device__ __forceinline__ int exponent_of(float x) { return (int)(__float_as_uint(x) >> 23) - 127; }

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
    float factor[2];        // of the scores, to base-2 exponents; |scale| goes here, its sign to q
    float m[2], l[2];
    float z[NG][2];         // sums of p z over this lane's tokens
    float gain[NG][2];      // powers of two (see the head of this file)
    // sums of p s c: row pairs (e, e + 1), odd columns times 16, all times 2^-24 gain
    // (from release on without those factors, and of p v too)
    float acc[NM][4];

    // qrow: q rows of the run's G heads
    __device__ __forceinline__ void begin(const uint16_t *qrow, int G, float qk_scale, int lane)
    {
        const int tig = lane & 3;
        uint4 w[NW];
        load_q(w, qrow, G, lane);
        float mx = 0.f;
#pragma unroll
        for (int j = 0; j < NW; ++j) {
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
            gain[c][0] = gain[c][1] = pow2_of(kMostGain);
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

    // M's new place where a score passes it: y0, y1 the lane's largest scores.  Their
    // weights are powers of two then, and lose nothing where weights are rounded.
    // down[h]: what the sums acc are the caller's to scale by.
    __device__ __forceinline__ bool raise(float y0, float y1, float (&down)[2])
    {
        if (!__any_sync(0xffffffffu, y0 > m[0] + kWeightTop || y1 > m[1] + kWeightTop)) return false;
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) {
            y0 = fmaxf(y0, __shfl_xor_sync(0xffffffffu, y0, off));
            y1 = fmaxf(y1, __shfl_xor_sync(0xffffffffu, y1, off));
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float y = h ? y1 : y0, to = y > m[h] + kWeightTop ? y + kWeightRest : m[h];
            down[h] = fast_exp2(m[h] - to);
            m[h] = to;
            l[h] *= down[h];
#pragma unroll
            for (int c = 0; c < NG; ++c) z[c][h] *= down[h];
        }
        return true;
    }

    // The gains after M moved, or where the unit's weights p, with V's parameters vp,
    // pass 2^15: a gain takes the move's power of two up, so that what was the largest
    // p s gain stays it, and falls where something passes that, to 2^7 of it.  (A NaN is
    // no maximum: it is on its way to its own columns.)
    template <int U>
    __device__ __forceinline__ void regain(const float (&p)[U][4], const uint32_t (&vp)[U][2][NG], const float (&down)[2])
    {
        constexpr uint32_t EXP = 0x7f800000u;
#pragma unroll
        for (int c = 0; c < NG; ++c) {
            uint32_t top = 0;  // of the heads' p s, as bf16 pairs
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float sa = bf_lo(vp[u][0][c]), sb = bf_lo(vp[u][1][c]);
                const float t0 = fmaxf(0.f, fmaxf(p[u][0] * sa, p[u][2] * sb)), t1 = fmaxf(0.f, fmaxf(p[u][1] * sa, p[u][3] * sb));
                top = __vmaxu2(top, __byte_perm(__float_as_uint(t0), __float_as_uint(t1), 0x7632));
            }
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, off));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float t = h ? bf_hi(top) : bf_lo(top), old = gain[c][h];
                // (1 / x of a power of two: its exponent, 127 too high, from 254)
                float g = fminf(old * __uint_as_float(2 * (127u << 23) - (__float_as_uint(down[h]) & EXP)), pow2_of(kMostGain));
                if (t * g >= 0x1p15f) g = __uint_as_float(((2 * 127u + 7u) << 23) - (__float_as_uint(t) & EXP));
                const float r = g * down[h] * __uint_as_float(2 * (127u << 23) - __float_as_uint(old));
                gain[c][h] = g;
#pragma unroll
                for (int i = 4 * c; i < 4 * c + 4; ++i) {
                    acc[i][h] *= r;
                    acc[i][2 + h] *= r;
                }
            }
        }
    }

    // The first `count` (or more) of a stage's U tiles in 4 bits.  In place of those that
    // are missing the last one is read once more, without weight: one tile by itself
    // takes nearly as long as two.
    template <int U>
    __device__ __forceinline__ void tiles4(const uint8_t *stage, int count, int lane)
    {
        constexpr int TILE = kQ4TileBytes<D>;
        const int gid = lane >> 2, tig = lane & 3;
        float x[U][4];
        uint32_t vp[U][2][NG];
        float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            {
                const uint8_t *tile = stage + min(u, count - 1) * TILE;
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
                }
                x0 = fmaxf(x0, fmaxf(x[u][0], x[u][2]));
                x1 = fmaxf(x1, fmaxf(x[u][1], x[u][3]));
            }
        }
        float down[2] = {1.f, 1.f};
        bool moved = raise(x0 * factor[0], x1 * factor[1], down);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool in = u == 0 || u < count;
            const float m0 = in ? -m[0] : -INFINITY, m1 = in ? -m[1] : -INFINITY;
            x[u][0] = fast_exp2(fmaf(x[u][0], factor[0], m0));
            x[u][1] = fast_exp2(fmaf(x[u][1], factor[1], m1));
            x[u][2] = fast_exp2(fmaf(x[u][2], factor[0], m0));
            x[u][3] = fast_exp2(fmaf(x[u][3], factor[1], m1));
            l[0] += x[u][0] + x[u][2];
            l[1] += x[u][1] + x[u][3];
        }
        uint32_t b[U][NG][2];
        auto weights = [&]() {  // rounded; the largest, as fp16 numbers
            uint32_t top = 0;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int c = 0; c < NG; ++c) {
                    const float2 g = make_float2(gain[c][0], gain[c][1]);
                    const float sa = bf_lo(vp[u][0][c]), sb = bf_lo(vp[u][1][c]);
                    const float2 pa = __fmul2_rn(make_float2(x[u][0], x[u][1]), g);
                    const float2 pb = __fmul2_rn(make_float2(x[u][2], x[u][3]), g);
                    b[u][c][0] = f16_pair(pa.x * sa, pa.y * sa);
                    b[u][c][1] = f16_pair(pb.x * sb, pb.y * sb);
                    top = __vmaxu2(top, __vmaxu2(b[u][c][0], b[u][c][1]));
                }
            return top;
        };
        // (2^15 and what is above, infinity and NaN too, carries into the sign)
        if (!moved) moved = __any_sync(0xffffffffu, ((weights() + 0x08000800u) & 0x80008000u) != 0);
        if (moved) {
            regain<U>(x, vp, down);
            weights();
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint8_t *tile = stage + min(u, count - 1) * TILE;
#pragma unroll
            for (int c = 0; c < NG; ++c) {
                const float za = bf_hi(vp[u][0][c]), zb = bf_hi(vp[u][1][c]);
                z[c][0] = fmaf(x[u][0], za, fmaf(x[u][2], zb, z[c][0]));
                z[c][1] = fmaf(x[u][1], za, fmaf(x[u][3], zb, z[c][1]));
                const uint32_t b0 = movmatrix_trans(b[u][c][0]), b1 = movmatrix_trans(b[u][c][1]);
                const uint4 v = *reinterpret_cast<const uint4 *>(tile + 8 * D + 512 * c + 16 * lane);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t h = w[i] >> 8;
                    mma_f16_16816(acc[4 * c + i], w[i] & 0x000f000fu, w[i] & 0x00f000f0u, h & 0x000f000fu, h & 0x00f000f0u,
                                  b0, b1);
                }
            }
        }
    }

    // The tensor cores' sums lose what falls under an fp32 digit, always toward zero,
    // and codes are never negative: sums of thousands of tiles drift (16384 tokens of flat
    // weights in one warp: the output 1.3e-2 off, 65536 tokens 3.6e-2), and z undoes most of
    // such a sum.  So now and then the sums' mean over a group's columns moves to the
    // sum of p z, exactly but for fp32 rounding: what stays is as small as the output.
    __device__ __forceinline__ void rebalance()
    {
#pragma unroll
        for (int c = 0; c < NG; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float x = 0.f;
#pragma unroll
                for (int i = 4 * c; i < 4 * c + 4; ++i) x += fmaf(acc[i][2 + h], 0.0625f, acc[i][h]);
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
                x *= 1.f / 64.f;
#pragma unroll
                for (int i = 4 * c; i < 4 * c + 4; ++i) {
                    acc[i][h] -= x;
                    acc[i][2 + h] = fmaf(x, -16.f, acc[i][2 + h]);
                }
                // (an eighth each: eight lanes hold parts of the sum)
                z[c][h] = fmaf(x, pow2_of(21 - exponent_of(gain[c][h])), z[c][h]);
            }
    }

    // The tiles in 4 bits are done: the sums themselves.  (bf16 values take no factor of
    // 16: it would carry an odd column's from 2^124 on past their range.)
    __device__ __forceinline__ void release()
    {
#pragma unroll
        for (int c = 0; c < NG; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int e = exponent_of(gain[c][h]);
                const float f = pow2_of(24 - e), odd = pow2_of(20 - e);
#pragma unroll
                for (int i = 4 * c; i < 4 * c + 4; ++i) {
                    acc[i][h] *= f;
                    acc[i][2 + h] *= odd;
                }
            }
    }

    // A tile of bf16 rows, of which the first `valid` are tokens: its K's scores (qw
    // as load_q gives it), then its V.
    static __device__ __forceinline__ void load_q(uint4 (&qw)[NW], const uint16_t *qrow, int G, int lane)
    {
        const int gid = lane >> 2, tig = lane & 3;
#pragma unroll
        for (int j = 0; j < NW; ++j)
            qw[j] = gid < G ? *reinterpret_cast<const uint4 *>(qrow + gid * D + 64 * (j >> 1) + 32 * (j & 1) + 8 * tig)
                            : make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ void scores16(float (&y)[4], const uint16_t *rows, int valid, const uint4 (&qw)[NW],
                                             float qk_scale, int lane)
    {
        const int gid = lane >> 2, tig = lane & 3;
        const uint16_t *k0 = rows + gid * D, *k1 = k0 + 8 * D;
        float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NW; ++j) {
            const int at = 64 * (j >> 1) + 32 * (j & 1) + 8 * tig;
            const uint4 a = *reinterpret_cast<const uint4 *>(k0 + at), b = *reinterpret_cast<const uint4 *>(k1 + at);
            mma_bf16_16816(x, a.x, b.x, a.y, b.y, qw[j].x, qw[j].y);
            mma_bf16_16816(x, a.z, b.z, a.w, b.w, qw[j].z, qw[j].w);
        }
        const float no = -INFINITY;
        y[0] = gid < valid ? x[0] * qk_scale : no;
        y[1] = gid < valid ? x[1] * qk_scale : no;
        y[2] = gid + 8 < valid ? x[2] * qk_scale : no;
        y[3] = gid + 8 < valid ? x[3] * qk_scale : no;
        float down[2];
        if (raise(fmaxf(y[0], y[2]), fmaxf(y[1], y[3]), down)) {
            const float f0 = down[0], f1 = down[1];
#pragma unroll
            for (int i = 0; i < NM; ++i) {
                acc[i][0] *= f0;
                acc[i][1] *= f1;
                acc[i][2] *= f0;
                acc[i][3] *= f1;
            }
        }
    }
    __device__ __forceinline__ void values16(const float (&y)[4], const uint16_t *rows, int valid, int lane)
    {
        const int gid = lane >> 2, tig = lane & 3;
        uint4 vw[4][NG];
#pragma unroll
        for (int r = 0; r < 4; ++r) {  // (what lies past the context may be anything)
            const int t = 2 * tig + (r & 1) + 4 * (r & 2);
            const uint16_t *v = rows + t * D;
#pragma unroll
            for (int c = 0; c < NG; ++c)
                vw[r][c] = t < valid ? *reinterpret_cast<const uint4 *>(v + 64 * c + 8 * gid) : make_uint4(0u, 0u, 0u, 0u);
        }
        const float p0 = fast_exp2(y[0] - m[0]), p1 = fast_exp2(y[1] - m[1]);
        const float p2 = fast_exp2(y[2] - m[0]), p3 = fast_exp2(y[3] - m[1]);
        l[0] += p0 + p2;
        l[1] += p1 + p3;
        const uint32_t b0 = movmatrix_trans(bf16_pair(p0, p1)), b1 = movmatrix_trans(bf16_pair(p2, p3));
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
                    a[2 * r + 1] = __byte_perm(w0, w1, 0x7632);
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
                    o[2 * i] = acc[4 * c + i][h] + z[c][h];
                    o[2 * i + 1] = acc[4 * c + i][2 + h] + z[c][h];
                }
                const int at = head * D + 64 * c + 8 * gid;
                if (split) {
                    *reinterpret_cast<float4 *>(slot + at) = make_float4(o[0], o[1], o[2], o[3]);
                    *reinterpret_cast<float4 *>(slot + at + 4) = make_float4(o[4], o[5], o[6], o[7]);
                } else {
                    const float il = 1.f / l[h];
                    uint4 w;
                    w.x = bf16_pair(o[0] * il, o[1] * il);
                    w.y = bf16_pair(o[2] * il, o[3] * il);
                    w.z = bf16_pair(o[4] * il, o[5] * il);
                    w.w = bf16_pair(o[6] * il, o[7] * il);
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
__global__ void __launch_bounds__(kQ4Threads, 1) q4_attn_kernel(const __grid_constant__ Q4Args a)
{
    constexpr int TILE = kQ4TileBytes<D>, U = kQ4Unit<D>, STAGE = U * TILE;
    constexpr int TILE16 = kQ4Tile * 2 * D;  // K or V of a tile in bf16
    static_assert(TILE16 <= STAGE, "a unit is a stage");
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((128u - (smem_u32(smem_raw) & 127u)) & 127u);
    const int G = a.G, MF = q4_record_floats(D, G);
    float *recs = reinterpret_cast<float *>(smem + (size_t)kQ4Warps * kQ4Stages * STAGE);  // [warps][MF]
    int4 *chains = reinterpret_cast<int4 *>(recs + kQ4Warps * MF);                          // [warps]
    uint64_t *bars = reinterpret_cast<uint64_t *>(chains + kQ4Warps);
    // costs before a thread's sequences, from its warp's on, and of a warp's
    int64_t *base = reinterpret_cast<int64_t *>(bars + kQ4Warps * kQ4Stages), *tops = base + kQ4Threads;
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const int bid = blockIdx.x, S = a.S;
    if (tid == 0) {
        for (int i = 0; i < kQ4Warps * kQ4Stages; ++i) mbar_init(smem_u32(&bars[i]), 1);
        fence_mbar_init();
    }
    __shared__ int2 part;  // by_part: this CTA's entry of ws_run
    if (lane == 0) chains[warp].x = -1;
    if (tid == 0) part = make_int2(-1, -1);
    grid_launch_dependents();
    grid_dependency_wait();

    // ---- the cost before each thread's sequences ----
    const int per = (S + kQ4Threads - 1) / kQ4Threads;
    {
        const int lo = min(S, tid * per), hi = min(S, lo + per);
        int64_t sum = 0;
        for (int s = lo; s < hi; ++s) {
            const Q4Seq<D> q = q4_seq<D>(a, s);
            sum += (int64_t)q.cost() * a.Hkv;
            if (s % a.P == bid) {
                const int32_t n = a.lens[s], p = a.packed[s];
                if (n != q.n || p != q.p || (a.k_new && n > 0 && !q.append)) report(a.err, KV_ERR_DEVICE_BOUNDS);
                if (q.n == 0) {  // no softmax: zeros
                    uint4 *row = reinterpret_cast<uint4 *>(a.out + (int64_t)s * a.Hkv * G * D);
                    for (int i = 0; i < a.Hkv * G * (D / 8); ++i) row[i] = make_uint4(0u, 0u, 0u, 0u);
                    for (int g = 0; g < a.Hkv && !a.by_part; ++g) a.ws_run[(int64_t)s * a.Hkv + g] = make_int2(0, 0);
                }
            }
        }
        int64_t incl = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int64_t v = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += v;
        }
        base[tid] = incl - sum;
        if (lane == 31) tops[warp] = incl;
        __syncthreads();
    }
    int64_t upto = lane < kQ4Warps ? tops[lane] : 0;  // the cost up to the end of warp `lane`'s sequences
#pragma unroll
    for (int off = 1; off < kQ4Warps; off <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, upto, off);
        if (lane >= off) upto += v;
    }
    // Equal shares of the cost, rounded up, but for the last: CTAs, and in a CTA its warps.
    // The last one's roundings leave it a tile's cost: a warp's 15 of kQ4MinPart, a CTA's
    // 151 at the most, and then it has four times as much.
    // (Divisions take 0.1 us each in this chain, those of 64 bits 0.5.)
    const int64_t W = __shfl_sync(0xffffffffu, upto, kQ4Warps - 1);
    const uint32_t least = (uint32_t)min(W, (int64_t)UINT32_MAX);
    const int NC = (int)min((uint32_t)a.P, (least / kQ4MinPart<D> + kQ4Spread - 1) / kQ4Spread + (least < kQ4MinPart<D>));
    if (bid >= NC || W == 0) {
        if (a.by_part && tid == 0) a.ws_run[bid] = make_int2(-1, -1);
        return;
    }
    const int64_t wq = (W >> 32) == 0 ? (int64_t)((uint32_t)(W - 1) / (uint32_t)NC + 1u) : (W - 1) / NC + 1;
    const int64_t c0 = bid * wq;
    const int32_t cn = (int32_t)min(wq, W - c0);  // this CTA's
    const int nw = max(1, min(kQ4Warps, cn / kQ4MinPart<D>));
    const int32_t nq = (int32_t)((uint32_t)(cn - 1) / (uint32_t)nw + 1u);
    auto warp_begin = [&](int w) { return min(w * nq, cn); };

    if (warp < nw) {
        const int32_t w0 = warp_begin(warp);
        // a run's tiles from cost x on
        auto tile_from = [&](const Q4Run<D> &r, int32_t x) { return q4_tile_at(r.q, x - r.begin); };
        // the run after r that has tiles in this part; false if there is none
        auto next = [&](Q4Run<D> &r) {
            r.begin += r.q.cost();
            if (++r.g == a.Hkv) {
                r.g = 0;
                do {
                    if (r.begin >= r.stop || ++r.s >= S) return false;
                    r.q = q4_seq<D>(a, r.s);
                } while (r.q.n == 0);
            }
            if (r.begin >= r.stop) return false;
            r.i0 = 0;
            r.i1 = tile_from(r, r.stop);
            return true;
        };
        // The runs from the one that is worked on to the one whose tiles are asked for
        // (three at most: the units of the ring are of two).
        __shared__ alignas(16) int32_t boxes[kQ4Warps][4][8];
        static_assert(kQ4Stages + 1 <= 4, "boxes");
        auto box = [&](int k) { return smem_u32(boxes[warp][k & 3]); };
        int asked = 0;                         // the latter's box
        int32_t at, ahead_i1, ahead_t4, head;  // its next tile, end, tiles in 4 bits, KV head
        // ---- the run at the part's start ----
        bool go;
        {
            Q4Run<D> run;
            // the last thread whose sequences start at or before w0 (with any cost)
            int64_t x = c0 + w0;
            const int k = __popc(__ballot_sync(0xffffffffu, lane < kQ4Warps && upto <= x));  // warps before
            const int64_t before = __shfl_sync(0xffffffffu, upto, max(k - 1, 0));
            x -= k > 0 ? before : 0;
            const int t = 31 - __clz((int)__ballot_sync(0xffffffffu, base[k * 32 + lane] <= x));
            x -= base[k * 32 + t];  // cost from the sequence's start on
            run.s = (k * 32 + t) * per;
            run.q = q4_seq<D>(a, run.s);
            while (x >= (int64_t)run.q.cost() * a.Hkv) {
                x -= (int64_t)run.q.cost() * a.Hkv;
                run.q = q4_seq<D>(a, ++run.s);
            }
            run.g = (int32_t)((uint32_t)x / (uint32_t)run.q.cost());
            run.begin = w0 - (int32_t)((uint32_t)x - (uint32_t)run.g * (uint32_t)run.q.cost());
            run.i0 = tile_from(run, w0);
            run.stop = warp_begin(warp + 1);
            run.i1 = tile_from(run, run.stop);
            // (the part may start past this run's last tile; it has one of the next then)
            go = run.i0 < run.i1 || next(run);
            put_run(box(0), run);
            at = run.i0;
            ahead_i1 = run.i1;
            ahead_t4 = run.q.tiles4();
            head = run.g;
        }

        // ---- the ring: units of this warp's tiles, piece after piece.  A unit is up
        // to kQ4Unit tiles in 4 bits, or the K or the V of one in bf16 ----
        uint8_t *ring = smem + (size_t)warp * kQ4Stages * STAGE;
        const uint32_t ring_addr = smem_u32(ring), bar0 = smem_u32(&bars[warp * kQ4Stages]);
        const uint64_t policy = l2_policy_evict_first();
        const int per_block = a.bs / kQ4Tile;
        bool more = go;          // there is a run whose tiles are asked for
        // The places of tiles [from, from + 32), one a lane, for head 0: a sequence's
        // runs share them, so that short ones load them once.
        int32_t from = at - 32;
        const uint8_t *src = nullptr;
        uint32_t good = 0;       // lanes with one
        bool v_next = false;     // a bf16 tile's V is next
        uint32_t issue_stage = 0;
        auto issue = [&]() {     // the next unit, if there is one
            if (!more) return;
            if (at >= ahead_i1) {
                Q4Run<D> ahead = get_run<D>(box(asked));
                const int32_t s = ahead.s;
                more = next(ahead);
                if (!more) return;
                put_run(box(++asked), ahead);
                if (lane < (G * D * 2 + 127) / 128)  // its q is needed next
                    prefetch_l2(a.q + ((int64_t)ahead.s * a.Hkv + ahead.g) * G * D + lane * 64);
                at = 0;
                ahead_i1 = ahead.i1;
                ahead_t4 = ahead.q.tiles4();
                head = ahead.g;
                if (from != 0 || s != ahead.s) from = -32;
            }
            const bool packed = at < ahead_t4;
            const int32_t end = packed ? min(at + U, min(ahead_i1, ahead_t4)) : at + 1;
            if (end > from + 32) {  // the next 32 tiles' places
                from = at;
                const Q4Run<D> ahead = get_run<D>(box(asked));
                const int32_t i = at + lane, b = (int32_t)((uint32_t)i / (uint32_t)per_block), t = i - b * per_block;
                const bool in4 = i < ahead_t4;
                int32_t id = -1;
                if (i < ahead.q.tiles())
                    id = in4 ? a.table4[(int64_t)ahead.s * a.max_blocks4 + b] : a.table[(int64_t)ahead.s * a.max_blocks + b];
                const bool ok = id >= 0 && (int64_t)id + (in4 ? a.pages_per_block4 : a.pages_per_block) <= a.pool_pages;
                if (i < ahead_i1 && !ok) report(a.err, KV_ERR_DEVICE_BOUNDS);
                src = a.pool + (int64_t)id * a.page_bytes + t * (in4 ? TILE : TILE16);
                good = __ballot_sync(0xffffffffu, ok);
            }
            const int off = at - from, n = end - at;
            const uint32_t bar = bar0 + issue_stage * 8;
            const uint32_t bytes = packed ? TILE : TILE16;
            if (lane == off) mbar_arrive_expect_tx(bar, __popc((good >> off) & ((1u << n) - 1u)) * bytes);
            __syncwarp();
            if ((uint32_t)(lane - off) < (uint32_t)n && ((good >> lane) & 1u))
                bulk_load(ring_addr + issue_stage * STAGE + (lane - off) * TILE,
                          src + (int64_t)(((v_next ? a.Hkv : 0) + head) * per_block) * bytes, bytes, bar, policy);
            if (packed || v_next) at = end;
            v_next = !packed && !v_next;
            issue_stage = issue_stage + 1 == kQ4Stages ? 0 : issue_stage + 1;
        };
#pragma unroll 1
        for (int st = 0; st < kQ4Stages; ++st) issue();

        // run r's entry of ws_run: it starts, ends in this CTA
        auto note = [&](int32_t r, bool first, bool last) {
            if (a.by_part) {
                if (first && !last) part.x = r;
                if (last && !first) part.y = r;
                return;
            }
            if (first) a.ws_run[r].x = bid;
            if (last) a.ws_run[r].y = first ? bid : bid + 1;
        };

        bool dead = false;
        uint32_t stage = 0, parity = 0;
        for (int k = 0; go && k <= asked; ++k) {
            Q4State<D> st;
            int32_t i, i0, i1, end4;
            {
                const Q4Run<D> run = get_run<D>(box(k));
                st.begin(a.q + ((int64_t)run.s * a.Hkv + run.g) * G * D, G, a.qk_scale, lane);
                i = i0 = run.i0;
                i1 = run.i1;
                end4 = min(run.i1, run.q.tiles4());
            }
            auto tile_in = [&]() { return ring + stage * STAGE; };
            auto stage_done = [&]() {
                if (++stage == kQ4Stages) {
                    stage = 0;
                    parity ^= 1u;
                }
            };
            auto unit_done = [&](int again) {
                stage_done();
                // the stages are refilled by bulk copies next: after this warp's reads
                fence_proxy_async_smem();
                __syncwarp();
#pragma unroll 1
                for (; again > 0; --again) issue();
            };
            for (; i < end4; i += U) {
                wait_phase(bar0 + stage * 8, parity, a.err, dead);
                if ((i - i0) % kQ4Rebalance == kQ4Rebalance - U) st.rebalance();
                // (a lone tile takes its warp nearly as long as two, but of d = 64's four one
                // is often enough alone; and where there are many short runs the kernel waits
                // for its instructions, so that less code counts)
                if (D == 128 || i + U <= end4)
                    st.template tiles4<U>(tile_in(), end4 - i, lane);
                else
#pragma unroll 1
                    for (int32_t u = i; u < end4; ++u) st.template tiles4<1>(tile_in() + (u - i) * TILE, 1, lane);
                unit_done(1);
            }
            if (i0 < end4) st.release();
            for (i = max(i0, end4); i < i1; ++i) {
                const Q4Run<D> run = get_run<D>(box(k));
                const int32_t r = run.s * a.Hkv + run.g, tok0 = i * kQ4Tile, valid = run.q.n - tok0;
                // The new row, lanes [0, D / 8) its K and the next D / 8 its V: it goes
                // to its tile's copy in shared memory and, once that has landed, to the
                // pool (no other unit holds that row).
                const int32_t fresh = a.k_new && run.q.append && valid <= kQ4Tile ? valid - 1 : -1;
                int32_t place = -1;
                uint4 row = make_uint4(0u, 0u, 0u, 0u), qw[D / 32];
                if (fresh >= 0 && lane < D / 4) {
                    place = a.table[(int64_t)run.s * a.max_blocks + (run.q.n - 1) / a.bs];
                    row = *reinterpret_cast<const uint4 *>((lane < D / 8 ? a.k_new : a.v_new) + (int64_t)r * D +
                                                           lane % (D / 8) * 8);
                }
                Q4State<D>::load_q(qw, a.q + (int64_t)r * G * D, G, lane);
                auto put_row = [&](int kv) {
                    if (fresh < 0) return;
                    if (lane / (D / 8) == kv)
                        *reinterpret_cast<uint4 *>(tile_in() + (fresh * D + lane % (D / 8) * 8) * 2) = row;
                    __syncwarp();
                };
                float y[4];
                wait_phase(bar0 + stage * 8, parity, a.err, dead);
                put_row(0);
                st.scores16(y, reinterpret_cast<const uint16_t *>(tile_in()), valid, qw, a.qk_scale, lane);
                stage_done();
                wait_phase(bar0 + stage * 8, parity, a.err, dead);
                put_row(1);
                st.values16(y, reinterpret_cast<const uint16_t *>(tile_in()), valid, lane);
                if (place >= 0 && (int64_t)place + a.pages_per_block <= a.pool_pages) {
                    const int kv = lane / (D / 8), c = lane % (D / 8);
                    uint16_t *dst = reinterpret_cast<uint16_t *>(a.pool + (int64_t)place * a.page_bytes) +
                                    ((int64_t)(kv * a.Hkv + run.g) * a.bs + (run.q.n - 1) % a.bs) * D;
                    *reinterpret_cast<uint4 *>(dst + c * 8) = row;
                }
                unit_done(2);
            }
            const Q4Run<D> run = get_run<D>(box(k));
            const Q4Seq<D> q = run.q;
            const int32_t r = run.s * a.Hkv + run.g;
            // ---- end of a piece: t0, t1 are the CTA's tiles of the run ----
            const int32_t t0 = tile_from(run, 0), t1 = tile_from(run, cn);
            const bool first = t0 == 0, last = t1 == q.tiles(), split = !(first && last);
            const bool alone = run.i0 == t0 && run.i1 == t1;
            // (a run that goes on in the next warp is the last here: the ring is free)
            if (alone)
                st.store(a.out + (int64_t)r * G * D, a.ws_part + ((int64_t)r + bid) * MF, split, G, lane);
            else
                st.store(nullptr, run.i0 != t0 ? recs + warp * MF : reinterpret_cast<float *>(ring), true, G, lane);
            if (lane == 0 && run.i0 == t0) {  // (one that goes on from an earlier warp is merged there)
                note(r, first, last);
                if (!alone) {
                    const int32_t last_tile = run.begin + q.cost_to(t1 - 1);
                    int e = warp;
                    while (e + 1 < nw && warp_begin(e + 1) <= last_tile) ++e;
                    chains[warp] = make_int4(r, e - warp, split ? 1 : 0, 0);
                }
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
        auto rec = [&](int k) {
            return k == 0 ? reinterpret_cast<const float *>(smem + (size_t)w * kQ4Stages * STAGE) : recs + (w + k) * MF;
        };
        float M = rec(0)[G * D + h], L = 0.f;
        for (int k = 1; k <= ch.y; ++k) M = fmaxf(M, rec(k)[G * D + h]);
        float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = 0; k <= ch.y; ++k) {
            const float *r = rec(k);
            const float e = fast_exp2(r[G * D + h] - M);
            const float4 o = *reinterpret_cast<const float4 *>(r + c * 4);
            L = __fmaf_rn(r[G * D + G + h], e, L);
            O.x = __fmaf_rn(o.x, e, O.x);
            O.y = __fmaf_rn(o.y, e, O.y);
            O.z = __fmaf_rn(o.z, e, O.z);
            O.w = __fmaf_rn(o.w, e, O.w);
        }
        if (ch.z == 0) {
            store_column(a.out + (int64_t)ch.x * (G * D) + c * 4, O, L);
        } else {
            float *slot = a.ws_part + ((int64_t)ch.x + bid) * MF;
            *reinterpret_cast<float4 *>(slot + c * 4) = O;
            if (c * 4 % D == 0) {
                slot[G * D + h] = M;
                slot[G * D + G + h] = L;
            }
        }
    }
    if (a.by_part && tid == 0) a.ws_run[bid] = part;
}

}  // namespace kvp

// one entry per head dim: the CTAs that are resident at once (launch false), or the
// kernel and its combine
int kvp_q4_attn_d64(int G, const kvp::Q4Args *a, int sm_count, cudaStream_t st, bool launch, int *P_out);
int kvp_q4_attn_d128(int G, const kvp::Q4Args *a, int sm_count, cudaStream_t st, bool launch, int *P_out);
