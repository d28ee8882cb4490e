// rotary.cu -- rotary positions with the append: a step's or a prompt chunk's
// q and k rows turned to their positions, k and v written into the paged pool.
//
// A rotary embedding (Su et al., 2021) turns each pair (x, y) of a head's
// rotated columns by the angle pos * f_i:
//     x' = m (x cos - y sin),   y' = m (y cos + x sin)
// with f_i the pair's frequency and m a magnitude (1, or the attention factor
// of a stretched context).  The pairs are columns (i, i + rot/2) (half layout)
// or (2i, 2i + 1) (interleaved); columns past `rot` pass through.
//
// Angles.  pos * f_i in fp32 is off by 4e-3 rad at position 65536.  Here a
// frequency is a 64-bit fixed-point fraction of a turn (kv_rotary_steps), and
// pos * step modulo 2^64 is the exact fraction of a turn, whatever the
// position: two integer multiplies, and sincospif on 31 bits of the result.
//
// Bound by HBM for prompts (each row read and written once) and by latency for
// a decode step.  A token's cos and sin are computed once, into shared memory,
// for all heads.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "pool_internal.h"
#include "ptx.cuh"
#include "stream_order.h"

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotShared = 3;     // CTAs an SM holds of those that tokens share
constexpr int kMaxHeadDim = 512;  // kv_pool_create's limit

struct RotaryArgs {
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
    int64_t page_bytes, n_pages;
    float magnitude;
    int32_t pages_per_block, max_blocks;
    int32_t S, Hq, Hkv, D, bs, rot;
    int32_t items;              // of a row (see rotary_kernel)
    int32_t run, longer;        // tokens of a group; the first `longer` groups have one more
};

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

// Two chunks of the half layout, columns 8c .. of either half (c, s: the cos and
// sin of the pairs, two at a time)
__device__ __forceinline__ void turn_halves(uint4 &a, uint4 &b, const float2 (&c)[4], const float2 (&s)[4])
{
    uint32_t *x = reinterpret_cast<uint32_t *>(&a), *y = reinterpret_cast<uint32_t *>(&b);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float2 u = unpack2(x[e]), v = unpack2(y[e]), ns = make_float2(-s[e].x, -s[e].y);
        const float2 p = __ffma2_rn(u, c[e], __fmul2_rn(v, ns)), q = __ffma2_rn(v, c[e], __fmul2_rn(u, s[e]));
        x[e] = pack2(p.x, p.y);
        y[e] = pack2(q.x, q.y);
    }
}

// a chunk of four adjacent pairs (c, s: the first four pairs' in c[0 .. 1], s[0 .. 1])
__device__ __forceinline__ void turn_adjacent(uint4 &a, const float2 (&c)[4], const float2 (&s)[4])
{
    uint32_t *x = reinterpret_cast<uint32_t *>(&a);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float ce = e & 1 ? c[e / 2].y : c[e / 2].x, se = e & 1 ? s[e / 2].y : s[e / 2].x;
        const float2 u = unpack2(x[e]);
        const float2 p = __ffma2_rn(u, make_float2(ce, ce), __fmul2_rn(make_float2(u.y, u.x), make_float2(-se, se)));
        x[e] = pack2(p.x, p.y);
    }
}

// A token's threads are a GROUP of a CTA's.  Its Hq + 2 Hkv rows (q, k, v) are
// cut alike into items: a pair of chunks that turn together (half layout), a
// chunk that turns (adjacent pairs) or one that passes through; a thread keeps
// its item and goes from row to row.  The rows' addresses need the token alone,
// so each thread loads its first kRotBatch rows before the position, the angles
// and the slot, four dependent loads away, are known.
//
// Tokens of many items have a CTA of their own, the whole of it their group:
// 16000 tokens of 40 q and 8 KV heads, half of each head turned (460 MB): 98.7 us
// with the loads after the position, 81.0 with them before, 74.8 with an item a
// thread (issue slots had been 79% taken; 6.15 TB/s).
//
// Tokens whose items are fewer than a smaller group's batches, where there are
// enough of them to fill the GPU, share CTAs that stay: a group of 128 to 8
// threads takes a run of adjacent tokens, looks its sequence up once, and has the
// next token's rows on their way after the last's are stored.  A CTA each / so:
// 32000 tokens of 16 and 4 heads of 128 184 us / 65.7; 16000 of 32 and 8 of 128
// 110 / 65.8 (5.97 TB/s); 1600 of 16 and 4 of 64 11.0 / 6.5; 21500 of 2 and 1
// heads of 64 114 / 7.8 (13.3 with no groups below a warp).
// Batches and CTAs an SM holds are the most that the registers allow; runs for
// the large tokens too measured 84 us where a CTA each measured 73.
//
// Pointers are not __restrict__: the kernel may be resident while the grid
// before it still writes what it reads, and a const __restrict__ pointer may be
// read through the non-coherent path, which the wait below does not order.
template <bool INTERLEAVED, int GROUP>
constexpr int kRotBatch = GROUP == kRotThreads ? 4 : INTERLEAVED ? 6 : 3;
template <bool INTERLEAVED, int GROUP>
constexpr int kRotResident = GROUP == kRotThreads && INTERLEAVED ? 5 : kRotShared;

template <bool INTERLEAVED, int GROUP>
__global__ void __launch_bounds__(kRotThreads, kRotResident<INTERLEAVED, GROUP>) rotary_kernel(const __grid_constant__ RotaryArgs a)
{
    constexpr int PER = kRotThreads / GROUP, BATCH = kRotBatch<INTERLEAVED, GROUP>;
    constexpr int PAIRS = GROUP < 32 ? 8 * GROUP : kMaxHeadDim / 2;  // (no more, with an item of a row a thread)
    // times the magnitude; of a group's token, and of the one before it
    __shared__ __align__(16) float cosines[2][PER][PAIRS], sines[2][PER][PAIRS];
    const int lane = threadIdx.x & 31, tid = threadIdx.x & (GROUP - 1), sub = threadIdx.x / GROUP;
    const int group = blockIdx.x * PER + sub;
    const int t0 = GROUP == kRotThreads ? blockIdx.x : group * a.run + min(group, a.longer);
    const int t_end = GROUP == kRotThreads ? t0 + 1 : t0 + a.run + (group < a.longer);
    // (a warp's groups take turns together)
    const int turns_end = GROUP < 32 ? t0 + a.run + (a.longer > 0) : t_end;
    const int turned = INTERLEAVED ? a.rot / 8 : a.rot / 16;
    const int items = a.items;  // of a row: those that turn, then the others
    const int step = GROUP / items;  // rows at a time
    const int item = tid % items, r0 = tid / items;
    const bool turns = item < turned, pair = !INTERLEAVED && turns;
    const int at = turns ? item : item + a.rot / 8 - turned;  // the item's (first) chunk
    const int q_rows = a.q ? a.Hq : 0, all_rows = r0 < step ? q_rows + (a.k ? 2 * a.Hkv : 0) : 0;
    int t = t0;
    auto load = [&](int r, uint4 &x, uint4 &y) {
        const int g = r - q_rows;
        const uint16_t *src = g < 0          ? a.q + t * a.q_stride + r * a.D
                              : g < a.Hkv ? a.k + t * a.k_stride + g * a.D
                                          : a.v + t * a.v_stride + (g - a.Hkv) * a.D;
        src += at * 8;
        x = *reinterpret_cast<const uint4 *>(src);
        if (pair) y = *reinterpret_cast<const uint4 *>(src + a.rot / 2);
    };
    uint4 x[BATCH], y[BATCH];
    kvp::grid_dependency_wait();
    kvp::grid_launch_dependents();
    int32_t s = 0, n = 0, end = 0;  // the token's sequence, its context, the token past it
    for (int i = t0, buf = 0; i < turns_end; ++i, buf ^= 1) {
        const bool live = GROUP >= 32 || i < t_end;  // else: the last token once more, without rows
        t = live ? i : t_end - 1;
        const int rows = live ? all_rows : 0;
#pragma unroll
        for (int b = 0; b < BATCH; ++b)
            if (r0 + b * step < rows) load(r0 + b * step, x[b], y[b]);
        if (GROUP < 32 ? __any_sync(0xffffffffu, t >= end) : t >= end) {
            s = a.starts ? seq_of_token<GROUP < 32 ? GROUP : 32>(a.starts, a.S, t, lane) : t;
            n = a.ctx_lens[s];
            end = a.starts ? a.starts[s + 1] : t + 1;
        }
        const int32_t pos = n - (end - t);
        // the token's slot: a sequence without a context (n <= 0) keeps its pages as
        // they are, a position outside the table or a page outside the pool is reported
        // (as is t >= end: a bad array)
        uint8_t *slot = nullptr;
        if (a.k && n > 0) {
            bool ok = t < end && pos >= 0 && pos < a.max_blocks * a.bs;
            if (ok) {
                const int32_t phys = a.table[(int64_t)s * a.max_blocks + pos / a.bs];
                ok = phys >= 0 && (int64_t)phys + a.pages_per_block <= a.n_pages;
                if (ok) slot = a.pool + (int64_t)phys * a.page_bytes + (int64_t)(pos % a.bs) * a.D * 2 + at * 16;
            }
            if (!ok && tid == 0) atomicCAS(a.err, 0, KV_ERR_DEVICE_BOUNDS);
        }
        const int32_t by = a.positions ? a.positions[t] : pos;
        for (int i = tid; i < a.rot / 2; i += GROUP) {
            const uint64_t turn = (uint64_t)(int64_t)by * a.steps[i] + (1ull << 31);
            float sn, cn;
            sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &sn, &cn);
            cosines[buf][sub][i] = cn * a.magnitude;
            sines[buf][sub][i] = sn * a.magnitude;
        }
        // (the other buffer was read before this barrier, and is written after it)
        if (GROUP <= 32)
            __syncwarp();
        else
            asm volatile("bar.sync %0, %1;" ::"r"(1 + sub), "n"(GROUP) : "memory");
        float2 c[4] = {}, sn[4] = {};  // of the item's pairs
        if (turns) {
#pragma unroll
            for (int e = 0; e < (INTERLEAVED ? 2 : 4); ++e) {
                c[e] = *reinterpret_cast<const float2 *>(cosines[buf][sub] + item * (INTERLEAVED ? 4 : 8) + 2 * e);
                sn[e] = *reinterpret_cast<const float2 *>(sines[buf][sub] + item * (INTERLEAVED ? 4 : 8) + 2 * e);
            }
        }
        const int64_t head_bytes = (int64_t)a.bs * a.D * 2;  // of one KV head in a block
        uint8_t *q_dst = reinterpret_cast<uint8_t *>(a.q_out + (int64_t)t * a.Hq * a.D) + at * 16;
        auto finish = [&](int r, uint4 &x0, uint4 &y0) {
            const int g = r - q_rows;
            if (g >= 0 && !slot) return;
            uint8_t *dst = g < 0 ? q_dst + r * a.D * 2 : slot + g * head_bytes;  // v's heads follow k's
            if (turns && g < a.Hkv) {
                if constexpr (INTERLEAVED)
                    turn_adjacent(x0, c, sn);
                else
                    turn_halves(x0, y0, c, sn);
            }
            *reinterpret_cast<uint4 *>(dst) = x0;
            if (pair) *reinterpret_cast<uint4 *>(dst + a.rot) = y0;
        };
        for (int r = r0;;) {
#pragma unroll
            for (int b = 0; b < BATCH; ++b)
                if (r + b * step < rows) finish(r + b * step, x[b], y[b]);
            r += BATCH * step;
            if (r >= rows) break;
#pragma unroll
            for (int b = 0; b < BATCH; ++b)
                if (r + b * step < rows) load(r + b * step, x[b], y[b]);
        }
    }
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

// a row stride that holds the row and keeps 16-byte chunks aligned
bool stride_ok(int64_t stride, int64_t row) { return stride >= row && stride % 8 == 0; }

}  // namespace

extern "C" {

int kv_rotary_freqs(const kv_rotary_desc *d, double *inv_freq)
{
    if (!d || !inv_freq || d->rot_dim < 2 || d->rot_dim % 2 || d->rot_dim > kMaxHeadDim) return KV_ERR_INVALID_ARG;
    if (!(d->base > 1.0) || !std::isfinite(d->base)) return KV_ERR_INVALID_ARG;
    const bool scaled = d->scaling != KV_ROTARY_PLAIN;
    if (d->scaling < KV_ROTARY_PLAIN || d->scaling > KV_ROTARY_BY_PARTS) return KV_ERR_INVALID_ARG;
    if (scaled && (!(d->factor >= 1.0) || !std::isfinite(d->factor))) return KV_ERR_INVALID_ARG;
    const bool parts = d->scaling == KV_ROTARY_BY_PARTS;
    if (parts && (d->original_len < 1 || !(d->low_turns >= 0.0) || !(d->high_turns > d->low_turns) ||
                  !std::isfinite(d->high_turns)))
        return KV_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925286766559;
    for (int i = 0; i < d->rot_dim / 2; ++i) {
        const double f = std::pow(d->base, -2.0 * i / d->rot_dim);
        double keep = scaled ? 0.0 : 1.0;
        if (parts) {
            const double turns = d->original_len * f / two_pi;
            keep = std::min(1.0, std::max(0.0, (turns - d->low_turns) / (d->high_turns - d->low_turns)));
        }
        inv_freq[i] = scaled ? f * keep + f / d->factor * (1.0 - keep) : f;
    }
    return KV_OK;
}

int kv_rotary_steps(const double *inv_freq, int n, uint64_t *steps)
{
    if (!inv_freq || !steps || n < 1) return KV_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i)
        if (!std::isfinite(inv_freq[i])) return KV_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i) {
        const double turns = inv_freq[i] / 6.283185307179586476925286766559;
        double frac = turns - std::floor(turns);  // in [0, 1]
        if (frac >= 1.0) frac = 0.0;
        steps[i] = (uint64_t)std::ldexp(frac, 64);
    }
    return KV_OK;
}

int kv_append_rotary(kv_pool *p, int layout, const kv_rotary *rot, const uint16_t *q, int64_t q_stride, uint16_t *q_out,
                     const uint16_t *k, int64_t k_stride, const uint16_t *v, int64_t v_stride, const int32_t *positions,
                     const int32_t *dev_q_starts, int T, const int32_t *dev_table, const int32_t *dev_ctx_lens,
                     int max_blocks, int S, int Hq, void *stream)
{
    if (!p || !rot || layout < 0 || layout >= p->desc.num_layouts) return KV_ERR_INVALID_ARG;
    if (S < 0 || T < 0 || max_blocks < 1 || Hq < 0 || Hq > 65536) return KV_ERR_INVALID_ARG;
    if (!dev_q_starts && T != S) return KV_ERR_INVALID_ARG;
    if (T > 0 && S == 0) return KV_ERR_INVALID_ARG;
    const kv_layout &L = p->desc.layouts[layout];
    const int64_t D = L.head_dim, Hkv = L.num_kv_heads;
    if (rot->rot_dim < 0 || rot->rot_dim > D || !std::isfinite(rot->magnitude)) return KV_ERR_INVALID_ARG;
    if (rot->interleaved < 0 || rot->interleaved > 1) return KV_ERR_INVALID_ARG;
    if (rot->rot_dim % 16) return KV_ERR_UNSUPPORTED;  // whole 16-byte chunks of either half
    if (rot->rot_dim > 0 && (!rot->steps || ((uintptr_t)rot->steps & 7u))) return KV_ERR_INVALID_ARG;
    if ((int64_t)max_blocks * p->desc.block_size >= INT32_MAX) return KV_ERR_INVALID_ARG;
    if (T == 0) return KV_OK;
    if (!dev_table || !dev_ctx_lens) return KV_ERR_INVALID_ARG;
    if (!q && !k) return KV_ERR_INVALID_ARG;
    if (q && (Hq < 1 || !q_out || !aligned16(q) || !aligned16(q_out) || !stride_ok(q_stride, Hq * D)))
        return KV_ERR_INVALID_ARG;
    if (q && q == q_out && q_stride != Hq * D) return KV_ERR_INVALID_ARG;  // in place: the same rows
    if (!k != !v) return KV_ERR_INVALID_ARG;
    if (k && (!aligned16(k) || !aligned16(v) || !stride_ok(k_stride, Hkv * D) || !stride_ok(v_stride, Hkv * D)))
        return KV_ERR_INVALID_ARG;
    RotaryArgs a{};
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
    a.page_bytes = (int64_t)p->page_bytes;
    a.n_pages = p->n_pages;
    a.magnitude = rot->magnitude;
    a.pages_per_block = p->pages_per_block[layout];
    a.max_blocks = max_blocks;
    a.S = S;
    a.Hq = Hq;
    a.Hkv = (int32_t)Hkv;
    a.D = (int32_t)D;
    a.bs = p->desc.block_size;
    a.rot = rot->rot_dim;
    a.items = (rot->interleaved ? a.rot / 8 : a.rot / 16) + (a.D - a.rot) / 8;
    const int64_t token_items = (int64_t)a.items * ((q ? Hq : 0) + (k ? 2 * Hkv : 0));
    const int64_t resident = (int64_t)kRotShared * std::max(1, p->sm_count);
    const int batch = rot->interleaved ? kRotBatch<true, 32> : kRotBatch<false, 32>;
    int per = 1;  // groups of a CTA (see rotary_kernel)
    while (kRotThreads / per > 8 && kRotThreads / (2 * per) >= a.items && T >= 2 * per * resident &&
           token_items <= batch * (kRotThreads / (2 * per)))
        per *= 2;
    a.run = (int32_t)(T / (per * resident));
    a.longer = (int32_t)(T % (per * resident));
    void (*kernel)(RotaryArgs) = nullptr;
    switch (kRotThreads / per) {
    case 256: kernel = rot->interleaved ? rotary_kernel<true, 256> : rotary_kernel<false, 256>; break;
    case 128: kernel = rot->interleaved ? rotary_kernel<true, 128> : rotary_kernel<false, 128>; break;
    case 64: kernel = rot->interleaved ? rotary_kernel<true, 64> : rotary_kernel<false, 64>; break;
    case 32: kernel = rot->interleaved ? rotary_kernel<true, 32> : rotary_kernel<false, 32>; break;
    case 16: kernel = rot->interleaved ? rotary_kernel<true, 16> : rotary_kernel<false, 16>; break;
    default: kernel = rot->interleaved ? rotary_kernel<true, 8> : rotary_kernel<false, 8>; break;
    }
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(per == 1 ? T : resident));  // (T >= per * resident)
    cfg.blockDim = dim3(kRotThreads);
    cfg.stream = (cudaStream_t)stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, a) != cudaSuccess)
        return KV_ERR_CUDA;
    kvp_note_stream(stream, false);
    return KV_OK;
}

}  // extern "C"
