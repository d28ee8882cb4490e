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
// a decode step.  A CTA takes one token: its cos and sin are computed once,
// into shared memory, for all heads.
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
};

// largest s with starts[s] <= t (starts ascending, starts[0] <= t): 32 probes a
// round trip; the whole warp, converged
__device__ __forceinline__ int seq_of_token(const int32_t *starts, int S, int t, int lane)
{
    int lo = 0, n = S;  // the answer is in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32;
        const int i = lo + lane * step;
        const unsigned le = __ballot_sync(0xffffffffu, lane * step < n && starts[i] <= t);
        const int k = 31 - __clz((int)(le | 1u));
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

constexpr int kRotBatch = 4;  // rows a thread loads before it needs the token's position

// One CTA per token.  Its Hq + 2 Hkv rows (q, k, v) are cut alike into items: a
// pair of chunks that turn together (half layout), a chunk that turns (adjacent
// pairs) or one that passes through; a thread keeps its item and goes from row
// to row.  The rows' addresses need the token alone, so each thread loads its
// first kRotBatch rows before the position, the angles and the slot, four
// dependent loads away, are known.  16000 tokens of 40 q and 8 KV heads, half of
// each head turned (460 MB): 98.7 us with the loads after the position, 81.0
// with them before, 73.4 with an item a thread (issue slots had been 79% taken; 6.27 TB/s).
// Pointers are not __restrict__: the kernel may be resident while the grid
// before it still writes what it reads, and a const __restrict__ pointer may be
// read through the non-coherent path, which the wait below does not order.
template <bool INTERLEAVED>
__global__ void __launch_bounds__(kRotThreads) rotary_kernel(const __grid_constant__ RotaryArgs a)
{
    __shared__ __align__(16) float cosines[kMaxHeadDim / 2], sines[kMaxHeadDim / 2];  // times the magnitude
    const int tid = threadIdx.x, lane = tid & 31, t = blockIdx.x;
    const int turned = INTERLEAVED ? a.rot / 8 : a.rot / 16;
    const int items = a.items;  // of a row: those that turn, then the others
    const int step = kRotThreads / items;  // rows at a time
    const int item = tid % items, r0 = tid / items;
    const bool turns = item < turned, pair = !INTERLEAVED && turns;
    const int at = turns ? item : item + a.rot / 8 - turned;  // the item's (first) chunk
    const int q_rows = a.q ? a.Hq : 0, rows = r0 < step ? q_rows + (a.k ? 2 * a.Hkv : 0) : 0;
    const uint16_t *qs = a.q + (int64_t)t * a.q_stride + at * 8, *ks = a.k + (int64_t)t * a.k_stride + at * 8,
                   *vs = a.v + (int64_t)t * a.v_stride + at * 8;
    auto load = [&](int r, uint4 &x, uint4 &y) {
        const int g = r - q_rows;
        const uint16_t *src = g < 0 ? qs + r * a.D : g < a.Hkv ? ks + g * a.D : vs + (g - a.Hkv) * a.D;
        x = *reinterpret_cast<const uint4 *>(src);
        if (pair) y = *reinterpret_cast<const uint4 *>(src + a.rot / 2);
    };
    uint4 x[kRotBatch], y[kRotBatch];
    kvp::grid_dependency_wait();
    kvp::grid_launch_dependents();
#pragma unroll
    for (int b = 0; b < kRotBatch; ++b)
        if (r0 + b * step < rows) load(r0 + b * step, x[b], y[b]);
    const int s = a.starts ? seq_of_token(a.starts, a.S, t, lane) : t;
    const int32_t n = a.ctx_lens[s];
    const int32_t end = a.starts ? a.starts[s + 1] : t + 1;  // past the sequence's tokens; t past it: a bad array
    const int32_t pos = n - (end - t);
    // the token's slot: a sequence without a context (n <= 0) keeps its pages as
    // they are, a position outside the table or a page outside the pool is reported
    uint8_t *slot = nullptr;
    if (a.k && n > 0) {
        bool ok = t < end && pos >= 0 && pos < a.max_blocks * a.bs;
        if (ok) {
            const int32_t phys = a.table[(int64_t)s * a.max_blocks + pos / a.bs];
            ok = phys >= 0 && (int64_t)phys + a.pages_per_block <= a.n_pages;
            if (ok) slot = a.pool + (int64_t)phys * a.page_bytes + (int64_t)(pos % a.bs) * a.D * 2;
        }
        if (!ok && tid == 0) atomicCAS(a.err, 0, KV_ERR_DEVICE_BOUNDS);
    }
    {
        const int32_t by = a.positions ? a.positions[t] : pos;
        for (int i = tid; i < a.rot / 2; i += kRotThreads) {
            const uint64_t turn = (uint64_t)(int64_t)by * a.steps[i] + (1ull << 31);
            float sn, cn;
            sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &sn, &cn);
            cosines[i] = cn * a.magnitude;
            sines[i] = sn * a.magnitude;
        }
    }
    __syncthreads();
    float2 c[4] = {}, sn[4] = {};  // of the item's pairs
    if (turns) {
#pragma unroll
        for (int e = 0; e < (INTERLEAVED ? 2 : 4); ++e) {
            c[e] = *reinterpret_cast<const float2 *>(cosines + item * (INTERLEAVED ? 4 : 8) + 2 * e);
            sn[e] = *reinterpret_cast<const float2 *>(sines + item * (INTERLEAVED ? 4 : 8) + 2 * e);
        }
    }
    const int64_t head_bytes = (int64_t)a.bs * a.D * 2;  // of one KV head in a block
    uint8_t *q_dst = reinterpret_cast<uint8_t *>(a.q_out + (int64_t)t * a.Hq * a.D) + at * 16;
    if (slot) slot += at * 16;
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
#pragma unroll
    for (int b = 0; b < kRotBatch; ++b)
        if (r0 + b * step < rows) finish(r0 + b * step, x[b], y[b]);
    for (int r = r0 + kRotBatch * step; r < rows; r += step) {
        load(r, x[0], y[0]);
        finish(r, x[0], y[0]);
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
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)T);
    cfg.blockDim = dim3(kRotThreads);
    cfg.stream = (cudaStream_t)stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, rot->interleaved ? rotary_kernel<true> : rotary_kernel<false>, a) != cudaSuccess)
        return KV_ERR_CUDA;
    kvp_note_stream(stream, false);
    return KV_OK;
}

}  // extern "C"
