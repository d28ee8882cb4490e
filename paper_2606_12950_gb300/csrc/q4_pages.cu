// q4_pages.cu -- cache blocks packed into 4 bits and back (KV_Q4 layouts), and
// the call on sequence tables that moves a chat's old tokens there
// (kv_seq_pack).
//
// A group of 64 columns of a token's row: z = min x, s = bf16((max x - z) / 15),
// c = the code nearest to (x - z) / s, ties to even.  The quotient is D i (D = x
// - z, i = 1 / s), corrected once by its residual, q + (D - q s) i, which rounds
// to the nearest fp32 quotient: where D / s is a code and a half exactly, so is
// the corrected quotient, and adding 1.5 * 2^23 rounds it to even.
//
// Bound by HBM, and close to it by instructions: a value is read in 2 bytes and written
// in 9/16, or the other way.  2040 blocks of 64 KB (171 MB) are packed in 29.6 us (5.8
// TB/s; 36.7 one value an instruction, every lane finding its groups' parameters) and
// unpacked in 26; 4000 packed and read back 111.6 us (671 MB, 6.0 TB/s), 6000 read back
// 80.5 (504 MB, 6.26 TB/s).
// A warp takes a tile (16 tokens of a KV head, K and V): K's rows as 16-byte
// chunks of 8 columns, four lanes a row, V's eight lanes a row, so that each lane
// holds what its words of the packed tile are made of (q4_format.h) and a group's
// least and greatest values are found by shuffles among 4 or 8 lanes.
#include <algorithm>
#include <mutex>
#include <new>
#include <vector>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "pages_internal.h"
#include "pool_internal.h"
#include "ptx.cuh"
#include "q4_format.h"
#include "seqtab_internal.h"
#include "stream_order.h"

namespace {

constexpr int kPackThreads = 128, kUnpackThreads = 256;
constexpr float kSpanLimit = 0x1p80f;   // spans from here on are NaN
constexpr float kScaleLeast = 0x1p-100f;  // scales below are 0

template <int N>
struct PackParams {
    uint8_t *pool;
    int64_t page_bytes;
    int32_t Hkv;
    int32_t tiles;   // of a head in a block
    int32_t at[N][2];  // source page, destination page
};

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// The least value and the greatest one's negative of a chunk, NaN if one is: a
// pair, so that a step among lanes is one shuffle and one minimum.
__device__ __forceinline__ __nv_bfloat162 extremes(const uint4 &x)
{
    const __nv_bfloat162 *p = reinterpret_cast<const __nv_bfloat162 *>(&x);
    const __nv_bfloat162 mn = __hmin2_nan(__hmin2_nan(p[0], p[1]), __hmin2_nan(p[2], p[3]));
    const __nv_bfloat162 mx = __hmax2_nan(__hmax2_nan(p[0], p[1]), __hmax2_nan(p[2], p[3]));
    return __halves2bfloat162(__hmin_nan(mn.x, mn.y), __hneg(__hmax_nan(mx.x, mx.y)));
}
__device__ __forceinline__ __nv_bfloat162 shuffled(__nv_bfloat162 v, int off)
{
    const uint32_t w = __shfl_xor_sync(0xffffffffu, *reinterpret_cast<uint32_t *>(&v), off);
    return *reinterpret_cast<const __nv_bfloat162 *>(&w);
}

// Of N values a lane, each to be joined over N lanes (of those whose numbers differ
// in bits N / 2 * STEP .. STEP): the one that this lane's bits name, joined.  log2 N
// rounds of N / 2, N / 4, .. shuffles.
template <int N, int STEP>
__device__ __forceinline__ __nv_bfloat162 joined(__nv_bfloat162 (&e)[N], int lane)
{
#pragma unroll
    for (int n = N / 2; n > 0; n /= 2) {
        const bool up = (lane & (n * STEP)) != 0;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const __nv_bfloat162 keep = up ? e[i + n] : e[i], give = up ? e[i] : e[i + n];
            e[i] = __hmin2_nan(keep, shuffled(give, n * STEP));
        }
    }
    return e[0];
}

// A group's parameters, (s, z) as they are stored, and about 1 / s; each lane that
// shares the group's row computes another group's.
__device__ __forceinline__ uint32_t params_of(__nv_bfloat162 ext, float &inv)
{
    const float lo = __bfloat162float(ext.x), span = -__bfloat162float(ext.y) - lo;
    // span / 15, rounded to the nearest fp32: a quotient corrected by its residual
    const float q = span * (1.f / 15.f);
    __nv_bfloat16 s = __float2bfloat16_rn(__fmaf_rn(__fmaf_rn(-q, 15.f, span), 1.f / 15.f, q));
    if (!(__bfloat162float(s) >= kScaleLeast)) s = __float2bfloat16_rn(0.f);
    if (!(span < kSpanLimit)) s = __ushort_as_bfloat16(0x7fc0);  // NaN
    const float f = __bfloat162float(s);
    inv = f > 0.f ? __fdividef(1.f, f) : 0.f;
    return (uint32_t)__bfloat16_as_ushort(s) | (__float_as_uint(lo) & 0xFFFF0000u);
}

// As the codes take them, two values at a time.
struct Group {
    float2 ns, nz, inv;  // -s, -z, 1 / s
    __device__ __forceinline__ Group(uint32_t word, float i)
    {
        ns = make_float2(-lo_f(word), -lo_f(word));
        nz = make_float2(-hi_f(word), -hi_f(word));
        inv = make_float2(i, i);
    }
};

// kCodeBase plus the codes of a word's two values (0 where s = 0; anything in a NaN
// group), whole numbers.
constexpr float kCodeBase = 12582912.f;  // 1.5 * 2^23
__device__ __forceinline__ float2 based_codes(uint32_t w, const Group &g)
{
    const float2 d = __fadd2_rn(make_float2(lo_f(w), hi_f(w)), g.nz), q = __fmul2_rn(d, g.inv);
    return __fadd2_rn(__ffma2_rn(__ffma2_rn(q, g.ns, d), g.inv, q), make_float2(kCodeBase, kCodeBase));
}
// the next word's codes, 256 times, added
__device__ __forceinline__ float2 with_next(float2 based, float2 next)
{
    return __ffma2_rn(__fadd2_rn(next, make_float2(-kCodeBase, -kCodeBase)), make_float2(256.f, 256.f), based);
}
// Codes are joined as fp32 sums above kCodeBase, whose low 16 bits four of them are:
// the integer units, which split and compare the bf16 pairs, have less to spare.
__device__ __forceinline__ float four(float2 based) { return __fmaf_rn(based.y - kCodeBase, 16.f, based.x); }
__device__ __forceinline__ uint32_t eight(float lo, float hi)
{
    return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x5410);
}

template <int D, int N>
__global__ void __launch_bounds__(kPackThreads, 6) pack_blocks_kernel(const __grid_constant__ PackParams<N> p)
{
    constexpr int NG = D / kQ4Group, NW = D / 32, TILE = kQ4TileBytes<D>;
    kvp::grid_dependency_wait();
    kvp::grid_launch_dependents();
    const int unit = blockIdx.y * (kPackThreads / 32) + (threadIdx.x >> 5);  // (head, tile)
    if (unit >= p.Hkv * p.tiles) return;
    const int lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;

    const int64_t kv = (int64_t)p.Hkv * p.tiles * 32 * D;  // bytes of a block's K
    const uint8_t *src = p.pool + (int64_t)p.at[blockIdx.x][0] * p.page_bytes + (int64_t)unit * 32 * D;
    uint8_t *dst = p.pool + (int64_t)p.at[blockIdx.x][1] * p.page_bytes + (int64_t)unit * TILE;
    uint4 k[2][NW], v[4][NG];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int j = 0; j < NW; ++j)
            k[r][j] = *reinterpret_cast<const uint4 *>(src + (gid + 8 * r) * 2 * D +
                                                       2 * (64 * (j >> 1) + 32 * (j & 1) + 8 * tig));
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < NG; ++c)
            v[r][c] = *reinterpret_cast<const uint4 *>(src + kv + (2 * tig + (r & 1) + 4 * (r & 2)) * 2 * D +
                                                       2 * (64 * c + 8 * gid));
    // ---- K: four lanes hold a row, and each finds the parameters of one of the
    // tile's groups that lie with them (or of one of two, twice) ----
    {
        __nv_bfloat162 ext[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = i & 1, c = NG == 2 ? i >> 1 : 0;  // (row, group)
            ext[i] = __hmin2_nan(extremes(k[r][2 * c]), extremes(k[r][2 * c + 1]));
        }
        float inv;
        const uint32_t mine = params_of(joined<4, 1>(ext, lane), inv);
        if (tig < 2 * NG)
            *(reinterpret_cast<uint32_t *>(dst + 16 * D) + (gid + 8 * (tig & 1)) * 2 * NG + (tig >> 1)) = mine;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            uint32_t codes[NW];
#pragma unroll
            for (int c = 0; c < NG; ++c) {
                const int from = (lane & ~3) + 2 * c + r;
                const Group g(__shfl_sync(0xffffffffu, mine, from), __shfl_sync(0xffffffffu, inv, from));
#pragma unroll
                for (int j = 2 * c; j < 2 * c + 2; ++j) {
                    const uint32_t *w = reinterpret_cast<const uint32_t *>(&k[r][j]);
                    codes[j] = eight(four(with_next(based_codes(w[0], g), based_codes(w[1], g))),
                                     four(with_next(based_codes(w[2], g), based_codes(w[3], g))));
                }
            }
            uint8_t *row = dst + (gid + 8 * r) * (D / 2) + tig * (D / 8);
            if constexpr (NW == 4)
                *reinterpret_cast<uint4 *>(row) = make_uint4(codes[0], codes[1], codes[2], codes[3]);
            else
                *reinterpret_cast<uint2 *>(row) = make_uint2(codes[0], codes[1]);
        }
    }
    // ---- V: eight lanes hold a row's group, four rows and NG groups each ----
    {
        __nv_bfloat162 ext[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) ext[i] = extremes(v[i & 3][NG == 2 ? i >> 2 : 0]);
        float inv;
        const uint32_t mine = params_of(joined<8, 4>(ext, lane), inv);
        if (gid < 4 * NG)
            *(reinterpret_cast<uint32_t *>(dst + 16 * D) + (2 * tig + (gid & 1) + 4 * (gid & 2)) * 2 * NG + NG + (gid >> 2)) = mine;
#pragma unroll
        for (int c = 0; c < NG; ++c) {
            // tokens a, a + 8 (r = 0, 2) are a word's low half, a + 1 and a + 9 its high one
            float2 half[2][4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int from = tig + 4 * (4 * c + r);
                uint32_t word = __shfl_sync(0xffffffffu, mine, from);
                const float i = __shfl_sync(0xffffffffu, inv, from);
                // (a NaN group's codes are 0: the sums are other tokens' too)
                const bool ok = (word & 0x7fffu) < 0x7f80u;
                word = ok ? word : 0u;
                const Group g(word, i);
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const float2 b = based_codes(ok ? reinterpret_cast<const uint32_t *>(&v[r][c])[m] : 0u, g);
                    half[r & 1][m] = r < 2 ? b : with_next(half[r & 1][m], b);
                }
            }
            *reinterpret_cast<uint4 *>(dst + 8 * D + 512 * c + 16 * lane) =
                make_uint4(eight(four(half[0][0]), four(half[1][0])), eight(four(half[0][1]), four(half[1][1])),
                           eight(four(half[0][2]), four(half[1][2])), eight(four(half[0][3]), four(half[1][3])));
        }
    }
}

// bf16(s c + z) of two codes of a word
__device__ __forceinline__ uint32_t values_of(uint32_t w, int a, int b, float s, float z)
{
    const float x = __uint_as_float(((w >> (4 * a)) & 15u) | 0x4B000000u) - 8388608.f;
    const float y = __uint_as_float(((w >> (4 * b)) & 15u) | 0x4B000000u) - 8388608.f;
    __nv_bfloat162 v = __floats2bfloat162_rn(__fmaf_rn(x, s, z), __fmaf_rn(y, s, z));
    return *reinterpret_cast<uint32_t *>(&v);
}

template <int D, int N>
__global__ void __launch_bounds__(kUnpackThreads) unpack_blocks_kernel(const __grid_constant__ PackParams<N> p)
{
    constexpr int NG = D / kQ4Group, NW = D / 32, TILE = kQ4TileBytes<D>;
    kvp::grid_dependency_wait();
    kvp::grid_launch_dependents();
    const int unit = blockIdx.y * (kUnpackThreads / 32) + (threadIdx.x >> 5);  // (head, tile)
    if (unit >= p.Hkv * p.tiles) return;
    const int lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    const int64_t kv = (int64_t)p.Hkv * p.tiles * 32 * D;
    const uint8_t *src = p.pool + (int64_t)p.at[blockIdx.x][0] * p.page_bytes + (int64_t)unit * TILE;
    uint8_t *dst = p.pool + (int64_t)p.at[blockIdx.x][1] * p.page_bytes + (int64_t)unit * 32 * D;
    uint32_t k[2][NW], v[NG][4], kp[2][NG], vp[4][NG];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const uint8_t *row = src + (gid + 8 * r) * (D / 2) + tig * (D / 8);
#pragma unroll
        for (int j = 0; j < NW; j += 2) {
            const uint2 w = *reinterpret_cast<const uint2 *>(row + 4 * j);
            k[r][j] = w.x;
            k[r][j + 1] = w.y;
        }
#pragma unroll
        for (int c = 0; c < NG; ++c) kp[r][c] = *(reinterpret_cast<const uint32_t *>(src + 16 * D) + (gid + 8 * r) * 2 * NG + c);
    }
#pragma unroll
    for (int c = 0; c < NG; ++c) {
        const uint4 w = *reinterpret_cast<const uint4 *>(src + 8 * D + 512 * c + 16 * lane);
        v[c][0] = w.x;
        v[c][1] = w.y;
        v[c][2] = w.z;
        v[c][3] = w.w;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            vp[r][c] = *(reinterpret_cast<const uint32_t *>(src + 16 * D) +
                         (2 * tig + (r & 1) + 4 * (r & 2)) * 2 * NG + NG + c);
    }
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int j = 0; j < NW; ++j) {
            const float s = lo_f(kp[r][j >> 1]), z = hi_f(kp[r][j >> 1]);
            const uint32_t w = k[r][j];
            *reinterpret_cast<uint4 *>(dst + (gid + 8 * r) * 2 * D + 2 * (64 * (j >> 1) + 32 * (j & 1) + 8 * tig)) =
                make_uint4(values_of(w, 0, 1, s, z), values_of(w, 2, 3, s, z), values_of(w, 4, 5, s, z),
                           values_of(w, 6, 7, s, z));
        }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < NG; ++c) {
            const float s = lo_f(vp[r][c]), z = hi_f(vp[r][c]);
            const int nib = 4 * (r & 1) + (r & 2);
            *reinterpret_cast<uint4 *>(dst + kv + (2 * tig + (r & 1) + 4 * (r & 2)) * 2 * D + 2 * (64 * c + 8 * gid)) =
                make_uint4(values_of(v[c][0], nib, nib + 1, s, z), values_of(v[c][1], nib, nib + 1, s, z),
                           values_of(v[c][2], nib, nib + 1, s, z), values_of(v[c][3], nib, nib + 1, s, z));
        }
}

// one launch of n pairs (n <= N)
template <int N>
int pack_launch(const kv_pool *p, int layout, int n, const int32_t *src, const int32_t *dst, bool unpack, cudaStream_t st)
{
    PackParams<N> c;
    c.pool = reinterpret_cast<uint8_t *>(p->desc.device_base);
    c.page_bytes = (int64_t)p->page_bytes;
    c.Hkv = p->desc.layouts[layout].num_kv_heads;
    c.tiles = p->desc.block_size / kQ4Tile;
    for (int i = 0; i < n; ++i) {
        c.at[i][0] = src[i];
        c.at[i][1] = dst[i];
    }
    const int threads = unpack ? kUnpackThreads : kPackThreads, per_cta = threads / 32;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)n, (unsigned)((c.Hkv * c.tiles + per_cta - 1) / per_cta));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    void (*kernel)(PackParams<N>) =
        kvp_head_dim(p->desc.layouts[layout]) == 64
            ? (unpack ? unpack_blocks_kernel<64, N> : pack_blocks_kernel<64, N>)
            : (unpack ? unpack_blocks_kernel<128, N> : pack_blocks_kernel<128, N>);
    if (cudaLaunchKernelEx(&cfg, kernel, c) != cudaSuccess) return KV_ERR_CUDA;
    kvp_note_stream(st, false);
    return KV_OK;
}

// parameter blocks of three sizes: a launch's cost grows with its bytes
constexpr int kPackSmall = 120;   // 1 KB
constexpr int kPackMid = 504;     // 4 KB
constexpr int kPackLarge = 2040;  // 16 KB

int pack_run(const kv_pool *p, int layout, int n, const int32_t *src, const int32_t *dst, bool unpack, void *stream)
{
    cudaStream_t st = (cudaStream_t)stream;
    for (int i = 0; i < n;) {
        const int m = std::min(n - i, kPackLarge);
        const int rc = m <= kPackSmall ? pack_launch<kPackSmall>(p, layout, m, src + i, dst + i, unpack, st)
                       : m <= kPackMid ? pack_launch<kPackMid>(p, layout, m, src + i, dst + i, unpack, st)
                                       : pack_launch<kPackLarge>(p, layout, m, src + i, dst + i, unpack, st);
        if (rc) return rc;
        i += m;
    }
    return KV_OK;
}

// a bf16 layout and a 4-bit one of the same geometry
int check_layouts(const kv_pool *p, int layout, int q4_layout)
{
    if (!p || layout < 0 || layout >= p->desc.num_layouts || q4_layout < 0 || q4_layout >= p->desc.num_layouts)
        return KV_ERR_INVALID_ARG;
    const kv_layout &L = p->desc.layouts[layout], &Q = p->desc.layouts[q4_layout];
    if (kvp_is_q4(L) || !kvp_is_q4(Q)) return KV_ERR_UNSUPPORTED;
    if (L.num_kv_heads != Q.num_kv_heads || L.head_dim != kvp_head_dim(Q)) return KV_ERR_INVALID_ARG;
    return KV_OK;
}

int pack_call(kv_pool *p, int layout, int q4_layout, int n, const int32_t *src, const int32_t *dst, bool unpack, void *stream)
{
    int rc = check_layouts(p, layout, q4_layout);
    if (rc) return rc;
    if (n < 0) return KV_ERR_INVALID_ARG;
    if (n == 0) return KV_OK;
    if (!src || !dst || !kvp_on_device(p)) return KV_ERR_INVALID_ARG;
    const int from = unpack ? q4_layout : layout, to = unpack ? layout : q4_layout;
    {
        // every id a live block of its layout, no destination twice.  Marks go to
        // the pool's tally, which is all zeros between calls.
        std::lock_guard<std::mutex> g(p->mu);
        auto live = [&](int32_t id, int l) {
            return id >= 0 && id < p->n_pages && p->owner[(size_t)id] == l && p->refcnt[(size_t)id] > 0;
        };
        bool ok = true;
        int marked = 0;
        for (; ok && marked < n; ++marked) {
            ok = live(src[marked], from) && live(dst[marked], to) && !p->tally[(size_t)dst[marked]];
            if (!ok) break;
            p->tally[(size_t)dst[marked]] = 1;
        }
        for (int i = 0; i < marked; ++i) p->tally[(size_t)dst[i]] = 0;
        if (!ok) return KV_ERR_INVALID_ARG;
    }
    return pack_run(p, layout, n, src, dst, unpack, stream);
}

}  // namespace

extern "C" {

int kv_pack_blocks(kv_pool *p, int layout, int q4_layout, int n, const int32_t *src, const int32_t *dst, void *stream)
{
    return pack_call(p, layout, q4_layout, n, src, dst, false, stream);
}

int kv_unpack_blocks(kv_pool *p, int q4_layout, int layout, int n, const int32_t *src, const int32_t *dst, void *stream)
{
    return pack_call(p, layout, q4_layout, n, src, dst, true, stream);
}

int kv_seq_pack(kv_seqtab *t, kv_seqtab *t4, int n, const int32_t *slots, int keep, void *stream, int32_t *n_packed)
{
    if (!t || !t4 || !t->pool || t->pool != t4->pool || t->S != t4->S || n < 0 || (n > 0 && !slots) || keep < 1)
        return KV_ERR_INVALID_ARG;
    int rc = check_layouts(t->pool, t->layout, t4->layout);
    if (rc) return rc;
    if (n_packed) *n_packed = 0;
    try {
        std::vector<int32_t> src, dst;
        std::vector<uint8_t> seen((size_t)t->S, 0);
        auto range = [&](int32_t s, int &from, int &to) {  // blocks of slot s to pack: [from, to)
            from = t4->lens[(size_t)s] / t->bs;
            to = std::max(from, (int)(std::max<int64_t>(0, (int64_t)t->lens[(size_t)s] - keep) / t->bs));
        };
        for (int i = 0; i < n; ++i) {
            const int32_t s = slots[i];
            if (s < 0 || s >= t->S || seen[(size_t)s]) return KV_ERR_INVALID_ARG;
            seen[(size_t)s] = 1;
            const int32_t done = t4->lens[(size_t)s];
            if (done % t->bs || t4->held[(size_t)s] != done / t->bs || done > t->lens[(size_t)s]) return KV_ERR_INVALID_ARG;
            int from, to;
            range(s, from, to);
            if (to > t4->max_blocks) return KV_ERR_INVALID_ARG;
            for (int b = from; b < to; ++b) {
                const int32_t id = t->table[(size_t)s * t->max_blocks + b];
                if (id < 0) return KV_ERR_INVALID_ARG;  // given up
                src.push_back(id);
            }
        }
        if (src.empty()) return KV_OK;
        if (!kvp_on_device(t->pool)) return KV_ERR_INVALID_ARG;
        const int m = (int)src.size();
        dst.resize((size_t)m);
        rc = kv_alloc_blocks(t4->pool, t4->layout, m, dst.data());
        if (rc) return rc;
        rc = pack_run(t->pool, t->layout, m, src.data(), dst.data(), false, stream);
        if (!rc) rc = kv_free_blocks(t->pool, t->layout, m, src.data());
        if (rc) {  // as before the call
            kv_free_blocks(t4->pool, t4->layout, m, dst.data());
            return rc;
        }
        for (int i = 0, k = 0; i < n; ++i) {
            const int32_t s = slots[i];
            int from, to;
            range(s, from, to);
            for (int b = from; b < to; ++b) {
                kvp_seqtab_set_entry(t, s, b, -1);
                kvp_seqtab_set_entry(t4, s, b, dst[(size_t)k++]);
            }
            if (to > from) {
                t4->held[(size_t)s] = to;
                t4->lens[(size_t)s] = to * t->bs;
            }
        }
        t->counters.blocks_held -= m;
        t4->counters.blocks_held += m;
        if (n_packed) *n_packed = m;
    } catch (const std::bad_alloc &) {
        return KV_ERR_OUT_OF_BLOCKS;
    }
    return KV_OK;
}

}  // extern "C"
