// prompt_impl.cuh -- causal attention of prompt chunks over the paged pool,
// with a sliding window and sinks, on the fifth-generation tensor cores.
//
// A query at position p of its sequence sees the tokens j <= p with
// j > p - window or j < sinks (window 0: all).  The query heads of a KV head
// share its K and V, so a Q tile's 128 rows are TQ = floor(128 / G)
// consecutive tokens x G heads of one (sequence, KV head), and an item, the
// unit of work, is two Q tiles (2 TQ tokens) over their common key range, in
// 128-key tiles:
//   S = Q K^T     tcgen05.mma, M = 128 rows, N = 128 keys, fp32 in TMEM
//   softmax       one thread per row, S read from TMEM, base 2, lazy rescale
//   O += P V      tcgen05.mma, P (bf16) over S in TMEM, V from shared memory
// While one Q tile's four warps run the softmax the tensor core works on the
// other's.
//
// CTAs stay and take one item after another, so that the next item's K and V
// (a warp each, TMA, 16-token boxes, 128-byte swizzle, two stages, released
// apart) and Q load while the last tiles of the one before are worked on and
// its output is written.  One warp issues the MMAs; one looks up the next
// item, loads Q and checks V (below).
//
// Keys.  An item's tiles are those of the sinks, then those from its first
// query's window on up to its last query; a tile in which some query of the
// item does not see some token (the diagonal, the window's edge, the sinks'
// edge) is masked element by element, the others are not looked at.
// 16-token boxes that no query of the item sees are not loaded: their table
// entries may be gone (kv_seq_evict).
//
// NaN and infinities.  A weight of 0 times a NaN is NaN in the MMA.  So in
// masked tiles the rows of V that no query sees are cleared, and rows that some
// query sees and that hold a NaN or an infinity are cleared too and noted; at
// the end each row adds the noted tokens that it sees itself.
//
// What bounds it, and what it measured.  At d = 128 (32 q / 8 KV heads): the
// chain S -> softmax -> P.V -> S of a Q tile, 2450 clocks for two 128 x 128
// tiles where the tensor core's own time is 2048, and the power limit: 16384
// tokens with a window of 4096 (963 GFLOP) 658 us, 1460 TFLOP/s (a plain library
// product 1705 sustained; the lowest seen on any GPU 600 us).  At d = 64: the softmax warps, 2440
// clocks where the exponentials are 1100 (each warp's own latencies; two Q tiles
// leave a sub-partition two warps): 5 causal prompts of 700 to 2500 tokens, 16
// heads, 69 to 78 us.  Short items pay 5 us for a CTA's start and about 8000
// clocks an item (masked tiles, output): 9 ragged chunks, window 1024, 67 to 74
// us for 52 GFLOP.
//
// Few rows (KS > 1): an item's key tiles are split over KS items, each leaving
// per row one fp32 record (o, running max, sum) that prompt_merge_kernel merges.
#pragma once

#include "attn_impl.cuh"

namespace kvp {

constexpr int kPrRows = 128;   // rows of a Q tile: the MMA's M
constexpr int kPrTiles = 2;    // Q tiles per item
constexpr int kPrKeys = 128;   // keys per tile: S's N, P.V's K
// Keys whose weights are handed over first: at d = 128, where S of the next tile
// waits for P.V, 96, so that the tensor core, which takes the Q tiles in turn,
// does not run out of them before the others are there; at d = 64 all.
template <int D>
constexpr int kPrFirst = D == 64 ? 128 : 96;
constexpr int kPrStages = 2;
constexpr int kPrSlots = 4;    // published items: the softmax warps hold one until its output is written
constexpr int kPrSoft = kPrTiles * 128;     // softmax threads, one per row
constexpr int kPrThreads = kPrSoft + 128;   // + K and V load warps, MMA warp, scheduling warp
// Registers a thread, by warpgroup: launched with 168; a softmax thread holds a
// row's 128 scores, the others need fewer.  2 x 128 x 200 + 128 x 104 = 384 x 168.
constexpr int kPrRegsLaunch = 168, kPrRegsSoft = 200, kPrRegsOther = 104;
static_assert(kPrSoft * kPrRegsSoft + 128 * kPrRegsOther <= kPrThreads * kPrRegsLaunch, "what the launch holds");
constexpr int kPrMasked = 16;  // masked tiles of an item: 3 on the diagonal, 3 at the window's edge, 2 of sinks at most
constexpr int kPrMaxSplits = 16;
// TMEM's 512 columns.  At d = 128: per Q tile S (128, fp32) with P (64, bf16
// pairs) over it, and O (128).  At d = 64 O takes half of that and P has columns
// of its own: S of the next tile is computed while the softmax still works on
// this one, so that only the softmax's own time counts.
constexpr uint32_t kPrTmem = 512;
template <int D>
struct PrCols {
    static constexpr bool SEP = D == 64;  // P apart from S
    static __device__ __forceinline__ uint32_t s(int q) { return SEP ? q * 128 : q * 256; }
    static __device__ __forceinline__ uint32_t p(int q) { return SEP ? 256 + q * 64 : q * 256; }
    static __device__ __forceinline__ uint32_t o(int q) { return SEP ? 384 + q * 64 : q * 256 + 128; }
};

struct PromptArgs {
    const uint16_t *q;
    uint16_t *out;
    const uint16_t *pool;
    const int32_t *starts;
    const int32_t *table;
    const int32_t *ctx_lens;
    int32_t *err;
    float *ws;             // KS > 1: the splits' o [KS][T][Hq][D], unnormalised, then (m, l) [KS][T][Hq]
    int64_t rows_per_page;
    int64_t pool_pages;
    int32_t pages_per_block;
    int32_t max_blocks;
    int32_t S, Hkv, G, bs, T;
    int32_t max_q;         // the longest chunk by the caller's word: n_items goes by it
    int32_t n_items;       // tiles * Hkv * KS
    int32_t KS;
    int32_t window, sinks; // window 0: the whole context
    float sign;            // 1, or what the scores are multiplied by first: -1 or 0 with the scale's sign
    float qk_scale;        // |scale| * log2(e) (1 where the scale is 0)
};

// An item: tokens [row0, row0 + ntok) of q, positions p0 .. p1 of sequence s,
// KV head g, and its key tiles.
struct PrItem {
    int32_t s;         // -1: no more items
    int32_t row0;      // q row of its first token
    int32_t ntok;
    int32_t p0, p1;    // positions of its first and last token
    int32_t lo;        // first token of the first query's window
    int32_t head;      // key tiles of the sinks before the window's tiles
    int32_t gap;       // key tiles left out between the two
    int32_t t0, nt;    // the tiles of this split: the first one, how many
    int32_t g, ks;
    __device__ __forceinline__ int32_t key0(int32_t t) const
    {
        const int32_t i = t0 + t;
        return (i < head ? i : i + gap) * kPrKeys;
    }
    // some query does not see some token of the tile at k0
    __device__ __forceinline__ bool masked(const PromptArgs &a, int32_t k0) const
    {
        return k0 + kPrKeys - 1 > p0 || (a.window > 0 && k0 <= p1 - a.window && k0 + kPrKeys > a.sinks);
    }
    // some query sees some token of [tok, tok + n)
    __device__ __forceinline__ bool sees(const PromptArgs &a, int32_t tok, int32_t n) const
    {
        return tok <= p1 && (tok + n > lo || tok < a.sinks);
    }
};

// shared memory (offsets from a 1024-byte aligned base)
template <int D>
struct PrSmem {
    static constexpr int HALVES = D / 64;
    static constexpr uint32_t KV_HALF = kPrKeys * 128;
    static constexpr uint32_t KV_TILE = HALVES * KV_HALF;
    static constexpr uint32_t STAGE = 2 * KV_TILE;
    static constexpr uint32_t Q_HALF = kPrRows * 128;
    static constexpr uint32_t Q_TILE = HALVES * Q_HALF;
    static constexpr uint32_t ST_OFF = kPrTiles * Q_TILE;
    static constexpr uint32_t X_OFF = ST_OFF + kPrStages * STAGE;       // 4 KB per softmax warp for the output
    static constexpr uint32_t BAR_OFF = X_OFF + kPrSoft / 32 * 4096;
    static constexpr int NBARS = 36;
    static constexpr uint32_t SLOT_OFF = BAR_OFF + NBARS * 8;
    static constexpr uint32_t ITEM_OFF = SLOT_OFF + 16;                 // [kPrSlots] PrItem
    static constexpr uint32_t NOTE_OFF = ITEM_OFF + kPrSlots * sizeof(PrItem); // [2] PrNotes
    static constexpr uint32_t BYTES = NOTE_OFF + 2 * (kPrMasked * 5 + 1) * 4;
};
// noted rows of an item's masked tiles
struct PrNotes {
    int32_t n;
    int32_t key0[kPrMasked];
    uint32_t rows[kPrMasked][4];
};

__device__ __forceinline__ uint32_t pr_pack(float lo, float hi)
{
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&v);
}

// Row tiles in the order of their key ranges, the longest first, for up to 32
// sequences (one a lane): CTAs that take every P-th of them then end at about
// the same time (five causal prompts of 700 to 2500 tokens, 16 heads of 64: the
// longest-running CTA had twice the shortest's work with the tiles in sequence
// order).
struct PrOrder {
    int32_t start, n;     // this lane's sequence: first row of q, length
    int32_t ctx, nq, nt;  // tokens before the chunk (>= 0), the chunk's, its row tiles
    int32_t reach;        // most keys of a tile by this measure, in kUnits
    static constexpr int kUnits = 64;
    // tiles of this lane's sequence with at least kUnits x keys up to their last
    // token (or the reach): the last ones.  (The quotient need not be exact, only
    // the same for the same x and never smaller for a larger one.)
    __device__ __forceinline__ int at_least(int32_t x, float inv) const
    {
        if (nt == 0 || x > min((ctx + nq) / kUnits, reach)) return 0;
        return nt - max(0, min(nt - 1, __float2int_ru((float)(x * kUnits - ctx) * inv) - 1));
    }
    // the tile of rank `rank`: its lane (-1: none), and its number in the sequence
    __device__ __forceinline__ int find(int rank, int TT, int lane, int &tile) const
    {
        if ((int)__reduce_add_sync(0xffffffffu, (unsigned)nt) <= rank) return -1;
        const float inv = 1.f / (float)TT;
        int32_t lo = -1, hi = reach + 1;  // count(lo) > rank >= count(hi)
        while (hi - lo > 1) {
            const int32_t mid = lo + (hi - lo) / 2;
            if ((int)__reduce_add_sync(0xffffffffu, (unsigned)at_least(mid, inv)) > rank)
                lo = mid;
            else
                hi = mid;
        }
        const int here = at_least(lo, inv), more = at_least(lo + 1, inv);
        const int j = rank - (int)__reduce_add_sync(0xffffffffu, (unsigned)more);  // among those with lo keys
        int incl = here - more;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += v;
        }
        const int l = __ffs((int)__ballot_sync(0xffffffffu, incl > j)) - 1;
        tile = __shfl_sync(0xffffffffu, nt - here + j - (incl - (here - more)), l);
        return l;
    }
};
__device__ __forceinline__ PrOrder pr_order(const PromptArgs &a, int TT, int lane)
{
    PrOrder o{};
    if (lane < a.S) {
        o.start = a.starts[lane];
        o.n = a.ctx_lens[lane];
        o.nq = max(0, a.starts[lane + 1] - o.start);
        o.nt = (o.nq + TT - 1) / TT;
        o.ctx = max(0, min(o.n, a.max_blocks * a.bs) - o.nq);
    }
    o.reach = (int32_t)__reduce_max_sync(0xffffffffu, (unsigned)(o.ctx + o.nq)) / PrOrder::kUnits;
    if (a.window > 0) o.reach = min(o.reach, a.window / PrOrder::kUnits + TT / PrOrder::kUnits);
    return o;
}

// Where the last item was found, of more sequences than PrOrder takes: items
// are asked for in ascending order, so that the search goes on from there.
struct PrCursor {
    int32_t s0 = 0, before = 0;  // sequences [s0, s0 + 32), row tiles of those before
};

// Item i (a converged warp); ntok = 0 where there is none.  `order`: the row
// tiles by their key ranges, or null: in sequence order.
__device__ __forceinline__ PrItem pr_item(const PromptArgs &a, int i, int TT, int lane, const PrOrder *order,
                                          PrCursor &cur)
{
    PrItem w{};
    w.ks = i % a.KS;
    i /= a.KS;
    w.g = i % a.Hkv;
    const int rank = i / a.Hkv;
    int tile = rank, st = 0, nq = 0;
    int32_t n = 0;
    if (order) {
        const int l = order->find(rank, TT, lane, tile);
        if (l < 0) return w;
        w.s = l;
        st = __shfl_sync(0xffffffffu, order->start, l);
        nq = __shfl_sync(0xffffffffu, order->nq, l);
        n = __shfl_sync(0xffffffffu, order->n, l);
    } else {
        int l = -1;
        for (; cur.s0 < a.S; cur.s0 += 32) {
            const int s = cur.s0 + lane;
            int first = 0, cnt = 0;
            if (s < a.S) {
                first = a.starts[s];
                cnt = max(0, a.starts[s + 1] - first);
            }
            const int nt = (cnt + TT - 1) / TT;
            int incl = nt;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, incl, off);
                if (lane >= off) incl += v;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, cur.before + incl > tile);
            if (hit) {
                l = __ffs((int)hit) - 1;
                tile -= cur.before + __shfl_sync(0xffffffffu, incl - nt, l);
                st = __shfl_sync(0xffffffffu, first, l);
                nq = __shfl_sync(0xffffffffu, cnt, l);
                w.s = cur.s0 + l;
                break;
            }
            cur.before += __shfl_sync(0xffffffffu, incl, 31);
        }
        if (l < 0) return w;
        n = a.ctx_lens[w.s];
    }
    const int i0 = tile * TT;  // its first token in the chunk
    w.row0 = st + i0;
    if (st < 0 || (int64_t)st + nq > a.T) {  // a bad array: nothing of it is touched
        report(a.err, KV_ERR_DEVICE_BOUNDS);
        return w;
    }
    // a chunk longer than the caller's bound: the last row tiles, of any sequence,
    // may have no items.  (Where some have none, a chunk with an item is longer:
    // were none, n_items would be enough.)
    if (nq > a.max_q) report(a.err, KV_ERR_DEVICE_BOUNDS);
    w.ntok = min(TT, nq - i0);
    const int32_t cap = a.max_blocks * a.bs;
    if (n < nq || n > cap) {
        report(a.err, KV_ERR_DEVICE_BOUNDS);
        n = n > cap ? cap : max(n, 0);
    }
    w.p0 = n - nq + i0;
    w.p1 = w.p0 + w.ntok - 1;
    if (w.p1 < 0) return w;
    w.lo = a.window > 0 ? max(0, w.p0 - a.window + 1) : 0;
    const int32_t sk = min(a.sinks, w.lo);  // sinks before the window
    w.head = (sk + kPrKeys - 1) / kPrKeys;
    w.gap = max(0, w.lo / kPrKeys - w.head);
    const int32_t all = w.p1 / kPrKeys + 1 - w.gap;
    w.t0 = (int32_t)((int64_t)w.ks * all / a.KS);
    w.nt = (int32_t)((int64_t)(w.ks + 1) * all / a.KS) - w.t0;
    return w;
}

// Pool row of token tok's K for KV head g, or -1 outside the pool.
__device__ __forceinline__ int32_t pr_pool_row(const PromptArgs &a, int s, int g, int32_t tok)
{
    const int32_t blk = tok / a.bs;
    const int32_t phys = a.table[(int64_t)s * a.max_blocks + blk];
    if (phys < 0 || (int64_t)phys + a.pages_per_block > a.pool_pages) return -1;
    return (int32_t)((int64_t)phys * a.rows_per_page + (int64_t)g * a.bs + (tok - blk * a.bs));
}

// wait_phase with its slow part out of the way
__device__ __forceinline__ void pr_wait(uint32_t bar, uint32_t parity, int32_t *err, bool &dead)
{
    if (__builtin_expect(!mbar_try_wait(bar, parity), 0)) wait_phase(bar, parity, err, dead);
}
// bits 0 .. n of a word (none for n < 0, all from 31 on)
__device__ __forceinline__ uint32_t pr_bits(int n) { return n < 0 ? 0u : 0xffffffffu >> (31 - min(n, 31)); }
// The columns that a row sees of 32 (column k is seen when k <= hi and not wl >=
// k >= sk), and its scores of the others to -inf.
__device__ __forceinline__ uint32_t pr_seen(int hi, int wl, int sk)
{
    return pr_bits(hi) & ~(pr_bits(wl) & ~pr_bits(sk - 1));
}
__device__ __forceinline__ void pr_mask(uint32_t (&x)[32], uint32_t seen)
{
#pragma unroll
    for (int k = 0; k < 32; ++k)
        if (!(seen >> k & 1u)) x[k] = 0xff800000u;
}
// and times -1 or 0, where the scale is negative or 0
__device__ __forceinline__ void pr_times(uint32_t (&x)[32], float f)
{
#pragma unroll
    for (int k = 0; k < 32; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * f);
}
// and their maximum, in four chains
__device__ __forceinline__ void pr_max(const uint32_t (&x)[32], float (&mx)[4])
{
#pragma unroll
    for (int k = 0; k < 32; k += 2)
        mx[(k >> 1) & 3] = fmaxf(fmaxf(mx[(k >> 1) & 3], __uint_as_float(x[k])), __uint_as_float(x[k + 1]));
}

// the weights of 32 scores as bf16 pairs, and their sums, in four chains (begun
// anew with `first`)
__device__ __forceinline__ void pr_weights(const uint32_t (&x)[32], uint32_t (&pw)[16], float2 (&r)[4], float scale,
                                           float m, bool first)
{
    const float2 sc = make_float2(scale, scale), nm = make_float2(-m, -m);
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        float2 y = __ffma2_rn(make_float2(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), sc, nm);
        y.x = fast_exp2(y.x);
        y.y = fast_exp2(y.y);
        pw[i / 2] = pr_pack(y.x, y.y);
        r[(i >> 1) & 3] = first && i < 8 ? y : __fadd2_rn(r[(i >> 1) & 3], y);
    }
}

template <int D>
__global__ void __launch_bounds__(kPrThreads, 1)
prompt_attn_kernel(const __grid_constant__ CUtensorMap tmap, const __grid_constant__ CUtensorMap qmap,
                   const __grid_constant__ CUtensorMap omap, const __grid_constant__ PromptArgs a)
{
    using L = PrSmem<D>;
    constexpr int HALVES = L::HALVES;
    using C = PrCols<D>;
    constexpr bool SEP = C::SEP;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t sbase = smem_u32(smem);
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + L::BAR_OFF);
    uint32_t *tslot = reinterpret_cast<uint32_t *>(smem + L::SLOT_OFF);
    PrItem *items = reinterpret_cast<PrItem *>(smem + L::ITEM_OFF);
    PrNotes *notes = reinterpret_cast<PrNotes *>(smem + L::NOTE_OFF);
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    // K and V of a stage loaded, free (V of a masked tile: loaded is V_RAW, and
    // FULL_V follows its check); per Q tile: S done, P of the first kPrFirst keys and of any others written, O done; an item's Q
    // loaded, used; an item published, read; its notes complete, read; per Q
    // tile (SEP): S read; all MMAs done
    constexpr int FULL_K = 0, EMPTY_K = 2, FULL_V = 4, EMPTY_V = 6, V_RAW = 8;
    constexpr int S_FULL = 10, P_FULL = 12, O_DONE = 16, Q_FULL = 18, Q_FREE = 19, NOTED = 20, NOTE_FREE = 22,
                  S_FREE = 24, ITEM_FULL = 26, ITEM_EMPTY = ITEM_FULL + kPrSlots, FIN = ITEM_EMPTY + kPrSlots;
    static_assert(kPrStages == 2 && kPrTiles == 2 && FIN < L::NBARS, "the barriers' numbers");

    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const int G = a.G, Hq = a.Hkv * G, TQ = kPrRows / G, TT = kPrTiles * TQ;
    constexpr int K_WARP = kPrSoft / 32, V_WARP = K_WARP + 1, MMA_WARP = K_WARP + 2, PLAN_WARP = K_WARP + 3;

    if (tid < L::NBARS) {
        int n = 1;
        if ((tid >= P_FULL && tid < O_DONE) || (tid >= S_FREE && tid < ITEM_FULL)) n = 128;
        if (tid >= NOTE_FREE && tid < S_FREE) n = kPrSoft / 32;
        if (tid >= ITEM_EMPTY && tid < FIN) n = kPrSoft / 32 + 3;
        mbar_init(bar(tid), n);
        fence_mbar_init();
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(tslot), kPrTmem);
        tmem_relinquish();
    }
    if (tid == 32) prefetch_tensormap(&tmap);
    if (tid == 64) prefetch_tensormap(&qmap);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tbase = *tslot;
    bool dead = false;
    grid_dependency_wait();
    grid_launch_dependents();

    // item k as the planning warp published it; each reading warp gives its slot
    // back at once
    auto item = [&](int k) {
        pr_wait(bar(ITEM_FULL + k % kPrSlots), (uint32_t)(k / kPrSlots) & 1u, a.err, dead);
        const PrItem w = items[k % kPrSlots];
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(ITEM_EMPTY + k % kPrSlots));
        return w;
    };

    if (warp >= K_WARP) {
        reg_dec<kPrRegsOther>();
        if (warp == PLAN_WARP) {
            // ---- the items' order, Q, and the check of V in masked tiles ----
            int turn = 0, pub = 0;   // rounds of items looked up, items published
            // (with an item a CTA the order is worth nothing)
            const bool sorted = a.S <= 32 && a.n_items > (int)gridDim.x;
            PrOrder order{};
            PrCursor cursor;
            if (sorted) order = pr_order(a, TT, lane);
            auto look_up = [&]() {   // the next item that has tokens, or the end
                PrItem w{};
                w.s = -1;
                const int P = gridDim.x, b = blockIdx.x;
                while ((int64_t)turn * P < a.n_items) {  // an item of each round of P, forwards and backwards in turn
                    const int64_t i = (int64_t)turn * P + (turn & 1 ? P - 1 - b : b);
                    ++turn;
                    if (i >= a.n_items) continue;
                    w = pr_item(a, (int)i, TT, lane, sorted ? &order : nullptr, cursor);
                    if (w.ntok > 0) break;
                    w.s = -1;
                }
                return w;
            };
            auto publish = [&](const PrItem &w) {
                const int sl = pub % kPrSlots;
                if (pub >= kPrSlots)
                    pr_wait(bar(ITEM_EMPTY + sl), (uint32_t)(pub / kPrSlots - 1) & 1u, a.err, dead);
                if (lane == 0) {
                    items[sl] = w;
                    mbar_arrive(bar(ITEM_FULL + sl));
                }
                __syncwarp();
                ++pub;
            };
            const uint64_t pol = l2_policy_evict_normal();
            // An item is published while the one before is worked on, and looked up
            // (3000 clocks and more) while the one before that is.
            PrItem w = look_up();
            publish(w);
            PrItem after{};
            bool have = false;  // `after` has been looked up
            int qn = 0, cnt = 0;        // items with Q loaded; tiles so far
            uint32_t vn = 0;            // parities: bit st, masked tiles of stage st so far
            for (int k = 0; w.s >= 0; ++k) {
                if (w.nt > 0) {
                    if (qn > 0) pr_wait(bar(Q_FREE), (uint32_t)(qn - 1) & 1u, a.err, dead);
                    if (lane == 0) {
                        const int nqt = (w.ntok + TQ - 1) / TQ;
                        mbar_arrive_expect_tx(bar(Q_FULL), (uint32_t)(nqt * HALVES * TQ * G * 128));
                        for (int t = 0; t < nqt; ++t)
                            for (int h = 0; h < HALVES; ++h)
                                tma_load_3d(sbase + t * L::Q_TILE + h * L::Q_HALF, &qmap, h * 64, w.g * G,
                                            w.row0 + t * TQ, bar(Q_FULL), pol);
                    }
                    __syncwarp();
                    ++qn;
                }
                PrItem next{};
                bool posted = false;
                auto post_next = [&]() {
                    if (posted) return;
                    if (!have) after = look_up();
                    next = after;
                    publish(next);
                    have = next.s < 0;  // nothing more to look up
                    posted = true;
                };
                if (have) post_next();
                // V of masked tiles: rows that no query sees are cleared, and so
                // are rows with a NaN or an infinity, which are noted
                PrNotes &nb = notes[k & 1];
                int n_masked = 0;
                if (k >= 2) pr_wait(bar(NOTE_FREE + (k & 1)), (uint32_t)((k >> 1) - 1) & 1u, a.err, dead);
                for (int t = 0; t < w.nt; ++t, ++cnt) {
                    const int k0 = w.key0(t), st = cnt % kPrStages;
                    if (!w.masked(a, k0)) {
                        if (!posted) {
                            post_next();
                        } else if (!have) {
                            after = look_up();
                            have = true;
                        }
                        continue;
                    }
                    pr_wait(bar(V_RAW + st), vn >> st & 1u, a.err, dead);
                    vn ^= 1u << st;
                    uint8_t *vt = smem + L::ST_OFF + st * L::STAGE + L::KV_TILE;
#pragma unroll 1
                    for (int q4 = 0; q4 < 4; ++q4) {
                        const int r = q4 * 32 + lane;
                        const bool any = w.sees(a, k0 + r, 1);
                        // x * 0 + acc: acc stays 0 while every value is finite
                        __nv_bfloat162 acc[2] = {__floats2bfloat162_rn(0.f, 0.f), __floats2bfloat162_rn(0.f, 0.f)};
                        const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
                        if (__any_sync(0xffffffffu, any)) {
#pragma unroll
                            for (int c = 0; c < D / 8; ++c) {
                                const uint4 x = *reinterpret_cast<const uint4 *>(vt + r * 128 + (c / 8) * L::KV_HALF +
                                                                                 ((c ^ r) & 7) * 16);
                                acc[0] = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&x.x), zero, acc[0]);
                                acc[1] = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&x.y), zero, acc[1]);
                                acc[0] = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&x.z), zero, acc[0]);
                                acc[1] = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&x.w), zero, acc[1]);
                            }
                        }
                        const bool odd = ((*reinterpret_cast<uint32_t *>(&acc[0]) | *reinterpret_cast<uint32_t *>(&acc[1])) &
                                          0x7fff7fffu) != 0;
                        if (!any || odd)
#pragma unroll
                            for (int c = 0; c < D / 8; ++c)  // (the order that spreads the lanes over the banks)
                                *reinterpret_cast<uint4 *>(vt + r * 128 + (c / 8) * L::KV_HALF + ((c ^ r) & 7) * 16) =
                                    make_uint4(0u, 0u, 0u, 0u);
                        __syncwarp();
                        const uint32_t bits = __ballot_sync(0xffffffffu, any && odd);
                        if (lane == 0) nb.rows[n_masked][q4] = bits;
                    }
                    if (lane == 0) nb.key0[n_masked] = k0;
                    ++n_masked;
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(FULL_V + st));
                    if (t > 0) post_next();  // (the first tile's check is waited for first)
                }
                post_next();
                if (lane == 0) {
                    nb.n = n_masked;
                    mbar_arrive(bar(NOTED + (k & 1)));
                }
                __syncwarp();
                w = next;
            }
        } else if (warp != MMA_WARP) {
            // ---- TMA producer warps, one of K and one of V: one box per lane ----
            const bool is_v = warp == V_WARP;
            const uint64_t pol = l2_policy_evict_normal();
            constexpr int NBOX = kPrKeys / kTile * HALVES;
            const int full0 = is_v ? FULL_V : FULL_K, empty0 = is_v ? EMPTY_V : EMPTY_K;
            const int j = lane / HALVES, h = lane % HALVES;
            int cnt = 0;
            for (int k = 0;; ++k) {
                const PrItem w = item(k);
                if (w.s < 0) break;
                // pool row of this lane's box of tile t: -1 outside the pool, -2 not wanted
                auto box_row = [&](int t) {
                    if (lane >= NBOX || t >= w.nt) return -2;
                    const int32_t tok = w.key0(t) + j * kTile;
                    if (!w.sees(a, tok, kTile)) return -2;
                    const int32_t y = pr_pool_row(a, w.s, w.g, tok);
                    return y < 0 ? -1 : y + (is_v ? a.Hkv * a.bs : 0);
                };
                int32_t y = box_row(0);
                for (int t = 0; t < w.nt; ++t, ++cnt) {
                    const int st = cnt % kPrStages;
                    const int32_t y_next = box_row(t + 1);
                    const bool bad = __any_sync(0xffffffffu, y == -1);
                    const uint32_t n = __popc(__ballot_sync(0xffffffffu, y >= 0));
                    const uint32_t full = bar(is_v && w.masked(a, w.key0(t)) ? V_RAW + st : full0 + st);
                    if (cnt >= kPrStages)
                        pr_wait(bar(empty0 + st), (uint32_t)(cnt / kPrStages - 1) & 1u, a.err, dead);
                    if (lane == 0) {
                        if (bad || n == 0) {
                            if (bad) report(a.err, KV_ERR_DEVICE_BOUNDS);
                            mbar_arrive(full);  // complete the phase without data
                        } else {
                            mbar_arrive_expect_tx(full, n * kHalfBytes);
                        }
                    }
                    __syncwarp();
                    if (!bad && y >= 0)
                        tma_load_2d(sbase + L::ST_OFF + st * L::STAGE + (is_v ? L::KV_TILE : 0) + h * L::KV_HALF +
                                        j * (kTile * 128),
                                    &tmap, h * 64, y, full, pol);
                    __syncwarp();
                    y = y_next;
                }
            }
            // drain: the last stages' loads have landed
            if (lane == 0)
                for (int c = max(0, cnt - kPrStages); c < cnt; ++c)
                    pr_wait(bar(full0 + c % kPrStages), (uint32_t)(c / kPrStages) & 1u, a.err, dead);
        } else {
            // ---- MMA issuer: S_0(0) S_1(0) | PV_0(t) S_0(t+1) PV_1(t) S_1(t+1) | ... (SEP:
            // S_0(t+1) S_1(t+1) PV_0(t) PV_1(t)); the pipe runs one thread's MMAs in issue order, so S_a(t+1), or S_a(0) of
            // the next item, overwrites P only after PV_a(t) has read it.  O is
            // overwritten by PV_a(0) of the next item once its P is there, which
            // the softmax warps write after they have read O ----
            const uint32_t el = elect_one();
            constexpr uint32_t ID_S = idesc_bf16_f32(kPrRows, kPrKeys, 0, 0);
            constexpr uint32_t ID_O = idesc_bf16_f32(kPrRows, D, 0, 1);
            int cnt = 0, qn = 0;           // tiles, items with Q so far
            uint32_t pn = 0;               // parities: bit q, tiles of Q tile q so far
            uint32_t sn = 0, used = 0;     // (SEP) waits on S_FREE so far; S written before
            auto issue_s = [&](int q, int c) {
                const uint32_t ka = sbase + L::ST_OFF + (c % kPrStages) * L::STAGE;
                const uint32_t qa = sbase + q * L::Q_TILE;
                // (rolled: three copies of it are less in the instruction caches, 121 ->
                // 115 us for 6 sequences of 80 / 16 heads and a window of 68; P.V,
                // which the next S waits for, is not: 147 -> 165 for 8192 causal
                // tokens of 16 heads of 64)
#pragma unroll 1
                for (int kk = 0; kk < D / 16; ++kk)
                    umma_bf16(tbase + C::s(q), smem_desc_sw128(qa + (kk / 4) * L::Q_HALF + (kk % 4) * 32, 16, 1024),
                              smem_desc_sw128(ka + (kk / 4) * L::KV_HALF + (kk % 4) * 32, 16, 1024), ID_S, kk > 0, el);
                umma_commit(bar(S_FULL + q), el);
            };
            auto issue_pv = [&](int q, int c, int half, bool more) {
                const uint32_t va = sbase + L::ST_OFF + (c % kPrStages) * L::STAGE + L::KV_TILE;
                constexpr int STEPS = kPrKeys / 16, FIRST = kPrFirst<D> / 16;
#pragma unroll
                for (int kk = half ? FIRST : 0; kk < (half ? STEPS : FIRST); ++kk) {
                    umma_bf16_tmem_a(tbase + C::o(q), tbase + C::p(q) + kk * 8,
                                     smem_desc_sw128(va + kk * (16 * 128), L::KV_HALF, 1024), ID_O, more || kk > 0, el);
                }
            };
            auto wait_k = [&](int c) {
                pr_wait(bar(FULL_K + c % kPrStages), (uint32_t)(c / kPrStages) & 1u, a.err, dead);
            };
            for (int k = 0;; ++k) {
                const PrItem w = item(k);
                if (w.s < 0) break;
                if (w.nt == 0) continue;
                const int nqt = (w.ntok + TQ - 1) / TQ;
                pr_wait(bar(Q_FULL), (uint32_t)qn & 1u, a.err, dead);
                ++qn;
                wait_k(cnt);
                // S of tile c for Q tile q; with SEP once the softmax has read the one before
                auto next_s = [&](int q, int c) {
                    if (SEP) {
                        if (used >> q & 1u) {
                            pr_wait(bar(S_FREE + q), sn >> q & 1u, a.err, dead);
                            sn ^= 1u << q;
                        }
                        used |= 1u << q;
                    }
                    tc_fence_after();
                    issue_s(q, c);
                };
                for (int q = 0; q < nqt; ++q) next_s(q, cnt);
                umma_commit(bar(EMPTY_K + cnt % kPrStages), el);
                if (w.nt == 1) umma_commit(bar(Q_FREE), el);
                for (int t = 0; t < w.nt; ++t, ++cnt) {
                    const int st = cnt % kPrStages;
                    const bool next = t + 1 < w.nt;
                    auto k_used = [&]() {  // K of tile cnt + 1, and Q after its last tile
                        umma_commit(bar(EMPTY_K + (cnt + 1) % kPrStages), el);
                        if (t + 2 == w.nt) umma_commit(bar(Q_FREE), el);
                    };
                    if (SEP && next) {
                        wait_k(cnt + 1);
                        for (int q = 0; q < nqt; ++q) next_s(q, cnt + 1);
                        k_used();
                    }
                    pr_wait(bar(FULL_V + st), (uint32_t)(cnt / kPrStages) & 1u, a.err, dead);
                    for (int q = 0; q < nqt; ++q) {
                        pr_wait(bar(P_FULL + 2 * q), pn >> q & 1u, a.err, dead);
                        tc_fence_after();
                        issue_pv(q, cnt, 0, t > 0);
                        if (kPrFirst<D> < kPrKeys) {
                            pr_wait(bar(P_FULL + 2 * q + 1), pn >> q & 1u, a.err, dead);
                            tc_fence_after();
                            issue_pv(q, cnt, 1, true);
                        }
                        pn ^= 1u << q;
                        if (SEP || !next) umma_commit(bar(O_DONE + q), el);
                        if (q == nqt - 1) umma_commit(bar(EMPTY_V + st), el);
                        if (!SEP && next) {
                            if (q == 0) wait_k(cnt + 1);
                            next_s(q, cnt + 1);
                            if (q == nqt - 1) k_used();
                        }
                    }
                }
            }
            // every MMA has completed before TMEM is released
            umma_commit(bar(FIN), el);
            pr_wait(bar(FIN), 0u, a.err, dead);
        }
    } else {
        // ---- softmax: thread r of Q tile qa owns its row r ----
        reg_inc<kPrRegsSoft>();
        const int qa = tid / kPrRows, r = tid % kPrRows;
        const int itok = qa * TQ + r / G, hrow = r % G;  // the row's token in the item, its head in the group
        const uint32_t trow = tbase + ((uint32_t)((warp % 4) * 32) << 16);
        const uint32_t ts = trow + C::s(qa), tp = trow + C::p(qa), to = trow + C::o(qa);
        const float scale = a.qk_scale;
        uint8_t *xb = smem + L::X_OFF + warp * 4096;
        int pn = 0, on = 0;  // tiles of this Q tile, waits on O_DONE so far
        for (int k = 0;; ++k) {
            // read where needed: its fields and a row's scores together are more
            // than the registers
            const PrItem &w = items[k % kPrSlots];
            pr_wait(bar(ITEM_FULL + k % kPrSlots), (uint32_t)(k / kPrSlots) & 1u, a.err, dead);
            if (w.s < 0) break;
            auto give_back = [&]() {  // the item and its notes
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(bar(NOTE_FREE + (k & 1)));
                    mbar_arrive(bar(ITEM_EMPTY + k % kPrSlots));
                }
            };
            if (qa * TQ >= w.ntok) {  // no tokens in this Q tile
                pr_wait(bar(NOTED + (k & 1)), (uint32_t)(k >> 1) & 1u, a.err, dead);
                give_back();
                continue;
            }
            float m_run = kMaxStart, l_run = 0.f;
            // tile t: whether it is masked; this row sees its columns [.., hi], of
            // which from the window's edge on or below sk
            bool mk;
            int hi, sk;
            auto tile_of = [&](int t) {
                const int k0 = w.key0(t);
                mk = w.masked(a, k0) | (a.sign != 1.f);
                hi = w.p0 + itok - k0;
                sk = a.sinks - k0;
            };
            tile_of(0);
            for (int t = 0; t < w.nt; ++t, ++pn) {
                pr_wait(bar(S_FULL + qa), (uint32_t)pn & 1u, a.err, dead);
                __syncwarp();
                tc_fence_after();
                // A masked tile: its scores masked in TMEM, 32 columns at a time, and
                // read like any other's.  Rolled, because what runs now and then is
                // rarely in the instruction caches: with the masks unrolled over the
                // 128 scores a tile took 700 clocks more, and skipping the weights of
                // unseen columns in a second copy of that code cost more than it
                // saved (6 sequences of 64 / 16 heads, window 68: 96 us unrolled, 111
                // with the copy, 93 so).
                if (__builtin_expect(mk, 0)) {
                    const int wl = a.window > 0 ? hi - a.window : -1;
#pragma unroll 1
                    for (int c = 0; c < 128; c += 32) {
                        const uint32_t seen = pr_seen(hi - c, wl - c, sk - c);
                        if (a.sign == 1.f && __all_sync(0xffffffffu, seen == 0xffffffffu)) continue;
                        uint32_t x[32];
                        tmem_ld32(ts + c, x);
                        tmem_wait_ld();
                        if (a.sign != 1.f) pr_times(x, a.sign);
                        pr_mask(x, seen);
                        tmem_st32(ts + c, x);
                    }
                    tmem_wait_st();
                }
                uint32_t v[4][32];  // the row's scores
                tmem_ld32(ts, v[0]);
                tmem_ld32(ts + 32, v[1]);
                tmem_ld32(ts + 64, v[2]);
                tmem_ld32(ts + 96, v[3]);
                tmem_wait_ld();
                if (SEP) {
                    tc_fence_before();
                    mbar_arrive(bar(S_FREE + qa));
                }
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < 4; ++c) pr_max(v[c], mx);
                if (SEP && t > 0) {  // the tile before: its P read, its O there
                    pr_wait(bar(O_DONE + qa), (uint32_t)on++ & 1u, a.err, dead);
                    __syncwarp();
                    tc_fence_after();
                }
                const float cmax = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
                // The reference m_run moves only when a tile exceeds it by 2^8 (o and l
                // share it, so the ratio is exact).  A warp's lanes read and write
                // TMEM together: all rows of a warp are scaled when one of them asks
                // for it, the others by 1
                const bool rise = cmax > m_run + 8.f;
                if (__builtin_expect(__any_sync(0xffffffffu, rise), 0)) {
                    const float al = rise ? fast_exp2(m_run - cmax) : 1.f;  // 0 when nothing came before
                    l_run *= al;
                    if (t >= 1) {
                        uint32_t o[16];
#pragma unroll 1
                        for (int cb = 0; cb < D / 16; ++cb) {
                            tmem_ld16(to + cb * 16, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * al);
                            tmem_st16(to + cb * 16, o);
                        }
                    }
                    if (rise) m_run = cmax;
                    __syncwarp();
                }
                // p = 2^(s * scale - m_run), as bf16 pairs over the first columns of S,
                // handed over in two parts
                uint32_t pw[2][16];
                float2 r2[4];
                pr_weights(v[0], pw[0], r2, scale, m_run, true);
                tmem_st16(tp, pw[0]);
                pr_weights(v[1], pw[1], r2, scale, m_run, false);
                tmem_st16(tp + 16, pw[1]);
                tile_of(t + 1);  // (the loads it needs, before they are waited for)
                pr_weights(v[2], pw[0], r2, scale, m_run, false);
                tmem_st16(tp + 32, pw[0]);
                if (kPrFirst<D> == 96) {
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(bar(P_FULL + 2 * qa));
                }
                pr_weights(v[3], pw[1], r2, scale, m_run, false);
                tmem_st16(tp + 48, pw[1]);
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(bar(P_FULL + 2 * qa + (kPrFirst<D> == 96 ? 1 : 0)));
                const float2 r1 = __fadd2_rn(__fadd2_rn(r2[0], r2[1]), __fadd2_rn(r2[2], r2[3]));
                l_run += r1.x + r1.y;
            }
            // ---- the rows' outputs, or this split's records (rolled: it runs once an item) ----
            if (w.nt > 0) pr_wait(bar(O_DONE + qa), (uint32_t)on++ & 1u, a.err, dead);
            pr_wait(bar(NOTED + (k & 1)), (uint32_t)(k >> 1) & 1u, a.err, dead);
            __syncwarp();
            tc_fence_after();
            const bool row_ok = r < TQ * G && itok < w.ntok;
            const int64_t qrow_off = ((int64_t)(w.row0 + itok) * Hq + w.g * G + hrow) * D;
            const int p = w.p0 + itok, nt = w.nt;  // this row's position; the item's tiles
            const PrNotes &nb = notes[k & 1];
            const int n_notes = nb.n * 4;
            bool any_note = false;
            for (int b = lane; b < n_notes; b += 32) any_note |= nb.rows[b / 4][b % 4] != 0;
            if (__any_sync(0xffffffffu, any_note)) {
                // noted tokens that this row sees: added to O in TMEM
#pragma unroll 1
                for (int cb = 0; cb < D / 32; ++cb) {
                    uint32_t o[32];
                    tmem_ld32(to + cb * 32, o);
                    tmem_wait_ld();
#pragma unroll 1
                    for (int b = 0; b < n_notes; ++b)
                        for (uint32_t bits = nb.rows[b / 4][b % 4]; bits; bits &= bits - 1) {
                            const int tok = nb.key0[b / 4] + b % 4 * 32 + __ffs((int)bits) - 1;
                            if (!row_ok || tok > p || (a.window > 0 && tok <= p - a.window && tok >= a.sinks)) continue;
                            const int32_t y = pr_pool_row(a, w.s, w.g, tok);
                            if (y < 0) continue;
                            const uint16_t *kr = a.pool + (int64_t)y * D, *vr = kr + (int64_t)a.Hkv * a.bs * D;
                            float s = 0.f;
#pragma unroll 1
                            for (int e = 0; e < D; ++e) s = fmaf(bf_lo(a.q[qrow_off + e]), bf_lo(kr[e]), s);
                            const float pj = fast_exp2(fmaf(s * a.sign, scale, -m_run));
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                o[i] = __float_as_uint(fmaf(pj, bf_lo(vr[cb * 32 + i]), __uint_as_float(o[i])));
                        }
                    __syncwarp();
                    tmem_st32(to + cb * 32, o);
                    tmem_wait_st();
                }
            }
            const bool blind = p < 0;  // the row sees nothing: zeros
            const float inv = blind || nt == 0 ? 0.f : 1.f / l_run;
            const bool rec = a.KS > 1;
            const int64_t rec_row = ((int64_t)w.ks * a.T + w.row0 + itok) * Hq + w.g * G + hrow;
            const unsigned long long orow =
                !row_ok || dead ? 0ull
                                : rec ? reinterpret_cast<unsigned long long>(a.ws + rec_row * D)
                                      : reinterpret_cast<unsigned long long>(a.out + qrow_off);
            const int g_out = w.g * G, tok_out = w.row0 + itok + (rec ? w.ks * a.T : 0);  // (of lane 0: the box's corner)
            give_back();
            // 128 bytes of each row through shared memory.  A warp whose 32 rows are
            // whole tokens of the chunk sends them as one TMA box; otherwise eight
            // lanes write 128 consecutive bytes.
            const bool box = 32 % G == 0 && __all_sync(0xffffffffu, orow != 0ull);
            auto send = [&](int part, const uint4 (&x)[8]) {
                if (lane == 0) bulk_wait_read();  // a box before has been read
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    *reinterpret_cast<uint4 *>(xb + lane * 128 + ((i ^ (lane & 7)) * 16)) = x[i];
                if (box) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_3d(&omap, smem_u32(xb), part * (rec ? 32 : 64), g_out, tok_out);
                        bulk_commit();
                    }
                    return;
                }
                __syncwarp();
                // (all loads first: the compiler cannot know that the stores go elsewhere)
                uint4 y[8];
                unsigned long long dst[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int rr = i * 4 + lane / 8;
                    y[i] = *reinterpret_cast<const uint4 *>(xb + rr * 128 + ((lane % 8) ^ (rr & 7)) * 16);
                    dst[i] = __shfl_sync(0xffffffffu, orow, rr);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (dst[i]) *reinterpret_cast<uint4 *>(dst[i] + part * 128 + lane % 8 * 16) = y[i];
                __syncwarp();
            };
            if (rec) {
#pragma unroll 1
                for (int cb = 0; cb < D / 32 && nt > 0; ++cb) {
                    uint32_t o[32];
                    tmem_ld32(to + cb * 32, o);
                    tmem_wait_ld();
                    uint4 x[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                    send(cb, x);
                }
                if (orow)
                    reinterpret_cast<float2 *>(a.ws + (int64_t)a.KS * a.T * Hq * D)[rec_row] =
                        make_float2(blind || nt == 0 ? -INFINITY : m_run, l_run);
            } else {
#pragma unroll 1
                for (int cb = 0; cb < D / 64; ++cb) {
                    uint32_t o[2][32] = {};
                    if (nt > 0) {
                        tmem_ld32(to + cb * 64, o[0]);
                        tmem_ld32(to + cb * 64 + 32, o[1]);
                        tmem_wait_ld();
                    }
                    uint4 x[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        uint32_t y[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int c = 8 * (i % 4) + 2 * e;
                            y[e] = pr_pack(__uint_as_float(o[i / 4][c]) * inv, __uint_as_float(o[i / 4][c + 1]) * inv);
                        }
                        x[i] = blind ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(y[0], y[1], y[2], y[3]);
                    }
                    send(cb, x);
                }
            }
            tc_fence_before();  // O has been read: the next item's P may let it be overwritten
        }
        if (lane == 0) bulk_wait_all();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_dealloc(tbase, kPrTmem);
}

// Merge of the KS records of each (row, query head): a warp each, D / 32
// columns a lane.  The records' maxima and sums first, a record a lane, then
// their outputs with the weights known, so that no load waits for another (16
// records one after another: 20 us for 512 rows).  A row without records (no
// split saw anything) is zero.
template <int D>
__global__ void __launch_bounds__(256) prompt_merge_kernel(const float *ws, uint16_t *out, int64_t n_rows, int KS)
{
    grid_dependency_wait();
    grid_launch_dependents();
    constexpr int C = D / 32;
    static_assert(kPrMaxSplits <= 32, "a record a lane");
    const int64_t i = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    const int lane = threadIdx.x & 31;
    if (i >= n_rows) return;
    const int64_t next = n_rows * D;
    const float *rec = ws + i * D;
    const float2 ml = lane < KS ? reinterpret_cast<const float2 *>(ws + KS * next)[lane * n_rows + i]
                                : make_float2(-INFINITY, 0.f);
    const float m = ml.x, l = ml.y;
    float M = m;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
    const float wgt = m == -INFINITY ? 0.f : fast_exp2(m - M);
    float L = m == -INFINITY ? 0.f : wgt * l;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) L += __shfl_xor_sync(0xffffffffu, L, off);
    const unsigned there = __ballot_sync(0xffffffffu, m != -INFINITY);
    float O[C] = {};
#pragma unroll 8
    for (int k = 0; k < KS; ++k) {
        const float w = __shfl_sync(0xffffffffu, wgt, k);
        if (!(there >> k & 1u)) continue;
        const float *o = rec + k * next + lane * C;
        if constexpr (C == 4) {
            const float4 x = *reinterpret_cast<const float4 *>(o);
            O[0] = fmaf(x.x, w, O[0]);
            O[1] = fmaf(x.y, w, O[1]);
            O[2] = fmaf(x.z, w, O[2]);
            O[3] = fmaf(x.w, w, O[3]);
        } else {
            const float2 x = *reinterpret_cast<const float2 *>(o);
            O[0] = fmaf(x.x, w, O[0]);
            O[1] = fmaf(x.y, w, O[1]);
        }
    }
    const float inv = there ? 1.f / L : 0.f;
    uint32_t y[C / 2];
#pragma unroll
    for (int c = 0; c < C / 2; ++c) y[c] = pr_pack(O[2 * c] * inv, O[2 * c + 1] * inv);
    uint32_t *dst = reinterpret_cast<uint32_t *>(out + i * D + lane * C);
    if constexpr (C == 4)
        *reinterpret_cast<uint2 *>(dst) = make_uint2(y[0], y[1]);
    else
        *dst = y[0];
}

template <int D>
inline size_t prompt_smem_bytes() { return 1024 + (size_t)PrSmem<D>::BYTES; }

}  // namespace kvp
