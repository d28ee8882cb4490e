// pages.cu -- copies of cache pages on the device, and the calls on sequence
// tables that need them: forks whose partial last block becomes each fork's
// own (kv_seq_fork), and live blocks moved together so that whole superpages
// and chunks are free for kv_pool_trim (kv_pool_compact).
//
// The copy is bound by HBM: a block's rows are read and written once.  4000
// blocks of 64 KB (524 MB read and written, three launches) take 82.5 us, 6.35
// TB/s; 48 partial ones 7.8 us, the call's own time on the host.  A block is
// several CTAs' work (gridDim.y), each thread with four 16-byte loads in flight.
// The (source, destination, tokens) triples travel as kernel parameters, like a
// table sync's words, so the caller's arrays may change right after the call.
#include <algorithm>
#include <mutex>
#include <new>
#include <vector>

#include <cuda_runtime.h>

#include "pages_internal.h"
#include "pool_internal.h"
#include "q4_format.h"
#include "ptx.cuh"
#include "seqtab_internal.h"
#include "stream_order.h"

namespace {

constexpr int kCopyThreads = 256;
constexpr int kCopyBatch = 4;  // 16-byte loads in flight per thread

template <int N>
struct CopyParams {
    uint8_t *pool;
    int64_t page_bytes;
    int64_t seg_stride;  // bytes of one KV head's K (or V) in a block
    int32_t row_bytes;
    int32_t segs;        // 2 * Hkv
    int32_t bs;
    int32_t at[N][3];    // source page, destination page, tokens
};

// gridDim.x pairs, gridDim.y CTAs each.
template <int N>
__global__ void __launch_bounds__(kCopyThreads) copy_blocks_kernel(const __grid_constant__ CopyParams<N> p)
{
    kvp::grid_dependency_wait();
    kvp::grid_launch_dependents();
    const int32_t *at = p.at[blockIdx.x];
    const uint8_t *src = p.pool + (int64_t)at[0] * p.page_bytes;
    uint8_t *dst = p.pool + (int64_t)at[1] * p.page_bytes;
    // a block copied whole is one run of bytes; else the first rows of each
    // head's K and V are
    const bool whole = at[2] == p.bs;
    const int segs = whole ? 1 : p.segs;
    const int per = (int)((whole ? p.segs * p.seg_stride : (int64_t)at[2] * p.row_bytes) / 16);  // chunks of a run
    const int total = segs * per;
    const int stride = gridDim.y * kCopyThreads;
    for (int i0 = blockIdx.y * kCopyThreads + threadIdx.x; i0 < total; i0 += stride * kCopyBatch) {
        uint4 w[kCopyBatch];
        int64_t off[kCopyBatch];
#pragma unroll
        for (int b = 0; b < kCopyBatch; ++b) {
            const int i = i0 + b * stride;
            if (i < total) {
                const int seg = whole ? 0 : i / per;
                off[b] = seg * p.seg_stride + (int64_t)(i - seg * per) * 16;
                w[b] = *reinterpret_cast<const uint4 *>(src + off[b]);
            }
        }
#pragma unroll
        for (int b = 0; b < kCopyBatch; ++b)
            if (i0 + b * stride < total) *reinterpret_cast<uint4 *>(dst + off[b]) = w[b];
    }
}

// one launch of n pairs (n <= N)
template <int N>
int copy_launch(const kv_pool *p, int layout, int n, const int32_t *src, const int32_t *dst, const int32_t *tokens,
                cudaStream_t st)
{
    const kv_layout &L = p->desc.layouts[layout];
    CopyParams<N> c;
    c.pool = reinterpret_cast<uint8_t *>(p->desc.device_base);
    c.page_bytes = (int64_t)p->page_bytes;
    c.row_bytes = 2 * L.head_dim;
    c.seg_stride = (int64_t)p->desc.block_size * c.row_bytes;
    c.segs = 2 * L.num_kv_heads;
    if (kvp_is_q4(L)) {  // copied whole, or (no tokens) not at all
        c.row_bytes = 0;
        c.seg_stride = (int64_t)p->block_bytes[layout];
        c.segs = 1;
    }
    c.bs = p->desc.block_size;
    for (int i = 0; i < n; ++i) {
        c.at[i][0] = src[i];
        c.at[i][1] = dst[i];
        c.at[i][2] = tokens ? tokens[i] : c.bs;
    }
    const int64_t chunks = (int64_t)c.segs * c.seg_stride / 16;
    const int64_t per_cta = (int64_t)kCopyThreads * kCopyBatch;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)n, (unsigned)std::min<int64_t>((chunks + per_cta - 1) / per_cta, 64));
    cfg.blockDim = dim3(kCopyThreads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, copy_blocks_kernel<N>, c) != cudaSuccess) return KV_ERR_CUDA;
    kvp_note_stream(st, false);
    return KV_OK;
}

// parameter blocks of three sizes: a launch's cost grows with its bytes
constexpr int kCopySmall = 80;   // 1 KB
constexpr int kCopyMid = 336;    // 4 KB
constexpr int kCopyLarge = 1360;  // 16 KB

}  // namespace

int kvp_copy_pages(const kv_pool *p, int layout, int n, const int32_t *src, const int32_t *dst, const int32_t *tokens,
                   void *stream)
{
    cudaStream_t st = (cudaStream_t)stream;
    for (int i = 0; i < n;) {
        const int m = std::min(n - i, kCopyLarge);
        const int32_t *tk = tokens ? tokens + i : nullptr;
        const int rc = m <= kCopySmall ? copy_launch<kCopySmall>(p, layout, m, src + i, dst + i, tk, st)
                       : m <= kCopyMid ? copy_launch<kCopyMid>(p, layout, m, src + i, dst + i, tk, st)
                                       : copy_launch<kCopyLarge>(p, layout, m, src + i, dst + i, tk, st);
        if (rc) return rc;
        i += m;
    }
    return KV_OK;
}

extern "C" {

int kv_copy_blocks(kv_pool *p, int layout, int n, const int32_t *src, const int32_t *dst, const int32_t *tokens,
                   void *stream)
{
    if (!p || layout < 0 || layout >= p->desc.num_layouts || n < 0) return KV_ERR_INVALID_ARG;
    if (n == 0) return KV_OK;
    if (!src || !dst) return KV_ERR_INVALID_ARG;
    if (tokens && kvp_is_q4(p->desc.layouts[layout]))
        for (int i = 0; i < n; ++i)
            if (tokens[i] > 0 && tokens[i] < p->desc.block_size) return KV_ERR_UNSUPPORTED;
    {
        // every id a live block; no destination twice, none that is also a
        // source: the copies run side by side.  Marks go to the pool's tally,
        // which is all zeros between calls.
        std::lock_guard<std::mutex> g(p->mu);
        bool ok = true;
        int marked = 0;
        for (int i = 0; i < n && ok; ++i) {
            for (const int32_t id : {src[i], dst[i]})
                ok = ok && id >= 0 && id < p->n_pages && p->owner[(size_t)id] == layout && p->refcnt[(size_t)id] > 0;
            ok = ok && (!tokens || (tokens[i] >= 0 && tokens[i] <= p->desc.block_size));
        }
        for (; ok && marked < n; ++marked) {
            if (p->tally[(size_t)dst[marked]]) {
                ok = false;
                break;
            }
            p->tally[(size_t)dst[marked]] = 1;
        }
        for (int i = 0; i < n && ok; ++i) ok = p->tally[(size_t)src[i]] == 0;
        for (int i = 0; i < marked; ++i) p->tally[(size_t)dst[i]] = 0;
        if (!ok) return KV_ERR_INVALID_ARG;
    }
    return kvp_copy_pages(p, layout, n, src, dst, tokens, stream);
}

int kv_seq_fork(kv_seqtab *t, int src, int n, const int32_t *dsts, void *stream)
{
    if (!t || !t->pool || src < 0 || src >= t->S || n < 0 || (n > 0 && !dsts)) return KV_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i) {
        const int32_t d = dsts[i];
        if (d < 0 || d >= t->S || d == src) return KV_ERR_INVALID_ARG;
        if (t->held[(size_t)d] != 0 || t->lens[(size_t)d] != 0) return KV_ERR_INVALID_ARG;
    }
    if (n == 0) return KV_OK;
    const int32_t len = t->lens[(size_t)src];
    const int full = len / t->bs, tail = len % t->bs;
    const int32_t *row = &t->table[(size_t)src * t->max_blocks];
    if (tail > 0 && row[full] < 0) return KV_ERR_INVALID_ARG;  // the last token's page was given up
    if (tail > 0 && kvp_is_q4(t->pool->desc.layouts[t->layout])) return KV_ERR_UNSUPPORTED;
    try {
        std::vector<int32_t> seen(dsts, dsts + n), shared, own((size_t)n), from((size_t)n), rows((size_t)n);
        std::sort(seen.begin(), seen.end());
        if (std::adjacent_find(seen.begin(), seen.end()) != seen.end()) return KV_ERR_INVALID_ARG;
        for (int i = 0; i < full; ++i)
            if (row[i] >= 0) shared.push_back(row[i]);
        int rc = KV_OK;
        if (tail > 0) {
            rc = kv_alloc_blocks(t->pool, t->layout, n, own.data());
            if (rc) return rc;
        }
        int refs = 0;
        for (; refs < n && !rc; ++refs) {
            rc = kv_block_ref(t->pool, t->layout, (int)shared.size(), shared.data());
            if (rc) break;
        }
        if (!rc && tail > 0) {
            std::fill(from.begin(), from.end(), row[full]);
            std::fill(rows.begin(), rows.end(), tail);
            rc = kvp_copy_pages(t->pool, t->layout, n, from.data(), own.data(), rows.data(), stream);
        }
        if (rc) {  // as before the call
            for (int i = 0; i < refs; ++i) kv_free_blocks(t->pool, t->layout, (int)shared.size(), shared.data());
            if (tail > 0) kv_free_blocks(t->pool, t->layout, n, own.data());
            return rc;
        }
        for (int i = 0; i < n; ++i) {
            const int32_t d = dsts[i];
            for (int b = 0; b < full; ++b)
                if (row[b] >= 0) kvp_seqtab_set_entry(t, d, b, row[b]);
            if (tail > 0) kvp_seqtab_set_entry(t, d, full, own[(size_t)i]);
            t->held[(size_t)d] = full + (tail > 0 ? 1 : 0);
            t->lens[(size_t)d] = len;
            t->counters.blocks_held += (int64_t)shared.size() + (tail > 0 ? 1 : 0);
        }
    } catch (const std::bad_alloc &) {
        return KV_ERR_OUT_OF_BLOCKS;
    }
    return KV_OK;
}

int kv_pool_compact(kv_pool *p, int max_moves, void *stream, int *n_moves)
{
    if (!p || max_moves < 0) return KV_ERR_INVALID_ARG;
    if (n_moves) *n_moves = 0;
    try {
        std::lock_guard<std::mutex> g(p->mu);
        const int nl = p->desc.num_layouts;
        // what kv_pool_trim gives back at once: a chunk of a VMM pool, else a superpage
        const int64_t region = (int64_t)p->super_pages * (p->vmm.active ? p->vmm.supers_per_chunk : 1);
        const size_t n_regions = (size_t)((p->n_pages + region - 1) / region);
        // a block can move when every reference to it is an entry of an open table
        std::vector<int32_t> refs((size_t)p->n_pages, 0);
        for (const kv_seqtab *t : p->seqtabs)
            for (int s = 0; s < t->S; ++s)
                for (int i = 0; i < t->held[(size_t)s]; ++i) {
                    const int32_t id = t->table[(size_t)s * t->max_blocks + i];
                    if (id >= 0 && id < p->n_pages) ++refs[(size_t)id];
                }
        struct Region {
            int64_t live = 0;  // pages
            bool fixed = false;
            std::vector<int32_t> blocks;
        };
        std::vector<Region> R(n_regions);
        for (int64_t id = 0; id < p->n_pages; ++id) {
            if (p->refcnt[(size_t)id] <= 0) continue;
            Region &r = R[(size_t)(id / region)];
            r.live += p->pages_per_block[p->owner[(size_t)id]];
            r.fixed |= refs[(size_t)id] != p->refcnt[(size_t)id];
            r.blocks.push_back((int32_t)id);
        }
        // room: free blocks of each layout per region, already cut from superpages,
        // and (in a chunk) free superpages that can be
        std::vector<std::vector<int32_t>> room[KV_MAX_LAYOUTS], supers(n_regions);
        for (int l = 0; l < nl; ++l) {
            room[l].resize(n_regions);
            for (int32_t id : p->free_blocks[l]) room[l][(size_t)(id / region)].push_back(id);
        }
        for (int32_t sp : p->super_free) supers[(size_t)((int64_t)sp * p->super_pages / region)].push_back(sp);
        // emptied from the least full on, into the fullest that have room
        std::vector<int32_t> order;
        for (size_t r = 0; r < n_regions; ++r)
            if (R[r].live > 0) order.push_back((int32_t)r);
        std::sort(order.begin(), order.end(), [&](int32_t x, int32_t y) {
            return R[(size_t)x].live != R[(size_t)y].live ? R[(size_t)x].live < R[(size_t)y].live : x > y;
        });
        std::vector<int32_t> src[KV_MAX_LAYOUTS], dst[KV_MAX_LAYOUTS], cut[KV_MAX_LAYOUTS];
        int moves = 0;
        int64_t spare[KV_MAX_LAYOUTS] = {0, 0, 0, 0}, spare_supers = 0;
        size_t into[KV_MAX_LAYOUTS], super_from = order.size();  // taken from the back of `order`
        for (int l = 0; l < nl; ++l) {
            into[l] = order.size();
            for (int32_t r : order) spare[l] += (int64_t)room[l][(size_t)r].size();
        }
        for (int32_t r : order) spare_supers += (int64_t)supers[(size_t)r].size();
        for (int32_t k : order) {
            Region &r = R[(size_t)k];
            int64_t need[KV_MAX_LAYOUTS] = {0, 0, 0, 0}, cuts = 0;
            for (int32_t id : r.blocks) ++need[p->owner[(size_t)id]];
            // (this region's own room does not count)
            for (int l = 0; l < nl; ++l) {
                const int64_t per = p->super_pages / p->pages_per_block[l];
                const int64_t more = need[l] - (spare[l] - (int64_t)room[l][(size_t)k].size());
                if (more > 0) cuts += (more + per - 1) / per;
            }
            if (r.fixed || (int64_t)r.blocks.size() + moves > max_moves ||
                cuts > spare_supers - (int64_t)supers[(size_t)k].size())
                continue;  // it stays, and later ones may move into it
            for (int l = 0; l < nl; ++l) {
                spare[l] -= (int64_t)room[l][(size_t)k].size();
                room[l][(size_t)k].clear();
            }
            spare_supers -= (int64_t)supers[(size_t)k].size();
            supers[(size_t)k].clear();
            for (int32_t id : r.blocks) {
                const int l = p->owner[(size_t)id];
                if (spare[l] == 0) {
                    while (supers[(size_t)order[super_from - 1]].empty()) --super_from;
                    std::vector<int32_t> &f = supers[(size_t)order[super_from - 1]];
                    const int32_t step = p->pages_per_block[l];
                    for (int32_t off = 0; off + step <= p->super_pages; off += step)
                        room[l][(size_t)order[super_from - 1]].push_back(f.back() * p->super_pages + off);
                    spare[l] += p->super_pages / step;
                    cut[l].push_back(f.back());
                    f.pop_back();
                    --spare_supers;
                    into[l] = super_from;
                }
                while (room[l][(size_t)order[into[l] - 1]].empty()) --into[l];
                auto &f = room[l][(size_t)order[into[l] - 1]];
                src[l].push_back(id);
                dst[l].push_back(f.back());
                R[(size_t)order[into[l] - 1]].fixed = true;  // it has taken moves: not emptied any more
                f.pop_back();
                --spare[l];
                ++moves;
            }
        }
        if (moves == 0) return KV_OK;
        std::vector<int32_t> to((size_t)p->n_pages, -1);
        for (int l = 0; l < nl; ++l)
            for (size_t i = 0; i < src[l].size(); ++i) to[(size_t)src[l][i]] = dst[l][i];
        // (what is needed below first, so that nothing there can fail but the copies)
        std::vector<int32_t> keep[KV_MAX_LAYOUTS], cut_all;
        for (int l = 0; l < nl; ++l) {
            std::vector<int32_t> taken = dst[l];
            std::sort(taken.begin(), taken.end());
            auto take = [&](int32_t id) {
                if (!std::binary_search(taken.begin(), taken.end(), id)) keep[l].push_back(id);
            };
            for (int32_t id : p->free_blocks[l]) take(id);
            for (int32_t sp : cut[l])
                for (int32_t off = 0; off + p->pages_per_block[l] <= p->super_pages; off += p->pages_per_block[l]) take(sp * p->super_pages + off);
            keep[l].insert(keep[l].end(), src[l].begin(), src[l].end());
            cut_all.insert(cut_all.end(), cut[l].begin(), cut[l].end());
        }
        std::sort(cut_all.begin(), cut_all.end());
        // a failed copy leaves the tables and the allocator as they were: only
        // free blocks have been written
        for (int l = 0; l < nl; ++l) {
            const int rc = kvp_copy_pages(p, l, (int)src[l].size(), src[l].data(), dst[l].data(), nullptr, stream);
            if (rc) return rc;
        }
        for (int l = 0; l < nl; ++l) {
            for (size_t i = 0; i < src[l].size(); ++i) {
                const size_t a = (size_t)src[l][i], b = (size_t)dst[l][i];
                p->refcnt[b] = p->refcnt[a];
                p->owner[b] = (int8_t)l;
                p->refcnt[a] = 0;
                p->owner[a] = -1;
            }
            p->free_blocks[l].assign(keep[l].begin(), keep[l].end());  // (within its room)
            p->carved_blocks[l] += (int64_t)cut[l].size() * (p->super_pages / p->pages_per_block[l]);
            if (p->vmm.active)
                for (int32_t sp : cut[l]) p->vmm.free_supers[(size_t)(sp / p->vmm.supers_per_chunk)] -= 1;
        }
        p->super_free.erase(std::remove_if(p->super_free.begin(), p->super_free.end(),
                                           [&](int32_t sp) {
                                               return std::binary_search(cut_all.begin(), cut_all.end(), sp);
                                           }),
                            p->super_free.end());
        for (kv_seqtab *t : p->seqtabs)
            for (int s = 0; s < t->S; ++s)
                for (int i = 0; i < t->held[(size_t)s]; ++i) {
                    const int32_t id = t->table[(size_t)s * t->max_blocks + i];
                    if (id >= 0 && id < p->n_pages && to[(size_t)id] >= 0)
                        kvp_seqtab_set_entry(t, s, i, to[(size_t)id]);
                }
        if (n_moves) *n_moves = moves;
    } catch (const std::bad_alloc &) {
        return KV_ERR_OUT_OF_BLOCKS;
    }
    return KV_OK;
}

}  // extern "C"
