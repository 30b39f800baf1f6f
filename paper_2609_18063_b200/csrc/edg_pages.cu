// Pages of a cache: fork, grow, free, compact, copy -- the state (reference counts, page table, lengths) lives on the device.
//
// The bookkeeping is integer work over small arrays: one CTA does what has an order (which page goes to whom), many do what has
// none (sharing, releasing, copying rows).  Every result is a function of the lists alone: free pages are given out in ascending order along
// the list by prefix sums, counts are changed by integer atomics.  Latency bounds fork / reserve / free (a launch or two of a few
// dependent trips to L2), HBM the copies.  Measured: 64 forks, one position more for each of them (a copied page in four layers each) and 32
// releases 33 us, 20 of them on the GPU; 48 sequences of 4,096 pages of 74 KB compacted in 45 us where the moved pages' bytes take 22.
#include "edg_ptx.cuh"

namespace edg {
namespace {

constexpr int kBook = 1024;                   // threads of the bookkeeping CTA, and the longest list

struct Move { int32_t src, dst, bytes, pad; };

struct PagesWorkspace {
    int32_t* status;
    int32_t* n_moves;                         // moves to carry out
    Move* moves;                              // [max(n_pages, kBook)]
    int32_t* list;                            // [n_pages]: free pages taken, or where a page moves to
};
inline size_t moves_of(const edg_page_pool& p) { return p.n_pages > kBook ? (size_t)p.n_pages : (size_t)kBook; }
inline size_t pages_bytes(const edg_page_pool& p) { return round_up(kCtrlBytes + 256 + moves_of(p) * sizeof(Move) + (size_t)p.n_pages * 4, 256); }
inline PagesWorkspace pages_workspace(void* ws, const edg_page_pool& p) {
    uint8_t* b = static_cast<uint8_t*>(ws);
    PagesWorkspace w;
    w.status = reinterpret_cast<int32_t*>(b);
    w.n_moves = reinterpret_cast<int32_t*>(b + kCtrlBytes);
    w.moves = reinterpret_cast<Move*>(b + kCtrlBytes + 256);
    w.list = reinterpret_cast<int32_t*>(w.moves + moves_of(p));
    return w;
}

__device__ __forceinline__ void raise(int32_t* status, int32_t code) { atomicCAS(status, 0, code); }
__device__ __forceinline__ int pages_for(int len, int page) { return (int)(((long long)len + page - 1) / page); }

// Exclusive prefix sum over the CTA's kBook threads; total to all.  Two barriers.
template <typename I>
__device__ __forceinline__ I block_scan(I v, I* s_warp, I& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    I x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const I y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    const I w = s_warp[lane];
    I z = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const I y = __shfl_up_sync(0xFFFFFFFFu, z, o);
        if (lane >= o) z += y;
    }
    total = __shfl_sync(0xFFFFFFFFu, z, 31);
    const I before = warp == 0 ? 0 : __shfl_sync(0xFFFFFFFFu, z, warp - 1);
    __syncthreads();
    return before + x - v;
}

__global__ void __launch_bounds__(128) fork_kernel(const edg_page_pool p, int n, const int32_t* parents, const int32_t* children, int32_t* status) {
    const int i = blockIdx.x, c = children[i], a = parents[i];
    int bad = c < 0 || c >= p.n_seqs || a < 0 || a >= p.n_seqs;
    for (int j = threadIdx.x; j < n; j += blockDim.x) bad |= (j < i && children[j] == c) || children[j] == a;
    if (!bad) bad = p.lens[c] != 0;          // (only the CTA that may change it reads past this point)
    bad = __syncthreads_or(bad);
    if (bad) {
        if (threadIdx.x == 0) raise(status, EDG_E_RANGE);
        return;
    }
    const int len = p.lens[a];
    const int np = len < 0 ? 0 : min(pages_for(len, p.page), p.max_pages);
    for (int j = threadIdx.x; j < np; j += blockDim.x) {
        const int pg = p.table[(size_t)a * p.max_pages + j];
        p.table[(size_t)c * p.max_pages + j] = pg;
        if (pg >= 0 && pg < p.n_pages) atomicAdd(&p.refs[pg], 1);
        else raise(status, EDG_E_RANGE);
    }
    if (threadIdx.x == 0) p.lens[c] = len;
}

__global__ void __launch_bounds__(128) free_kernel(const edg_page_pool p, int n, const int32_t* seqs, int32_t* status) {
    const int i = blockIdx.x, s = seqs[i];
    int twice = 0;
    for (int j = threadIdx.x; j < i; j += blockDim.x) twice |= seqs[j] == s;
    twice = __syncthreads_or(twice);
    if (s < 0 || s >= p.n_seqs) {
        if (threadIdx.x == 0) raise(status, EDG_E_RANGE);
        return;
    }
    if (twice) return;
    const int len = p.lens[s];
    const int np = len < 0 ? 0 : min(pages_for(len, p.page), p.max_pages);
    for (int j = threadIdx.x; j < np; j += blockDim.x) {
        const int pg = p.table[(size_t)s * p.max_pages + j];
        p.table[(size_t)s * p.max_pages + j] = -1;
        if (pg < 0 || pg >= p.n_pages) { raise(status, EDG_E_RANGE); continue; }
        if (atomicSub(&p.refs[pg], 1) <= 0) {                       // nobody held it
            atomicAdd(&p.refs[pg], 1);
            raise(status, EDG_E_RANGE);
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) p.lens[s] = 0;
}

__global__ void __launch_bounds__(kBook) reserve_kernel(const edg_page_pool p, int n, const int32_t* seqs, const int32_t* counts, int row_bytes,
                                                        const PagesWorkspace w) {
    __shared__ int s_seq[kBook], s_last[kBook], s_first[kBook + 1], s_warp[32];
    __shared__ long long s_sums[32];
    const int i = threadIdx.x;
    const int seq = i < n ? seqs[i] : -1, cnt = i < n ? counts[i] : 0;
    s_seq[i] = seq;
    bool ok = i < n && seq >= 0 && seq < p.n_seqs && cnt >= 0;
    int old = 0, last = -1;
    __syncthreads();
    if (ok)
        for (int j = 0; j < i; ++j) ok = ok && s_seq[j] != seq;
    if (ok) {
        old = p.lens[seq];
        ok = old >= 0 && (long long)old + cnt <= (long long)p.max_pages * p.page;
    }
    const int p_old = ok ? pages_for(old, p.page) : 0, p_new = ok ? pages_for(old + cnt, p.page) : 0;
    const bool partial = ok && cnt > 0 && old % p.page != 0;
    if (partial) {
        last = p.table[(size_t)seq * p.max_pages + p_old - 1];
        if (last < 0 || last >= p.n_pages) { ok = false; last = -1; }
    }
    if (i < n && !ok) raise(w.status, EDG_E_RANGE);
    s_last[i] = last;
    __syncthreads();
    bool copy = false;
    if (ok && last >= 0) {                                          // all holders but the last one copy
        int rank = 0;
        for (int j = 0; j < i; ++j) rank += s_last[j] == last;
        copy = rank < p.refs[last] - 1;
    }
    // (1024 sequences of up to 2^31 pages: the sum has 64 bits.  What is beyond the pool counts as one page beyond it.)
    long long all;
    const long long before = block_scan<long long>(ok ? p_new - p_old + (copy ? 1 : 0) : 0, s_sums, all);
    const int total = (int)min(all, p.n_pages + 1ll), first = (int)min(before, p.n_pages + 1ll);
    s_first[i] = first;
    if (i == 0) s_first[kBook] = total;
    // the lowest `total` free pages, in ascending order
    int found = 0;
    for (int b = 0; b < p.n_pages && found < total; b += kBook * 8) {
        const int at = b + i * 8;
        unsigned mask = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (at + j < p.n_pages && p.refs[at + j] == 0) mask |= 1u << j;
        int here;
        int k = found + block_scan(__popc(mask), s_warp, here);
        while (mask != 0 && k < total) {
            w.list[k++] = at + __ffs(mask) - 1;
            mask &= mask - 1;
        }
        found += here;
    }
    __syncthreads();                                                // (the list and s_first are there)
    const bool enough = found >= total;
    if (i == 0) {
        if (!enough) raise(w.status, EDG_E_SLOTS);
        *w.n_moves = enough ? n : 0;
    }
    if (i < n) {
        Move m = {-1, -1, 0, 0};
        if (enough && copy) { m.src = last; m.dst = w.list[first]; m.bytes = (old % p.page) * row_bytes; }
        w.moves[i] = m;
    }
    if (!enough) return;
    if (copy) {
        atomicSub(&p.refs[last], 1);
        p.table[(size_t)seq * p.max_pages + p_old - 1] = w.list[first];
    }
    if (ok) p.lens[seq] = old + cnt;
    s_last[i] = p_old - (copy ? 1 : 0);                             // table column of this entry's first page
    __syncthreads();
    for (int k = i; k < total; k += kBook) {                        // pages one by one: whose they are is looked up
        int lo = 0, hi = n - 1;
        while (lo < hi) {                                           // last entry with s_first <= k
            const int mid = (lo + hi + 1) >> 1;
            if (s_first[mid] <= k) lo = mid; else hi = mid - 1;
        }
        const int pg = w.list[k];
        p.refs[pg] = 1;
        p.table[(size_t)s_seq[lo] * p.max_pages + s_last[lo] + k - s_first[lo]] = pg;
    }
}

__device__ __forceinline__ void copy_bytes(uint8_t* dst, const uint8_t* src, int64_t bytes, int tid, int threads) {
    const uint4* s = reinterpret_cast<const uint4*>(src);
    uint4* d = reinterpret_cast<uint4*>(dst);
    const int n = (int)(bytes / 16);
    int i = tid;
    for (; i + 3 * threads < n; i += 4 * threads) {
        uint4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = ld_stream16(s + i + j * threads);
#pragma unroll
        for (int j = 0; j < 4; ++j) __stcs(d + i + j * threads, v[j]);
    }
    for (; i < n; i += threads) __stcs(d + i, ld_stream16(s + i));
}

constexpr int kPiece = 16384;                 // bytes that a CTA copies at a time

// the moves, piece by piece over all layers; then (TABLE) the table's pages are renamed and the counts follow
template <bool TABLE>
__global__ void __launch_bounds__(256) move_kernel(const edg_page_pool p, const edg_page_cache c, const PagesWorkspace w) {
    const int64_t page_bytes = (int64_t)c.page * c.row_bytes;
    const int pieces = (int)((page_bytes + kPiece - 1) / kPiece), moves = *w.n_moves;
    const int64_t work = (int64_t)moves * c.n_layers * pieces;
    for (int64_t k = blockIdx.x; k < work; k += gridDim.x) {
        const int piece = (int)(k % pieces), layer = (int)(k / pieces % c.n_layers);
        const Move m = w.moves[k / pieces / c.n_layers];
        const int64_t from = (int64_t)piece * kPiece, bytes = min((int64_t)m.bytes - from, (int64_t)kPiece);
        if (m.src < 0 || bytes <= 0) continue;
        uint8_t* base = static_cast<uint8_t*>(c.base) + layer * c.layer_stride + from;
        copy_bytes(base + m.dst * page_bytes, base + m.src * page_bytes, bytes, threadIdx.x, 256);
    }
    if (!TABLE) return;
    const int64_t entries = (int64_t)p.n_seqs * p.max_pages, at = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
    for (int64_t k = at; k < entries; k += step) {
        const int pg = p.table[k];
        if (pg >= 0 && pg < p.n_pages) {
            const int to = w.list[pg];
            if (to != pg) p.table[k] = to;
        }
    }
    for (int64_t k = at; k < moves; k += step) {
        const Move m = w.moves[k];
        p.refs[m.dst] = m.pad;                                      // (the count of the page that moved)
        p.refs[m.src] = 0;
    }
}

// which pages move where: pages in use at u and behind to the free ones before u
__global__ void __launch_bounds__(kBook) compact_kernel(const edg_page_pool p, int page_bytes, const PagesWorkspace w) {
    __shared__ int s_warp[32];
    const int i = threadIdx.x;
    int used = 0;
    for (int b = i; b < p.n_pages; b += kBook) used += p.refs[b] > 0;
    int u;
    block_scan(used, s_warp, u);
    int from = 0, to = 0;                     // pages that move, and places for them, found so far
    for (int b = 0; b < p.n_pages; b += kBook * 8) {
        const int at = b + i * 8;
        unsigned src = 0, dst = 0;
        int r[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            r[j] = at + j < p.n_pages ? p.refs[at + j] : 0;
            if (at + j < p.n_pages) {
                w.list[at + j] = at + j;
                if (r[j] > 0 && at + j >= u) src |= 1u << j;
                if (r[j] <= 0 && at + j < u) dst |= 1u << j;
            }
        }
        int n_src, n_dst;
        int ks = from + block_scan(__popc(src), s_warp, n_src), kd = to + block_scan(__popc(dst), s_warp, n_dst);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (src >> j & 1u) { w.moves[ks].src = at + j; w.moves[ks].pad = r[j]; w.moves[ks].bytes = page_bytes; ++ks; }
            if (dst >> j & 1u) w.moves[kd++].dst = at + j;
        }
        from += n_src;
        to += n_dst;
    }
    __syncthreads();
    for (int k = i; k < from; k += kBook) w.list[w.moves[k].src] = w.moves[k].dst;
    if (i == 0) *w.n_moves = from;
}

__global__ void __launch_bounds__(256) copy_kernel(const edg_page_cache d, const edg_page_cache s, int n, const int32_t* dst_pages,
                                                   const int32_t* src_pages, int32_t* status) {
    const int i = blockIdx.x, to = dst_pages[i], from = src_pages[i];
    const bool same = d.base == s.base;
    if (to < 0 || to >= d.n_pages || from < 0 || from >= s.n_pages) {
        if (threadIdx.x == 0) raise(status, EDG_E_RANGE);
        return;
    }
    int later = 0, read = 0;
    for (int j = threadIdx.x; j < n; j += 256) {
        later |= j > i && dst_pages[j] == to;
        read |= same && j != i && src_pages[j] == to;
    }
    later = __syncthreads_or(later);
    read = __syncthreads_or(read);
    if (read) {
        if (threadIdx.x == 0) raise(status, EDG_E_RANGE);
        return;
    }
    if (later || (same && from == to)) return;
    const int64_t bytes = (int64_t)d.page * d.row_bytes;
    for (int layer = blockIdx.y; layer < d.n_layers; layer += gridDim.y)
        copy_bytes(static_cast<uint8_t*>(d.base) + layer * d.layer_stride + to * bytes,
                   static_cast<const uint8_t*>(s.base) + layer * s.layer_stride + from * bytes, bytes, threadIdx.x, 256);
}

int32_t check_pool(const edg_page_pool* p) {
    if (!p || !p->refs || !p->table || !p->lens) return EDG_E_INVAL;
    if (!aligned(p->refs, 4) || !aligned(p->table, 4) || !aligned(p->lens, 4)) return EDG_E_INVAL;
    if (p->n_pages < 1 || p->page < 1 || p->n_seqs < 1 || p->max_pages < 1) return EDG_E_SHAPE;
    if ((int64_t)p->max_pages * p->page > 0x7FFFFFFF || (int64_t)p->n_pages > (1 << 26)) return EDG_E_SHAPE;
    return EDG_OK;
}
int32_t check_cache(const edg_page_cache* c) {
    if (!c || !c->base || !aligned(c->base, 16)) return EDG_E_INVAL;
    if (c->n_layers < 1 || c->n_pages < 1 || c->page < 1 || c->row_bytes < 16 || c->row_bytes % 16 != 0 || c->layer_stride % 16 != 0) return EDG_E_SHAPE;
    const int64_t page_bytes = (int64_t)c->page * c->row_bytes;
    if (page_bytes > (1 << 28) || (c->n_layers > 1 && c->layer_stride < page_bytes * c->n_pages)) return EDG_E_SHAPE;
    return EDG_OK;
}
int32_t check_both(const edg_page_pool* p, const edg_page_cache* c) {
    int32_t rc = check_pool(p);
    if (rc == EDG_OK) rc = check_cache(c);
    if (rc == EDG_OK && (p->n_pages != c->n_pages || p->page != c->page)) rc = EDG_E_SHAPE;
    return rc;
}
int32_t check_scratch(const edg_page_pool* p, const void* ws, size_t bytes) {
    if (!ws) return EDG_E_INVAL;
    return aligned(ws, 256) && bytes >= pages_bytes(*p) ? EDG_OK : EDG_E_WORKSPACE;
}
int32_t launched() {
    EDG_CUDA_TRY(cudaGetLastError());
    return EDG_OK;
}

}  // namespace
}  // namespace edg

using namespace edg;

extern "C" int32_t edg_pages_workspace_bytes(const edg_page_pool* pool, size_t* bytes) {
    const int32_t rc = check_pool(pool);
    if (rc != EDG_OK) return rc;
    if (!bytes) return EDG_E_INVAL;
    *bytes = pages_bytes(*pool);
    return EDG_OK;
}

extern "C" int32_t edg_pages_fork(const edg_page_pool* pool, int32_t n, const int32_t* parents, const int32_t* children, void* workspace,
                                  size_t workspace_bytes, void* stream) {
    int32_t rc = check_pool(pool);
    if (rc == EDG_OK && (!parents || !children || n < 1 || n > kBook)) rc = EDG_E_INVAL;
    if (rc == EDG_OK) rc = check_scratch(pool, workspace, workspace_bytes);
    if (rc != EDG_OK) return rc;
    fork_kernel<<<n, 128, 0, static_cast<cudaStream_t>(stream)>>>(*pool, n, parents, children, static_cast<int32_t*>(workspace));
    return launched();
}

extern "C" int32_t edg_pages_reserve(const edg_page_pool* pool, const edg_page_cache* cache, int32_t n, const int32_t* seqs, const int32_t* counts,
                                     void* workspace, size_t workspace_bytes, void* stream) {
    int32_t rc = check_both(pool, cache);
    if (rc == EDG_OK && (!seqs || !counts || n < 1 || n > kBook)) rc = EDG_E_INVAL;
    if (rc == EDG_OK) rc = check_scratch(pool, workspace, workspace_bytes);
    if (rc != EDG_OK) return rc;
    const PagesWorkspace w = pages_workspace(workspace, *pool);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    reserve_kernel<<<1, kBook, 0, st>>>(*pool, n, seqs, counts, cache->row_bytes, w);
    rc = launched();
    if (rc != EDG_OK) return rc;
    const int64_t pieces = ((int64_t)cache->page * cache->row_bytes + kPiece - 1) / kPiece, work = pieces * n * cache->n_layers, most = 8ll * sm_count();
    move_kernel<false><<<(int)(work < most ? work : most), 256, 0, st>>>(*pool, *cache, w);
    return launched();
}

extern "C" int32_t edg_pages_free(const edg_page_pool* pool, int32_t n, const int32_t* seqs, void* workspace, size_t workspace_bytes, void* stream) {
    int32_t rc = check_pool(pool);
    if (rc == EDG_OK && (!seqs || n < 1 || n > kBook)) rc = EDG_E_INVAL;
    if (rc == EDG_OK) rc = check_scratch(pool, workspace, workspace_bytes);
    if (rc != EDG_OK) return rc;
    free_kernel<<<n, 128, 0, static_cast<cudaStream_t>(stream)>>>(*pool, n, seqs, static_cast<int32_t*>(workspace));
    return launched();
}

extern "C" int32_t edg_pages_compact(const edg_page_pool* pool, const edg_page_cache* cache, void* workspace, size_t workspace_bytes, void* stream) {
    int32_t rc = check_both(pool, cache);
    if (rc == EDG_OK) rc = check_scratch(pool, workspace, workspace_bytes);
    if (rc != EDG_OK) return rc;
    const PagesWorkspace w = pages_workspace(workspace, *pool);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    compact_kernel<<<1, kBook, 0, st>>>(*pool, cache->page * cache->row_bytes, w);
    rc = launched();
    if (rc != EDG_OK) return rc;
    move_kernel<true><<<8 * sm_count(), 256, 0, st>>>(*pool, *cache, w);
    return launched();
}

extern "C" int32_t edg_pages_copy(const edg_page_cache* dst, const edg_page_cache* src, int32_t n, const int32_t* dst_pages, const int32_t* src_pages,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    int32_t rc = check_cache(dst);
    if (rc == EDG_OK) rc = check_cache(src);
    if (rc != EDG_OK) return rc;
    if (!dst_pages || !src_pages || n < 1 || n > 65535 || !workspace) return EDG_E_INVAL;
    if (dst->page != src->page || dst->row_bytes != src->row_bytes || dst->n_layers != src->n_layers) return EDG_E_SHAPE;
    if (dst->base == src->base && (dst->n_pages != src->n_pages || dst->layer_stride != src->layer_stride)) return EDG_E_SHAPE;
    if (!aligned(workspace, 256) || workspace_bytes < kCtrlBytes) return EDG_E_WORKSPACE;
    copy_kernel<<<dim3(n, dst->n_layers < 64 ? dst->n_layers : 64), 256, 0, static_cast<cudaStream_t>(stream)>>>(
        *dst, *src, n, dst_pages, src_pages, static_cast<int32_t*>(workspace));
    return launched();
}
