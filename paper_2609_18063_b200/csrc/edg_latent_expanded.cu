// Latent attention, expanded form (prompts): keys and values of every head are written out once, then plain causal attention over them.
//
//     K[h,j] = W_uk[h] c_j,  V[h,j] = W_uv[h] c_j            (expand_kernel: one product of 128 cache rows with a head's weights each)
//     y[t,h] = softmax(scale (q_nope . K[h,j] + q_rope . p_j)) V[h]        (prompt_kernel)
//
// 2 (d_n + d_r + d_v) operations a pair of rows against 2 (2 d_l + d_r) in the latent space, 3.4 times fewer at 128 / 64 / 128 / 512; the writing out costs
// 2 d_l (d_n + d_v) a position and head, which some hundred new rows a sequence earn back.
//
// prompt_kernel: a CTA takes pairs of tiles of 128 new rows of a head; while the softmax of one runs, the tensor cores work on the other.  S of
// a tile (128 x 128) lies in tensor memory, two threads to a row with half of its columns each.  P goes back over S as bf16 and is the A
// operand of P V from there, the first half of it while the other is still being made.  O is rescaled only when a row's maximum has grown by
// more than 2^8.  Keys and values come by TMA in chunks of 64 columns through one ring of eight (K of a tile, V of it, K of the next: the tile
// after that takes what S has read).  Positions behind a sequence's end are padded to 128; their values are written as zeros, their scores
// never looked at.
//
// K is rounded to bf16, by 2^-8 of a value at most: the operands of a product have one type, and the queries' is bf16.  V and P are rounded to fp16, by
// 2^-11, wherever that holds their range: |V| is at most d_l times the largest of a row of W_uv times the largest of a cache row, so the exponents of
// these tell, for a tile of positions, whether V stays below 2^15 and whether it is large enough for what fp16 cuts off at 2^-25 not to count.  In
// other tiles both are bf16, which holds any range.  Maxima, sums and O are fp32.  Of a standard normal batch the outputs before their own rounding are
// 0.1% off in the mean square (0.2% with V and P in bf16).
//
// 4,430 new rows of three sequences of 7,103 positions, 32 heads of 128 + 64 / 128, 512 latent columns: 232 to 282 us, by the box; under a
// profiler the plan and the look through W_uv 5, expand_kernel 64 to 67 (62 GFLOP: 1.0 PFLOP/s; its limits are the weights, which every CTA reads from
// L2, and its two rounds of CTAs), prompt_kernel 190 (185 GFLOP of rows that see one another: 1.0 PFLOP/s).  A pair of tiles takes 3,900
// clocks, with products under way for 3,260 (2,600 by their operations); S of a tile, its softmax (2,050) and P V follow one another, since neither tensor memory has room for a third S nor shared
// memory for P.
#include "edg_latent.cuh"
#include "edg_umma.cuh"

namespace edg {

struct ExpandedParams {
    LatentSeqs s;
    const uint16_t* cache;
    uint16_t *K, *V, *Rp;       // [heads][rows][dn], [heads][rows][dv], [rows][64] (rotated part and zeros)
    int32_t *q_pre, *kv_pre;    // [n + 1] pairs of row tiles before a sequence; tiles of 128 positions before it
    int32_t* next;              // the next pair of row tiles (of a head) to be taken
    const uint16_t* W_uv;
    int32_t* w_range;           // [kScan] exponents of the largest values of rows of W_uv: most << 16 | least
    int32_t* halves;            // [rows / 128] whether V of a tile of positions, and P beside it, is fp16
    void* y;
    int32_t* status;
    int heads, dn, dr, dv, dl, out_dtype;
    int rows;                   // rows of K and V that there is room for, a multiple of 128
    int more_than;              // sequences of more new rows than this are taken
    int max_new, splits;
    int64_t total_len;
    float scale;
};

namespace {

struct XSeq { int a, fresh, len, pairs, tiles; };
__device__ __forceinline__ XSeq xsequence(const ExpandedParams& p, int i) {
    XSeq q;
    q.a = min(max(p.s.cu[i], 0), p.s.T);
    q.fresh = max(min(p.s.cu[i + 1], p.s.T) - q.a, 0);
    q.len = min(max(p.s.lens[i], 0), p.s.max_pages << p.s.page_shift);
    const bool mine = q.fresh > p.more_than;
    q.pairs = mine ? (q.fresh + 255) >> 8 : 0;
    q.tiles = mine ? (q.len + 127) >> 7 : 0;
    return q;
}

constexpr int kSms = 148;                   // what a launch is sized by

// Biased exponents of the largest magnitudes of rows (of cache or W_uv): the most and the least of them, rows of zeros aside.
struct Exponents {
    unsigned most = 0, least = 511;
    __device__ __forceinline__ void row(unsigned magnitude) {            // (bits of a bf16 without its sign)
        if (magnitude == 0) return;
        most = max(most, magnitude >> 7);
        least = min(least, magnitude >> 7);
    }
    __device__ __forceinline__ void join(unsigned packed) { most = max(most, packed >> 16); least = min(least, packed & 0xFFFFu); }
    __device__ __forceinline__ unsigned packed() const { return most << 16 | least; }
};
// V is a sum of d_l <= 2^9 products of values below 2^(e - 126): below 2^15 where the two exponents add up to 258 at most.  Where they add up to 246 at least,
// V of rows without outliers is some 2^-7 and more, of which fp16 cuts off 2^-25: a value has to be 2^-9 of that before bf16 would hold it better.
__device__ __forceinline__ bool fits_half(const Exponents& w, const Exponents& c) { return w.most + c.most <= 258 && w.least + c.least >= 246; }

// CTAs of the plan that look through W_uv
constexpr int kScan = 128;
__device__ __forceinline__ void scan_values(const ExpandedParams& p, int cta) {
    __shared__ unsigned s_range[8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rows = p.heads * p.dv;
    Exponents e;
#pragma unroll 4
    for (int r = cta * 8 + warp; r < rows; r += kScan * 8) {
        const uint16_t* w = p.W_uv + (size_t)r * p.dl + lane * 8;
        uint32_t m = 0;
        if (lane * 8 < p.dl) m = bf16_magnitudes(m, __ldg(reinterpret_cast<const uint4*>(w)));
        if (256 + lane * 8 < p.dl) m = bf16_magnitudes(m, __ldg(reinterpret_cast<const uint4*>(w + 256)));
        e.row(__reduce_max_sync(0xFFFFFFFFu, max(m & 0xFFFFu, m >> 16)));
    }
    if (lane == 0) s_range[warp] = e.packed();
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int i = 1; i < 8; ++i) e.join(s_range[i]);
    p.w_range[cta] = (int32_t)e.packed();
}

// prefix sums over the sequences, and the caller's bounds; the other CTAs look through W_uv meanwhile
__global__ void __launch_bounds__(256) prompt_plan_kernel(const __grid_constant__ ExpandedParams p) {
    pdl_launch_dependents();
    if (blockIdx.x > 0) {
        scan_values(p, blockIdx.x - 1);
        return;
    }
    if (threadIdx.x == 0) *p.next = 0;
    __shared__ int s_q[8], s_k[8];
    __shared__ long long s_l[8], s_f[8];
    const int tid = threadIdx.x, per = (p.s.n + 255) / 256, i0 = min(tid * per, p.s.n), i1 = min(i0 + per, p.s.n);
    int q = 0, k = 0;
    long long len = 0, fresh = 0;
    bool ok = tid != 0 || (p.s.cu[0] == 0 && p.s.cu[p.s.n] <= p.s.T);
    for (int i = i0; i < i1; ++i) {
        const XSeq x = xsequence(p, i);
        q += x.pairs;
        k += x.tiles;
        len += x.len;
        fresh += x.fresh;
        ok = ok && p.s.cu[i + 1] >= p.s.cu[i] && x.fresh <= p.max_new && x.len >= p.s.lens[i];
    }
    const int lane = tid & 31, warp = tid >> 5, own_q = q, own_k = k;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {                                    // sums up to and with this lane's
        const int a = __shfl_up_sync(0xFFFFFFFFu, q, d), b = __shfl_up_sync(0xFFFFFFFFu, k, d);
        if (lane >= d) { q += a; k += b; }
        len += __shfl_xor_sync(0xFFFFFFFFu, len, d);
        fresh += __shfl_xor_sync(0xFFFFFFFFu, fresh, d);
    }
    if (lane == 31) { s_q[warp] = q; s_k[warp] = k; s_l[warp] = len; s_f[warp] = fresh; }
    __syncthreads();
    q -= own_q;
    k -= own_k;
    len = fresh = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (j < warp) { q += s_q[j]; k += s_k[j]; }
        len += s_l[j];
        fresh += s_f[j];
    }
    if (!ok || len > p.total_len) latent_raise(p.status, EDG_E_RANGE);
    const bool none = len > p.total_len || fresh > p.s.T;                // (sequences that overlap, or more than there is room for: nothing is done)
    if (none) q = k = 0;
    for (int i = i0; i < i1; ++i) {
        XSeq x = xsequence(p, i);
        if (none) x.pairs = x.tiles = 0;
        p.q_pre[i] = q;
        p.kv_pre[i] = k;
        q += x.pairs;
        k += x.tiles;
        if (i == p.s.n - 1) { p.q_pre[p.s.n] = q; p.kv_pre[p.s.n] = k; }
    }
    if (k * 128ll > p.rows && tid == 255) latent_raise(p.status, EDG_E_RANGE);
}

// ---------------------------------------------------------------- keys and values

constexpr int kXThreads = 256;              // warp 0 loads, warp 1 issues products, warps 4-7 write out
constexpr int kXRing = 12;                  // chunks of weights in flight: four behind the cache rows, eight where these lay
constexpr uint32_t kChunk = 16384;          // 128 rows of 64 columns
constexpr uint32_t kXOut = 12 * kChunk, kXBars = kXOut + 4 * 8192, kXBytes = kXBars + 256 + 1024;

// The cache rows are the A operand of all products of a CTA.  They go on to tensor memory (256 columns of it): with both operands in shared
// memory the products take all of its 128 bytes a clock, and the arrival of the weights comes on top (7,500 rows, 32 heads of 128: 88 us, and 69 from here).
__global__ void __launch_bounds__(kXThreads, 1) expand_kernel(const __grid_constant__ ExpandedParams p, const __grid_constant__ CUtensorMap c_map,
                                                              const __grid_constant__ CUtensorMap uk_map, const __grid_constant__ CUtensorMap uv_map) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    const uint32_t sb = smem_u32(smem);
    uint64_t* w_full = reinterpret_cast<uint64_t*>(smem + kXBars);       // [kXRing]
    uint64_t* w_empty = w_full + kXRing;
    uint64_t* c_full = w_empty + kXRing;
    uint64_t* a_full = c_full + 1;                                       // the cache rows are in tensor memory
    uint64_t* d_full = a_full + 1;                                       // [2]
    uint64_t* d_empty = d_full + 2;                                      // [2]
    uint32_t* s_tmem = reinterpret_cast<uint32_t*>(d_empty + 2);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < kXRing; ++i) { mbar_init(&w_full[i], 1); mbar_init(&w_empty[i], 1); }
        mbar_init(c_full, 1);
        mbar_init(a_full, 4);
        for (int i = 0; i < 2; ++i) { mbar_init(&d_full[i], 1); mbar_init(&d_empty[i], 4); }
        fence_barrier_init();
    }
    if (warp == 1) tmem_alloc(s_tmem, 512);
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *s_tmem;
    __shared__ unsigned s_rows[4], s_weights[4];                         // exponents by warp: of this tile's cache rows, of W_uv
    const int tile = blockIdx.x, split = blockIdx.y;
    const int h0 = (int)((int64_t)p.heads * split / p.splits), h1 = (int)((int64_t)p.heads * (split + 1) / p.splits);
    const bool there = tile < p.kv_pre[p.s.n] && (tile + 1) * 128 <= p.rows;
    const int nc = p.dl / 64;
    auto chunk_at = [](int slot) { return (uint32_t)(slot < 4 ? slot + 8 : slot - 4) * kChunk; };      // (the cache rows come to chunks 0-7)
    if (there) {
        const int seq = find_sequence(p.kv_pre, p.s.n, tile, lane);
        const XSeq q = xsequence(p, seq);
        const int pos0 = (tile - p.kv_pre[seq]) * 128;
        if (warp == 0) {
            const int br = min(1 << p.s.page_shift, 128), boxes = 128 / br, outside = p.s.n_pages << p.s.page_shift;
            int coord = outside;
            const int at = pos0 + lane * br;
            if (lane < boxes && at < q.len) {
                const int pg = p.s.table[(size_t)seq * p.s.max_pages + (at >> p.s.page_shift)];
                if (pg >= 0 && pg < p.s.n_pages) coord = (pg << p.s.page_shift) + (at & ((1 << p.s.page_shift) - 1));
                else latent_raise(p.status, EDG_E_RANGE);
            }
            if (elected()) mbar_expect_tx(c_full, nc * kChunk);
            __syncwarp();
            for (int b = 0; b < boxes; ++b) {
                const int y = __shfl_sync(0xFFFFFFFFu, coord, b);
                if (elected())
                    for (int c = 0; c < nc; ++c) tma_2d(sb + c * kChunk + b * br * 128, &c_map, c * 64, y, c_full);
                __syncwarp();
            }
            if (elected()) {
                RingAt w;
                bool moved = false;
                for (int h = h0; h < h1; ++h)
                    for (int kv = 0; kv < 2; ++kv) {
                        const int n = kv == 0 ? p.dn : p.dv;
                        const CUtensorMap* map = kv == 0 ? &uk_map : &uv_map;
                        for (int c = 0; c < nc; ++c) {
                            role_wait(&w_empty[w.slot], w.phase ^ 1, p.status);
                            if (w.slot >= 4 && !moved) { role_wait(a_full, 0, p.status); moved = true; }
                            mbar_expect_tx(&w_full[w.slot], n * 128);
                            tma_2d(sb + chunk_at(w.slot), map, c * 64, h * n, &w_full[w.slot]);
                            w.next(kXRing);
                        }
                    }
                // (no arrival of a product may come after the block's end)
                for (int i = 0; i < kXRing; ++i, w.next(kXRing)) role_wait(&w_empty[w.slot], w.phase ^ 1, p.status);
            }
            __syncwarp();
        } else if (warp == 1) {
            if (elected()) {                                             // (one thread: see the products of prompt_kernel)
                const uint32_t dw = desc_lo(sb);
                RingAt w;
                int j = 0;
                role_wait(a_full, 0, p.status);
                for (int h = h0; h < h1; ++h)
                    for (int kv = 0; kv < 2; ++kv, ++j) {
                        const uint32_t id = idesc_bf16(128, kv == 0 ? p.dn : p.dv), d = tmem + (j & 1) * 128;
                        role_wait(&d_empty[j & 1], ((uint32_t)(j >> 1) & 1) ^ 1, p.status);
                        for (int c = 0; c < nc; ++c) {
                            role_wait(&w_full[w.slot], w.phase, p.status);
                            tc_fence_after();
                            const uint32_t a = tmem + 256 + c * 32, b = dw + (chunk_at(w.slot) >> 4);
#pragma unroll
                            for (int k = 0; k < 4; ++k) umma_ts(d, a + k * 8, b + k * 2, id, c + k > 0);
                            umma_done(&w_empty[w.slot]);
                            w.next(kXRing);
                        }
                        umma_done(&d_full[j & 1]);
                    }
            }
            __syncwarp();
        } else if (warp >= 4) {
            const int wq = warp & 3, row = wq * 32 + lane;
            const uint32_t lanes = (uint32_t)(wq * 32) << 16;
            const bool held = pos0 + row < q.len;
            // A cache row that is not finite makes its scores NaN for all that see it; its values are zeros, so that rows that do not see
            // it stay what they are (their weight of zero times NaN would not).
            uint32_t most = 0;
            role_wait(c_full, 0, p.status);
            for (int c = 0; c < nc; ++c) {
                uint32_t v[32];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint4 x = *reinterpret_cast<const uint4*>(smem + c * kChunk + row * 128 + ((j ^ (row & 7)) * 16));
                    most = bf16_magnitudes(most, x);
                    v[4 * j] = x.x; v[4 * j + 1] = x.y; v[4 * j + 2] = x.z; v[4 * j + 3] = x.w;
                }
                tmem_st(tmem + lanes + 256 + c * 32, v);
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(a_full);
            const bool finite = !bf16_not_finite(most);
            Exponents rows, weights;
            rows.row(held && finite ? max(most & 0xFFFFu, most >> 16) : 0u);
            weights.join((unsigned)p.w_range[tid - 128]);
            static_assert(kScan == 128, "one to a thread");
            rows.most = __reduce_max_sync(0xFFFFFFFFu, rows.most);
            rows.least = __reduce_min_sync(0xFFFFFFFFu, rows.least);
            weights.most = __reduce_max_sync(0xFFFFFFFFu, weights.most);
            weights.least = __reduce_min_sync(0xFFFFFFFFu, weights.least);
            if (lane == 0) { s_rows[wq] = rows.packed(); s_weights[wq] = weights.packed(); }
            barrier_sync(1, 128);
#pragma unroll
            for (int i = 0; i < 4; ++i) { rows.join(s_rows[i]); weights.join(s_weights[i]); }
            const bool in_half = fits_half(weights, rows);
            if (split == 0 && tid == 128) p.halves[tile] = in_half;
            if (split == 0) {                                            // the rotated part of this thread's row
                uint4* out = reinterpret_cast<uint4*>(p.Rp + ((size_t)tile * 128 + row) * 64);
                const int at = pos0 + row;
                int pg = -1;
                if (held) pg = p.s.table[(size_t)seq * p.s.max_pages + (at >> p.s.page_shift)];
                const bool ok = pg >= 0 && pg < p.s.n_pages;
                const uint4* src = reinterpret_cast<const uint4*>(
                    p.cache + (((size_t)(ok ? pg : 0) << p.s.page_shift) + (at & ((1 << p.s.page_shift) - 1))) * (p.dl + p.dr) + p.dl);
#pragma unroll
                for (int c = 0; c < 8; ++c) out[c] = ok && c * 8 < p.dr ? src[c] : make_uint4(0, 0, 0, 0);
            }
            int j = 0;
            for (int h = h0; h < h1; ++h)
                for (int kv = 0; kv < 2; ++kv, ++j) {
                    const int n = kv == 0 ? p.dn : p.dv;
                    const bool keep = held && (kv == 0 || finite);
                    uint8_t* stage = smem + kXOut + wq * 8192;
                    role_wait(&d_full[j & 1], (uint32_t)(j >> 1) & 1, p.status);
                    tc_fence_after();
                    auto round = [&](auto pair) {
#pragma unroll 2
                        for (int c = 0; c < n; c += 16) {
                            uint32_t v[16];
                            tmem_ld(tmem + lanes + (j & 1) * 128 + c, v);
                            uint32_t o[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) o[i] = keep ? pair(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])) : 0u;
#pragma unroll
                            for (int x = 0; x < 2; ++x)
                                *reinterpret_cast<uint4*>(stage + lane * 256 + (((c / 8 + x) ^ (lane & 7)) * 16)) = make_uint4(o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]);
                        }
                    };
                    if (kv == 1 && in_half) round([](float a, float b) { return half_pair(a, b); });
                    else round([](float a, float b) { return bf16_pair(a, b); });
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&d_empty[j & 1]);
                    // (the 32 rows lie one behind another: whole lines, by way of shared memory; a row's own thread wrote 16 bytes to each of 32 lines)
                    uint16_t* out = (kv == 0 ? p.K : p.V) + ((size_t)h * p.rows + (size_t)tile * 128 + wq * 32) * n;
                    const int pieces = n / 8;
#pragma unroll 4
                    for (int x = lane; x < 32 * pieces; x += 32) {
                        const int rr = x / pieces, c = x - rr * pieces;
                        *reinterpret_cast<uint4*>(out + (size_t)x * 8) = *reinterpret_cast<const uint4*>(stage + rr * 256 + ((c ^ (rr & 7)) * 16));
                    }
                    __syncwarp();
                }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_free(tmem, 512);
}

// ---------------------------------------------------------------- attention

constexpr int kPThreads = 640;              // warp 0 takes work and loads, 1 issues products, 4-11 and 12-19 are the softmax of a tile of rows each
constexpr int kPRing = 8;
constexpr uint32_t kPQ = 0, kPRingAt = 6 * kChunk, kPBars = kPRingAt + kPRing * kChunk, kPItems = kPBars + 320, kPMax = kPItems + 64,
                   kPBytes = kPMax + 2048;

// Two tiles of 128 new rows of one head, and what they see.  h < 0: there is no more.  (Read until the item is done.)
struct alignas(16) Item { int h, kv0, pos0, token, rows, n[2], unused; };

__global__ void __launch_bounds__(kPThreads, 1) prompt_kernel(const __grid_constant__ ExpandedParams p, const __grid_constant__ CUtensorMap qn_map,
                                                              const __grid_constant__ CUtensorMap qr_map, const __grid_constant__ CUtensorMap k_map,
                                                              const __grid_constant__ CUtensorMap r_map, const __grid_constant__ CUtensorMap v_map) {
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sb = smem_u32(smem);
    uint64_t* kv_empty = reinterpret_cast<uint64_t*>(smem + kPBars);     // [kPRing] the groups below, read
    uint64_t* kv_full = kv_empty + kPRing;                                  // [kPRing] keys of a tile, its values, the next keys ...: never more than chunks
    uint64_t* q_full = kv_full + kPRing;                                      // [2]
    uint64_t* s_full = q_full + 2;                                       // [2]
    uint64_t* p_full = s_full + 2;                                       // [2]
    uint64_t* p_half = p_full + 2;                                       // [2] the first 32 columns of both halves of a tile's P
    uint64_t* o_done = p_half + 2;                                       // [2]
    uint64_t* q_empty = o_done + 2;                                      // [2] the last S of a tile of rows is there
    uint64_t* item_full = q_empty + 2;                                   // [2]
    uint64_t* item_empty = item_full + 2;                                // [2]
    uint32_t* s_tmem = reinterpret_cast<uint32_t*>(item_empty + 2);
    Item* s_item = reinterpret_cast<Item*>(smem + kPItems);              // [2]
    float* s_max = reinterpret_cast<float*>(smem + kPMax);               // [tile][half of the columns][row]
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if ((sb & 1023) != 0) {                                              // (the swizzle counts on it)
        if (tid == 0) latent_raise(p.status, EDG_E_INVAL);
        return;
    }
    if (tid == 0) {
        for (int i = 0; i < kPRing; ++i) mbar_init(&kv_empty[i], 1);
        for (int i = 0; i < kPRing; ++i) mbar_init(&kv_full[i], 1);
        for (int i = 0; i < 2; ++i) { mbar_init(&q_full[i], 1); mbar_init(&s_full[i], 1); mbar_init(&p_full[i], 8); mbar_init(&p_half[i], 8); mbar_init(&o_done[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&q_empty[i], 1); mbar_init(&item_full[i], 1); mbar_init(&item_empty[i], 17); s_item[i].h = -1; }
        fence_barrier_init();
        prefetch_map(&qn_map);
        prefetch_map(&qr_map);
        prefetch_map(&k_map);
        prefetch_map(&r_map);
        prefetch_map(&v_map);
    }
    if (warp == 1) tmem_alloc(s_tmem, 512);
    pdl_wait_prior_grid();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *s_tmem;
    // A CTA takes pairs of tiles one after another: the next one's queries and keys are loaded, and its first tile begun, while the second tile
    // of this one is finished (a CTA a pair stood for 5,000 clocks before its first S and 5,000 after its last, of some 75,000).
    RingAt it;
    {
        const int nkc = (p.dn + 63) / 64, nvc = (p.dv + 63) / 64;        // chunks of keys (and one of rotated parts), of values
        if (warp >= 4) {
            // ========================================= softmax: two threads to a row, 64 columns each (one thread's 128 took 2000 clocks from S to P,
            // on the way from one product of a tile to the next)
            const int i = (warp - 4) >> 3, half = ((warp - 4) >> 2) & 1, wq = warp & 3, row = i * 128 + wq * 32 + lane;
            const uint32_t st = tmem + ((uint32_t)(wq * 32) << 16) + i * 128, ot = st + 256;
            const float k2 = p.scale * 1.4426950408889634f;
            float* my_max = s_max + (i * 2 + half) * 128 + wq * 32 + lane;
            float* their_max = s_max + (i * 2 + 1 - half) * 128 + wq * 32 + lane;
            uint32_t done = 0;                                           // tiles, of all items
            // (An item's place is given back when it is done: what of it is needed at its end takes no registers in between.)
            while (true) {
            role_wait(&item_full[it.slot], it.phase, p.status);
            const Item& x = s_item[it.slot];
            if (x.h < 0) break;
            auto item_done = [&]() {
                __syncwarp();
                if (lane == 0) mbar_arrive(&item_empty[it.slot]);
                it.next(2);
            };
            const int pos = x.pos0 + row, mine = x.n[i];                 // positions 0 .. pos are seen
            float m = -INFINITY, l = 0.f;                                // (l: of this thread's columns)
            for (int t = 0; t < mine; ++t, ++done) {
                const int in_half = __ldcg(p.halves + (x.kv0 >> 7) + t);        // (there long before it is used)
                role_wait(&s_full[i], done & 1, p.status);
                tc_fence_after();
                const int seen = pos + 1 - t * 128 - half * 64;          // of these columns
                const bool part = __any_sync(0xFFFFFFFFu, seen < 64);
                uint32_t v[64];
                tmem_ld(st + half * 64, v);
                float mt;
                {
                    float a[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    if (part) {
#pragma unroll
                        for (int j = 0; j < 64; ++j)
                            if (j >= seen) v[j] = 0xFF800000u;
                    }
#pragma unroll
                    for (int j = 0; j < 64; j += 8)
#pragma unroll
                        for (int y = 0; y < 4; ++y) a[y] = max3(a[y], __uint_as_float(v[j + y]), __uint_as_float(v[j + 4 + y]));
                    mt = max3(max3(a[0], a[1], a[2]), a[3], a[3]);
                    // the other half's (whose reader is done with it before the next S can be there: it takes all of P)
                    *my_max = mt;
                    tc_fence_before();
                    barrier_sync(1 + i, 256);
                    tc_fence_after();
                    mt = max3(mt, *their_max, *their_max) * k2;          // (the scale is positive)
                    if (!(mt < INFINITY)) { l = __int_as_float(0x7FFFFFFF); mt = -INFINITY; }      // NaN or infinity among them: so is the row
                    mt = fmaxf(m, mt);
                }
                if (t == 0) m = mt;
                const bool grown = mt > m + 8.f;
                if (__any_sync(0xFFFFFFFFu, grown)) {                    // (the same rows in both halves; each takes every second 16 columns of O)
                    const float alpha = grown ? exp2_approx(m - mt) : 1.f;
                    if (grown) { m = mt; l *= alpha; }
                    role_wait(&o_done[i], (done - 1) & 1, p.status);
                    tc_fence_after();
                    for (int c = half * 16; c < p.dv; c += 32) {
                        uint32_t o[16];
                        tmem_ld(ot + c, o);
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
                        tmem_st(ot + c, o);
                    }
                    tmem_st_wait();
                }
                // (2^4 times 2^(s - m): what fp16 cuts off is then 2^-29 of the largest weight, below what sums of 32 bits lose anyway.  No more than
                // that: values up to 2^123 stay finite on their way)
                const float mm = m == -INFINITY ? 0.f : 4.f - m;
                float2 sum = make_float2(0.f, 0.f);
                auto weights = [&](auto pair) {
#pragma unroll
                    for (int c = 0; c < 64; c += 32) {
                        uint32_t o[16];
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const float x = exp2_approx(fmaf(__uint_as_float(v[c + j]), k2, mm)), y = exp2_approx(fmaf(__uint_as_float(v[c + j + 1]), k2, mm));
                            sum.x += x;
                            sum.y += y;
                            o[j / 2] = pair(x, y);
                        }
                        tmem_st(st + half * 32 + c / 2, o);              // (over the scores of the first half, which all have read: the barrier above)
                        if (c == 0) {                                    // (half of P V can begin)
                            tmem_st_wait();
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&p_half[i]);
                        }
                    }
                };
                if (in_half != 0) weights([](float a, float b) { return half_pair(a, b); });
                else weights([](float a, float b) { return bf16_pair(a, b); });
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[i]);
                l += sum.x + sum.y;
            }
            // ---- out
            // (straight from the registers, a sector at a time: by way of the queries' place, for whole lines, the next queries came 6,000 clocks later)
            uint16_t* const out = row < x.rows ? static_cast<uint16_t*>(p.y) + ((size_t)(x.token + row) * p.heads + x.h) * p.dv : nullptr;
            if (mine == 0) {                                             // rows that see nothing, or none
                if (out != nullptr)
                    for (int c = half * 16; c < p.dv; c += 32) {
                        *reinterpret_cast<uint4*>(out + c) = make_uint4(0, 0, 0, 0);
                        *reinterpret_cast<uint4*>(out + c + 8) = make_uint4(0, 0, 0, 0);
                    }
                item_done();
                continue;
            }
            // (A sum goes to the place of the other half's maximum, whose one reader is this thread: behind the last tile nothing tells that the
            // other has read this one's.)
            *their_max = l;
            barrier_sync(1 + i, 256);
            l += *my_max;
            barrier_sync(1 + i, 256);                                    // (the next item's maxima go there)
            const float inv = l == 0.f ? 0.f : 1.f / l;
            role_wait(&o_done[i], (done - 1) & 1, p.status);
            tc_fence_after();
            for (int c = half * 16; c < p.dv; c += 32) {                 // (the two halves take every second 16 columns)
                uint32_t v[16], o[8];
                tmem_ld(ot + c, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float a = l == 0.f ? 0.f : __uint_as_float(v[2 * j]) * inv, b = l == 0.f ? 0.f : __uint_as_float(v[2 * j + 1]) * inv;
                    if (p.out_dtype == EDG_F16) {
                        const __half2 y = __floats2half2_rn(a, b);
                        o[j] = *reinterpret_cast<const uint32_t*>(&y);
                    } else o[j] = bf16_pair(a, b);
                }
                if (out != nullptr) {
                    *reinterpret_cast<uint4*>(out + c) = make_uint4(o[0], o[1], o[2], o[3]);
                    *reinterpret_cast<uint4*>(out + c + 8) = make_uint4(o[4], o[5], o[6], o[7]);
                }
                __syncwarp();
            }
            tc_fence_before();
            item_done();
            }
        } else {
            if (warp == 0) {
            // ========================================= loads
            uint32_t begun[2] = {0, 0};
            Item x = {};
            auto queries = [&](int i) {
                if (x.n[i] == 0) return;
                role_wait(&q_empty[i], (begun[i]++ & 1) ^ 1, p.status);
                if (elected()) {
                    mbar_expect_tx(&q_full[i], (nkc + 1) * kChunk);
                    for (int c = 0; c < nkc; ++c) tma_3d(sb + kPQ + (i * 3 + c) * kChunk, &qn_map, c * 64, x.h, x.token + i * 128, &q_full[i]);
                    tma_3d(sb + kPQ + (i * 3 + nkc) * kChunk, &qr_map, 0, x.h, x.token + i * 128, &q_full[i]);
                }
                __syncwarp();
            };
            // Groups (the keys of a tile, its values, the next keys ...) take the ring's chunks in turn and are read in that order: a group waits
            // until those before it have left it room.
            RingAt f, old;
            int at = 0, held = 0;                                        // place of the next chunk; chunks that have not been read
            bool old_keys = true;
            auto room_left = [&]() {
                role_wait(&kv_empty[old.slot], old.phase, p.status);
                held -= old_keys ? nkc + 1 : nvc;
                old_keys = !old_keys;
                old.next(kPRing);
            };
            auto room = [&](int chunks) {
                held += chunks;
                while (held > kPRing) room_left();
            };
            // ---- work: the last pairs of a sequence see the most, they go first.  (The next one is taken when all of this one's loads are on their
            // way, not before: taken a whole pair ahead, the last CTA had 82 of 67 tiles on average.)
            const int pairs = p.q_pre[p.s.n], total = pairs * p.heads;
            auto next_item = [&]() {
                int w = 0;
                if (lane == 0) w = atomicAdd(p.next, 1);
                w = __shfl_sync(0xFFFFFFFFu, w, 0);
                x.h = -1;
                if (w >= 0 && w < total) {
                    const int pair = pairs - 1 - w / p.heads, seq = min(find_sequence(p.q_pre, p.s.n, pair, lane), p.s.n - 1);
                    const XSeq q = xsequence(p, seq);
                    const int r0 = (pair - p.q_pre[seq]) * 256;
                    x.h = w % p.heads;
                    x.kv0 = p.kv_pre[seq] * 128;
                    const bool fits = x.kv0 + q.tiles * 128 <= p.rows;
                    x.pos0 = q.len - q.fresh + r0;                       // position of the pair's first row
                    x.token = q.a + r0;
                    x.rows = fits ? q.fresh - r0 : 0;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {                        // tiles of 128 positions that a tile of rows sees something of
                        const int last = min(r0 + i * 128 + 127, q.fresh - 1);      // its last row
                        x.n[i] = fits && r0 + i * 128 < q.fresh ? max((q.len - q.fresh + last + 128) >> 7, 0) : 0;
                    }
                }
                role_wait(&item_empty[it.slot], it.phase ^ 1, p.status);
                if (lane == 0) {
                    s_item[it.slot] = x;
                    mbar_arrive(&item_full[it.slot]);
                }
                __syncwarp();
                it.next(2);
                return x.h >= 0;
            };
            while (next_item()) {
            const int nt = max(x.n[0], x.n[1]);
            queries(0);
            for (int t = 0; t < nt; ++t) {
                const int row = x.kv0 + t * 128;
                room(nkc + 1);
                if (elected()) {
                    mbar_expect_tx(&kv_full[f.slot], (nkc + 1) * kChunk);
                    for (int c = 0; c < nkc; ++c) tma_3d(sb + kPRingAt + ((at + c) & (kPRing - 1)) * kChunk, &k_map, c * 64, row, x.h, &kv_full[f.slot]);
                    tma_2d(sb + kPRingAt + ((at + nkc) & (kPRing - 1)) * kChunk, &r_map, 0, row, &kv_full[f.slot]);
                }
                __syncwarp();
                at = (at + nkc + 1) & (kPRing - 1);
                f.next(kPRing);
                if (t == 0) queries(1);                         // (free later than the first tile's, and needed later)
                room(nvc);
                if (elected()) {
                    mbar_expect_tx(&kv_full[f.slot], nvc * kChunk);
                    for (int c = 0; c < nvc; ++c) tma_3d(sb + kPRingAt + ((at + c) & (kPRing - 1)) * kChunk, &v_map, c * 64, row, x.h, &kv_full[f.slot]);
                }
                __syncwarp();
                at = (at + nvc) & (kPRing - 1);
                f.next(kPRing);
            }
            }
            while (held > 0) room_left();                                // (no arrival may come after the block's end)
            for (int i = 0; i < 2; ++i) role_wait(&q_empty[i], (begun[i] & 1) ^ 1, p.status);
        } else if (warp == 1) {
            // ========================================= products, by one thread: for each tile of rows O += P V of a tile of positions, then S of the
            // next.  (What it does between two products is time in which the tensor cores wait: they hold two or three products of 65 clocks.)
            if (elected()) {
                const uint32_t id_s = idesc_bf16(128, 128), id_any = idesc_bf16(128, p.dv, false, true);
                const uint32_t dq = desc_lo(sb + kPQ), dk = desc_lo(sb + kPRingAt), dv = desc_lo(sb + kPRingAt, kChunk);
                const int rks = p.dr / 16;
                RingAt f;                                                // the next group (keys or values) to wait for
                int at = 0, read = 0;                                    // ring place of the next group; groups that have been read
                uint32_t tiles[2] = {0, 0}, begun[2] = {0, 0};           // tiles of positions, tiles of rows with any
                auto take = [&](int chunks) { const int a = at; at = (at + chunks) & (kPRing - 1); return a; };
                auto loaded = [&](RingAt g) {
                    role_wait(&kv_full[g.slot], g.phase, p.status);
                    tc_fence_after();
                };
                auto release = [&]() { umma_done(&kv_empty[read++ & (kPRing - 1)]); };
                auto scores = [&](int i, int k, bool last) {
                    const uint32_t st = tmem + i * 128;
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        if (c < nkc) {
                            const uint32_t a = dq + (((i * 3 + c) * kChunk) >> 4), b = dk + ((((k + c) & (kPRing - 1)) * kChunk) >> 4);
#pragma unroll
                            for (int s = 0; s < 4; ++s) umma_ss(st, a + s * 2, b + s * 2, id_s, c + s > 0);
                        }
                    const uint32_t a = dq + (((i * 3 + nkc) * kChunk) >> 4), b = dk + ((((k + nkc) & (kPRing - 1)) * kChunk) >> 4);
#pragma unroll
                    for (int s = 0; s < 4; ++s)
                        if (s < rks) umma_ss(st, a + s * 2, b + s * 2, id_s, true);
                    umma_done(&s_full[i]);
                    if (last) umma_done(&q_empty[i]);
                };
                while (true) {
                    role_wait(&item_full[it.slot], it.phase, p.status);
                    const int n[2] = {s_item[it.slot].n[0], s_item[it.slot].n[1]};
                    const bool end = s_item[it.slot].h < 0;
                    const int first = s_item[it.slot].kv0 >> 7;
                    mbar_arrive(&item_empty[it.slot]);
                    it.next(2);
                    if (end) break;
                    const int nt = max(n[0], n[1]);
                    int k = 0;
                    if (nt > 0) {
                        k = take(nkc + 1);
                        loaded(f);
                        f.next(kPRing);
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            if (n[i] > 0) {
                                role_wait(&q_full[i], begun[i]++ & 1, p.status);
                                tc_fence_after();
                                scores(i, k, n[i] == 1);
                            }
                        release();
                    }
                    for (int t = 0; t < nt; ++t) {
                        const uint32_t types = __ldcg(p.halves + first + t) != 0 ? kIdescTypes : 0u, id_o = id_any - types;
                        const int v = take(nvc);
                        const RingAt fv = f;                             // the values, and the next keys
                        f.next(kPRing);
                        const bool more = t + 1 < nt;
                        const RingAt fk = f;
                        if (more) { k = take(nkc + 1); f.next(kPRing); }
                        const bool whole = nvc == 1 || v + 1 < kPRing;   // (values that go round the ring's end: a chunk at a time)
                        const uint32_t b = dv + ((v * kChunk) >> 4);
                        bool seen_v = false, seen_k = false;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t o = tmem + 256 + i * 128, pt = tmem + i * 128;
                            if (t < n[i]) {
                                if (!seen_v) loaded(fv);
                                seen_v = true;
                                role_wait(&p_half[i], tiles[i] & 1, p.status);
                                tc_fence_after();
                                if (whole) {                             // (16 positions each: 0-31, 64-95, then the others)
#pragma unroll
                                    for (int x = 0; x < 8; ++x) {
                                        const int s = (x & 1) | (x & 2) << 1 | (x & 4) >> 1;
                                        if (x == 4) {
                                            role_wait(&p_full[i], tiles[i]++ & 1, p.status);
                                            tc_fence_after();
                                        }
                                        umma_ts(o, pt + s * 8, b + ((s * 2048) >> 4), id_o, t + x > 0);
                                    }
                                } else {
                                    role_wait(&p_full[i], tiles[i]++ & 1, p.status);
                                    tc_fence_after();
                                    const uint32_t id0 = idesc_bf16(128, 64, false, true) - types, id1 = idesc_bf16(128, p.dv - 64, false, true) - types;
#pragma unroll
                                    for (int s = 0; s < 8; ++s) {
                                        umma_ts(o, pt + s * 8, b + ((s * 2048) >> 4), id0, t + s > 0);
                                        umma_ts(o + 64, pt + s * 8, dv + ((s * 2048) >> 4), id1, t + s > 0);
                                    }
                                }
                                umma_done(&o_done[i]);
                            }
                            if (i == 1) release();                       // (the values)
                            if (t + 1 < n[i]) {
                                if (!seen_k) loaded(fk);
                                seen_k = true;
                                scores(i, k, t + 2 == n[i]);
                            }
                        }
                        if (more) release();
                    }
                }
            }
            __syncwarp();
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_free(tmem, 512);
}

struct ExpandedLayout { int rows; size_t q_pre, kv_pre, next, range, halves, K, V, Rp, bytes; };

ExpandedLayout expanded_layout(const edg_latent_desc& d, int n_seqs, int T, int64_t total_len) {
    ExpandedLayout L;
    const int64_t with = n_seqs < T ? n_seqs : T, rows = (total_len + 127) / 128 * 128 + 128 * with;
    L.rows = (int)(rows < 0x7FFFFF00 ? rows : 0x7FFFFF00);
    L.q_pre = 0;
    L.kv_pre = round_up(((size_t)n_seqs + 1) * 4, 256);
    L.next = 2 * L.kv_pre;
    L.range = L.next + 256;
    L.halves = L.range + kScan * 4;
    L.Rp = round_up(L.halves + (size_t)rows / 128 * 4, 256);
    L.K = L.Rp + (size_t)rows * 128;
    L.V = round_up(L.K + (size_t)rows * d.heads * d.d_nope * 2, 256);
    L.bytes = round_up(L.V + (size_t)rows * d.heads * d.d_v * 2, 256);
    return L;
}

}  // namespace

size_t expanded_workspace(const edg_latent_desc& d, int n_seqs, int T, int64_t total_len) { return expanded_layout(d, n_seqs, T, total_len).bytes; }

int32_t run_expanded(const edg_latent_desc& d, const LatentSeqs& s, int max_new, int64_t total_len, int more_than, const void* q, const void* q_rope,
                     const void* W_uk, const void* W_uv, const void* cache, void* y, int32_t* status, void* scratch, cudaStream_t st) {
    const ExpandedLayout L = expanded_layout(d, s.n, s.T, total_len);
    uint8_t* ws = static_cast<uint8_t*>(scratch);
    ExpandedParams p = {};
    p.s = s;
    p.cache = static_cast<const uint16_t*>(cache);
    p.K = reinterpret_cast<uint16_t*>(ws + L.K);
    p.V = reinterpret_cast<uint16_t*>(ws + L.V);
    p.Rp = reinterpret_cast<uint16_t*>(ws + L.Rp);
    p.q_pre = reinterpret_cast<int32_t*>(ws + L.q_pre);
    p.kv_pre = reinterpret_cast<int32_t*>(ws + L.kv_pre);
    p.next = reinterpret_cast<int32_t*>(ws + L.next);
    p.W_uv = static_cast<const uint16_t*>(W_uv);
    p.w_range = reinterpret_cast<int32_t*>(ws + L.range);
    p.halves = reinterpret_cast<int32_t*>(ws + L.halves);
    p.y = y;
    p.status = status;
    p.heads = d.heads;
    p.dn = d.d_nope;
    p.dr = d.d_rope;
    p.dv = d.d_v;
    p.dl = d.d_latent;
    p.out_dtype = d.out_dtype;
    p.rows = L.rows;
    p.more_than = more_than;
    p.max_new = max_new;
    p.total_len = total_len;
    p.scale = d.scale;
    // the heads of a tile of positions are shared out so that the CTAs' rounds take the least, a CTA's start counted as a head
    const int64_t tiles = L.rows / 128;
    int64_t least = 0;
    for (int x = 1; x <= d.heads; ++x) {
        const int64_t cost = (tiles * x + kSms - 1) / kSms * ((d.heads + x - 1) / x + 1);
        if (x == 1 || cost < least) { least = cost; p.splits = x; }
    }
    static OncePerDevice once;
    EDG_CUDA_TRY(once([] {
        const cudaError_t e = allow_smem(kXBytes, expand_kernel);
        return e == cudaSuccess ? allow_smem(kPBytes, prompt_kernel) : e;
    }));
    CUtensorMap c_map, uk_map, uv_map, qn_map, qr_map, k_map, r_map, v_map;
    const uint64_t row = (uint64_t)latent_row(d), dl = (uint64_t)d.d_latent, H = (uint64_t)d.heads, dn = (uint64_t)d.d_nope, dr = (uint64_t)d.d_rope,
                   dv = (uint64_t)d.d_v, rows = (uint64_t)L.rows, T = (uint64_t)s.T, ldq = (uint64_t)latent_ldq(d);
    {
        const uint64_t dims[2] = {row, (uint64_t)d.n_pages * d.page};
        const uint32_t box[2] = {64, (uint32_t)(d.page < 128 ? d.page : 128)};
        EDG_CUDA_TRY(make_map(&c_map, cache, 2, dims, &row, box));
    }
    {
        const uint64_t dims[2] = {dl, H * dn};
        const uint32_t box[2] = {64, (uint32_t)dn};
        EDG_CUDA_TRY(make_map(&uk_map, W_uk, 2, dims, &dl, box));
    }
    {
        const uint64_t dims[2] = {dl, H * dv};
        const uint32_t box[2] = {64, (uint32_t)dv};
        EDG_CUDA_TRY(make_map(&uv_map, W_uv, 2, dims, &dl, box));
    }
    const uint32_t rows128[3] = {64, 128, 1}, tokens128[3] = {64, 1, 128};
    {
        const uint64_t dims[3] = {dn, H, T}, strides[2] = {dn + dr, ldq};
        EDG_CUDA_TRY(make_map(&qn_map, q, 3, dims, strides, tokens128));
    }
    {
        const uint64_t dims[3] = {dr, H, T}, own[2] = {dr, H * dr}, in_q[2] = {dn + dr, ldq};
        EDG_CUDA_TRY(make_map(&qr_map, q_rope != nullptr ? q_rope : static_cast<const uint16_t*>(q) + dn, 3, dims, q_rope != nullptr ? own : in_q, tokens128));
    }
    {
        const uint64_t dims[3] = {dn, rows, H}, strides[2] = {dn, rows * dn};
        EDG_CUDA_TRY(make_map(&k_map, p.K, 3, dims, strides, rows128));
    }
    {
        const uint64_t dims[3] = {dv, rows, H}, strides[2] = {dv, rows * dv};
        EDG_CUDA_TRY(make_map(&v_map, p.V, 3, dims, strides, rows128));
    }
    {
        const uint64_t dims[2] = {64, rows}, stride = 64;
        EDG_CUDA_TRY(make_map(&r_map, p.Rp, 2, dims, &stride, rows128));
    }
    prompt_plan_kernel<<<1 + kScan, 256, 0, st>>>(p);
    EDG_CUDA_TRY(cudaGetLastError());
    EDG_CUDA_TRY(launch_pdl(expand_kernel, dim3((unsigned)tiles, p.splits), kXThreads, kXBytes, st, p, c_map, uk_map, uv_map));
    const int64_t pairs = (int64_t)d.heads * (s.T / 256 + (s.n < s.T ? s.n : s.T));       // at most
    EDG_CUDA_TRY(launch_pdl(prompt_kernel, dim3((unsigned)(pairs < kSms ? pairs : kSms)), kPThreads, kPBytes, st, p, qn_map, qr_map, k_map, r_map, v_map));
    return EDG_OK;
}

}  // namespace edg
