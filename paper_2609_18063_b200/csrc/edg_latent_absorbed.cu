// Latent attention, absorbed form: queries are brought to the latent space, and every cache row is read once for all heads.
//
//     q_lat[t,h] = W_uk[h]^T q_nope            (absorb_kernel)
//     s = scale (q_lat . c_j + q_rope . p_j),  O = sum_j 2^(s_j - m) c_j,  l = sum_j 2^(s_j - m)     (absorbed_kernel, over pieces of a sequence)
//     y[t,h] = W_uv[h] (sum over pieces of O) / (sum of l)                                           (combine_kernel)
//
// A sequence's (row, head) pairs are the rows of one matrix product with its cache rows: 2 (2 d_l + d_r) operations a pair and
// position against 2 (d_l + d_r) bytes a position -- 32 rows are bound by HBM, 128 by either.  absorbed_kernel gives a CTA R = 16, 32 or 64 rows
// and streams tiles of 64 positions through shared memory by TMA.  With so few rows the second product is turned round: S = Q C^T
// has the rows along M (64, of which R count), O^T = C^T P^T the latent dimension along M (128 at a time) and the rows along N, so that
// O of all 512 columns takes 4 R columns of tensor memory and no lane of it idles.  C is both operands from one copy: K-major in the first
// product, MN-major in the second.  Eight warps take S, two to 16 rows with half of the columns each, which exchange maxima once a tile.  O is
// rescaled only when a row's maximum has grown by more than 2^8 since it was last (p stays below 2^8, l and O are fp32).
//
// All positions of a batch form one line of tiles, sequence after sequence; groups of CTAs (a CTA per R rows of a sequence, side by side
// on the same tiles, which the second then finds in L2) take equal stretches of it, whatever the lengths.  What a group has of a sequence is a piece;
// combine_kernel adds them up in order.
//
// Rounded to bf16, by 2^-8 of a value at most: q_lat and p, which are operands beside the cache's bf16 (l sums p as it was rounded).  O, m and l
// are fp32 throughout; the latent sums go into the last product as two bf16 parts, 16 bits in all.
//
// Of the cache, 512 + 64 columns: 8 sequences of 65,536 positions, 128 heads (R = 64, two CTAs side by side) 219 to 252 us, by the box -- 3,000 clocks a tile, of which the
// products take 2,100 and shared memory 2,500 (36 products of 37 clocks for S, whose M = 64 is half of what the tensor cores take; 16 of 49
// for O; the copies of 74 KB); 32 sequences of 1 to 8,191, 32 heads (R = 32) 52 to 54 us -- the tiles by themselves come at 6.5 TB/s (16 us), the
// rest is absorb_kernel (9), the first tile (6) and combine_kernel (15, of W_uv and the code's first fetch more than of the pieces: half as
// many rows to a CTA took as long).
#include "edg_latent.cuh"
#include "edg_mma.cuh"
#include "edg_umma.cuh"

namespace edg {

constexpr int kGroupMost = 8;               // CTAs side by side at most; sequences of more rows come in several units
constexpr int kPiece = 2;                   // tiles that a piece costs beside its own: queries, epilogue, nothing overlapped
constexpr int kSms = 148;                   // CTAs of the attention kernel: one to an SM

inline int absorbed_rows(int64_t most_rows) { return most_rows <= 16 ? 16 : (most_rows <= 32 ? 32 : 64); }

struct AbsorbedParams {
    LatentSeqs s;
    const uint16_t *q, *q_rope, *W_uk, *W_uv;
    uint16_t* q_lat;            // [T * heads][dl + 64], the rotated part padded with zeros
    float* part;                // [slots][group][R][dl]
    float2* ml;                 // [slots][group][R]: maximum (in powers of two), sum
    long long* tile_pre;        // [n + 1] tiles before a sequence
    int32_t* unit_pre;          // [n + 1] units before it
    int32_t* row_pre;           // [n + 1] new rows before it, of the sequences that are taken
    void* y;
    int32_t* status;
    int heads, dn, dr, dv, dl, out_dtype, hr;
    int64_t ldq, ldr;
    float scale;
    int R, group, groups, max_slots;
    int max_new, most;          // the caller's bound; sequences of up to `most` new rows are taken
    long long total_len;        // the caller's bound on the sum of lens
};

namespace {

struct Seq { int a, rows, len, fresh, units, kt; };     // first new row, (row, head) pairs, positions, new rows, units, tiles of 64 positions
__device__ __forceinline__ Seq sequence(const AbsorbedParams& p, int i) {
    Seq q;
    q.a = min(max(p.s.cu[i], 0), p.s.T);
    q.fresh = max(min(p.s.cu[i + 1], p.s.T) - q.a, 0);
    q.len = min(max(p.s.lens[i], 0), p.s.max_pages << p.s.page_shift);
    q.rows = q.fresh <= p.most ? q.fresh * p.heads : 0;
    q.units = ((q.rows + p.R - 1) / p.R + p.group - 1) / p.group;
    q.kt = (q.len + 63) >> 6;
    return q;
}
// places on the line that a unit takes: its tiles, behind kPiece that stand for what a piece costs beside them; and a group's share of a line of W
__device__ __forceinline__ long long unit_length(const Seq& q) { return q.kt > 0 ? q.kt + kPiece : 0; }
// (quotients of 64 bits take some hundred clocks: nearly all fit 32)
__device__ __forceinline__ long long quotient(long long a, long long b) {
    return ((a | b) >> 31) == 0 ? (long long)((unsigned)a / (unsigned)b) : a / b;
}
__device__ __forceinline__ long long stretch(long long W, int groups) { return quotient(W + groups - 1, groups); }

// ---------------------------------------------------------------- queries to the latent space

// Prefix sums over the sequences, and the caller's bounds: 128 threads.
__device__ __forceinline__ void plan_sequences(const AbsorbedParams& p) {
        __shared__ long long s_t[128], s_l[128];
        __shared__ int s_u[128], s_r[128];
        const int tid = threadIdx.x, per = (p.s.n + 127) / 128, i0 = min(tid * per, p.s.n), i1 = min(i0 + per, p.s.n);
        long long t = 0, len = 0;
        int u = 0, rows = 0;
        bool ok = tid != 0 || (p.s.cu[0] == 0 && p.s.cu[p.s.n] <= p.s.T);
        for (int i = i0; i < i1; ++i) {
            const Seq q = sequence(p, i);
            t += q.units * unit_length(q);
            u += q.units;
            rows += q.rows > 0 ? q.fresh : 0;
            len += q.len;
            ok = ok && p.s.cu[i + 1] >= p.s.cu[i] && q.fresh <= p.max_new && q.len >= p.s.lens[i];
        }
        s_l[tid] = len;
        s_t[tid] = t;
        s_u[tid] = u;
        s_r[tid] = rows;
        __syncthreads();
        if (tid == 127)                                                  // (the sum sizes nothing here; it is a bound all the same)
            for (int j = 0; j < 127; ++j) len += s_l[j];
        if (!ok || len > p.total_len) latent_raise(p.status, EDG_E_RANGE);
        t = 0;
        u = rows = 0;
        for (int j = 0; j < tid; ++j) { t += s_t[j]; u += s_u[j]; rows += s_r[j]; }
        for (int i = i0; i < i1; ++i) {
            const Seq q = sequence(p, i);
            p.tile_pre[i] = t;
            p.unit_pre[i] = u;
            p.row_pre[i] = rows;
            t += q.units * unit_length(q);
            u += q.units;
            rows += q.rows > 0 ? q.fresh : 0;
            if (i == p.s.n - 1) { p.tile_pre[p.s.n] = t; p.unit_pre[p.s.n] = u; p.row_pre[p.s.n] = rows; }
        }
}
__global__ void __launch_bounds__(128) plan_kernel(const __grid_constant__ AbsorbedParams p) {
    pdl_launch_dependents();
    plan_sequences(p);
}

// A CTA: 64 latent columns of one head, up to 64 rows.  Where every sequence is taken the last CTA of the grid makes the prefix sums; else
// plan_kernel has made them, and rows are counted over the sequences that are taken.
__global__ void __launch_bounds__(128) absorb_kernel(const __grid_constant__ AbsorbedParams p) {
    pdl_launch_dependents();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
    const int ctiles = p.dl / 64;
    const bool all = p.most >= p.max_new;
    if (all && blockIdx.x == gridDim.x - 1) {
        if (blockIdx.y == 0) plan_sequences(p);
        return;
    }
    __shared__ int s_row[64];                                           // new rows of this CTA, or -1
    if (!all) {
        pdl_wait_prior_grid();
        const int rows = p.row_pre[p.s.n];
        if ((int)blockIdx.y * 64 >= rows) return;
        if (tid < 64) {
            const int a = blockIdx.y * 64 + tid;
            int lo = 0, hi = p.s.n;                                      // ends row_pre[1..n] that are <= a
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (p.row_pre[mid + 1] <= a) lo = mid + 1; else hi = mid;
            }
            s_row[tid] = lo < p.s.n ? p.s.cu[lo] + a - p.row_pre[lo] : -1;
        }
    } else if (tid < 64) {
        const int a = blockIdx.y * 64 + tid;
        s_row[tid] = a < p.s.T ? a : -1;
    }
    constexpr int kPitch = 72;                                          // elements of a row of W in shared memory: 64 and padding
    __shared__ __align__(16) uint16_t s_w[128 * kPitch];
    const int h = blockIdx.x / ctiles, c0 = (blockIdx.x % ctiles) * 64, row = p.dl + 64;
    {
        uint4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int n = k * 16 + (tid >> 3), c = (tid & 7) * 8;
            if (n < p.dn) v[k] = __ldg(reinterpret_cast<const uint4*>(p.W_uk + ((size_t)h * p.dn + n) * p.dl + c0 + c));
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k * 16 < p.dn) *reinterpret_cast<uint4*>(s_w + (k * 16 + (tid >> 3)) * kPitch + (tid & 7) * 8) = v[k];
    }
    __syncthreads();
    if (c0 == 0)                                                        // the rotated part, zeros behind it
        for (int i = tid; i < 64 * 8; i += 128) {
            const int t = s_row[i >> 3], c = (i & 7) * 8;
            if (t < 0) break;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (c < p.dr) v = *reinterpret_cast<const uint4*>(p.q_rope + (size_t)t * p.ldr + h * p.hr + c);
            *reinterpret_cast<uint4*>(p.q_lat + ((size_t)t * p.heads + h) * row + p.dl + c) = v;
        }
    const int ks = p.dn / 16;
    for (int t0 = 0; t0 < 64 && s_row[t0] >= 0; t0 += 16) {
        float d[2][4] = {};
        const int ra = s_row[t0 + g], rb = s_row[t0 + g + 8];
        const bool r0 = ra >= 0, r1 = rb >= 0;
        const uint16_t* q0 = p.q + (size_t)max(ra, 0) * p.ldq + h * (p.dn + p.dr) + 2 * t4;
        const uint16_t* q1 = p.q + (size_t)max(rb, 0) * p.ldq + h * (p.dn + p.dr) + 2 * t4;
#pragma unroll 4
        for (int k = 0; k < ks; ++k) {
            const uint32_t a0 = r0 ? *reinterpret_cast<const uint32_t*>(q0 + k * 16) : 0u, a1 = r1 ? *reinterpret_cast<const uint32_t*>(q1 + k * 16) : 0u;
            const uint32_t a2 = r0 ? *reinterpret_cast<const uint32_t*>(q0 + k * 16 + 8) : 0u, a3 = r1 ? *reinterpret_cast<const uint32_t*>(q1 + k * 16 + 8) : 0u;
            uint32_t b[4];                                              // k rows 0-7 and 8-15 of columns 0-7, then of columns 8-15
            const uint32_t at = smem_u32(s_w + (k * 16 + (lane & 15)) * kPitch + warp * 16 + (lane >> 4) * 8);
            asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(b[0]), "=r"(b[1]), "=r"(b[2]), "=r"(b[3]) : "r"(at));
            mma16816_bf16(d[0], a0, a1, a2, a3, b[0], b[1]);
            mma16816_bf16(d[1], a0, a1, a2, a3, b[2], b[3]);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int c = c0 + warp * 16 + j * 8 + 2 * t4;
            if (r0) *reinterpret_cast<uint32_t*>(p.q_lat + ((size_t)ra * p.heads + h) * row + c) = bf16_pair(d[j][0], d[j][1]);
            if (r1) *reinterpret_cast<uint32_t*>(p.q_lat + ((size_t)rb * p.heads + h) * row + c) = bf16_pair(d[j][2], d[j][3]);
        }
    }
}

// ---------------------------------------------------------------- attention over pieces

constexpr int kThreads = 384;               // warps 0 and 3 load, 1 and 2 issue products, 4-11 softmax and epilogue
constexpr uint32_t kUnit = 16384, kRope = 8192;      // 64 positions x 128 latent columns; x 64 rotated ones

constexpr int kFull = 4;                    // "tile is there" barriers: more than tiles that fit the ring of rotated parts

// Shared memory by R: Q [dl/64 + 1 chunks][R rows][128 bytes], P [R][128 bytes], rings of rotated parts and of units of 128 columns.
template <int R> struct Plan {
    static constexpr int NV = R == 64 ? 8 : (R == 32 ? 10 : 11), NR = R == 64 ? 2 : 3;
    static constexpr uint32_t q = 0, p = 9 * R * 128, rope = p + R * 128, unit = rope + NR * kRope, bars = unit + NV * kUnit;
    static constexpr uint32_t alpha = bars + (NV + NR + 2 * kFull + 12) * 8, most = alpha + 64 * 4, end = most + 2 * 2 * 64 * 4, bytes = end + 1024;
    static constexpr uint32_t columns = R == 64 ? 512 : 256;            // of tensor memory: S twice 64, O 4 R
    static_assert(bytes <= 227 * 1024, "shared memory");
    static_assert(p % 1024 == 0 && rope % 1024 == 0 && unit % 1024 == 0, "swizzle atoms");
};

// The pieces of a CTA, one after the other; every role walks them for itself.
struct Walk {
    int seq, unit, ug, tile;    // tile: place within the unit's part of the line
    long long left;
    Seq q;
    // the piece
    int row0, rows, t0, t1, slot;
    __device__ __forceinline__ bool next(const AbsorbedParams& p, int g, int r) {
        while (left > 0 && seq < p.s.n) {
            q = sequence(p, seq);
            if (ug >= q.units || q.kt == 0) { unit += q.units - ug; ++seq; ug = 0; tile = 0; continue; }
            const int end = (int)min((long long)q.kt + kPiece, tile + left);
            left -= end - tile;
            t0 = max(tile - kPiece, 0);
            t1 = max(end - kPiece, 0);
            slot = g + unit;
            const int first = (ug * p.group + r) * p.R;
            row0 = q.a * p.heads + first;
            rows = min(q.rows - first, p.R);
            tile = end;
            if (tile == q.kt + kPiece) { tile = 0; ++ug; ++unit; }
            if (rows > 0 && t1 > t0) { first_row = first; return true; }
        }
        return false;
    }
    int first_row;              // row0 within the sequence
};

template <int R>
__global__ void __launch_bounds__(kThreads, 1) absorbed_kernel(const __grid_constant__ AbsorbedParams p, const __grid_constant__ CUtensorMap kv_map,
                                                               const __grid_constant__ CUtensorMap q_map) {
    using P = Plan<R>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    const uint32_t sb = smem_u32(smem);
    uint64_t* v_empty = reinterpret_cast<uint64_t*>(smem + P::bars);     // [NV]
    uint64_t* r_empty = v_empty + P::NV;                                 // [NR]
    uint64_t* t_full = r_empty + P::NR;                                  // [kFull][2]: rotated parts and the first half of the units, the others
    uint64_t* q_full = t_full + 2 * kFull;
    uint64_t* q_empty = q_full + 1;
    uint64_t* s_full = q_empty + 1;                                      // [2]
    uint64_t* s_empty = s_full + 2;                                      // [2]
    uint64_t* p_full = s_empty + 2;
    uint64_t* pv_done = p_full + 1;
    uint64_t* o_empty = pv_done + 1;
    uint32_t* s_tmem = reinterpret_cast<uint32_t*>(o_empty + 1);
    float* s_alpha = reinterpret_cast<float*>(smem + P::alpha);
    float* s_most = reinterpret_cast<float*>(smem + P::most);             // [2][half of the columns][row]
    __shared__ long long s_tiles[kThreads / 32], s_fresh[kThreads / 32], s_from[2];
    __shared__ int s_units[kThreads / 32], s_at[3];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = blockIdx.x / p.group, r = blockIdx.x % p.group;
    if (tid == 0) {
        for (int i = 0; i < P::NV; ++i) mbar_init(&v_empty[i], 1);
        for (int i = 0; i < P::NR; ++i) mbar_init(&r_empty[i], 1);
        for (int i = 0; i < 2 * kFull; ++i) mbar_init(&t_full[i], 1);
        mbar_init(q_full, 1);
        mbar_init(q_empty, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(&s_full[i], 1); mbar_init(&s_empty[i], 8); }
        mbar_init(p_full, 8);
        mbar_init(pv_done, 1);
        mbar_init(o_empty, 8);
        fence_barrier_init();
    }
    if (warp == 1) tmem_alloc(s_tmem, P::columns);
    if (warp == 0 && elected()) { prefetch_map(&kv_map); prefetch_map(&q_map); }
    // ---- this group's stretch of the line of tiles, and the sequence it begins in
    {
        const int per = (p.s.n + kThreads - 1) / kThreads, i0 = min(tid * per, p.s.n), i1 = min(i0 + per, p.s.n);
        long long t = 0, fresh = 0;
        int u = 0;
        for (int i = i0; i < i1; ++i) {
            const Seq q = sequence(p, i);
            t += q.units * unit_length(q);
            u += q.units;
            fresh += q.fresh;
        }
        long long xt = t;
        int xu = u;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long yt = __shfl_up_sync(0xFFFFFFFFu, xt, o);
            const int yu = __shfl_up_sync(0xFFFFFFFFu, xu, o);
            if (lane >= o) { xt += yt; xu += yu; }
            fresh += __shfl_xor_sync(0xFFFFFFFFu, fresh, o);
        }
        if (lane == 31) { s_tiles[warp] = xt; s_units[warp] = xu; s_fresh[warp] = fresh; }
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        long long W = 0, before = xt - t, all_fresh = 0;
        int ub = xu - u;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) { before += s_tiles[w]; ub += s_units[w]; }
            W += s_tiles[w];
            all_fresh += s_fresh[w];
        }
        if (all_fresh > p.s.T) W = 0;                                    // (sequences that overlap: reported, and no end of work otherwise)
        const long long each = stretch(W, p.groups), start = min(each * g, W), end = min(start + each, W);
        if (tid == 0) { s_from[1] = end - start; if (end <= start) { s_from[0] = 0; s_at[0] = s_at[1] = s_at[2] = 0; } }
        if (end > start && t > 0 && before <= start && start < before + t) {
            for (int i = i0; i < i1; ++i) {
                const Seq q = sequence(p, i);
                const long long here = q.units * unit_length(q);
                if (start < before + here) {
                    const int ug = (int)quotient(start - before, unit_length(q));
                    s_at[0] = i;
                    s_at[1] = ug;
                    s_at[2] = ub + ug;
                    s_from[0] = start - before - ug * unit_length(q);
                    break;
                }
                before += here;
                ub += q.units;
            }
        }
        __syncthreads();
    }
    Walk w;
    w.seq = s_at[0];
    w.ug = s_at[1];
    w.unit = s_at[2];
    w.tile = (int)s_from[0];
    w.left = s_from[1];
    const uint32_t tmem = *s_tmem;
    const int NU = p.dl / 128, n1 = (NU + 1) / 2;                        // units of 128 columns; the first half of them

    if (warp == 0 || warp == 3) {
        // ============================================= loads: warp 0 takes the first 64 columns of every unit, the rotated parts and Q, warp 3 the
        // other 64.  A warp issues a copy every 100 clocks, and every 500 with an arrival between two of them (8 KB copies, one SM): so
        // one barrier a tile, and two warps (a page of 16 makes 36 copies of a tile).
        const int br = min(1 << p.s.page_shift, 64), boxes = 64 / br, outside = p.s.n_pages << p.s.page_shift, half = warp == 0 ? 0 : 1;
        RingAt v, ro, f;
        uint32_t q_phase = 1;
        bool waited = false;
        while (w.next(p, g, r)) {
            const int32_t* table = p.s.table + (size_t)w.seq * p.s.max_pages;
            int base = -64, coord = 0;                                   // boxes base .. base + 31 are known, one to a lane
            for (int t = w.t0; t < w.t1; ++t) {
                if ((t + 1) * boxes - base > 32) {
                    base = t * boxes;
                    const int at = (base + lane) * br;                   // first position of the lane's box
                    coord = outside;
                    if (at < w.q.len) {
                        const int pg = table[at >> p.s.page_shift];
                        if (pg >= 0 && pg < p.s.n_pages) coord = (pg << p.s.page_shift) + (at & ((1 << p.s.page_shift) - 1));
                        else latent_raise(p.status, EDG_E_RANGE);
                    }
                }
                int y[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) y[b] = __shfl_sync(0xFFFFFFFFu, coord, (t * boxes - base + min(b, boxes - 1)) & 31);
                role_wait(&r_empty[ro.slot], ro.phase ^ 1, p.status);
                if (half == 0 && elected()) {
                    mbar_expect_tx(&t_full[2 * f.slot], kRope + n1 * kUnit);
                    if (n1 < NU) mbar_expect_tx(&t_full[2 * f.slot + 1], (NU - n1) * kUnit);
#pragma unroll
                    for (int b = 0; b < 4; ++b)
                        if (b < boxes) tma_2d(sb + P::rope + ro.slot * kRope + b * br * 128, &kv_map, p.dl, y[b], &t_full[2 * f.slot]);
                }
                ro.next(P::NR);
                for (int u = 0; u < NU; ++u) {
                    role_wait(&v_empty[v.slot], v.phase ^ 1, p.status);
                    if (elected()) {
#pragma unroll
                        for (int b = 0; b < 4; ++b)
                            if (b < boxes) tma_2d(sb + P::unit + v.slot * kUnit + half * kRope + b * br * 128, &kv_map, u * 128 + half * 64, y[b], &t_full[2 * f.slot + (u >= n1)]);
                    }
                    v.next(P::NV);
                }
                f.next(kFull);
                if (half == 0 && t == w.t0) {                            // (behind the first tile: that does not wait for the kernel before)
                    if (!waited) { pdl_wait_prior_grid(); waited = true; }
                    role_wait(q_empty, q_phase, p.status);
                    q_phase ^= 1;
                    if (elected()) {
                        mbar_expect_tx(q_full, (p.dl / 64 + 1) * R * 128);
                        for (int c = 0; c <= p.dl / 64; ++c) tma_2d(sb + P::q + c * R * 128, &q_map, c * 64, w.row0, q_full);
                    }
                }
                __syncwarp();
            }
        }
        if (!waited) pdl_wait_prior_grid();
        if (half == 0) {                                                 // (no arrival of a product may come after the block's end)
            for (int i = 0; i < P::NV; ++i, v.next(P::NV)) role_wait(&v_empty[v.slot], v.phase ^ 1, p.status);
            for (int i = 0; i < P::NR; ++i, ro.next(P::NR)) role_wait(&r_empty[ro.slot], ro.phase ^ 1, p.status);
            role_wait(q_empty, q_phase, p.status);
        }
    } else if (warp == 1) {
        // ============================================= S of every tile, in two halves as they arrive.  (O is another warp's: what queues up
        // behind a product covers two or three of them, a wait costs as much, and each warp's products cover the other's waits.)
        if (elected()) {
            const uint32_t id_s = idesc_bf16(64, 64);
            const uint32_t dq = desc_lo(sb + P::q), dk0 = desc_lo(sb + P::unit), dr0 = desc_lo(sb + P::rope);
            const int rks = p.dr / 16;
            RingAt ks, kr, f;
            int n = 0;                                                       // tiles issued
            uint32_t q_phase = 0;
            while (w.next(p, g, r)) {
                role_wait(q_full, q_phase, p.status);
                q_phase ^= 1;
                for (int t = w.t0; t < w.t1; ++t, ++n) {
                    const int buf = n & 1;
                    role_wait(&s_empty[buf], ((uint32_t)(n >> 1) & 1) ^ 1, p.status);
                    role_wait(&t_full[2 * f.slot], f.phase, p.status);
                    uint32_t at[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (u < NU) {
                            at[u] = dk0 + ((ks.slot * kUnit) >> 4);
                            ks.next(P::NV);
                        }
                    tc_fence_after();
                    const uint32_t d = tmem + buf * 64, dr = dr0 + ((kr.slot * kRope) >> 4);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < rks) umma_ss(d, dq + ((NU * 2 * R * 128 + k * 32) >> 4), dr + ((k * 32) >> 4), id_s, k > 0);
                    umma_done(&r_empty[kr.slot]);
#pragma unroll
                    for (int u = 0; u < 2; ++u)
                        if (u < n1)
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                umma_ss(d, dq + (((u * 2 + (k >> 2)) * R * 128 + (k & 3) * 32) >> 4), at[u] + (((k >> 2) * kRope + (k & 3) * 32) >> 4), id_s, true);
                    if (n1 == NU) {
                        umma_done(&s_full[buf]);
                        if (t == w.t1 - 1) umma_done(q_empty);
                    }
                    if (n1 < NU) {
                        role_wait(&t_full[2 * f.slot + 1], f.phase, p.status);
                        tc_fence_after();
#pragma unroll
                        for (int u = 1; u < 4; ++u)
                            if (u >= n1 && u < NU)
#pragma unroll
                                for (int k = 0; k < 8; ++k)
                                    umma_ss(d, dq + (((u * 2 + (k >> 2)) * R * 128 + (k & 3) * 32) >> 4), at[u] + (((k >> 2) * kRope + (k & 3) * 32) >> 4), id_s, true);
                        umma_done(&s_full[buf]);
                        if (t == w.t1 - 1) umma_done(q_empty);
                    }
                    f.next(kFull);
                    kr.next(P::NR);
                }
            }
        }
        __syncwarp();
    } else if (warp == 2) {
        // ============================================= O += C^T P^T of every tile
        if (elected()) {
            const uint32_t id_o = idesc_bf16(128, R, true, false);
            const uint32_t dp = desc_lo(sb + P::p), dv0 = desc_lo(sb + P::unit, kRope), o0 = tmem + 128;
            RingAt vs;
            int n = 0;
            uint32_t o_phase = 1;
            while (w.next(p, g, r)) {
                role_wait(o_empty, o_phase, p.status);
                o_phase ^= 1;
                for (int t = w.t0; t < w.t1; ++t, ++n) {
                    role_wait(p_full, (uint32_t)n & 1, p.status);            // (whose writers have seen S: the units are there)
                    tc_fence_after();
                    RingAt at[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (u < NU) { at[u] = vs; vs.next(P::NV); }
                    const bool more = t > w.t0;
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (u < NU) {
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                umma_ss(o0 + u * R, dv0 + ((at[u].slot * kUnit + k * 2048) >> 4), dp + ((k * 32) >> 4), id_o, more || k > 0);
                            umma_done(&v_empty[at[u].slot]);
                        }
                    umma_done(pv_done);
                }
            }
        }
        __syncwarp();
    } else if (warp >= 4) {
        // ============================================= softmax, rescaling, epilogue
        // A product of M = 64 leaves its rows in 16 lanes of every 32; a load of that shape gives a lane two rows (gq, gq + 8 of the warp's
        // 16), and of them the columns 8 j + 2 cq and the next.  Two warps share the rows, 32 columns each.
        const int wq = warp & 3, half = (warp >> 2) - 1, gq = lane >> 2, cq = lane & 3;
        const bool mine = wq * 16 < R;
        const uint32_t lanes = (uint32_t)(wq * 32) << 16;
        const float k2 = p.scale * 1.4426950408889634f;
        RingAt vn;                                                       // units of the next tile (to clear rows behind the end)
        int n = 0;
        while (w.next(p, g, r)) {
            float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};      // (l: this lane's share)
            int sees[2];                                                 // positions that a row sees: up to its own
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = wq * 16 + gq + 8 * i;
                sees[i] = mine && row < w.rows ? min(w.q.len, w.q.len - w.q.fresh + (w.first_row + row) / p.heads + 1) : 0;
            }
            // (The first time round these warps go through the motions on whatever tensor memory holds, and forget it: the loads take longer than
            // the fetching of this code, which took 4000 clocks of the first tile.)
            for (int t = n == 0 ? w.t0 - 1 : w.t0; t < w.t1; ++t) {
                const int buf = n & 1;
                const bool dry = t < w.t0, first = t <= w.t0;
                if (!dry) role_wait(&s_full[buf], (uint32_t)(n >> 1) & 1, p.status);
                tc_fence_after();
                if (t == w.t0) { m[0] = m[1] = -INFINITY; l[0] = l[1] = 0.f; }
                float s[2][8], mt[2] = {-INFINITY, -INFINITY};
                if (mine) {
                    uint32_t v[16];
                    tmem_ld_rows16(tmem + lanes + buf * 64 + half * 32, v);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int seen = sees[i] - t * 64 - half * 32 - 2 * cq;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            s[i][2 * j] = __uint_as_float(v[4 * j + 2 * i]) * k2;
                            s[i][2 * j + 1] = __uint_as_float(v[4 * j + 2 * i + 1]) * k2;
                        }
                        if (seen < 26) {                                 // (the last two of the lane's columns are 24 and 25 from its first)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                if (8 * j >= seen) s[i][2 * j] = -INFINITY;
                                if (8 * j + 1 >= seen) s[i][2 * j + 1] = -INFINITY;
                            }
                        }
                        float a = fmaxf(fmaxf(fmaxf(s[i][0], s[i][1]), fmaxf(s[i][2], s[i][3])), fmaxf(fmaxf(s[i][4], s[i][5]), fmaxf(s[i][6], s[i][7])));
                        a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
                        mt[i] = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
                    }
                    if (cq == 0) {
                        s_most[(buf * 2 + half) * 64 + wq * 16 + gq] = mt[0];
                        s_most[(buf * 2 + half) * 64 + wq * 16 + gq + 8] = mt[1];
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && !dry) mbar_arrive(&s_empty[buf]);
                // One barrier brings the other half's maxima and whether any row has grown (which either half of it tells).  A tile later the
                // maxima go to the other buffer, and nobody is two tiles ahead: the barrier again.
                const bool rescale = barrier_or(1, 256, !first && (mt[0] > m[0] + 8.f || mt[1] > m[1] + 8.f)) && !first;      // (-infinity: anything is more)
                if (first || rescale) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        if (mine) mt[i] = fmaxf(mt[i], s_most[(buf * 2 + 1 - half) * 64 + wq * 16 + gq + 8 * i]);
                    if (first) { m[0] = mt[0]; m[1] = mt[1]; }
                }
                if (n > 0) role_wait(pv_done, (uint32_t)(n - 1) & 1, p.status);       // O is complete, P has been read
                if (rescale) {
                    const bool grown0 = mt[0] > m[0] + 8.f, grown1 = mt[1] > m[1] + 8.f;
                    const float a0 = grown0 ? exp2_approx(m[0] - mt[0]) : 1.f, a1 = grown1 ? exp2_approx(m[1] - mt[1]) : 1.f;
                    if (grown0) { m[0] = mt[0]; l[0] *= a0; }
                    if (grown1) { m[1] = mt[1]; l[1] *= a1; }
                    if (mine && cq == 0 && half == 0) { s_alpha[wq * 16 + gq] = a0; s_alpha[wq * 16 + gq + 8] = a1; }
                    barrier_sync(1, 256);
                    tc_fence_after();
                    for (int u = half; u < NU; u += 2)
#pragma unroll
                        for (int c = 0; c < R; c += 16) {
                            uint32_t v[16];
                            tmem_ld(tmem + lanes + 128 + u * R + c, v);
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * s_alpha[c + j]);
                            tmem_st(tmem + lanes + 128 + u * R + c, v);
                        }
                    tmem_st_wait();
                    tc_fence_before();
                }
                if (mine) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float mm = m[i] == -INFINITY ? 0.f : m[i];
                        const int row = wq * 16 + gq + 8 * i;
                        uint8_t* out = smem + P::p + row * 128 + cq * 4;
                        float la = 0.f, lb = 0.f;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {                    // two positions to a word, under the swizzle
                            const uint32_t o = bf16_pair(exp2_approx(s[i][2 * j] - mm), exp2_approx(s[i][2 * j + 1] - mm));
                            la += bf16_lo(o);                            // (what the product sums)
                            lb += bf16_hi(o);
                            *reinterpret_cast<uint32_t*>(out + (((j + half * 4) ^ (row & 7)) * 16)) = o;
                        }
                        l[i] += la + lb;
                    }
                }
                if (dry) continue;
                const int held = w.q.len - t * 64;                       // positions of the tile that exist: clear the rows behind them
                const RingAt vt = vn;
                vn.slot += NU;
                if (vn.slot >= P::NV) vn.slot -= P::NV;
                if (held < 64) {
                    RingAt c = vt;
                    for (int u = 0; u < NU; ++u) {
                        uint8_t* unit = smem + P::unit + c.slot * kUnit;
                        for (int i = held * 8 + (tid - 128); i < 512; i += 256) {
                            *reinterpret_cast<uint4*>(unit + i * 16) = make_uint4(0, 0, 0, 0);
                            *reinterpret_cast<uint4*>(unit + kRope + i * 16) = make_uint4(0, 0, 0, 0);
                        }
                        c.next(P::NV);
                    }
                }
                // Of the new rows themselves some see less than others: one that is not finite is NaN by its score for those that see it, and
                // must not reach the others by their weight of zero.
                const int own = max(w.q.len - w.q.fresh + 1 - t * 64, 0);
                if (own < min(held, 64))
                    for (int i = own + warp - 4; i < min(held, 64); i += 8) {
                        uint32_t most = 0;
                        RingAt c = vt;
                        for (int u = 0; u < NU; ++u, c.next(P::NV))
                            if (lane < 16) most = bf16_magnitudes(most, *reinterpret_cast<const uint4*>(smem + P::unit + c.slot * kUnit + (lane >> 3) * kRope + i * 128 + (lane & 7) * 16));
                        if (__any_sync(0xFFFFFFFFu, bf16_not_finite(most))) {
                            c = vt;
                            for (int u = 0; u < NU; ++u, c.next(P::NV))
                                if (lane < 16) *reinterpret_cast<uint4*>(smem + P::unit + c.slot * kUnit + (lane >> 3) * kRope + i * 128 + (lane & 7) * 16) = make_uint4(0, 0, 0, 0);
                        }
                    }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full);
                ++n;
            }
            // ---- the piece's sums
            role_wait(pv_done, (uint32_t)(n - 1) & 1, p.status);
            tc_fence_after();
            const bool fits = w.slot < p.max_slots;
            const size_t at = ((size_t)w.slot * p.group + r) * R;
            // (the other half's sums by way of the maxima's place: the buffer that the last tile did not use, and the next will)
            float* shared = s_most + (n & 1) * 128;
            float sum[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                sum[i] = group_sum<4>(l[i]);
                if (half == 1 && mine && cq == 0) shared[wq * 16 + gq + 8 * i] = sum[i];
            }
            barrier_sync(1, 256);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = wq * 16 + gq + 8 * i;
                if (fits && half == 0 && cq == 0 && mine && row < w.rows) p.ml[at + row] = make_float2(m[i], sum[i] + shared[row]);
            }
            for (int u = half; u < NU; u += 2)
#pragma unroll
                for (int c = 0; c < R; c += 16) {
                    uint32_t v[16];
                    tmem_ld(tmem + lanes + 128 + u * R + c, v);
                    if (fits)
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (c + j < w.rows) p.part[(at + c + j) * p.dl + u * 128 + wq * 32 + lane] = __uint_as_float(v[j]);
                }
            barrier_sync(1, 256);                                        // (read before the next tile's maxima)
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(o_empty);
        }
    }
    pdl_launch_dependents();
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_free(tmem, P::columns);
}

// ---------------------------------------------------------------- sums of the pieces, and out of the latent space

constexpr int kCombine = 512;

// A CTA: one head of 16 rows.  A warp adds up the pieces of a row and leaves its latent sums in shared memory as two bf16 parts, 16 bits of
// them in all; then every warp takes 32 values of W_uv over a quarter of the latent columns, asked for before anything else (eight values over
// all of them read the sums from shared memory four times as often: 5000 clocks instead of 1500).
__global__ void __launch_bounds__(kCombine, 1) combine_kernel(const __grid_constant__ AbsorbedParams p) {
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float s_weight[16][kSms];
    __shared__ int s_row[16];                                           // new rows of this CTA, or -1
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
    const int h = blockIdx.x, t0 = blockIdx.y * 16, pitch = p.dl * 2 + 64, kb = p.dl / 32;
    const int v0 = (warp & 3) * 32, quarter = warp >> 2, kq = kb / 4;    // (d_latent is a multiple of 128)
    const bool all = p.most >= p.max_new;
    if (!all) {
        pdl_wait_prior_grid();
        if (t0 >= p.row_pre[p.s.n]) return;
    }
    // lane t4 of a quad takes columns 8 t4 .. 8 t4 + 7 of every 32, of both operands: any order of k will do
    uint4 w[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (v0 + j * 8 < p.dv && k < kq)
                w[j][k] = __ldg(reinterpret_cast<const uint4*>(p.W_uv + ((size_t)h * p.dv + v0 + j * 8 + g) * p.dl + t4 * 8 + (quarter * kq + k) * 32));
    pdl_wait_prior_grid();
    {
        int first = 0, count = 0, row = -1;
        const int32_t* ends = all ? p.s.cu : p.row_pre;
        const int seq = find_sequence(ends, p.s.n, t0 + warp, lane);
        const Seq q = seq < p.s.n ? sequence(p, seq) : Seq{};
        const int t = q.a + t0 + warp - ends[min(seq, p.s.n)];
        const bool there = q.rows > 0 && t < p.s.T;
        if (there) {
            const long long W = p.tile_pre[p.s.n], before = p.tile_pre[seq];
            const int units = p.unit_pre[seq], in = (t - q.a) * p.heads + h, rt = in / p.R, ug = rt / p.group;
            row = (rt - ug * p.group) * p.R + in - rt * p.R;
            if (q.kt > 0) {
                const long long each = stretch(W, p.groups), at = before + ug * unit_length(q) + kPiece;
                const int g0 = (int)quotient(at, each), g1 = (int)quotient(at + q.kt - 1, each);
                first = g0 + units + ug;
                count = first >= 0 ? max(min(g1 - g0 + 1, p.max_slots - first), 0) : 0;
            }
        }
        const size_t step = (size_t)p.group * p.R, at = (size_t)first * step + row;
        // weights of the pieces: 2^(m - largest m)
        float2 ml[(kSms + 31) / 32];
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int k = 0; k < (kSms + 31) / 32; ++k)
            if (k * 32 + lane < count) {
                ml[k] = p.ml[at + (k * 32 + lane) * step];
                top = fmaxf(top, ml[k].x);
            }
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
        const float mm = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int k = 0; k < (kSms + 31) / 32; ++k)
            if (k * 32 + lane < count) {
                const float e = exp2f(ml[k].x - mm);
                s_weight[warp][k * 32 + lane] = e;
                sum = fmaf(ml[k].y, e, sum);
            }
        sum = warp_sum(sum);
        if (lane == 0) s_row[warp] = there ? t : -1;
        __syncwarp();
        float4 o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int j = 0; j < count; ++j) {
            const float e = s_weight[warp][j];
            const float4* src = reinterpret_cast<const float4*>(p.part + (at + j * step) * p.dl) + lane;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k * 128 < p.dl) {
                    const float4 v = __ldcs(src + k * 32);
                    o[k].x = fmaf(v.x, e, o[k].x); o[k].y = fmaf(v.y, e, o[k].y); o[k].z = fmaf(v.z, e, o[k].z); o[k].w = fmaf(v.w, e, o[k].w);
                }
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;                  // (nothing seen: zeros; NaN stays)
        uint8_t* hi = smem + warp * pitch + lane * 8;
        uint8_t* lo = hi + 16 * pitch;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k * 128 < p.dl) {
                const float x = o[k].x * inv, y = o[k].y * inv, z = o[k].z * inv, u = o[k].w * inv;
                const uint32_t h0 = bf16_pair(x, y), h1 = bf16_pair(z, u);
                *reinterpret_cast<uint2*>(hi + k * 256) = make_uint2(h0, h1);
                *reinterpret_cast<uint2*>(lo + k * 256) = make_uint2(bf16_pair(x - bf16_lo(h0), y - bf16_hi(h0)), bf16_pair(z - bf16_lo(h1), u - bf16_hi(h1)));
            }
    }
    __syncthreads();
    float d[4][4] = {};
    const uint8_t* a0 = smem + g * pitch + t4 * 16 + quarter * kq * 64;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (k < kq)
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const uint8_t* a = a0 + part * 16 * pitch + k * 64;
                const uint4 x = *reinterpret_cast<const uint4*>(a), z = *reinterpret_cast<const uint4*>(a + 8 * pitch);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (v0 + j * 8 < p.dv) {
                        mma16816_bf16(d[j], x.x, z.x, x.y, z.y, w[j][k].x, w[j][k].y);
                        mma16816_bf16(d[j], x.z, z.z, x.w, z.w, w[j][k].z, w[j][k].w);
                    }
            }
    // the quarters meet in shared memory: [quarter][row][value]
    __syncthreads();
    float* s_d = reinterpret_cast<float*>(smem);
    constexpr int kRow = 132;                                            // floats of a row: 128 and padding
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float* out = s_d + (quarter * 16 + g) * kRow + v0 + j * 8 + 2 * t4;
        *reinterpret_cast<float2*>(out) = make_float2(d[j][0], d[j][1]);
        *reinterpret_cast<float2*>(out + 8 * kRow) = make_float2(d[j][2], d[j][3]);
    }
    __syncthreads();
    const int r = tid >> 5, v = lane * 4, t = s_row[r];
    if (t < 0 || v >= p.dv) return;
    float4 y = *reinterpret_cast<const float4*>(s_d + r * kRow + v);
#pragma unroll
    for (int i = 1; i < 4; ++i) {
        const float4 x = *reinterpret_cast<const float4*>(s_d + (i * 16 + r) * kRow + v);
        y.x += x.x; y.y += x.y; y.z += x.z; y.w += x.w;
    }
    const size_t at = ((size_t)t * p.heads + h) * p.dv + v;
    uint2 o;
    if (p.out_dtype == EDG_F16) {
        const __half2 a = __floats2half2_rn(y.x, y.y), b = __floats2half2_rn(y.z, y.w);
        o = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    } else o = make_uint2(bf16_pair(y.x, y.y), bf16_pair(y.z, y.w));
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.y) + at) = o;
}

struct AbsorbedLayout { int R, group, groups, slots; size_t tile_pre, unit_pre, row_pre, q_lat, ml, part, bytes; };

AbsorbedLayout absorbed_layout(const edg_latent_desc& d, int n_seqs, int T, int max_new) {
    AbsorbedLayout L;
    const int64_t rows = (int64_t)max_new * d.heads, taken = (int64_t)n_seqs * max_new, all = (taken < T ? taken : T) * d.heads;
    L.R = absorbed_rows(rows);
    const int64_t tiles = (rows + L.R - 1) / L.R;
    L.group = (int)(tiles < kGroupMost ? tiles : kGroupMost);
    L.groups = kSms / L.group;
    // units: every sequence with rows has one and a part of one more at most
    const int64_t with = n_seqs < T ? n_seqs : T;
    L.slots = (int)(L.groups + with + all / ((int64_t)L.R * L.group) + 1);
    const size_t rows_all = (size_t)kSms * L.R + (size_t)(with + 1) * L.R * L.group + (size_t)all;
    L.tile_pre = kCtrlBytes;
    L.unit_pre = round_up(L.tile_pre + ((size_t)n_seqs + 1) * 8, 256);
    L.row_pre = round_up(L.unit_pre + ((size_t)n_seqs + 1) * 4, 256);
    L.q_lat = round_up(L.row_pre + ((size_t)n_seqs + 1) * 4, 256);
    L.ml = round_up(L.q_lat + (size_t)T * d.heads * (d.d_latent + 64) * 2, 256);
    L.part = round_up(L.ml + rows_all * 8, 256);
    L.bytes = round_up(L.part + rows_all * d.d_latent * 4, 256);
    return L;
}

}  // namespace

size_t absorbed_workspace(const edg_latent_desc& d, int n_seqs, int T, int most) { return absorbed_layout(d, n_seqs, T, most).bytes; }

int32_t run_absorbed(const edg_latent_desc& d, const LatentSeqs& s, int max_new, int64_t total_len, int most, const void* q, const void* q_rope,
                     const void* W_uk, const void* W_uv, const void* cache, void* y, void* workspace, cudaStream_t st) {
    const AbsorbedLayout L = absorbed_layout(d, s.n, s.T, most);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    AbsorbedParams p = {};
    p.s = s;
    p.q = static_cast<const uint16_t*>(q);
    p.ldq = latent_ldq(d);
    p.q_rope = q_rope != nullptr ? static_cast<const uint16_t*>(q_rope) : p.q + d.d_nope;
    p.ldr = q_rope != nullptr ? (int64_t)d.heads * d.d_rope : p.ldq;
    p.hr = q_rope != nullptr ? d.d_rope : d.d_nope + d.d_rope;
    p.W_uk = static_cast<const uint16_t*>(W_uk);
    p.W_uv = static_cast<const uint16_t*>(W_uv);
    p.q_lat = reinterpret_cast<uint16_t*>(ws + L.q_lat);
    p.part = reinterpret_cast<float*>(ws + L.part);
    p.ml = reinterpret_cast<float2*>(ws + L.ml);
    p.tile_pre = reinterpret_cast<long long*>(ws + L.tile_pre);
    p.unit_pre = reinterpret_cast<int32_t*>(ws + L.unit_pre);
    p.row_pre = reinterpret_cast<int32_t*>(ws + L.row_pre);
    p.y = y;
    p.status = static_cast<int32_t*>(workspace);
    p.heads = d.heads;
    p.dn = d.d_nope;
    p.dr = d.d_rope;
    p.dv = d.d_v;
    p.dl = d.d_latent;
    p.out_dtype = d.out_dtype;
    p.scale = d.scale;
    p.R = L.R;
    p.group = L.group;
    p.groups = L.groups;
    p.max_slots = L.slots;
    p.max_new = max_new;
    p.total_len = total_len;
    p.most = most;
    static OncePerDevice once;
    EDG_CUDA_TRY(once([] {
        cudaError_t e = allow_smem(Plan<16>::bytes, absorbed_kernel<16>);
        if (e == cudaSuccess) e = allow_smem(Plan<32>::bytes, absorbed_kernel<32>);
        if (e == cudaSuccess) e = allow_smem(Plan<64>::bytes, absorbed_kernel<64>);
        return e;
    }));
    CUtensorMap kv_map, q_map;
    const uint64_t row = (uint64_t)latent_row(d), q_row = (uint64_t)d.d_latent + 64;
    const uint64_t kv_dims[2] = {row, (uint64_t)d.n_pages * d.page}, q_dims[2] = {q_row, (uint64_t)s.T * d.heads};
    const uint32_t kv_box[2] = {64, (uint32_t)(d.page < 64 ? d.page : 64)}, q_box[2] = {64, (uint32_t)L.R};
    EDG_CUDA_TRY(make_map(&kv_map, cache, 2, kv_dims, &row, kv_box));
    EDG_CUDA_TRY(make_map(&q_map, p.q_lat, 2, q_dims, &q_row, q_box));
    const int64_t rows = most >= max_new ? s.T : ((int64_t)s.n * most < s.T ? (int64_t)s.n * most : s.T);        // that can be taken
    if (most >= max_new) {
        absorb_kernel<<<dim3(d.heads * (d.d_latent / 64) + 1, (unsigned)((rows + 63) / 64)), 128, 0, st>>>(p);
        EDG_CUDA_TRY(cudaGetLastError());
    } else {
        plan_kernel<<<1, 128, 0, st>>>(p);
        EDG_CUDA_TRY(cudaGetLastError());
        EDG_CUDA_TRY(launch_pdl(absorb_kernel, dim3(d.heads * (d.d_latent / 64), (unsigned)((rows + 63) / 64)), 128, (size_t)0, st, p));
    }
    const dim3 grid(L.groups * L.group);
    EDG_CUDA_TRY(L.R == 16   ? launch_pdl(absorbed_kernel<16>, grid, kThreads, Plan<16>::bytes, st, p, kv_map, q_map)
                 : L.R == 32 ? launch_pdl(absorbed_kernel<32>, grid, kThreads, Plan<32>::bytes, st, p, kv_map, q_map)
                             : launch_pdl(absorbed_kernel<64>, grid, kThreads, Plan<64>::bytes, st, p, kv_map, q_map));
    EDG_CUDA_TRY(launch_pdl(combine_kernel, dim3(d.heads, (unsigned)((rows + 15) / 16)), kCombine,
                            (size_t)(32 * (d.d_latent * 2 + 64) > 4 * 16 * 132 * 4 ? 32 * (d.d_latent * 2 + 64) : 4 * 16 * 132 * 4), st, p));
    return EDG_OK;
}

}  // namespace edg
