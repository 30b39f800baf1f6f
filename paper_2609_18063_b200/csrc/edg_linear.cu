// y[t] = W x[t] + lora_scale B (A x[t]): one int4 projection for a few tokens.
//
//     y[t,n] = sum over groups of s[n,g] ( sum_k q[n,k] x[t,k] - z[n,g] sum_k x[t,k] )  +  lora_scale sum_r B[n,r] u[t,r],   u = A x
//
// Memory bounds it (N Kd / 2 bytes of codes for 2 T N Kd operations), so the design is about reading the codes at full width and
// doing little per code.  The codes are the A operand of m16n8k16 tensor-core products (16 rows), eight tokens the B operand; the
// codes go in as the fp16 subnormals that their bits are (edg_mma.cuh: five instructions for eight codes), the activations
// carry a power of two per token.  Sums of one group leave the accumulator with the zero point removed and the scale applied, in fp32.
//
// Record: codes [N/16 row tiles][Kd/128 blocks][2][32 lanes][16 bytes] -- lane 4g + t of half h holds, chunk by chunk (32 codes) of the
// block, the t-th word of row g + 8h, which is its operand of the product: a block of a row tile is two coalesced 16-byte loads a lane.
// Then (scale, zero) [N/16][Kd/128][16 rows][128/GS] with GS = 32, 64 or 128 codes to a pair (the largest of these that divides the group:
// the kernel then knows how many pairs a block has, one load a row).  Rows and codes beyond N and Kd are zero.
//
// A warp walks the blocks of its one or two row tiles (RT), 4 KB of codes in flight in registers; the warps of a CTA share the blocks of row
// tiles (WK of them) or take row tiles of their own, and a cluster of CTAs shares the input dimension where the row tiles alone do not fill
// the GPU.  Partial sums meet in shared memory, in a fixed order.
//
// 64,001 x 2,048 codes (74 MB with their scales): 1 token 18.1 us (4.1 TB/s), 8 20.5, 16 31, 64 97; 6,144 x 2,048 with an adapter of 16:
// 1 token 7.9, 64 23.5, 4,096 623 (ten times what its operations take); 1,024 x 1,024, 1 token: 6.7 (two launches and two waits for memory).
// From 16 tokens on the products bound it: a slice of the grid for every 8 or 16 tokens takes the codes apart again, and every 8
// tokens more cost 11 us of the first, 25 clocks a product and quarter of an SM.
#include <cooperative_groups.h>
#include <string.h>

#include "edg_mma.cuh"
#include "edg_ptx.cuh"

namespace edg {

bool zero_points_ok(const uint16_t* z, size_t n);      // edg_pack.cu

namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 256, kWarps = 8;

inline int pair_codes(int group) { return group % 128 == 0 ? 128 : (group % 64 == 0 ? 64 : 32); }
inline int blocks_of(int Kd) { return (Kd + 127) / 128; }
inline size_t tiles_of(int N) { return ((size_t)N + 15) / 16; }
inline size_t codes_bytes(const edg_linear_desc& d) { return tiles_of(d.N) * blocks_of(d.Kd) * 1024; }
inline size_t record_size(const edg_linear_desc& d) { return codes_bytes(d) + tiles_of(d.N) * blocks_of(d.Kd) * 64 * (128 / pair_codes(d.group)); }

int32_t check(const edg_linear_desc* d) {
    if (d == nullptr) return EDG_E_INVAL;
    if (d->N < 1 || d->N > (1 << 24) || d->Kd < 32 || d->Kd > 65536) return EDG_E_SHAPE;
    if (d->group < 32 || d->group % 32 != 0 || d->Kd % d->group != 0) return EDG_E_SHAPE;
    if (d->rank < 0 || d->rank > 64) return EDG_E_SHAPE;
    if (d->out_dtype != EDG_F32 && d->out_dtype != EDG_F16 && d->out_dtype != EDG_BF16) return EDG_E_INVAL;
    if (d->ldx != 0 && (d->ldx < d->Kd || d->ldx % 8 != 0)) return EDG_E_SHAPE;
    if (d->ldy != 0 && d->ldy < d->N) return EDG_E_SHAPE;
    return EDG_OK;
}

// canonical <-> record.  Codes of a word keep their order: code k of it in bits 4k..4k+3.
void repack_linear(const edg_linear_desc& d, uint8_t* rec, uint8_t* codes, uint16_t* sc, uint16_t* ze, bool to_record) {
    const int nb = blocks_of(d.Kd), gs = pair_codes(d.group), per = 128 / gs;
    uint8_t* rz = rec + codes_bytes(d);
    for (int n = 0; n < d.N; ++n) {
        const size_t tile = n >> 4;
        const int row = n & 15, half = row >> 3, g = row & 7;
        for (int w = 0; w < d.Kd / 8; ++w) {                  // word w of the row: chunk w / 4, lane w % 4 of the quad
            const int b = w >> 4, chunk = (w >> 2) & 3, t = w & 3;
            uint8_t* r = rec + ((tile * nb + b) * 2 + half) * 512 + (g * 4 + t) * 16 + chunk * 4;
            uint8_t* c = codes + (size_t)n * (d.Kd / 2) + (size_t)w * 4;
            if (to_record) memcpy(r, c, 4); else memcpy(c, r, 4);
        }
        for (int p = 0; p < d.Kd / gs; ++p) {
            uint16_t* r = reinterpret_cast<uint16_t*>(rz + (((tile * nb + p / per) * 16 + row) * per + p % per) * 4);
            const size_t k = (size_t)n * (d.Kd / d.group) + (size_t)p * gs / d.group;
            if (to_record) { r[0] = sc[k]; r[1] = ze[k]; } else { sc[k] = r[0]; ze[k] = r[1]; }
        }
    }
}

struct LinearParams {
    const uint8_t* codes;
    const uint8_t* sz;
    const uint16_t* x;
    const float* u;             // [T][rank] or null
    const uint16_t* B;
    void* y;
    int N, Kd, T, rank, out_dtype, ldx;
    size_t ldy;
    int tiles, blocks;          // row tiles; blocks of 128 codes of the input dimension
    int wk;                     // warps that share their row tiles; RT kWarps / wk row tiles to a unit
    int cluster, cta_blocks;    // CTAs that share the input dimension; blocks of each
    float lora_scale;
};
static_assert(kThreads % (kWarps * 32) == 0, "a thread keeps its row");

// u[t][r] = A[r] . x[t]: a warp per (token, rank)
__global__ void __launch_bounds__(128) linear_u_kernel(const uint16_t* A, const uint16_t* x, float* u, int Kd, int ldx, int rank) {
    pdl_launch_dependents();
    const int r = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31, t = blockIdx.y;
    if (r >= rank) return;
    const uint4* a = reinterpret_cast<const uint4*>(A + (size_t)r * Kd);
    const uint4* b = reinterpret_cast<const uint4*>(x + (size_t)t * ldx);
    float s = 0.f;
#pragma unroll 4
    for (int i = lane; i < Kd / 8; i += 32) {
        const uint4 v = __ldg(a + i), w = __ldg(b + i);
        s = fmaf(bf16_lo(v.x), bf16_lo(w.x), s); s = fmaf(bf16_hi(v.x), bf16_hi(w.x), s);
        s = fmaf(bf16_lo(v.y), bf16_lo(w.y), s); s = fmaf(bf16_hi(v.y), bf16_hi(w.y), s);
        s = fmaf(bf16_lo(v.z), bf16_lo(w.z), s); s = fmaf(bf16_hi(v.z), bf16_hi(w.z), s);
        s = fmaf(bf16_lo(v.w), bf16_lo(w.w), s); s = fmaf(bf16_hi(v.w), bf16_hi(w.w), s);
    }
    s = warp_sum(s);
    if (lane == 0) u[(size_t)t * rank + r] = s;
}

// Shared memory: activations [blocks][4 chunks][NT][32 lanes] 16 bytes; sums of them [blocks][128/GS][NT * 8] float; scales of the tokens
// [NT * 8]; partial sums [kWarps][16 RT rows][NT * 8] float; A x of the tokens [NT * 8][rank rounded to 8] float.
template <int GS, int NT, int RT> constexpr size_t linear_smem(int blocks, int rank) {
    return (size_t)blocks * (NT * 2048 + (128 / GS) * NT * 32) + NT * 8 * 4 + kWarps * 16 * RT * NT * 8 * 4 + (size_t)NT * 32 * ((rank + 7) & ~7);
}

constexpr int kResident = 2;                  // CTAs that share an SM

template <int GS, int NT, int RT>
__global__ void __launch_bounds__(kThreads, kResident) linear_kernel(const __grid_constant__ LinearParams p) {
    constexpr int PB = 128 / GS;                       // (scale, zero) pairs of a row in a block
    constexpr int TN = NT * 8, RR = 16 * RT;
    constexpr int kAhead = 4 / RT;                     // blocks in flight per warp
    extern __shared__ __align__(16) uint8_t smem[];
    uint4* s_x = reinterpret_cast<uint4*>(smem);
    float* s_sum = reinterpret_cast<float*>(smem + (size_t)p.cta_blocks * NT * 2048);
    float* s_scale = s_sum + (size_t)p.cta_blocks * PB * TN;
    float* s_red = s_scale + TN;
    float* s_u = s_red + kWarps * RR * TN;
    const int ru = (p.rank + 7) & ~7;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
    const int rank_c = (int)(blockIdx.x % p.cluster), unit0 = (int)(blockIdx.x / p.cluster), n_units_grid = (int)(gridDim.x / p.cluster);
    const int t0 = blockIdx.y * TN, nt = min(TN, p.T - t0);
    const int b0 = rank_c * p.cta_blocks, nb = min(p.cta_blocks, p.blocks - b0);        // this CTA's blocks
    const int wr = kWarps / p.wk;                      // row tiles of a unit, RT at a time
    const int tiles = (p.tiles + RT - 1) / RT;
    const int my_tile = warp / p.wk, my_k = warp % p.wk;
    const int per_unit = nb > my_k ? (nb - my_k + p.wk - 1) / p.wk : 0;                 // this warp's blocks of a unit
    const int units = (tiles + wr - 1) / wr;

    // ---- the first blocks of codes are asked for before anything else
    uint4 c0[kAhead][RT], c1[kAhead][RT];
    uint32_t z0[kAhead][RT][PB], z1[kAhead][RT][PB];
    auto load = [&](int slot, int i, const uint8_t* c, const uint8_t* z) {
        c0[slot][i] = ld_stream16(c);
        c1[slot][i] = ld_stream16(c + 512);
        if constexpr (PB == 1) {
            z0[slot][i][0] = ld_stream4(z);
            z1[slot][i][0] = ld_stream4(z + 32);
        } else if constexpr (PB == 2) {
            const uint2 a = __ldg(reinterpret_cast<const uint2*>(z)), b = __ldg(reinterpret_cast<const uint2*>(z + 64));
            z0[slot][i][0] = a.x; z0[slot][i][1] = a.y; z1[slot][i][0] = b.x; z1[slot][i][1] = b.y;
        } else {
            const uint4 a = ld_stream16(z), b = ld_stream16(z + 128);
            z0[slot][i][0] = a.x; z0[slot][i][1] = a.y; z0[slot][i][2] = a.z; z0[slot][i][3] = a.w;
            z1[slot][i][0] = b.x; z1[slot][i][1] = b.y; z1[slot][i][2] = b.z; z1[slot][i][3] = b.w;
        }
    };
    // A warp's blocks of a unit, rounded up to the slots: a block's slot is its number, known when the loop is unrolled.
    const int padded = (per_unit + kAhead - 1) / kAhead * kAhead;
    int lu = unit0, li = 0;                            // the next block to ask for, and where it lies
    const size_t first = ((size_t)(unit0 * wr + my_tile) * RT * p.blocks + b0 + my_k), jump = (size_t)n_units_grid * wr * RT * p.blocks - (size_t)padded * p.wk;
    const uint8_t *lc = p.codes + first * 1024 + lane * 16, *lz = p.sz + first * (64 * PB) + g * (4 * PB);
    auto load_next = [&](int slot) {
#pragma unroll
        for (int i = 0; i < RT; ++i)
            if (li < per_unit && (lu * wr + my_tile) * RT + i < p.tiles) load(slot, i, lc + (size_t)i * p.blocks * 1024, lz + (size_t)i * p.blocks * (64 * PB));
        lc += p.wk * 1024;
        lz += p.wk * 64 * PB;
        if (++li == padded) {
            li = 0;
            lu += n_units_grid;
            lc += jump * 1024;
            lz += jump * (64 * PB);
        }
    };
    if (padded > 0) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) load_next(j);
    }

    // ---- activations: largest magnitude per token, then operands and sums of groups
    {
        uint32_t* s_max = reinterpret_cast<uint32_t*>(s_scale);
        if (tid < TN) s_max[tid] = 0u;
        __syncthreads();
        const int chunks = nb * 4;
        auto raw = [&](int c, int n) -> uint4 {        // eight activations of token n: word t4 of chunk c
            const int k = (b0 * 4 + c) * 32 + t4 * 8;
            if (n < nt && k < p.Kd) return __ldg(reinterpret_cast<const uint4*>(p.x + (size_t)(t0 + n) * p.ldx + k));
            return make_uint4(0, 0, 0, 0);
        };
        // Groups of GS codes go to the warps in turn.  The first ones stay in registers from the search for the largest magnitude to the
        // operands; what does not fit is read again.
        constexpr int GC = GS / 32, kRoom = 8, kKeep = kRoom / (NT * GC) > 0 ? kRoom / (NT * GC) : 1;
        uint4 keep[kKeep][GC][NT];
        uint32_t m[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) m[j] = 0u;
        auto magnitude = [&](int j, const uint4& v) {
            const float f[8] = {bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y), bf16_lo(v.z), bf16_hi(v.z), bf16_lo(v.w), bf16_hi(v.w)};
            m[j] = max(m[j], abs_max8(f));
        };
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            const int c = (warp + i * kWarps) * GC;
#pragma unroll
            for (int x = 0; x < GC; ++x)
#pragma unroll
                for (int j = 0; j < NT; ++j) keep[i][x][j] = c < chunks ? raw(c + x, j * 8 + g) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < kKeep; ++i)
#pragma unroll
            for (int x = 0; x < GC; ++x)
#pragma unroll
                for (int j = 0; j < NT; ++j) magnitude(j, keep[i][x][j]);
        for (int c = (warp + kKeep * kWarps) * GC; c < chunks; c += kWarps * GC)
#pragma unroll
            for (int x = 0; x < GC; ++x)
#pragma unroll
                for (int j = 0; j < NT; ++j) magnitude(j, raw(c + x, j * 8 + g));
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const uint32_t v = group_max<4>(m[j]);
            if (t4 == 0 && v != 0u) atomicMax(&s_max[j * 8 + g], v);
        }
        __syncthreads();
        float sc[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) sc[j] = vector_scale(s_max[j * 8 + g]);
        auto operands = [&](int c, int j, const uint4 (&v)[GC]) {
            float sum = 0.f;
#pragma unroll
            for (int x = 0; x < GC; ++x) {
                const float f[8] = {bf16_lo(v[x].x), bf16_hi(v[x].x), bf16_lo(v[x].y), bf16_hi(v[x].y), bf16_lo(v[x].z), bf16_hi(v[x].z), bf16_lo(v[x].w), bf16_hi(v[x].w)};
                s_x[(size_t)((c + x) * NT + j) * 32 + lane] = permute8_s(f, sc[j]);
                sum += ((f[0] + f[1]) + (f[2] + f[3])) * sc[j] + ((f[4] + f[5]) + (f[6] + f[7])) * sc[j];
            }
            sum = group_sum<4>(sum);
            if (t4 == 0) s_sum[(c / GC) * TN + j * 8 + g] = sum * kScaleS;
        };
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            const int c = (warp + i * kWarps) * GC;
            if (c < chunks) {
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    uint4 v[GC];
#pragma unroll
                    for (int x = 0; x < GC; ++x) v[x] = keep[i][x][j];
                    operands(c, j, v);
                }
            }
        }
        for (int c = (warp + kKeep * kWarps) * GC; c < chunks; c += kWarps * GC)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                uint4 v[GC];
#pragma unroll
                for (int x = 0; x < GC; ++x) v[x] = raw(c + x, j * 8 + g);
                operands(c, j, v);
            }
        __syncthreads();
        if (tid < TN) s_scale[tid] = kUnscaleS * vector_unscale(vector_scale(s_max[tid]));
        __syncthreads();
    }

    bool u_there = p.rank == 0;
    for (int unit = unit0; unit < units; unit += n_units_grid) {
        const int tile = unit * wr + my_tile;
        float acc[RT][NT][4];
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j][0] = acc[i][j][1] = acc[i][j][2] = acc[i][j][3] = 0.f;
        auto block = [&](int s, int n) {
            const int lb = my_k + n * p.wk;            // block within this CTA's
            float d[RT][NT][4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t q0[RT][4], q1[RT][4];
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const uint32_t w0[4] = {c0[s][i].x, c0[s][i].y, c0[s][i].z, c0[s][i].w}, w1[4] = {c1[s][i].x, c1[s][i].y, c1[s][i].z, c1[s][i].w};
                    dequant_word_s(w0[c], q0[i]);
                    dequant_word_s(w1[c], q1[i]);
                }
                const uint4* xb = s_x + (size_t)((lb * 4 + c) * NT) * 32 + lane;
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const uint4 b = xb[j * 32];
#pragma unroll
                    for (int i = 0; i < RT; ++i) {
                        if (c % (GS / 32) == 0) mma16816_zero(d[i][j], q0[i][0], q1[i][0], q0[i][1], q1[i][1], b.x, b.y);
                        else mma16816(d[i][j], q0[i][0], q1[i][0], q0[i][1], q1[i][1], b.x, b.y);
                    }
#pragma unroll
                    for (int i = 0; i < RT; ++i) mma16816(d[i][j], q0[i][2], q1[i][2], q0[i][3], q1[i][3], b.z, b.w);
                }
                if (c % (GS / 32) == GS / 32 - 1) {
                    const int pi = c / (GS / 32);
                    float2 f0[RT], f1[RT];
#pragma unroll
                    for (int i = 0; i < RT; ++i) {
                        f0[i] = __half22float2(u32_as_h2(z0[s][i][pi]));
                        f1[i] = __half22float2(u32_as_h2(z1[s][i][pi]));
                    }
                    const float2* sm = reinterpret_cast<const float2*>(s_sum + (lb * PB + pi) * TN) + t4;
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        const float2 xs = sm[j * 4];
#pragma unroll
                        for (int i = 0; i < RT; ++i) {
                            acc[i][j][0] = fmaf(f0[i].x, fmaf(-f0[i].y, xs.x, d[i][j][0]), acc[i][j][0]);
                            acc[i][j][1] = fmaf(f0[i].x, fmaf(-f0[i].y, xs.y, d[i][j][1]), acc[i][j][1]);
                            acc[i][j][2] = fmaf(f1[i].x, fmaf(-f1[i].y, xs.x, d[i][j][2]), acc[i][j][2]);
                            acc[i][j][3] = fmaf(f1[i].x, fmaf(-f1[i].y, xs.y, d[i][j][3]), acc[i][j][3]);
                        }
                    }
                }
            }
        };
        for (int i = 0; i < padded; i += kAhead)
#pragma unroll
            for (int s = 0; s < kAhead; ++s) {
                if (i + s < per_unit && tile < tiles) block(s, i + s);
                load_next(s);
            }
        // ---- partial sums meet: [warp][row][token]
        float* red = s_red + warp * RR * TN;
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                *reinterpret_cast<float2*>(red + (i * 16 + g) * TN + j * 8 + 2 * t4) = make_float2(acc[i][j][0], acc[i][j][1]);
                *reinterpret_cast<float2*>(red + (i * 16 + g + 8) * TN + j * 8 + 2 * t4) = make_float2(acc[i][j][2], acc[i][j][3]);
            }
        __syncthreads();
        if (p.cluster > 1) {                           // this CTA's sums over its warps, scaled, into the first warp's of each row tile
            for (int o = tid; o < wr * RR * TN; o += kThreads) {
                const int x = o / (RR * TN), at = o - x * RR * TN;
                float* s = s_red + x * p.wk * RR * TN + at;
                float v = s[0];
                for (int k = 1; k < p.wk; ++k) v += s[k * RR * TN];
                s[0] = v * s_scale[at % TN];
            }
            __syncwarp();
            cluster_arrive();
            cluster_wait();
        }
        if (!u_there) {                                // (A x comes from the kernel before, which has run beside this one)
            pdl_wait_prior_grid();
            for (int i = tid; i < nt * ru; i += kThreads) {
                const int tok = i / ru, r = i - tok * ru;
                s_u[i] = r < p.rank ? p.lora_scale * __ldcg(p.u + (size_t)(t0 + tok) * p.rank + r) : 0.f;
            }
            __syncthreads();
            u_there = true;
        }
        // outputs of the unit, spread over the cluster's CTAs: a thread keeps its row, consecutive threads take consecutive rows
        const int rows = wr * RR, row = tid & (rows - 1), rt = row / RR, n = unit * rows + row;
        const int tstep = p.cluster * kThreads / rows, tok0 = (rank_c * kThreads + tid) / rows;
        const cg::cluster_group cluster = cg::this_cluster();
        const float* src = s_red + rt * p.wk * RR * TN + (row & (RR - 1)) * TN;
        auto value = [&](int tok) {
            float v = 0.f;
            if (p.cluster > 1) {
                float f[8];
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (c < p.cluster) f[c] = *cluster.map_shared_rank(src + tok, c);
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (c < p.cluster) v += f[c];
            } else {
                for (int k = 0; k < p.wk; ++k) v += src[tok + k * RR * TN];
                v *= s_scale[tok];
            }
            return v;
        };
        auto store = [&](int tok, float v) {
            const size_t at = (size_t)(t0 + tok) * p.ldy + n;
            if (p.out_dtype == EDG_F32) store_out(static_cast<float*>(p.y), at, v);
            else if (p.out_dtype == EDG_F16) store_out(static_cast<__half*>(p.y), at, v);
            else static_cast<uint16_t*>(p.y)[at] = bf16_rn(v);
        };
        if (n < p.N) {
            if (p.rank == 0) {
                for (int tok = tok0; tok < nt; tok += tstep) store(tok, value(tok));
            } else {
                // four tokens at a time against eight ranks of this row of B
                const uint16_t* Bn = p.B + (size_t)n * p.rank;
                const bool wide = (p.rank & 7) == 0;
                for (int q0 = tok0; q0 < nt; q0 += 4 * tstep) {
                    float e[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) e[q] = q0 + q * tstep < nt ? value(q0 + q * tstep) : 0.f;
                    for (int r = 0; r < ru; r += 8) {
                        float bv[8];
                        if (wide) {
                            const uint4 w = __ldg(reinterpret_cast<const uint4*>(Bn + r));
                            bv[0] = bf16_lo(w.x); bv[1] = bf16_hi(w.x); bv[2] = bf16_lo(w.y); bv[3] = bf16_hi(w.y);
                            bv[4] = bf16_lo(w.z); bv[5] = bf16_hi(w.z); bv[6] = bf16_lo(w.w); bv[7] = bf16_hi(w.w);
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j) bv[j] = r + j < p.rank ? bf16_bits_to_float(Bn[r + j]) : 0.f;
                        }
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int tok = q0 + q * tstep;
                            if (tok < nt) {
                                const float4 a = *reinterpret_cast<const float4*>(s_u + tok * ru + r), b = *reinterpret_cast<const float4*>(s_u + tok * ru + r + 4);
                                e[q] = fmaf(bv[0], a.x, e[q]); e[q] = fmaf(bv[1], a.y, e[q]); e[q] = fmaf(bv[2], a.z, e[q]); e[q] = fmaf(bv[3], a.w, e[q]);
                                e[q] = fmaf(bv[4], b.x, e[q]); e[q] = fmaf(bv[5], b.y, e[q]); e[q] = fmaf(bv[6], b.z, e[q]); e[q] = fmaf(bv[7], b.w, e[q]);
                            }
                        }
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (q0 + q * tstep < nt) store(q0 + q * tstep, e[q]);
                }
            }
        }
        __syncwarp();
        // (the next unit's partial sums wait until these have been read)
        if (p.cluster > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();
    }
    if (!u_there) pdl_wait_prior_grid();
}

constexpr size_t kMost = 200 * 1024;
struct LinearPlan { int nt, rt, wk, cluster, cta_blocks, grid; size_t smem; int64_t cost; };

// Tokens of a pass (8 NT), row tiles of a warp (RT), warps that share them, CTAs that share the input dimension: what takes the least by the rounds that a CTA's
// warps make.  In clocks: a block of 128 codes 200 + 100 NT of a warp with seven beside it and half as much more with fifteen (of two row tiles
// 300 + 150 NT), the sums' meeting 700 + 60 NT a row tile and 1500 more in a cluster, the activations 1500 + 60 NT a block at the start.  Against
// every shape of a launch at 13 sizes (1 to 64 tokens) this took 0 to 16% longer than the best; four or eight tiles of tokens never were that.
// Two row tiles at once share the activations' operands: 64,001 rows, 16 tokens 32.5 -> 31 us; 6,144 rows, 16 tokens 11.1 -> 8.8.
template <int GS, int NT, int RT> void plan_linear(const LinearParams& p, int sms, LinearPlan& best) {
    const int slices = (p.T + NT * 8 - 1) / (NT * 8);
    for (int c = 1; c <= 8; c *= 2)
        for (int wk = 1; wk <= kWarps; wk *= 2) {
            const int each = (p.blocks + c - 1) / c;
            const size_t bytes = linear_smem<GS, NT, RT>(each, p.rank);
            if (bytes > kMost || (c > 1 && each * (c - 1) >= p.blocks)) continue;      // (every CTA has blocks)
            int resident = (int)((220 * 1024) / (bytes + 1024));
            resident = resident < 1 ? 1 : (resident > kResident ? kResident : resident);
            const int units = ((p.tiles + RT - 1) / RT + kWarps / wk - 1) / (kWarps / wk), room = sms * resident / c > 0 ? sms * resident / c : 1;
            const int64_t all = (int64_t)units * slices, rounds = (all + room - 1) / room;
            const int beside = all * c > sms ? resident : 1;                           // CTAs that share an SM's pipes
            const int64_t cost = rounds * ((int64_t)((each + wk - 1) / wk) * (RT == 1 ? 200 + 100 * NT : 300 + 150 * NT) * (beside > 1 ? 3 : 2) / 2 + 700 + 60 * NT * RT + (c > 1 ? 1500 : 0)) +
                                 1500 + each * 60 * NT;
            if (best.cost >= 0 && cost >= best.cost) continue;
            best = {NT, RT, wk, c, each, (int)((units + rounds - 1) / rounds), bytes, cost};
        }
}

template <int GS, int NT, int RT> int32_t launch_linear(LinearParams& p, const LinearPlan& plan, cudaStream_t st) {
    static OncePerDevice once;
    EDG_CUDA_TRY(once([] { return allow_smem(kMost, linear_kernel<GS, NT, RT>); }));
    p.wk = plan.wk;
    p.cluster = plan.cluster;
    p.cta_blocks = plan.cta_blocks;
    const dim3 grid(plan.grid * plan.cluster, (p.T + NT * 8 - 1) / (NT * 8));
    EDG_CUDA_TRY(p.rank > 0 ? launch_pdl_cluster(p.cluster, linear_kernel<GS, NT, RT>, grid, kThreads, plan.smem, st, p)
                            : launch_cluster(p.cluster, linear_kernel<GS, NT, RT>, grid, kThreads, plan.smem, st, p));
    return EDG_OK;
}

template <int GS> int32_t launch_gs(LinearParams& p, cudaStream_t st) {
    const int sms = sm_count();
    LinearPlan plan;
    plan.cost = -1;
    plan_linear<GS, 1, 1>(p, sms, plan);
    plan_linear<GS, 1, 2>(p, sms, plan);
    if (p.T > 8) { plan_linear<GS, 2, 1>(p, sms, plan); plan_linear<GS, 2, 2>(p, sms, plan); }
    if (plan.cost < 0) return EDG_E_SHAPE;
    switch (plan.nt * 10 + plan.rt) {
        case 11: return launch_linear<GS, 1, 1>(p, plan, st);
        case 12: return launch_linear<GS, 1, 2>(p, plan, st);
        case 21: return launch_linear<GS, 2, 1>(p, plan, st);
        default: return launch_linear<GS, 2, 2>(p, plan, st);
    }
}

}  // namespace
}  // namespace edg

using namespace edg;

extern "C" int32_t edg_linear_record_bytes(const edg_linear_desc* desc, size_t* bytes) {
    const int32_t rc = check(desc);
    if (rc != EDG_OK) return rc;
    if (!bytes) return EDG_E_INVAL;
    *bytes = record_size(*desc);
    return EDG_OK;
}

extern "C" int32_t edg_pack_linear(const edg_linear_desc* desc, const uint8_t* codes, const uint16_t* scales, const uint16_t* zeros, void* record) {
    const int32_t rc = check(desc);
    if (rc != EDG_OK) return rc;
    if (!codes || !scales || !zeros || !record) return EDG_E_INVAL;
    if (!zero_points_ok(zeros, (size_t)desc->N * (desc->Kd / desc->group))) return EDG_E_RANGE;
    memset(record, 0, record_size(*desc));
    repack_linear(*desc, static_cast<uint8_t*>(record), const_cast<uint8_t*>(codes), const_cast<uint16_t*>(scales), const_cast<uint16_t*>(zeros), true);
    return EDG_OK;
}

extern "C" int32_t edg_unpack_linear(const edg_linear_desc* desc, const void* record, uint8_t* codes, uint16_t* scales, uint16_t* zeros) {
    const int32_t rc = check(desc);
    if (rc != EDG_OK) return rc;
    if (!codes || !scales || !zeros || !record) return EDG_E_INVAL;
    repack_linear(*desc, static_cast<uint8_t*>(const_cast<void*>(record)), codes, scales, zeros, false);
    return EDG_OK;
}

extern "C" int32_t edg_linear_workspace_bytes(const edg_linear_desc* desc, int32_t T, size_t* bytes) {
    const int32_t rc = check(desc);
    if (rc != EDG_OK) return rc;
    if (!bytes || T < 1 || T > 65535) return EDG_E_INVAL;
    *bytes = round_up((size_t)T * (desc->rank > 0 ? desc->rank : 1) * sizeof(float), 256);
    return EDG_OK;
}

extern "C" int32_t linear_int4_lora(const edg_linear_desc* desc, const void* record, int32_t T, const void* x, const void* A, const void* B,
                                    void* y, void* workspace, size_t workspace_bytes, void* stream) {
    const int32_t rc = check(desc);
    if (rc != EDG_OK) return rc;
    if (!record || !x || !y || !workspace || T < 1 || T > 65535) return EDG_E_INVAL;
    if (desc->rank > 0 && (!A || !B)) return EDG_E_INVAL;
    const size_t out = desc->out_dtype == EDG_F32 ? 4 : 2;
    if (!aligned(record, 256) || !aligned(x, 16) || !aligned(y, out) || (desc->rank > 0 && (!aligned(A, 16) || !aligned(B, 16)))) return EDG_E_INVAL;
    size_t need = 0;
    edg_linear_workspace_bytes(desc, T, &need);
    if (!aligned(workspace, 256) || workspace_bytes < need) return EDG_E_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    LinearParams p = {};
    p.codes = static_cast<const uint8_t*>(record);
    p.sz = p.codes + codes_bytes(*desc);
    p.x = static_cast<const uint16_t*>(x);
    p.B = static_cast<const uint16_t*>(B);
    p.y = y;
    p.N = desc->N;
    p.Kd = desc->Kd;
    p.T = T;
    p.rank = desc->rank;
    p.out_dtype = desc->out_dtype;
    p.ldx = desc->ldx != 0 ? desc->ldx : desc->Kd;
    p.ldy = (size_t)(desc->ldy != 0 ? desc->ldy : desc->N);
    p.tiles = (int)tiles_of(desc->N);
    p.blocks = blocks_of(desc->Kd);
    p.lora_scale = desc->lora_scale;
    if (p.rank > 0) {
        float* u = static_cast<float*>(workspace);
        p.u = u;
        linear_u_kernel<<<dim3((p.rank + 3) / 4, T), 128, 0, st>>>(static_cast<const uint16_t*>(A), p.x, u, p.Kd, p.ldx, p.rank);
        EDG_CUDA_TRY(cudaGetLastError());
    }
    switch (pair_codes(desc->group)) {
        case 32: return launch_gs<32>(p, st);
        case 64: return launch_gs<64>(p, st);
        default: return launch_gs<128>(p, st);
    }
}
