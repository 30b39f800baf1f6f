// New rows of a latent cache: norm, rotation, write into pages; the queries' positional parts are rotated with them.
//
//     c = v / sqrt(mean v^2 + eps) * gain,     (a, b) -> (a cos - b sin, a sin + b cos) at angle position * inv_freq
//
// Bound by HBM for prompts (each row read and written once) and by latency for a step of decoding.  A row is a warp's, or with few rows a CTA's:
// one warp of it takes the cache row, all of them the heads of its query; a lane rotates pairs of eight consecutive values.  Angles are formed and brought to
// [-pi, pi] in double (a position of 10^5 and more leaves no digit of the angle in fp32), sine and cosine are fp32.  A value is rounded
// once, when it is written.  Measured with 32 heads and 512 + 64 columns: 64 rows of as many sequences 4.2 us in a graph (a wait for the
// sequence's place, one for the row), 4,430 rows 10.6 (46 MB: 4.3 TB/s, half of it from L2; 16.4 with all of it from memory).
#include "edg_latent.cuh"

namespace edg {
namespace {

constexpr int kAppendThreads = 256;

struct AppendParams {
    LatentSeqs s;
    const uint16_t *kv, *gain, *q;
    uint16_t *q_rope, *cache;
    const float* inv_freq;
    int32_t* status;
    int heads, dn, dr, dl, ldkv, halves;
    int64_t ldq;
    float eps;
};

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) { return (uint32_t)bf16_rn(a) | ((uint32_t)bf16_rn(b) << 16); }

// Eight values of a rotated part: values 8j.. of it (pairs lie beside one another), or values 4j.. of both halves.
__device__ __forceinline__ uint4 load8(const uint16_t* in, int j, int dr, bool halves) {
    if (!halves) return *reinterpret_cast<const uint4*>(in + 8 * j);
    const uint2 a = *reinterpret_cast<const uint2*>(in + 4 * j), b = *reinterpret_cast<const uint2*>(in + dr / 2 + 4 * j);
    return make_uint4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ void rotate8(const uint4& in, uint16_t* out, int j, int dr, bool halves, const float2* cs) {
    if (halves) {
        const float x[4] = {bf16_lo(in.x), bf16_hi(in.x), bf16_lo(in.y), bf16_hi(in.y)}, y[4] = {bf16_lo(in.z), bf16_hi(in.z), bf16_lo(in.w), bf16_hi(in.w)};
        float u[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 c = cs[4 * j + i];
            u[i] = x[i] * c.x - y[i] * c.y;
            v[i] = x[i] * c.y + y[i] * c.x;
        }
        *reinterpret_cast<uint2*>(out + 4 * j) = make_uint2(pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]));
        *reinterpret_cast<uint2*>(out + dr / 2 + 4 * j) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
    } else {
        const uint32_t w[4] = {in.x, in.y, in.z, in.w};
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 c = cs[4 * j + i];
            const float x = bf16_lo(w[i]), y = bf16_hi(w[i]);
            o[i] = pack_bf16(x * c.x - y * c.y, x * c.y + y * c.x);
        }
        *reinterpret_cast<uint4*>(out + 8 * j) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// 16-byte pieces of queries that a lane has in flight.  (With eight a thread needs 79 registers, and 4,430 rows take the warps of an SM a second
// time round: 13.3 us instead of 10.6.)
constexpr int kPieces = 4;

// WARPS: warps that share a row.  All that does not depend on the row's place is asked for first: the search for the sequence, its length, its
// page and the angles are a chain of four trips to memory, and run beside it.
template <int WARPS>
__global__ void __launch_bounds__(kAppendThreads, 4) append_kernel(const __grid_constant__ AppendParams p) {
    constexpr int kRows = kAppendThreads / 32 / WARPS;
    __shared__ float2 s_cs[kAppendThreads / 32][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = blockIdx.x * kRows + warp / WARPS, share = warp % WARPS;
    if (t >= p.s.T) return;
    const bool halves = p.halves != 0;
    const uint16_t* kv = p.kv + (size_t)t * p.ldkv;
    uint4 v[2] = {}, rot = {};
    if (share == 0) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (i * 256 + lane * 8 < p.dl) v[i] = *reinterpret_cast<const uint4*>(kv + i * 256 + lane * 8);
        if (lane < p.dr / 8) rot = load8(kv + p.dl, lane, p.dr, halves);
    }
    const int per = p.dr / 8, all = p.q != nullptr ? p.heads * per : 0, dh = p.dn + p.dr;
    const uint16_t* q = p.q + (size_t)t * p.ldq + p.dn;
    uint4 w[kPieces];
    auto ask = [&](int i0) {
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int i = i0 + (k * WARPS + share) * 32 + lane, h = i / per;
            if (i < all) w[k] = load8(q + h * dh, i - h * per, p.dr, halves);
        }
    };
    ask(0);
    const float freq = lane < p.dr / 2 ? p.inv_freq[lane] : 0.f;
    const int seq = find_sequence(p.s.cu, p.s.n, t, lane);
    if (seq >= p.s.n) return;                                            // behind the last sequence
    const int pos = p.s.lens[seq] - p.s.cu[seq + 1] + t;
    int row = -1;
    if (pos >= 0 && (pos >> p.s.page_shift) < p.s.max_pages) {
        const int pg = p.s.table[(size_t)seq * p.s.max_pages + (pos >> p.s.page_shift)];
        if (pg >= 0 && pg < p.s.n_pages) row = (pg << p.s.page_shift) + (pos & ((1 << p.s.page_shift) - 1));
    }
    if (row < 0) {
        if (lane == 0) latent_raise(p.status, EDG_E_RANGE);
        return;
    }
    float2* cs = s_cs[warp];
    if (lane < p.dr / 2) {
        double a = (double)pos * (double)freq;
        a -= 6.283185307179586476925 * rint(a * 0.15915494309189533577);
        float sn, cn;
        sincosf((float)a, &sn, &cn);
        cs[lane] = make_float2(cn, sn);
    }
    __syncwarp();
    if (share == 0) {
        uint16_t* out = p.cache + (size_t)row * (p.dl + p.dr);
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t x[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) { ss = fmaf(bf16_lo(x[j]), bf16_lo(x[j]), ss); ss = fmaf(bf16_hi(x[j]), bf16_hi(x[j]), ss); }
        }
        ss = warp_sum(ss);
        const float r = 1.f / sqrtf(ss / (float)p.dl + p.eps);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = i * 256 + lane * 8;
            if (c < p.dl) {
                uint4 g = make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);
                if (p.gain != nullptr) g = __ldg(reinterpret_cast<const uint4*>(p.gain + c));
                uint4 o;
                o.x = pack_bf16(bf16_lo(v[i].x) * r * bf16_lo(g.x), bf16_hi(v[i].x) * r * bf16_hi(g.x));
                o.y = pack_bf16(bf16_lo(v[i].y) * r * bf16_lo(g.y), bf16_hi(v[i].y) * r * bf16_hi(g.y));
                o.z = pack_bf16(bf16_lo(v[i].z) * r * bf16_lo(g.z), bf16_hi(v[i].z) * r * bf16_hi(g.z));
                o.w = pack_bf16(bf16_lo(v[i].w) * r * bf16_lo(g.w), bf16_hi(v[i].w) * r * bf16_hi(g.w));
                *reinterpret_cast<uint4*>(out + c) = o;
            }
        }
        if (lane < p.dr / 8) rotate8(rot, out + p.dl, lane, p.dr, halves, cs);
    }
    for (int i0 = 0; i0 < all; i0 += kPieces * WARPS * 32) {
        if (i0 > 0) ask(i0);
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int i = i0 + (k * WARPS + share) * 32 + lane, h = i / per;
            if (i < all) rotate8(w[k], p.q_rope + ((size_t)t * p.heads + h) * p.dr, i - h * per, p.dr, halves, cs);
        }
    }
}

}  // namespace
}  // namespace edg

using namespace edg;

extern "C" int32_t latent_append(const edg_latent_desc* desc, int32_t n_seqs, int32_t T, const int32_t* cu, const int32_t* lens, const int32_t* table,
                                 const void* kv, const void* gain, float eps, const float* inv_freq, const void* q, void* q_rope, void* cache,
                                 void* workspace, size_t workspace_bytes, void* stream) {
    const int32_t rc = check_latent(desc);
    if (rc != EDG_OK) return rc;
    if (!cu || !lens || !table || !kv || !inv_freq || !cache || !workspace || n_seqs < 1 || n_seqs > 65535 || T < 1 || !(eps >= 0.f)) return EDG_E_INVAL;
    if ((q == nullptr) != (q_rope == nullptr)) return EDG_E_INVAL;
    if (!aligned(cu, 4) || !aligned(lens, 4) || !aligned(table, 4) || !aligned(kv, 16) || !aligned(gain, 16) || !aligned(inv_freq, 4) || !aligned(q, 16) ||
        !aligned(q_rope, 16) || !aligned(cache, 16))
        return EDG_E_INVAL;
    if (!aligned(workspace, 256) || workspace_bytes < kCtrlBytes) return EDG_E_WORKSPACE;
    AppendParams p = {};
    p.s = {cu, lens, table, n_seqs, T, desc->max_pages, __builtin_ctz((unsigned)desc->page), desc->n_pages};
    p.kv = static_cast<const uint16_t*>(kv);
    p.gain = static_cast<const uint16_t*>(gain);
    p.q = static_cast<const uint16_t*>(q);
    p.q_rope = static_cast<uint16_t*>(q_rope);
    p.cache = static_cast<uint16_t*>(cache);
    p.inv_freq = inv_freq;
    p.status = static_cast<int32_t*>(workspace);
    p.heads = desc->heads;
    p.dn = desc->d_nope;
    p.dr = desc->d_rope;
    p.dl = desc->d_latent;
    p.ldkv = latent_ldkv(*desc);
    p.ldq = latent_ldq(*desc);
    p.halves = desc->rope_halves;
    p.eps = eps;
    // Few rows: the warps of a CTA share one; many: a warp each (4430 rows of 32 heads 10.6 us in a graph, with two warps to a row 11.9, with four
    // 14.0; 64 rows the other way round).
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (T < 1024) append_kernel<8><<<T, kAppendThreads, 0, st>>>(p);
    else append_kernel<1><<<(T + 7) / 8, kAppendThreads, 0, st>>>(p);
    EDG_CUDA_TRY(cudaGetLastError());
    return EDG_OK;
}
