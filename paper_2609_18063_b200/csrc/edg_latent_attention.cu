// Latent attention: y[t,h] = W_uv[h] sum_j softmax_j( scale (q_nope . W_uk[h] c_j + q_rope . p_j) ) c_j over the rows of a paged cache.
//
// A CTA takes one head of one new row: it brings the query to the latent space, walks the cache rows 128 at a time with a running
// maximum and sum, and multiplies by W_uv at the end.
#include "edg_latent.cuh"

namespace edg {
namespace {

struct AttendParams {
    LatentSeqs s;
    const uint16_t *q, *q_rope, *W_uk, *W_uv, *cache;
    void* y;
    int32_t* status;
    int heads, dn, dr, dv, dl, out_dtype;
    int64_t ldq, ldr;           // elements between rows of q and of the rotated parts
    int hr;                     // elements between heads of the rotated parts
    float scale;
    int max_new;
    int64_t total_len;
};

constexpr int kThreads = 128;

__global__ void __launch_bounds__(kThreads) attend_kernel(const __grid_constant__ AttendParams p) {
    __shared__ float s_q[576], s_o[512], s_p[kThreads], s_red[8];
    __shared__ int s_row[kThreads], s_at[3];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, t = blockIdx.x, h = blockIdx.y;
    if (t == 0 && h == 0 && tid == 0) {                       // the bounds that the caller gave
        long long all = 0;
        bool ok = p.s.cu[0] == 0 && p.s.cu[p.s.n] <= p.s.T;
        for (int i = 0; i < p.s.n; ++i) {
            all += max(p.s.lens[i], 0);
            ok = ok && p.s.cu[i + 1] >= p.s.cu[i] && p.s.cu[i + 1] - p.s.cu[i] <= p.max_new;
        }
        if (!ok || all > p.total_len) latent_raise(p.status, EDG_E_RANGE);
    }
    if (warp == 0) {
        const int seq = find_sequence(p.s.cu, p.s.n, t, lane);
        if (lane == 0) {
            s_at[0] = seq;
            s_at[1] = seq < p.s.n ? p.s.lens[seq] - p.s.cu[seq + 1] + t + 1 : 0;     // positions seen
        }
    }
    __syncthreads();
    const int seq = s_at[0];
    if (seq >= p.s.n) return;
    int len = s_at[1];
    const int most = p.s.max_pages << p.s.page_shift;
    if (len > most) { len = most; if (tid == 0) latent_raise(p.status, EDG_E_RANGE); }
    const uint16_t* q = p.q + (size_t)t * p.ldq + h * (p.dn + p.dr);
    for (int c = tid; c < p.dl; c += kThreads) {
        float a = 0.f;
        for (int n = 0; n < p.dn; ++n) a = fmaf(bf16_bits_to_float(q[n]), bf16_bits_to_float(p.W_uk[((size_t)h * p.dn + n) * p.dl + c]), a);
        s_q[c] = a * p.scale;
    }
    for (int c = tid; c < p.dr; c += kThreads) s_q[p.dl + c] = bf16_bits_to_float(p.q_rope[(size_t)t * p.ldr + h * p.hr + c]) * p.scale;
    float o[4] = {0.f, 0.f, 0.f, 0.f}, top = -INFINITY, sum = 0.f;
    const int row = p.dl + p.dr;
    for (int j0 = 0; j0 < len; j0 += kThreads) {
        __syncthreads();
        const int j = j0 + tid;
        int r = -1;
        if (j < len) {
            const int pg = p.s.table[(size_t)seq * p.s.max_pages + (j >> p.s.page_shift)];
            if (pg >= 0 && pg < p.s.n_pages) r = (pg << p.s.page_shift) + (j & ((1 << p.s.page_shift) - 1));
            else latent_raise(p.status, EDG_E_RANGE);
        }
        float sc = -INFINITY;
        if (r >= 0) {
            const uint4* k = reinterpret_cast<const uint4*>(p.cache + (size_t)r * row);
            sc = 0.f;
            for (int c = 0; c < row / 8; ++c) {
                const uint4 v = __ldg(k + c);
                const float* a = s_q + c * 8;
                sc = fmaf(bf16_lo(v.x), a[0], sc); sc = fmaf(bf16_hi(v.x), a[1], sc); sc = fmaf(bf16_lo(v.y), a[2], sc); sc = fmaf(bf16_hi(v.y), a[3], sc);
                sc = fmaf(bf16_lo(v.z), a[4], sc); sc = fmaf(bf16_hi(v.z), a[5], sc); sc = fmaf(bf16_lo(v.w), a[6], sc); sc = fmaf(bf16_hi(v.w), a[7], sc);
            }
        }
        float m = sc;
        for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, x));
        if (lane == 0) s_red[warp] = m;
        s_row[tid] = r;
        __syncthreads();
        m = fmaxf(fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])), top);
        const float fade = m == -INFINITY ? 1.f : expf(top - m), e = r < 0 ? 0.f : expf(sc - m);
        const float part = warp_sum(e);
        if (lane == 0) s_red[4 + warp] = part;
        s_p[tid] = e;
        __syncthreads();
        sum = sum * fade + ((s_red[4] + s_red[5]) + (s_red[6] + s_red[7]));
        top = m;
        for (int i = 0; i < 4; ++i) o[i] *= fade;
        for (int k = 0; k < kThreads && j0 + k < len; ++k) {
            if (s_row[k] < 0) continue;
            const uint16_t* v = p.cache + (size_t)s_row[k] * row;
            for (int i = 0; i < 4; ++i)
                if (tid + i * kThreads < p.dl) o[i] = fmaf(s_p[k], bf16_bits_to_float(v[tid + i * kThreads]), o[i]);
        }
    }
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    for (int i = 0; i < 4; ++i)
        if (tid + i * kThreads < p.dl) s_o[tid + i * kThreads] = o[i] * inv;
    __syncthreads();
    for (int n = tid; n < p.dv; n += kThreads) {
        float a = 0.f;
        for (int c = 0; c < p.dl; ++c) a = fmaf(s_o[c], bf16_bits_to_float(p.W_uv[((size_t)h * p.dv + n) * p.dl + c]), a);
        const size_t at = ((size_t)t * p.heads + h) * p.dv + n;
        if (p.out_dtype == EDG_F16) store_out(static_cast<__half*>(p.y), at, a);
        else static_cast<uint16_t*>(p.y)[at] = bf16_rn(a);
    }
}

}  // namespace
}  // namespace edg

using namespace edg;

extern "C" int32_t edg_latent_workspace_bytes(const edg_latent_desc* desc, int32_t n_seqs, int32_t T, int32_t max_new, int64_t total_len, size_t* bytes) {
    const int32_t rc = check_latent(desc);
    if (rc != EDG_OK) return rc;
    if (!bytes || n_seqs < 1 || n_seqs > 65535 || T < 1 || max_new < 1 || total_len < 0) return EDG_E_INVAL;
    *bytes = absorbed_workspace(*desc, n_seqs, T, max_new);
    return EDG_OK;
}

extern "C" int32_t latent_attention(const edg_latent_desc* desc, int32_t n_seqs, int32_t T, int32_t max_new, int64_t total_len, const int32_t* cu,
                                    const int32_t* lens, const int32_t* table, const void* q, const void* q_rope, const void* W_uk, const void* W_uv,
                                    const void* cache, void* y, void* workspace, size_t workspace_bytes, void* stream) {
    const int32_t rc = check_latent(desc);
    if (rc != EDG_OK) return rc;
    if (!cu || !lens || !table || !q || !W_uk || !W_uv || !cache || !y || !workspace || n_seqs < 1 || n_seqs > 65535 || T < 1 || max_new < 1 ||
        max_new > T || total_len < 0)
        return EDG_E_INVAL;
    if (!aligned(cu, 4) || !aligned(lens, 4) || !aligned(table, 4) || !aligned(q, 16) || !aligned(q_rope, 16) || !aligned(W_uk, 16) || !aligned(W_uv, 16) ||
        !aligned(cache, 16) || !aligned(y, 16))
        return EDG_E_INVAL;
    size_t need = 0;
    edg_latent_workspace_bytes(desc, n_seqs, T, max_new, total_len, &need);
    if (!aligned(workspace, 256) || workspace_bytes < need) return EDG_E_WORKSPACE;
    const bool absorbed = desc->form == EDG_LATENT_ABSORBED || (desc->form == EDG_LATENT_AUTO && max_new <= 128);
    if (absorbed) {
        const LatentSeqs s = {cu, lens, table, n_seqs, T, desc->max_pages, __builtin_ctz((unsigned)desc->page), desc->n_pages};
        return run_absorbed(*desc, s, max_new, q, q_rope, W_uk, W_uv, cache, y, workspace, static_cast<cudaStream_t>(stream));
    }
    AttendParams p = {};
    p.s = {cu, lens, table, n_seqs, T, desc->max_pages, __builtin_ctz((unsigned)desc->page), desc->n_pages};
    p.q = static_cast<const uint16_t*>(q);
    p.q_rope = q_rope != nullptr ? static_cast<const uint16_t*>(q_rope) : p.q + desc->d_nope;
    p.ldq = latent_ldq(*desc);
    p.ldr = q_rope != nullptr ? (int64_t)desc->heads * desc->d_rope : p.ldq;
    p.hr = q_rope != nullptr ? desc->d_rope : desc->d_nope + desc->d_rope;
    p.W_uk = static_cast<const uint16_t*>(W_uk);
    p.W_uv = static_cast<const uint16_t*>(W_uv);
    p.cache = static_cast<const uint16_t*>(cache);
    p.y = y;
    p.status = static_cast<int32_t*>(workspace);
    p.heads = desc->heads;
    p.dn = desc->d_nope;
    p.dr = desc->d_rope;
    p.dv = desc->d_v;
    p.dl = desc->d_latent;
    p.out_dtype = desc->out_dtype;
    p.scale = desc->scale;
    p.max_new = max_new;
    p.total_len = total_len;
    attend_kernel<<<dim3(T, desc->heads), kThreads, 0, static_cast<cudaStream_t>(stream)>>>(p);
    EDG_CUDA_TRY(cudaGetLastError());
    return EDG_OK;
}
