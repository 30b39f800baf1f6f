// What the latent-attention translation units share: descriptor checks, the sequences of a batch, the scratch layout.
#pragma once

#include "edg_common.cuh"

namespace edg {

inline int32_t check_latent(const edg_latent_desc* d) {
    if (d == nullptr) return EDG_E_INVAL;
    auto part = [](int v, int most) { return v >= 16 && v <= most && v % 16 == 0; };
    if (d->heads < 1 || d->heads > 256 || !part(d->d_nope, 128) || !part(d->d_rope, 64) || !part(d->d_v, 128)) return EDG_E_SHAPE;
    if (d->d_latent < 128 || d->d_latent > 512 || d->d_latent % 128 != 0) return EDG_E_SHAPE;
    if (d->page < 16 || d->page > 256 || (d->page & (d->page - 1)) != 0) return EDG_E_SHAPE;
    if (d->n_pages < 1 || d->max_pages < 1 || (int64_t)d->n_pages * d->page > 0x7FFFFFFF || (int64_t)d->max_pages * d->page > 0x7FFFFFFF) return EDG_E_SHAPE;
    if (d->out_dtype != EDG_F16 && d->out_dtype != EDG_BF16) return EDG_E_INVAL;
    if (d->rope_halves != 0 && d->rope_halves != 1) return EDG_E_INVAL;
    if (d->form < EDG_LATENT_AUTO || d->form > EDG_LATENT_EXPANDED) return EDG_E_INVAL;
    if (!(d->scale > 0.f) || d->scale > 3.4e38f) return EDG_E_INVAL;
    if (d->ldkv != 0 && (d->ldkv < d->d_latent + d->d_rope || d->ldkv % 8 != 0)) return EDG_E_SHAPE;
    if (d->ldq != 0 && (d->ldq < d->heads * (d->d_nope + d->d_rope) || d->ldq % 8 != 0)) return EDG_E_SHAPE;
    return EDG_OK;
}

inline int latent_row(const edg_latent_desc& d) { return d.d_latent + d.d_rope; }
inline int latent_ldkv(const edg_latent_desc& d) { return d.ldkv != 0 ? d.ldkv : latent_row(d); }
inline int latent_ldq(const edg_latent_desc& d) { return d.ldq != 0 ? d.ldq : d.heads * (d.d_nope + d.d_rope); }

// The sequences of a call as the kernels get them.
struct LatentSeqs {
    const int32_t* cu;          // [n + 1]
    const int32_t* lens;        // [n]
    const int32_t* table;       // [n][max_pages]
    int n, T, max_pages, page_shift, n_pages;
};

// The absorbed form (edg_latent_absorbed.cu) of sequences of up to `most` new rows: scratch, control block included, and the launches.
size_t absorbed_workspace(const edg_latent_desc& d, int n_seqs, int T, int most);
int32_t run_absorbed(const edg_latent_desc& d, const LatentSeqs& s, int max_new, int64_t total_len, int most, const void* q, const void* q_rope,
                     const void* W_uk, const void* W_uv, const void* cache, void* y, void* workspace, cudaStream_t st);
// The expanded form (edg_latent_expanded.cu) of sequences of more new rows than `more_than`: scratch, a control block not among it.
size_t expanded_workspace(const edg_latent_desc& d, int n_seqs, int T, int64_t total_len);
int32_t run_expanded(const edg_latent_desc& d, const LatentSeqs& s, int max_new, int64_t total_len, int more_than, const void* q, const void* q_rope,
                     const void* W_uk, const void* W_uv, const void* cache, void* y, int32_t* status, void* scratch, cudaStream_t st);

#ifdef __CUDACC__

// Sequence of row t: the i with cu[i] <= t < cu[i + 1], or n where t lies behind the last one.  A whole warp looks: 32 places at a time.
__device__ __forceinline__ int find_sequence(const int32_t* cu, int n, int t, int lane) {
    int lo = 0, hi = n;                                  // the number of ends cu[1..n] that are <= t
    while (hi > lo) {
        const int step = (hi - lo + 31) / 32, at = lo + lane * step;
        const bool le = at < hi && cu[at + 1] <= t;
        const int c = __popc(__ballot_sync(0xFFFFFFFFu, le));
        if (c == 0) return lo;
        const int nlo = lo + (c - 1) * step + 1;
        hi = min(hi, lo + c * step);
        lo = nlo;
    }
    return lo;
}

__device__ __forceinline__ void latent_raise(int32_t* status, int32_t code) { atomicCAS(status, 0, code); }

#endif

}  // namespace edg
