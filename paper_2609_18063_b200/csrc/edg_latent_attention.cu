// Latent attention: the call, and which of its two forms a sequence takes.
#include "edg_latent.cuh"

namespace edg {
namespace {

// Up to how many new rows a sequence is taken in the absorbed form when the caller leaves it open.  Its work grows with them, the expanded
// form's hardly does below 128 (32 heads of 128, 512 latent columns, microseconds absorbed / expanded):
//     8 sequences of 2,000 positions:   16 rows  68 / 186    64: 223 / 187    128: 428 / 190
//     one of 1,000:                     16 rows  31 /  34    64:  39 /  34    128:  60 /  35
//     4 of 16,000:                      16 rows 142 / 711    64: 497 / 716    128: 948 / 694
constexpr int kAbsorbedMost = 64;
// Where some sequence has more, the others cost four launches in the absorbed form (20-40 us with little to do).  They are expanded along when
// they are short: a prompt of 1,024 rows beside 8 sequences of 500 positions takes 83 us so and 100 in two forms, beside 4 of 4,000 197 and 179.
// Their positions are known by their bound alone; 100 more for each stand for the CTAs of a sequence.
constexpr int64_t kAlongPositions = 5000;
bool expanded_along(const edg_latent_desc& d, int n_seqs, int max_new, int64_t total_len) {
    const int64_t others = (total_len > max_new ? total_len - max_new : 0) + 100ll * (n_seqs - 1);
    return n_seqs == 1 || others * (d.heads > 32 ? d.heads : 32) <= kAlongPositions * 32;
}

struct Forms {
    bool absorbed, expanded;
    int most;                   // new rows of a sequence in the absorbed form
    size_t first, bytes;        // scratch: where the expanded form's begins, and all of it
};
Forms forms(const edg_latent_desc& d, int n_seqs, int T, int max_new, int64_t total_len) {
    Forms f;
    if (d.form == EDG_LATENT_AUTO) f.most = max_new <= kAbsorbedMost ? max_new : (expanded_along(d, n_seqs, max_new, total_len) ? 0 : kAbsorbedMost);
    else f.most = d.form == EDG_LATENT_ABSORBED ? max_new : 0;
    f.absorbed = f.most > 0;
    f.expanded = max_new > f.most;
    // (scratch for both where the form is open, so that what serves some bounds serves all smaller ones)
    const int kept = d.form == EDG_LATENT_AUTO && max_new > kAbsorbedMost ? kAbsorbedMost : max_new;
    f.first = round_up(d.form != EDG_LATENT_EXPANDED ? absorbed_workspace(d, n_seqs, T, kept) : kCtrlBytes, 256);
    f.bytes = f.first + (f.expanded ? expanded_workspace(d, n_seqs, T, total_len) : 0);
    return f;
}

}  // namespace
}  // namespace edg

using namespace edg;

extern "C" int32_t edg_latent_workspace_bytes(const edg_latent_desc* desc, int32_t n_seqs, int32_t T, int32_t max_new, int64_t total_len, size_t* bytes) {
    const int32_t rc = check_latent(desc);
    if (rc != EDG_OK) return rc;
    if (!bytes || n_seqs < 1 || n_seqs > 65535 || T < 1 || T > 65535 || max_new < 1 || total_len < 0 || total_len > 0x7FFFFFFF) return EDG_E_INVAL;
    *bytes = forms(*desc, n_seqs, T, max_new, total_len).bytes;
    return EDG_OK;
}

extern "C" int32_t latent_attention(const edg_latent_desc* desc, int32_t n_seqs, int32_t T, int32_t max_new, int64_t total_len, const int32_t* cu,
                                    const int32_t* lens, const int32_t* table, const void* q, const void* q_rope, const void* W_uk, const void* W_uv,
                                    const void* cache, void* y, void* workspace, size_t workspace_bytes, void* stream) {
    const int32_t rc = check_latent(desc);
    if (rc != EDG_OK) return rc;
    if (!cu || !lens || !table || !q || !W_uk || !W_uv || !cache || !y || !workspace || n_seqs < 1 || n_seqs > 65535 || T < 1 || T > 65535 ||
        max_new < 1 || max_new > T || total_len < 0 || total_len > 0x7FFFFFFF)
        return EDG_E_INVAL;
    if (!aligned(cu, 4) || !aligned(lens, 4) || !aligned(table, 4) || !aligned(q, 16) || !aligned(q_rope, 16) || !aligned(W_uk, 16) || !aligned(W_uv, 16) ||
        !aligned(cache, 16) || !aligned(y, 16))
        return EDG_E_INVAL;
    const Forms f = forms(*desc, n_seqs, T, max_new, total_len);
    if (!aligned(workspace, 256) || workspace_bytes < f.bytes) return EDG_E_WORKSPACE;
    const LatentSeqs s = {cu, lens, table, n_seqs, T, desc->max_pages, __builtin_ctz((unsigned)desc->page), desc->n_pages};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (f.absorbed) {
        const int32_t e = run_absorbed(*desc, s, max_new, total_len, f.most, q, q_rope, W_uk, W_uv, cache, y, workspace, st);
        if (e != EDG_OK) return e;
    }
    if (f.expanded)
        return run_expanded(*desc, s, max_new, total_len, f.most, q, q_rope, W_uk, W_uv, cache, y, static_cast<int32_t*>(workspace),
                            static_cast<uint8_t*>(workspace) + f.first, st);
    return EDG_OK;
}
