// Entry points of the attention operators (include/ibp.h): checks of the arguments, then one or
// two launches on the caller's stream. Nothing is allocated, copied or synchronized here.
#include <hip/hip_runtime.h>

#include "ibp_attn_checks.hpp"

namespace ibp {
namespace {

using namespace attn;

ibp_status prompt_impl(const ibp_attn *a, const ibp_rows *q, const ibp_rows *k, const ibp_rows *v,
                       const int32_t *d_q_starts, const int32_t *d_k_starts, uint32_t n_seqs, const ibp_rows *out,
                       float *d_lse, void *workspace, uint64_t workspace_bytes, void *stream) {
    attn::Shape s;
    attn::Rows rq, rk, rv, ro;
    attn::Packed p;
    IBP_TRY(take_shape(a, s));
    IBP_TRY(take_rows(q, "q", rq));
    IBP_TRY(take_rows(k, "k", rk));
    IBP_TRY(take_rows(v, "v", rv));
    IBP_TRY(take_rows(out, "out", ro));
    if (v->rows != k->rows) return fail(IBP_EINVAL, "k and v must have the same rows");
    if (out->rows < q->rows) return fail(IBP_ENOMEM, "out has fewer rows than q");
    IBP_TRY(take_starts(d_q_starts, d_k_starts, n_seqs, q->rows, k->rows, p));
    IBP_TRY(take_workspace(workspace, workspace_bytes, attn::prompt_needs(s.q_heads, s.dim, q->rows, k->rows, n_seqs)));
    return launched(attn::launch_prompt(s, rq, rk, rv, p, ro, d_lse, static_cast<uint8_t *>(workspace),
                                        static_cast<hipStream_t>(stream)));
}

ibp_status key_weights_impl(const ibp_attn *a, const ibp_rows *q, const ibp_rows *k, const int32_t *d_q_starts,
                            const int32_t *d_k_starts, uint32_t n_seqs, const float *d_lse, float *d_weights,
                            void *workspace, uint64_t workspace_bytes, void *stream) {
    attn::Shape s;
    attn::Rows rq, rk;
    attn::Packed p;
    IBP_TRY(take_shape(a, s));
    IBP_TRY(take_rows(q, "q", rq));
    IBP_TRY(take_rows(k, "k", rk));
    IBP_TRY(take_starts(d_q_starts, d_k_starts, n_seqs, q->rows, k->rows, p));
    if (q->rows && !d_lse) return fail(IBP_EINVAL, "lse is null");
    if (k->rows && !d_weights) return fail(IBP_EINVAL, "weights are null");
    IBP_TRY(take_workspace(workspace, workspace_bytes, attn::key_weights_workspace(s.q_heads, s.kv_heads, k->rows, n_seqs)));
    return launched(attn::launch_key_weights(s, rq, rk, p, d_lse, d_weights, static_cast<float *>(workspace),
                                             static_cast<hipStream_t>(stream)));
}

ibp_status decode_impl(const ibp_attn *a, const ibp_rows *q, const ibp_pages *pages, const int32_t *d_lens,
                       uint32_t max_len, const ibp_rows *out, float *d_lse, float *d_weights, uint64_t weights_stride,
                       void *workspace, uint64_t workspace_bytes, void *stream) {
    attn::Shape s;
    attn::Rows rq, ro;
    attn::Pages pg;
    IBP_TRY(take_shape(a, s));
    if (s.causal) return fail(IBP_EINVAL, "a new token sees its whole cache: no IBP_ATTN_CAUSAL here");
    IBP_TRY(take_rows(q, "q", rq));
    IBP_TRY(take_rows(out, "out", ro));
    if (out->rows < q->rows) return fail(IBP_ENOMEM, "out has fewer rows than q");
    IBP_TRY(take_pages(pages, max_len, pg));
    IBP_TRY(check_paged((uint32_t)q->rows, s.kv_heads, d_lens));
    if (d_weights && weights_stride < max_len) return fail(IBP_ENOMEM, "weights have fewer slots than max_len");
    const uint32_t len = pg.n_pages ? max_len : 0;   // an empty pool holds no tokens
    const attn::DecodePlan plan = attn::plan_decode((uint32_t)q->rows, s.q_heads, s.kv_heads, s.dim, len, d_weights != nullptr);
    IBP_TRY(take_workspace(workspace, workspace_bytes, q->rows ? plan.bytes : 0));
    return launched(attn::launch_decode(s, rq, pg, d_lens, (uint32_t)q->rows, len, ro, d_lse, d_weights, weights_stride,
                                        plan, static_cast<uint8_t *>(workspace), static_cast<hipStream_t>(stream)));
}

ibp_status evict_impl(const ibp_attn *a, const ibp_pages *pages, const int32_t *d_lens, uint32_t n_seqs,
                      uint32_t max_len, uint32_t budget, uint32_t recent, const int32_t *d_next,
                      const float *d_weights, const int32_t *d_positions, uint64_t stride, float *d_new_weights,
                      int32_t *d_new_positions, uint64_t new_stride, int32_t *d_new_lens, void *workspace,
                      uint64_t workspace_bytes, void *stream) {
    attn::Shape s;
    attn::Evict e{};
    IBP_TRY(take_shape(a, s));
    IBP_TRY(take_pages(pages, max_len, e.pg));
    IBP_TRY(check_paged(n_seqs, s.kv_heads, d_lens));
    if (max_len > kMaxEvictSlots) return fail(IBP_EINVAL, "max_len is too large for an eviction");
    if (budget == 0 || budget > kMaxRows) return fail(IBP_EINVAL, "budget must be at least 1");
    if (recent > budget) return fail(IBP_EINVAL, "more recent positions than the budget");
    if (n_seqs == 0) return IBP_OK;
    if (!d_next || !d_weights || !d_positions || !d_new_weights || !d_new_positions || !d_new_lens)
        return fail(IBP_EINVAL, "an array of the eviction is null");
    const uint64_t kept = budget < max_len ? budget : max_len;
    if (stride < max_len) return fail(IBP_EINVAL, "weights have fewer slots than max_len");
    if (new_stride < kept) return fail(IBP_ENOMEM, "the new weights have fewer slots than what is kept");
    if ((d_new_weights == d_weights || d_new_positions == d_positions) && new_stride != stride)
        return fail(IBP_EINVAL, "in place the arrays must have the same stride");
    e.kv_heads = s.kv_heads;
    e.row_bytes = s.dim * 2;
    e.lens = d_lens;
    e.next = d_next;
    e.n_seqs = n_seqs;
    e.max_len = e.pg.n_pages ? max_len : 0;          // an empty pool holds no tokens
    e.budget = budget;
    e.recent = recent;
    e.weights = d_weights;
    e.positions = d_positions;
    e.new_weights = d_new_weights;
    e.new_positions = d_new_positions;
    e.new_lens = d_new_lens;
    e.stride = stride;
    e.new_stride = new_stride;
    IBP_TRY(take_workspace(workspace, workspace_bytes, attn::evict_workspace(n_seqs, s.kv_heads, max_len, budget)));
    return launched(attn::launch_evict(e, static_cast<uint8_t *>(workspace), static_cast<hipStream_t>(stream)));
}

}  // namespace
}  // namespace ibp

using namespace ibp;

extern "C" {

ibp_status ibp_attn_prompt_workspace(uint32_t q_heads, uint32_t head_dim, uint64_t q_rows, uint64_t k_rows, uint32_t n_seqs,
                                     uint64_t *bytes) {
    clear_error();
    if (!bytes) return fail(IBP_EINVAL, "bytes is null");
    if (q_heads == 0 || q_heads > 65536 || head_dim == 0 || head_dim % 8 || head_dim > 256 || q_rows > kMaxRows || k_rows > kMaxRows)
        return fail(IBP_EINVAL, "bad sizes");
    *bytes = attn::prompt_workspace(q_heads, head_dim, q_rows, k_rows, n_seqs);
    return IBP_OK;
}

ibp_status ibp_attn_prompt(const ibp_attn *a, const ibp_rows *q, const ibp_rows *k, const ibp_rows *v,
                           const int32_t *d_q_starts, const int32_t *d_k_starts, uint32_t n_seqs, const ibp_rows *out,
                           float *d_lse, void *workspace, uint64_t workspace_bytes, void *stream) {
    clear_error();
    return guarded([&] {
        return prompt_impl(a, q, k, v, d_q_starts, d_k_starts, n_seqs, out, d_lse, workspace, workspace_bytes, stream);
    });
}

ibp_status ibp_attn_key_weights_workspace(uint32_t q_heads, uint32_t kv_heads, uint64_t k_rows, uint32_t n_seqs,
                                          uint64_t *bytes) {
    clear_error();
    if (!bytes) return fail(IBP_EINVAL, "bytes is null");
    if (kv_heads == 0 || q_heads == 0 || q_heads % kv_heads || q_heads > 65536 || k_rows > kMaxRows)
        return fail(IBP_EINVAL, "bad sizes");
    *bytes = attn::key_weights_workspace(q_heads, kv_heads, k_rows, n_seqs);
    return IBP_OK;
}

ibp_status ibp_attn_key_weights(const ibp_attn *a, const ibp_rows *q, const ibp_rows *k, const int32_t *d_q_starts,
                                const int32_t *d_k_starts, uint32_t n_seqs, const float *d_lse, float *d_weights,
                                void *workspace, uint64_t workspace_bytes, void *stream) {
    clear_error();
    return guarded([&] {
        return key_weights_impl(a, q, k, d_q_starts, d_k_starts, n_seqs, d_lse, d_weights, workspace, workspace_bytes, stream);
    });
}

ibp_status ibp_attn_decode_workspace(uint32_t n_seqs, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim,
                                     uint32_t max_len, int weights, uint64_t *bytes) {
    clear_error();
    if (!bytes) return fail(IBP_EINVAL, "bytes is null");
    if (kv_heads == 0 || q_heads == 0 || q_heads % kv_heads || q_heads > 65536 || head_dim == 0 || head_dim % 8 ||
        head_dim > 256 || max_len > kMaxRows || (uint64_t)n_seqs * kv_heads > attn::kMaxGrid)
        return fail(IBP_EINVAL, "bad sizes");
    *bytes = n_seqs ? attn::decode_workspace(n_seqs, q_heads, kv_heads, head_dim, max_len, weights != 0) : 0;
    return IBP_OK;
}

ibp_status ibp_attn_decode(const ibp_attn *a, const ibp_rows *q, const ibp_pages *pages, const int32_t *d_lens,
                           uint32_t max_len, const ibp_rows *out, float *d_lse, float *d_weights,
                           uint64_t weights_stride, void *workspace, uint64_t workspace_bytes, void *stream) {
    clear_error();
    return guarded([&] {
        return decode_impl(a, q, pages, d_lens, max_len, out, d_lse, d_weights, weights_stride, workspace,
                           workspace_bytes, stream);
    });
}

ibp_status ibp_kv_evict_workspace(uint32_t n_seqs, uint32_t kv_heads, uint32_t max_len, uint32_t budget, uint64_t *bytes) {
    clear_error();
    if (!bytes) return fail(IBP_EINVAL, "bytes is null");
    if (kv_heads == 0 || max_len > kMaxEvictSlots || budget == 0 || budget > kMaxRows || (uint64_t)n_seqs * kv_heads > attn::kMaxGrid)
        return fail(IBP_EINVAL, "bad sizes");
    *bytes = attn::evict_workspace(n_seqs, kv_heads, max_len, budget);
    return IBP_OK;
}

ibp_status ibp_kv_evict(const ibp_attn *a, const ibp_pages *pages, const int32_t *d_lens, uint32_t n_seqs,
                        uint32_t max_len, uint32_t budget, uint32_t recent, const int32_t *d_next,
                        const float *d_weights, const int32_t *d_positions, uint64_t stride, float *d_new_weights,
                        int32_t *d_new_positions, uint64_t new_stride, int32_t *d_new_lens, void *workspace,
                        uint64_t workspace_bytes, void *stream) {
    clear_error();
    return guarded([&] {
        return evict_impl(a, pages, d_lens, n_seqs, max_len, budget, recent, d_next, d_weights, d_positions, stride,
                          d_new_weights, d_new_positions, new_stride, d_new_lens, workspace, workspace_bytes, stream);
    });
}

}  // extern "C"
