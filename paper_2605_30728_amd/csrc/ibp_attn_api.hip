// Entry points of the attention operators (include/ibp.h): checks of the arguments, then one or
// two launches on the caller's stream. Nothing is allocated, copied or synchronized here.
#include <cmath>

#include <hip/hip_runtime.h>

#include "ibp_attn.hpp"
#include "ibp_internal.hpp"

namespace ibp {
namespace {

constexpr uint64_t kMaxRows = 0x7fffff00ull;      // rows and slots are counted in 31 bits
constexpr uint64_t kMaxEvictSlots = 0x7f000000ull;   // so that a block's last rounds and two numbers per move fit 31 bits
constexpr uint64_t kMaxRowStride = 1ull << 23;    // elements: 64 rows stay within 2^31 bytes

bool aligned(const void *p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

ibp_status take_shape(const ibp_attn *a, attn::Shape &s) {
    if (!a) return fail(IBP_EINVAL, "attention parameters are null");
    if (a->type != IBP_BF16 && a->type != IBP_F16) return fail(IBP_EINVAL, "type must be IBP_BF16 or IBP_F16");
    if (a->flags & ~(uint32_t)IBP_ATTN_CAUSAL) return fail(IBP_EINVAL, "unknown attention flags");
    if (a->kv_heads == 0 || a->q_heads == 0 || a->q_heads % a->kv_heads || a->q_heads > 65536)
        return fail(IBP_EINVAL, "query heads must be a positive multiple of the KV heads, at most 65536");
    if (a->head_dim == 0 || a->head_dim % 8 || a->head_dim > 256)
        return fail(IBP_EINVAL, "head_dim must be a multiple of 8 from 8 to 256");
    if (!std::isfinite(a->scale) || a->scale < 1e-30f || a->scale > 1e30f) return fail(IBP_EINVAL, "scale must be positive, from 1e-30 to 1e30");
    s = attn::Shape{a->q_heads, a->kv_heads, a->q_heads / a->kv_heads, a->head_dim, a->scale,
                    a->scale * 1.4426950408889634f, a->type == IBP_F16, (a->flags & IBP_ATTN_CAUSAL) != 0};
    return IBP_OK;
}

ibp_status take_rows(const ibp_rows *r, const char *what, attn::Rows &out) {
    if (!r) return fail(IBP_EINVAL, std::string(what) + " is null");
    if (r->rows > kMaxRows) return fail(IBP_EINVAL, std::string(what) + ": too many rows for one call");
    if (r->rows && !r->data) return fail(IBP_EINVAL, std::string(what) + ": data is null");
    if (!aligned(r->data, 16)) return fail(IBP_EINVAL, std::string(what) + ": data must be 16-byte aligned");
    if (r->row_stride % 8 || r->head_stride % 8)
        return fail(IBP_EINVAL, std::string(what) + ": strides must be multiples of 8 elements");
    if (r->row_stride > kMaxRowStride || r->head_stride > 1ull << 40)
        return fail(IBP_EINVAL, std::string(what) + ": stride too large");
    out = attn::Rows{r->data, (int64_t)r->row_stride, (int64_t)r->head_stride};
    return IBP_OK;
}

ibp_status take_starts(const int32_t *d_q_starts, const int32_t *d_k_starts, uint32_t n_seqs, uint64_t q_rows,
                       uint64_t k_rows, attn::Packed &p) {
    if (n_seqs && (!d_q_starts || !d_k_starts)) return fail(IBP_EINVAL, "sequence starts are null");
    if (!aligned(d_q_starts, 4) || !aligned(d_k_starts, 4)) return fail(IBP_EINVAL, "sequence starts must be 4-byte aligned");
    if (n_seqs > 1u << 24) return fail(IBP_EINVAL, "too many sequences for one call");
    p = attn::Packed{d_q_starts, d_k_starts, n_seqs, (uint32_t)q_rows, (uint32_t)k_rows};
    return IBP_OK;
}

ibp_status take_pages(const ibp_pages *g, uint64_t max_len, attn::Pages &out) {
    if (!g) return fail(IBP_EINVAL, "pages are null");
    if (g->page_tokens == 0 || g->page_tokens > 1u << 24) return fail(IBP_EINVAL, "page_tokens must be from 1 to 2^24");
    if (g->n_pages > kMaxRows) return fail(IBP_EINVAL, "too many pages");
    if (g->n_pages && (!g->keys || !g->values)) return fail(IBP_EINVAL, "page data is null");
    if (!aligned(g->keys, 16) || !aligned(g->values, 16)) return fail(IBP_EINVAL, "page data must be 16-byte aligned");
    const uint64_t strides[] = {g->key_page_stride,   g->key_head_stride,   g->key_token_stride,
                                g->value_page_stride, g->value_head_stride, g->value_token_stride};
    for (uint64_t x : strides) {
        if (x % 8) return fail(IBP_EINVAL, "page strides must be multiples of 8 elements");
        if (x > 1ull << 40) return fail(IBP_EINVAL, "page stride too large");
    }
    if (max_len > kMaxRows) return fail(IBP_EINVAL, "max_len is too large");
    if (max_len > (uint64_t)g->table_pages * g->page_tokens)
        return fail(IBP_ERANGE, "max_len is more than the page table holds");
    if (max_len && !g->d_table) return fail(IBP_EINVAL, "page table is null");
    if (!aligned(g->d_table, 4)) return fail(IBP_EINVAL, "page table must be 4-byte aligned");
    out = attn::Pages{};
    out.k = attn::Pool{g->keys, (int64_t)g->key_page_stride, (int64_t)g->key_head_stride, (int64_t)g->key_token_stride};
    out.v = attn::Pool{g->values, (int64_t)g->value_page_stride, (int64_t)g->value_head_stride, (int64_t)g->value_token_stride};
    out.table = g->d_table;
    out.table_stride = g->table_pages;
    out.n_pages = (uint32_t)g->n_pages;
    out.page_tokens = g->page_tokens;
    attn::page_division(g->page_tokens, out.page_magic, out.page_shift);
    return IBP_OK;
}

ibp_status take_workspace(void *workspace, uint64_t have, uint64_t need) {
    if (need == 0) return IBP_OK;
    if (!workspace) return fail(IBP_EINVAL, "workspace is null");
    if (!aligned(workspace, 16)) return fail(IBP_EINVAL, "workspace must be 16-byte aligned");
    if (have < need) return fail(IBP_ENOMEM, "workspace too small");
    return IBP_OK;
}

ibp_status launched(hipError_t e) {
    if (e == hipSuccess) return IBP_OK;
    if (e == hipErrorInvalidConfiguration) return fail(IBP_EINVAL, "too much work for one launch");
    return fail(IBP_EHIP, std::string("attention kernel: ") + hipGetErrorString(e));
}

ibp_status check_paged(uint32_t n_seqs, uint32_t kv_heads, const int32_t *d_lens) {
    if ((uint64_t)n_seqs * kv_heads > attn::kMaxGrid) return fail(IBP_EINVAL, "too many sequences for one call");
    if (n_seqs && !d_lens) return fail(IBP_EINVAL, "sequence lengths are null");
    return IBP_OK;
}

#define IBP_TRY(expr)                              \
    do {                                           \
        const ibp_status st_ = (expr);             \
        if (st_ != IBP_OK) return st_;             \
    } while (0)

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
