// Checks of the arguments that the attention and KV cache entry points share; each fills what the launchers take.
#pragma once

#include <cmath>
#include <string>

#include "ibp_attn.hpp"
#include "ibp_internal.hpp"

namespace ibp {
namespace attn {

inline constexpr uint64_t kMaxRows = 0x7fffff00ull;      // rows and slots are counted in 31 bits
inline constexpr uint64_t kMaxEvictSlots = 0x7f000000ull;   // so that a block's last rounds and two numbers per move fit 31 bits
inline constexpr uint64_t kMaxRowStride = 1ull << 23;    // elements: 64 rows stay within 2^31 bytes

inline bool aligned(const void *p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

inline ibp_status take_shape(const ibp_attn *a, Shape &s) {
    if (!a) return fail(IBP_EINVAL, "attention parameters are null");
    if (a->type != IBP_BF16 && a->type != IBP_F16) return fail(IBP_EINVAL, "type must be IBP_BF16 or IBP_F16");
    if (a->flags & ~(uint32_t)IBP_ATTN_CAUSAL) return fail(IBP_EINVAL, "unknown attention flags");
    if (a->kv_heads == 0 || a->q_heads == 0 || a->q_heads % a->kv_heads || a->q_heads > 65536)
        return fail(IBP_EINVAL, "query heads must be a positive multiple of the KV heads, at most 65536");
    if (a->head_dim == 0 || a->head_dim % 8 || a->head_dim > 256)
        return fail(IBP_EINVAL, "head_dim must be a multiple of 8 from 8 to 256");
    if (!std::isfinite(a->scale) || a->scale < 1e-30f || a->scale > 1e30f) return fail(IBP_EINVAL, "scale must be positive, from 1e-30 to 1e30");
    s = Shape{a->q_heads, a->kv_heads, a->q_heads / a->kv_heads, a->head_dim, a->scale,
                    a->scale * 1.4426950408889634f, a->type == IBP_F16, (a->flags & IBP_ATTN_CAUSAL) != 0};
    return IBP_OK;
}

inline ibp_status take_rows(const ibp_rows *r, const char *what, Rows &out) {
    if (!r) return fail(IBP_EINVAL, std::string(what) + " is null");
    if (r->rows > kMaxRows) return fail(IBP_EINVAL, std::string(what) + ": too many rows for one call");
    if (r->rows && !r->data) return fail(IBP_EINVAL, std::string(what) + ": data is null");
    if (!aligned(r->data, 16)) return fail(IBP_EINVAL, std::string(what) + ": data must be 16-byte aligned");
    if (r->row_stride % 8 || r->head_stride % 8)
        return fail(IBP_EINVAL, std::string(what) + ": strides must be multiples of 8 elements");
    if (r->row_stride > kMaxRowStride || r->head_stride > 1ull << 40)
        return fail(IBP_EINVAL, std::string(what) + ": stride too large");
    out = Rows{r->data, (int64_t)r->row_stride, (int64_t)r->head_stride};
    return IBP_OK;
}

inline ibp_status take_starts(const int32_t *d_q_starts, const int32_t *d_k_starts, uint32_t n_seqs, uint64_t q_rows,
                       uint64_t k_rows, Packed &p) {
    if (n_seqs && (!d_q_starts || !d_k_starts)) return fail(IBP_EINVAL, "sequence starts are null");
    if (!aligned(d_q_starts, 4) || !aligned(d_k_starts, 4)) return fail(IBP_EINVAL, "sequence starts must be 4-byte aligned");
    if (n_seqs > 1u << 24) return fail(IBP_EINVAL, "too many sequences for one call");
    p = Packed{d_q_starts, d_k_starts, n_seqs, (uint32_t)q_rows, (uint32_t)k_rows};
    return IBP_OK;
}

inline ibp_status take_pages(const ibp_pages *g, uint64_t max_len, Pages &out) {
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
    out = Pages{};
    out.k = Pool{g->keys, (int64_t)g->key_page_stride, (int64_t)g->key_head_stride, (int64_t)g->key_token_stride};
    out.v = Pool{g->values, (int64_t)g->value_page_stride, (int64_t)g->value_head_stride, (int64_t)g->value_token_stride};
    out.table = g->d_table;
    out.table_stride = g->table_pages;
    out.n_pages = (uint32_t)g->n_pages;
    out.page_tokens = g->page_tokens;
    page_division(g->page_tokens, out.page_magic, out.page_shift);
    return IBP_OK;
}

inline ibp_status take_workspace(void *workspace, uint64_t have, uint64_t need) {
    if (need == 0) return IBP_OK;
    if (!workspace) return fail(IBP_EINVAL, "workspace is null");
    if (!aligned(workspace, 16)) return fail(IBP_EINVAL, "workspace must be 16-byte aligned");
    if (have < need) return fail(IBP_ENOMEM, "workspace too small");
    return IBP_OK;
}

inline ibp_status launched(hipError_t e) {
    if (e == hipSuccess) return IBP_OK;
    if (e == hipErrorInvalidConfiguration) return fail(IBP_EINVAL, "too much work for one launch");
    return fail(IBP_EHIP, std::string("attention kernel: ") + hipGetErrorString(e));
}

inline ibp_status check_paged(uint32_t n_seqs, uint32_t kv_heads, const int32_t *d_lens) {
    if ((uint64_t)n_seqs * kv_heads > kMaxGrid) return fail(IBP_EINVAL, "too many sequences for one call");
    if (n_seqs && !d_lens) return fail(IBP_EINVAL, "sequence lengths are null");
    return IBP_OK;
}

#define IBP_TRY(expr)                              \
    do {                                           \
        const ibp_status st_ = (expr);             \
        if (st_ != IBP_OK) return st_;             \
    } while (0)

}  // namespace attn
}  // namespace ibp
