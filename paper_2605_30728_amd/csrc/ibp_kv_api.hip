// Entry points that write a paged KV cache and that hold it in 4 bits (include/ibp.h): checks of the arguments, then
// one or two launches on the caller's stream. Nothing is allocated, copied or synchronized here.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "ibp_attn_checks.hpp"
#include "ibp_kv_cache.hpp"

namespace ibp {
namespace {

using namespace attn;

// What is written must not lie in itself: no two rows, heads, pages or slots of it in the same place, as a stride of 0 has them
// or rows as far apart as the heads (queries turned in place would be turned again and again). From the smallest stride on, each is
// at least what those before it span; that takes any order of the dimensions, padding, and outputs in turns.
struct Dim {
    int64_t stride;
    uint64_t count;
};
template <size_t N>
bool apart(Dim (&&dims)[N], uint32_t width) {
    std::sort(dims, dims + N, [](const Dim &x, const Dim &y) { return x.stride < y.stride; });
    __int128 span = width;               // (2^31 pages of 2^40 values each do not fit 64 bits)
    for (const Dim &d : dims) {
        if (d.count <= 1) continue;
        if (d.stride < span) return false;
        span += (__int128)d.stride * (d.count - 1);
    }
    return true;
}
ibp_status take_apart(const Rows &r, uint64_t rows, uint32_t heads, uint32_t width, const char *what) {
    if (!rows || apart({{r.row, rows}, {r.head, heads}}, width)) return IBP_OK;
    return fail(IBP_EINVAL, std::string(what) + ": rows and heads that are written must not overlap");
}
ibp_status take_apart(const Pages &g, uint32_t heads, uint32_t width) {
    if (!g.n_pages) return IBP_OK;
    for (const attn::Pool &p : {g.k, g.v})
        if (!apart({{p.page, g.n_pages}, {p.head, heads}, {p.token, g.page_tokens}}, width))
            return fail(IBP_EINVAL, "pages, heads and slots that are written must not overlap");
    return IBP_OK;
}

// Packed rows of n_seqs sequences, or one row per sequence where there are no starts.
ibp_status take_packed(const int32_t *d_starts, uint32_t n_seqs, uint64_t rows, const ibp_pages *pages) {
    if (!aligned(d_starts, 4)) return fail(IBP_EINVAL, "sequence starts must be 4-byte aligned");
    if (n_seqs > 1u << 24) return fail(IBP_EINVAL, "too many sequences for one call");
    if (!d_starts && rows != n_seqs) return fail(IBP_EINVAL, "without starts every sequence has one row");
    if (rows && n_seqs && pages->n_pages && pages->table_pages && !pages->d_table) return fail(IBP_EINVAL, "page table is null");
    return IBP_OK;
}

ibp_status append_impl(bool four, const ibp_attn *p, const ibp_rows *k, const ibp_rows *v, const ibp_rows *q, const ibp_rows *q_out,
                       const ibp_rotation *rotation, const int32_t *d_starts, uint32_t n_seqs, const ibp_pages *pages,
                       const int32_t *d_lens, const int32_t *d_next, float *d_weights, int32_t *d_positions, uint64_t stride, void *stream) {
    Shape s;
    Append a{};
    IBP_TRY(take_shape(p, s));
    IBP_TRY(take_rows(k, "k", a.k));
    IBP_TRY(take_rows(v, "v", a.v));
    if (v->rows != k->rows) return fail(IBP_EINVAL, "k and v must have the same rows");
    if (!q != !q_out) return fail(IBP_EINVAL, "q and q_out: both or neither");
    if (q) {
        IBP_TRY(take_rows(q, "q", a.q));
        IBP_TRY(take_rows(q_out, "q_out", a.q_out));
        if (q->rows != k->rows) return fail(IBP_EINVAL, "q and k must have the same rows");
        if (q_out->rows < q->rows) return fail(IBP_ENOMEM, "q_out has fewer rows than q");
        if (q_out->data == q->data && (q_out->row_stride != q->row_stride || q_out->head_stride != q->head_stride))
            return fail(IBP_EINVAL, "in place q and q_out must have the same strides");
        IBP_TRY(take_apart(a.q_out, q->rows, s.q_heads, s.dim, "q_out"));
    }
    if (rotation && rotation->turned) {
        if (rotation->turned % 8 || rotation->turned > s.dim) return fail(IBP_EINVAL, "turned values must be a multiple of 8, at most head_dim");
        if (rotation->positions == 0 || rotation->positions > kMaxRows) return fail(IBP_EINVAL, "a rotation must have from 1 to 2^31 - 257 positions");
        if (!rotation->d_table) return fail(IBP_EINVAL, "rotation table is null");
        if (!aligned(rotation->d_table, 16)) return fail(IBP_EINVAL, "rotation table must be 16-byte aligned");
        a.rotation = rotation->d_table;
        a.positions = (uint32_t)rotation->positions;
        a.turned = rotation->turned;
        a.halves = rotation->halves != 0;
    }
    IBP_TRY(take_pages(pages, 0, a.pg));
    IBP_TRY(take_apart(a.pg, s.kv_heads, four ? record_bytes(s.dim) / 2 : s.dim));
    IBP_TRY(take_packed(d_starts, n_seqs, k->rows, pages));
    if (n_seqs && (!d_lens || !d_next)) return fail(IBP_EINVAL, "sequence lengths are null");
    if (!aligned(d_lens, 4) || !aligned(d_next, 4) || !aligned(d_weights, 4) || !aligned(d_positions, 4))
        return fail(IBP_EINVAL, "arrays must be 4-byte aligned");
    a.f16 = s.f16;
    a.four = four;
    a.q_heads = q ? s.q_heads : 0;
    a.kv_heads = s.kv_heads;
    a.dim = s.dim;
    a.starts = d_starts;
    a.n_seqs = n_seqs;
    a.rows = (uint32_t)k->rows;
    a.lens = d_lens;
    a.next = d_next;
    a.weights = d_weights;
    a.places = d_positions;
    a.stride = stride;
    return launched(launch_append(a, static_cast<hipStream_t>(stream)));
}

ibp_status read4_impl(const ibp_attn *p, const ibp_pages *pages, const int32_t *d_lens, uint32_t n_seqs, const int32_t *d_starts,
                      const int32_t *d_first, const ibp_rows *k, const ibp_rows *v, void *stream) {
    Shape s;
    Read4 r{};
    IBP_TRY(take_shape(p, s));
    IBP_TRY(take_rows(k, "k", r.k));
    IBP_TRY(take_rows(v, "v", r.v));
    if (v->rows != k->rows) return fail(IBP_EINVAL, "k and v must have the same rows");
    IBP_TRY(take_apart(r.k, k->rows, s.kv_heads, s.dim, "k"));
    IBP_TRY(take_apart(r.v, v->rows, s.kv_heads, s.dim, "v"));
    IBP_TRY(take_pages(pages, 0, r.pg));
    IBP_TRY(take_packed(d_starts, n_seqs, k->rows, pages));
    if (n_seqs && !d_lens) return fail(IBP_EINVAL, "sequence lengths are null");
    if (!aligned(d_lens, 4) || !aligned(d_first, 4)) return fail(IBP_EINVAL, "arrays must be 4-byte aligned");
    r.f16 = s.f16;
    r.kv_heads = s.kv_heads;
    r.dim = s.dim;
    r.starts = d_starts;
    r.first = d_first;
    r.n_seqs = n_seqs;
    r.rows = (uint32_t)k->rows;
    r.lens = d_lens;
    return launched(launch_read4(r, static_cast<hipStream_t>(stream)));
}

ibp_status decode4_impl(const ibp_attn *p, const ibp_rows *q, const ibp_pages *pages, const int32_t *d_lens, uint32_t max_len,
                        const ibp_rows *out, float *d_lse, float *d_weights, uint64_t weights_stride, void *workspace,
                        uint64_t workspace_bytes, void *stream) {
    Shape s;
    Rows rq, ro;
    Pages pg;
    IBP_TRY(take_shape(p, s));
    if (s.causal) return fail(IBP_EINVAL, "a new token sees its whole cache: no IBP_ATTN_CAUSAL here");
    IBP_TRY(take_rows(q, "q", rq));
    IBP_TRY(take_rows(out, "out", ro));
    if (out->rows < q->rows) return fail(IBP_ENOMEM, "out has fewer rows than q");
    IBP_TRY(take_apart(ro, q->rows, s.q_heads, s.dim, "out"));
    IBP_TRY(take_pages(pages, max_len, pg));
    IBP_TRY(check_paged((uint32_t)q->rows, s.kv_heads, d_lens));
    if (d_weights && weights_stride < max_len) return fail(IBP_ENOMEM, "weights have fewer slots than max_len");
    const uint32_t len = pg.n_pages ? max_len : 0;   // an empty pool holds no tokens
    const DecodePlan plan = plan_decode4((uint32_t)q->rows, s.q_heads, s.kv_heads, s.dim, len, d_weights != nullptr);
    IBP_TRY(take_workspace(workspace, workspace_bytes, q->rows ? plan.bytes : 0));
    return launched(launch_decode4(s, rq, pg, d_lens, (uint32_t)q->rows, len, ro, d_lse, d_weights, weights_stride, plan,
                                   static_cast<uint8_t *>(workspace), static_cast<hipStream_t>(stream)));
}

}  // namespace
}  // namespace ibp

using namespace ibp;

extern "C" {

ibp_status ibp_kv_append(const ibp_attn *a, const ibp_rows *k, const ibp_rows *v, const ibp_rows *q, const ibp_rows *q_out,
                         const ibp_rotation *rotation, const int32_t *d_starts, uint32_t n_seqs, const ibp_pages *pages,
                         const int32_t *d_lens, const int32_t *d_next, float *d_weights, int32_t *d_positions, uint64_t stride,
                         void *stream) {
    clear_error();
    return guarded([&] {
        return append_impl(false, a, k, v, q, q_out, rotation, d_starts, n_seqs, pages, d_lens, d_next, d_weights, d_positions, stride, stream);
    });
}

ibp_status ibp_kv4_record(uint32_t head_dim, uint32_t *bytes) {
    clear_error();
    if (!bytes) return fail(IBP_EINVAL, "bytes is null");
    if (head_dim == 0 || head_dim % 8 || head_dim > 256) return fail(IBP_EINVAL, "head_dim must be a multiple of 8 from 8 to 256");
    *bytes = record_bytes(head_dim);
    return IBP_OK;
}

ibp_status ibp_kv4_append(const ibp_attn *a, const ibp_rows *k, const ibp_rows *v, const ibp_rows *q, const ibp_rows *q_out,
                          const ibp_rotation *rotation, const int32_t *d_starts, uint32_t n_seqs, const ibp_pages *pages,
                          const int32_t *d_lens, const int32_t *d_next, float *d_weights, int32_t *d_positions, uint64_t stride,
                          void *stream) {
    clear_error();
    return guarded([&] {
        return append_impl(true, a, k, v, q, q_out, rotation, d_starts, n_seqs, pages, d_lens, d_next, d_weights, d_positions, stride, stream);
    });
}

ibp_status ibp_kv4_read(const ibp_attn *a, const ibp_pages *pages, const int32_t *d_lens, uint32_t n_seqs, const int32_t *d_starts,
                        const int32_t *d_first, const ibp_rows *k, const ibp_rows *v, void *stream) {
    clear_error();
    return guarded([&] { return read4_impl(a, pages, d_lens, n_seqs, d_starts, d_first, k, v, stream); });
}

ibp_status ibp_attn_decode4_workspace(uint32_t n_seqs, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim, uint32_t max_len,
                                      int weights, uint64_t *bytes) {
    clear_error();
    if (!bytes) return fail(IBP_EINVAL, "bytes is null");
    if (kv_heads == 0 || q_heads == 0 || q_heads % kv_heads || q_heads > 65536 || head_dim == 0 || head_dim % 8 ||
        head_dim > 256 || max_len > kMaxRows || (uint64_t)n_seqs * kv_heads > kMaxGrid)
        return fail(IBP_EINVAL, "bad sizes");
    *bytes = n_seqs ? decode4_workspace(n_seqs, q_heads, kv_heads, head_dim, max_len, weights != 0) : 0;
    return IBP_OK;
}

ibp_status ibp_attn_decode4(const ibp_attn *a, const ibp_rows *q, const ibp_pages *pages, const int32_t *d_lens, uint32_t max_len,
                            const ibp_rows *out, float *d_lse, float *d_weights, uint64_t weights_stride, void *workspace,
                            uint64_t workspace_bytes, void *stream) {
    clear_error();
    return guarded([&] {
        return decode4_impl(a, q, pages, d_lens, max_len, out, d_lse, d_weights, weights_stride, workspace, workspace_bytes, stream);
    });
}

}  // extern "C"
