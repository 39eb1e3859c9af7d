// Launchers of the attention kernels over KV tensors (ibp_attn_*.hip, ibp_kv_evict.hip).
#pragma once

#include <cstdint>

#include <hip/hip_runtime.h>

#include "ibp.h"

namespace ibp {
namespace attn {

// Rows of a 2-byte type as [row][head][dim]; strides in elements.
struct Rows {
    void *data;
    int64_t row, head;
};

// What every attention kernel is told; sizes are checked by the entry points.
struct Shape {
    uint32_t q_heads, kv_heads, group;   // group = q_heads / kv_heads
    uint32_t dim;                        // a multiple of 8, at most 256
    float scale;                         // > 0
    float scale_log2;                    // scale * log2(e)
    bool f16;                            // else bf16
    bool causal;
};

// Packed sequences: rows [starts[s], starts[s + 1]) belong to sequence s.
struct Packed {
    const int32_t *q_starts, *k_starts;
    uint32_t n_seqs;
    uint32_t q_rows, k_rows;             // rows of the tensors: no start beyond them is followed
};

hipError_t launch_prompt(const Shape &a, const Rows &q, const Rows &k, const Rows &v, const Packed &p, const Rows &out,
                         float *lse, uint8_t *workspace, hipStream_t stream);
// What a call needs (nothing where the tiles fill the chip by themselves), and what is enough for it and for every
// call of fewer rows.
uint64_t prompt_needs(uint32_t q_heads, uint32_t dim, uint64_t q_rows, uint64_t k_rows, uint32_t n_seqs);
uint64_t prompt_workspace(uint32_t q_heads, uint32_t dim, uint64_t q_rows, uint64_t k_rows, uint32_t n_seqs);

// partial: the workspace (unused, may be null, where it has 0 bytes).
uint64_t key_weights_workspace(uint32_t q_heads, uint32_t kv_heads, uint64_t k_rows, uint32_t n_seqs);
hipError_t launch_key_weights(const Shape &a, const Rows &q, const Rows &k, const Packed &p, const float *lse,
                              float *weights, float *partial, hipStream_t stream);

// A paged pool of K or V rows; strides in elements.
struct Pool {
    void *data;
    int64_t page, head, token;
};

struct Pages {
    Pool k, v;
    const int32_t *table;                // [n_seqs][table_stride]
    uint32_t table_stride;               // pages per sequence in the table
    uint32_t n_pages;
    uint32_t page_tokens;
    uint32_t page_magic;                 // slot / page_tokens = mulhi(slot, page_magic) >> page_shift (magic 0: >> shift)
    uint32_t page_shift;
};

// slot / page_tokens for slots below 2^31 as a multiply-high and a shift.
void page_division(uint32_t page_tokens, uint32_t &magic, uint32_t &shift);

// How a decode call is split over the cache's length, and the workspace it needs.
struct DecodePlan {
    uint32_t head_blocks;                // blocks of at most 16 query heads per KV head
    uint32_t split_tokens;               // slots per split, a multiple of 128
    uint32_t splits;                     // splits of the longest sequence
    uint64_t stats_off, out_off, scores_off, bytes;
};
DecodePlan plan_decode(uint32_t n_seqs, uint32_t q_heads, uint32_t kv_heads, uint32_t dim, uint32_t max_len,
                       bool weights);
// Enough for the plan of this and of every smaller call (fewer sequences, a smaller max_len).
uint64_t decode_workspace(uint32_t n_seqs, uint32_t q_heads, uint32_t kv_heads, uint32_t dim, uint32_t max_len, bool weights);

hipError_t launch_decode(const Shape &a, const Rows &q, const Pages &pg, const int32_t *lens, uint32_t n_seqs,
                         uint32_t max_len, const Rows &out, float *lse, float *weights, uint64_t weights_stride,
                         const DecodePlan &plan, uint8_t *workspace, hipStream_t stream);

struct Evict {
    Pages pg;
    uint32_t kv_heads, row_bytes;
    const int32_t *lens, *next;
    uint32_t n_seqs, max_len, budget, recent;
    const float *weights;
    const int32_t *positions;
    float *new_weights;
    int32_t *new_positions, *new_lens;
    uint64_t stride, new_stride;         // slots per head of the arrays
};
uint64_t evict_workspace(uint32_t n_seqs, uint32_t kv_heads, uint32_t max_len, uint32_t budget);
hipError_t launch_evict(const Evict &e, uint8_t *workspace, hipStream_t stream);

// Blocks that one launch may have (a grid's threads are counted in 32 bits).
inline constexpr uint64_t kMaxGrid = 0xFFFFFFFFull / 1024;

}  // namespace attn
}  // namespace ibp
