// What the decode kernels of 16-bit and of 4-bit caches share: their arguments, and the kernel that joins the blocks of
// a sequence (in ibp_attn_decode.hip).
#pragma once

#include "ibp_attn.hpp"

namespace ibp {
namespace attn {

struct DecodeArgs {
    Rows q, out;
    Pages pg;
    const int32_t *lens;
    float *lse, *weights;
    uint64_t weights_stride;
    float *stats;                // [n_seqs][q_heads][splits] pairs: reference (in scores) and sum
    float *partial;              // [n_seqs][q_heads][splits][dim]
    float *scores;               // [n_seqs][q_heads][scores_stride], null: not asked for
    uint32_t scores_stride;
    uint32_t n_seqs, q_heads, kv_heads, group, head_blocks, dim, max_len;
    uint32_t split_tokens, splits;
    float scale, scale_log2;
};

inline constexpr uint32_t kMaxSplits = 1024;

__device__ __forceinline__ int slots_of(const DecodeArgs &a, uint32_t seq) {
    return min(max(a.lens[seq], 0), (int)a.max_len);
}

// Joins the splits (where there are several) and adds the slots' weights (where they are asked for); blocks of that launch.
uint64_t decode_join_blocks(const DecodeArgs &a);
void launch_decode_join(const DecodeArgs &a, bool f16, hipStream_t stream);

}  // namespace attn
}  // namespace ibp
