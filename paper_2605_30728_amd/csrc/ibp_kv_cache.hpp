// Launchers of the kernels that write a paged KV cache and that read one of 4-bit records.
#pragma once

#include "ibp_attn.hpp"

namespace ibp {
namespace attn {

// A record: what a 4-bit cache holds of one token of one head, in groups of 32 values.
inline constexpr uint32_t kGroupValues = 32, kGroupBytes = 16;
__host__ __device__ constexpr uint32_t record_groups(uint32_t dim) { return (dim + kGroupValues - 1) / kGroupValues; }
__host__ __device__ constexpr uint32_t record_bytes(uint32_t dim) { return (record_groups(dim) * (kGroupBytes + 4) + 15) / 16 * 16; }

struct Append {
    bool f16, four;                      // four: pools of records
    uint32_t q_heads, kv_heads, dim;     // q_heads 0: no queries
    Rows q, q_out, k, v;
    const float *rotation;               // [positions][turned / 2] pairs of cosine and sine
    uint32_t positions, turned;
    bool halves;
    const int32_t *starts;               // null: one row per sequence
    uint32_t n_seqs, rows;
    Pages pg;
    const int32_t *lens, *next;
    float *weights;                      // [n_seqs][kv_heads][stride], null: not kept
    int32_t *places;                     // the slots' positions, the same
    uint64_t stride;
};
hipError_t launch_append(const Append &a, hipStream_t stream);

struct Read4 {
    bool f16;
    uint32_t kv_heads, dim;
    Rows k, v;
    const int32_t *starts, *first;       // null: one row per sequence; sequences from slot 0 on
    uint32_t n_seqs, rows;
    Pages pg;
    const int32_t *lens;
};
hipError_t launch_read4(const Read4 &r, hipStream_t stream);

DecodePlan plan_decode4(uint32_t n_seqs, uint32_t q_heads, uint32_t kv_heads, uint32_t dim, uint32_t max_len, bool weights);
uint64_t decode4_workspace(uint32_t n_seqs, uint32_t q_heads, uint32_t kv_heads, uint32_t dim, uint32_t max_len, bool weights);
hipError_t launch_decode4(const Shape &a, const Rows &q, const Pages &pg, const int32_t *lens, uint32_t n_seqs,
                          uint32_t max_len, const Rows &out, float *lse, float *weights, uint64_t weights_stride,
                          const DecodePlan &plan, uint8_t *workspace, hipStream_t stream);

}  // namespace attn
}  // namespace ibp
