// Attention of one new token per sequence over a paged cache of 4-bit records.
//
// The cache's length is split over blocks, which the decode of 16-bit caches' second kernel joins:
//   x_j = scale sum_d q_d k_jd,   out = sum_j p_j v_j,   k and v = centre + (code - 7.5) step of their group of 32.
#include <algorithm>

#include "ibp_attn_decode.hpp"
#include "ibp_attn_wave.hpp"
#include "ibp_kv_cache.hpp"

namespace ibp {
namespace attn {

namespace {

using namespace dev;

// Four values of a record from place d on.
template <class T>
__device__ __forceinline__ f32x4 values_at(const uint8_t *record, uint32_t d, uint32_t groups) {
    const uint32_t code = *reinterpret_cast<const uint16_t *>(record + d / 2);
    const uint8_t *meta = record + groups * kGroupBytes + d / kGroupValues * 2;
    const float step = T::value(*reinterpret_cast<const uint16_t *>(meta)), centre = T::value(*reinterpret_cast<const uint16_t *>(meta + groups * 2));
    f32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __builtin_fmaf((float)(code >> 4 * i & 15) - 7.5f, step, centre);
    return x;
}

// A wave per split and query head, slot by slot; a lane has four values of the head.
template <class T>
__global__ __launch_bounds__(64) void k_attn_decode4(DecodeArgs a) {
    const uint32_t head = blockIdx.x % a.q_heads, seq = blockIdx.x / a.q_heads % a.n_seqs, split = blockIdx.x / a.q_heads / a.n_seqs;
    const uint32_t kv = head / a.group, groups = record_groups(a.dim), d = threadIdx.x * 4;
    const int len = slots_of(a, seq), from = split * a.split_tokens, to = from < len ? from + min(len - from, (int)a.split_tokens) : from;
    if (from >= to && split) return;
    const bool in = d < a.dim;
    const float inf = __builtin_inff(), c = a.scale_log2;
    float q[4] = {};
    if (in)
        for (int i = 0; i < 4; ++i)
            q[i] = T::value(*(reinterpret_cast<const uint16_t *>(a.q.data) + (int64_t)seq * a.q.row + (int64_t)head * a.q.head + d + i));
    float m = -inf, l = 0.f;
    f32x4 acc{};
    float *sp = a.scores ? a.scores + ((int64_t)seq * a.q_heads + head) * a.scores_stride : nullptr;
    for (int slot = from; slot < to; ++slot) {
        const uint32_t i = a.pg.page_magic ? __umulhi(slot, a.pg.page_magic) >> a.pg.page_shift : (uint32_t)slot >> a.pg.page_shift;
        const int32_t page = a.pg.table[(int64_t)seq * a.pg.table_stride + i];
        const bool there = (uint32_t)page < a.pg.n_pages;
        float x = -inf;
        f32x4 v{};
        if (there) {
            const int64_t row = slot - i * a.pg.page_tokens;
            const uint8_t *kr = (const uint8_t *)a.pg.k.data + ((int64_t)page * a.pg.k.page + (int64_t)kv * a.pg.k.head + row * a.pg.k.token) * 2;
            const uint8_t *vr = (const uint8_t *)a.pg.v.data + ((int64_t)page * a.pg.v.page + (int64_t)kv * a.pg.v.head + row * a.pg.v.token) * 2;
            float sum = 0.f;
            if (in) {
                const f32x4 k = values_at<T>(kr, d, groups);
                v = values_at<T>(vr, d, groups);
                for (int y = 0; y < 4; ++y) sum = __builtin_fmaf(q[y], k[y], sum);
            }
            for (int y = 1; y < 64; y <<= 1) sum += __shfl_xor(sum, y);
            x = sum;
        }
        if (sp && threadIdx.x == 0) sp[slot] = x;
        if (x > m) {
            const float keep = m == -inf ? 0.f : exp2_fast((m - x) * c);
            l *= keep;
            acc *= keep;
            m = x;
        }
        if (!there) continue;
        const float p = exp2_fast((x - (m == -inf ? 0.f : m)) * c);
        l += p;
        acc += p * v;
    }
    const bool last = a.splits == 1;
    const int64_t part = ((int64_t)seq * a.q_heads + head) * a.splits + split;
    if (threadIdx.x == 0) {
        if (last && a.lse) a.lse[(int64_t)seq * a.q_heads + head] = l == 0.f ? -inf : m * a.scale + __logf(l);
        if (!last || a.weights) {
            a.stats[part * 2] = m;
            a.stats[part * 2 + 1] = l;
        }
    }
    if (!in) return;
    if (last) {
        acc *= l == 0.f ? 0.f : 1.f / l;
        *reinterpret_cast<u32x2 *>((uint8_t *)a.out.data + ((int64_t)seq * a.out.row + (int64_t)head * a.out.head + d) * 2) =
            u32x2{T::pack_out(acc[0], acc[1]), T::pack_out(acc[2], acc[3])};
    } else {
        *reinterpret_cast<f32x4 *>(a.partial + part * a.dim + d) = acc;
    }
}

}  // namespace

DecodePlan plan_decode4(uint32_t n_seqs, uint32_t q_heads, uint32_t kv_heads, uint32_t dim, uint32_t max_len, bool weights) {
    return plan_decode(n_seqs, q_heads, kv_heads, dim, max_len, weights);
}

uint64_t decode4_workspace(uint32_t n_seqs, uint32_t q_heads, uint32_t kv_heads, uint32_t dim, uint32_t max_len, bool weights) {
    return decode_workspace(n_seqs, q_heads, kv_heads, dim, max_len, weights);
}

hipError_t launch_decode4(const Shape &s, const Rows &q, const Pages &pg, const int32_t *lens, uint32_t n_seqs,
                          uint32_t max_len, const Rows &out, float *lse, float *weights, uint64_t weights_stride,
                          const DecodePlan &plan, uint8_t *workspace, hipStream_t stream) {
    if (n_seqs == 0) return hipSuccess;
    const uint64_t blocks = (uint64_t)n_seqs * plan.splits * s.q_heads;
    DecodeArgs a{q, out, pg, lens, lse, weights, weights_stride, (float *)(workspace + plan.stats_off),
                 (float *)(workspace + plan.out_off), weights ? (float *)(workspace + plan.scores_off) : nullptr,
                 (max_len + 31) / 32 * 32, n_seqs, s.q_heads, s.kv_heads, s.group, plan.head_blocks, s.dim, max_len,
                 plan.split_tokens, plan.splits, s.scale, s.scale_log2};
    if (blocks > kMaxGrid || decode_join_blocks(a) > kMaxGrid) return hipErrorInvalidConfiguration;
    if (s.f16) k_attn_decode4<F16><<<dim3((uint32_t)blocks), dim3(64), 0, stream>>>(a);
    else k_attn_decode4<Bf16><<<dim3((uint32_t)blocks), dim3(64), 0, stream>>>(a);
    launch_decode_join(a, s.f16, stream);
    return hipGetLastError();
}

}  // namespace attn
}  // namespace ibp
