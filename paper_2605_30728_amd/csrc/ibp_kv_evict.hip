// Eviction from a paged KV cache by accumulated attention weight.
//
// Of the n slots of a (sequence, KV head), m = min(n, budget) are kept: first those of the
// `recent` newest positions, then by weight, ties to the lowest slot. A kept slot below m stays
// where it is; the k-th freed slot below m takes the k-th kept slot from m on, so nothing is read
// that is written and the moves are as few as they can be.
//
// k_evict_select finds the m-th largest of the slots' 32-bit keys digit by digit (a radix select),
// marks what is kept and pairs the moves; k_evict_move copies the K and V rows.
#include "ibp_attn.hpp"
#include "ibp_attn_wave.hpp"

#include <algorithm>

namespace ibp {
namespace attn {

namespace {

using namespace dev;

struct EvictArgs {
    Evict e;
    int32_t *counts;             // [n_seqs][kv_heads] moves
    int32_t *moves;              // [n_seqs][kv_heads][move_stride] pairs: to, from
    uint32_t move_stride;
};

constexpr int kThreads = 1024;

// Larger keys are kept first: weights in the order of their values (NaN as the lowest, -0 as 0),
// above them all the positions that are kept anyway.
__device__ __forceinline__ uint32_t key_of(float w, bool guarded) {
    uint32_t u = __float_as_uint(w);
    if ((u & 0x7fffffffu) > 0x7f800000u) u = 0xff800000u;
    if (u == 0x80000000u) u = 0;
    u = u & 0x80000000u ? ~u : u | 0x80000000u;
    return guarded ? 0xffffffffu : u;
}

// Inclusive sum over the block of one small number per thread; total: the block's.
__device__ __forceinline__ int block_scan(int x, int *wave_sums, int &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int sum = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(sum, d);
        if (lane >= d) sum += y;
    }
    __syncthreads();
    if (lane == 63) wave_sums[wave] = sum;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        const int s = wave_sums[w];
        if (w < wave) before += s;
        total += s;
    }
    return before + sum;
}

__global__ __launch_bounds__(kThreads) void k_evict_select(EvictArgs a) {
    __shared__ uint32_t bins[256];
    __shared__ int wave_sums[kThreads / 64];
    __shared__ uint32_t chosen[2];
    const Evict &e = a.e;
    const uint32_t seq = blockIdx.x / e.kv_heads;
    const int n = min(max(e.lens[seq], 0), (int)e.max_len), m = min(n, (int)e.budget);
    const int64_t newest = (int64_t)e.next[seq] - e.recent;
    const float *w = e.weights + (int64_t)blockIdx.x * e.stride;
    const int32_t *pos = e.positions + (int64_t)blockIdx.x * e.stride;
    float *new_w = e.new_weights + (int64_t)blockIdx.x * e.new_stride;
    int32_t *new_pos = e.new_positions + (int64_t)blockIdx.x * e.new_stride;
    int32_t *moves = a.moves + (int64_t)blockIdx.x * a.move_stride * 2;
    auto key = [&](int i) { return key_of(w[i], pos[i] >= newest); };

    if (m == n) {                        // everything is kept
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const float x = w[i];
            const int32_t y = pos[i];
            new_w[i] = x;
            new_pos[i] = y;
        }
        if (threadIdx.x == 0) a.counts[blockIdx.x] = 0;
        return;
    }

    // the m-th largest key and how many of those equal to it are kept
    uint32_t prefix = 0, left = m;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (threadIdx.x < 256) bins[threadIdx.x] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const uint32_t k = key(i);
            if (shift == 24 || k >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&bins[k >> shift & 255], 1u);
        }
        __syncthreads();
        if (threadIdx.x < 64) {          // the digit at which the count from above reaches `left`
            uint32_t b[4], sum = 0;
#pragma unroll
            for (int x = 0; x < 4; ++x) sum += b[x] = bins[255 - (threadIdx.x * 4 + x)];
            uint32_t upto = sum;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t y = __shfl_up(upto, d);
                if ((int)threadIdx.x >= d) upto += y;
            }
            uint32_t above = upto - sum;
            if (above < left && upto >= left) {
                int x = 0;
                while (above + b[x] < left) above += b[x++];
                chosen[0] = 255 - (threadIdx.x * 4 + x);
                chosen[1] = left - above;
            }
        }
        __syncthreads();
        prefix |= chosen[0] << shift;
        left = chosen[1];
    }

    // the freed slots below m and the kept ones from m on, each in ascending order
    int ties = 0, holes = 0, movers = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        const uint32_t k = i < n ? key(i) : 0;
        int total;
        const bool tie = i < n && k == prefix;
        const int nth = ties + block_scan(tie, wave_sums, total);
        ties += total;
        const bool keep = i < n && (k > prefix || (tie && nth <= (int)left));
        const bool hole = i < m && !keep, mover = i >= m && keep;
        const int both = block_scan(hole ? 1 : mover ? 1 << 16 : 0, wave_sums, total);
        if (hole) moves[(holes + (both & 0xffff) - 1) * 2] = i;
        if (mover) moves[(movers + (both >> 16) - 1) * 2 + 1] = i;
        holes += total & 0xffff;
        movers += total >> 16;
    }
    if (threadIdx.x == 0) a.counts[blockIdx.x] = holes;

    // the arrays: what stays, then what moves (in place too: nothing below m is read for a move)
    for (int i = threadIdx.x; i < m; i += kThreads) {
        const float x = w[i];
        const int32_t y = pos[i];
        new_w[i] = x;
        new_pos[i] = y;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < holes; i += kThreads) {
        const int to = moves[i * 2], of = moves[i * 2 + 1];
        new_w[to] = w[of];
        new_pos[to] = pos[of];
    }
}

constexpr int kMoveThreads = 256;

// A block takes moves x, x + per, ... of a (sequence, KV head), 16 bytes of K or V per thread.
__global__ __launch_bounds__(kMoveThreads) void k_evict_move(EvictArgs a, uint32_t per) {
    const Evict &e = a.e;
    const uint32_t sh = blockIdx.x / per, x = blockIdx.x % per, seq = sh / e.kv_heads, kv = sh % e.kv_heads;
    if (kv == 0 && x == 0 && threadIdx.x == 0) e.new_lens[seq] = min(min(max(e.lens[seq], 0), (int)e.max_len), (int)e.budget);
    const int count = a.counts[sh];
    const int32_t *moves = a.moves + (int64_t)sh * a.move_stride * 2;
    const int32_t *table = e.pg.table + (int64_t)seq * e.pg.table_stride;
    const uint32_t chunks = e.row_bytes / 16, items = 2 * chunks;        // of K, then of V
    auto at = [&](const Pool &p, uint32_t slot, bool &there) {
        const uint32_t i = e.pg.page_magic ? __umulhi(slot, e.pg.page_magic) >> e.pg.page_shift : slot >> e.pg.page_shift;
        const int32_t page = table[i];
        there = (uint32_t)page < e.pg.n_pages;
        return (uint8_t *)p.data + ((int64_t)(there ? page : 0) * p.page + (int64_t)(slot - i * e.pg.page_tokens) * p.token + (int64_t)kv * p.head) * 2;
    };
    const uint64_t total = (uint64_t)count * items;
    for (uint64_t t = (uint64_t)x * kMoveThreads + threadIdx.x; t < total; t += (uint64_t)per * kMoveThreads) {
        const uint32_t mv = (uint32_t)(t / items), it = (uint32_t)(t % items);
        const Pool &p = it < chunks ? e.pg.k : e.pg.v;
        const uint32_t byte = (it < chunks ? it : it - chunks) * 16;
        bool to_there, of_there;
        uint8_t *to = at(p, moves[mv * 2], to_there);
        const uint8_t *of = at(p, moves[mv * 2 + 1], of_there);
        if (to_there && of_there) *reinterpret_cast<u32x4 *>(to + byte) = *reinterpret_cast<const u32x4 *>(of + byte);
    }
}

uint64_t up256(uint64_t x) { return (x + 255) / 256 * 256; }

}  // namespace

uint64_t evict_workspace(uint32_t n_seqs, uint32_t kv_heads, uint32_t max_len, uint32_t budget) {
    const uint64_t rows = (uint64_t)n_seqs * kv_heads, most = std::min(budget, max_len);
    return up256(rows * 4) + up256(rows * most * 8);
}

hipError_t launch_evict(const Evict &e, uint8_t *workspace, hipStream_t stream) {
    const uint64_t rows = (uint64_t)e.n_seqs * e.kv_heads;
    if (rows == 0) return hipSuccess;
    EvictArgs a{e, (int32_t *)workspace, (int32_t *)(workspace + up256(rows * 4)), std::min(e.budget, e.max_len)};
    // blocks per head for the copies: enough to fill the chip, 8 KiB of copies at least
    const uint64_t bytes = (uint64_t)std::min(e.budget, e.max_len - std::min(e.budget, e.max_len)) * e.row_bytes * 2;
    const uint32_t per = (uint32_t)std::min<uint64_t>(std::max<uint64_t>(bytes / 8192, 1), std::max<uint64_t>(2048 / rows, 1));
    if (rows * per > kMaxGrid) return hipErrorInvalidConfiguration;
    k_evict_select<<<dim3((uint32_t)rows), dim3(kThreads), 0, stream>>>(a);
    k_evict_move<<<dim3((uint32_t)(rows * per)), dim3(kMoveThreads), 0, stream>>>(a, per);
    return hipGetLastError();
}

}  // namespace attn
}  // namespace ibp
