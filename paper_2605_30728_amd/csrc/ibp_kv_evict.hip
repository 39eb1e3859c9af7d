// Eviction from a paged KV cache by accumulated attention weight.
//
// Of the n slots of a (sequence, KV head), m = min(n, budget) are kept: first those of the
// `recent` newest positions, then by weight, ties to the lowest slot. A kept slot below m stays
// where it is; the k-th freed slot below m takes the k-th kept slot from m on, so nothing is read
// that is written and the moves are as few as they can be.
//
// k_evict_select, a block per (sequence, KV head), finds the m-th largest of the slots' 32-bit keys
// in three digits (a radix select), ranks what is kept by ballots, pairs the moves and writes the
// new arrays; k_evict_move copies the K and V rows, or the first kernel does where they are few.
//
// Bound by the latency of the selection's passes, since a (sequence, KV head) is one block's: weights and positions
// are read from HBM once, later passes find their keys in LDS. The copies are bound by HBM. 32 heads of 32,768
// slots of 128 down to 4,096: 64 us (131 MB); 128 heads of 2,049 slots, one too many: 11 us.
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

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2048;
constexpr uint32_t kFewMoves = 128;       // moves per head that the first kernel makes by itself

// Larger keys are kept first: weights in the order of their values (NaN as the lowest, -0 as 0),
// above them all the positions that are kept anyway. No slot has key 0.
__device__ __forceinline__ uint32_t key_of(float w, bool guarded) {
    uint32_t u = __float_as_uint(w);
    if ((u & 0x7fffffffu) > 0x7f800000u) u = 0xff800000u;
    if (u == 0x80000000u) u = 0;
    u = u & 0x80000000u ? ~u : u | 0x80000000u;
    return guarded ? 0xffffffffu : u;
}

// Copies the rows of moves: a wave takes 64 / pieces of them at a time, a piece being 16 bytes of
// K's row or, after those, of V's; move0, move0 + stride, ... of `count` by this wave, N rounds' loads before
// their stores (no row that is written is read).
template <int N>
__device__ __forceinline__ void copy_rows(const Evict &e, const int32_t *moves, uint32_t seq, uint32_t kv, uint32_t count,
                                          uint32_t wave, uint32_t waves) {
    const uint32_t lane = threadIdx.x & 63, chunks = e.row_bytes / 16, pieces = 2 * chunks;
    const uint32_t sub = lane / pieces, piece = lane - sub * pieces, at_once = 64 / pieces;
    const Pool &p = piece < chunks ? e.pg.k : e.pg.v;
    uint8_t *base = (uint8_t *)p.data + (int64_t)kv * p.head * 2 + (piece < chunks ? piece : piece - chunks) * 16;
    const int64_t page_bytes = p.page * 2, token_bytes = p.token * 2;
    const int32_t *table = e.pg.table + (int64_t)seq * e.pg.table_stride;
    auto row = [&](uint32_t slot, bool &there) {
        const uint32_t i = e.pg.page_magic ? __umulhi(slot, e.pg.page_magic) >> e.pg.page_shift : slot >> e.pg.page_shift;
        const int32_t page = table[i];
        there = (uint32_t)page < e.pg.n_pages;
        return base + (there ? page : 0) * page_bytes + (int64_t)(slot - i * e.pg.page_tokens) * token_bytes;
    };
    for (uint64_t mv = sub < at_once ? (uint64_t)wave * at_once + sub : count; mv < count; mv += (uint64_t)waves * at_once * N) {
        uint8_t *to[N];
        u32x4 x[N];
        bool both[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint64_t t = mv + (uint64_t)i * waves * at_once;
            const uint64_t pair = min(t, (uint64_t)count - 1);
            bool to_there, of_there;
            to[i] = row(moves[pair * 2], to_there);
            x[i] = *reinterpret_cast<const u32x4 *>(row(moves[pair * 2 + 1], of_there));
            both[i] = to_there && of_there && t < count;
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (both[i]) *reinterpret_cast<u32x4 *>(to[i]) = x[i];
    }
}

__device__ __forceinline__ int kept_of(const Evict &e, int n) { return min(n, (int)e.budget); }
__device__ __forceinline__ int slots_of(const Evict &e, uint32_t seq) { return min(max(e.lens[seq], 0), (int)e.max_len); }

// Sums over the waves before this one, and over all of them, of two numbers that each wave has.
struct Before {
    int x, y, all_x, all_y;
};
__device__ __forceinline__ Before before_wave(int x, int y, int (*sums)[2]) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        sums[wave][0] = x;
        sums[wave][1] = y;
    }
    __syncthreads();
    Before b{};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const int sx = sums[w][0], sy = sums[w][1];
        b.x += w < wave ? sx : 0;
        b.y += w < wave ? sy : 0;
        b.all_x += sx;
        b.all_y += sy;
    }
    return b;
}

// Wave w has the slots [w, w + 1) * 64 rounds, 64 in each of its rounds, a multiple of four. The keys of up to KEYS
// slots are held in LDS, KEYS = 0: computed again in every pass. (Loops over LDS rather than keys in
// registers: unrolled over 32 registers the passes are so long that fetching their code takes
// longer than they do.)
template <int KEYS, bool MOVE>
__global__ __launch_bounds__(kThreads) void k_evict_select(EvictArgs a) {
    __shared__ uint32_t held[KEYS ? KEYS : 1];
    __shared__ uint32_t bins[kBins];
    __shared__ int sums[kWaves][2];
    __shared__ uint32_t chosen[2];
    __shared__ int32_t pairs[MOVE ? 2 * kFewMoves : 1];
    const Evict &e = a.e;
    const uint32_t seq = blockIdx.x / e.kv_heads, kv = blockIdx.x % e.kv_heads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = slots_of(e, seq), m = kept_of(e, n);
    const int64_t newest = (int64_t)e.next[seq] - e.recent;
    const float *w = e.weights + (int64_t)blockIdx.x * e.stride;
    const int32_t *pos = e.positions + (int64_t)blockIdx.x * e.stride;
    float *new_w = e.new_weights + (int64_t)blockIdx.x * e.new_stride;
    int32_t *new_pos = e.new_positions + (int64_t)blockIdx.x * e.new_stride;
    int32_t *moves = a.moves + (int64_t)blockIdx.x * a.move_stride * 2;
    if (MOVE && kv == 0 && threadIdx.x == 0) e.new_lens[seq] = m;

    const int rounds = (n + 4 * kThreads - 1) / (4 * kThreads) * 4, first = wave * rounds * 64 + lane;
    // what stays below m, and what the movers then replace (in place: the same values)
    for (int i = threadIdx.x; i < m; i += kThreads) {
        const float x = w[i];
        const int32_t y = pos[i];
        new_w[i] = x;
        new_pos[i] = y;
    }
    if (m == n) {                                    // everything is kept
        if (threadIdx.x == 0) a.counts[blockIdx.x] = 0;
        return;
    }

    const int end = n - 1;
    auto key_at = [&](int slot) {
        const uint32_t k = key_of(w[min(slot, end)], pos[min(slot, end)] >= newest);
        return slot < n ? k : 0u;
    };
    auto each = [&](auto &&f) {                      // f(slot, key) over the wave's slots, in order
        for (int r = 0; r < rounds; r += 4) {
            uint32_t k[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int slot = first + (r + i) * 64;
                if constexpr (KEYS != 0) k[i] = held[slot];
                else k[i] = key_at(slot);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) f(first + (r + i) * 64, k[i]);
        }
    };

    // the m-th largest key and how many of those equal to it are kept
    uint32_t prefix = 0, left = m;
#pragma unroll 1
    for (int digit = 0; digit < 3; ++digit) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0;
        const uint32_t last = digit == 2 ? 1023 : 2047;
        for (int i = threadIdx.x; i < kBins; i += kThreads) bins[i] = 0;
        __syncthreads();
        if (digit == 0) {                            // (a wave reads back only the keys that it wrote)
            constexpr int kBatch = KEYS == 4096 ? 4 : KEYS == 16384 ? 8 : 16;    // loads on their way together
            for (int r0 = 0; r0 < rounds; r0 += kBatch) {
                float bw[kBatch];
                int32_t bp[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    bw[i] = w[min(first + (r0 + i) * 64, end)];
                    bp[i] = pos[min(first + (r0 + i) * 64, end)];
                }
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    const int slot = first + (r0 + i) * 64;
                    if (r0 + i >= rounds) break;
                    const uint32_t k = slot < n ? key_of(bw[i], bp[i] >= newest) : 0u;
                    if constexpr (KEYS != 0) held[slot] = k;
                    if (slot < n) atomicAdd(&bins[k >> 21], 1u);
                }
            }
        } else {
            const int above = digit == 1 ? 21 : 10;
            const uint32_t want = prefix >> above;
            each([&](int, uint32_t k) {              // (key 0 of no slot is below every prefix)
                if (k >> above == want) atomicAdd(&bins[k >> shift & last], 1u);
            });
        }
        __syncthreads();
        // two bins per thread, the highest first: the one at which the count from above reaches `left`
        const uint32_t hi = last - threadIdx.x * 2;
        const uint32_t b0 = threadIdx.x * 2 <= last ? bins[hi] : 0, b1 = threadIdx.x * 2 < last ? bins[hi - 1] : 0;
        const uint32_t upto = ::ibp::dev::wave_incl_scan(b0 + b1);
        const Before before = before_wave(__builtin_amdgcn_readlane((int)upto, 63), 0, sums);
        const uint32_t above = (uint32_t)before.x + upto - b0 - b1;
        if (above < left && above + b0 + b1 >= left) {
            const bool second = above + b0 < left;
            chosen[0] = second ? hi - 1 : hi;
            chosen[1] = left - above - (second ? b0 : 0);
        }
        __syncthreads();
        prefix |= chosen[0] << shift;
        left = chosen[1];
    }

    // How many of a wave's slots are kept on either side of m, and of those how many equal the last
    // key kept: of these the first `left` in the order of the slots are, so that a wave's holes
    // (freed slots below m) and movers (kept ones from m on) follow from four counts.
    int more_lo = 0, more_hi = 0, tie_lo = 0, tie_hi = 0;
    each([&](int slot, uint32_t k) {
        const uint64_t lo = __ballot(slot < m), more = __ballot(k > prefix), tie = __ballot(k == prefix);
        more_lo += __popcll(more & lo);
        more_hi += __popcll(more & ~lo);
        tie_lo += __popcll(tie & lo);
        tie_hi += __popcll(tie & ~lo);
    });
    const int ties = tie_lo + tie_hi;
    int tie_at = before_wave(ties, 0, sums).x;
    const int kept_ties = min(max((int)left - tie_at, 0), ties), kept_lo = min(kept_ties, tie_lo);
    const int slots_lo = min(max(m - wave * rounds * 64, 0), rounds * 64);
    const Before moved = before_wave(slots_lo - more_lo - kept_lo, more_hi + kept_ties - kept_lo, sums);
    int hole_at = moved.x, mover_at = moved.y;
    const int n_holes = moved.all_x;

    const uint64_t below = (1ull << lane) - 1;
    int32_t *to_list = MOVE ? pairs : moves;         // (the few moves of this kernel stay in LDS)
    each([&](int slot, uint32_t k) {
        const uint64_t tie = __ballot(k == prefix);
        const bool keep = k > prefix || (k == prefix && tie_at + __popcll(tie & below) < (int)left);
        tie_at += __popcll(tie);
        const bool hole = slot < m && !keep, mover = slot >= m && keep;
        const uint64_t h = __ballot(hole), v = __ballot(mover);
        if (hole) to_list[(hole_at + __popcll(h & below)) * 2] = slot;
        if (mover) to_list[(mover_at + __popcll(v & below)) * 2 + 1] = slot;
        hole_at += __popcll(h);
        mover_at += __popcll(v);
    });
    __syncthreads();                                 // (in place nothing below m is read for a move)
    if constexpr (MOVE) copy_rows<1>(e, to_list, seq, kv, n_holes, wave, kWaves);
    for (int i0 = threadIdx.x; i0 < n_holes; i0 += 4 * kThreads) {
        int to[4], at[4];
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = min(i0 + j * kThreads, n_holes - 1);
            to[j] = to_list[i * 2];
            const int of = to_list[i * 2 + 1];
            x[j] = w[of];
            at[j] = pos[of];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i0 + j * kThreads < n_holes) {
                new_w[to[j]] = x[j];
                new_pos[to[j]] = at[j];
            }
    }
    if (threadIdx.x == 0) a.counts[blockIdx.x] = n_holes;
}

constexpr int kMoveThreads = 256;

// `per` blocks for each (sequence, KV head), 16 bytes of K or V per thread and round.
__global__ __launch_bounds__(kMoveThreads) void k_evict_move(EvictArgs a, uint32_t per) {
    const Evict &e = a.e;
    const uint32_t sh = blockIdx.x / per, x = blockIdx.x % per, seq = sh / e.kv_heads, kv = sh % e.kv_heads;
    if (kv == 0 && x == 0 && threadIdx.x == 0) e.new_lens[seq] = kept_of(e, slots_of(e, seq));
    const int32_t *moves = a.moves + (int64_t)sh * a.move_stride * 2;
    copy_rows<2>(e, moves, seq, kv, a.counts[sh], x * (kMoveThreads / 64) + (threadIdx.x >> 6), per * (kMoveThreads / 64));
}

template <bool MOVE>
void select(const EvictArgs &a, uint32_t rows, hipStream_t stream) {
    const dim3 grid(rows), block(kThreads);
    if (a.e.max_len <= 4096) k_evict_select<4096, MOVE><<<grid, block, 0, stream>>>(a);
    else if (a.e.max_len <= 16384) k_evict_select<16384, MOVE><<<grid, block, 0, stream>>>(a);
    else if (a.e.max_len <= 36864) k_evict_select<36864, MOVE><<<grid, block, 0, stream>>>(a);
    else k_evict_select<0, MOVE><<<grid, block, 0, stream>>>(a);
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
    const uint32_t kept = std::min(e.budget, e.max_len);
    const uint64_t bytes = (uint64_t)std::min(kept, e.max_len - kept) * e.row_bytes * 2;   // moved per head at most
    // few moves: in the first kernel (a token too many in each of 16 x 8 heads of 2,049 slots: 11.0 us; when this was
    // chosen 10.3, with a second launch 12.7), unless the new lengths replace those that its other blocks read
    if (std::min(kept, e.max_len - kept) <= kFewMoves && e.new_lens != e.lens) {
        select<true>(a, (uint32_t)rows, stream);
        return hipGetLastError();
    }
    // blocks per head for the copies: enough to fill the chip, 8 KiB of copies at least
    const uint32_t per = (uint32_t)std::min<uint64_t>(std::max<uint64_t>(bytes / 8192, 1), std::max<uint64_t>(2048 / rows, 1));
    if (rows * per > kMaxGrid) return hipErrorInvalidConfiguration;
    select<false>(a, (uint32_t)rows, stream);
    k_evict_move<<<dim3((uint32_t)(rows * per)), dim3(kMoveThreads), 0, stream>>>(a, per);
    return hipGetLastError();
}

}  // namespace attn
}  // namespace ibp
