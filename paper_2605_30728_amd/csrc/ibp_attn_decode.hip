// Attention of one new token per sequence over a paged KV cache.
//
// The cache's length is split over blocks, and within a block over its waves; each wave runs
// through its slots 32 at a time with a running reference and sum, a block joins its waves, and
// a second kernel joins the blocks of a sequence:
//   m = max_x m_x,  l = sum_x l_x 2^(m_x - m),  out = sum_x acc_x 2^(m_x - m) / l.
// Where the slots' accumulated weights are asked for, the scores are kept and the second kernel
// adds exp(s - lse) of every slot, in the order of the query heads.
//
// Bound by HBM: every slot's key and value are read once and used by the heads that share them (up to
// 16 as the columns of one matrix product). They go to registers a chunk ahead of their use, the values on to
// LDS, which turns them for the second product; the weights are rounded to the inputs' type for it (float16's
// lifted first, by kLift), their sum is of the unrounded ones. 131,071 slots of 8 heads of 128 in bf16: 101 us, 5.3 TB/s; 64 sequences of up to
// 8,192 slots with the slots' weights: 249 us, 4.5 TB/s of what the call has to move (the scores'
// way through the workspace comes on top). Short caches are bound by two launches: 1,531 slots in 13 us.
#include "ibp_attn_decode.hpp"
#include "ibp_attn_wave.hpp"

#include <algorithm>

namespace ibp {
namespace attn {

namespace {

using namespace dev;

constexpr int kWaves = 4;

// Slots that a wave takes at a time: what its registers hold of K and V while they are on their
// way, with two waves per SIMD.
template <int DIM>
constexpr int chunk_slots() { return DIM <= 128 ? 32 : 16; }

template <class T, int DIM, bool FULL>
__global__ __launch_bounds__(64 * kWaves, 2) void k_attn_decode(DecodeArgs a) {
    constexpr int kChunk = chunk_slots<DIM>(), KT = kChunk / 16;
    constexpr uint64_t kAll = (1ull << kChunk) - 1;
    constexpr int KS = DIM / 32, DT = DIM / 16, RB = Tile<DIM>::kRowBytes, CH = Tile<DIM>::kChunks;
    constexpr int kChunkBytes = kChunk * RB, VL = kChunkBytes / 1024, kRowsPer = 64 / CH;
    constexpr int kJoin = 16 * (DIM + 4) * 4;        // a wave's sums, for the join
    constexpr int kWaveBytes = kChunkBytes > kJoin ? kChunkBytes : kJoin;
    __shared__ __align__(128) uint8_t lds[kWaves * kWaveBytes];
    __shared__ float stat[kWaves][2][16];

    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), quarter = lane >> 4, col = lane & 15;
    const uint32_t hb = blockIdx.x % (a.kv_heads * a.head_blocks), rest = blockIdx.x / (a.kv_heads * a.head_blocks);
    // (splits outermost: those that no sequence reaches come last; and sequences turned by one from split
    // to split, so that each one's splits run on all XCDs)
    const uint32_t split = rest / a.n_seqs, seq = (rest % a.n_seqs + split) % a.n_seqs;
    const uint32_t kv = hb / a.head_blocks, head0 = kv * a.group + hb % a.head_blocks * 16;
    const int heads = min((int)((kv + 1) * a.group - head0), 16);
    const int len = uniform(slots_of(a, seq));
    const int from = split * a.split_tokens, to = from < len ? from + min(len - from, (int)a.split_tokens) : from;
    if (from >= to && !(split == 0)) return;

    Frag q[KS];
    {
        const uint8_t *qp = (const uint8_t *)a.q.data + ((int64_t)seq * a.q.row + (int64_t)(head0 + min(col, heads - 1)) * a.q.head) * 2;
#pragma unroll
        for (int x = 0; x < KS; ++x) q[x] = load_head<FULL>(qp, x * 32 + quarter * 8, a.dim);
    }

    // lane i < kChunk of a wave (and i + kChunk ...) knows the page of slot i of a chunk, and its place there
    const int32_t *table = a.pg.table + (int64_t)seq * a.pg.table_stride;
    int page = 0, place = 0;
    auto find = [&](int chunk) {
        const uint32_t s = min(chunk + (lane & (kChunk - 1)), len - 1);
        const uint32_t i = a.pg.page_magic ? __umulhi(s, a.pg.page_magic) >> a.pg.page_shift : s >> a.pg.page_shift;
        place = (int)(s - i * a.pg.page_tokens);
        page = table[i];
    };

    const float inf = __builtin_inff();
    const float c = a.scale_log2;
    float m = -inf, ref = 0.f, l = 0.f;     // reference, what scores are taken relative to (0 while there is none), sum
    f32x4 acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = f32x4{};
    uint8_t *vt = lds + wave * kWaveBytes;

    constexpr int kStep = kWaves * kChunk;
    Frag kf[KT][KS], vf[VL];
    uint64_t live = 0;                   // bit i: slot i of the chunk is there
    const uint8_t *kbase = (const uint8_t *)a.pg.k.data + (int64_t)kv * a.pg.k.head * 2;
    const uint8_t *vbase = (const uint8_t *)a.pg.v.data + (int64_t)kv * a.pg.v.head * 2;
    auto of_slot = [](int64_t x, int slot) {         // lane `slot`'s x
        return (int64_t)((uint64_t)(uint32_t)__shfl((int)(x >> 32), slot) << 32 | (uint32_t)__shfl((int)x, slot));
    };
    // the loads of a chunk whose pages are known, and the look-up of the next one's, so that
    // nothing waits for a look-up
    auto load = [&](int chunk) {
        const bool in = (uint32_t)page < a.pg.n_pages;
        live = __ballot(in && chunk + (lane & (kChunk - 1)) < len) & kAll;
        const int64_t pg = in ? page : 0;
        const int64_t ko = (pg * a.pg.k.page + (int64_t)place * a.pg.k.token) * 2, vo = (pg * a.pg.v.page + (int64_t)place * a.pg.v.token) * 2;
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            const uint8_t *kp = kbase + of_slot(ko, j * 16 + col);
#pragma unroll
            for (int x = 0; x < KS; ++x) kf[j][x] = load_head<FULL>(kp, x * 32 + quarter * 8, a.dim);
        }
#pragma unroll
        for (int i = 0; i < VL; ++i)
            vf[i] = load_head<FULL>(vbase + of_slot(vo, i * kRowsPer + lane / CH), lane % CH * 8, a.dim);
        find(chunk + kStep);
    };

    int chunk = from + wave * kChunk;
    if (chunk < to) {
        find(chunk);
        load(chunk);
    }
    for (; chunk < to; chunk += kStep) {
        f32x4 s[KT];
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            s[j] = f32x4{};
#pragma unroll
            for (int x = 0; x < KS; ++x) s[j] = T::mfma16(kf[j][x], q[x], s[j]);
        }
        const uint64_t now = live;
        if (now != kAll) {      // slots that are not there: no score, and no value that a weight of 0 could meet
#pragma unroll
            for (int j = 0; j < KT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!(now >> (j * 16 + quarter * 4 + i) & 1)) s[j][i] = -inf;
#pragma unroll
            for (int i = 0; i < VL; ++i) {
                const bool in = now >> (i * kRowsPer + lane / CH) & 1;
                vf[i] = Frag{in ? vf[i][0] : 0, in ? vf[i][1] : 0, in ? vf[i][2] : 0, in ? vf[i][3] : 0};
            }
        }
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int row = i * kRowsPer + lane / CH, ch = lane % CH;
            *reinterpret_cast<Frag *>(vt + row * RB + ((ch ^ Tile<DIM>::template columns<16>(row)) << 4)) = vf[i];
        }
        if (chunk + kStep < to) load(chunk + kStep);
        if (a.scores && col < heads) {
            float *sp = a.scores + ((int64_t)seq * a.q_heads + head0 + col) * a.scores_stride + chunk + quarter * 4;
#pragma unroll
            for (int j = 0; j < KT; ++j) *reinterpret_cast<f32x4 *>(sp + j * 16) = s[j];
        }
        float top = s[0][0];
#pragma unroll
        for (int j = 0; j < KT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, s[j][i]);
        top = max_halves(max_quarters(top));
        if (__any(top > m)) {
            const float next = fmaxf(m, top);
            const float keep = m == -inf ? 0.f : exp2_fast((m - next) * c);
            l *= keep;
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] *= keep;
            m = next;
            ref = m == -inf ? 0.f : m;
        }
        u32x2 p[KT];
#pragma unroll
        for (int j = 0; j < KT; ++j) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[j][i] = exp2_fast(__builtin_fmaf(s[j][i] - ref, c, (float)T::kLift));
                l += s[j][i];
            }
            p[j][0] = T::pack(s[j][0], s[j][1]);
            p[j][1] = T::pack(s[j][2], s[j][3]);
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const int key = quarter * 4 + (col >> 2), at = d * 16 + (col & 3) * 4;
            const u32x2 lo = read_columns<DIM, 16>(vt, key, at);
            if constexpr (KT == 1) {
                acc[d] = T::mfma16(lo, p[0], acc[d]);
            } else {
                const u32x2 hi = read_columns<DIM, 16>(vt, key + 16, at);
                acc[d] = T::mfma16(Frag{lo[0], lo[1], hi[0], hi[1]}, Frag{p[0][0], p[0][1], p[1][0], p[1][1]}, acc[d]);
            }
        }
    }

    // the block's waves joined: lane's column is a head, its registers dims quarter * 4 + i
    constexpr float unit = 1.f / (1 << T::kLift);
    l = sum_halves(sum_quarters(l)) * unit;
    if (quarter == 0) {
        stat[wave][0][col] = m;
        stat[wave][1][col] = l;
    }
    __syncthreads();
    float *mine = reinterpret_cast<float *>(vt);
#pragma unroll
    for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4 *>(mine + col * (DIM + 4) + d * 16 + quarter * 4) = acc[d] * unit;
    __syncthreads();
    const int h = threadIdx.x >> 4;          // 16 heads, 16 threads each
    if (h >= heads) return;
    float top = -inf, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, stat[w][0][h]);
    float part[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        part[w] = part_of(stat[w][0][h], stat[w][1][h], top, c);
        if (!(part[w] < 0.f)) sum += part[w] * stat[w][1][h];
    }
    const uint32_t head = head0 + h;
    const bool last = a.splits == 1;
    const float inv = !last ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
    for (int d = (threadIdx.x & 15) * 4; d < (int)a.dim; d += 64) {
        f32x4 x{};
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            if (!(part[w] < 0.f)) x += part[w] * *reinterpret_cast<const f32x4 *>(reinterpret_cast<float *>(lds + w * kWaveBytes) + h * (DIM + 4) + d);
        x *= inv;
        if (last) {
            u32x2 o;
            o[0] = T::pack_out(x[0], x[1]);
            o[1] = T::pack_out(x[2], x[3]);
            *reinterpret_cast<u32x2 *>((uint8_t *)a.out.data + ((int64_t)seq * a.out.row + (int64_t)head * a.out.head + d) * 2) = o;
        } else {
            *reinterpret_cast<f32x4 *>(a.partial + (((int64_t)seq * a.q_heads + head) * a.splits + split) * a.dim + d) = x;
        }
    }
    if ((threadIdx.x & 15) == 0) {
        if (last && a.lse) a.lse[(int64_t)seq * a.q_heads + head] = sum == 0.f ? -inf : top * a.scale + __logf(sum);
        if (!last || a.weights) {
            float *st = a.stats + (((int64_t)seq * a.q_heads + head) * a.splits + split) * 2;
            st[0] = top;
            st[1] = sum;
        }
    }
}

constexpr int kJoinThreads = 256;
constexpr int kJoinSlots = 4 * kJoinThreads; // slots whose weights a block of the second kernel adds

// Dims that a block of the second kernel joins: the whole head where it has few splits (64
// sequences of 8 heads, 11 splits: 18 us, in blocks of 64 dims 31), 64 where the way through them is long
// (512 splits of 256 dims: 16 rounds of its threads instead of 128).
inline uint32_t join_dims(uint32_t dim, uint32_t splits) { return splits > 64 ? std::min(dim, 64u) : dim; }

// x over the block's threads, by `op` with neutral element `none`.
template <class Op>
__device__ __forceinline__ float block_reduce(float x, float none, float *waves, Op op) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x = op(x, __shfl_xor(x, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
    __syncthreads();
    x = none;
#pragma unroll
    for (int w = 0; w < kJoinThreads / 64; ++w) x = op(x, waves[w]);
    return x;
}

// Of the blocks of a (sequence, KV head), one for each query head and join_dims dims joins that
// head's splits (where there are several); the others add the weights of kJoinSlots slots.
template <class T>
__global__ __launch_bounds__(kJoinThreads) void k_attn_decode_join(DecodeArgs a, uint32_t weight_blocks, uint32_t dims) {
    __shared__ float part[kMaxSplits];
    __shared__ f32x4 sums[kJoinThreads];
    __shared__ float waves[kJoinThreads / 64];
    const uint32_t dim_blocks = (a.dim + dims - 1) / dims, per = weight_blocks + (a.splits > 1 ? a.group * dim_blocks : 0);
    const uint32_t x = blockIdx.x % per, kv = blockIdx.x / per % a.kv_heads, seq = blockIdx.x / per / a.kv_heads;
    const int len = slots_of(a, seq);
    const int n = len > 0 ? (int)((len + a.split_tokens - 1) / a.split_tokens) : 1;
    const float inf = __builtin_inff(), c = a.scale_log2;
    if (x >= weight_blocks) {
        const uint32_t head = kv * a.group + (x - weight_blocks) / dim_blocks, d0 = (x - weight_blocks) % dim_blocks * dims;
        const int64_t at = ((int64_t)seq * a.q_heads + head) * a.splits;
        const f32x2 *st = reinterpret_cast<const f32x2 *>(a.stats) + at;
        float top = -inf, sum = 0.f;
        for (int y = threadIdx.x; y < n; y += kJoinThreads) top = fmaxf(top, st[y][0]);
        top = block_reduce(top, -inf, waves, [](float u, float v) { return fmaxf(u, v); });
        for (int y = threadIdx.x; y < n; y += kJoinThreads) {
            const f32x2 s = st[y];
            part[y] = part_of(s[0], s[1], top, c);
            if (!(part[y] < 0.f)) sum += part[y] * s[1];
        }
        sum = block_reduce(sum, 0.f, waves, [](float u, float v) { return u + v; });
        // four dims per thread, the splits shared out over the groups of threads that hold all dims
        const int quads = dims / 4, groups = kJoinThreads / quads;
        const int q = threadIdx.x % quads, y0 = threadIdx.x / quads, d = d0 + q * 4;
        const float *pp = a.partial + at * a.dim + d;
        f32x4 o{};
        if (d < (int)a.dim && y0 < groups) {
#pragma unroll 4
            for (int y = y0; y < n; y += groups) {
                const f32x4 v = *reinterpret_cast<const f32x4 *>(pp + (int64_t)y * a.dim);
                if (!(part[y] < 0.f)) o += part[y] * v;
            }
        }
        sums[threadIdx.x] = o;
        __syncthreads();
        if (y0 != 0 || d >= (int)a.dim) return;
        for (int y = 1; y < groups; ++y) o += sums[y * quads + q];
        o *= sum == 0.f ? 0.f : 1.f / sum;
        u32x2 w;
        w[0] = T::pack_out(o[0], o[1]);
        w[1] = T::pack_out(o[2], o[3]);
        *reinterpret_cast<u32x2 *>((uint8_t *)a.out.data + ((int64_t)seq * a.out.row + (int64_t)head * a.out.head + d) * 2) = w;
        if (a.lse && d == 0) a.lse[(int64_t)seq * a.q_heads + head] = sum == 0.f ? -inf : top * a.scale + __logf(sum);
        return;
    }
    if ((int)(x * kJoinSlots) >= len) return;
    const int lane = threadIdx.x & 63, slot = x * kJoinSlots + threadIdx.x * 4;
    float w[4] = {};
    for (uint32_t g0 = 0; g0 < a.group; g0 += 64) {          // (64 heads' references and sums at a time)
        const int heads = min((int)(a.group - g0), 64);
        __syncthreads();
        for (int h = threadIdx.x >> 6; h < heads; h += kJoinThreads / 64) {
            const f32x2 *st = reinterpret_cast<const f32x2 *>(a.stats) + ((int64_t)seq * a.q_heads + kv * a.group + g0 + h) * a.splits;
            float top = -inf, sum = 0.f;
            for (int y = lane; y < n; y += 64) top = fmaxf(top, st[y][0]);
#pragma unroll
            for (int y = 1; y < 64; y <<= 1) top = fmaxf(top, __shfl_xor(top, y));
            for (int y = lane; y < n; y += 64) {
                const f32x2 s = st[y];
                const float f = part_of(s[0], s[1], top, c);
                if (!(f < 0.f)) sum += f * s[1];
            }
#pragma unroll
            for (int y = 1; y < 64; y <<= 1) sum += __shfl_xor(sum, y);
            if (lane == 0) {
                part[h * 2] = top == -inf ? 0.f : top;
                part[h * 2 + 1] = sum == 0.f ? 0.f : 1.f / sum;
            }
        }
        __syncthreads();
        if (slot >= len) continue;
        const float *sp = a.scores + ((int64_t)seq * a.q_heads + kv * a.group + g0) * a.scores_stride + slot;
#pragma unroll 4
        for (int h = 0; h < heads; ++h) {
            const f32x4 s = *reinterpret_cast<const f32x4 *>(sp + (int64_t)h * a.scores_stride);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] += exp2_fast((s[i] - part[h * 2]) * c) * part[h * 2 + 1];
        }
    }
    float *out = a.weights + ((int64_t)seq * a.kv_heads + kv) * a.weights_stride + slot;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (slot + i < len) out[i] += w[i];
}

template <class T>
void decode_of(const DecodeArgs &a, uint32_t blocks, hipStream_t stream) {
    const dim3 grid(blocks), block(64 * kWaves);
    if (a.dim == 64) k_attn_decode<T, 64, true><<<grid, block, 0, stream>>>(a);
    else if (a.dim < 64) k_attn_decode<T, 64, false><<<grid, block, 0, stream>>>(a);
    else if (a.dim < 128) k_attn_decode<T, 128, false><<<grid, block, 0, stream>>>(a);
    else if (a.dim == 128) k_attn_decode<T, 128, true><<<grid, block, 0, stream>>>(a);
    else if (a.dim < 256) k_attn_decode<T, 256, false><<<grid, block, 0, stream>>>(a);
    else k_attn_decode<T, 256, true><<<grid, block, 0, stream>>>(a);
}

uint64_t up256(uint64_t x) { return (x + 255) / 256 * 256; }

}  // namespace

DecodePlan plan_decode(uint32_t n_seqs, uint32_t q_heads, uint32_t kv_heads, uint32_t dim, uint32_t max_len,
                       bool weights) {
    DecodePlan p{};
    p.head_blocks = (q_heads / kv_heads + 15) / 16;
    // a single sequence: the 512 blocks that the chip holds at once (131,071 slots of 8 heads of
    // 128: 99 us, with 1,024 blocks 103, with 2,048 109). Several, whose lengths differ: up to 1,024
    // blocks (24 sequences of up to 6,000 slots of one head of 256: 27 us, with 512 31), and more of
    // 768 slots (64 sequences of up to 8,192 slots: blocks of 4,096 slots 294 us, of 768 to 1,024 259,
    // of 256 267). At least 128 slots, a chunk or two per wave.
    const uint64_t rows = std::max<uint64_t>((uint64_t)n_seqs * kv_heads * p.head_blocks, 1), len = std::max<uint64_t>(max_len, 1);
    uint64_t t = n_seqs > 1 ? std::min<uint64_t>((len * rows + 1023) / 1024, 768) : (len * rows + 511) / 512;
    t = std::max<uint64_t>(t, (len + kMaxSplits - 1) / kMaxSplits);
    t = std::max<uint64_t>((std::min(t, len) + 127) / 128 * 128, 128);   // (below 2^31, however many heads there are)
    p.split_tokens = (uint32_t)t;
    p.splits = (uint32_t)((len + t - 1) / t);
    const uint64_t parts = (uint64_t)n_seqs * q_heads * p.splits;
    p.stats_off = 0;
    p.out_off = up256(parts * 8);
    p.scores_off = p.out_off + (p.splits > 1 ? up256(parts * dim * 4) : 0);
    p.bytes = p.scores_off + (weights ? up256((uint64_t)n_seqs * q_heads * ((max_len + 31ull) / 32 * 32) * 4) : 0);
    return p;
}

// What plan_decode needs at most for up to n_seqs sequences of up to max_len slots. Fewer slots can need more: a
// split's length goes in steps of 128, so 8,192 slots of a sequence of 8 KV heads make 64 splits and 8,193
// slots 33. By plan_decode's rule a sequence has a split for every 128 slots at most, and no more than both 768
// slots each and 1,024 blocks among all sequences (each rounded up) come to; this grows with both sizes.
uint64_t decode_workspace(uint32_t n_seqs, uint32_t q_heads, uint32_t kv_heads, uint32_t dim, uint32_t max_len, bool weights) {
    const uint64_t n = n_seqs, len = std::max<uint64_t>(max_len, 1), blocks = (uint64_t)kv_heads * ((q_heads / kv_heads + 15) / 16);
    const uint64_t splits = std::min(n * std::min<uint64_t>((len + 127) / 128, kMaxSplits),
                                     std::max((1024 + blocks - 1) / blocks + n, n * ((len + 767) / 768)));
    return up256(splits * q_heads * 8) + (len > 128 ? up256(splits * q_heads * dim * 4) : 0) +
           (weights ? up256(n * q_heads * ((max_len + 31ull) / 32 * 32) * 4) : 0);
}

namespace {
uint32_t join_weight_blocks(const DecodeArgs &a) { return a.weights ? (a.max_len + kJoinSlots - 1) / kJoinSlots : 0; }
}  // namespace

uint64_t decode_join_blocks(const DecodeArgs &a) {
    const uint32_t dims = join_dims(a.dim, a.splits), dim_blocks = (a.dim + dims - 1) / dims;
    return (uint64_t)a.n_seqs * a.kv_heads * (join_weight_blocks(a) + (a.splits > 1 ? a.group * dim_blocks : 0));
}

void launch_decode_join(const DecodeArgs &a, bool f16, hipStream_t stream) {
    const uint32_t join = (uint32_t)decode_join_blocks(a), dims = join_dims(a.dim, a.splits);
    if (join == 0) return;
    if (f16) k_attn_decode_join<F16><<<dim3(join), dim3(kJoinThreads), 0, stream>>>(a, join_weight_blocks(a), dims);
    else k_attn_decode_join<Bf16><<<dim3(join), dim3(kJoinThreads), 0, stream>>>(a, join_weight_blocks(a), dims);
}

hipError_t launch_decode(const Shape &s, const Rows &q, const Pages &pg, const int32_t *lens, uint32_t n_seqs,
                         uint32_t max_len, const Rows &out, float *lse, float *weights, uint64_t weights_stride,
                         const DecodePlan &plan, uint8_t *workspace, hipStream_t stream) {
    if (n_seqs == 0) return hipSuccess;
    const uint64_t blocks = (uint64_t)n_seqs * plan.splits * s.kv_heads * plan.head_blocks;
    DecodeArgs a{q, out, pg, lens, lse, weights, weights_stride, (float *)(workspace + plan.stats_off),
                 (float *)(workspace + plan.out_off), weights ? (float *)(workspace + plan.scores_off) : nullptr,
                 (max_len + 31) / 32 * 32, n_seqs, s.q_heads, s.kv_heads, s.group, plan.head_blocks, s.dim, max_len,
                 plan.split_tokens, plan.splits, s.scale, s.scale_log2};
    if (blocks > kMaxGrid || decode_join_blocks(a) > kMaxGrid) return hipErrorInvalidConfiguration;
    if (s.f16) decode_of<F16>(a, (uint32_t)blocks, stream);
    else decode_of<Bf16>(a, (uint32_t)blocks, stream);
    launch_decode_join(a, s.f16, stream);
    return hipGetLastError();
}

void page_division(uint32_t page_tokens, uint32_t &magic, uint32_t &shift) {
    // d = page_tokens > 1 not a power of two, k = ceil(log2 d): with magic = ceil(2^(31 + k) / d)
    // (below 2^32, since 2^k < 2 d), n magic / 2^(31 + k) exceeds n / d by less than
    // n / 2^(31 + k) <= 1 / 2^k <= 1 / d for n < 2^31, so its floor is n / d's
    uint32_t k = 0;
    while ((1ull << k) < page_tokens) ++k;
    if ((1ull << k) == page_tokens) {
        magic = 0;
        shift = k;
        return;
    }
    magic = (uint32_t)(((1ull << (31 + k)) + page_tokens - 1) / page_tokens);
    shift = k - 1;
}

}  // namespace attn
}  // namespace ibp
