// The attention weight that every key received from the rows of its sequence:
//   w[j] = sum over the query heads of its KV head and the rows i that see it of exp(s_ij - lse_i),
// s_ij as in attention over prompts and lse_i what that left behind. A block holds 64 keys per
// wave as matrix fragments and streams the rows of one query head past them; the query heads of
// a KV head are added up by a second kernel, so that the result never depends on an order.
//
// Of the pairs of a causal prompt each costs DIM multiply-adds, a subtraction, an exponential and an addition, and
// nothing of that size is written. 64 keys a wave, since every row fragment read from LDS then feeds two matrix
// instructions (with 32 keys LDS is as busy as they are); rows reach LDS by direct loads, issued a tile before the one
// that reads them. 8,192 rows of 32 heads of 128 in bf16: 351 to 357 us with the sum over heads, 0.77 to 0.78 PFLOP/s
// of the pairs that count, with the matrix unit busy for 0.40 of the time (11 packed prompts in f16: 82 us, 0.26). What
// holds both units up shows in the compiled code: the compiler waits for a tile's loads right behind their issue, before
// the first fragment of the tile at hand is read, which costs every 64 rows a load's latency; and where some pairs of
// a tile do not count (four tiles or more of every block in a causal prompt) each score reads its row's lse from LDS
// in a branch of its own (settle).
#include "ibp_attn.hpp"
#include "ibp_attn_wave.hpp"

#include <algorithm>

namespace ibp {
namespace attn {

namespace {

using namespace dev;

struct WeightArgs {
    Rows q, k;
    Packed p;
    const float *lse;
    float *out;                  // [splits][q_heads][k_rows]
    uint32_t q_heads, kv_heads, group, dim;
    uint32_t tiles, splits;      // per head: at least the tiles of all sequences; blocks that share a tile's rows
    float scale_log2;
    uint32_t causal;
};

constexpr int kWaves = 4;
constexpr int kBlockKeys = 64 * kWaves;
constexpr float kLog2e = 1.4426950408889634f;

// Scores of 32 rows (fragments from LDS) and the wave's 64 keys (k): next; beside them, in turns, the
// weights exp(s - lse) of the 32 rows before them, added up per register (sum). The
// two are about as much work for the matrix as for the vector unit, and they only run beside each other in
// turns (8,192 rows of 32 heads of 128: all products first 371 us, in turns 364).
// lse: of the rows of s, times log2(e) and never NaN; rows that count for nothing have an infinite one.
template <class T, int DIM>
__device__ __forceinline__ void step(const uint8_t *__restrict qt, int row_in_tile, const Frag (*k)[DIM / 16], f32x16 *s,
                                     f32x16 *next, const float *lse, f32x16 *sum, float c) {
    constexpr int KS = DIM / 16, kAhead = 2;
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    f32x4 ls[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) ls[i] = *reinterpret_cast<const f32x4 *>(lse + i * 8 + half * 4);
    Frag ahead[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) ahead[x] = read_rows<DIM>(qt, row_in_tile + col, x * 2 + half);
#pragma unroll
    for (int x = 0; x < KS; ++x) {
        const Frag now = ahead[x % kAhead];
        if (x + kAhead < KS) ahead[x % kAhead] = read_rows<DIM>(qt, row_in_tile + col, (x + kAhead) * 2 + half);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            __builtin_amdgcn_sched_barrier(0);
            next[j] = T::mfma32(now, k[j][x], x == 0 ? f32x16{} : next[j]);
#pragma unroll
            for (int n = (x * 2 + j) * 16 / KS; n < (x * 2 + j + 1) * 16 / KS; ++n) {
                const int i = n % 16, y = n / 16;
                sum[y][i] += exp2_fast(__builtin_fmaf(s[y][i], c, -ls[i >> 2][i & 3]));
                asm volatile("" : "+v"(sum[y][i]));                   // (here, not where it is used)
            }
        }
    }
    __builtin_amdgcn_sched_barrier(0);
}

// The scores s of 32 rows before their step, where some pair of them does not count (from row `end` on, or
// before row `seen` of a column; rows relative to the first): -inf, whatever score and lse are; where
// a row's lse (raw) is NaN, so are the scores that count.
__device__ __forceinline__ void settle(f32x16 *s, const float *raw, const int *seen, int end) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int from = seen[j] - half * 4, to = end - half * 4;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int at = (i >> 2) * 8 + (i & 3);
            const float x = raw[at + half * 4];
            s[j][i] = at < from || at >= to ? -__builtin_inff() : x != x ? x : s[j][i];
        }
    }
}

// The scores of rows without an lse (raw: -inf) likewise: they may be NaN, which no lse takes away.
__device__ __forceinline__ void leave_out(f32x16 *s, const float *raw) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const bool none = raw[(i >> 2) * 8 + (i & 3) + half * 4] == -__builtin_inff();
#pragma unroll
        for (int j = 0; j < 2; ++j) s[j][i] = none ? -__builtin_inff() : s[j][i];
    }
}

template <class T, int DIM>
__global__ __launch_bounds__(64 * kWaves, DIM <= 128 ? 2 : 1) void k_attn_key_weights(WeightArgs a) {
    constexpr int N = 64, RB = Tile<DIM>::kRowBytes, KS = DIM / 16;
    constexpr int kTileBytes = N * RB, kLoads = kTileBytes / 1024 / kWaves;
    __shared__ __align__(128) uint8_t lds[3 * kTileBytes];   // rows of three tiles
    __shared__ __align__(16) float lse_tile[3][N], lse_raw[3][N];

    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    // One long sequence: one head after the other on an XCD, where they can be dealt out evenly; the blocks that
    // run there at a time read the same rows, which its cache holds (8,192 rows of 32 heads of 128: 348 us, in the
    // other order 364). Several: all heads of a tile, then the next tile, which leaves the long ones no
    // tail (11 sequences, the longest of 2,501 rows: 82 us, head after head 92).
    uint32_t head, t, split;
    const uint32_t b = blockIdx.x;
    if (a.p.n_seqs == 1 && a.q_heads % 8 == 0) {
        const uint32_t i = b >> 3, per = a.tiles * a.splits;
        head = (b & 7) + 8 * (i / per);
        t = i % per / a.splits;
        split = i % per % a.splits;
    } else {
        head = b / a.splits % a.q_heads;
        split = b % a.splits;
        t = b / a.splits / a.q_heads;
    }
    SeqTile st;
    if (!find_tile<true>(a.p.q_starts, a.p.k_starts, a.p.n_seqs, a.p.q_rows, a.p.k_rows, kBlockKeys, t, st)) return;
    const int q_len = st.q_len, k_len = st.k_len, past = k_len - q_len;
    const uint32_t kv = head / a.group;
    const int tile = st.tiles - 1 - st.rank, key0 = tile * kBlockKeys + wave * 64;   // (the first keys are seen by the most rows)

    // the tiles of rows that see a key of this block, and this block's share of them
    const int first = (a.causal ? max(tile * kBlockKeys - past, 0) : 0) / N, rows_end = (q_len + N - 1) / N;
    const int per_split = (max(rows_end - first, 0) + (int)a.splits - 1) / (int)a.splits;
    const int n0 = first + (int)split * per_split, n1 = min(n0 + per_split, rows_end);
    const int wave_all = a.causal ? max(min(key0 + 63, k_len - 1) - past, 0) : 0;    // the first row that sees all of the wave's keys
    const int seen[2] = {a.causal ? key0 + col - past : 0, a.causal ? key0 + 32 + col - past : 0};

    const uint32_t q_stride = (uint32_t)a.q.row * 2;
    const uint8_t *qp = (const uint8_t *)a.q.data + ((int64_t)st.q0 * a.q.row + (int64_t)head * a.q.head) * 2;
    const float *lse = a.lse + (int64_t)head * a.p.q_rows + st.q0;
    uint32_t q_off[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) q_off[i] = tile_source<DIM, true>((i * kWaves + wave) * 64 + lane, q_stride, a.dim);
    auto load_tile = [&](int n, int buf) {                   // (empty past the last tile: zeros)
        const int rows = n < n1 ? min(q_len - n * N, N) : 0;
        const Rsrc r = descriptor(rows ? qp + (int64_t)n * N * q_stride : qp, rows ? (rows - 1) * q_stride + a.dim * 2 : 0);
        uint8_t *at = lds + buf * kTileBytes + wave * 1024;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load_to_lds(r, at + i * kWaves * 1024, q_off[i]);
    };
    const float inf = __builtin_inff();
    auto load_lse = [&](int n) {                             // (no row past the end weighs anything)
        const int row = n * N + (int)threadIdx.x;
        return threadIdx.x < N && row < q_len ? lse[row] : inf;
    };
    auto put_lse = [&](int buf, float x) {
        if (threadIdx.x >= N) return;
        lse_raw[buf][threadIdx.x] = x;
        lse_tile[buf][threadIdx.x] = x == -inf || x != x ? inf : x * kLog2e;
    };

    f32x16 sum[2] = {f32x16{}, f32x16{}};
    if (n0 < n1) {
        float l0 = load_lse(n0), l1 = load_lse(n0 + 1);
        load_tile(n0, 0);
        load_tile(n0 + 1, 1);
        Frag k[2][KS];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int key = min(key0 + j * 32 + col, k_len - 1);
            const uint8_t *kp = (const uint8_t *)a.k.data + ((int64_t)(st.k0 + key) * a.k.row + (int64_t)kv * a.k.head) * 2;
#pragma unroll
            for (int x = 0; x < KS; ++x) k[j][x] = load_head<false>(kp, x * 16 + half * 8, a.dim);
        }
        put_lse(0, l0);
        put_lse(1, l1);
        tiles_loaded();
        f32x16 s0[2], s1[2];                                 // of rows 0 to 31 and 32 to 63 of a tile
#pragma unroll
        for (int j = 0; j < 2; ++j) s0[j] = f32x16{};
#pragma unroll
        for (int x = 0; x < KS; ++x)
#pragma unroll
            for (int j = 0; j < 2; ++j) s0[j] = T::mfma32(read_rows<DIM>(lds, col, x * 2 + half), k[j][x], s0[j]);
        int here = 0, then = 1, free = 2;                    // places of this tile, the next one and the one after
        for (int n = n0; n < n1; ++n) {
            const float raw = lse_raw[here][lane];
            const float next_lse = load_lse(n + 2);
            load_tile(n + 2, free);
            const int row0 = n * N;
            const uint8_t *qt = lds + here * kTileBytes, *qn = lds + then * kTileBytes;
            const bool special = row0 < wave_all || row0 + N > q_len || __any(raw != raw), none = __any(raw == -inf);
            if (special) {
                const int from[2] = {seen[0] - row0, seen[1] - row0};
                settle(s0, lse_raw[here], from, q_len - row0);
            }
            if (none) leave_out(s0, lse_raw[here]);
            step<T, DIM>(qt, 32, k, s0, s1, lse_tile[here], sum, a.scale_log2);
            if (special) {
                const int from[2] = {seen[0] - row0 - 32, seen[1] - row0 - 32};
                settle(s1, lse_raw[here] + 32, from, q_len - row0 - 32);
            }
            if (none) leave_out(s1, lse_raw[here] + 32);
            step<T, DIM>(qn, 0, k, s1, s0, lse_tile[here] + 32, sum, a.scale_log2);
            put_lse(free, next_lse);
            tiles_loaded();                                  // (the next tile's second step reads tile n + 2, every wave's share)
            const int old = here;
            here = then;
            then = free;
            free = old;
        }
    }

    float *out = a.out + ((int64_t)split * a.q_heads + head) * a.p.k_rows + st.k0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        float w = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) w += sum[j][i];
        w = sum_halves(w);
        const int key = key0 + j * 32 + col;
        if (half == 0 && key < k_len) out[key] = w;
    }
}

// The sums of all splits and query heads of a KV head, in their order.
__global__ __launch_bounds__(256) void k_sum_heads(const float *partial, float *weights, uint32_t q_heads, uint32_t kv_heads,
                                                   uint32_t splits, uint32_t k_rows, const int32_t *k_starts, uint32_t n_seqs) {
    const uint32_t per = (k_rows + 255) / 256, kv = blockIdx.x / per, j = blockIdx.x % per * 256 + threadIdx.x;
    const int from = clamp_row(k_starts[0], k_rows), to = clamp_row(k_starts[n_seqs], k_rows);
    if ((int64_t)j < from || (int64_t)j >= to) return;       // rows of no sequence
    const uint32_t group = q_heads / kv_heads;
    float w = 0.f;
    for (uint32_t x = 0; x < splits; ++x) {
        const float *p = partial + ((int64_t)x * q_heads + kv * group) * k_rows + j;
#pragma unroll 4
        for (uint32_t g = 0; g < group; ++g) w += p[(int64_t)g * k_rows];
    }
    weights[(int64_t)kv * k_rows + j] = w;
}

// Blocks that share a tile's rows: up to four, which evens out what keys at a sequence's start and end are
// seen by; one where many sequences are on their way (an empty share still costs its block's start).
uint32_t splits_of(uint32_t n_seqs) { return std::min(std::max(32 / std::max(n_seqs, 1u), 1u), 4u); }

template <class T>
hipError_t weights_of(const WeightArgs &a, uint32_t blocks, hipStream_t stream) {
    const dim3 grid(blocks), block(64 * kWaves);
    if (a.dim <= 64) k_attn_key_weights<T, 64><<<grid, block, 0, stream>>>(a);
    else if (a.dim <= 96) k_attn_key_weights<T, 96><<<grid, block, 0, stream>>>(a);
    else if (a.dim <= 128) k_attn_key_weights<T, 128><<<grid, block, 0, stream>>>(a);
    else k_attn_key_weights<T, 256><<<grid, block, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_key_weights(const Shape &s, const Rows &q, const Rows &k, const Packed &p, const float *lse,
                              float *weights, float *partial, hipStream_t stream) {
    if (p.n_seqs == 0 || p.k_rows == 0) return hipSuccess;
    const uint32_t splits = splits_of(p.n_seqs);
    const uint64_t tiles = p.k_rows / kBlockKeys + (uint64_t)p.n_seqs;
    const uint64_t blocks = tiles * s.q_heads * splits, sum_blocks = (uint64_t)(p.k_rows + 255) / 256 * s.kv_heads;
    if (blocks > kMaxGrid || sum_blocks > kMaxGrid) return hipErrorInvalidConfiguration;
    const bool one = s.group == 1 && splits == 1;
    WeightArgs a{q, k, p, lse, one ? weights : partial, s.q_heads, s.kv_heads, s.group, s.dim, (uint32_t)tiles, splits,
                 s.scale_log2, s.causal ? 1u : 0u};
    hipError_t e = s.f16 ? weights_of<F16>(a, (uint32_t)blocks, stream) : weights_of<Bf16>(a, (uint32_t)blocks, stream);
    if (e != hipSuccess || one) return e;
    k_sum_heads<<<dim3((uint32_t)sum_blocks), dim3(256), 0, stream>>>(partial, weights, s.q_heads, s.kv_heads, splits, p.k_rows,
                                                                      p.k_starts, p.n_seqs);
    return hipGetLastError();
}

uint64_t key_weights_workspace(uint32_t q_heads, uint32_t kv_heads, uint64_t k_rows, uint32_t n_seqs) {
    const uint32_t splits = splits_of(n_seqs);
    return q_heads == kv_heads && splits == 1 ? 0 : (uint64_t)splits * q_heads * k_rows * sizeof(float);
}

}  // namespace attn
}  // namespace ibp
