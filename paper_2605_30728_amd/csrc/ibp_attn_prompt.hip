// Attention over whole prompts.
//
// Row i of a sequence with keys k_j and values v_j: with s_ij = scale * q_i . k_j over the keys
// that i sees,  out_i = sum_j exp(s_ij) v_j / sum_j exp(s_ij)  and  lse_i = ln sum_j exp(s_ij),
// in one pass over the keys with a running reference m and a running sum: what has been added up
// so far is scaled by exp(m_old - m_new) when the reference moves.
//
// Every pair of a row and a key costs 4 DIM operations of the matrix unit and, beside it, an exponential. Keys and values are read from HBM about once (the heads
// that share them run on one XCD). A wave holds 32 rows' queries, weights and sums in registers, four waves share
// the tiles of 64 keys (32 of wide heads) that LDS holds, two of K and two of V. The weights are rounded to the
// inputs' type for the product with the values, as the matrix unit takes them (float16's lifted first, by kLift);
// their sum is of the unrounded ones. 8,192 rows of 32 heads of 128 in bf16, causal: 512 to 553 us, 0.99 to 1.07 PFLOP/s of
// the pairs that count, with the matrix unit busy for 0.59 of the time and LDS for 0.30 (of 16 heads of 64, with
// half the products per exponential, 0.35 and 0.18).
#include "ibp_attn.hpp"
#include "ibp_attn_wave.hpp"

#include <algorithm>
#include <type_traits>

namespace ibp {
namespace attn {

namespace {

using namespace dev;

struct PromptArgs {
    Rows q, k, v, out;
    Packed p;
    float *lse;
    uint32_t q_heads, kv_heads, group, dim;
    uint32_t tiles;              // per head: at least the tiles of all sequences
    uint32_t splits;             // blocks that share a tile's keys
    f32x2 *stats;                // splits > 1: [split][q_heads][q rows] reference (in scores) and sum
    float *partial;              //   [split][q_heads][q rows][dim]
    float scale, scale_log2;
    float lazy, huge;            // lazy<T>() and huge<T>() as scores: over scale_log2
    uint32_t causal;
};

constexpr int kWaves = 4;        // of a block, 32 rows each
constexpr int kBlockRows = 32 * kWaves;
// All exponents of a row are taken relative to one rounded product, reference times c. What that is off by, up to 2^-24
// of it (twice that where weights are lifted), is common to the row's weights and cancels, as long as these are
// numbers of the type: a row whose reference gets larger than this is done key by key.
template <class T>
constexpr float huge() { return T::kLift ? 0x1p23f : 0x1p26f; }
// How far (in powers of two) weights may exceed those of the reference: 2^8; in float16, with what they are lifted by, 2^15.
template <class T>
constexpr float lazy() { return T::kLift ? 15.f - T::kLift : 8.f; }

template <int DIM>
constexpr int key_tile() { return DIM <= 128 ? 64 : 32; }

// What a block leaves of a row: the row's output and lse, or its part of them.
__device__ __forceinline__ int64_t part_at(const PromptArgs &a, int split, int head, int row) {
    return ((int64_t)split * a.q_heads + head) * a.p.q_rows + row;
}

// One row, key by key in 32 bits, by one wave: lanes are keys for the scores and columns for the
// sum. Only for rows whose tiles hold infinities or NaN in places that the row does not see, and rows of huge scores.
template <class T, int DIM>
__device__ void attend_row(const PromptArgs &a, int row, int head, int split, const uint8_t *kp, const uint8_t *vp,
                           int from, int keys) {
    const int lane = threadIdx.x & 63;
    const uint16_t *q = (const uint16_t *)a.q.data + (int64_t)row * a.q.row + (int64_t)head * a.q.head;
    const float inf = __builtin_inff();
    float m = -inf, l = 0.f, acc[(DIM + 63) / 64] = {};
    for (int k0 = from; k0 < keys; k0 += 64) {
        float s = -inf;
        if (k0 + lane < keys) {
            const uint16_t *k = (const uint16_t *)kp + (int64_t)(k0 + lane) * a.k.row;
            s = 0.f;
            for (int d = 0; d < (int)a.dim; ++d) s = __builtin_fmaf(T::value(q[d]), T::value(k[d]), s);
        }
        float top = s;
        for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
        const float next = fmaxf(m, top), keep = m == -inf ? 0.f : exp2_fast((m - next) * a.scale_log2);
        const float p = exp2_fast((s - (next == -inf ? 0.f : next)) * a.scale_log2);
        l *= keep;
        for (float &x : acc) x *= keep;
        float sum = p;
        for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x);
        l += sum;
        m = next;
        for (int j = 0; j < min(keys - k0, 64); ++j) {
            const uint16_t *v = (const uint16_t *)vp + (int64_t)(k0 + j) * a.v.row;
            const float w = __shfl(p, j);
#pragma unroll
            for (int x = 0; x < (DIM + 63) / 64; ++x)
                if (lane + 64 * x < (int)a.dim) acc[x] = __builtin_fmaf(w, T::value(v[lane + 64 * x]), acc[x]);
        }
    }
    if (a.splits > 1) {
        const int64_t at = part_at(a, split, head, row);
        if (lane == 0) a.stats[at] = f32x2{m, l};
#pragma unroll
        for (int x = 0; x < (DIM + 63) / 64; ++x)
            if (lane + 64 * x < (int)a.dim) a.partial[at * a.dim + lane + 64 * x] = acc[x];
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t *out = (uint16_t *)a.out.data + (int64_t)row * a.out.row + (int64_t)head * a.out.head;
#pragma unroll
    for (int x = 0; x < (DIM + 63) / 64; ++x)
        if (lane + 64 * x < (int)a.dim) out[lane + 64 * x] = (uint16_t)T::pack_out(l == 0.f ? 0.f : acc[x] * inv, 0.f);
    if (a.lse && lane == 0) a.lse[(int64_t)head * a.p.q_rows + row] = l == 0.f ? -inf : m * a.scale + __logf(l);
}

// A wave's share of a tile of K or V on its way into LDS.
template <int LOADS>
__device__ __forceinline__ void load_tile(uint8_t *__restrict to, Rsrc r, const uint32_t *off) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load_to_lds(r, to + i * kWaves * 1024, off[i]);
}

// What the exponents of a row with reference m are relative to. (Not fused: the lift would take a register all the time,
// and of those the kernel of 128 wide heads has none left.)
template <class T>
__device__ __forceinline__ float base_of(float m, float c) {
#pragma clang fp contract(off)
    return m * c - (float)T::kLift;
}

// A row's running state in its lanes (both halves of the wave agree on m).
struct Running {
    float m, l;                  // reference (a score) and sum of the weights relative to it
    bool odd;                    // the row has to be done key by key (as one with an infinite reference has)
};

// The step of tile n for 32 rows of a wave: the weights p of its scores s, the products of the last tile's
// weights `last` with its values (PV), and the next tile's scores `next` (S). The three do not depend on one
// another, and the matrix unit only runs beside the vector unit where one wave's instructions
// alternate: a matrix instruction that waits for its unit keeps the SIMD's other wave from issuing vector
// instructions. So they are written down in turns, one matrix instruction, then its share of the
// exponentials, and kept in that order. (Scores, softmax and values one after the other: 538
// us for 8,192 rows of 32 heads of 128; with the two waves of a SIMD in opposite phases: 538; in turns: 508.)
// kt, vt: the next tile's keys and the last one's values. On their way to k_to and v_to are the
// keys after those and this tile's values. What is read and what is being loaded do not overlap (restrict
// says so to the compiler, which else waits for the loads before it reads anything).
template <class T, int DIM, int N, int LOADS, bool PV, bool S>
__device__ __forceinline__ void step(const uint8_t *__restrict kt, const uint8_t *__restrict vt, uint8_t *__restrict k_to,
                                     uint8_t *__restrict v_to, Rsrc kr, Rsrc vr, const uint32_t *k_off,
                                     const uint32_t *v_off, const Frag *q, f32x16 *s, f32x16 *next, const Frag *last, Frag *p,
                                     f32x16 *acc, Running &r, float c, float lazy, float huge) {
    constexpr int DT = DIM / 32, NT = N / 32, kPv = PV ? NT * 2 * DT : 0, kS = S ? NT * (DIM / 16) : 0;
    constexpr int kAll = kPv + kS, kElems = S ? NT * 16 : 0;
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const float inf = __builtin_inff();
    if constexpr (S) {
        load_tile<LOADS>(v_to, vr, v_off);
        load_tile<LOADS>(k_to, kr, k_off);
    }
    auto fragment = [&](int f) {
        if (f < kPv) {                   // 16 keys of 32 columns of the values, in the order of the weights' keys
            const int x = f / DT, d = f % DT;
            const int key = (x >> 1) * 32 + (x & 1) * 16 + half * 4 + ((lane & 15) >> 2);
            const int at = d * 32 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
            const u32x2 lo = read_columns<DIM, 32>(vt, key, at), hi = read_columns<DIM, 32>(vt, key + 8, at);
            return Frag{lo[0], lo[1], hi[0], hi[1]};
        }
        const int x = (f - kPv) / NT, j = (f - kPv) % NT;
        return read_rows<DIM>(kt, j * 32 + col, x * 2 + half);
    };
    constexpr int kAhead = 4;            // fragments read ahead
    Frag ahead[kAhead];
#pragma unroll
    for (int f = 0; f < kAhead && f < kAll; ++f) ahead[f] = fragment(f);

    // the first four shares: the highest score; then the reference, which moves only where a score
    // is far above it (any reference gives the same result); from then on the weights
    constexpr int kTop = kAll >= 16 ? 4 : 1;
    float top = -inf, to = r.m, mc = 0.f, sum = 0.f;
#pragma unroll
    for (int f = 0; f < kAll; ++f) {
        __builtin_amdgcn_sched_barrier(0);
        const Frag now = ahead[f % kAhead];
        if (f + kAhead < kAll) ahead[f % kAhead] = fragment(f + kAhead);
        if (f < kPv) {
            acc[f % DT] = T::mfma32(now, last[f / DT], acc[f % DT]);
        } else {
            const int x = (f - kPv) / NT, j = (f - kPv) % NT;
            next[j] = T::mfma32(now, q[x], x == 0 ? f32x16{} : next[j]);
        }
        if constexpr (S) {
            if (f < kTop) {
#pragma unroll
                for (int e = f * kElems / kTop; e < (f + 1) * kElems / kTop; ++e) top = fmaxf(top, s[e / 16][e % 16]);
            } else {
                if (f == kTop) {
                    top = max_halves(top);
                    to = top > r.m + lazy ? fmaxf(r.m, top) : r.m;
                    mc = to == -inf ? 0.f : base_of<T>(to, c);
                }
                constexpr int kShares = kAll - kTop;
                const int e0 = (f - kTop) * (kElems / 2) / kShares * 2, e1 = (f - kTop + 1) * (kElems / 2) / kShares * 2;
#pragma unroll
                for (int e = e0; e < e1; e += 2) {
                    const float a = exp2_fast(__builtin_fmaf(s[e / 16][e % 16], c, -mc));
                    const float b = exp2_fast(__builtin_fmaf(s[e / 16][e % 16 + 1], c, -mc));
                    sum += a + b;
                    uint32_t w = T::pack(a, b);
                    asm volatile("" : "+v"(w), "+v"(sum));       // (here, not where it is used)
                    p[e / 8][e % 8 / 2] = w;
                }
            }
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (S) {
        if (__any(to != r.m)) {          // what there is so far is relative to the old reference
            const float keep = r.m == -inf ? 0.f : exp2_fast((r.m - to) * c);
            r.l *= keep;
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] *= keep;
            r.m = fabsf(to) >= huge ? inf : to;
        }
        r.l += sum;
    }
}

template <class T, int DIM>
__global__ __launch_bounds__(64 * kWaves, DIM <= 128 ? 2 : 1) void k_attn_prompt(PromptArgs a) {
    constexpr int N = key_tile<DIM>(), RB = Tile<DIM>::kRowBytes;
    constexpr int KS = DIM / 16, DT = DIM / 32, NT = N / 32;
    constexpr int kTileBytes = N * RB, kLoads = kTileBytes / 1024 / kWaves;
    __shared__ __align__(128) uint8_t lds[4 * kTileBytes];    // K of two tiles, V of two tiles

    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;

    // the head, tile and split of this block: the heads that share keys run on one XCD where they
    // can be dealt out evenly, tiles with the most keys first
    uint32_t head, t, split;
    const uint32_t b = blockIdx.x;
    if (a.kv_heads % 8 == 0) {
        const uint32_t i = b >> 3, per = a.group * a.splits * a.tiles;
        head = ((b & 7) + 8 * (i / per)) * a.group + i % per % a.group;
        split = i % per / a.group % a.splits;
        t = i % per / a.group / a.splits;
    } else {
        head = b % a.q_heads;
        split = b / a.q_heads % a.splits;
        t = b / a.q_heads / a.splits;
    }
    SeqTile st;
    if (!find_tile<false>(a.p.q_starts, a.p.k_starts, a.p.n_seqs, a.p.q_rows, a.p.k_rows, kBlockRows, t, st)) return;
    const int tile = st.rank;
    const int q_len = st.q_len, k_len = st.k_len;
    const int past = k_len - q_len;                            // causal: row i sees keys j <= i + past
    const int row = tile * kBlockRows + wave * 32 + col;
    const int seen_row = min(row, q_len - 1);
    const int limit = a.causal ? min(max(seen_row + past + 1, 0), k_len) : k_len;   // keys that this lane's row sees
    const int wave_first = min(tile * kBlockRows + wave * 32, q_len - 1);
    const int wave_all = a.causal ? min(max(wave_first + past + 1, 0), k_len) : k_len;   // keys that all its rows see
    const int block_last = min(tile * kBlockRows + kBlockRows - 1, q_len - 1);
    const int keys = a.causal ? min(max(block_last + past + 1, 0), k_len) : k_len;
    const int all_tiles = (keys + N - 1) / N, per_split = (all_tiles + a.splits - 1) / a.splits;
    const int first_tile = min((int)split * per_split, all_tiles), n_tiles = min(first_tile + per_split, all_tiles);

    const uint32_t kv = head / a.group;
    const uint32_t k_stride = (uint32_t)a.k.row * 2, v_stride = (uint32_t)a.v.row * 2;
    const uint8_t *kp = (const uint8_t *)a.k.data + ((int64_t)st.k0 * a.k.row + (int64_t)kv * a.k.head) * 2;
    const uint8_t *vp = (const uint8_t *)a.v.data + ((int64_t)st.k0 * a.v.row + (int64_t)kv * a.v.head) * 2;

    uint32_t k_off[kLoads], v_off[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int slot = (i * kWaves + wave) * 64 + lane;
        k_off[i] = tile_source<DIM, true>(slot, k_stride, a.dim);
        v_off[i] = tile_source<DIM, false>(slot, v_stride, a.dim);
    }
    uint8_t *const lk = lds + wave * 1024, *const lv = lk + 2 * kTileBytes;
    auto tile_of = [&](const uint8_t *p, uint32_t stride, int n) {       // (empty past the last tile: zeros)
        const int rows = n < n_tiles ? min(k_len - n * N, N) : 0;
        return descriptor(rows ? p + (int64_t)n * N * stride : p, rows ? (rows - 1) * stride + a.dim * 2 : 0);
    };
    const bool some = first_tile < n_tiles;
    if (some) {
        load_tile<kLoads>(lk + (first_tile & 1) * kTileBytes, tile_of(kp, k_stride, first_tile), k_off);
        load_tile<kLoads>(lk + (~first_tile & 1) * kTileBytes, tile_of(kp, k_stride, first_tile + 1), k_off);
    }

    Frag q[KS];
    {
        const uint8_t *qp = (const uint8_t *)a.q.data + ((int64_t)(st.q0 + seen_row) * a.q.row + (int64_t)head * a.q.head) * 2;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = load_head<false>(qp, s * 16 + half * 8, a.dim);
    }

    const float inf = __builtin_inff();
    const float c = a.scale_log2;
    Running r{-inf, 0.f, false};
    f32x16 acc[DT], s0[NT], s1[NT];
    Frag p0[NT * 2], p1[NT * 2];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = f32x16{};

    // keys from a row's limit on have no score; `at` is tile n's first key
    auto hide = [&](f32x16 *s, int at) {
        const int end = limit - at - half * 4;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (j * 32 + (i >> 2) * 8 + (i & 3) >= end) s[j][i] = -inf;
    };
    // a weight of zero must not meet an infinity or NaN: rows that do not see all of such a tile are
    // done again, key by key
    auto look = [&](const uint8_t *vt) {
#pragma unroll 4
        for (int x = lane * 16; x < kTileBytes; x += 1024)
            r.odd |= has_nonfinite<T>(*reinterpret_cast<const Frag *>(vt + x));
    };
    auto tile_n = [&](auto pv, int n, f32x16 *s, f32x16 *next, const Frag *last, Frag *p) {
        tiles_loaded();
        const uint8_t *kt = lds + (~n & 1) * kTileBytes, *vt = lds + (2 + (~n & 1)) * kTileBytes;
        if (n * N + N > wave_all) hide(s, n * N);
        if (pv.value && n * N > wave_all) look(vt);
        step<T, DIM, N, kLoads, pv.value, true>(kt, vt, lk + (n & 1) * kTileBytes, lv + (n & 1) * kTileBytes,
                                                tile_of(kp, k_stride, n + 2), tile_of(vp, v_stride, n), k_off, v_off, q, s, next,
                                                last, p, acc, r, c, a.lazy, a.huge);
    };
    if (some) {
        tiles_loaded();
#pragma unroll
        for (int j = 0; j < NT; ++j) s0[j] = f32x16{};
#pragma unroll
        for (int x = 0; x < KS; ++x)
#pragma unroll
            for (int j = 0; j < NT; ++j)
                s0[j] = T::mfma32(read_rows<DIM>(lds + (first_tile & 1) * kTileBytes, j * 32 + col, x * 2 + half), q[x], s0[j]);
        tile_n(std::false_type{}, first_tile, s0, s1, p1, p0);
        for (int n = first_tile + 1; n < n_tiles; n += 2) {
            tile_n(std::true_type{}, n, s1, s0, p0, p1);
            if (n + 1 < n_tiles) tile_n(std::true_type{}, n + 1, s0, s1, p1, p0);
        }
        tiles_loaded();                  // the last tile's values
        const uint8_t *vt = lds + (2 + (~n_tiles & 1)) * kTileBytes;
        if (n_tiles * N > wave_all) look(vt);
        const bool even = (n_tiles - first_tile) & 1;        // whose weights the last tile left
#pragma unroll
        for (int x = 0; x < NT * 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) p0[x][i] = even ? p0[x][i] : p1[x][i];
        step<T, DIM, N, kLoads, true, false>(nullptr, vt, nullptr, nullptr, tile_of(kp, 0, n_tiles), tile_of(vp, 0, n_tiles), k_off,
                                             v_off, q, s0, s1, p0, p1, acc, r, c, a.lazy, a.huge);
    }
    const float m = r.m;
    float l = r.l;
    const bool odd = r.odd || m == inf;
    if (__any(odd)) {
        const int rows = min(q_len - (tile * kBlockRows + wave * 32), 32);
        for (int r = 0; r < rows; ++r)
            attend_row<T, DIM>(a, st.q0 + row - col + r, head, split, kp, vp, first_tile * N,
                               min(uniform(__shfl(limit, r)), n_tiles * N));
        return;
    }

    constexpr float unit = 1.f / (1 << T::kLift);
    l = sum_halves(l) * unit;
    if (row >= q_len) return;
    if (a.splits > 1) {
        const int64_t at = part_at(a, split, head, st.q0 + row);
        if (half == 0) a.stats[at] = f32x2{m, l};
        float *pp = a.partial + at * a.dim;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int to = d * 32 + i * 8 + half * 4;
                if (to < (int)a.dim)
                    *reinterpret_cast<f32x4 *>(pp + to) =
                        f32x4{acc[d][i * 4], acc[d][i * 4 + 1], acc[d][i * 4 + 2], acc[d][i * 4 + 3]} * unit;
            }
        return;
    }
    const float inv = l == 0.f ? 0.f : unit / l;
    if (__any(l == 0.f)) {               // (a weight of 0 may have met an infinity)
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[d] = l == 0.f ? f32x16{} : acc[d];
    }
    uint8_t *op = (uint8_t *)a.out.data + ((int64_t)(st.q0 + row) * a.out.row + (int64_t)head * a.out.head) * 2;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = d * 32 + i * 8 + half * 4;
            u32x2 w;
            w[0] = T::pack_out(acc[d][i * 4] * inv, acc[d][i * 4 + 1] * inv);
            w[1] = T::pack_out(acc[d][i * 4 + 2] * inv, acc[d][i * 4 + 3] * inv);
            if (at < (int)a.dim) *reinterpret_cast<u32x2 *>(op + at * 2) = w;
        }
    if (a.lse && half == 0)
        a.lse[(int64_t)head * a.p.q_rows + st.q0 + row] = l == 0.f ? -inf : m * a.scale + __logf(l);
}

// Joins the splits of 32 rows of a tile, four dims per thread:
//   m = max_x m_x,  l = sum_x l_x 2^(m_x - m),  out = sum_x acc_x 2^(m_x - m) / l.
constexpr int kMaxSplits = 8;

template <class T>
__global__ __launch_bounds__(256) void k_attn_prompt_join(PromptArgs a) {
    constexpr int block_rows = kBlockRows, parts = block_rows / 32;
    const uint32_t b = blockIdx.x / parts, head = b % a.q_heads, t = b / a.q_heads;
    SeqTile st;
    if (!find_tile<false>(a.p.q_starts, a.p.k_starts, a.p.n_seqs, a.p.q_rows, a.p.k_rows, block_rows, t, st)) return;
    const int row0 = st.rank * block_rows + blockIdx.x % parts * 32, rows = min(st.q_len - row0, 32);
    const int quads = a.dim / 4;
    const float inf = __builtin_inff();
    for (int i = threadIdx.x; i < rows * quads; i += 256) {
        const int r = i / quads, d = (i - r * quads) * 4, row = st.q0 + row0 + r;
        f32x2 s[kMaxSplits];
        f32x4 x[kMaxSplits];
        float top = -inf;
#pragma unroll
        for (int y = 0; y < kMaxSplits; ++y) {
            const int64_t at = part_at(a, min(y, (int)a.splits - 1), head, row);
            s[y] = a.stats[at];
            x[y] = *reinterpret_cast<const f32x4 *>(a.partial + at * a.dim + d);
            top = fmaxf(top, s[y][0]);
        }
        float sum = 0.f;
        f32x4 o{};
#pragma unroll
        for (int y = 0; y < kMaxSplits; ++y) {
            const float f = part_of(s[y][0], s[y][1], top, a.scale_log2);
            if (y < (int)a.splits && !(f < 0.f)) {
                sum += f * s[y][1];
                o += f * x[y];
            }
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        u32x2 w;
        w[0] = T::pack_out(o[0] * inv, o[1] * inv);
        w[1] = T::pack_out(o[2] * inv, o[3] * inv);
        *reinterpret_cast<u32x2 *>((uint8_t *)a.out.data + ((int64_t)row * a.out.row + (int64_t)head * a.out.head + d) * 2) = w;
        if (a.lse && d == 0) a.lse[(int64_t)head * a.p.q_rows + row] = sum == 0.f ? -inf : top * a.scale + __logf(sum);
    }
}

template <class T>
hipError_t prompt_of(const PromptArgs &a, uint32_t blocks, hipStream_t stream) {
    const dim3 grid(blocks), block(64 * kWaves);
    if (a.dim <= 64) k_attn_prompt<T, 64><<<grid, block, 0, stream>>>(a);
    else if (a.dim <= 96) k_attn_prompt<T, 96><<<grid, block, 0, stream>>>(a);
    else if (a.dim <= 128) k_attn_prompt<T, 128><<<grid, block, 0, stream>>>(a);
    else k_attn_prompt<T, 256><<<grid, block, 0, stream>>>(a);
    if (a.splits > 1) k_attn_prompt_join<T><<<dim3(a.tiles * a.q_heads * kWaves), dim3(256), 0, stream>>>(a);
    return hipGetLastError();
}

// What the tiles of all sequences come to at most.
uint64_t tiles_of(uint64_t q_rows, uint64_t n_seqs) { return q_rows / kBlockRows + n_seqs; }

constexpr uint64_t kPlaces = 512;        // blocks that the chip holds at once

// Blocks that share a tile's keys: as many as leave none of the chip's places empty, each with at least 512 keys of a
// sequence of average length (1,000 rows of 16 heads of 64 against 9,001 keys: 59 us, in one block each 125).
uint32_t splits_of(uint32_t q_heads, uint64_t q_rows, uint64_t k_rows, uint64_t n_seqs) {
    const uint64_t blocks = tiles_of(q_rows, n_seqs) * q_heads;
    if (n_seqs == 0 || blocks == 0) return 1;
    return (uint32_t)std::max<uint64_t>(std::min<uint64_t>({(uint64_t)kMaxSplits, kPlaces / blocks, k_rows / n_seqs / 512}), 1);
}

uint64_t up256(uint64_t x) { return (x + 255) / 256 * 256; }

// Of a call: what its parts take (none where one block per tile does).
uint64_t prompt_parts(uint32_t q_heads, uint32_t dim, uint64_t q_rows, uint64_t splits) {
    const uint64_t parts = splits > 1 ? splits * q_heads * q_rows : 0;
    return up256(parts * 8) + up256(parts * dim * 4);
}

}  // namespace

uint64_t prompt_needs(uint32_t q_heads, uint32_t dim, uint64_t q_rows, uint64_t k_rows, uint32_t n_seqs) {
    return prompt_parts(q_heads, dim, q_rows, splits_of(q_heads, q_rows, k_rows, n_seqs));
}

// Fewer rows make fewer blocks, which are split more: of every number of splits that the keys
// allow, with the most rows that are split that often.
uint64_t prompt_workspace(uint32_t q_heads, uint32_t dim, uint64_t q_rows, uint64_t k_rows, uint32_t n_seqs) {
    uint64_t most = 0;
    for (uint64_t splits = 2; n_seqs && splits <= std::min<uint64_t>(kMaxSplits, k_rows / n_seqs / 512); ++splits) {
        const uint64_t tiles = kPlaces / splits / q_heads;
        if (tiles >= n_seqs) most = std::max(most, prompt_parts(q_heads, dim, std::min(q_rows, (tiles - n_seqs + 1) * kBlockRows - 1), splits));
    }
    return most;
}

hipError_t launch_prompt(const Shape &s, const Rows &q, const Rows &k, const Rows &v, const Packed &p, const Rows &out,
                         float *lse, uint8_t *workspace, hipStream_t stream) {
    if (p.n_seqs == 0 || p.q_rows == 0) return hipSuccess;
    const uint64_t tiles = tiles_of(p.q_rows, p.n_seqs);
    const uint32_t splits = splits_of(s.q_heads, p.q_rows, p.k_rows, p.n_seqs);
    const uint64_t blocks = tiles * s.q_heads * splits;
    if (blocks > kMaxGrid) return hipErrorInvalidConfiguration;
    PromptArgs a{q, k, v, out, p, lse, s.q_heads, s.kv_heads, s.group, s.dim, (uint32_t)tiles, splits,
                 (f32x2 *)workspace, (float *)(workspace + up256((uint64_t)splits * s.q_heads * p.q_rows * 8)), s.scale,
                 s.scale_log2, (s.f16 ? lazy<F16>() : lazy<Bf16>()) / s.scale_log2, (s.f16 ? huge<F16>() : huge<Bf16>()) / s.scale_log2,
                 s.causal ? 1u : 0u};
    return s.f16 ? prompt_of<F16>(a, (uint32_t)blocks, stream) : prompt_of<Bf16>(a, (uint32_t)blocks, stream);
}

}  // namespace attn
}  // namespace ibp
