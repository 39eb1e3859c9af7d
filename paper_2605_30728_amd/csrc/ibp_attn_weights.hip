// The attention weight that every key received from the rows of its sequence:
//   w[j] = sum over the query heads of its KV head and the rows i that see it of exp(s_ij - lse_i),
// s_ij as in attention over prompts and lse_i what that left behind. A block holds 64 keys per
// wave as matrix fragments and streams the rows of one query head past them; the query heads of
// a KV head are added up by a second kernel, so that the result never depends on an order.
#include "ibp_attn.hpp"
#include "ibp_attn_wave.hpp"

namespace ibp {
namespace attn {

namespace {

using namespace dev;

struct WeightArgs {
    Rows q, k;
    Packed p;
    const float *lse;
    float *out;                  // [q_heads][k_rows]
    uint32_t q_heads, kv_heads, group, dim;
    uint32_t tiles;
    float scale_log2;
    uint32_t causal;
};

constexpr int kWaves = 4;
constexpr int kBlockKeys = 64 * kWaves;
constexpr float kLog2e = 1.4426950408889634f;

template <int DIM>
constexpr int row_tile() { return DIM <= 128 ? 64 : 32; }

template <class T, int DIM>
__global__ __launch_bounds__(64 * kWaves, DIM <= 128 ? 2 : 1) void k_attn_key_weights(WeightArgs a) {
    constexpr int N = row_tile<DIM>(), RB = Tile<DIM>::kRowBytes, KS = DIM / 16, NT = N / 32;
    constexpr int kTileBytes = N * RB, kLoads = kTileBytes / 1024 / kWaves;
    __shared__ __align__(128) uint8_t lds[2 * kTileBytes];
    __shared__ __align__(16) float lse_tile[2][N];

    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    uint32_t head, t;
    const uint32_t b = blockIdx.x;
    if (a.q_heads % 8 == 0) {            // one head's rows stay in one XCD's cache
        const uint32_t i = b >> 3;
        head = (b & 7) * (a.q_heads / 8) + i % (a.q_heads / 8);
        t = i / (a.q_heads / 8);
    } else {
        head = b % a.q_heads;
        t = b / a.q_heads;
    }
    SeqTile st;
    if (!find_tile<true>(a.p.q_starts, a.p.k_starts, a.p.n_seqs, a.p.q_rows, a.p.k_rows, kBlockKeys, t, st)) return;
    const int q_len = st.q_len, k_len = st.k_len, past = k_len - q_len;
    const uint32_t kv = head / a.group;
    const int tile = st.tiles - 1 - st.rank, key0 = tile * kBlockKeys + wave * 64;   // (the first keys are seen by the most rows)

    Frag k[2][KS];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int key = min(key0 + j * 32 + col, k_len - 1);
        const uint8_t *kp = (const uint8_t *)a.k.data + ((int64_t)(st.k0 + key) * a.k.row + (int64_t)kv * a.k.head) * 2;
#pragma unroll
        for (int x = 0; x < KS; ++x) k[j][x] = load_head<false>(kp, x * 16 + half * 8, a.dim);
    }

    const uint32_t q_stride = (uint32_t)a.q.row * 2;
    const uint8_t *qp = (const uint8_t *)a.q.data + ((int64_t)st.q0 * a.q.row + (int64_t)head * a.q.head) * 2;
    const float *lse = a.lse + (int64_t)head * a.p.q_rows + st.q0;
    uint32_t q_off[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) q_off[i] = tile_source<DIM, true>((i * kWaves + wave) * 64 + lane, q_stride, a.dim);
    auto load_tile = [&](int n, int buf) {
        const int rows = min(q_len - n * N, N);
        const Rsrc r = descriptor(qp + (int64_t)n * N * q_stride, (rows - 1) * q_stride + a.dim * 2);
        uint8_t *at = lds + buf * kTileBytes + wave * 1024;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load_to_lds(r, at + i * kWaves * 1024, q_off[i]);
    };
    const float inf = __builtin_inff();
    auto load_lse = [&](int n) {         // rows that count nowhere get an infinite one
        const int row = n * N + (int)threadIdx.x;
        const float x = threadIdx.x < N && row < q_len ? lse[row] : inf;
        return x == -inf ? inf : x * kLog2e;
    };

    // the first row that sees a key of this block, and of this wave; the first that sees all of the wave's
    const int first = a.causal ? max(tile * kBlockKeys - past, 0) : 0;
    const int wave_any = a.causal ? max(key0 - past, 0) : 0;
    const int wave_all = a.causal ? max(min(key0 + 63, k_len - 1) - past, 0) : 0;
    const int n0 = first / N, n1 = (q_len + N - 1) / N;

    f32x16 sum[2] = {f32x16{}, f32x16{}};
    if (n0 < n1) {
        load_tile(n0, n0 & 1);
        const float x = load_lse(n0);
        if (threadIdx.x < N) lse_tile[n0 & 1][threadIdx.x] = x;
    }
    for (int n = n0; n < n1; ++n) {
        tiles_loaded();
        float next_lse = 0.f;
        if (n + 1 < n1) {
            load_tile(n + 1, (n + 1) & 1);
            next_lse = load_lse(n + 1);
        }
        const int row0 = n * N;
        if (row0 + N > wave_any && key0 < k_len) {
            const uint8_t *qt = lds + (n & 1) * kTileBytes;
            const bool masked = row0 < wave_all || row0 + N > q_len;
#pragma unroll
            for (int y = 0; y < NT; ++y) {
                f32x16 s[2] = {f32x16{}, f32x16{}};
#pragma unroll
                for (int x = 0; x < KS; ++x) {
                    const Frag f = read_rows<DIM>(qt, y * 32 + col, x * 2 + half);
                    s[0] = T::mfma32(f, k[0][x], s[0]);
                    s[1] = T::mfma32(f, k[1][x], s[1]);
                }
                f32x4 ls[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    ls[i] = *reinterpret_cast<const f32x4 *>(&lse_tile[n & 1][y * 32 + i * 8 + half * 4]);
                // (a pair that does not count is left out after the exponential: its score and the
                // row's lse may be anything)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int seen = a.causal ? key0 + j * 32 + col - past : 0;   // the first row that sees this key
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float e = exp2_fast(__builtin_fmaf(s[j][i], a.scale_log2, -ls[i >> 2][i & 3]));
                        if (masked) {
                            const int row = row0 + y * 32 + (i >> 2) * 8 + half * 4 + (i & 3);
                            e = row < seen || row >= q_len ? 0.f : e;
                        }
                        sum[j][i] += e;
                    }
                }
            }
        }
        if (n + 1 < n1 && threadIdx.x < N) lse_tile[(n + 1) & 1][threadIdx.x] = next_lse;
    }

    float *out = a.out + (int64_t)head * a.p.k_rows + st.k0;
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

__global__ __launch_bounds__(256) void k_sum_heads(const float *partial, float *weights, uint32_t group, uint32_t k_rows,
                                                   const int32_t *k_starts, uint32_t n_seqs) {
    const uint32_t per = (k_rows + 255) / 256, kv = blockIdx.x / per, j = blockIdx.x % per * 256 + threadIdx.x;
    const int from = clamp_row(k_starts[0], k_rows), to = clamp_row(k_starts[n_seqs], k_rows);
    if ((int64_t)j < from || (int64_t)j >= to) return;       // rows of no sequence
    const float *p = partial + (int64_t)kv * group * k_rows + j;
    float w = 0.f;
    for (uint32_t g = 0; g < group; ++g) w += p[(int64_t)g * k_rows];
    weights[(int64_t)kv * k_rows + j] = w;
}

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
    const uint64_t tiles = p.k_rows / kBlockKeys + (uint64_t)p.n_seqs;
    const uint64_t blocks = tiles * s.q_heads, sum_blocks = (uint64_t)(p.k_rows + 255) / 256 * s.kv_heads;
    if (blocks > kMaxGrid || sum_blocks > kMaxGrid) return hipErrorInvalidConfiguration;
    const bool one = s.group == 1;
    WeightArgs a{q, k, p, lse, one ? weights : partial, s.q_heads, s.kv_heads, s.group, s.dim, (uint32_t)tiles,
                 s.scale_log2, s.causal ? 1u : 0u};
    hipError_t e = s.f16 ? weights_of<F16>(a, (uint32_t)blocks, stream) : weights_of<Bf16>(a, (uint32_t)blocks, stream);
    if (e != hipSuccess || one) return e;
    k_sum_heads<<<dim3((uint32_t)sum_blocks), dim3(256), 0, stream>>>(partial, weights, s.group, p.k_rows, p.k_starts,
                                                                      p.n_seqs);
    return hipGetLastError();
}

}  // namespace attn
}  // namespace ibp
