// Attention of one new token per sequence over a paged cache of 4-bit records.
//
// As in the decode of 16-bit caches the cache's length is split over blocks and a block's waves, and its second kernel
// joins the blocks. Keys and values are never widened to what they stand for, whose rounding to 16 bits would show: a
// code is exact as the 16-bit number 16 + code (its bits below those of 16), so that with groups g of 32 values
//   x_j = scale sum_g [ step_jg sum_d q_d (16 + c_jd)  -  47/2 step_jg sum_d q_d  +  centre_jg sum_d q_d ]
//   out_d = sum_j (p_j step_jg) (16 + c_jd)  -  47/2 sum_j (p_j step_jg)  +  sum_j p_j centre_jg.
// A group is what one 16x16x32 product sums over for the keys; the last two terms of a score are one more product of a
// record's steps and centres with the queries' sums, split into three 16-bit parts (24 bits).
//
// The weights times steps p_j step_jg are rounded for the product with the codes, and the same rounded ones meet 16 + c and 47/2. In
// bfloat16 that would show as much as the rounding of the output does (error against 64 bits 0.0023 of the output instead of
// 0.0017), so a bfloat16 cache's are float16 numbers (39 us for the long cache below instead of 37.5 then), its steps scaled so that
// the largest so far is from 2^14 to 2^15, which leaves float16's small numbers to small weights: they have 11 bits
// down to 2^-28 of the largest step and are there down to 2^-39. A float16 cache's are two bfloat16 parts, 16 bits at any
// size (for a bfloat16 cache that took 45 us then).
//
// Centres meet weights that are rounded less: values may lie in their centres alone, with signs by which sums are far below what is
// added up (weights of 8 bits were off by 0.005 of such an output, more than its own rounding). A bfloat16 cache's are two bfloat16
// parts, 16 bits at any size, side by side along one product's k of 32 (131,071 slots 47.9 us a call when that was chosen, 45.8 with one
// part, 50.9 with weights in 32 bits). float16 has too few exponents for parts: those weights stay in 32 bits, and so does the
// product (24 sequences of heads of 256 up to 6,000 slots 26.6 us a call, 26.0 with weights of 16 bits).
//
// A chunk of 64 slots is about 730 vector instructions and 56 matrix ones for a head of 128 in bfloat16, with the records' loads of
// the next half chunk on their way (131,071 slots of 8 heads of 128: 43 us of which some 7 are a block's start and end, 168 MB, 4.7 TB/s
// in between; vector unit busy 0.63, LDS 0.36, matrix unit 0.17; in float16, with two parts and the centres in 32 bits, 56 us).
// 64 sequences of up to 8,192 slots with the slots' weights: 97 us (4.0 TB/s; in float16 117). Three waves a SIMD hide what a wave waits
// for its products; two, as heads above 128 have them, took 125 us a call there instead of 116 when that was measured. Short
// caches are bound by one wave's instructions, one after another at some 8 cycles: 1,531 slots 8 us, no less than their 16-bit decode.
#include <algorithm>
#include <type_traits>

#include "ibp_attn_decode.hpp"
#include "ibp_attn_wave.hpp"
#include "ibp_kv_cache.hpp"

namespace ibp {
namespace attn {

namespace {

using namespace dev;

constexpr int kWaves = 4;
constexpr int kChunk = 64;               // slots that a wave takes at a time: a lane looks up each one's page

// A chunk's keys, then its values, in LDS: rows of codes of an odd number of 16-byte pieces, so that the 16 keys of a product are in
// different banks; the records' steps and centres as they are; and the steps in 32 bits, [group][slot].
template <int G>
struct Rec {
    static constexpr int kMetaFrags = (G + 3) / 4, kCodes = G * kGroupBytes;
    static constexpr int kRow = (G | 1) * 16, kMetaRow = kMetaFrags * 16;
    static constexpr int kMeta = kChunk * kRow, kSteps = kMeta + kChunk * kMetaRow + 16, kBytes = kSteps + G * kChunk * 4;
};

// What turns codes into 16-bit numbers: where they lie in these, and 16. Kept out of the compiler's sight, in a scalar and a
// vector register, so that masking and setting are one instruction (constants it would take apart).
template <class T>
struct Widen {
    uint32_t mask, sixteen;
    __device__ __forceinline__ Widen() {
        asm("s_mov_b32 %0, %1" : "=s"(mask) : "n"(std::is_same_v<T, Bf16> ? 0x00780078 : 0x03c003c0));
        asm("v_mov_b32 %0, %1" : "=v"(sixteen) : "n"(std::is_same_v<T, Bf16> ? 0x41804180 : 0x4c004c00));
    }
    // Eight codes, values i and i + 4 of them side by side.
    __device__ __forceinline__ Frag operator()(uint32_t x) const {
        constexpr bool b = std::is_same_v<T, Bf16>;
        return Frag{((b ? x << 3 : x << 6) & mask) | sixteen, ((b ? x >> 1 : x << 2) & mask) | sixteen,
                    ((b ? x >> 5 : x >> 2) & mask) | sixteen, ((b ? x >> 9 : x >> 6) & mask) | sixteen};
    }
};

// The two 16-bit halves of a dword as numbers.
template <class T>
__device__ __forceinline__ float low(uint32_t x) {
    return T::value((uint16_t)x);
}
template <class T>
__device__ __forceinline__ float high(uint32_t x) {
    if constexpr (std::is_same_v<T, Bf16>) return __uint_as_float(x & 0xffff0000u);
    else return T::value((uint16_t)(x >> 16));
}

// 16 rows of 16 codes, transposed over 16 lanes: lane i gets code i of the rows whose addresses the lanes pass.
__device__ __forceinline__ u32x2 read_codes(const uint8_t *p) {
    typedef int v2i __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr4_b64_v2i32((IBP_LDS(v2i) *)p));
}
// Four rows of 16 16-bit numbers, the same.
__device__ __forceinline__ u32x2 read_numbers(const uint8_t *p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((IBP_LDS(s16x4) *)p));
}

// 16x16x4 of 32-bit numbers: A and B have k = l / 16, one number a lane; C as of the other products of 16 rows.
__device__ __forceinline__ f32x4 mfma_f32(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// The largest of x over a wave.
__device__ __forceinline__ float max_wave(float x) {
    auto turned = [](float v, auto by) {             // of the 16 lanes that a lane is one of
        return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x120 + decltype(by)::value, 0xf, 0xf, true));
    };
    x = fmaxf(x, turned(x, std::integral_constant<int, 8>{}));
    x = fmaxf(x, turned(x, std::integral_constant<int, 4>{}));
    x = fmaxf(x, turned(x, std::integral_constant<int, 2>{}));
    x = fmaxf(x, turned(x, std::integral_constant<int, 1>{}));
    return __uint_as_float((uint32_t)uniform((int)__float_as_uint(max_halves(max_quarters(x)))));
}

// Key `row` of the t-th product of a chunk is this slot of it: those that a quarter of the wave has
// of all four products are spread over the banks.
__device__ __forceinline__ int slot_of(int t, int row) { return t * 16 + (row ^ (t & 1) * 8); }

// Three waves a SIMD for heads of up to 128, two above, whose 168 and 256 registers hold what a wave has in work but for a few that
// spill into the loop: nine of heads of 97 to 128 in float16, of heads above 224 eight in bfloat16 and 13 in float16.
template <class T, int G>
__global__ __launch_bounds__(64 * kWaves, G <= 4 ? 3 : 2) void k_attn_decode4(DecodeArgs a) {
    using R = Rec<G>;
    constexpr int DIM = G * kGroupValues, DT = DIM / 16, MF = R::kMetaFrags;
    constexpr bool kHalf = std::is_same_v<T, F16>;
    using P = std::conditional_t<kHalf, Bf16, F16>;  // of the weights times steps, kParts numbers each
    constexpr int kParts = kHalf ? 2 : 1;
    constexpr int kJoin = 16 * (DIM + 4) * 4;        // a wave's sums, for the join
    constexpr int kWaveBytes = R::kBytes > kJoin ? R::kBytes : kJoin;
    __shared__ __align__(128) uint8_t lds[kWaves * kWaveBytes];
    __shared__ float stat[kWaves][2][16];
    __shared__ __align__(16) float sums[kWaves][16][16];

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

    Frag raw[G];                         // the queries, used once the first records are on their way
    {
        const uint8_t *qp = (const uint8_t *)a.q.data + ((int64_t)seq * a.q.row + (int64_t)(head0 + min(col, heads - 1)) * a.q.head) * 2;
#pragma unroll
        for (int g = 0; g < G; ++g) raw[g] = load_head<false>(qp, g * kGroupValues + quarter * 8, a.dim);
    }

    // lane i looks up the page of slot i of a chunk
    const int32_t *table = a.pg.table + (int64_t)seq * a.pg.table_stride;
    int page = 0, place = 0;
    auto find = [&](int chunk) {
        const uint32_t s = min(chunk + lane, len - 1);
        const uint32_t i = a.pg.page_magic ? __umulhi(s, a.pg.page_magic) >> a.pg.page_shift : s >> a.pg.page_shift;
        place = (int)(s - i * a.pg.page_tokens);
        page = table[i];
    };

    const Widen<T> widen;
    const Widen<P> widen_p;
    const float inf = __builtin_inff();
    const float c = a.scale_log2;
    float m = -inf, ref = 0.f, l = 0.f;     // reference, what scores are taken relative to (0 while there is none), sum
    f32x4 acc[DT], z{};                     // out, and the weighted sums of steps and centres
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = f32x4{};
    // the queries, in the order of Widen, and the products' second operand for steps and centres
    Frag q[G], qs[MF];
    float back = 1.f;                    // what its product is to be multiplied with
    {
        float side[MF * 8];              // -47/2 sum and sum of every group, in the order of a record's steps and centres
#pragma unroll
        for (int i = 0; i < MF * 8; ++i) side[i] = 0.f;
        float top = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const Frag f = raw[g];
            float x = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) x += low<T>(f[i]) + high<T>(f[i]);
            x = sum_halves(sum_quarters(x));
            side[g] = -23.5f * x;
            side[G + g] = x;
            top = fmaxf(top, fabsf(side[g]));
            q[g] = Frag{(f[0] & 0xffffu) | f[2] << 16, f[0] >> 16 | (f[2] & 0xffff0000u), (f[1] & 0xffffu) | f[3] << 16,
                        f[1] >> 16 | (f[3] & 0xffff0000u)};
        }
        if constexpr (kHalf) {           // float16: the largest brought to 2^14, so that no part is lost below or above
            const int e = top > 0.f && top < __builtin_inff() ? (int)(__float_as_uint(top) >> 23) - 127 - 14 : 0;
            back = __builtin_amdgcn_ldexpf(1.f, e);
#pragma unroll
            for (int i = 0; i < MF * 8; ++i) side[i] = __builtin_amdgcn_ldexpf(side[i], -e);
        }
        // quarter 0, 1 and 2 have the first, second and third part
#pragma unroll
        for (int i = 0; i < MF * 8; i += 2) {
            float x = side[i], y = side[i + 1];
            uint32_t part = T::pack(x, y);
#pragma unroll
            for (int n = 1; n < 3; ++n) {
                x -= low<T>(part);
                y -= high<T>(part);
                const uint32_t next = T::pack(x, y);
                part = quarter >= n ? next : part;
            }
            qs[i / 8][i % 8 / 2] = quarter == 3 ? 0u : part;
        }
    }

    uint8_t *tile = lds + wave * kWaveBytes, *meta = tile + R::kMeta;
    float *steps = reinterpret_cast<float *>(tile + R::kSteps);

    // Keys and values take turns in the same registers and the same LDS: values are on their way during the products with the keys, the
    // next chunk's keys during those with the values. A lane loads pieces of codes, neighbours neighbouring ones, and
    // the steps and centres of its own slot.
    constexpr int kStep = kWaves * kChunk;
    Frag codes[G], numbers[MF];
    int64_t value_at = 0;                // of this lane's slot
    uint64_t live = 0;                   // bit i: slot i of the chunk is there
    const uint8_t *kbase = (const uint8_t *)a.pg.k.data + (int64_t)kv * a.pg.k.head * 2;
    const uint8_t *vbase = (const uint8_t *)a.pg.v.data + (int64_t)kv * a.pg.v.head * 2;
    auto of_slot = [](int64_t x, int slot) {         // lane `slot`'s x
        return (int64_t)((uint64_t)(uint32_t)__shfl((int)(x >> 32), slot) << 32 | (uint32_t)__shfl((int)x, slot));
    };
    auto load = [&](const uint8_t *base, int64_t at) {
#pragma unroll
        for (int i = 0; i < MF; ++i) numbers[i] = *reinterpret_cast<const Frag *>(base + at + R::kCodes + i * 16);
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int x = i * 64 + lane;
            codes[i] = *reinterpret_cast<const Frag *>(base + of_slot(at, x / G) + x % G * 16);
        }
    };
    auto load_keys = [&](int chunk) {
        const bool in = (uint32_t)page < a.pg.n_pages;
        live = __ballot(in && chunk + lane < len);
        const int64_t pg = in ? page : 0;
        value_at = (pg * a.pg.v.page + (int64_t)place * a.pg.v.token) * 2;
        load(kbase, (pg * a.pg.k.page + (int64_t)place * a.pg.k.token) * 2);
    };
    // A bfloat16 cache's value steps are scaled by 2^shift: the largest so far, which is below `limit`, to 2^14 .. 2^15.
    int shift = 0;
    float limit = 0.f;
    auto raise = [&](float top, const float (&step)[G]) {      // a larger one, and with it what there is so far
        if (top == inf) {
            top = 0.f;
#pragma unroll
            for (int g = 0; g < G; ++g) top = fmaxf(top, fabsf(step[g]) < inf ? fabsf(step[g]) : 0.f);
            top = max_wave(top);
            if (top < limit || top == 0.f) return;
        }
        const int e = (int)(__float_as_uint(top) >> 23) - 127, next = 14 - e;
        if (limit > 0.f) {
            const float less = __builtin_amdgcn_ldexpf(1.f, next - shift);
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] *= less;
        }
        shift = next;
        limit = __builtin_amdgcn_ldexpf(2.f, e);
    };
    auto store = [&](uint64_t live, bool of_values) {
        const bool there = live >> lane & 1;         // else steps and centres of 0: it counts for nothing
#pragma unroll
        for (int i = 0; i < MF; ++i) {
#pragma unroll
            for (int w = 0; w < 4; ++w)              // (what follows a record's numbers may be anything)
                numbers[i][w] = i * 4 + w < G && there ? numbers[i][w] : 0u;
            *reinterpret_cast<Frag *>(meta + lane * R::kMetaRow + i * 16) = numbers[i];
        }
        float step[G];
#pragma unroll
        for (int g = 0; g < G; ++g) step[g] = g % 2 ? high<T>(numbers[g / 8][g % 8 / 2]) : low<T>(numbers[g / 8][g % 8 / 2]);
        if (!kHalf && of_values) {
            float top = 0.f;
#pragma unroll
            for (int g = 0; g < G; ++g) top = fmaxf(top, fabsf(step[g]));        // (NaN is left out)
            top = max_wave(top);
            if (top >= limit && top > 0.f) raise(top, step);
#pragma unroll
            for (int g = 0; g < G; ++g) step[g] = __builtin_amdgcn_ldexpf(step[g], shift);
        }
#pragma unroll
        for (int g = 0; g < G; ++g) steps[g * kChunk + lane] = step[g];
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int x = i * 64 + lane;
            *reinterpret_cast<Frag *>(tile + x / G * R::kRow + x % G * 16) = codes[i];
        }
    };

    int chunk = from + wave * kChunk;
    if (chunk < to) {
        find(chunk);
        load_keys(chunk);
    }
    for (; chunk < to; chunk += kStep) {
        const uint64_t now = live;
        store(now, false);
        load(vbase, value_at);
        find(chunk + kStep);

        f32x4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int row = slot_of(t, col), mine = slot_of(t, quarter * 4);
            f32x4 side{};
#pragma unroll
            for (int f = 0; f < MF; ++f) side = T::mfma16(*reinterpret_cast<const Frag *>(meta + row * R::kMetaRow + f * 16), qs[f], side);
            f32x4 x[G];
#pragma unroll
            for (int g = 0; g < G; ++g)
                x[g] = T::mfma16(widen(*reinterpret_cast<const uint32_t *>(tile + row * R::kRow + g * kGroupBytes + quarter * 4)), q[g], f32x4{});
            s[t] = side * back;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const f32x4 step = *reinterpret_cast<const f32x4 *>(steps + g * kChunk + mine);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[t][i] = __builtin_fmaf(step[i], x[g][i], s[t][i]);
            }
        }
        if (now != ~0ull) {
            const uint64_t there[2] = {now >> (quarter * 4), now >> (quarter * 4 ^ 8)};      // of even and of odd products
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!(there[t & 1] >> (t * 16 + i) & 1)) s[t][i] = -inf;
        }
        if (a.scores && col < heads) {
            float *sp = a.scores + ((int64_t)seq * a.q_heads + head0 + col) * a.scores_stride + chunk;
#pragma unroll
            for (int t = 0; t < 4; ++t) *reinterpret_cast<f32x4 *>(sp + slot_of(t, quarter * 4)) = s[t];
        }
        float top = s[0][0];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][i]);
        top = max_halves(max_quarters(top));
        if (__any(top > m)) {
            const float next = fmaxf(m, top);
            const float keep = m == -inf ? 0.f : exp2_fast((m - next) * c);
            l *= keep;
            z *= keep;
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] *= keep;
            m = next;
            ref = m == -inf ? 0.f : m;
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[t][i] = exp2_fast((s[t][i] - ref) * c);
                l += s[t][i];
            }
        }

        store(now, true);
        if (chunk + kStep < to) load_keys(chunk + kStep);
        const uint8_t *transposed = tile + slot_of(col >> 2, quarter * 4 + (col & 3)) * R::kRow;
        constexpr uint32_t minus = kHalf ? 0xc1bcc1bcu : 0xcde0cde0u;     // -47/2
        const Frag less = Frag{minus, minus, minus, minus};
#pragma unroll
        for (int g = 0; g < G; ++g) {
            Frag p[kParts][2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const f32x4 u = s[y * 2] * *reinterpret_cast<const f32x4 *>(steps + g * kChunk + slot_of(y * 2, quarter * 4));
                const f32x4 v = s[y * 2 + 1] * *reinterpret_cast<const f32x4 *>(steps + g * kChunk + slot_of(y * 2 + 1, quarter * 4));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[0][y][i] = P::pack(u[i], v[i]);
                    if constexpr (kParts == 2) p[1][y][i] = P::pack(u[i] - low<P>(p[0][y][i]), v[i] - high<P>(p[0][y][i]));
                }
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const u32x2 x = read_codes(transposed + g * kGroupBytes + half * 8);
                f32x4 o = acc[g * 2 + half];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const Frag code = widen_p(x[y]);
#pragma unroll
                    for (int n = 0; n < kParts; ++n) {
                        o = P::mfma16(less, p[n][y], o);
                        o = P::mfma16(code, p[n][y], o);
                    }
                }
                acc[g * 2 + half] = o;
            }
        }
        // the centres, last: mixed with the products above their weights cost registers (heads of 128 in bfloat16 spilled 20)
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const u32x2 x = read_numbers(meta + slot_of(t, quarter * 4 + (col >> 2)) * R::kMetaRow + (col & 3) * 8);
            if constexpr (kHalf) {
#pragma unroll
                for (int i = 0; i < 4; ++i) z = mfma_f32(i % 2 ? high<T>(x[i / 2]) : low<T>(x[i / 2]), s[t][i], z);
            } else {
                const u32x2 p = {T::pack(s[t][0], s[t][1]), T::pack(s[t][2], s[t][3])};
                z = T::mfma16(Frag{x[0], x[1], x[0], x[1]},
                              Frag{p[0], p[1], T::pack(s[t][0] - low<T>(p[0]), s[t][1] - high<T>(p[0])),
                                   T::pack(s[t][2] - low<T>(p[1]), s[t][3] - high<T>(p[1]))}, z);
            }
        }
    }

    // the block's waves joined: lane's column is a head, its registers dims quarter * 4 + i (of z: a record's numbers)
    l = sum_halves(sum_quarters(l));
    if (quarter == 0) {
        stat[wave][0][col] = m;
        stat[wave][1][col] = l;
    }
    *reinterpret_cast<f32x4 *>(&sums[wave][col][quarter * 4]) = z;
    __syncthreads();
    float *mine = reinterpret_cast<float *>(tile);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
        const float centre = sums[wave][col][G + d / 2];
        f32x4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (kHalf ? acc[d][i] : __builtin_amdgcn_ldexpf(acc[d][i], -shift)) + centre;
        *reinterpret_cast<f32x4 *>(mine + col * (DIM + 4) + d * 16 + quarter * 4) = x;
    }
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

template <class T>
void decode4_of(const DecodeArgs &a, uint32_t blocks, hipStream_t stream) {
    const dim3 grid(blocks), block(64 * kWaves);
    switch (record_groups(a.dim)) {
    case 1: k_attn_decode4<T, 1><<<grid, block, 0, stream>>>(a); break;
    case 2: k_attn_decode4<T, 2><<<grid, block, 0, stream>>>(a); break;
    case 3: k_attn_decode4<T, 3><<<grid, block, 0, stream>>>(a); break;
    case 4: k_attn_decode4<T, 4><<<grid, block, 0, stream>>>(a); break;
    case 5: k_attn_decode4<T, 5><<<grid, block, 0, stream>>>(a); break;
    case 6: k_attn_decode4<T, 6><<<grid, block, 0, stream>>>(a); break;
    case 7: k_attn_decode4<T, 7><<<grid, block, 0, stream>>>(a); break;
    default: k_attn_decode4<T, 8><<<grid, block, 0, stream>>>(a); break;
    }
}

uint64_t up256(uint64_t x) { return (x + 255) / 256 * 256; }
uint32_t scores_stride(uint32_t max_len) { return (max_len + 63) / 64 * 64; }

constexpr uint32_t kMinSplit = kWaves * kChunk;      // a chunk for every wave
constexpr uint32_t kManySplit = 768;                 // slots per split, where sequences are many

}  // namespace

DecodePlan plan_decode4(uint32_t n_seqs, uint32_t q_heads, uint32_t kv_heads, uint32_t dim, uint32_t max_len, bool weights) {
    DecodePlan p{};
    p.head_blocks = (q_heads / kv_heads + 15) / 16;
    // a single sequence: about 512 blocks (131,071 slots of 8 heads of 128: 46.3 us a call, with 768 blocks 47.5, with 1,536
    // 52.6). Several, whose lengths differ: up to 1,024 blocks, and more of 768 slots (64 sequences of
    // up to 8,192 slots: 112.6 us a call, of 512 slots 114.3, of 1,536 119.2, of 2,048 117.6).
    const uint64_t rows = std::max<uint64_t>((uint64_t)n_seqs * kv_heads * p.head_blocks, 1), len = std::max<uint64_t>(max_len, 1);
    uint64_t t = n_seqs > 1 ? std::min<uint64_t>((len * rows + 1023) / 1024, kManySplit) : (len * rows + 511) / 512;
    t = std::max<uint64_t>(t, (len + kMaxSplits - 1) / kMaxSplits);
    t = (std::min(t, len) + kMinSplit - 1) / kMinSplit * kMinSplit;
    p.split_tokens = (uint32_t)t;
    p.splits = (uint32_t)((len + t - 1) / t);
    const uint64_t parts = (uint64_t)n_seqs * q_heads * p.splits;
    p.stats_off = 0;
    p.out_off = up256(parts * 8);
    p.scores_off = p.out_off + (p.splits > 1 ? up256(parts * dim * 4) : 0);
    p.bytes = p.scores_off + (weights ? up256((uint64_t)n_seqs * q_heads * scores_stride(max_len) * 4) : 0);
    return p;
}

// What plan_decode4 needs at most for up to n_seqs sequences of up to max_len slots: by its rule a sequence has a split for
// every kMinSplit slots at most, and no more than both kManySplit slots each and 1,024 blocks among all sequences
// (each rounded up) come to; this grows with both sizes.
uint64_t decode4_workspace(uint32_t n_seqs, uint32_t q_heads, uint32_t kv_heads, uint32_t dim, uint32_t max_len, bool weights) {
    const uint64_t n = n_seqs, len = std::max<uint64_t>(max_len, 1), blocks = (uint64_t)kv_heads * ((q_heads / kv_heads + 15) / 16);
    const uint64_t splits = std::min(n * std::min<uint64_t>((len + kMinSplit - 1) / kMinSplit, kMaxSplits),
                                     std::max((1024 + blocks - 1) / blocks + n, n * ((len + kManySplit - 1) / kManySplit)));
    return up256(splits * q_heads * 8) + (len > kMinSplit ? up256(splits * q_heads * dim * 4) : 0) +
           (weights ? up256(n * q_heads * scores_stride(max_len) * 4) : 0);
}

hipError_t launch_decode4(const Shape &s, const Rows &q, const Pages &pg, const int32_t *lens, uint32_t n_seqs,
                          uint32_t max_len, const Rows &out, float *lse, float *weights, uint64_t weights_stride,
                          const DecodePlan &plan, uint8_t *workspace, hipStream_t stream) {
    if (n_seqs == 0) return hipSuccess;
    const uint64_t blocks = (uint64_t)n_seqs * plan.splits * s.kv_heads * plan.head_blocks;
    DecodeArgs a{q, out, pg, lens, lse, weights, weights_stride, (float *)(workspace + plan.stats_off),
                 (float *)(workspace + plan.out_off), weights ? (float *)(workspace + plan.scores_off) : nullptr,
                 scores_stride(max_len), n_seqs, s.q_heads, s.kv_heads, s.group, plan.head_blocks, s.dim, max_len,
                 plan.split_tokens, plan.splits, s.scale, s.scale_log2};
    if (blocks > kMaxGrid || decode_join_blocks(a) > kMaxGrid) return hipErrorInvalidConfiguration;
    if (s.f16) decode4_of<F16>(a, (uint32_t)blocks, stream);
    else decode4_of<Bf16>(a, (uint32_t)blocks, stream);
    launch_decode_join(a, s.f16, stream);
    return hipGetLastError();
}

}  // namespace attn
}  // namespace ibp
