// New rows of keys and values into a paged cache, keys (and queries) turned by their positions on the way; and the rows
// of a 4-bit cache back to 16 bits.
//
//   (x, y) -> (x c - y s, x s + y c) for the pairs of a head's first values, c and s of the row's position,
//   every product and sum rounded to 32 bits, the results once to the type (or held in 4 bits):
//   per 32 values  centre = type((lo + hi) / 2),  step = type(2/15 max(hi - centre, centre - lo)),
//   code = round((x - centre) / step + 7.5) clamped to 0 .. 15,  value = centre + (code - 7.5) step.
#include "ibp_attn_wave.hpp"
#include "ibp_kv_cache.hpp"

#include <algorithm>

// What is held in 4 bits is defined operation by operation: nothing is fused but where it says so.
#pragma clang fp contract(off)

namespace ibp {
namespace attn {

namespace {

using namespace dev;

constexpr int kThreads = 256;

// The sequence of a packed row and how many rows of it come from this one on (this one among them); false: in none.
// Every wave looks for itself, 64 starts at a time: of ascending ones the last that is not above the row.
__device__ __forceinline__ bool find_row(const int32_t *starts, uint32_t n_seqs, uint32_t rows, uint32_t row, uint32_t &seq, int &back) {
    if (!starts) {
        seq = row;
        back = 1;
        return true;
    }
    uint32_t lo = 0, hi = n_seqs;
    const int lane = threadIdx.x & 63;
    bool any = false;
    while (hi - lo > 1 || !any) {
        const uint32_t step = (hi - lo + 63) / 64, at = lo + lane * step;
        const uint64_t below = __ballot(at < hi && starts[min(at, hi - 1)] <= (int)row);
        if (!below) return false;
        lo += (63 - __builtin_clzll(below)) * step;
        hi = min(lo + step, hi);
        any = true;
    }
    seq = (uint32_t)uniform((int)lo);
    back = uniform(min(starts[seq + 1], (int)rows)) - (int)row;
    return back > 0;
}

// The place of a slot in a pool of pages: false where its page is not there.
struct Place {
    int64_t page;
    uint32_t row;
};
__device__ __forceinline__ bool find_slot(const Pages &pg, uint32_t seq, int64_t slot, Place &p) {
    if (slot < 0 || slot >= (int64_t)pg.table_stride * pg.page_tokens || slot >= 0x7fffffff) return false;
    const uint32_t s = (uint32_t)slot, i = pg.page_magic ? __umulhi(s, pg.page_magic) >> pg.page_shift : s >> pg.page_shift;
    const int32_t page = pg.table[(int64_t)seq * pg.table_stride + i];
    p.page = page;
    p.row = s - i * pg.page_tokens;
    return (uint32_t)page < pg.n_pages;
}

__device__ __forceinline__ uint8_t *at_slot(const Pool &p, const Place &x, uint32_t head) {
    return (uint8_t *)p.data + (x.page * p.page + (int64_t)head * p.head + (int64_t)x.row * p.token) * 2;
}

template <class T>
__device__ __forceinline__ f32x4 widen(u32x2 x) {
    return f32x4{T::value((uint16_t)x[0]), T::value((uint16_t)(x[0] >> 16)), T::value((uint16_t)x[1]), T::value((uint16_t)(x[1] >> 16))};
}
template <class T>
__device__ __forceinline__ u32x2 narrow(f32x4 x) {
    return u32x2{T::pack(x[0], x[1]), T::pack(x[2], x[3])};
}

// x a + y b, each product and the sum rounded.
__device__ __forceinline__ float turned(float x, float a, float y, float b) { return x * a + y * b; }

// A head's quad `to` (four values from there on) after turning.
template <class T>
__device__ __forceinline__ f32x4 turned_quad(const Append &a, const uint8_t *head, const float *angles, uint32_t to) {
    const f32x4 x = widen<T>(*reinterpret_cast<const u32x2 *>(head + to * 2));
    if (to >= a.turned) return x;
    const uint32_t half = a.turned / 2;
    f32x4 o;
    if (a.halves) {
        const bool second = to >= half;
        const uint32_t pair = second ? to - half : to;
        const f32x4 y = widen<T>(*reinterpret_cast<const u32x2 *>(head + (second ? pair : to + half) * 2));
        const f32x4 *cs = reinterpret_cast<const f32x4 *>(angles + pair * 2);
        const f32x4 c0 = cs[0], c1 = cs[1];
        const f32x4 c = {c0[0], c0[2], c1[0], c1[2]}, s = {c0[1], c0[3], c1[1], c1[3]};
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = second ? turned(y[i], s[i], x[i], c[i]) : turned(x[i], c[i], -y[i], s[i]);
    } else {
        const f32x4 cs = *reinterpret_cast<const f32x4 *>(angles + to);
        o = f32x4{turned(x[0], cs[0], -x[1], cs[1]), turned(x[0], cs[1], x[1], cs[0]),
                  turned(x[2], cs[2], -x[3], cs[3]), turned(x[2], cs[3], x[3], cs[2])};
    }
    return o;
}

// Eight values of a head, in the lanes of its group of 32 (four in a row), as their dword of codes; step and centre.
template <class T>
__device__ __forceinline__ uint32_t codes_of(const float *x, uint32_t there, uint16_t &step16, uint16_t &centre16) {
    float lo = __builtin_inff(), hi = -__builtin_inff();
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < (int)there) {
            lo = fminf(lo, x[i]);
            hi = fmaxf(hi, x[i]);
            bad |= !(fabsf(x[i]) < __builtin_inff());
        }
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
        lo = fminf(lo, __shfl_xor(lo, d));
        hi = fmaxf(hi, __shfl_xor(hi, d));
        bad |= __shfl_xor((int)bad, d) != 0;
    }
    centre16 = (uint16_t)T::pack(lo * 0.5f + hi * 0.5f, 0.f);
    const float centre = T::value(centre16);
    step16 = (uint16_t)T::pack(fmaxf(hi - centre, centre - lo) * (2.f / 15.f), 0.f);
    const float step = T::value(step16);
    if (bad || !(fabsf(centre) < __builtin_inff()) || !(step < __builtin_inff())) {
        centre16 = step16 = (uint16_t)(T::kExp | (T::kExp >> 1 & ~T::kExp));      // (quiet NaN)
        return 0;
    }
    const float inverse = step >= 0x1p-126f ? 1.f / step : 0.f;
    uint32_t code = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = rintf((x[i] - centre) * inverse + 7.5f);
        code |= (uint32_t)fminf(fmaxf(y, 0.f), 15.f) << (4 * i);
    }
    return there < 8 ? code & (there ? 0xffffffffu >> (32 - 4 * there) : 0u) : code;
}

// A block per row; a thread takes eight values of a head at a time, `octs` (a power of two, at least
// the head's) threads per head.
template <class T, bool FOUR>
__global__ __launch_bounds__(kThreads) void k_kv_append(Append a, uint32_t octs_log2) {
    const uint32_t row = blockIdx.x;
    uint32_t seq;
    int back;
    if (!find_row(a.starts, a.n_seqs, a.rows, row, seq, back)) return;
    const int64_t slot = (int64_t)a.lens[seq] - back, position = (int64_t)a.next[seq] - back;
    const float *angles = a.rotation + min(max(position, (int64_t)0), (int64_t)a.positions - 1) * a.turned;
    Place place;
    const bool there = find_slot(a.pg, seq, slot, place);
    const uint32_t heads = a.q_heads + 2 * a.kv_heads, octs = 1u << octs_log2, half = a.turned / 2;
    for (uint32_t item = threadIdx.x; item < heads << octs_log2; item += kThreads) {
        const uint32_t h = item >> octs_log2, oct = item & (octs - 1), d = oct * 8;
        const bool is_q = h < a.q_heads, is_k = !is_q && h < a.q_heads + a.kv_heads;
        const uint32_t head = is_q ? h : is_k ? h - a.q_heads : h - a.q_heads - a.kv_heads;
        const Rows &in = is_q ? a.q : is_k ? a.k : a.v;
        const uint8_t *from = (const uint8_t *)in.data + ((int64_t)row * in.row + (int64_t)head * in.head) * 2;
        if (!is_q && !there) continue;
        if (FOUR && !is_q) {
            const uint32_t groups = record_groups(a.dim);
            if (d >= groups * kGroupValues) continue;
            const uint32_t have = min(max((int)a.dim - (int)d, 0), 8);
            float x[8] = {};
            if (have) {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const f32x4 v = is_k ? turned_quad<T>(a, from, angles, d + 4 * y) : widen<T>(*reinterpret_cast<const u32x2 *>(from + (d + 4 * y) * 2));
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[4 * y + i] = v[i];
                }
            }
            uint16_t step, centre;
            const uint32_t code = codes_of<T>(x, have, step, centre);
            uint8_t *to = at_slot(is_k ? a.pg.k : a.pg.v, place, head);
            *reinterpret_cast<uint32_t *>(to + oct * 4) = code;
            if ((oct & 3) == 0) {
                uint8_t *meta = to + groups * kGroupBytes + oct / 4 * 2;
                *reinterpret_cast<uint16_t *>(meta) = step;
                *reinterpret_cast<uint16_t *>(meta + groups * 2) = centre;
            }
            continue;
        }
        if (d >= a.dim) continue;
        uint8_t *to = is_q ? (uint8_t *)a.q_out.data + ((int64_t)row * a.q_out.row + (int64_t)head * a.q_out.head) * 2
                           : at_slot(is_k ? a.pg.k : a.pg.v, place, head);
        if (h >= a.q_heads + a.kv_heads || d >= a.turned) {
            *reinterpret_cast<Frag *>(to + d * 2) = *reinterpret_cast<const Frag *>(from + d * 2);
            continue;
        }
        // both quads of four pairs: nothing that another thread writes is read, so that queries may be turned in place
        const uint32_t q0 = a.halves ? oct * 4 : d, q1 = a.halves ? half + oct * 4 : d + 4;
        const f32x4 x = turned_quad<T>(a, from, angles, q0), y = turned_quad<T>(a, from, angles, q1);
        *reinterpret_cast<u32x2 *>(to + q0 * 2) = narrow<T>(x);
        *reinterpret_cast<u32x2 *>(to + q1 * 2) = narrow<T>(y);
    }
    if (there && a.weights && slot < (int64_t)a.stride)
        for (uint32_t h = threadIdx.x; h < a.kv_heads; h += kThreads) {
            a.weights[((int64_t)seq * a.kv_heads + h) * a.stride + slot] = 0.f;
        }
    if (there && a.places && slot < (int64_t)a.stride)
        for (uint32_t h = threadIdx.x; h < a.kv_heads; h += kThreads)
            a.places[((int64_t)seq * a.kv_heads + h) * a.stride + slot] = (int32_t)position;
}

// A block per row, threads as above.
template <class T>
__global__ __launch_bounds__(kThreads) void k_kv4_read(Read4 a, uint32_t octs_log2) {
    const uint32_t row = blockIdx.x;
    uint32_t seq;
    int back;
    if (!find_row(a.starts, a.n_seqs, a.rows, row, seq, back)) return;
    const int64_t slot = (a.first ? (int64_t)a.first[seq] : 0) + (a.starts ? (int64_t)row - a.starts[seq] : 0);
    Place place;
    if (slot >= a.lens[seq] || !find_slot(a.pg, seq, slot, place)) return;
    const uint32_t octs = 1u << octs_log2, groups = record_groups(a.dim);
    for (uint32_t item = threadIdx.x; item < 2 * a.kv_heads << octs_log2; item += kThreads) {
        const uint32_t h = item >> octs_log2, oct = item & (octs - 1), d = oct * 8;
        if (d >= a.dim) continue;
        const bool is_k = h < a.kv_heads;
        const uint32_t head = is_k ? h : h - a.kv_heads;
        const uint8_t *from = at_slot(is_k ? a.pg.k : a.pg.v, place, head), *meta = from + groups * kGroupBytes + oct / 4 * 2;
        const Rows &out = is_k ? a.k : a.v;
        const uint32_t code = *reinterpret_cast<const uint32_t *>(from + oct * 4);
        const float step = T::value(*reinterpret_cast<const uint16_t *>(meta)), centre = T::value(*reinterpret_cast<const uint16_t *>(meta + groups * 2));
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf((float)(code >> 4 * i & 15) - 7.5f, step, centre);
        *reinterpret_cast<Frag *>((uint8_t *)out.data + ((int64_t)row * out.row + (int64_t)head * out.head + d) * 2) =
            Frag{T::pack(x[0], x[1]), T::pack(x[2], x[3]), T::pack(x[4], x[5]), T::pack(x[6], x[7])};
    }
}

uint32_t log2_up(uint32_t x) {
    uint32_t n = 0;
    while ((1u << n) < x) ++n;
    return n;
}

}  // namespace

hipError_t launch_append(const Append &a, hipStream_t stream) {
    if (a.rows == 0 || a.n_seqs == 0) return hipSuccess;
    if (a.rows > kMaxGrid) return hipErrorInvalidConfiguration;
    const uint32_t octs = log2_up(a.four ? record_groups(a.dim) * 4 : a.dim / 8);
    const dim3 grid(a.rows), block(kThreads);
    if (a.f16) {
        if (a.four) k_kv_append<F16, true><<<grid, block, 0, stream>>>(a, octs);
        else k_kv_append<F16, false><<<grid, block, 0, stream>>>(a, octs);
    } else {
        if (a.four) k_kv_append<Bf16, true><<<grid, block, 0, stream>>>(a, octs);
        else k_kv_append<Bf16, false><<<grid, block, 0, stream>>>(a, octs);
    }
    return hipGetLastError();
}

hipError_t launch_read4(const Read4 &r, hipStream_t stream) {
    if (r.rows == 0 || r.n_seqs == 0) return hipSuccess;
    if (r.rows > kMaxGrid) return hipErrorInvalidConfiguration;
    const uint32_t octs = log2_up(r.dim / 8);
    if (r.f16) k_kv4_read<F16><<<dim3(r.rows), dim3(kThreads), 0, stream>>>(r, octs);
    else k_kv4_read<Bf16><<<dim3(r.rows), dim3(kThreads), 0, stream>>>(r, octs);
    return hipGetLastError();
}

}  // namespace attn
}  // namespace ibp
