// New rows of keys and values into a paged cache, keys (and queries) turned by their positions on the way; and the rows
// of a 4-bit cache back to 16 bits.
//
//   (x, y) -> (x c - y s, x s + y c) for the pairs of a head's first values, c and s of the row's position,
//   every product and sum rounded to 32 bits, the results once to the type (or held in 4 bits):
//   per 32 values  centre = type((lo + hi) / 2),  step = type(2/15 max(hi - centre, centre - lo)),
//   code = round((x - centre) / step + 7.5) clamped to 0 .. 15,  value = centre + (code - 7.5) step.
//
// Large calls are bound by HBM: 8,192 rows of 32/8 heads of 128 in bfloat16 39.5 us into 16-bit pages (206 MB, 5.2 TB/s, as a large
// copy) and 45 into records (182 MB, 4.0 TB/s, with the conversions between the loads and the stores), 32,768 slots of 8 heads of
// 128 read back 29.5 us (176 MB, 6.0 TB/s: 134 of them written around the caches). Small ones by the look-ups, each of
// which waits for the one before (the row's sequence, its length, its page): one row 2.7 us, 64 rows 3.6, into records 4.6,
// of which a launch is about 2.
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
    if (pg.n_pages == 0 || slot < 0 || slot >= (int64_t)pg.table_stride * pg.page_tokens || slot >= 0x7fffffff) return false;
    const uint32_t s = (uint32_t)slot, i = pg.page_magic ? __umulhi(s, pg.page_magic) >> pg.page_shift : s >> pg.page_shift;
    const int32_t page = pg.table[(int64_t)seq * pg.table_stride + i];
    p.page = page;
    p.row = s - i * pg.page_tokens;
    return (uint32_t)page < pg.n_pages;
}

// Where the first head's row is, the same for a whole wave, and how far apart the heads are, in bytes: what a lane's own head needs beside
// is one product.
struct Heads {
    uint8_t *first;
    int64_t step;
};
__device__ __forceinline__ Heads heads_at(const Pool &p, const Place &x) {
    return Heads{(uint8_t *)p.data + (x.page * p.page + (int64_t)x.row * p.token) * 2, p.head * 2};
}
__device__ __forceinline__ Heads heads_at(const Rows &r, uint32_t row) {
    return Heads{(uint8_t *)r.data + (int64_t)row * r.row * 2, r.head * 2};
}
__device__ __forceinline__ uint8_t *head_of(const Heads &h, uint32_t head) { return h.first + (int64_t)head * h.step; }
__device__ __forceinline__ Heads either(bool first, const Heads &a, const Heads &b) {
    return Heads{first ? a.first : b.first, first ? a.step : b.step};
}

template <class T>
__device__ __forceinline__ f32x4 widen(u32x2 x) {
    return f32x4{T::value((uint16_t)x[0]), T::value((uint16_t)(x[0] >> 16)), T::value((uint16_t)x[1]), T::value((uint16_t)(x[1] >> 16))};
}
// A number that is rounded to 32 bits before it is to 16: the instructions that do both at once for float16 round once.
template <class T>
__device__ __forceinline__ float rounded(float x) {
    if constexpr (T::kExp == F16::kExp) asm("" : "+v"(x));
    return x;
}
template <class T>
__device__ __forceinline__ uint32_t narrow(float x, float y) {
    return T::pack(rounded<T>(x), rounded<T>(y));
}
template <class T>
__device__ __forceinline__ u32x2 narrow(f32x4 x) {
    return u32x2{narrow<T>(x[0], x[1]), narrow<T>(x[2], x[3])};
}

// x a + y b, each product and the sum rounded.
__device__ __forceinline__ float turned(float x, float a, float y, float b) { return x * a + y * b; }

// Cosines and sines of four pairs.
struct Angles {
    f32x4 c, s;
};
__device__ __forceinline__ Angles angles_at(const float *p) {
    const f32x4 x = *reinterpret_cast<const f32x4 *>(p), y = *reinterpret_cast<const f32x4 *>(p + 4);
    return Angles{f32x4{x[0], x[2], y[0], y[2]}, f32x4{x[1], x[3], y[1], y[3]}};
}
__device__ __forceinline__ f32x4 first_of(f32x4 x, f32x4 y, const Angles &a) {
    return f32x4{turned(x[0], a.c[0], -y[0], a.s[0]), turned(x[1], a.c[1], -y[1], a.s[1]), turned(x[2], a.c[2], -y[2], a.s[2]),
                 turned(x[3], a.c[3], -y[3], a.s[3])};
}
__device__ __forceinline__ f32x4 second_of(f32x4 x, f32x4 y, const Angles &a) {
    return f32x4{turned(x[0], a.s[0], y[0], a.c[0]), turned(x[1], a.s[1], y[1], a.c[1]), turned(x[2], a.s[2], y[2], a.c[2]),
                 turned(x[3], a.s[3], y[3], a.c[3])};
}
// Eight values, four pairs of neighbours.
__device__ __forceinline__ void turn_neighbours(f32x4 &u, f32x4 &v, const Angles &a) {
    const f32x4 x = {u[0], u[2], v[0], v[2]}, y = {u[1], u[3], v[1], v[3]};
    const f32x4 p = first_of(x, y, a), q = second_of(x, y, a);
    u = f32x4{p[0], q[0], p[1], q[1]};
    v = f32x4{p[2], q[2], p[3], q[3]};
}

// x of lane ^ D, of the four that a lane is one of.
template <int D>
__device__ __forceinline__ float beside(float x) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), D == 1 ? 0xb1 : 0x4e, 0xf, 0xf, true));
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
    lo = fminf(lo, beside<1>(lo));
    hi = fmaxf(hi, beside<1>(hi));
    lo = fminf(lo, beside<2>(lo));
    hi = fmaxf(hi, beside<2>(hi));
    bad = (__ballot(bad) >> (threadIdx.x & 60) & 15) != 0;
    centre16 = (uint16_t)narrow<T>(lo * 0.5f + hi * 0.5f, 0.f);
    const float centre = T::value(centre16);
    step16 = (uint16_t)narrow<T>(fmaxf(hi - centre, centre - lo) * (2.f / 15.f), 0.f);
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

// A store of a large call (N items a lane): around the caches, which its rows would leave unread (32,768 slots read back 29 us instead
// of 38, 8,192 rows appended 47 instead of 49 when that was chosen). What a small call writes is read next, and stays.
template <int N, class X>
__device__ __forceinline__ void put(uint8_t *to, X x) {
    if constexpr (N == 1) *reinterpret_cast<X *>(to) = x;
    else __builtin_nontemporal_store(x, reinterpret_cast<X *>(to));
}

// What a row's wave needs of its sequence. Asked for behind the loads of the row's values, which need none of it.
struct Where {
    uint32_t seq;
    int64_t slot, position;
    Place place;
    bool there;
    const float *angles;
};
__device__ __forceinline__ bool find_where(const Append &a, uint32_t row, Where &w) {
    int back;
    if (!find_row(a.starts, a.n_seqs, a.rows, row, w.seq, back)) return false;
    w.slot = (int64_t)a.lens[w.seq] - back;
    w.position = (int64_t)a.next[w.seq] - back;
    w.angles = a.rotation + min(max(w.position, (int64_t)0), (int64_t)a.positions - 1) * a.turned;
    w.there = find_slot(a.pg, w.seq, w.slot, w.place);
    return true;
}

// Items, of eight values each, that a lane has on their way together: four fill the chip's memory system (8,192 rows appended 39 us,
// with two 41.5, with eight 40; into records 45, with two 53). In calls of too few rows for that one each is sooner done
// (64 rows 3.5 us instead of 5.5). Four into records keep 12 to 14 scalar registers in vector ones' lanes.
constexpr int kMany = 4;
constexpr uint64_t kFewWaves = 2048;     // (of so many items)

// Waves are shared out as `parts` per row: each takes 64 N items of its heads, first of those that stay 16 bits wide (`wide`
// parts: queries, and without FOUR keys and values), then of those that are held in 4. A lane's items are the same eight
// values of several heads, `octs` (a power of two, at least the head's) lanes per head, so that it needs the angles once.
template <class T, bool FOUR, int N>
__global__ __launch_bounds__(kThreads) void k_kv_append(Append a, uint32_t wide_log2, uint32_t four_log2, uint32_t wide, uint32_t parts) {
    const uint32_t wave = (uint32_t)uniform((int)(blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)));
    const uint32_t row = wave / parts, part = wave - row * parts, lane = threadIdx.x & 63;
    if (row >= a.rows) return;
    const uint32_t half = a.turned / 2;
    Where w;
    if (part < wide) {
        const uint32_t heads = a.q_heads + (FOUR ? 0 : 2 * a.kv_heads), oct = lane & ((1u << wide_log2) - 1), d = oct * 8;
        const uint32_t head0 = ((part * N * 64) + lane) >> wide_log2, head_step = 64u >> wide_log2;
        // both quads of four pairs, so that nothing that another lane writes is read: queries may be turned in place
        const bool turn = d < a.turned, apart = turn && a.halves;
        const uint32_t q0 = apart ? oct * 4 : d, q1 = apart ? half + oct * 4 : d + 4;
        const Heads in_q = heads_at(a.q, row), in_k = heads_at(a.k, row), in_v = heads_at(a.v, row);
        u32x2 x[N], y[N];
        auto in_heads = [&](int n, uint32_t &head, uint32_t &which) {
            const uint32_t h = head0 + n * head_step;
            which = h < a.q_heads ? 0 : h < a.q_heads + a.kv_heads ? 1 : 2;
            head = which == 0 ? h : which == 1 ? h - a.q_heads : h - a.q_heads - a.kv_heads;
            return h < heads && d < a.dim;
        };
#pragma unroll
        for (int n = 0; n < N; ++n) {
            uint32_t head, which;
            if (!in_heads(n, head, which)) continue;
            const bool mixed = which != 2;
            const uint8_t *from = head_of(either(which == 0, in_q, either(which == 1, in_k, in_v)), head);
            x[n] = *reinterpret_cast<const u32x2 *>(from + (mixed ? q0 : d) * 2);
            y[n] = *reinterpret_cast<const u32x2 *>(from + (mixed ? q1 : d + 4) * 2);
        }
        if (!find_where(a, row, w)) return;
        const Heads out_q = heads_at(a.q_out, row), out_k = heads_at(a.pg.k, w.place), out_v = heads_at(a.pg.v, w.place);
        Angles at{};
        if (turn) at = angles_at(w.angles + oct * 8);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            uint32_t head, which;
            if (!in_heads(n, head, which) || (which != 0 && !w.there)) continue;
            const bool mixed = which != 2;
            uint8_t *to = head_of(either(which == 0, out_q, either(which == 1, out_k, out_v)), head);
            if (mixed && turn) {
                f32x4 u = widen<T>(x[n]), v = widen<T>(y[n]);
                if (a.halves) {
                    const f32x4 p = first_of(u, v, at);
                    v = second_of(u, v, at);
                    u = p;
                } else {
                    turn_neighbours(u, v, at);
                }
                x[n] = narrow<T>(u);
                y[n] = narrow<T>(v);
            }
            put<N>(to + (mixed ? q0 : d) * 2, x[n]);
            put<N>(to + (mixed ? q1 : d + 4) * 2, y[n]);
        }
    } else if constexpr (FOUR) {
        const uint32_t groups = record_groups(a.dim), oct = lane & ((1u << four_log2) - 1), d = oct * 8;
        const uint32_t head0 = (((part - wide) * N * 64) + lane) >> four_log2, head_step = 64u >> four_log2;
        const uint32_t have = min(max((int)a.dim - (int)d, 0), 8);
        const bool turn = d < a.turned;
        // of pairs that are apart the other quads
        uint32_t other[2], pair[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t at = d + 4 * i;
            other[i] = at < half ? at + half : at - half;
            pair[i] = at < half ? at : at - half;
        }
        const Heads in_k = heads_at(a.k, row), in_v = heads_at(a.v, row);
        u32x2 x[N][2], y[N][2];
        auto in_heads = [&](int n, uint32_t &head, bool &is_k) {
            const uint32_t h = head0 + n * head_step;
            is_k = h < a.kv_heads;
            head = is_k ? h : h - a.kv_heads;
            return h < 2 * a.kv_heads && oct < groups * 4;
        };
#pragma unroll
        for (int n = 0; n < N; ++n) {
            uint32_t head;
            bool is_k;
            if (!in_heads(n, head, is_k) || !have) continue;
            const uint8_t *from = head_of(either(is_k, in_k, in_v), head);
#pragma unroll
            for (int i = 0; i < 2; ++i) x[n][i] = *reinterpret_cast<const u32x2 *>(from + (d + 4 * i) * 2);
            if (is_k && turn && a.halves) {
#pragma unroll
                for (int i = 0; i < 2; ++i) y[n][i] = *reinterpret_cast<const u32x2 *>(from + other[i] * 2);
            }
        }
        if (!find_where(a, row, w) || !w.there) return;
        const Heads out_k = heads_at(a.pg.k, w.place), out_v = heads_at(a.pg.v, w.place);
        Angles at[2]{};
        if (turn) {
            if (a.halves) {
#pragma unroll
                for (int i = 0; i < 2; ++i) at[i] = angles_at(w.angles + pair[i] * 2);
            } else {
                at[0] = angles_at(w.angles + d);
            }
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            uint32_t head;
            bool is_k;
            if (!in_heads(n, head, is_k)) continue;
            f32x4 u{}, v{};
            if (have) {
                u = widen<T>(x[n][0]);
                v = widen<T>(x[n][1]);
                if (is_k && turn) {
                    if (a.halves) {
                        const f32x4 p = widen<T>(y[n][0]), q = widen<T>(y[n][1]);
                        u = d < half ? first_of(u, p, at[0]) : second_of(p, u, at[0]);
                        v = d + 4 < half ? first_of(v, q, at[1]) : second_of(q, v, at[1]);
                    } else {
                        turn_neighbours(u, v, at[0]);
                    }
                }
            }
            const float z[8] = {u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
            uint16_t step, centre;
            const uint32_t code = codes_of<T>(z, have, step, centre);
            uint8_t *to = head_of(either(is_k, out_k, out_v), head);
            *reinterpret_cast<uint32_t *>(to + oct * 4) = code;
            if ((oct & 3) == 0) {
                uint8_t *meta = to + groups * kGroupBytes + oct / 4 * 2;
                *reinterpret_cast<uint16_t *>(meta) = step;
                *reinterpret_cast<uint16_t *>(meta + groups * 2) = centre;
            }
        }
    }
    if (part != parts - 1 || !w.there || w.slot >= (int64_t)a.stride) return;
    const int64_t at = (int64_t)w.seq * a.kv_heads * a.stride + w.slot;
    for (uint32_t h = lane; h < a.kv_heads; h += 64) {
        if (a.weights) a.weights[at + h * a.stride] = 0.f;
        if (a.places) a.places[at + h * a.stride] = (int32_t)w.position;
    }
}

// A step is rounded, so that the ends of a group that holds the type's largest number may lie beyond it (a float16 group of +-65504
// has a step of 8736 and ends at +-65520, which would round to infinity): they are held to it. (In a branch that hardly any group takes: 32,768 slots of 8 heads
// of 128 29.1 us a call, 29.4 with all values held.)
template <class T>
constexpr float kLargest = T::kExp == F16::kExp ? 65504.f : 0x1.fep127f;

// The same shares of a row; a lane's values are the same eight of several heads.
template <class T, int N>
__global__ __launch_bounds__(kThreads) void k_kv4_read(Read4 a, uint32_t octs_log2, uint32_t parts) {
    const uint32_t wave = (uint32_t)uniform((int)(blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)));
    const uint32_t row = wave / parts, part = wave - row * parts, lane = threadIdx.x & 63;
    if (row >= a.rows) return;
    uint32_t seq;
    int back;
    if (!find_row(a.starts, a.n_seqs, a.rows, row, seq, back)) return;
    const int64_t slot = (a.first ? (int64_t)a.first[seq] : 0) + (a.starts ? (int64_t)row - a.starts[seq] : 0);
    Place place;
    if (slot >= a.lens[seq] || !find_slot(a.pg, seq, slot, place)) return;
    const uint32_t groups = record_groups(a.dim), oct = lane & ((1u << octs_log2) - 1), d = oct * 8;
    const uint32_t head0 = ((part * N * 64) + lane) >> octs_log2, head_step = 64u >> octs_log2;
    if (d >= a.dim) return;
    const Heads in_k = heads_at(a.pg.k, place), in_v = heads_at(a.pg.v, place), out_k = heads_at(a.k, row), out_v = heads_at(a.v, row);
    uint32_t code[N];
    uint16_t step[N], centre[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const uint32_t h = min(head0 + n * head_step, 2 * a.kv_heads - 1);
        const bool is_k = h < a.kv_heads;
        const uint8_t *from = head_of(either(is_k, in_k, in_v), is_k ? h : h - a.kv_heads), *meta = from + groups * kGroupBytes + oct / 4 * 2;
        code[n] = *reinterpret_cast<const uint32_t *>(from + oct * 4);
        step[n] = *reinterpret_cast<const uint16_t *>(meta);
        centre[n] = *reinterpret_cast<const uint16_t *>(meta + groups * 2);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const uint32_t h = head0 + n * head_step;
        if (h >= 2 * a.kv_heads) return;
        const bool is_k = h < a.kv_heads;
        const float s = T::value(step[n]), c = T::value(centre[n]);
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf((float)(code[n] >> 4 * i & 15) - 7.5f, s, c);
        if (__builtin_fmaf(fabsf(s), 7.5f, fabsf(c)) > kLargest<T> && fabsf(s) < __builtin_inff() && fabsf(c) < __builtin_inff()) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_fmed3f(x[i], -kLargest<T>, kLargest<T>);
        }
        put<N>(head_of(either(is_k, out_k, out_v), is_k ? h : h - a.kv_heads) + d * 2,
               Frag{narrow<T>(x[0], x[1]), narrow<T>(x[2], x[3]), narrow<T>(x[4], x[5]), narrow<T>(x[6], x[7])});
    }
}

uint32_t log2_up(uint32_t x) {
    uint32_t n = 0;
    while ((1u << n) < x) ++n;
    return n;
}

// Waves of `items` items a lane that `heads` heads of 2^octs_log2 of them make.
uint64_t parts_of(uint64_t heads, uint32_t octs_log2, int items) { return ((heads << octs_log2) + 64 * items - 1) / (64 * items); }

// A row's parts times the rows, as blocks; 0: more than a launch has.
uint32_t blocks_of(uint64_t rows, uint64_t parts) {
    const uint64_t blocks = (rows * parts + kThreads / 64 - 1) / (kThreads / 64);
    return blocks > kMaxGrid || rows > kMaxGrid ? 0 : (uint32_t)blocks;
}

}  // namespace

hipError_t launch_append(const Append &a, hipStream_t stream) {
    if (a.rows == 0 || a.n_seqs == 0) return hipSuccess;
    const uint32_t wide_log2 = log2_up(a.dim / 8), four_log2 = log2_up(record_groups(a.dim) * 4);
    const uint64_t wide_heads = a.q_heads + (a.four ? 0ull : 2ull * a.kv_heads), four_heads = a.four ? 2ull * a.kv_heads : 0;
    auto launch = [&](auto kernel, int items) {
        const uint64_t wide = parts_of(wide_heads, wide_log2, items), parts = wide + parts_of(four_heads, four_log2, items);
        const uint32_t blocks = blocks_of(a.rows, parts);
        if (!blocks) return hipErrorInvalidConfiguration;
        kernel<<<dim3(blocks), dim3(kThreads), 0, stream>>>(a, wide_log2, four_log2, (uint32_t)wide, (uint32_t)parts);
        return hipGetLastError();
    };
    const bool many = a.rows * (parts_of(wide_heads, wide_log2, kMany) + parts_of(four_heads, four_log2, kMany)) >= kFewWaves;
    auto of_type = [&](auto type) {
        using T = decltype(type);
        if (many) return launch(a.four ? k_kv_append<T, true, kMany> : k_kv_append<T, false, kMany>, kMany);
        return launch(a.four ? k_kv_append<T, true, 1> : k_kv_append<T, false, 1>, 1);
    };
    return a.f16 ? of_type(F16{}) : of_type(Bf16{});
}

hipError_t launch_read4(const Read4 &r, hipStream_t stream) {
    if (r.rows == 0 || r.n_seqs == 0) return hipSuccess;
    const uint32_t octs = log2_up(r.dim / 8);
    auto launch = [&](auto kernel, int items) {
        const uint64_t parts = parts_of(2ull * r.kv_heads, octs, items);
        const uint32_t blocks = blocks_of(r.rows, parts);
        if (!blocks) return hipErrorInvalidConfiguration;
        kernel<<<dim3(blocks), dim3(kThreads), 0, stream>>>(r, octs, (uint32_t)parts);
        return hipGetLastError();
    };
    auto of_type = [&](auto type) {
        using T = decltype(type);
        if (r.rows * parts_of(2ull * r.kv_heads, octs, kMany) >= kFewWaves) return launch(k_kv4_read<T, kMany>, kMany);
        return launch(k_kv4_read<T, 1>, 1);
    };
    return r.f16 ? of_type(F16{}) : of_type(Bf16{});
}

}  // namespace attn
}  // namespace ibp
