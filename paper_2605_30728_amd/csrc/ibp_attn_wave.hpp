// Pieces that the attention kernels share: matrix fragments of the two 2-byte types, the LDS
// tile layout and its loads, exchange between a wave's lanes.
//
// Fragment layouts of the matrix instructions used (l = lane):
//   32x32x16  A: row l % 32, k = (l / 32) * 8 .. + 7     B: column l % 32, the same k
//             C: column l % 32, register i is row (i / 4) * 8 + (l / 32) * 4 + i % 4
//   16x16x32  A: row l % 16, k = (l / 16) * 8 .. + 7     B: column l % 16, the same k
//             C: column l % 16, register i is row (l / 16) * 4 + i
//   16x16x16  A and B: k = (l / 16) * 4 .. + 3, C the same
// The k of a product may be in any order as long as A and B agree on it: the kernels compute
// scores transposed (keys as rows), so that the registers of a C tile, rounded to 2 bytes, are
// the B fragment of the product with the values, whose A fragment takes its keys in that order.
#pragma once

#include <cstdint>

#include <hip/hip_runtime.h>

#include "ibp_wave.hpp"

namespace ibp {
namespace attn {
namespace dev {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

#define IBP_LDS(T) __attribute__((address_space(3))) T

// Eight 2-byte values in four registers.
using Frag = u32x4;

struct Bf16 {
    static constexpr uint32_t kExp = 0x7f80u;    // exponent bits: all set in infinities and NaN
    static constexpr int kLift = 0;
    static __device__ __forceinline__ float value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
    static __device__ __forceinline__ f32x16 mfma32(Frag a, Frag b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    }
    static __device__ __forceinline__ f32x4 mfma16(Frag a, Frag b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    }
    static __device__ __forceinline__ f32x4 mfma16(u32x2 a, u32x2 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, a), __builtin_bit_cast(s16x4, b), c, 0,
                                                         0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y) {   // round to nearest even
        const f32x2 v = {x, y};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
    }
    static __device__ __forceinline__ uint32_t pack_out(float x, float y) { return pack(x, y); }
};

struct F16 {
    static constexpr uint32_t kExp = 0x7c00u;
    // Softmax weights carry this power of two until their row is done. float16 has few exponents: a weight below 2^-14
    // loses bits and one below 2^-25 counts for nothing in the product with the values, while the sum of the
    // weights still has it, so that one key far above many others would take what those add up to. Its numbers above 1 are
    // free: lifted, a weight keeps its bits down to 2^-26 and is there down to 2^-37.
    static constexpr int kLift = 12;
    static __device__ __forceinline__ float value(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
    static __device__ __forceinline__ f32x16 mfma32(Frag a, Frag b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
    }
    static __device__ __forceinline__ f32x4 mfma16(Frag a, Frag b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
    }
    static __device__ __forceinline__ f32x4 mfma16(u32x2 a, u32x2 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4, a), __builtin_bit_cast(f16x4, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y) {
        const f32x2 v = {x, y};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
    }
    // An output is a mean of values: finite where they are, though its weights' rounding may take it past the largest.
    static __device__ __forceinline__ float in_range(float x) {
        return fabsf(x) < __builtin_inff() ? __builtin_amdgcn_fmed3f(x, -65504.f, 65504.f) : x;
    }
    static __device__ __forceinline__ uint32_t pack_out(float x, float y) { return pack(in_range(x), in_range(y)); }
};

// 2^x; a result below the normal range is 0.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// x of this lane and of lane ^ 32, combined.
__device__ __forceinline__ float max_halves(float x) {
    const u32x2 r = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
    const u32x2 r = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// The same with lane ^ 16.
__device__ __forceinline__ float max_quarters(float x) {
    const u32x2 r = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_quarters(float x) {
    const u32x2 r = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Rows of a head of DIM values in LDS, as 16-byte chunks whose places are permuted within the
// row so that the lanes of one read spread over all banks: `rows` for reads of one chunk of many
// consecutive rows (a fragment's own rows), `columns` for transposing reads (half a wave at a time
// 32 or 64 bytes of consecutive rows: WIDE 16 or 32 columns of eight or four of them). Rows are 128, 256
// or 512 bytes wide (96 values are padded to 256 bytes).
template <int DIM>
struct Tile {
    static constexpr int kRowBytes = DIM <= 64 ? 128 : DIM <= 128 ? 256 : 512;
    static constexpr int kChunks = kRowBytes / 16;
    static __device__ __forceinline__ int rows(int row) { return DIM <= 64 ? (row >> 1) & 7 : row & 15; }
    template <int WIDE>
    static __device__ __forceinline__ int columns(int row) {
        if (WIDE == 32) return DIM <= 64 ? ((row >> 1) & 1) << 2 : (row & 3) << 2;
        return DIM <= 64 ? ((row >> 1) & 3) << 1 : (row & 7) << 1;
    }
};

// Byte offset, in a tensor of `stride` bytes per row, that a lane loads for 16-byte chunk
// `slot` of a tile; out of every tile's range where the chunk holds no values of the head.
constexpr uint32_t kNowhere = 0x80000000u;
// ROWS: laid out as `rows`, else as 32 wide `columns`.
template <int DIM, bool ROWS>
__device__ __forceinline__ uint32_t tile_source(int slot, uint32_t stride, int dim) {
    const int row = slot / Tile<DIM>::kChunks;
    const int c = (slot % Tile<DIM>::kChunks) ^ (ROWS ? Tile<DIM>::rows(row) : Tile<DIM>::template columns<32>(row));
    return c * 8 < dim ? row * stride + c * 16 : kNowhere;
}

// A fragment's row of a `rows` tile: chunk c of row r.
template <int DIM>
__device__ __forceinline__ Frag read_rows(const uint8_t *tile, int row, int c) {
    return *reinterpret_cast<const Frag *>(tile + row * Tile<DIM>::kRowBytes + ((c ^ Tile<DIM>::rows(row)) << 4));
}

// Four rows of 16 values, transposed over 16 lanes: lane i of the 16 gets value i of the rows
// r0 .. r0 + 3, when it passes row r0 + i / 4 and column c0 + (i % 4) * 4 here.
template <int DIM, int WIDE>
__device__ __forceinline__ u32x2 read_columns(const uint8_t *tile, int row, int col) {
    const uint8_t *p = tile + row * Tile<DIM>::kRowBytes + (((col >> 3) ^ Tile<DIM>::template columns<WIDE>(row)) << 4) + (col & 7) * 2;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((IBP_LDS(s16x4) *)p));
}

// What a part with this reference and sum counts for beside the common reference; below zero: it
// saw no key at all (one that only saw NaN has a reference of -inf too, but a sum of NaN).
__device__ __forceinline__ float part_of(float ref, float sum, float top, float c) {
    return ref == -__builtin_inff() ? (sum == 0.f ? -1.f : 1.f) : exp2_fast((ref - top) * c);
}

using Rsrc = __amdgpu_buffer_rsrc_t;

// A descriptor of `bytes` bytes from p on: a load beyond them gives zeros.
__device__ __forceinline__ Rsrc descriptor(const void *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, 0x00020000);
}

// 16 bytes per lane straight into LDS at `to` + lane * 16.
__device__ __forceinline__ void load_to_lds(Rsrc r, uint8_t *to, uint32_t offset) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (IBP_LDS(void) *)to, 16, (int)offset, 0, 0, 0);
}

// Waits for this wave's loads into LDS and for its reads of LDS, then for the other waves.
__device__ __forceinline__ void tiles_loaded() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Whether any of a fragment's values is infinite or NaN.
template <class T>
__device__ __forceinline__ bool has_nonfinite(Frag f) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        bad |= (f[i] & T::kExp) == T::kExp || (f[i] & (T::kExp << 16)) == T::kExp << 16;
    return bad;
}

// Eight values from place d of a head on; zeros where the head (of `dim` values, a multiple of 8)
// ends before that. Nothing beyond the head is read. FULL: it never does.
template <bool FULL>
__device__ __forceinline__ Frag load_head(const uint8_t *head, int d, int dim) {
    if constexpr (FULL) return *reinterpret_cast<const Frag *>(head + d * 2);
    const Frag f = *reinterpret_cast<const Frag *>(head + min(d, dim - 8) * 2);
    const bool in = d < dim;
    return Frag{in ? f[0] : 0, in ? f[1] : 0, in ? f[2] : 0, in ? f[3] : 0};
}

// The sequence and tile of block `t`, where a packed sequence of n rows makes ceil(n / tile_rows)
// tiles, `rank` the tile's number. Of up to 64 sequences the blocks come in falling order of rank
// over all of them, so that where a tile's work grows with its rank the long ones are not left
// for the end; of more, sequence by sequence. Every wave works this out by itself. False: no such tile.
struct SeqTile {
    int q0, q_len, k0, k_len, rank, tiles;
};
__device__ __forceinline__ int clamp_row(int x, int rows) { return min(max(x, 0), rows); }

template <bool BY_KEYS>
__device__ __forceinline__ bool find_tile(const int32_t *q_starts, const int32_t *k_starts, int n_seqs, int q_rows,
                                          int k_rows, int tile_rows, int t, SeqTile &out) {
    const int lane = threadIdx.x & 63;
    for (int s0 = 0; s0 < n_seqs; s0 += 64) {
        const int s = s0 + lane;
        int q0 = 0, q1 = 0, k0 = 0, k1 = 0;
        if (s < n_seqs) {
            q0 = clamp_row(q_starts[s], q_rows);
            q1 = clamp_row(q_starts[s + 1], q_rows);
            k0 = clamp_row(k_starts[s], k_rows);
            k1 = clamp_row(k_starts[s + 1], k_rows);
        }
        const int n = max(BY_KEYS ? k1 - k0 : q1 - q0, 0);
        const int mine = (n + tile_rows - 1) / tile_rows;
        const int sum = (int)::ibp::dev::wave_incl_scan((uint32_t)mine), all = __builtin_amdgcn_readlane(sum, 63);
        if (t >= all) {
            t -= all;
            continue;
        }
        int at, rank;
        if (n_seqs > 64) {
            at = __builtin_ctzll(__ballot(sum > t));
            rank = __builtin_amdgcn_readlane(mine, at) - 1 - (t - __builtin_amdgcn_readlane(sum - mine, at));
        } else {
            // lane i counts the sequences that have a tile of rank top - i, then 64 ranks further down
            int top = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) top = max(top, __shfl_xor(top, d));
            int done = 0;
            for (int first = uniform(top) - 1;; first -= 64) {
                int have = 0;
                for (int i = 0; i < n_seqs; ++i) have += __builtin_amdgcn_readlane(mine, i) > max(first - lane, -1) && first >= lane;
                const int upto = done + (int)::ibp::dev::wave_incl_scan((uint32_t)have);
                const uint64_t past = __ballot(upto > t);
                if (past) {
                    const int i = __builtin_ctzll(past);
                    rank = first - i;
                    const int nth = t - __builtin_amdgcn_readlane(upto - have, i);
                    const uint64_t those = __ballot(mine > rank);
                    at = __builtin_ctzll(__ballot(mine > rank && __popcll(those & ((1ull << lane) - 1)) == nth));
                    break;
                }
                done = __builtin_amdgcn_readlane(upto, 63);
            }
        }
        out.rank = rank;
        out.tiles = __builtin_amdgcn_readlane(mine, at);
        out.q0 = __builtin_amdgcn_readlane(q0, at);
        out.q_len = __builtin_amdgcn_readlane(max(q1 - q0, 0), at);
        out.k0 = __builtin_amdgcn_readlane(k0, at);
        out.k_len = __builtin_amdgcn_readlane(max(k1 - k0, 0), at);
        return true;
    }
    return false;
}

}  // namespace dev
}  // namespace attn
}  // namespace ibp
