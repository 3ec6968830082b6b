// Device helpers of the attention over packed sequences (gfx950): tiles in LDS, and the two
// kinds of matrix product that its kernels are made of, for bf16 and fp32.
#pragma once

#include "prompt.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace a2t {
namespace prompt {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;

constexpr int kThreads = 256;
constexpr int kTile = 64;            // rows of a tile in LDS
constexpr float kLn2 = 0.693147180559945309417f;
constexpr float kLog2e = 1.44269504088896340736f;

struct bf16_t {
    uint16_t bits;
};

__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
    const bf16x2 v = {(__bf16)a, (__bf16)b};   // round to nearest even
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float swap_max(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float swap_sum(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// Sequence of block y of the launch, and the block's place among the sequence's.
template <int N>
__device__ __forceinline__ int sequence_of(const SeqTable<N>& t, int y, int* place) {
    if (N == 1) {
        *place = y;
        return 0;
    }
    const int lane = threadIdx.x & 63;
    int z = -1;
#pragma unroll
    for (int i = 0; i < (N + 63) / 64; ++i) {
        const int at = 64 * i + lane;
        const int first = at < t.count ? t.block0[at < N ? at : 0] : 0x7fffffff;
        z += __builtin_popcountll(__ballot(y >= first));
    }
    z = uniform(z);
    *place = y - t.block0[z];
    return z;
}

// A tile holds kTile rows of a head, RB bytes each, in 16-byte chunks.  Chunk c of row r is at
// place c ^ swizzle(r) of its row, so that neither way of reading it has a bank conflict: the 16
// rows of a quarter of a row read (one chunk of each) lie in 16 different places of 256 bytes, and
// the four rows x 64 bytes that half of a transposed read touches do as well.
template <typename T, int D>
struct Tile {
    static constexpr int RB = D * (int)sizeof(T);
    static constexpr int CPR = RB / 16;          // chunks of a row
    static constexpr int STEPS = RB / 32;        // steps of a product over the head dimension
    static constexpr int DB = D / 32;            // blocks of 32 dimensions
    static constexpr int BYTES = kTile * RB;
    static constexpr int PER = kTile * CPR / kThreads;   // chunks of a tile that a thread moves
    static __device__ __forceinline__ int swizzle(int r) {
        return CPR == 8 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : ((r & 3) << 2) | ((r >> 2) & 3);
    }
    static __device__ __forceinline__ int at(int r, int c) { return r * RB + ((c ^ swizzle(r)) << 4); }
};

// Operand of a row for a product over the head dimension, step s: 16 bytes, the lane's half of
// the step's 32.  (A row's dimensions come in the same order on both sides of a product.)
template <typename T, int D>
__device__ __forceinline__ u32x4 row_operand(const char* tile, int r, int s, int h) {
    return *reinterpret_cast<const u32x4*>(tile + Tile<T, D>::at(r, 2 * s + h));
}
// acc[row of a][row of b] += sum over the step's dimensions.  acc's register r of lane l holds
// a's row 8 (r / 4) + 4 (l / 32) + r % 4 and b's row l % 32.
template <typename T>
__device__ __forceinline__ void mma_step(const u32x4& a, const u32x4& b, f32x16& acc) {
    if constexpr (sizeof(T) == 2) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), acc, 0, 0, 0);
    }
}

// acc[db][dimension of block db][column] += sum over 32 rows of the tile (from row r0, a multiple
// of 32) of tile[row][dimension] p[row][column], p laid out like mma_step's acc (a's rows = the
// tile's).  bf16: p is rounded to bf16, half a step of 2^-8 of each value; the sum is fp32.
// Rows may come in any order as long as both sides agree, so p's registers are operands as they are.
template <int D, typename T>
__device__ __forceinline__ void mma_rows(const char* tile, int r0, const f32x16& p, f32x16 (&acc)[D / 32]) {
    const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
    using Tl = Tile<T, D>;
    if constexpr (sizeof(T) == 2) {
        typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
        const int l16 = lane & 15, lg = lane >> 4;
        const int row = 4 * h + (l16 >> 2), chunk = 2 * (lg & 1) + ((l16 & 3) >> 1);
        const uint32_t base = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)(tile + r0 * Tl::RB);
        const uint32_t a0 = base + Tl::at(row, chunk) + 8 * (l16 & 1), a1 = base + Tl::at(row + 8, chunk) + 8 * (l16 & 1);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const u32x4 pk = {pack_bf16x2(p[8 * c], p[8 * c + 1]), pack_bf16x2(p[8 * c + 2], p[8 * c + 3]),
                              pack_bf16x2(p[8 * c + 4], p[8 * c + 5]), pack_bf16x2(p[8 * c + 6], p[8 * c + 7])};
            const bf16x8 b = __builtin_bit_cast(bf16x8, pk);
#pragma unroll
            for (int db = 0; db < D / 32; ++db) {
                auto read = [&](uint32_t at) {
                    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s16x4*)(uintptr_t)((at ^ (64 * db)) + 16 * c * Tl::RB));
                };
                const s16x4 x = read(a0), y = read(a1);
                typedef __attribute__((__vector_size__(8 * sizeof(short)))) short s16x8;
                const s16x8 xy = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
                acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, xy), b, acc[db], 0, 0, 0);
            }
        }
    } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = 8 * (r >> 2) + 4 * h + (r & 3);
#pragma unroll
            for (int db = 0; db < D / 32; ++db) {
                const float a = *reinterpret_cast<const float*>(tile + Tl::at(r0 + row, 8 * db + (l32 >> 2)) + 4 * (l32 & 3));
                acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p[r], acc[db], 0, 0, 0);
            }
        }
    }
}

// A tile on its way from memory to LDS through registers: chunk i of a thread is chunk
// (tid % CPR) of row tid / CPR + i * (256 / CPR).
template <typename T, int D>
struct Moving {
    using Tl = Tile<T, D>;
    u32x4 x[Tl::PER];
    template <class RowPtr>   // row of the tile -> its first byte in memory
    __device__ __forceinline__ void load(RowPtr&& row) {
#pragma unroll
        for (int i = 0; i < Tl::PER; ++i) {
            const int r = threadIdx.x / Tl::CPR + i * (kThreads / Tl::CPR), c = threadIdx.x % Tl::CPR;
            x[i] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(row(r)) + 16 * c);
        }
    }
    __device__ __forceinline__ void store(char* tile) const {
#pragma unroll
        for (int i = 0; i < Tl::PER; ++i) {
            const int r = threadIdx.x / Tl::CPR + i * (kThreads / Tl::CPR), c = threadIdx.x % Tl::CPR;
            *reinterpret_cast<u32x4*>(tile + Tl::at(r, c)) = x[i];
        }
    }
};

// Four consecutive dimensions (registers 4 a .. 4 a + 3 of a block of acc) of the lane's column,
// as stored: the lanes of a column, l and l ^ 32, hold every second four.
template <typename T>
__device__ __forceinline__ void store4(T* to, float a, float b, float c, float d) {
    if constexpr (sizeof(T) == 2) {
        uint2 w = {pack_bf16x2(a, b), pack_bf16x2(c, d)};
        *reinterpret_cast<uint2*>(to) = w;
    } else {
        *reinterpret_cast<float4*>(to) = make_float4(a, b, c, d);
    }
}

}  // namespace
}  // namespace prompt
}  // namespace a2t
