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

// A tile holds kTile rows of a head, RB bytes each, in blocks of 1 KiB (RPB rows) that lie 1,040
// bytes apart.  Within a block the 16-byte chunks of its rows are interleaved so that neither way of
// reading has a bank conflict: 16 rows' chunk c lie in 16 different places of 256 bytes (row reads), and
// so do four rows x 64 bytes (transposed reads); and so that a lane's addresses differ by
// constants: one register for all steps of a product (an exclusive-or of row and chunk, without the 16
// bytes, took one a step).
template <typename T, int D>
struct Tile {
    static constexpr int RB = D * (int)sizeof(T);
    static constexpr int CPR = RB / 16;          // chunks of a row
    static constexpr int STEPS = RB / 32;        // steps of a product over the head dimension
    static constexpr int DB = D / 32;            // blocks of 32 dimensions
    static constexpr int RPB = 1024 / RB;        // rows of a block
    static constexpr int BLOCK = 1040;
    static constexpr int BYTES = kTile / RPB * BLOCK;
    static_assert(RPB == 2 || RPB == 4 || RPB == 8, "rows of 128, 256 or 512 bytes");
    // chunk c of row r
    static __device__ __forceinline__ int at(int r, int c) {
        const int block = r / RPB * BLOCK, q = r % RPB;
        if (RPB == 4) return block + (c >> 2) * 256 + q * 64 + (c & 3) * 16;
        if (RPB == 2) return block + (c >> 3) * 256 + q * 128 + (c & 7) * 16;
        return block + (c >> 2) * 512 + (q >> 2) * 256 + (q & 3) * 64 + (((c & 3) ^ ((q >> 2) << 1)) * 16);
    }
    // row of a block and chunk that place j of it holds
    static __device__ __forceinline__ int row_of(int j) {
        return RPB == 4 ? (j >> 2) & 3 : RPB == 2 ? (j >> 3) & 1 : ((j >> 4) & 1) * 4 + ((j >> 2) & 3);
    }
    static __device__ __forceinline__ int chunk_of(int j) {
        return RPB == 4 ? (j >> 4) * 4 + (j & 3) : RPB == 2 ? (j >> 4) * 8 + (j & 7) : (j >> 5) * 4 + ((j & 3) ^ (((j >> 4) & 1) << 1));
    }
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
        const char* const from = tile + Tl::at(row, chunk) + 8 * (l16 & 1);   // rows r0 + 16 c + row and 8 further, block db
        const char* const from8 = tile + Tl::at(row + 8, chunk) + 8 * (l16 & 1);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const u32x4 pk = {pack_bf16x2(p[8 * c], p[8 * c + 1]), pack_bf16x2(p[8 * c + 2], p[8 * c + 3]),
                              pack_bf16x2(p[8 * c + 4], p[8 * c + 5]), pack_bf16x2(p[8 * c + 6], p[8 * c + 7])};
            const bf16x8 b = __builtin_bit_cast(bf16x8, pk);
#pragma unroll
            for (int db = 0; db < D / 32; ++db) {
                auto read = [&](const char* at) {
                    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + Tl::at(r0 + 16 * c, 4 * db)));
                };
                const s16x4 x = read(from), y = read(from8);
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

// ---- bf16: LDS reads issued ahead as assembly, in groups of at most 16 registers.  The compiler,
// left to itself, requests all of a product's operands at once, which costs the 256 registers that a
// wave of two on a SIMD has (spills to memory, whose reloads then wait for the next tile too), or waits
// for each before the next.  A group's registers hold nothing until lds_wait() has named them; LDS
// reads return in order, so that waiting for all but the N youngest is enough, and any read of the
// compiler's between them makes the wait longer, never shorter.
template <int OFF>
__device__ __forceinline__ u32x4 read16(uint32_t at) {
    u32x4 r;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(r) : "v"(at), "i"(OFF));
    return r;
}
template <int OFF>
__device__ __forceinline__ uint2 read8t(uint32_t at) {
    uint2 r;
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r) : "v"(at), "i"(OFF));
    return r;
}
template <int N>
__device__ __forceinline__ void lds_wait(u32x4 (&a)[4]) {
    asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(a[0]), "+v"(a[1]), "+v"(a[2]), "+v"(a[3]) : "i"(N));
}
template <int N>
__device__ __forceinline__ void lds_wait(u32x4 (&a)[2]) {
    asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(a[0]), "+v"(a[1]) : "i"(N));
}
template <int N>
__device__ __forceinline__ void lds_wait(uint2 (&a)[8]) {
    asm volatile("s_waitcnt lgkmcnt(%8)"
                 : "+v"(a[0]), "+v"(a[1]), "+v"(a[2]), "+v"(a[3]), "+v"(a[4]), "+v"(a[5]), "+v"(a[6]), "+v"(a[7])
                 : "i"(N));
}
template <int N>
__device__ __forceinline__ void lds_wait(uint2 (&a)[4]) {
    asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(a[0]), "+v"(a[1]), "+v"(a[2]), "+v"(a[3]) : "i"(N));
}

// Row reads of a lane: its row of the tile at LDS address `tile` (row r of it), operand of step K.
template <int D>
struct RowReads {
    using Tl = Tile<bf16_t, D>;
    uint32_t even, odd;   // of even and odd steps (D 128: 32 bytes apart)
    __device__ __forceinline__ RowReads(uint32_t tile, int r, int h) : even(tile + Tl::at(r, h)), odd(tile + Tl::at(r, 2 + h)) {}
    template <int K, int ROWS = 0>   // of the row ROWS further (a multiple of 32)
    __device__ __forceinline__ u32x4 step() const {
        constexpr int OFF = ROWS / Tl::RPB * Tl::BLOCK;
        if constexpr (D == 128) return read16<OFF + (K >> 1) * 256 + (K & 1) * 32>(even);
        else return read16<OFF + (K >> 1) * 512>(K & 1 ? odd : even);
    }
};
// Transposed reads: rows r0 + 16 C .. + 15 of the tile (r0 a multiple of 32), all blocks of 32
// dimensions; group C of a 32-row block.
template <int D>
struct TransReads {
    using Tl = Tile<bf16_t, D>;
    uint32_t from;
    __device__ __forceinline__ TransReads(uint32_t tile, int r0) {
        const int lane = threadIdx.x & 63, l16 = lane & 15, lg = lane >> 4;
        from = tile + Tl::at(r0 + 4 * (lane >> 5) + (l16 >> 2), 2 * (lg & 1) + ((l16 & 3) >> 1)) + 8 * (l16 & 1);
    }
    template <int C, int DB0>   // blocks DB0 and DB0 + 1 alone
    __device__ __forceinline__ void pair(uint2 (&x)[4]) const {
        constexpr int BLOCK = D == 128 ? 256 : 512, OFF = 16 * C / Tl::RPB * Tl::BLOCK + DB0 * BLOCK, FAR = 8 / Tl::RPB * Tl::BLOCK;
        x[0] = read8t<OFF>(from), x[1] = read8t<OFF + FAR>(from);
        x[2] = read8t<OFF + BLOCK>(from), x[3] = read8t<OFF + BLOCK + FAR>(from);
    }
    template <int C, int DB0 = 0>
    __device__ __forceinline__ void group(uint2 (&x)[D / 16]) const {
        if constexpr (DB0 < D / 32) {
            constexpr int OFF = 16 * C / Tl::RPB * Tl::BLOCK + DB0 * (D == 128 ? 256 : 512);
            x[2 * DB0] = read8t<OFF>(from);
            x[2 * DB0 + 1] = read8t<OFF + 8 / Tl::RPB * Tl::BLOCK>(from);
            group<C, DB0 + 1>(x);
        }
    }
};
__device__ __forceinline__ bf16x8 pack8(const f32x16& p, int c) {
    const u32x4 pk = {pack_bf16x2(p[8 * c], p[8 * c + 1]), pack_bf16x2(p[8 * c + 2], p[8 * c + 3]),
                      pack_bf16x2(p[8 * c + 4], p[8 * c + 5]), pack_bf16x2(p[8 * c + 6], p[8 * c + 7])};
    return __builtin_bit_cast(bf16x8, pk);
}
// acc[db] += rows of a transposed group times the packed values of the same rows
template <int D>
__device__ __forceinline__ void mma_group(const uint2 (&x)[D / 16], const bf16x8& p, f32x16 (&acc)[D / 32]) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
        const u32x4 a = {x[2 * db].x, x[2 * db].y, x[2 * db + 1].x, x[2 * db + 1].y};
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), p, acc[db], 0, 0, 0);
    }
}

// A tile's way from memory into LDS: 1 KiB blocks, PER of them a wave, 16 bytes a lane, without
// registers between.  Lane j of a block fills place j % CPR of the block's row j / CPR; the address it
// reads picks the chunk that belongs there.  Written as assembly: of the builtin's loads the compiler
// waits for all before it reads any LDS, the next tile's with this one's.  What it counts itself
// stays right (loads return in order, so that more of them outstanding than it knows make its waits
// longer, never shorter); wait_tiles() is the wait for these.
template <typename T, int D, int WAVES = 4>
struct Coming {
    using Tl = Tile<T, D>;
    static constexpr int PER = kTile / Tl::RPB / WAVES;  // blocks of a wave
    static_assert(PER >= 1, "a wave moves whole blocks");
    static __device__ __forceinline__ void block(const char* base, uint32_t at, uint32_t lds) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(at), "s"(base) : "memory");
    }
    // rows lo .. lo + 63, those past `last` read row `last`
    static __device__ __forceinline__ void rows(const char* base, int64_t stride, int lo, int last, int w, uint32_t lds) {
        const int lane = threadIdx.x & 63, r0 = w * PER * Tl::RPB, row = Tl::row_of(lane);
        const uint32_t byte = Tl::chunk_of(lane) * 16;
        const char* first = base + (lo + r0) * stride;
        lds += w * PER * Tl::BLOCK;
        if (lo + kTile - 1 <= last) {
            const uint32_t at = (uint32_t)row * (uint32_t)stride + byte;
#pragma unroll
            for (int i = 0; i < PER; ++i) block(first + i * Tl::RPB * stride, at, lds + i * Tl::BLOCK);
        } else {
            first = base + lo * stride;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                block(first, (uint32_t)min(r0 + i * Tl::RPB + row, last - lo) * (uint32_t)stride + byte, lds + i * Tl::BLOCK);
        }
    }
};
__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)uniform((int)(uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)(p));
}
__device__ __forceinline__ void wait_tiles() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

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
