// Rows held in 4 bits (A2T_MX4 caches): where they are, and how a block is encoded.
//
// A head's row of K (rotated) or V is D / 32 blocks of 32 elements: 16 bytes of e2m1 codes
// (element i of the block in bits 4 (i % 2) .. + 3 of byte i / 2) and one e8m0 byte, the
// block's scale 2^(byte - 127).  Both are what the matrix instructions with block scales
// and the scaled conversions take, so that a score product reads K as it is stored and V
// becomes fp16 at two elements an instruction, without a multiplication.
//
// Scale: the exponent of the block's largest magnitude a less 2, so that a lies in [4, 8)
// units, and one more where a would be 7 or above, which is nearer to 8 than to 6, the
// largest element.  Against saturating there this halves the largest error (relative error
// of N(0, 1) rows 0.112 against 0.115, of Student t rows with 4 degrees 0.129 against 0.131;
// 15-level integers with a bf16 scale per block 0.097 and 0.131, and a third more work to
// unpack).  Held between 2^-124 and 2^125 every value is a normal bf16 number.
#pragma once

#include "a2t_internal.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace a2t {

constexpr int kMxBlock = 32;              // elements of a block
constexpr int kMxLeast = 3, kMxMost = 252;   // scale bytes
constexpr int kMxNaN = 255;               // a block that holds an infinity or a NaN: reads as NaN

// Bytes of a pool of `rows` head rows (codes of every row, then their scales).
inline int64_t mx4_pool_bytes(int64_t rows, int head_dim) { return rows * (head_dim / 2 + head_dim / kMxBlock); }

// A pool and its rows: row x has its codes at codes + x D / 2 and its scales at scales + x D / 32.
// The rows of the ring [L][S][Hkv][unit_rows] come first, then the kept regions'.
struct Mx4Pool {
    uint8_t* codes;
    uint8_t* scales;
};
__host__ __device__ inline int64_t mx4_heads(const DevState& st) { return (int64_t)st.L * st.S * st.Hkv; }
__host__ __device__ inline Mx4Pool mx4_pool(const DevState& st, void* pool) {
    uint8_t* p = static_cast<uint8_t*>(pool);
    return {p, p + mx4_heads(st) * ((int64_t)st.unit_rows + st.kept_rows) * (st.D / 2)};
}
// first row of a head's ring and of its kept region
__host__ __device__ inline int64_t mx4_ring_row(const DevState& st, int layer, int s, int g) {
    return (((int64_t)layer * st.S + s) * st.Hkv + g) * st.unit_rows;
}
__host__ __device__ inline int64_t mx4_kept_row(const DevState& st, int layer, int s, int g) {
    return mx4_heads(st) * st.unit_rows + (((int64_t)layer * st.S + s) * st.Hkv + g) * st.kept_rows;
}

// scale byte of a block whose largest magnitude has these fp32 bits (sign cleared; as integers
// the bits of an infinity and of every NaN are above those of any number)
__host__ __device__ inline int mx4_scale(uint32_t largest) {
    if (largest >= 0x7f800000u) return kMxNaN;
    const int e = (int)((largest + 0x200000u) >> 23) - 2;
    return e < kMxLeast ? kMxLeast : e > kMxMost ? kMxMost : e;
}

// Workgroups (per split and KV head) of `rows` query rows each that cover query_rows.
inline int mx4_groups(int query_rows, int rows) { return (query_rows + rows - 1) / rows; }

// ---- reading rows back (any cache)
struct ReadDesc {
    int32_t s;
    int32_t kept;      // rows in the kept region
    int32_t head;      // ring head slot
    int32_t R;         // resident rows
    int64_t row0;      // first row of the stream in the packed output
};
template <int N>
struct ReadBatchT {
    int32_t count;
    int32_t layer0;       // first layer read
    int32_t max_R;
    int32_t rows;         // rows of a workgroup (set by the launcher)
    int64_t total_rows;   // rows per layer in the packed output
    ReadDesc d[N];
};
using ReadBatch = ReadBatchT<kMaxDesc>;

// Launchers (attn_mx4.hip, attn_mx4_rows.hip, mx4_rows.hip).  Each issues one kernel unless it says otherwise.
// MFMA attention (chunk and decode, D 64 or 128; the step's rows already stored), query_blocks (1 to 3)
// blocks of 16 query rows a workgroup.  Split partials as launch_attn_tile's.
hipError_t launch_attn_mx4(const DevState& st, const AttnBatch& b, int query_blocks, const void* q, void* o, hipStream_t stream,
                           const KTimer& kt);
// The same for many query rows: row_waves (2 or 4) x 32 of them a workgroup of twice as many waves.
hipError_t launch_attn_mx4_rows(const DevState& st, const AttnBatch& b, int row_waves, const void* q, void* o, hipStream_t stream,
                                const KTimer& kt);
// Encodes and stores a step's rows (launch_append of other caches).
hipError_t launch_append_mx4(const DevState& st, const AppendBatch& b, int n_layers, const void* k, const void* v,
                             hipStream_t stream, const KTimer& kt);
// Moves the rows that an eviction retains, by the new slots that launch_evict has written.
hipError_t launch_move_mx4(const DevState& st, const EvictBatch& b, hipStream_t stream, const KTimer& kt);
// Resident rows in cache order (any cache): k or v may be null.
hipError_t launch_read_rows(const DevState& st, const ReadBatch& b, int n_layers, void* k, void* v, hipStream_t stream,
                            const KTimer& kt);

}  // namespace a2t
