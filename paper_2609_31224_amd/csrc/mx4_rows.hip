// Rows of A2T_MX4 caches as they are written, and rows of any cache read back (gfx950).
//
//   append_mx4  rotates a step's keys by their positions, encodes K and V and stores
//               codes and scales in the ring.
//   move_mx4    copies the rows that an eviction retains into the kept region.
//   read_rows   resident rows in cache order: decoded (A2T_MX4) or copied.
#include "a2t_internal.h"
#include "a2t.h"
#include "launch.h"
#include "mx4_device.h"


#include <type_traits>

namespace a2t {
namespace {

constexpr int kRowThreads = 256;
constexpr int64_t kFullThreads = 256 * 1024;   // threads that fill the CUs

__device__ __forceinline__ void unpack8(const u32x4& r, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(r[e] << 16);
        x[2 * e + 1] = __uint_as_float(r[e] & 0xffff0000u);
    }
}
// Encodes a thread's 8 elements of a block that four neighbouring lanes share; *scale: its byte.
__device__ __forceinline__ uint32_t encode8(const float (&x)[8], int* scale) {
    uint32_t big = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) big = max(big, __float_as_uint(x[e]) & 0x7fffffffu);
    big = max(big, (uint32_t)__shfl_xor((int)big, 1));
    big = max(big, (uint32_t)__shfl_xor((int)big, 2));
    *scale = mx4_scale(big);
    const float s = __uint_as_float((uint32_t)*scale << 23);
    uint32_t c = 0;   // round to nearest even, saturating
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
    return *scale == kMxNaN ? 0u : c;
}

// One thread per (row, 8 dims of the lower half and their rotate-half partners of the upper one,
// `heads` KV heads one after the other), K and V: every element is loaded once, four lanes
// hold a block, and the next head's loads are in flight while one is encoded.  Bound by memory: 36
// layers of two steps of 1,024 rows of 8 heads of 128, 382 MB, take 68 us (5.6 TB/s; with one head
// a thread and nothing in flight 101).  A unit's rows take a launch's 4 to 5 us.
//
// The rotation is computed in 64 bits (products of a bf16 and an fp32 number are exact there)
// and rounded to fp32 once, so that what a key is encoded as follows from the inputs and the
// rotary table alone: two fp32 roundings would put one key in ~10^7 on the other side of a
// border between two codes, depending on the compiler's choice of fused operations.
template <class BT>
__global__ __launch_bounds__(kRowThreads) void append_mx4_kernel(DevState st, BT b, const uint16_t* k, const uint16_t* v,
                                                                 int heads) {
    const AppendDesc d = b.d[blockIdx.y];
    const uint32_t D = st.D, half = D / 2, tph = D / 16, groups = ((uint32_t)st.Hkv + heads - 1) / heads;
    const uint32_t x = blockIdx.x * kRowThreads + threadIdx.x;
    const uint32_t y = x / tph, r = y / groups;
    if (r >= (uint32_t)d.n) return;   // whole groups of four lanes: tph is a multiple of 4
    const uint32_t d0 = (x - y * tph) * 8, g0 = (y - r * groups) * heads, g1 = min(g0 + heads, (uint32_t)st.Hkv);
    int slot = d.slot0 + r;
    if (slot >= st.unit_rows) slot -= st.unit_rows;
    const int64_t in = (((int64_t)blockIdx.z * b.total_rows + d.in_row0 + r) * st.Hkv + g0) * D + d0;
    const uint16_t *pk = k + in, *pv = v + in;
    const float4* cs4 = reinterpret_cast<const float4*>(st.rope + ((int64_t)d.s * st.max_step_rows + r) * half + d0);
    u32x4 raw[4];
    auto load = [&] {
        raw[0] = *reinterpret_cast<const u32x4*>(pk);
        raw[1] = *reinterpret_cast<const u32x4*>(pk + half);
        raw[2] = *reinterpret_cast<const u32x4*>(pv);
        raw[3] = *reinterpret_cast<const u32x4*>(pv + half);
    };
    load();
    float4 cs[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) cs[e] = cs4[e];
    const Mx4Pool kp = mx4_pool(st, st.k_unit), vp = mx4_pool(st, st.v_unit);
    int64_t row = mx4_ring_row(st, b.layer0 + blockIdx.z, d.s, g0) + slot;
    for (uint32_t g = g0; g < g1; ++g, row += st.unit_rows) {
        const u32x4 klo = raw[0], khi = raw[1], vlo = raw[2], vhi = raw[3];
        if (g + 1 < g1) pk += D, pv += D, load();
        auto store = [&](const Mx4Pool& p, const float(&y)[8], uint32_t at) {
            int scale;
            const uint32_t code = encode8(y, &scale);
            *reinterpret_cast<uint32_t*>(p.codes + row * half + at / 2) = code;
            if (at % kMxBlock == 0) p.scales[row * (D / kMxBlock) + at / kMxBlock] = (uint8_t)scale;
        };
        float lo[8], hi[8], ylo[8], yhi[8];
        unpack8(klo, lo);
        unpack8(khi, hi);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double co = e & 1 ? cs[e / 2].z : cs[e / 2].x, si = e & 1 ? cs[e / 2].w : cs[e / 2].y;
            ylo[e] = (float)((double)lo[e] * co - (double)hi[e] * si);
            yhi[e] = (float)((double)hi[e] * co + (double)lo[e] * si);
        }
        store(kp, ylo, d0);
        store(kp, yhi, d0 + half);
        unpack8(vlo, lo);
        unpack8(vhi, hi);
        store(vp, lo, d0);
        store(vp, hi, d0 + half);
    }
}

// grid (layer, stream, rows): a wave takes every fourth row of the span that eviction has
// passed over and copies it, where it is kept, to the slot that the eviction's index pass found for
// it.  A chunk is a block's 16 bytes of codes, and its scale byte goes with it.  A unit's 3 rows of 36 layers
// of 2 x 8 heads take a launch's time (8.8 us with the launch that finds them), 60 rows of each of 16 streams 62 us with it.
template <class BT>
__global__ __launch_bounds__(kRowThreads) void move_mx4_kernel(DevState st, BT b) {
    const EvictDesc d = b.d[blockIdx.y];
    const int lane = threadIdx.x & 63, nb = st.D / kMxBlock, chunks = 2 * st.Hkv * nb, layer = blockIdx.x;
    const int64_t eb = (int64_t)d.s * ((int64_t)st.unit_rows + st.kept_rows);
    const Mx4Pool kp = mx4_pool(st, st.k_unit), vp = mx4_pool(st, st.v_unit);
    for (int x = blockIdx.z * (kRowThreads / 64) + (threadIdx.x >> 6); x < d.span; x += gridDim.z * (kRowThreads / 64)) {
        const int to = st.ev_slot[eb + d.kept + x];
        if (to < 0) continue;
        int from = d.head + x;
        if (from >= st.unit_rows) from -= st.unit_rows;
        for (int c = lane; c < chunks; c += 64) {
            const bool is_v = c >= chunks / 2;
            const int y = is_v ? c - chunks / 2 : c, g = y / nb, ch = y - g * nb;
            const Mx4Pool& p = is_v ? vp : kp;
            const int64_t src = (mx4_ring_row(st, layer, d.s, g) + from) * nb + ch;
            const int64_t dst = (mx4_kept_row(st, layer, d.s, g) + to) * nb + ch;
            reinterpret_cast<u32x4*>(p.codes)[dst] = reinterpret_cast<const u32x4*>(p.codes)[src];
            p.scales[dst] = p.scales[src];
        }
    }
}

// grid (rows / b.rows, stream, layer x {K, V}): a workgroup writes b.rows consecutive rows, a
// thread 16 bytes of every kRowThreads-th chunk of them, four loads ahead of their stores.  Bound by
// the writes, which are not read again soon and pass the caches by: 36 layers of 4,096 rows of 8 heads of 128 held in 4
// bits, 764 MB, take 115 us (6.7 TB/s; 21 sessions of two layers 64 us with cached stores and a load at a
// time, 44 so).
template <int DTYPE, class BT>
__global__ __launch_bounds__(kRowThreads) void read_rows_kernel(DevState st, BT b, char* k, char* v) {
    constexpr int EPT = DTYPE == A2T_F32 ? 4 : 8, EB = 16 / EPT;   // elements of a chunk, bytes of one
    constexpr int U = 4;
    const ReadDesc d = b.d[blockIdx.y];
    const bool is_v = blockIdx.z & 1;
    char* const out = is_v ? v : k;
    const int j0 = blockIdx.x * b.rows, rows = min(b.rows, d.R - j0);
    if (rows <= 0 || !out) return;
    const uint32_t D = st.D, cph = D / EPT, cpr = st.Hkv * cph;
    const int z = blockIdx.z >> 1, layer = b.layer0 + z;
    const uint32_t dr = kRowThreads / cpr, dc = kRowThreads - dr * cpr;   // from a thread's chunk to its next
    uint32_t r = threadIdx.x / cpr, c = threadIdx.x - r * cpr;
    char* const to = out + ((int64_t)z * b.total_rows + d.row0 + j0) * cpr * 16;
    const Mx4Pool p = mx4_pool(st, is_v ? st.v_unit : st.k_unit);
    const void* const pool_ring = is_v ? st.v_unit : st.k_unit;
    const void* const pool_kept = is_v ? st.v_kept : st.k_kept;
    while (r < (uint32_t)rows) {
        u32x4 x[U];
        uint32_t code[U], byte[U], at_r[U], at_c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            at_r[u] = r, at_c[u] = c;
            const int j = j0 + (int)min(r, (uint32_t)rows - 1);
            const uint32_t g = c / cph, d0 = (c - g * cph) * EPT;
            const bool in_kept = j < d.kept;
            int at = in_kept ? j : d.head + (j - d.kept);
            if (!in_kept && at >= st.unit_rows) at -= st.unit_rows;
            if constexpr (DTYPE == A2T_MX4) {
                const int64_t row = (in_kept ? mx4_kept_row(st, layer, d.s, g) : mx4_ring_row(st, layer, d.s, g)) + at;
                code[u] = *reinterpret_cast<const uint32_t*>(p.codes + row * (D / 2) + d0 / 2);
                byte[u] = p.scales[row * (D / kMxBlock) + d0 / kMxBlock];
            } else {
                const int64_t e = pool_index(st, layer, d.s, g, in_kept ? st.kept_rows : st.unit_rows, at) + d0;
                x[u] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(in_kept ? pool_kept : pool_ring) + e * EB);
            }
            r += dr, c += dc;
            if (c >= cpr) c -= cpr, ++r;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (DTYPE == A2T_MX4) {
                x[u] = mx4_to_bf16(code[u], __uint_as_float(byte[u] << 23));
                if (byte[u] == kMxNaN) x[u] = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};   // one NaN, as on the host
            }
            if (at_r[u] < (uint32_t)rows)
                __builtin_nontemporal_store(x[u], reinterpret_cast<u32x4*>(to + ((uint64_t)at_r[u] * cpr + at_c[u]) * 16));
        }
    }
}

}  // namespace

hipError_t launch_append_mx4(const DevState& st, const AppendBatch& b, int n_layers, const void* k, const void* v,
                             hipStream_t stream, const KTimer& kt) {
    // heads of a thread: more while the threads still fill the CUs
    const int64_t threads = (int64_t)b.max_n * b.count * n_layers * st.Hkv * (st.D / 16);
    int heads = 1;
    while (heads < st.Hkv && threads / (2 * heads) >= kFullThreads) heads *= 2;
    const int64_t per_stream = (int64_t)b.max_n * ((st.Hkv + heads - 1) / heads) * (st.D / 16);
    const dim3 grid((uint32_t)((per_stream + kRowThreads - 1) / kRowThreads), b.count, n_layers);
    const uint16_t *kk = static_cast<const uint16_t*>(k), *vv = static_cast<const uint16_t*>(v);
    return by_size<AppendBatchT>(b, [&](const auto& bb) {
        using B = std::decay_t<decltype(bb)>;
        return launch_kernel(append_mx4_kernel<B>, grid, dim3(kRowThreads), {stream, kt.start, kt.stop}, st, bb, kk, vv, heads);
    });
}

hipError_t launch_move_mx4(const DevState& st, const EvictBatch& b, hipStream_t stream, const KTimer& kt) {
    int span = 1;
    for (int i = 0; i < b.count; ++i) span = b.d[i].span > span ? b.d[i].span : span;
    const dim3 grid(st.L, b.count, span < 256 ? (span + 3) / 4 : 64);
    return by_size<EvictBatchT>(b, [&](const auto& bb) {
        using B = std::decay_t<decltype(bb)>;
        return launch_kernel(move_mx4_kernel<B>, grid, dim3(kRowThreads), {stream, kt.start, kt.stop}, st, bb);
    });
}

hipError_t launch_read_rows(const DevState& st, const ReadBatch& b, int n_layers, void* k, void* v, hipStream_t stream,
                            const KTimer& kt) {
    const int cpr = st.Hkv * st.D / (st.dtype == A2T_F32 ? 4 : 8);
    ReadBatch rb = b;
    // rows of a workgroup: eight chunks a thread, a row at least
    rb.rows = cpr > kRowThreads * 8 ? 1 : kRowThreads * 8 / cpr;
    const dim3 grid((b.max_R + rb.rows - 1) / rb.rows, b.count, 2 * n_layers);
    char *kk = static_cast<char*>(k), *vv = static_cast<char*>(v);
    return by_size<ReadBatchT>(rb, [&](const auto& bb) {
        using B = std::decay_t<decltype(bb)>;
        auto go = [&](auto kernel) {
            return launch_kernel(kernel, grid, dim3(kRowThreads), {stream, kt.start, kt.stop}, st, bb, kk, vv);
        };
        if (st.dtype == A2T_F32) return go(read_rows_kernel<A2T_F32, B>);
        if (st.dtype == A2T_BF16) return go(read_rows_kernel<A2T_BF16, B>);
        return go(read_rows_kernel<A2T_MX4, B>);
    });
}

}  // namespace a2t
