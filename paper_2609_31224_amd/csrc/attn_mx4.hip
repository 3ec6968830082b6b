// Causal attention of a step's rows over rows held in 4 bits (A2T_MX4 caches; chunk and decode;
// gfx950).  The layout of a block is in mx4.h.
//
//   attn_mx4  one workgroup = (key split, QB blocks of 16 query rows, KV head, stream),
//             8 waves: wave w takes every eighth 32-key block of the split; the eight
//             states are combined in LDS at the end.
//
// Scores: v_mfma_scale_f32_16x16x128_f8f6f4 multiplies K as it is stored, scales included,
// with Q in e2m3 (6 bits): a block of 32 rotated elements is scaled by a power of two and written as three
// e2m3 numbers an element, the later ones with scales 2^-4 and 2^-9 of the first one's.  The first is off by up to
// 1/4 unit where the largest element has 3.875 to 7.75 of them, two by up to 1/128, three by 1/4096: 2^-13.9 of
// the block's largest element.  The error is the same for the block's small elements, and their keys may be the
// large ones: with four channels of Q 50 times and four others of K 20 times the rest, outputs are off by 0.0178 of
// their size with two numbers, 0.0003 with three and 0.0026 with Q in bf16.  The third costs 10 % of the time of
// long chunks and of units, none of decode on many keys (1,024 rows onto 16,384 keys 283 -> 311 us, 16 sessions of 22 rows onto
// 8,192 63 -> 70).  (Two numbers in e4m3 take the products' time of four in e2m3.)  At head dim 128 that is
// three products per 16 keys, at 64 two: K times the first part with K times the second in one's 128 dims, and K
// times the third in half of the other's.
// Values: a lane's 16 bytes of V are a block, which the scaled conversion turns into fp16
// (exactly); transposed LDS reads then give the operand of v_mfma_f32_16x16x32_f16.  The few blocks
// that fp16 does not hold are added in fp32.  Probabilities are fp16, relative to a reference that
// a wave's largest one reaches or exceeds: off by up to 2^-11 of each, or 2^-25 of the largest.  (In bf16, at the
// same time, they were off by as much as the output's own rounding: with two parts a query an error against 64 bits of
// 0.0026 instead of 0.0020 relative, 64 sessions on 4,096 keys.  With three it is 0.0017, that of the bf16 output alone.)
// Nothing is shared between waves before the end, so there are no barriers in the loop; the
// next block's codes are in flight while one is computed.
//
// One block of rows (decode): bound by memory where there are many sessions (64 of 4,096 keys, 48 us a
// layer, 5.9 TB/s) or keys (one of 131,072: 26 us, 5.5 TB/s), by the launch and the way of the first loads for
// one session of 4,096 (7.5 us, and 4 of the merge).  Two and three blocks: bound by vector operations and products
// together, which overlap little (a product takes the vector units' time, attn_mx4_rows.hip): 16 sessions of 22 rows
// onto 8,192 keys 65 to 71 us, of which products are busy 33 %, vector operations 56 %.
#include "a2t_internal.h"
#include "launch.h"
#include "mx4_device.h"

#include <math.h>

#include <type_traits>

namespace a2t {
namespace {

constexpr int kWaves = 8;
constexpr int kKeyBlock = 32;    // keys of a wave's block
constexpr int kRows = 16;        // query rows of a product

// LDS accesses of the wave before this one come before those after it, whatever the compiler
// knows about their addresses in one lane (the hardware keeps a wave's LDS accesses in order)
__device__ __forceinline__ void wave_lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}
// max over the four lanes l % 16 + 16 i that hold one query column
__device__ __forceinline__ float col_max(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Lane l of a wave is (column l % 16, group lg = l / 16).
//   scores   S^T[16 keys x 16 queries]: A = K, lane: key l % 16, block lg of 32 dims; B = Q^T,
//            lane: query l % 16, block lg; scales: one byte of each operand's row and block
//            lg.  The lane gets keys 4 lg + e of its query.
//   values   O^T[16 dims x 16 queries]: the 32 keys are contracted in the order in which the
//            scores of two products lie in a lane, keys 4 lg + e and 16 + 4 lg + e; the lane
//            gets dims 4 lg + e of each 16.
// V in LDS: a key's 16-byte chunk c is at c ^ f(key), so that neither the four keys x four
// blocks of a store nor the eight keys x two chunks of half a transposed read share banks.
template <int D>
__device__ __forceinline__ int v_chunk(int key, int c) {
    const int y = D == 128 ? key & 7 : (key >> 1) & 3;
    return key * (D / 8) + (c ^ (2 * y | ((y >> 1) & 1)));
}

template <int D, int QB, int N>
__global__ __launch_bounds__(64 * kWaves, QB == 1 ? 4 : 2) void attn_mx4_kernel(DevState st, AttnBatchT<N> b, WgStart<N> start,
                                                                               const uint16_t* q, uint16_t* o) {
    constexpr int NB = D / kMxBlock;   // blocks of a row
    constexpr int CB = D / 2;          // bytes of a row's codes
    constexpr int DB = D / 16;         // 16-dim blocks of O
    constexpr int VL = D / 64;         // 16-byte loads of V per lane and key block
    constexpr int QP = D == 128 ? 3 : 2;   // products per 16 keys: one for each part of Q, or the first two in one
    constexpr int kInRegs = QB == 1 && D == 128 ? 2 : QP;   // products whose Q operand stays in registers, of one block of rows
    constexpr int kAhead = QB == 3 ? 2 : 4;   // V operands read ahead of the products (three spill with three blocks)
    constexpr int kStride = kWaves * kKeyBlock;
    constexpr bool kPipe = QB > 1;
    // (its chunks are found by exclusive or on their addresses: whole rows are aligned)
    __shared__ __align__(256) u32x4 s_mem[(kPipe ? 2 : 1) * kWaves * kKeyBlock * D / 8];   // V of each wave's block; at the end the states
    __shared__ u32x4 s_q[QB][QP][64];           // Q operands, their first 16 bytes
    __shared__ uint2 s_q2[QB][QP][64];          // ... the other 8
    __shared__ uint8_t s_qs[QB][64];            // ... and their scales
    __shared__ float2 s_ml[kWaves][kRows];
    f32x4(&s_part)[kWaves][DB][64] = *reinterpret_cast<f32x4(*)[kWaves][DB][64]>(s_mem);
    static_assert(sizeof(f32x4) * kWaves * DB * 64 <= sizeof(s_mem), "the states of one block of query rows fit");

    int wg;
    const AttnDesc d = b.d[stream_of(start, b.count, &wg)];
    const int G = st.G, M = G * d.n_q, R = d.R;
    const int blocks = (M + kRows - 1) / kRows, groups = (blocks + QB - 1) / QB;
    auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };   // divisions run on the vector ALU
    // linear block (split, query group, KV head), heads fastest: the workgroups of a head
    // share an XCD's L2 when the head count divides the 8 XCDs
    const int y = uniform(wg / st.Hkv), g = wg - y * st.Hkv;
    const int sp = uniform(y / groups), grp = groups - 1 - (y - sp * groups);
    if (sp >= d.splits) return;
    const int w = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, l16 = lane & 15, lg = lane >> 4;
    const int mw = grp * QB * kRows;   // the workgroup's first query row
    const int vis0 = R - d.n_q;
    const int g_shift = __builtin_ctz(G);   // (G is 1, 2, 4 or 8)
    // step row of lane ln's query of block x (past M: that of row M - 1)
    auto step_row = [&](int x, int ln) { return min(mw + x * kRows + (ln & 15), M - 1) >> g_shift; };
    const int last_i = uniform((min(M, mw + QB * kRows) - 1) / G);
    const int k_end = vis0 + last_i + 1;
    const int t0 = sp * d.tile_q + min(sp, d.tile_r), t1 = t0 + d.tile_q + (sp < d.tile_r ? 1 : 0);
    // this wave's key blocks: k0, k0 + kStride, ..; n of them
    const int k0 = t0 * kTileKeys + w * kKeyBlock;
    const int n = max(0, (min(k_end, t1 * kTileKeys) - k0 + kStride - 1) / kStride);

    const int kept = d.kept, head = d.head, ring_rows = st.unit_rows;
    const Mx4Pool kp = mx4_pool(st, st.k_unit), vp = mx4_pool(st, st.v_unit);
    const int64_t ring0 = mx4_ring_row(st, b.layer, d.s, g), kept0 = mx4_kept_row(st, b.layer, d.s, g);
    auto ring_slot = [&](int j) {
        const int slot = head + (j - kept);
        return slot >= ring_rows ? slot - ring_rows : slot;
    };
    auto row_of = [&](int j) -> int64_t {
        j = min(j, R - 1);   // keys past R read row R-1 and are masked
        return j < kept ? kept0 + j : ring0 + ring_slot(j);
    };
    // first row of a key block that is one run of rows
    auto run_of = [&](int kb, int64_t* row) {
        if (kb + kKeyBlock > R) return false;
        if (kb + kKeyBlock <= kept) {
            *row = kept0 + kb;
            return true;
        }
        const int slot = ring_slot(kb);
        *row = ring0 + slot;
        return kb >= kept && slot + kKeyBlock <= ring_rows;
    };

    f32x4 acc[QB][DB], lsum[QB];   // lsum: the sum of probabilities, in every element
    float mrun[QB];
#pragma unroll
    for (int x = 0; x < QB; ++x) {
        mrun[x] = -INFINITY;
        lsum[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < DB; ++c) acc[x][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    u32x4 kc[2], vc[VL];
    int ks[2], vs[VL];   // their scale bytes
    // where a key block's rows are: a run from `row` on, or each row on its own
    struct Place {
        int64_t row;
        bool run;
    };
    auto place_of = [&](int kb) {
        Place p{0, false};
        p.run = run_of(kb, &p.row);
        return p;
    };
    // (addresses are picked by branches, the loads are not: a value loaded on one side of a
    // branch would be waited for there)
    auto load_k = [&](int kb, const Place& at, int ln) {
        const int l16 = ln & 15, c = (ln >> 4) & (NB - 1);
        const uint8_t *p[2], *ps[2];
        if (at.run) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                p[t] = kp.codes + at.row * CB + (uint32_t)((16 * t + l16) * CB + 16 * c);
                ps[t] = kp.scales + at.row * NB + (uint32_t)((16 * t + l16) * NB + c);
            }
        } else {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int64_t row = row_of(kb + 16 * t + l16);
                p[t] = kp.codes + row * CB + 16 * c;
                ps[t] = kp.scales + row * NB + c;
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            kc[t] = gload16(p[t]);
            ks[t] = gload1(ps[t]);
        }
    };
    auto load_v = [&](int kb, const Place& at, int ln) {
        const uint8_t *p[VL], *ps[VL];
        if (at.run) {
#pragma unroll
            for (int j = 0; j < VL; ++j) {
                p[j] = vp.codes + at.row * CB + (uint32_t)(16 * (64 * j + ln));
                ps[j] = vp.scales + at.row * NB + (uint32_t)(64 * j + ln);
            }
        } else {
#pragma unroll
            for (int j = 0; j < VL; ++j) {
                const int c = (64 * j + ln) % NB;
                const int64_t row = row_of(kb + (64 * j + ln) / NB);
                p[j] = vp.codes + row * CB + 16 * c;
                ps[j] = vp.scales + row * NB + c;
            }
        }
#pragma unroll
        for (int j = 0; j < VL; ++j) {
            vc[j] = gload16(p[j]);
            vs[j] = gload1(ps[j]);
        }
    };
    auto load_first = [&] {
        if (n == 0) return;
        const Place at = place_of(k0);
        load_v(k0, at, lane);
        load_k(k0, at, lane);
    };

    // Q^T operands.  First the rows, rotated and scaled by scale * log2(e), to LDS: a thread
    // takes 8 dims of the lower half and their partners of the upper one.  Rows past M read row
    // M - 1 and are never stored.
    constexpr int kPad = kMxBlock + 4;   // a block's floats in LDS: 16 lanes' reads do not share banks
    constexpr int kItems = QB * kRows * (D / 16), kTurns = (kItems + 64 * kWaves - 1) / (64 * kWaves);
    float* const s_rows = reinterpret_cast<float*>(s_mem);
    static_assert(sizeof(float) * QB * kRows * NB * kPad <= sizeof(s_mem), "the rotated rows fit");
#pragma unroll
    for (int turn = 0; turn < kTurns; ++turn) {
        const int x = turn * 64 * kWaves + (int)threadIdx.x;
        const int r = x / (D / 16), d0 = (x - r * (D / 16)) * 8;
        const int m = min(mw + r, M - 1), i = m / G;
        const uint16_t* qp = q + ((int64_t)(d.q_row0 + i) * st.Hq + g * G + (m - i * G)) * D + d0;
        const float4* cp = reinterpret_cast<const float4*>(
            st.rope + ((int64_t)d.s * st.max_step_rows + d.rope_row0 + i) * (D / 2) + d0);
        const u32x4 a = *reinterpret_cast<const u32x4*>(qp), a2 = *reinterpret_cast<const u32x4*>(qp + D / 2);
        float4 cs[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) cs[e] = cp[e];
        if (turn == 0) {
            __builtin_amdgcn_sched_barrier(0);
            load_first();   // K and V behind them: loads return in order
        }
        if (kItems % (64 * kWaves) == 0 || x < kItems)
            mx4_rotate(a, a2, cs, st.scale_log2e, s_rows + (r * NB + d0 / kMxBlock) * kPad + d0 % kMxBlock,
                       s_rows + (r * NB + (d0 + D / 2) / kMxBlock) * kPad + (d0 + D / 2) % kMxBlock);
    }
    __syncthreads();
    // Then the operands, a lane a block: with one block of rows every wave makes them for
    // itself, else wave x makes those of the 16 rows x.
    i32x8 qv[QP];   // Q operands: of one block of rows, the last read for each block; else read as the block before is done with them
    int qs;            // ... and their first part's scales, read with them
    if (QB == 1 || w < QB) {
        const int x0 = QB == 1 ? 0 : w;
        u32x6 part[kMxQueryParts];
        const int scale = mx4_query(s_rows + ((x0 * kRows + l16) * NB + (lg & (NB - 1))) * kPad, part);
        auto put = [&](int k, const u32x6& x) {
            if (QB == 1 && k < kInRegs) {
                qv[k] = mx4_operand(x);
            } else if (QB > 1 || w == 0) {
                s_q[QB == 1 ? 0 : w][k][lane] = u32x4{x[0], x[1], x[2], x[3]};
                s_q2[QB == 1 ? 0 : w][k][lane] = make_uint2(x[4], x[5]);
            }
        };
        int mine = scale;
        if constexpr (D == 128) {
#pragma unroll
            for (int k = 0; k < QP; ++k) put(k, part[k]);
        } else {   // the last 64 dims of the products are the second part, and nothing
            put(0, lg < NB ? part[0] : part[1]);
            put(1, lg < NB ? part[2] : u32x6{0u, 0u, 0u, 0u, 0u, 0u});
            mine = lg < NB ? scale : mx4_query_scale(scale, 1);
        }
        if (QB == 1) qs = mine;
        else s_qs[w][lane] = (uint8_t)mine;
    }
    __syncthreads();   // V takes the rows' place

    // this wave's V: where the lane's block e (of 8 dims) of its first row goes, and the lane's
    // place in the transposed reads (16 lanes read 8 bytes each of four keys' 32 bytes).  The
    // swizzle and e (the 16-dim block c) touch the same bits of the address.
    constexpr int kBuf = kWaves * kKeyBlock * D * 2;   // bytes of a buffer
    const uint32_t s_v = lds_addr(s_mem) + w * (kKeyBlock * D * 2);
    const uint32_t v_in0 = s_v + 16 * v_chunk<D>(lane / NB, 4 * (lane % NB));
    const uint32_t v_out0 = s_v + 16 * v_chunk<D>(4 * lg + (l16 >> 2), (l16 & 3) >> 1) + 8 * (l16 & 1);
    auto v_store = [&](uint32_t v_in, int j, int e, const u32x4& x) {   // row 64 j / NB + lane / NB
        *reinterpret_cast<__attribute__((address_space(3))) u32x4*>((uintptr_t)((v_in ^ (16u * e)) + j * (64 / NB) * D * 2)) = x;
    };
    auto v_op = [&](uint32_t v_out, int c) {
        i16x4 h[2];
#pragma unroll
        for (int half = 0; half < 2; ++half)
            h[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) i16x4*)(uintptr_t)((v_out ^ (32u * c)) + half * 16 * D * 2));
        return __builtin_bit_cast(f16x8, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // LDS reads and matrix products stay in the order written; other vector operations move freely
    auto ordered = [] { __builtin_amdgcn_sched_barrier(0x6); };
    // nothing moves past; between two of these a product is followed by m vector operations
    auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
    const f16x8 ones = __builtin_bit_cast(f16x8, u32x4{0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u});

    f32x4 sc[QB][2];   // scores of a block, relative to the running reference
    f16x8 p[QB];       // its probabilities
    auto read_part = [&](int x, int k, int ln) {
        const u32x4 a = s_q[x][k][ln];
        const uint2 b2 = s_q2[x][k][ln];
        return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b2.x, (int)b2.y, 0, 0};
    };
    // those of block x that are not there yet
    auto read_q = [&](int x, int ln) {
#pragma unroll
        for (int k = QB == 1 ? kInRegs : 0; k < QP; ++k) qv[k] = read_part(x, k, ln);
        if (QB > 1) qs = s_qs[x][ln];
    };
    auto score = [&](int x, int ln) {   // and the operands of the next block
        const float mu = mrun[x] == -INFINITY ? 0.f : mrun[x];
#pragma unroll
        for (int t = 0; t < 2; ++t) sc[x][t] = f32x4{-mu, -mu, -mu, -mu};
#pragma unroll
        for (int k = 0; k < QP; ++k) {
            const int s = mx4_query_scale(qs, D == 128 ? k : 2 * k);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const i32x8 kv = {(int)kc[t][0], (int)kc[t][1], (int)kc[t][2], (int)kc[t][3], 0, 0, 0, 0};
                sc[x][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kv, qv[k], sc[x][t], 4, 2, 0, ks[t], 0, s);
            }
            if (x + 1 < QB) qv[k] = read_part(x + 1, k, ln);
            if (x + 1 < QB && k == QP - 1) qs = s_qs[x + 1][ln];
        }
    };
    // hides what a row does not see, and moves the reference, lazily: the first block with a score sets it, and it is
    // raised, and the running sums rescaled, only when a block exceeds it by more than 2^8.  (A row without
    // one yet, which sees none of the wave's keys or whose scores are all -infinity in fp32, has the wave look at every block.)
    bool unset = true;
    auto settle = [&](int kb, int ln) {
        if (kb + kKeyBlock - 1 > vis0) {   // some row does not see every key
#pragma unroll
            for (int x = 0; x < QB; ++x) {
                const int see = vis0 + step_row(x, ln) - kb - 4 * (ln >> 4);
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (16 * t + e > see) sc[x][t][e] = -INFINITY;
            }
        }
        float top[QB], most = -INFINITY;
#pragma unroll
        for (int x = 0; x < QB; ++x) {
            top[x] = fmaxf(fmaxf(sc[x][0][0], sc[x][0][1]), sc[x][0][2]);
            top[x] = fmaxf(fmaxf(top[x], sc[x][0][3]), sc[x][1][0]);
            top[x] = fmaxf(fmaxf(top[x], sc[x][1][1]), sc[x][1][2]);
            top[x] = fmaxf(top[x], sc[x][1][3]);
            most = fmaxf(most, top[x]);
        }
        if (unset || __any(most > 8.f)) {
#pragma unroll
            for (int x = 0; x < QB; ++x) {
                const float t = col_max(top[x]);
                const bool fresh = mrun[x] == -INFINITY;
                const float up = !fresh ? fmaxf(t, 0.f) : t == -INFINITY ? 0.f : t;
                mrun[x] = fresh ? t : mrun[x] + up;
                const float corr = __builtin_amdgcn_exp2f(fresh ? 0.f : -up);
                lsum[x] *= corr;
#pragma unroll
                for (int c = 0; c < DB; ++c) acc[x][c] *= corr;
#pragma unroll
                for (int t2 = 0; t2 < 2; ++t2) sc[x][t2] -= up;
            }
            bool none = false;
#pragma unroll
            for (int x = 0; x < QB; ++x) none |= mrun[x] == -INFINITY;
            unset = __any(none);
        }
    };
    auto weigh = [&](int x) {
        float pr[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) pr[e] = __builtin_amdgcn_exp2f(sc[x][e >> 2][e & 3]);
        p[x] = __builtin_bit_cast(f16x8, u32x4{mx4_pack_f16x2(pr[0], pr[1]), mx4_pack_f16x2(pr[2], pr[3]),
                                               mx4_pack_f16x2(pr[4], pr[5]), mx4_pack_f16x2(pr[6], pr[7])});
    };
    auto sum = [&](int x) { lsum[x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, p[x], lsum[x], 0, 0, 0); };
    // step m of 4 VL: a lane's 8 values of V to LDS as fp16
    auto take_v = [&](uint32_t v_in, int m) {
        v_store(v_in, m / 4, m % 4, mx4_to_f16(vc[m / 4][m % 4], __uint_as_float((uint32_t)vs[m / 4] << 23)));
    };
    // Blocks of V that fp16 does not hold (outside its range, or NaN) become zeros in LDS; odd says that
    // there are some.  add_odd gives the queries that see their keys these products in fp32, once the block's
    // scores are settled.  (Blocks of zeros have the lowest scale and are in order.)
    bool odd = false;
    auto odd_v = [&](uint32_t v_in) {
        bool any = false;
#pragma unroll
        for (int j = 0; j < VL; ++j) any |= mx4_odd(vs[j]);
        odd = __any(any);
        if (!odd) return;
        any = false;
#pragma unroll
        for (int j = 0; j < VL; ++j)
            if (mx4_odd(vs[j])) {
                any |= vs[j] == kMxNaN || (vc[j][0] | vc[j][1] | vc[j][2] | vc[j][3]) != 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) v_store(v_in, j, e, u32x4{0u, 0u, 0u, 0u});
            }
        odd = __any(any);
    };
    auto add_odd = [&](int kb) {
#pragma unroll 1
        for (int key = 0; key < kKeyBlock; ++key) {
            const int64_t row = row_of(kb + key);
            float pr[QB];   // the lane's queries': of lane (key % 16) / 4, scores key / 16, key % 4
#pragma unroll
            for (int x = 0; x < QB; ++x) {
                float s = sc[x][0][0];
#pragma unroll
                for (int e = 1; e < 8; ++e) s = 4 * (key >> 4) + (key & 3) == e ? sc[x][e >> 2][e & 3] : s;
                pr[x] = __builtin_amdgcn_exp2f(__shfl(s, 16 * ((key & 15) >> 2) + l16));
            }
#pragma unroll
            for (int c = 0; c < NB; ++c) {
                const int byte = gload1(vp.scales + row * NB + c);
                if (!mx4_odd(byte)) continue;
#pragma unroll
                for (int h = 0; h < 2; ++h) {   // dims 32 c + 16 h + 4 lg ..
                    const uint8_t* at = vp.codes + row * CB + 16 * c + 8 * h + 2 * lg;
                    const f32x4 v = mx4_to_f32(gload1(at) | gload1(at + 1) << 8, byte);
#pragma unroll
                    for (int x = 0; x < QB; ++x)
                        if (kb + key <= vis0 + step_row(x, lane)) acc[x][2 * c + h] += v * pr[x];
                }
            }
        }
    };
    f16x8 vv[kAhead + 1];   // V operands, read kAhead 16-dim blocks ahead of the products

    if constexpr (!kPipe) {
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            const int kb = k0 + i * kStride;
            // the block after it (past the last one: row R - 1 once more, one cache line)
            const int kb_next = i + 1 < n ? kb + kStride : R;
            const Place next = place_of(kb_next);
            // registers: no address of the lane is kept from one pass to the next
            int ln = lane;
            uint32_t v_in = v_in0, v_out = v_out0;
            asm volatile("" : "+v"(ln), "+v"(v_in), "+v"(v_out));
            read_q(0, ln);
            ordered();
#pragma unroll
            for (int m = 0; m < 4 * VL; ++m) take_v(v_in, m);
            odd_v(v_in);
            wave_lds_order();   // other lanes read these rows
            load_v(kb_next, next, ln);
            ordered();
            __builtin_amdgcn_s_setprio(1);
            score(0, ln);
            ordered();
            __builtin_amdgcn_s_setprio(0);
            load_k(kb_next, next, ln);   // into the registers that the products have read
#pragma unroll
            for (int c = 0; c < kAhead; ++c) vv[c] = v_op(v_out, c);
            ordered();
            settle(kb, ln);
            if (odd) add_odd(kb);
#pragma unroll
            for (int x = 0; x < QB; ++x) weigh(x), sum(x);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int c = 0; c < DB; ++c) {
                if (c + kAhead < DB) vv[(c + kAhead) % (kAhead + 1)] = v_op(v_out, c + kAhead);
                ordered();
#pragma unroll
                for (int x = 0; x < QB; ++x)
                    acc[x][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv[c % (kAhead + 1)], p[x], acc[x][c], 0, 0, 0);
                ordered();
            }
            __builtin_amdgcn_s_setprio(0);
            wave_lds_order();   // the next block takes this one's place
        }
    } else if (n > 0) {
        auto values = [&](int c) {
#pragma unroll
            for (int x = 0; x < QB; ++x)
                acc[x][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv[c % (kAhead + 1)], p[x], acc[x][c], 0, 0, 0);
        };
        {
            const int kb_next = n > 1 ? k0 + kStride : R;
            const Place next = place_of(kb_next);
#pragma unroll
            for (int m = 0; m < 4 * VL; ++m) take_v(v_in0, m);
            odd_v(v_in0);
            load_v(kb_next, next, lane);
            read_q(0, lane);
#pragma unroll
            for (int x = 0; x < QB; ++x) score(x, lane);
            fence();
            load_k(kb_next, next, lane);
            settle(k0, lane);
            if (odd) add_odd(k0);
        }
        // In each pass the probabilities and products of a block go with the next one's scores and V: the matrix
        // units work on one while the vector units work on the other.
#pragma unroll 1
        for (int i = 0; i + 1 < n; ++i) {
            const int kb = k0 + (i + 1) * kStride;   // the next block; K and V are in registers or on their way
            const int kb_next = i + 2 < n ? kb + kStride : R;
            const Place next = place_of(kb_next);
            int ln = lane;
            const uint32_t flip = i & 1 ? kBuf : 0;
            uint32_t v_in = v_in0 + (kBuf - flip), v_out = v_out0 + flip;
            asm volatile("" : "+v"(ln), "+v"(v_in), "+v"(v_out));
            // the two waves of a SIMD (w and w + 4) take turns in coming first: with the older one always
            // first it ended its keys a quarter earlier and left the other one alone
            if ((i ^ (w >> 2)) & 1) __builtin_amdgcn_s_setprio(2);
            else __builtin_amdgcn_s_setprio(0);
            wave_lds_order();   // other lanes wrote this block's rows
            read_q(0, ln);
            fence();
            weigh(0);
#pragma unroll
            for (int x = 0; x < QB; ++x) {
                if (x + 1 == QB) {
#pragma unroll
                    for (int c = 0; c < kAhead; ++c) vv[c] = v_op(v_out, c);
                }
                fence();
                score(x, ln);
                sum(x);
                if (x + 1 < QB) weigh(x + 1);
#pragma unroll
                for (int m = 0; m < 2 * QP + 1; ++m) {
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x2, 4, 0);
                    if (x + 1 < QB && m % 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                    if (x + 1 < QB && m == 2 * QP - 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                fence();
            }
            load_k(kb_next, next, ln);   // into the registers that the products have read
            fence();
#pragma unroll
            for (int c = 0; c < DB; ++c) {
                if (c + kAhead < DB) vv[(c + kAhead) % (kAhead + 1)] = v_op(v_out, c + kAhead);
                values(c);
                take_v(v_in, c);
                static_assert(DB == 4 * VL, "a step of V for each block of products");
                if (c + kAhead < DB) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
                for (int x = 0; x < QB; ++x) {
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x2, 3, 0);
                }
                fence();
            }
            odd_v(v_in);
            load_v(kb_next, next, ln);
            settle(kb, ln);
            if (odd) add_odd(kb);
        }
        __builtin_amdgcn_s_setprio(0);
        // the last block
        const uint32_t v_out = v_out0 + (n & 1 ? 0 : kBuf);
        wave_lds_order();
#pragma unroll
        for (int c = 0; c < kAhead; ++c) vv[c] = v_op(v_out, c);
#pragma unroll
        for (int x = 0; x < QB; ++x) weigh(x), sum(x);
#pragma unroll
        for (int c = 0; c < DB; ++c) {
            if (c + kAhead < DB) vv[(c + kAhead) % (kAhead + 1)] = v_op(v_out, c + kAhead);
            ordered();
            values(c);
            ordered();
        }
    }
    // combine the waves' states, one block of query rows after the other: each wave sums an
    // eighth of the dims
    const bool whole = d.splits == 1;
    float* po = st.ws + d.ws_off;
#pragma unroll
    for (int x = 0; x < QB; ++x) {
        __syncthreads();   // V, or the states of the block before
#pragma unroll
        for (int c = 0; c < DB; ++c) s_part[w][c][lane] = acc[x][c];
        if (lg == 0) s_ml[w][l16] = make_float2(mrun[x], lsum[x][0]);
        __syncthreads();
        const int mq = mw + x * kRows + l16;
        float mx = -INFINITY;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) mx = fmaxf(mx, s_ml[k][l16].x);
        auto weight = [&](int k) {
            const float m = s_ml[k][l16].x;
            return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mx);
        };
        float wt[kWaves], L = 0.f;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            wt[k] = weight(k);
            L += wt[k] * s_ml[k][l16].y;
        }
        // split partials: O / sum in fp16 (attn_merge_kernel; a split that sees no key of a row
        // is zeros with a maximum of -inf), else the bf16 output
        const float inv = L == 0.f && !whole ? 0.f : 1.f / L;
        const int64_t at = ((int64_t)sp * st.Hkv + g) * M + mq;
        for (int c = w; c < DB && mq < M; c += kWaves) {   // dims 16 c + 4 lg .. + 3
            f32x4 O = s_part[0][c][lane] * wt[0];
#pragma unroll
            for (int k = 1; k < kWaves; ++k) O += s_part[k][c][lane] * wt[k];
            O *= inv;
            if (whole) {
                const int i = mq >> g_shift;
                uint16_t* orow = o + ((int64_t)(d.q_row0 + i) * st.Hq + g * G + (mq - i * G)) * D;
                *reinterpret_cast<uint2*>(orow + 16 * c + 4 * lg) = make_uint2(pack_bf16x2(O[0], O[1]), pack_bf16x2(O[2], O[3]));
            } else {
                uint16_t* orow = reinterpret_cast<uint16_t*>(po) + at * D;
                *reinterpret_cast<uint2*>(orow + 16 * c + 4 * lg) = make_uint2(mx4_pack_f16x2(O[0], O[1]), mx4_pack_f16x2(O[2], O[3]));
            }
        }
        if (!whole && w == 0 && lg == 0 && mq < M)
            *reinterpret_cast<float2*>(po + (int64_t)d.splits * st.Hkv * M * (D / 2) + at * 2) =
                make_float2(mx == -INFINITY && L != 0.f ? 0.f : mx, L);   // a NaN sum keeps its weight
    }
}

}  // namespace

hipError_t launch_attn_mx4(const DevState& st, const AttnBatch& b, int query_blocks, const void* q, void* o, hipStream_t stream,
                           const KTimer& kt) {
    const uint16_t* qq = static_cast<const uint16_t*>(q);
    uint16_t* oo = static_cast<uint16_t*>(o);
    return by_size<AttnBatchT>(b, [&](const auto& bb) {
        constexpr int N = sizeof(bb.d) / sizeof(bb.d[0]);
        WgStart<N> start{};
        const dim3 grid = place_workgroups(b.count, &start, [&](int i) {
            return mx4_groups(st.G * b.d[i].n_q, kRows * query_blocks) * b.d[i].splits * st.Hkv;
        });
        auto go = [&](auto kernel) {
            const dim3 block(64 * kWaves);
            return launch_kernel(kernel, grid, block, {stream, kt.start, kt.stop}, st, bb, start, qq, oo);
        };
        auto sized = [&](auto dim) {
            constexpr int D = decltype(dim)::value;
            switch (query_blocks) {
                case 1: return go(attn_mx4_kernel<D, 1, N>);
                case 2: return go(attn_mx4_kernel<D, 2, N>);
                case 3: return go(attn_mx4_kernel<D, 3, N>);
                default: return hipErrorInvalidValue;
            }
        };
        if (st.D == 128) return sized(std::integral_constant<int, 128>{});
        if (st.D == 64) return sized(std::integral_constant<int, 64>{});
        return hipErrorInvalidValue;
    });
}

}  // namespace a2t
