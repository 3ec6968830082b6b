// Causal attention of a step's rows over rows held in 4 bits, for many query rows (gfx950).
//
//   attn_mx4_rows  one workgroup = (key split, RW x 32 query rows, KV head, stream),
//                  2 RW waves: a wave has 32 query rows; two groups of RW waves take the split's
//                  stages of keys in turn, and their states are combined in LDS at the end.
//
// The products are attn_mx4's (attn_mx4.hip), 32 by 32: a product holds up the vector units for
// ~20 cycles whatever its size (32x32x16 f16 adds 17 to 19 to a run of vector operations and takes 33 by itself,
// 16x16x32 adds 14 and takes 17), so that larger ones leave them more.  V is unpacked once a workgroup and stage,
// each wave its share, not once a wave.  Two of a query's three parts stay in registers; the third is read from LDS for
// each block.
// Bounds: vector operations (~105 a wave and block of 32 x 32, exponentials and their roundings half of them),
// products and what neither hides: 54 % and 42 % of the cycles of 1,024 rows onto 16,384 keys, at a clock that
// power holds at 1.85 to 2.0 GHz.  That launch takes 274 to 317 us, card by card, attn_mx4's waves of 48 rows 338 where it
// takes 274 (with two parts a query 251 to 283).
#include "a2t_internal.h"
#include "launch.h"
#include "mx4_device.h"

#include <math.h>

#include <type_traits>

namespace a2t {
namespace {

constexpr int kRows = 32;        // query rows of a wave
constexpr int kKeys = 32;        // keys of a block
constexpr int kGroups = 2;       // groups of waves that share a stage's V

// V in LDS: a key's 16-byte chunk c is at c ^ f(key): neither the four keys x four blocks (head dim
// 64: eight x two) of a store nor the four keys x four chunks of half a transposed read share banks.
template <int D>
__device__ __forceinline__ int v_chunk(int key, int c) {
    const int y = D == 128 ? key & 3 : (key >> 1) & 3;
    return key * (D / 8) + (c ^ (y | 4 * (D == 128 ? y : y & 1)));
}

// Lane l of a wave is (column l % 32, half h = l / 32).
//   scores   S^T[32 keys x 32 queries]: A = K, lane: key l % 32, 32 dims: block h of each 64;
//            B = Q^T, lane: query l % 32, the same dims; scales: the blocks'.  The lane gets keys
//            8 i + 4 h + e of its query.
//   values   O^T[32 dims x 32 queries]: 16 keys at a time, contracted in the order in which the
//            scores lie in a lane, keys 4 h + e and 8 + 4 h + e; the lane gets dims 8 i + 4 h + e of each 32.
template <int D, int RW, int N>
__global__ __launch_bounds__(64 * RW * kGroups, 2) void attn_mx4_rows_kernel(DevState st, AttnBatchT<N> b, WgStart<N> start,
                                                                            const uint16_t* q, uint16_t* o) {
    constexpr int NB = D / kMxBlock;   // blocks of a row: 32 dims of O each
    constexpr int CB = D / 2;          // bytes of a row's codes
    constexpr int KS = D / 64;         // products of 64 dims
    constexpr int SK = RW * 64 / NB, SB = SK / kKeys;   // keys, key blocks of a stage: a block of V a lane
    static_assert(SK % kKeys == 0, "whole key blocks");
    constexpr int kWaves = RW * kGroups;
    constexpr int kBuf = SK * D * 2;   // bytes of a stage's V
    constexpr int kPad = kMxBlock + 4;   // a block's floats in LDS: 16 lanes' reads do not share banks
    constexpr int kVBytes = 2 * kGroups * kBuf, kQBytes = RW * kRows * NB * kPad * 4, kMem = kVBytes > kQBytes ? kVBytes : kQBytes;
    static_assert(RW * NB * 4096 <= kMem, "a group's states fit");
    // (V's chunks are found by exclusive or on their addresses: whole rows are aligned)
    __shared__ __align__(256) uint8_t s_mem[kMem];   // rotated rows; V of two stages a group; at the end states
    __shared__ u32x4 s_q[RW][KS][64];     // third parts of the Q operands, their first 16 bytes
    __shared__ uint2 s_q2[RW][KS][64];    // ... and the other 8
    __shared__ float2 s_ml[RW][kRows];
    __shared__ int s_odd[2][kWaves], s_any;   // a stage's share, any stage has blocks that fp16 does not hold

    int wg;
    const AttnDesc d = b.d[stream_of(start, b.count, &wg)];
    const int G = st.G, M = G * d.n_q, R = d.R;
    const int groups = (M + RW * kRows - 1) / (RW * kRows);
    auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };   // divisions run on the vector ALU
    // linear block (split, query group, KV head), heads fastest: the workgroups of a head
    // share an XCD's L2 when the head count divides the 8 XCDs
    const int y = uniform(wg / st.Hkv), g = wg - y * st.Hkv;
    const int sp = uniform(y / groups), grp = groups - 1 - (y - sp * groups);
    if (sp >= d.splits) return;
    const int w = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, l16 = lane & 15, h = lane >> 5;
    const int kg = w / RW, rw = w - kg * RW;
    const int mw = (grp * RW + rw) * kRows;   // the wave's first query row
    const int vis0 = R - d.n_q;
    const int qi = min(mw + l32, M - 1) / G;   // step row of the lane's query (past M: that of row M - 1)
    const int t0 = sp * d.tile_q + min(sp, d.tile_r), t1 = t0 + d.tile_q + (sp < d.tile_r ? 1 : 0);
    auto end_of = [&](int m) { return min(vis0 + uniform((min(M, m) - 1) / G) + 1, t1 * kTileKeys); };
    const int k0 = t0 * kTileKeys;
    const int see_to = min(vis0 + qi, t1 * kTileKeys - 1);       // last key of the lane's query
    const int see_all = min(vis0 + uniform(min(mw, M - 1) / G) + 1, t1 * kTileKeys);   // keys that all the wave's queries see
    const int end = end_of((grp + 1) * RW * kRows);              // of the workgroup's keys
    const int end_w = mw < M ? end_of(mw + kRows) : 0;           // of the wave's
    const int passes = end > k0 ? ((end - k0 + SK - 1) / SK + kGroups - 1) / kGroups : 0;

    const int kept = d.kept, head = d.head, ring_rows = st.unit_rows;
    const Mx4Pool kp = mx4_pool(st, st.k_unit), vp = mx4_pool(st, st.v_unit);
    const int64_t ring0 = mx4_ring_row(st, b.layer, d.s, g), kept0 = mx4_kept_row(st, b.layer, d.s, g);
    // Where key j's row is (keys past R: row R - 1, and masked): a row of the kept region or of the ring.
    struct Row {
        bool in_kept;
        uint32_t at;
    };
    auto row_of = [&](int j) {
        j = min(j, R - 1);
        const uint32_t slot = head + (j - kept);
        return Row{j < kept, j < kept ? (uint32_t)j : min(slot, slot - ring_rows)};
    };
    // (selected without branches: a value loaded on one side of a branch would be waited for there, and the addresses
    // of a run of rows took 330 cycles a block, of ~1,500)
    auto pick = [](const Row& r, uint8_t* of_kept, uint8_t* of_ring, uint32_t row_bytes) {
        const uint64_t base = r.in_kept ? reinterpret_cast<uint64_t>(of_kept) : reinterpret_cast<uint64_t>(of_ring);
        return reinterpret_cast<const uint8_t*>(base + (uint64_t)r.at * row_bytes);
    };
    uint8_t* const k_ring = kp.codes + ring0 * CB + 16 * h;
    uint8_t* const k_kept = kp.codes + kept0 * CB + 16 * h;
    uint8_t* const ks_ring = kp.scales + ring0 * NB + (KS == 1 ? h : 0);
    uint8_t* const ks_kept = kp.scales + kept0 * NB + (KS == 1 ? h : 0);
    uint8_t* const v_ring = vp.codes + ring0 * CB + 16 * (lane % NB);
    uint8_t* const v_kept = vp.codes + kept0 * CB + 16 * (lane % NB);
    uint8_t* const vs_ring = vp.scales + ring0 * NB + lane % NB;
    uint8_t* const vs_kept = vp.scales + kept0 * NB + lane % NB;

    u32x4 kc[KS], vc;
    uint32_t ks;          // the K row's scale bytes, the lane's one of each 64 dims in bytes 0 and 2 once shifted
    int vs;               // the V block's
    auto load_k = [&](int kb) {
        const Row r = row_of(kb + l32);
        const uint8_t* const p = pick(r, k_kept, k_ring, CB);
#pragma unroll
        for (int t = 0; t < KS; ++t) kc[t] = gload16(p + 32 * t);
        const uint8_t* const ps = pick(r, ks_kept, ks_ring, NB);
        ks = KS == 1 ? gload1(ps) : gload4(ps);
    };
    // the wave's share of a stage's V: keys (64 / NB) rw .., a lane a block
    auto load_v = [&](int kb) {
        const Row r = row_of(kb + (64 * rw + lane) / NB);
        vc = gload16(pick(r, v_kept, v_ring, CB));
        vs = gload1(pick(r, vs_kept, vs_ring, NB));
    };
    auto stage_key = [&](int i) { return k0 + (i * kGroups + kg) * SK; };   // first key of the group's stage i
    auto lds_barrier = [] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    };

    // Q^T operands.  First the rows, rotated and scaled by scale * log2(e), to LDS: a thread
    // takes 8 dims of the lower half and their partners of the upper one.  Rows past M read row
    // M - 1 and are never stored.
    constexpr int kItems = RW * kRows * (D / 16), kTurns = (kItems + 64 * kWaves - 1) / (64 * kWaves);
    float* const s_rows = reinterpret_cast<float*>(s_mem);
#pragma unroll
    for (int turn = 0; turn < kTurns; ++turn) {
        const int x = turn * 64 * kWaves + (int)threadIdx.x;
        const int r = x / (D / 16), d0 = (x - r * (D / 16)) * 8;
        const int m = min(grp * RW * kRows + r, M - 1), i = m / G;
        const uint16_t* qp = q + ((int64_t)(d.q_row0 + i) * st.Hq + g * G + (m - i * G)) * D + d0;
        const float4* cp = reinterpret_cast<const float4*>(
            st.rope + ((int64_t)d.s * st.max_step_rows + d.rope_row0 + i) * (D / 2) + d0);
        const u32x4 a = *reinterpret_cast<const u32x4*>(qp), a2 = *reinterpret_cast<const u32x4*>(qp + D / 2);
        float4 cs[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) cs[e] = cp[e];
        if (turn == 0) {
            __builtin_amdgcn_sched_barrier(0);
            load_v(stage_key(0));   // K and V behind them: loads return in order
            load_k(stage_key(0));
        }
        if (kItems % (64 * kWaves) == 0 || x < kItems)
            mx4_rotate(a, a2, cs, st.scale_log2e, s_rows + (r * NB + d0 / kMxBlock) * kPad + d0 % kMxBlock,
                       s_rows + (r * NB + (d0 + D / 2) / kMxBlock) * kPad + (d0 + D / 2) % kMxBlock);
    }
    __syncthreads();
    // Then the wave's operands, a lane a block of each 64 dims.
    // first and second part; the third is in LDS, where the wave reads it for each block (registers)
    i32x8 qh[KS], ql[KS];
    int qs[KS];             // the first part's scales
    u32x6 q3[KS];
#pragma unroll
    for (int t = 0; t < KS; ++t) {
        u32x6 part[kMxQueryParts];
        qs[t] = mx4_query(s_rows + ((rw * kRows + l32) * NB + 2 * t + h) * kPad, part);
        qh[t] = mx4_operand(part[0]), ql[t] = mx4_operand(part[1]);
        q3[t] = part[2];
    }
    __syncthreads();   // V takes the rows' place
    if (kg == 0) {   // (both groups of waves have the same rows)
#pragma unroll
        for (int t = 0; t < KS; ++t) {
            s_q[rw][t][lane] = u32x4{q3[t][0], q3[t][1], q3[t][2], q3[t][3]};
            s_q2[rw][t][lane] = make_uint2(q3[t][4], q3[t][5]);
        }
    }
    __syncthreads();

    // V in LDS: where the lane's block e (of 8 dims) of its first row goes, and the lane's
    // place in the transposed reads (16 lanes read 8 bytes each of four keys' 32 bytes).  The
    // swizzle and e (the 32-dim block c) touch the same bits of the address.
    const uint32_t s_v = lds_addr(s_mem) + kg * (2 * kBuf);
    const uint32_t v_in0 = s_v + 16 * v_chunk<D>((64 * rw + lane) / NB, 4 * (lane % NB));
    const uint32_t v_out0 = s_v + 16 * v_chunk<D>(4 * h + (l16 >> 2), 2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1)) + 8 * (l16 & 1);
    auto v_op = [&](uint32_t v_out, int c, int j) {   // 16 keys j of a key block, 32 dims c
        i16x4 x[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
            x[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(uintptr_t)(
                (v_out ^ (64u * c)) + (16 * j + 8 * t) * D * 2));
        return __builtin_bit_cast(f16x8, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // The wave's share of a stage's V to LDS as fp16; blocks that fp16 does not hold become zeros there
    // and the stage odd.  (Blocks of zeros have the lowest scale and are in order.)
    auto take_v = [&](auto odd, int buf) {
        const uint32_t v_in = v_in0 + buf * kBuf;
        auto store = [&](int e, const u32x4& x) {
            *reinterpret_cast<__attribute__((address_space(3))) u32x4*>((uintptr_t)(v_in ^ (16u * e))) = x;
        };
#pragma unroll
        for (int e = 0; e < 4; ++e) store(e, mx4_to_f16(vc[e], __uint_as_float((uint32_t)vs << 23)));
        if constexpr (decltype(odd)::value)
            if (lane == 0) s_odd[buf][w] = 0;
        if (__any(mx4_odd(vs)) && mx4_odd(vs)) {
            if (vs == kMxNaN || (vc[0] | vc[1] | vc[2] | vc[3]) != 0) s_odd[buf][w] = s_any = 1;
#pragma unroll
            for (int e = 0; e < 4; ++e) store(e, u32x4{0u, 0u, 0u, 0u});
        }
    };

    f32x16 acc[NB], sc;
    // ref: mrun, or what every score in fp32 reaches before there was one (a score of -infinity has no weight)
    constexpr float kLowest = -3.40282347e38f;
    float mrun = -INFINITY, ref = kLowest, lsum[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < NB; ++c) acc[c] = f32x16{};
    auto score = [&] {
        const int k_scale = KS == 1 ? ks : ks >> (8 * h);
        sc = f32x16{};
        auto dims = [&](auto x) {
            constexpr int t = decltype(x)::value;
            const i32x8 kv = {(int)kc[t][0], (int)kc[t][1], (int)kc[t][2], (int)kc[t][3], 0, 0, 0, 0};
            const u32x4 a = s_q[rw][t][lane];
            const uint2 a2 = s_q2[rw][t][lane];
            const i32x8 q3 = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)a2.x, (int)a2.y, 0, 0};
            sc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kv, qh[t], sc, 4, 2, 2 * t, k_scale, 0, qs[t]);
            sc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kv, ql[t], sc, 4, 2, 2 * t, k_scale, 0, mx4_query_scale(qs[t], 1));
            sc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kv, q3, sc, 4, 2, 2 * t, k_scale, 0, mx4_query_scale(qs[t], 2));
        };
        dims(std::integral_constant<int, 0>());
        if constexpr (KS == 2) dims(std::integral_constant<int, 1>());
        asm volatile("" : "+v"(sc));   // (the compiler would put them off to where they are read)
    };
    // hides what a row does not see, and moves the reference, lazily: the first block with a score sets it, and it is
    // raised, and the running sums rescaled, only when a block exceeds it by more than 2^8
    auto settle = [&](int kb, bool first) {
        if (kb + kKeys > see_all) {   // some row does not see every key, or the split ends
            const int see = see_to - kb - 4 * h;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r >> 2) + (r & 3) > see) sc[r] = -INFINITY;
        }
        float half_top[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            half_top[x] = fmaxf(fmaxf(sc[8 * x], sc[8 * x + 1]), sc[8 * x + 2]);
            half_top[x] = fmaxf(fmaxf(half_top[x], sc[8 * x + 3]), sc[8 * x + 4]);
            half_top[x] = fmaxf(fmaxf(half_top[x], sc[8 * x + 5]), sc[8 * x + 6]);
        }
        const float top = fmaxf(fmaxf(fmaxf(half_top[0], sc[7]), half_top[1]), sc[15]);
        if (first || __any(top >= ref + 8.f)) {   // (the lowest plus 8 is the lowest)
            const auto z = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            const float t = fmaxf(mrun, fmaxf(__uint_as_float(z[0]), __uint_as_float(z[1])));
            const float corr = first ? 0.f : __builtin_amdgcn_exp2f(ref - t);
            if (first || t >= ref) {
                mrun = t;
                lsum[0] *= corr, lsum[1] *= corr;
#pragma unroll
                for (int c = 0; c < NB; ++c) acc[c] *= corr;
                ref = fmaxf(t, kLowest);
            }
        }
    };
    // gives the queries that see their keys the products of odd blocks, in fp32
    auto add_odd = [&](int kb) {
#pragma unroll 1
        for (int key = 0; key < kKeys; ++key) {
            const Row r = row_of(kb + key);
            const uint8_t* const codes = pick(r, v_kept, v_ring, CB) - 16 * (lane % NB);
            const uint8_t* const scales = pick(r, vs_kept, vs_ring, NB) - lane % NB;
            float s = sc[0];   // of lane half key / 4 % 2, element 4 (key / 8) + key % 4
#pragma unroll
            for (int r = 1; r < 16; ++r) s = 4 * (key >> 3) + (key & 3) == r ? sc[r] : s;
            const float pr = __builtin_amdgcn_exp2f(__shfl(s, 32 * ((key >> 2) & 1) + l32) - ref);
            if (kb + key > see_to) continue;
#pragma unroll
            for (int c = 0; c < NB; ++c) {
                const int byte = gload1(scales + c);
                if (!mx4_odd(byte)) continue;
#pragma unroll
                for (int i = 0; i < 4; ++i) {   // dims 32 c + 8 i + 4 h ..
                    const uint8_t* at = codes + 16 * c + 4 * i + 2 * h;
                    const f32x4 v = mx4_to_f32(gload1(at) | gload1(at + 1) << 8, byte);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[c][4 * i + e] += v[e] * pr;
                }
            }
        }
    };

    // The workgroup's keys: in each pass a wave has its block's probabilities, the next block's scores and its
    // block's products, and unpacks its share of the next stage's V.  Without `odd` the blocks that fp16
    // does not hold are left out; where there were some the workgroup begins again with it.  (Both in one loop:
    // the compiler copies all sums from block to block, 421 us instead of 320.)
    auto run = [&](auto odd) {
        mrun = -INFINITY, ref = kLowest, lsum[0] = lsum[1] = 0.f;
#pragma unroll
        for (int c = 0; c < NB; ++c) acc[c] = f32x16{};
        take_v(odd, 0);
        load_v(stage_key(1));
        score();
        load_k(SB > 1 ? stage_key(0) + kKeys : stage_key(1));
        asm volatile("" : "+v"(ks));   // (a byte on its way is not extended at the end of each pass)
        settle(stage_key(0), true);
        lds_barrier();
        int i = 0;
#pragma unroll 1
        for (; stage_key(i) < end_w; ++i) {
            uint32_t v_out = v_out0 + (i & 1) * kBuf;
#pragma unroll
            for (int blk = 0; blk < SB; ++blk, v_out += kKeys * D * 2) {
                const int kb = stage_key(i) + blk * kKeys;
                // the block after the next (past the last one: row R - 1)
                const int after = blk + 2 < SB ? kb + 2 * kKeys : stage_key(i + (SB > 1 ? 1 : 2)) + (SB > 1 ? (blk + 2 - SB) * kKeys : 0);
                if constexpr (decltype(odd)::value) {
                    int any = 0;
#pragma unroll
                    for (int x = 0; x < RW; ++x) any |= s_odd[i & 1][kg * RW + x];
                    if (uniform(any)) add_odd(kb);
                }
                f16x8 p[2], vv[2][NB];
#pragma unroll
                for (int c = 0; c < NB; ++c) vv[0][c] = v_op(v_out, c, 0);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    u32x4 x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t two = mx4_pack_f16x2(__builtin_amdgcn_exp2f(sc[8 * j + 2 * e] - ref), __builtin_amdgcn_exp2f(sc[8 * j + 2 * e + 1] - ref));
                        lsum[j] = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, two), f16x2{(_Float16)1.f, (_Float16)1.f}, lsum[j], false);
                        x[e] = two;
                    }
                    p[j] = __builtin_bit_cast(f16x8, x);
                }
                asm volatile("" : "+v"(p[0]), "+v"(p[1]), "+v"(lsum[0]), "+v"(lsum[1]));   // before the scores: in their registers
                if (blk == 0 && i + 1 < passes) take_v(odd, (i & 1) ^ 1);
                score();
                load_k(after);   // the one needed first
                if (blk == 0) load_v(stage_key(i + 2));
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int c = 0; c < NB; ++c) {
                        if (j == 0) {
                            vv[1][c] = v_op(v_out, c, 1);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                        acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vv[j][c], p[j], acc[c], 0, 0, 0);
                    }
                settle(blk + 1 < SB ? kb + kKeys : stage_key(i + 1), false);
            }
            lds_barrier();
        }
#pragma unroll 1
        for (; i < passes; ++i) {   // stages that other waves see
            if (i + 1 < passes) take_v(odd, (i & 1) ^ 1);
            load_v(stage_key(i + 2));
            lds_barrier();
        }
        __syncthreads();
    };
    if (passes > 0) {
        if (threadIdx.x == 0) s_any = 0;
        __syncthreads();
        run(std::false_type());
        if (s_any) {
            __syncthreads();
            load_v(stage_key(0));
            load_k(stage_key(0));
            run(std::true_type());
        }
    }
    float L = lsum[0] + lsum[1];
    {
        const auto z = __builtin_amdgcn_permlane32_swap(__float_as_uint(L), __float_as_uint(L), false, false);
        L = __uint_as_float(z[0]) + __uint_as_float(z[1]);
    }
    // combine the groups' states: the second one hands its to the first
    f32x4(&s_part)[RW][NB][4][64] = *reinterpret_cast<f32x4(*)[RW][NB][4][64]>(s_mem);
    if (kg == 1) {
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                s_part[rw][c][i][lane] = f32x4{acc[c][4 * i], acc[c][4 * i + 1], acc[c][4 * i + 2], acc[c][4 * i + 3]};
        if (h == 0) s_ml[rw][l32] = make_float2(mrun, L);
    }
    __syncthreads();
    const int mq = mw + l32;
    if (kg == 1 || mq >= M) return;
    {
        const float2 ml = s_ml[rw][l32];
        const float mx = fmaxf(mrun, ml.x);
        const float a = mrun == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mrun - mx);
        const float a2 = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - mx);
        mrun = mx;
        L = L * a + ml.y * a2;
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 x = s_part[rw][c][i][lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[c][4 * i + e] = acc[c][4 * i + e] * a + x[e] * a2;
            }
    }
    // split partials: O / sum in fp16 (attn_merge_kernel; a split that sees no key of a row
    // is zeros with a maximum of -inf), else the bf16 output
    const bool whole = d.splits == 1;
    float* po = st.ws + d.ws_off;
    const float inv = L == 0.f && !whole ? 0.f : 1.f / L;
    const int64_t at = ((int64_t)sp * st.Hkv + g) * M + mq;
    uint16_t* const orow = whole ? o + ((int64_t)(d.q_row0 + qi) * st.Hq + g * G + (mq - qi * G)) * D : reinterpret_cast<uint16_t*>(po) + at * D;
#pragma unroll
    for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // dims 32 c + 8 i + 4 h ..
            const float x0 = acc[c][4 * i] * inv, x1 = acc[c][4 * i + 1] * inv, x2 = acc[c][4 * i + 2] * inv, x3 = acc[c][4 * i + 3] * inv;
            *reinterpret_cast<uint2*>(orow + 32 * c + 8 * i + 4 * h) =
                whole ? make_uint2(pack_bf16x2(x0, x1), pack_bf16x2(x2, x3)) : make_uint2(mx4_pack_f16x2(x0, x1), mx4_pack_f16x2(x2, x3));
        }
    if (!whole && h == 0)
        *reinterpret_cast<float2*>(po + (int64_t)d.splits * st.Hkv * M * (D / 2) + at * 2) =
            make_float2(mrun == -INFINITY && L != 0.f ? 0.f : mrun, L);   // a NaN sum keeps its weight
}

}  // namespace

hipError_t launch_attn_mx4_rows(const DevState& st, const AttnBatch& b, int row_waves, const void* q, void* o, hipStream_t stream,
                                const KTimer& kt) {
    const uint16_t* qq = static_cast<const uint16_t*>(q);
    uint16_t* oo = static_cast<uint16_t*>(o);
    return by_size<AttnBatchT>(b, [&](const auto& bb) {
        constexpr int N = sizeof(bb.d) / sizeof(bb.d[0]);
        WgStart<N> start{};
        const dim3 grid = place_workgroups(b.count, &start, [&](int i) {
            return mx4_groups(st.G * b.d[i].n_q, kRows * row_waves) * b.d[i].splits * st.Hkv;
        });
        auto go = [&](auto kernel) {
            const dim3 block(64 * row_waves * kGroups);
            return launch_kernel(kernel, grid, block, {stream, kt.start, kt.stop}, st, bb, start, qq, oo);
        };
        auto sized = [&](auto dim) {
            constexpr int D = decltype(dim)::value;
            if (row_waves == 2) return go(attn_mx4_rows_kernel<D, 2, N>);
            if (row_waves == 4) return go(attn_mx4_rows_kernel<D, 4, N>);
            return hipErrorInvalidValue;
        };
        if (st.D == 128) return sized(std::integral_constant<int, 128>{});
        if (st.D == 64) return sized(std::integral_constant<int, 64>{});
        return hipErrorInvalidValue;
    });
}

}  // namespace a2t
