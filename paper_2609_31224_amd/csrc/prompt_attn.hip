// Causal attention over packed sequences, forward and gradients (gfx950).  Per query head and row i of
// a sequence, over the rows j <= i < until_j of the same sequence:
//   O_i = sum_j P_ij v_j,  P_ij = exp(scale q_i . k_j - lse_i),  lse_i = ln sum_j exp(scale q_i . k_j)
//   delta_i = dO_i . O_i,  dS_ij = P_ij (dO_i . v_j - delta_i)
//   dQ_i = scale sum_j dS_ij k_j,  dK_j = scale sum_i dS_ij q_i,  dV_j = sum_i P_ij dO_i
//
//   prompt_attn16, prompt_attn   forward (bf16, fp32): 128 packed query rows of a KV head a workgroup
//   prompt_dq                    dQ and delta, the same rows
//   prompt_dkv                   dK and dV: 128 keys a workgroup, every query row that sees them
//   prompt_join, prompt_add      sums of blocks that were split over workgroups
// The scores are computed again for each gradient (seven products where five would do): dQ summed over
// the key blocks would need sums in memory whose order changes from run to run, or a pass over as many
// partial sums as there are key blocks.
//
// Row m of a sequence is head m % G of a KV head's group at place m / G, so that the G heads share
// every key tile and a block's triangle at the diagonal is G times smaller.  Scores are S^T = K Q^T on 32 x
// 32 matrix instructions: a lane has 16 of 32 keys of its own query, a row's maximum needs one
// exchange between two lanes, and probabilities are the operand of O^T = V^T P^T as they lie in registers.
//
// Bound: the matrix units under the card's power (clock 1.9 to 2.0 GHz of 2.4; a library's product of
// 8,192^3 reaches 1.23 PFLOP/s) and, beside them, LDS reads and exponentials.  Measured, head dim 128,
// 32 heads on 8: forward of 16,384 rows 2.0 ms, 1.10 PFLOP/s; a ten-minute session of 13,200 rows under
// eviction 0.80 ms forward (0.94 PFLOP/s of visible pairs), dQ 1.05 ms (1.07), dK and dV 1.75 ms (0.85).  fp32,
// where the blocks fill the CUs (4,096 rows, the same heads): forward 0.74 of a library product's 154 TFLOP/s
// (1.20 ms at head dim 128, 0.60 at 64), dQ 0.80 and 0.79, dK and dV 0.78 and 0.80.
// Of the forms tried: tiles through registers instead of straight into LDS, 3.4 instead of 2.3 ms
// (the compiler took 296 registers, one wave a SIMD); scores a tile ahead of the exponentials, 2.3 ->
// 2.1; waves of 64 keys for dK and dV, one a SIMD, 1.25 ms instead of 0.86 at head dim 64 (at 128
// their sums alone are 256 registers and spill); priorities among a SIMD's waves, no change.
#include "launch.h"
#include "prompt_device.h"

#include <type_traits>

namespace a2t {
namespace prompt {
namespace {

// The key tiles of a block of queries at places first .. last: one or two runs of rows.
struct Runs {
    int start[2], end[2], tiles0, tiles;
    __device__ __forceinline__ void at(int t, int* lo, int* hi) const {
        const int second = t >= tiles0;
        *lo = start[second] + (t - (second ? tiles0 : 0)) * kTile;
        *hi = end[second];
    }
};
// Place and `until` of row r of a sequence's keys as the kernels read them.
__device__ __forceinline__ int2 key_place(const KeyRows& kv, int row0, int r) {
    return kv.meta ? kv.meta[row0 + r] : make_int2(r, kv.until[row0 + r]);
}
template <bool UNTIL>
__device__ __forceinline__ Runs key_runs(const KeyRows& kv, int row0, int n, int first, int last) {
    Runs r;
    r.start[0] = 0;
    r.end[0] = last + 1;
    r.start[1] = r.end[1] = 0;
    if (UNTIL && kv.meta) {   // lasting keys, then the passing ones that some query may still see
        const int all = uniform(kv.lasting[row0 + n - 1]), seen = uniform(kv.lasting[row0 + last]);
        r.end[0] = seen;
        r.start[1] = all + uniform(kv.first[row0 + first]);
        r.end[1] = all + (last + 1 - seen);
        if (r.end[1] < r.start[1]) r.end[1] = r.start[1];
    }
    r.tiles0 = (r.end[0] - r.start[0] + kTile - 1) / kTile;
    r.tiles = r.tiles0 + (r.end[1] - r.start[1] + kTile - 1) / kTile;
    return r;
}

// Which of keys lo .. lo + 63 of a tile (up to hi) some row of a wave's at places first .. last sees,
// by blocks of 32, and whether all rows see all of them.
struct Sees {
    bool block[2], all;
};
template <bool UNTIL>
__device__ __forceinline__ Sees sees(const int2* meta, int lo, int hi, int first, int last) {
    if constexpr (UNTIL) {
        const int lane = threadIdx.x & 63;
        const int2 m = meta[lane];
        const bool in = lo + lane < hi;
        const uint64_t some = __ballot(in && m.x <= last && m.y > first);
        return {(uint32_t)some != 0, (some >> 32) != 0, (bool)__all(in && m.x <= first && m.y > last)};
    } else {
        return {lo <= last, lo + 32 <= last, lo + kTile - 1 <= first};
    }
}
// Whether the query at place i sees key k of a tile.
template <bool UNTIL>
__device__ __forceinline__ bool visible(const int2* meta, int lo, int hi, int k, int i) {
    if constexpr (UNTIL) return lo + k < hi && meta[k].x <= i && i < meta[k].y;
    return lo + k <= i;
}

template <typename T, int D, bool UNTIL, int N>
__global__ __launch_bounds__(kThreads, (sizeof(T) * D <= 256 ? 2 : 1)) void prompt_attn_kernel(Args a, SeqTable<N> t) {
    using Tl = Tile<T, D>;
    constexpr int DB = Tl::DB;
    __shared__ __align__(1024) char s_k[2][Tl::BYTES];
    __shared__ __align__(1024) char s_v[2][Tl::BYTES];
    __shared__ int2 s_meta[2][UNTIL ? kTile : 1];

    const int g = blockIdx.x % a.Hkv, G = a.G;
    int sp = (int)(blockIdx.x / a.Hkv), place;   // split of the block's tiles
    const int y = sp / a.splits;
    sp -= y * a.splits;
    const int z = sequence_of(t, y, &place);
    const int n = t.rows[z], row0 = t.row0[z], M = G * n;
    const int m0 = ((M + kBlock - 1) / kBlock - 1 - place) * kBlock;   // the rows that see most come first
    const int base = uniform(m0 / G), rem = m0 - base * G;
    auto place_of = [&](int r) { return base + (int)(((uint32_t)(rem + r) * a.inv_g) >> 16); };   // of row m0 + r
    const int w = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
    const int rows = min(kBlock, M - m0);
    const bool busy = 32 * w < rows;
    const int r = min(32 * w + l32, rows - 1);
    const int i = place_of(r), hh = rem + r - (i - base) * G;
    const int i_first = uniform(place_of(min(32 * w, rows - 1))), i_last = uniform(place_of(min(32 * w + 31, rows - 1)));
    const Runs runs = key_runs<UNTIL>(a.kv, row0, n, base, uniform(place_of(rows - 1)));
    const int t0 = runs.tiles * sp / a.splits, t1 = runs.tiles * (sp + 1) / a.splits;

    const char* kp = static_cast<const char*>(a.kv.k) + ((int64_t)row0 * a.kv.k_stride + g * D) * sizeof(T);
    const char* vp = static_cast<const char*>(a.kv.v) + ((int64_t)row0 * a.kv.v_stride + g * D) * sizeof(T);
    int2 mm = {0, 0};
    auto load = [&](int tile) {
        int lo, hi;
        runs.at(tile, &lo, &hi);
        const int stage = tile & 1;
        Coming<T, D>::rows(kp, a.kv.k_stride * sizeof(T), lo, n - 1, w, lds_address(s_k[stage]));
        Coming<T, D>::rows(vp, a.kv.v_stride * sizeof(T), lo, n - 1, w, lds_address(s_v[stage]));
        if (UNTIL && threadIdx.x < kTile) mm = key_place(a.kv, row0, min(lo + (int)threadIdx.x, n - 1));
    };
    auto store = [&](int stage) {
        if (UNTIL && threadIdx.x < kTile) s_meta[stage][threadIdx.x] = mm;
    };
    if (t0 < t1) load(t0);

    u32x4 qop[Tl::STEPS];
    {
        const char* qp = static_cast<const char*>(a.q) + ((row0 + i) * a.q_stride + (g * G + hh) * D) * (int64_t)sizeof(T) + 16 * h;
#pragma unroll
        for (int s = 0; s < Tl::STEPS; ++s) qop[s] = *reinterpret_cast<const u32x4*>(qp + 32 * s);
    }
    if (t0 < t1) store(t0 & 1);

    // base-2 logarithms throughout: mref is the reference of the lane's row (its scaled scores less mref
    // are at most 8), sum of 2^(score - mref)
    const float c = a.scale_log2e;
    float mrun = -INFINITY, mref = 0.f, sum = 0.f;
    f32x16 acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[db][e] = 0.f;

    for (int tile = t0; tile < t1; ++tile) {
        const int stage = tile & 1;
        wait_tiles();
        __syncthreads();
        if (tile + 1 < t1) load(tile + 1);
        int lo, hi;
        runs.at(tile, &lo, &hi);
        const Sees what = sees<UNTIL>(s_meta[stage], lo, hi, i_first, i_last);
        if (busy && (what.block[0] || what.block[1])) {
            f32x16 s[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[b][e] = 0.f;
                if (what.block[b]) {
#pragma unroll
                    for (int k = 0; k < Tl::STEPS; ++k) mma_step<T>(row_operand<T, D>(s_k[stage], 32 * b + l32, k, h), qop[k], s[b]);
                }
            }
            if (!what.all) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (!visible<UNTIL>(s_meta[stage], lo, hi, 32 * b + 8 * (e >> 2) + 4 * h + (e & 3), i)) s[b][e] = -INFINITY;
            }
            float top = fmaxf(s[0][0], s[1][0]);
#pragma unroll
            for (int e = 1; e < 16; ++e) top = fmaxf(fmaxf(top, s[0][e]), s[1][e]);
            top = swap_max(top) * c;
            if (__any(top > mrun + 8.f)) {
                const float up = fmaxf(mrun, top), ref = up == -INFINITY ? 0.f : up;
                const float by = exp2_(mrun - ref);
                sum *= by;
#pragma unroll
                for (int db = 0; db < DB; ++db) acc[db] *= by;
                mrun = up;
                mref = ref;
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    s[b][e] = exp2_(__builtin_fmaf(s[b][e], c, -mref));
                    sum += s[b][e];
                }
                if (what.block[b]) mma_rows<D, T>(s_v[stage], 32 * b, s[b], acc);
            }
        }
        if (tile + 1 < t1) store(stage ^ 1);
    }

    if (32 * w + l32 >= rows) return;
    const float total = swap_sum(sum);
    if (a.splits > 1) {   // the split's own sums; prompt_join_kernel puts them together
        const int64_t at = ((int64_t)sp * a.total + row0 + i) * a.Hq + g * G + hh;
        if (h == 0) *reinterpret_cast<float2*>(a.part + (int64_t)a.splits * a.total * a.Hq * D + 2 * at) = make_float2(mrun, total);
        float* o = a.part + at * D + 4 * h;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int e = 0; e < 4; ++e) store4(o + 32 * db + 8 * e, acc[db][4 * e], acc[db][4 * e + 1], acc[db][4 * e + 2], acc[db][4 * e + 3]);
        return;
    }
    const float inv = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;   // a row without keys is zero
    const int64_t row = row0 + i;
    if (a.lse && h == 0) a.lse[(int64_t)(g * G + hh) * a.total + row] = (mref + __builtin_amdgcn_logf(total)) * kLn2;
    T* o = static_cast<T*>(a.o) + (row * a.Hq + g * G + hh) * D + 4 * h;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            store4(o + 32 * db + 8 * e, acc[db][4 * e] * inv, acc[db][4 * e + 1] * inv, acc[db][4 * e + 2] * inv, acc[db][4 * e + 3] * inv);
}

// The same for bf16, a tile ahead: the scores of the next tile run on the matrix units beside the
// exponentials of this one, and this one's products with V after them.  LDS reads are issued two
// groups ahead.
template <int D, bool UNTIL, int N>
__global__ __launch_bounds__(kThreads, 2) void prompt_attn16_kernel(Args a, SeqTable<N> t) {
    using T = bf16_t;
    using Tl = Tile<T, D>;
    constexpr int DB = Tl::DB, STEPS = Tl::STEPS;
    __shared__ __align__(1024) char s_k[2][Tl::BYTES];
    __shared__ __align__(1024) char s_v[2][Tl::BYTES];
    __shared__ int2 s_meta[2][UNTIL ? kTile : 1];

    const int g = blockIdx.x % a.Hkv, G = a.G;
    int sp = (int)(blockIdx.x / a.Hkv), place;   // split of the block's tiles
    const int y = sp / a.splits;
    sp -= y * a.splits;
    const int z = sequence_of(t, y, &place);
    const int n = t.rows[z], row0 = t.row0[z], M = G * n;
    const int m0 = ((M + kBlock - 1) / kBlock - 1 - place) * kBlock;   // the rows that see most come first
    const int base = uniform(m0 / G), rem = m0 - base * G;
    auto place_of = [&](int r) { return base + (int)(((uint32_t)(rem + r) * a.inv_g) >> 16); };   // of row m0 + r
    const int w = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
    const int rows = min(kBlock, M - m0);
    const int r = min(32 * w + l32, rows - 1);
    const int i = place_of(r), hh = rem + r - (i - base) * G;
    const int i_first = uniform(place_of(min(32 * w, rows - 1))), i_last = uniform(place_of(min(32 * w + 31, rows - 1)));
    const Runs runs = key_runs<UNTIL>(a.kv, row0, n, base, uniform(place_of(rows - 1)));
    const int t0 = runs.tiles * sp / a.splits, t1 = runs.tiles * (sp + 1) / a.splits;

    const char* kp = static_cast<const char*>(a.kv.k) + ((int64_t)row0 * a.kv.k_stride + g * D) * sizeof(T);
    const char* vp = static_cast<const char*>(a.kv.v) + ((int64_t)row0 * a.kv.v_stride + g * D) * sizeof(T);
    int2 mm = {0, 0};
    auto load_k = [&](int tile) {
        int lo, hi;
        runs.at(tile, &lo, &hi);
        Coming<T, D>::rows(kp, a.kv.k_stride * sizeof(T), lo, n - 1, w, lds_address(s_k[tile & 1]));
        if (UNTIL && threadIdx.x < kTile) mm = key_place(a.kv, row0, min(lo + (int)threadIdx.x, n - 1));
    };
    auto load_v = [&](int tile) {
        int lo, hi;
        runs.at(tile, &lo, &hi);
        Coming<T, D>::rows(vp, a.kv.v_stride * sizeof(T), lo, n - 1, w, lds_address(s_v[tile & 1]));
    };
    auto store_meta = [&](int tile) {
        if (UNTIL && threadIdx.x < kTile) s_meta[tile & 1][threadIdx.x] = mm;
    };
    if (t0 < t1) {
        load_k(t0);
        store_meta(t0);
        load_v(t0);
    }
    u32x4 qop[STEPS];
    {
        const char* qp = static_cast<const char*>(a.q) + ((row0 + i) * a.q_stride + (g * G + hh) * D) * (int64_t)sizeof(T) + 16 * h;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) qop[s] = *reinterpret_cast<const u32x4*>(qp + 32 * s);
    }

    // base-2 logarithms throughout: mref is the reference of the lane's row (its scaled scores less mref
    // are at most 8), sum of 2^(score - mref)
    const float c = a.scale_log2e;
    float mrun = -INFINITY, mref = 0.f, sum = 0.f, sum1 = 0.f, top = -INFINITY;
    f32x16 acc[DB], s[2], next[2];
    uint32_t pk[16];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[db][e] = 0.f;

    auto probability = [&](int e) {   // of the scores' pair e
        const float p = exp2_(__builtin_fmaf(s[e >> 3][(2 * e) & 15], c, -mref)), q = exp2_(__builtin_fmaf(s[e >> 3][(2 * e + 1) & 15], c, -mref));
        sum += p;
        sum1 += q;
        pk[e] = pack_bf16x2(p, q);
    };
    // scores of the tile in stage `st` into `next`; BESIDE: the probabilities of `s` with them
    auto scores = [&](int st, auto beside) {
        constexpr bool BESIDE = decltype(beside)::value;
        const RowReads<D> kr(lds_address(s_k[st]), l32, h);
        u32x4 x[4], y[4];
        auto group = [&](u32x4 (&f)[4], auto k) {   // two steps of both blocks of 32 keys
            constexpr int K = decltype(k)::value;
            f[0] = kr.template step<K>(), f[1] = kr.template step<K, 32>(), f[2] = kr.template step<K + 1>(), f[3] = kr.template step<K + 1, 32>();
        };
        auto products = [&](const u32x4 (&f)[4], int k) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                mma_step<T>(f[e], qop[k + e / 2], next[e & 1]);
                if constexpr (BESIDE) {
#pragma unroll
                    for (int x = 0; x < 8 / STEPS; ++x) probability(8 / STEPS * (2 * k + e) + x);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) next[b][e] = 0.f;
        using std::integral_constant;
#define A2T_I(k) integral_constant<int, k>{}
        group(x, A2T_I(0));
        group(y, A2T_I(2));
        lds_wait<4>(x);
        products(x, 0);
        if constexpr (D == 128) {
            group(x, A2T_I(4));
            lds_wait<4>(y);
            products(y, 2);
            group(y, A2T_I(6));
            lds_wait<4>(x);
            products(x, 4);
            lds_wait<0>(y);
            products(y, 6);
        } else {
            lds_wait<0>(y);
            products(y, 2);
        }
#undef A2T_I
    };
    // the tile's scores that a row does not see, and the largest of the rest
    auto finish = [&](int tile) {
        int lo, hi;
        runs.at(tile, &lo, &hi);
        const int2* meta = s_meta[tile & 1];
        if (!sees<UNTIL>(meta, lo, hi, i_first, i_last).all) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (!visible<UNTIL>(meta, lo, hi, 32 * b + 8 * (e >> 2) + 4 * h + (e & 3), i)) next[b][e] = -INFINITY;
        }
        float m = fmaxf(next[0][0], next[1][0]);
#pragma unroll
        for (int e = 1; e < 16; ++e) m = fmaxf(fmaxf(m, next[0][e]), next[1][e]);
        top = swap_max(m) * c;
#pragma unroll
        for (int b = 0; b < 2; ++b) s[b] = next[b];
    };

    if (t0 < t1) {
        wait_tiles();
        __syncthreads();
        if (t0 + 1 < t1) load_k(t0 + 1);
        scores(t0 & 1, std::false_type{});
        finish(t0);
        if (t0 + 1 < t1) store_meta(t0 + 1);
    }
    for (int tile = t0; tile < t1; ++tile) {
        // here: s and top are the tile's; its V and the next K are there once everybody has come
        wait_tiles();
        __syncthreads();
        if (tile + 2 < t1) load_k(tile + 2);
        if (tile + 1 < t1) load_v(tile + 1);
        if (__any(top > mrun + 8.f)) {
            const float up = fmaxf(mrun, top), ref = up == -INFINITY ? 0.f : up;
            const float by = exp2_(mrun - ref);
            sum *= by;
            sum1 *= by;
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] *= by;
            mrun = up;
            mref = ref;
        }
        const TransReads<D> vt(lds_address(s_v[tile & 1]), 0);
        if (tile + 1 < t1) {
            scores((tile + 1) & 1, std::true_type{});
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) probability(e);
        }
        uint2 x[D / 16], y[D / 16];
        auto products = [&](const uint2 (&f)[D / 16], int k) {
            mma_group<D>(f, __builtin_bit_cast(bf16x8, (u32x4{pk[4 * k], pk[4 * k + 1], pk[4 * k + 2], pk[4 * k + 3]})), acc);
        };
        vt.template group<0>(x);
        vt.template group<1>(y);
        lds_wait<D / 16>(x);
        products(x, 0);
        vt.template group<2>(x);
        lds_wait<D / 16>(y);
        products(y, 1);
        vt.template group<3>(y);
        lds_wait<D / 16>(x);
        products(x, 2);
        lds_wait<0>(y);
        products(y, 3);
        if (tile + 1 < t1) finish(tile + 1);
        if (tile + 2 < t1) store_meta(tile + 2);
    }

    if (32 * w + l32 >= rows) return;
    const float total = swap_sum(sum + sum1);
    if (a.splits > 1) {   // the split's own sums; prompt_join_kernel puts them together
        const int64_t at = ((int64_t)sp * a.total + row0 + i) * a.Hq + g * G + hh;
        if (h == 0) *reinterpret_cast<float2*>(a.part + (int64_t)a.splits * a.total * a.Hq * D + 2 * at) = make_float2(mrun, total);
        float* o = a.part + at * D + 4 * h;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int e = 0; e < 4; ++e) store4(o + 32 * db + 8 * e, acc[db][4 * e], acc[db][4 * e + 1], acc[db][4 * e + 2], acc[db][4 * e + 3]);
        return;
    }
    const float inv = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;   // a row without keys is zero
    const int64_t row = row0 + i;
    if (a.lse && h == 0) a.lse[(int64_t)(g * G + hh) * a.total + row] = (mref + __builtin_amdgcn_logf(total)) * kLn2;
    T* o = static_cast<T*>(a.o) + (row * a.Hq + g * G + hh) * D + 4 * h;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            store4(o + 32 * db + 8 * e, acc[db][4 * e] * inv, acc[db][4 * e + 1] * inv, acc[db][4 * e + 2] * inv, acc[db][4 * e + 3] * inv);
}

// ---- gradient with respect to the queries; delta goes to memory for the gradient of the keys.  bf16:
// P (dO . v - delta) is rounded to bf16 for its product with K, half a step of 2^-8 of each term.  delta
// comes from the O that was stored, whose rounding moves it by about 2^-9.3 |dO| |O|: little where a row's
// weight is on many keys and O is small beside v, but as much as all else where it is on few.  Blocks of
// queries with one or two key tiles in sight, which are then both in LDS, form it from the scores first, as
// sum_j P_ij dO_i . v_j in fp32: dQ and dK of sequences of 3 rows are 0.0023 off in the 2-norm instead of
// 0.0041, of 64 rows 0.0023 instead of 0.0028 (0.0017 is one rounding at the end).  Two products more for those
// blocks: 11 sequences of 64 to 1,599 rows, 32 heads on 8, 409 us forward and backward with and without.
template <typename T, int D, bool UNTIL, int N>
__global__ __launch_bounds__(kThreads, (sizeof(T) * D <= 256 ? 2 : 1)) void prompt_dq_kernel(Args a, SeqTable<N> t) {
    using Tl = Tile<T, D>;
    constexpr int DB = Tl::DB;
    __shared__ __align__(1024) char s_k[2][Tl::BYTES];
    __shared__ __align__(1024) char s_v[2][Tl::BYTES];
    __shared__ int2 s_meta[2][UNTIL ? kTile : 1];

    const int g = blockIdx.x % a.Hkv, G = a.G;
    int sp = (int)(blockIdx.x / a.Hkv), place;   // split of the block's tiles
    const int y = sp / a.splits;
    sp -= y * a.splits;
    const int z = sequence_of(t, y, &place);
    const int n = t.rows[z], row0 = t.row0[z], M = G * n;
    const int m0 = ((M + kBlock - 1) / kBlock - 1 - place) * kBlock;
    const int base = uniform(m0 / G), rem = m0 - base * G;
    auto place_of = [&](int r) { return base + (int)(((uint32_t)(rem + r) * a.inv_g) >> 16); };
    const int w = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
    const int rows = min(kBlock, M - m0);
    const bool busy = 32 * w < rows;
    const int r = min(32 * w + l32, rows - 1);
    const int i = place_of(r), hh = rem + r - (i - base) * G;
    const int i_first = uniform(place_of(min(32 * w, rows - 1))), i_last = uniform(place_of(min(32 * w + 31, rows - 1)));
    const Runs runs = key_runs<UNTIL>(a.kv, row0, n, base, uniform(place_of(rows - 1)));
    const bool few = sizeof(T) == 2 && runs.tiles <= 2;   // delta from the scores; such blocks are not split
    const int t0 = few ? (sp ? runs.tiles : 0) : runs.tiles * sp / a.splits, t1 = few ? runs.tiles : runs.tiles * (sp + 1) / a.splits;

    const char* kp = static_cast<const char*>(a.kv.k) + ((int64_t)row0 * a.kv.k_stride + g * D) * sizeof(T);
    const char* vp = static_cast<const char*>(a.kv.v) + ((int64_t)row0 * a.kv.v_stride + g * D) * sizeof(T);
    int2 mm = {0, 0};
    auto load = [&](int tile) {
        int lo, hi;
        runs.at(tile, &lo, &hi);
        const int stage = tile & 1;
        Coming<T, D>::rows(kp, a.kv.k_stride * sizeof(T), lo, n - 1, w, lds_address(s_k[stage]));
        Coming<T, D>::rows(vp, a.kv.v_stride * sizeof(T), lo, n - 1, w, lds_address(s_v[stage]));
        if (UNTIL && threadIdx.x < kTile) mm = key_place(a.kv, row0, min(lo + (int)threadIdx.x, n - 1));
    };
    auto store = [&](int stage) {
        if (UNTIL && threadIdx.x < kTile) s_meta[stage][threadIdx.x] = mm;
    };
    if (t0 < t1) load(t0);

    u32x4 qop[Tl::STEPS], dop[Tl::STEPS];
    const int64_t row = row0 + i, head = g * G + hh;
    float delta = 0.f;
    {
        const char* qp = static_cast<const char*>(a.q) + (row * a.q_stride + head * D) * (int64_t)sizeof(T) + 16 * h;
        const char* dp = static_cast<const char*>(a.d_o) + (row * a.Hq + head) * D * (int64_t)sizeof(T) + 16 * h;
        const char* op = static_cast<const char*>(a.o_in) + (row * a.Hq + head) * D * (int64_t)sizeof(T) + 16 * h;
#pragma unroll
        for (int s = 0; s < Tl::STEPS; ++s) {
            qop[s] = *reinterpret_cast<const u32x4*>(qp + 32 * s);
            dop[s] = *reinterpret_cast<const u32x4*>(dp + 32 * s);
            const u32x4 o = *reinterpret_cast<const u32x4*>(op + 32 * s);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (sizeof(T) == 2) {
                    delta += __uint_as_float(o[e] << 16) * __uint_as_float(dop[s][e] << 16);
                    delta += __uint_as_float(o[e] & 0xffff0000u) * __uint_as_float(dop[s][e] & 0xffff0000u);
                } else {
                    delta += __uint_as_float(o[e]) * __uint_as_float(dop[s][e]);
                }
            }
        }
    }
    delta = swap_sum(delta);
    float lse2 = a.lse[head * a.total + row] * kLog2e;
    if (lse2 == -INFINITY) lse2 = 0.f;   // a row without keys: nothing is visible below
    if (t0 < t1) store(t0 & 1);
    if (few && t0 + 1 < t1) {
        load(t0 + 1);
        store((t0 + 1) & 1);
    }

    const float c = a.scale_log2e;
    // P (dO . v - less) of the wave's rows and 32 keys of a tile, 0 where a key is not visible
    auto weights = [&](int stage, int b, int lo, int hi, bool all, float less, f32x16& p) {
        f32x16 s;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = p[e] = 0.f;
#pragma unroll
        for (int k = 0; k < Tl::STEPS; ++k) mma_step<T>(row_operand<T, D>(s_k[stage], 32 * b + l32, k, h), qop[k], s);
#pragma unroll
        for (int k = 0; k < Tl::STEPS; ++k) mma_step<T>(row_operand<T, D>(s_v[stage], 32 * b + l32, k, h), dop[k], p);
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] = exp2_(__builtin_fmaf(s[e], c, -lse2)) * (p[e] - less);
        if (!all) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (!visible<UNTIL>(s_meta[stage], lo, hi, 32 * b + 8 * (e >> 2) + 4 * h + (e & 3), i)) p[e] = 0.f;
        }
    };
    if (few && t0 < t1) {
        wait_tiles();
        __syncthreads();
        delta = 0.f;
        for (int tile = t0; busy && tile < t1; ++tile) {
            int lo, hi;
            runs.at(tile, &lo, &hi);
            const Sees what = sees<UNTIL>(s_meta[tile & 1], lo, hi, i_first, i_last);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if (!what.block[b]) continue;
                f32x16 p;
                weights(tile & 1, b, lo, hi, what.all, 0.f, p);
#pragma unroll
                for (int e = 0; e < 16; ++e) delta += p[e];
            }
        }
        delta = swap_sum(delta);
    }
    if (sp == 0 && 32 * w + l32 < rows && h == 0) a.delta[head * a.total + row] = delta;
    f32x16 acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[db][e] = 0.f;

    for (int tile = t0; tile < t1; ++tile) {
        const int stage = tile & 1;
        wait_tiles();
        __syncthreads();
        if (tile + 1 < t1 && !few) load(tile + 1);
        int lo, hi;
        runs.at(tile, &lo, &hi);
        const Sees what = sees<UNTIL>(s_meta[stage], lo, hi, i_first, i_last);
        if (busy) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if (!what.block[b]) continue;
                f32x16 p;
                weights(stage, b, lo, hi, what.all, delta, p);
                mma_rows<D, T>(s_k[stage], 32 * b, p, acc);
            }
        }
        if (tile + 1 < t1 && !few) store(stage ^ 1);
    }

    if (32 * w + l32 >= rows) return;
    if (a.splits > 1) {
        float* o = a.part + (((int64_t)sp * a.total + row) * a.Hq + head) * D + 4 * h;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int e = 0; e < 4; ++e) store4(o + 32 * db + 8 * e, acc[db][4 * e], acc[db][4 * e + 1], acc[db][4 * e + 2], acc[db][4 * e + 3]);
        return;
    }
    T* o = static_cast<T*>(a.dq) + row * a.q_stride + head * D + 4 * h;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            store4(o + 32 * db + 8 * e, acc[db][4 * e] * a.scale, acc[db][4 * e + 1] * a.scale, acc[db][4 * e + 2] * a.scale,
                   acc[db][4 * e + 3] * a.scale);
}

// ---- gradient with respect to keys and values, over all heads of the group.
// One workgroup = 128 keys of a KV head, 32 a wave, over tiles of 64 query rows of one head of the
// group after the other: one sum, in one fixed order.  Two waves share 32 keys (each takes half of a
// tile's rows; their sums are added at the end), two a SIMD, for one's products to run beside the
// other's exponentials.  That leaves 256 registers a wave: at head dim 128 both gradients' sums take
// 128 of them, and the keys' own rows of K and V are read from LDS with every tile (V in registers spills, and
// its reloads wait for the next tile as well: 2.6 instead of 1.8 ms; K's half makes no difference);
// at head dim 64 they stay in registers (0.76 instead of 0.85 ms for 8,192 rows of 32 heads).  fp32 rows of 512
// bytes do not fit either way: four waves, one a SIMD, everything in registers.
template <typename T, int D>
struct KeyShape {
    static constexpr bool kWide = Tile<T, D>::RB <= 256;
    static constexpr int kWaves = kWide ? 8 : 4;
};
template <typename T, int D, bool UNTIL, int N>
__global__ __launch_bounds__((64 * KeyShape<T, D>::kWaves), (KeyShape<T, D>::kWide ? 2 : 1)) void prompt_dkv_kernel(Args a, SeqTable<N> t) {
    using Tl = Tile<T, D>;
    constexpr int DB = Tl::DB, WAVES = KeyShape<T, D>::kWaves;
    constexpr bool WIDE = KeyShape<T, D>::kWide;
    using In = Coming<T, D, WAVES>;
    __shared__ __align__(1024) char s_tile[4][Tl::BYTES];            // Q and dO, two stages of each
    // where the operands of the wave's keys are
    constexpr bool KV_LDS = sizeof(T) == 2 && D == 128, V_LDS = KV_LDS || (sizeof(T) == 4 && WIDE);
    __shared__ __align__(1024) char s_v[V_LDS ? 2 : 1][V_LDS ? Tl::BYTES : 16];
    __shared__ __align__(1024) char s_k[KV_LDS ? 2 : 1][KV_LDS ? Tl::BYTES : 16];
    __shared__ __align__(16) float s_lse[2][kTile], s_delta[2][kTile];   // -lse / scale (fp32: -lse log2 e) and -delta of the tile's rows
    __shared__ int s_range[2][4];
    static_assert(!WIDE || 4 * Tl::BYTES >= 4 * DB * 16 * 256, "one gradient's sums of four waves fit the tiles");

    const int g = blockIdx.x % a.Hkv, G = a.G;
    int sp = (int)(blockIdx.x / a.Hkv), place;   // split of the block's tiles
    const int y = sp / a.splits;
    sp -= y * a.splits;
    const int z = sequence_of(t, y, &place);
    const int n = t.rows[z], row0 = t.row0[z];
    const int w = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
    const int kg = w & 3, rg = w >> 2;        // keys, rows of a tile that are the wave's
    const int k0 = place * kBlock + 32 * kg, key = min(k0 + l32, n - 1);
    const bool busy = k0 < n;
    // the lane's key: its place, and the first place that does not see it
    int2 me = {key, n};
    if constexpr (UNTIL) {
        me = key_place(a.kv, row0, key);
        me.y = max(min(me.y, n), 0);   // any number is allowed: differences of places stay within 32 bits
    }
    int j_min = me.x, j_max = me.x, u_min = me.y, u_max = me.y;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        j_min = min(j_min, __shfl_xor(j_min, d));
        j_max = max(j_max, __shfl_xor(j_max, d));
        u_min = min(u_min, __shfl_xor(u_min, d));
        u_max = max(u_max, __shfl_xor(u_max, d));
    }
    j_min = uniform(j_min), j_max = uniform(j_max), u_min = uniform(u_min), u_max = uniform(u_max);
    if (lane == 0) s_range[0][kg] = j_min, s_range[1][kg] = u_max;   // idle waves repeat the last key's
    __syncthreads();
    const int from = uniform(min(min(s_range[0][0], s_range[0][1]), min(s_range[0][2], s_range[0][3])));
    const int to = uniform(max(max(s_range[1][0], s_range[1][1]), max(s_range[1][2], s_range[1][3])));
    // places from .. to - 1, head by head; the split's tiles
    const int per_head = max(to - from + kTile - 1, 0) / kTile;
    const int t0 = (int)((int64_t)G * per_head * sp / a.splits), t1 = (int)((int64_t)G * per_head * (sp + 1) / a.splits);

    const char* kb = static_cast<const char*>(a.kv.k) + (row0 * a.kv.k_stride + g * D) * (int64_t)sizeof(T);
    const char* kp = kb + key * a.kv.k_stride * (int64_t)sizeof(T) + 16 * h;
    const char* vp = static_cast<const char*>(a.kv.v) + (row0 * a.kv.v_stride + g * D) * (int64_t)sizeof(T);
    u32x4 kop[KV_LDS ? 1 : Tl::STEPS], vop[V_LDS ? 1 : Tl::STEPS];
#pragma unroll
    for (int s = 0; s < Tl::STEPS; ++s) {
        if constexpr (!KV_LDS) kop[s] = *reinterpret_cast<const u32x4*>(kp + 32 * s);
        if constexpr (!V_LDS) vop[s] = *reinterpret_cast<const u32x4*>(vp + key * a.kv.v_stride * (int64_t)sizeof(T) + 16 * h + 32 * s);
    }

    const char* qp = static_cast<const char*>(a.q) + ((int64_t)row0 * a.q_stride + g * G * D) * sizeof(T);
    const char* dp = static_cast<const char*>(a.d_o) + ((int64_t)row0 * a.Hq + g * G) * D * sizeof(T);
    float2 stat = {0.f, 0.f};
    const float lse_by = sizeof(T) == 2 ? -1.f / a.scale : -kLog2e;
    auto load = [&](int hh, int lo, int stage) {
        In::rows(qp + hh * D * sizeof(T), a.q_stride * sizeof(T), lo, n - 1, w, lds_address(s_tile[stage]));
        In::rows(dp + hh * D * sizeof(T), (int64_t)a.Hq * D * sizeof(T), lo, n - 1, w, lds_address(s_tile[2 + stage]));
        if (threadIdx.x < kTile) {
            const int64_t at = (int64_t)(g * G + hh) * a.total + row0 + min(lo + (int)threadIdx.x, n - 1);
            stat = make_float2(a.lse[at], a.delta[at]);
        }
    };
    auto store = [&](int stage) {
        if (threadIdx.x < kTile) {
            s_lse[stage][threadIdx.x] = stat.x == -INFINITY ? 0.f : stat.x * lse_by;   // a row without keys sees none of these
            s_delta[stage][threadIdx.x] = -stat.y;
        }
    };
    int hh = per_head ? t0 / per_head : 0, lo = from + (t0 - hh * per_head) * kTile;
    if (t0 < t1) {
        if constexpr (V_LDS) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int first = min(place * kBlock + x * kTile, n - 1);
                In::rows(vp, a.kv.v_stride * sizeof(T), first, n - 1, w, lds_address(s_v[x]));
                if constexpr (KV_LDS) In::rows(kb, a.kv.k_stride * sizeof(T), first, n - 1, w, lds_address(s_k[x]));
            }
        }
        load(hh, lo, t0 & 1);
        store(t0 & 1);
    }

    const float c = a.scale_log2e;
    f32x16 ak[DB], av[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) ak[db][e] = av[db][e] = 0.f;

    // rows 32 b + 8 (e / 4) + 4 h + e % 4 of a tile, as the products' sums hold them
    auto init = [&](f32x16& x, const float* of, int b) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float4 y = *reinterpret_cast<const float4*>(of + 32 * b + 8 * q + 4 * h);
            x[4 * q] = y.x, x[4 * q + 1] = y.y, x[4 * q + 2] = y.z, x[4 * q + 3] = y.w;
        }
    };
    auto block = [&](const char* q, const char* d, const float* lse, const float* delta, int b, int first, bool all) {
        // bf16 starts the products from -lse / scale and -delta of their rows, so that no subtraction
        // comes after them; sums that start at -lse / scale would round to its size in fp32
        f32x16 s, p;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
        for (int k = 0; k < Tl::STEPS; ++k) mma_step<T>(row_operand<T, D>(q, 32 * b + l32, k, h), kop[k], s);
        init(p, delta, b);
#pragma unroll
        for (int k = 0; k < Tl::STEPS; ++k) {
            u32x4 v;
            if constexpr (V_LDS) v = row_operand<T, D>(s_v[0], 32 * kg + l32, k, h);
            else v = vop[k];
            mma_step<T>(row_operand<T, D>(d, 32 * b + l32, k, h), v, p);
        }
        f32x16 l;
        init(l, lse, b);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = exp2_(__builtin_fmaf(s[e], c, l[e]));
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] *= s[e];
        if (!all) {   // a pair that is not visible has no gradient, whatever its products were
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int i = first + 32 * b + 8 * (e >> 2) + 4 * h + (e & 3);
                if (i < me.x || i >= me.y) s[e] = p[e] = 0.f;
            }
        }
        mma_rows<D, T>(d, 32 * b, s, av);
        mma_rows<D, T>(q, 32 * b, p, ak);
    };
    // The same for bf16, with LDS reads in groups of eight registers, three of them under way: rows of Q,
    // rows of dO (with K's and V's where those are in LDS), then both transposed.
    auto block16 = [&](uint32_t q, uint32_t d, const float* lse, const float* delta, int b, int first, bool all) {
        f32x16 s, p;
        const int r = 32 * b + l32;
        const RowReads<D> qr(q, r, h), dr(d, r, h);
        const RowReads<D> kr(KV_LDS ? lds_address(s_k[0]) : 0, 32 * kg + l32, h), vr(KV_LDS ? lds_address(s_v[0]) : 0, 32 * kg + l32, h);
        const TransReads<D> qt(q, 32 * b), dt(d, 32 * b);
        constexpr int NQ = KV_LDS ? Tl::STEPS : Tl::STEPS / 2, ND = NQ, NT = DB / 2 * 2, ALL = NQ + ND + 2 * NT;
        constexpr int EXPS = 16 / Tl::STEPS;   // beside a product
        u32x4 f[3][2];
        uint2 tr[3][4];
        bf16x8 packed[2];
        using std::integral_constant;
        auto issue = [&](auto at) {
            constexpr int G = decltype(at)::value;
            if constexpr (G < NQ) {
                if constexpr (KV_LDS) f[G % 3][0] = qr.template step<G>(), f[G % 3][1] = kr.template step<G>();
                else f[G % 3][0] = qr.template step<2 * G>(), f[G % 3][1] = qr.template step<2 * G + 1>();
            } else if constexpr (G < NQ + ND) {
                constexpr int X = G - NQ;
                if constexpr (KV_LDS) f[G % 3][0] = dr.template step<X>(), f[G % 3][1] = vr.template step<X>();
                else f[G % 3][0] = dr.template step<2 * X>(), f[G % 3][1] = dr.template step<2 * X + 1>();
            } else if constexpr (G < ALL) {
                constexpr int X = (G - NQ - ND) % NT;   // half of the rows, pair of blocks of 32 dimensions
                if constexpr (G < NQ + ND + NT) dt.template pair<X / (NT / 2), 2 * (X % (NT / 2))>(tr[G % 3]);
                else qt.template pair<X / (NT / 2), 2 * (X % (NT / 2))>(tr[G % 3]);
            }
        };
        auto use = [&](auto at) {
            constexpr int G = decltype(at)::value;
            // reads of the two groups behind this one
            constexpr int R1 = G + 1 >= ALL ? 0 : G + 1 < NQ + ND ? 2 : 4, R2 = G + 2 >= ALL ? 0 : G + 2 < NQ + ND ? 2 : 4;
            if constexpr (G < NQ + ND) lds_wait<R1 + R2>(f[G % 3]);
            else lds_wait<R1 + R2>(tr[G % 3]);
            if constexpr (G < NQ) {
                if constexpr (KV_LDS) mma_step<T>(f[G % 3][0], f[G % 3][1], s);
                else mma_step<T>(f[G % 3][0], kop[2 * G], s), mma_step<T>(f[G % 3][1], kop[2 * G + 1], s);
            } else if constexpr (G < NQ + ND) {
                constexpr int X = G - NQ;
#pragma unroll
                for (int e = 0; e < (KV_LDS ? 1 : 2); ++e) {
                    const int at = KV_LDS ? X : 2 * X + e;
                    if constexpr (KV_LDS) mma_step<T>(f[G % 3][0], f[G % 3][1], p);
                    else mma_step<T>(f[G % 3][e], vop[at], p);
#pragma unroll
                    for (int i = 0; i < EXPS; ++i) s[EXPS * at + i] = exp2_(s[EXPS * at + i] * c);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                constexpr int X = (G - NQ - ND) % NT, HALF = X / (NT / 2), DB0 = 2 * (X % (NT / 2));
                constexpr bool OF_Q = G >= NQ + ND + NT;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const u32x4 o = {tr[G % 3][2 * e].x, tr[G % 3][2 * e].y, tr[G % 3][2 * e + 1].x, tr[G % 3][2 * e + 1].y};
                    f32x16& acc = (OF_Q ? ak : av)[DB0 + e];
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, o), packed[HALF], acc, 0, 0, 0);
                }
            }
        };
        auto weights = [&] {
#pragma unroll
            for (int e = 0; e < 16; ++e) p[e] *= s[e];
            if (!all) {   // a pair that is not visible has no gradient, whatever its products were
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int i = first + 32 * b + 8 * (e >> 2) + 4 * h + (e & 3);
                    if (i < me.x || i >= me.y) s[e] = p[e] = 0.f;
                }
            }
            packed[0] = pack8(s, 0), packed[1] = pack8(s, 1);
        };
        auto step = [&](auto at) {
            constexpr int G = decltype(at)::value;
            if constexpr (G < ALL) {
                if constexpr (G == NQ + ND) weights();
                if constexpr (G == NQ + ND + NT) packed[0] = pack8(p, 0), packed[1] = pack8(p, 1);
                use(at);
                issue(integral_constant<int, G + 3>{});
            }
        };
        init(s, lse, b);
        init(p, delta, b);
        issue(integral_constant<int, 0>{});
        issue(integral_constant<int, 1>{});
        issue(integral_constant<int, 2>{});
        static_assert(sizeof(T) == 4 || ALL <= 24, "steps of a block");
#define A2T_G(k) step(integral_constant<int, k>{});
        A2T_G(0) A2T_G(1) A2T_G(2) A2T_G(3) A2T_G(4) A2T_G(5) A2T_G(6) A2T_G(7) A2T_G(8)
        A2T_G(9) A2T_G(10) A2T_G(11) A2T_G(12) A2T_G(13) A2T_G(14) A2T_G(15) A2T_G(16) A2T_G(17)
        A2T_G(18) A2T_G(19) A2T_G(20) A2T_G(21) A2T_G(22) A2T_G(23)
#undef A2T_G
    };
    for (int tile = t0; tile < t1; ++tile) {
        const int stage = tile & 1;
        int next = lo + kTile, next_hh = hh;
        if (next >= to) next = from, next_hh = hh + 1;
        wait_tiles();
        __syncthreads();
        if (tile + 1 < t1) load(next_hh, next, stage ^ 1);
        auto visit = [&](int b) {
            const int first = lo + 32 * b, last = min(first + 32, n) - 1;
            if (!busy || last < j_min || first >= u_max) return;
            const bool all = first >= j_max && first + 32 <= u_min;
            if constexpr (sizeof(T) == 2) block16(lds_address(s_tile[stage]), lds_address(s_tile[2 + stage]), s_lse[stage], s_delta[stage], b, lo, all);
            else block(s_tile[stage], s_tile[2 + stage], s_lse[stage], s_delta[stage], b, lo, all);
        };
        if constexpr (WIDE) {
            visit(rg);
        } else {
            visit(0);
            visit(1);
        }
        if (tile + 1 < t1) store(stage ^ 1);
        lo = next;
        hh = next_hh;
    }

    if constexpr (WIDE) {   // the second half's sums to the first half's waves, one gradient after the other
        float* part = reinterpret_cast<float*>(s_tile[0]) + kg * (DB * 16 * 64) + lane;
        auto add = [&](f32x16 (&x)[DB]) {
            __syncthreads();
            if (rg == 1) {
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int e = 0; e < 16; ++e) part[(db * 16 + e) * 64] = x[db][e];
            }
            __syncthreads();
            if (rg == 0) {
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[db][e] += part[(db * 16 + e) * 64];
            }
        };
        add(ak);
        add(av);
    }
    if (rg || k0 + l32 >= n) return;
    if (a.splits > 1) {
        float* o = a.part + (((int64_t)sp * a.total + row0 + me.x) * a.Hkv + g) * 2 * D + 4 * h;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                store4(o + 32 * db + 8 * e, ak[db][4 * e], ak[db][4 * e + 1], ak[db][4 * e + 2], ak[db][4 * e + 3]);
                store4(o + D + 32 * db + 8 * e, av[db][4 * e], av[db][4 * e + 1], av[db][4 * e + 2], av[db][4 * e + 3]);
            }
        return;
    }
    // gradients lie as the caller's K and V do, whatever order the keys were read in
    T* ok = static_cast<T*>(a.dk) + (row0 + me.x) * a.k_out + g * D + 4 * h;
    T* ov = static_cast<T*>(a.dv) + (row0 + me.x) * a.v_out + g * D + 4 * h;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            store4(ok + 32 * db + 8 * e, ak[db][4 * e] * a.scale, ak[db][4 * e + 1] * a.scale, ak[db][4 * e + 2] * a.scale, ak[db][4 * e + 3] * a.scale);
            store4(ov + 32 * db + 8 * e, av[db][4 * e], av[db][4 * e + 1], av[db][4 * e + 2], av[db][4 * e + 3]);
        }
}

// ---- blocks whose tiles were split: the splits' sums put together, in order
// Four elements a thread; a row of the launch's sequences by its place among their rows.
template <int N>
__device__ __forceinline__ int64_t joined_row(const SeqTable<N>& t, int64_t r) {
    for (int z = 0; z < t.count; ++z) {   // few: launches of many sequences are not split
        if (r < t.rows[z]) return t.row0[z] + r;
        r -= t.rows[z];
    }
    return -1;
}
template <typename T, int D, int N>
__global__ __launch_bounds__(kThreads) void prompt_join_kernel(Args a, SeqTable<N> t) {
    const int64_t x = (int64_t)blockIdx.x * kThreads + threadIdx.x, rh = x / (D / 4);
    const int c = (int)(x % (D / 4)) * 4, head = (int)(rh % a.Hq);
    const int64_t row = joined_row(t, rh / a.Hq);
    if (row < 0) return;
    const float* ml = a.part + (int64_t)a.splits * a.total * a.Hq * D;
    auto at = [&](int sp) { return ((int64_t)sp * a.total + row) * a.Hq + head; };
    float m = -INFINITY;
    for (int sp = 0; sp < a.splits; ++sp) m = fmaxf(m, ml[2 * at(sp)]);
    const float ref = m == -INFINITY ? 0.f : m;
    float4 o = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
    for (int sp = 0; sp < a.splits; ++sp) {
        const float2 p = *reinterpret_cast<const float2*>(ml + 2 * at(sp));
        const float by = exp2_(p.x - ref);
        const float4 q = *reinterpret_cast<const float4*>(a.part + at(sp) * D + c);
        sum += by * p.y;
        o.x += by * q.x, o.y += by * q.y, o.z += by * q.z, o.w += by * q.w;
    }
    const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    if (a.lse && c == 0) a.lse[(int64_t)head * a.total + row] = (ref + __builtin_amdgcn_logf(sum)) * kLn2;
    store4(static_cast<T*>(a.o) + (row * a.Hq + head) * D + c, o.x * inv, o.y * inv, o.z * inv, o.w * inv);
}
// dQ, or dK and dV (WIDTH D or 2 D a head)
template <typename T, int D, bool KEYS, int N>
__global__ __launch_bounds__(kThreads) void prompt_add_kernel(Args a, SeqTable<N> t) {
    constexpr int WIDTH = KEYS ? 2 * D : D;
    const int heads = KEYS ? a.Hkv : a.Hq;
    const int64_t x = (int64_t)blockIdx.x * kThreads + threadIdx.x, rh = x / (WIDTH / 4);
    const int c = (int)(x % (WIDTH / 4)) * 4, head = (int)(rh % heads);
    const int64_t row = joined_row(t, rh / heads);
    if (row < 0) return;
    float4 o = {0.f, 0.f, 0.f, 0.f};
    for (int sp = 0; sp < a.splits; ++sp) {
        const float4 q = *reinterpret_cast<const float4*>(a.part + (((int64_t)sp * a.total + row) * heads + head) * WIDTH + c);
        o.x += q.x, o.y += q.y, o.z += q.z, o.w += q.w;
    }
    const bool v = KEYS && c >= D;
    const float by = v ? 1.f : a.scale;
    T* to = KEYS ? v ? static_cast<T*>(a.dv) + row * a.v_out + head * D + c - D : static_cast<T*>(a.dk) + row * a.k_out + head * D + c
                 : static_cast<T*>(a.dq) + row * a.q_stride + head * D + c;
    store4(to, o.x * by, o.y * by, o.z * by, o.w * by);
}

enum class Kernel { forward, dq, dkv };

template <Kernel K, typename T, int D, int N>
hipError_t join(const Args& a, const SeqTable<N>& s, hipStream_t stream) {
    int64_t rows = 0;
    for (int i = 0; i < s.count; ++i) rows += s.rows[i];
    const int64_t fours = rows * (K == Kernel::dkv ? (int64_t)a.Hkv * 2 : a.Hq) * (D / 4);
    const dim3 grid((uint32_t)((fours + kThreads - 1) / kThreads));
    if constexpr (K == Kernel::forward) return launch_kernel(prompt_join_kernel<T, D, N>, grid, dim3(kThreads), stream, a, s);
    else return launch_kernel(prompt_add_kernel<T, D, K == Kernel::dkv, N>, grid, dim3(kThreads), stream, a, s);
}
template <Kernel K, typename T, int D, bool UNTIL>
hipError_t launch(const Args& a, const SeqTable<kMaxSeqs>& t, int blocks, hipStream_t stream) {
    return by_count(t, [&](const auto& s) {
        constexpr int N = sizeof(s.rows) / sizeof(s.rows[0]);
        const dim3 grid((uint32_t)(blocks * a.splits * a.Hkv));
        hipError_t e;
        if constexpr (K == Kernel::forward && sizeof(T) == 2) e = launch_kernel(prompt_attn16_kernel<D, UNTIL, N>, grid, dim3(kThreads), stream, a, s);
        else if constexpr (K == Kernel::forward) e = launch_kernel(prompt_attn_kernel<T, D, UNTIL, N>, grid, dim3(kThreads), stream, a, s);
        else if constexpr (K == Kernel::dq) e = launch_kernel(prompt_dq_kernel<T, D, UNTIL, N>, grid, dim3(kThreads), stream, a, s);
        else e = launch_kernel(prompt_dkv_kernel<T, D, UNTIL, N>, grid, dim3(64 * KeyShape<T, D>::kWaves), stream, a, s);
        return e != hipSuccess || a.splits == 1 ? e : join<K, T, D, N>(a, s, stream);
    });
}
template <Kernel K>
hipError_t launch(const Shape& s, const Args& a, const SeqTable<kMaxSeqs>& t, int blocks, hipStream_t stream) {
    auto typed = [&](auto* type) {
        using T = std::remove_pointer_t<decltype(type)>;
        const bool u = a.kv.until != nullptr;
        if (s.head_dim == 128) return u ? launch<K, T, 128, true>(a, t, blocks, stream) : launch<K, T, 128, false>(a, t, blocks, stream);
        if (s.head_dim == 64) return u ? launch<K, T, 64, true>(a, t, blocks, stream) : launch<K, T, 64, false>(a, t, blocks, stream);
        return hipErrorInvalidValue;
    };
    return s.f32 ? typed((float*)nullptr) : typed((bf16_t*)nullptr);
}

}  // namespace

hipError_t launch_forward(const Shape& s, const Args& a, const SeqTable<kMaxSeqs>& t, int blocks, hipStream_t stream) {
    return launch<Kernel::forward>(s, a, t, blocks, stream);
}
hipError_t launch_dq(const Shape& s, const Args& a, const SeqTable<kMaxSeqs>& t, int blocks, hipStream_t stream) {
    return launch<Kernel::dq>(s, a, t, blocks, stream);
}
hipError_t launch_dkv(const Shape& s, const Args& a, const SeqTable<kMaxSeqs>& t, int blocks, hipStream_t stream) {
    return launch<Kernel::dkv>(s, a, t, blocks, stream);
}

}  // namespace prompt
}  // namespace a2t
