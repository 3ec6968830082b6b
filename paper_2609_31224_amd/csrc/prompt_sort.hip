// Keys sorted for attention over packed sequences with keys that expire (a2t_prompt_* with
// `until`).  Eviction keeps a few rows of every unit, so that a tile of 64 consecutive keys is
// never quite dead: sorted into lasting and passing keys, what a block of queries sees is two
// dense runs, and the kernels skip the rest (a ten-minute session with a budget of 4,096 rows: 52 %
// of the pairs of a causal triangle).  That costs a launch of one workgroup a sequence (17 us there, 5 for
// 3,000 rows) and one that copies K and V (28 us there).
#include "launch.h"
#include "prompt_device.h"

namespace a2t {
namespace prompt {
namespace {

constexpr int kScanThreads = 1024;
constexpr int kCopyRows = 16;    // rows of a copying workgroup

// One workgroup a sequence: counts of lasting keys and reach of the passing ones, by place.  A thread
// takes neighbouring places, so that the threads meet once.
template <int N>
__global__ __launch_bounds__(kScanThreads) void prompt_scan_kernel(SortArgs a, SeqTable<N> t) {
    constexpr int kWaves = kScanThreads / 64;
    constexpr int kNone = -0x7fffffff;
    const int n = t.rows[blockIdx.x], row0 = t.row0[blockIdx.x];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int per = (n + kScanThreads - 1) / kScanThreads;
    const int j0 = (int)min((int64_t)tid * per, (int64_t)n), j1 = min(j0 + per, n);
    __shared__ int s_count[kWaves], s_reach[kWaves];
    // eight places' values at a time
    auto each = [&](auto f) {
        for (int j = j0; j < j1; j += 8) {
            int until[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) until[e] = a.until[row0 + min(j + e, j1 - 1)];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (j + e < j1) f(j + e, until[e]);
        }
    };
    int count = 0, reach = kNone;
    each([&](int, int until) {
        if (until >= n) ++count;
        else reach = max(reach, until);
    });
    // of the threads before and this one
    int c = count, m = reach;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int oc = __shfl_up(c, d), om = __shfl_up(m, d);
        if (lane >= d) c += oc, m = max(m, om);
    }
    if (lane == 63) s_count[w] = c, s_reach[w] = m;
    // of the threads before alone
    c -= count;
    m = __shfl_up(m, 1);
    if (lane == 0) m = kNone;
    __syncthreads();
    for (int k = 0; k < w; ++k) c += s_count[k], m = max(m, s_reach[k]);
    each([&](int j, int until) {
        if (until >= n) {
            ++c;
        } else {
            m = max(m, until);
            a.reach[row0 + (j - c)] = m;
        }
        a.lasting[row0 + j] = c;
    });
}

template <int N>
__global__ __launch_bounds__(kThreads) void prompt_copy_kernel(SortArgs a, SeqTable<N> t) {
    int place;
    const int z = sequence_of(t, (int)blockIdx.x, &place);
    const int n = t.rows[z], row0 = t.row0[z], i0 = place * kCopyRows, rows = min(kCopyRows, n - i0);
    const int all = a.lasting[row0 + n - 1];
    auto sorted = [&](int j, bool* lasts) {
        const int seen = a.lasting[row0 + j];
        *lasts = seen > (j ? a.lasting[row0 + j - 1] : 0);
        return *lasts ? seen - 1 : all + j - seen;
    };
    if ((int)threadIdx.x < rows) {
        const int j = i0 + threadIdx.x;
        bool lasts;
        const int at = sorted(j, &lasts);
        a.meta[row0 + at] = make_int2(j, lasts ? 0x7fffffff : a.until[row0 + j]);
        // the first passing key that place j may still see: reach does not fall
        int lo = 0, hi = n - all;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (a.reach[row0 + mid] > j) hi = mid;
            else lo = mid + 1;
        }
        a.first[row0 + j] = lo;
    }
    const int chunks = a.row_bytes / 16;
    for (int x = threadIdx.x; x < rows * chunks; x += kThreads) {
        const int j = i0 + x / chunks, c = x % chunks;
        bool lasts;
        const int64_t to = (int64_t)(row0 + sorted(j, &lasts)) * a.row_bytes;
        reinterpret_cast<u32x4*>(static_cast<char*>(a.k_out) + to)[c] =
            reinterpret_cast<const u32x4*>(static_cast<const char*>(a.k) + (row0 + j) * a.k_stride)[c];
        reinterpret_cast<u32x4*>(static_cast<char*>(a.v_out) + to)[c] =
            reinterpret_cast<const u32x4*>(static_cast<const char*>(a.v) + (row0 + j) * a.v_stride)[c];
    }
}

}  // namespace

hipError_t launch_sort(const SortArgs& a, const SeqTable<kMaxSeqs>& t, hipStream_t stream) {
    hipError_t e = by_count(t, [&](const auto& s) {
        constexpr int N = sizeof(s.rows) / sizeof(s.rows[0]);
        return launch_kernel(prompt_scan_kernel<N>, dim3(t.count), dim3(kScanThreads), stream, a, s);
    });
    if (e != hipSuccess) return e;
    SeqTable<kMaxSeqs> u = t;
    int blocks = 0;
    for (int i = 0; i < t.count; ++i) {
        u.block0[i] = blocks;
        blocks += (t.rows[i] + kCopyRows - 1) / kCopyRows;
    }
    return by_count(u, [&](const auto& s) {
        constexpr int N = sizeof(s.rows) / sizeof(s.rows[0]);
        return launch_kernel(prompt_copy_kernel<N>, dim3(blocks), dim3(kThreads), stream, a, s);
    });
}

}  // namespace prompt
}  // namespace a2t
