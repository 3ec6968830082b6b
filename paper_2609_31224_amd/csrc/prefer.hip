// The preference loss of paired answers on given logits, and the log probabilities of
// target tokens (gfx950).  Public API: include/a2t.h (a2t_prefer_*).
//
//   prefer_rows_kernel  one workgroup per row (policy rows, then reference rows): (max, sum
//                       of exponentials) of the row and log p(target) = x_t - max - ln sum.
//   prefer_grad_kernel  one workgroup per policy row: the sums of the row's pair, the slope
//                       of the loss, and the gradient slope (p_v - [v = target]); one more
//                       workgroup writes the loss and every answer's ratio.
//   prefer_ratio_kernel one workgroup per answer between the two, where answers are long.
// The slope of a row depends on all rows of its pair, so the policy's logits are read twice.
// Sums of short answers are formed by every workgroup for its own pair, in the same order
// (deterministic, and one launch less), in 64 bits: a ratio is a small difference of large sums.
// That is work that grows with the square of an answer's rows: those of long ones are formed once.
#include "../../include/a2t.h"
#include "launch.h"
#include "overlap.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <type_traits>

namespace {

constexpr int kChunk = 8;             // elements of a chunk (16 bytes of bf16, 32 of fp32)
constexpr int kMaxPairs = A2T_PREFER_MAX_PAIRS;
constexpr int kAnswers = 2 * kMaxPairs;
// Policy logits that the gradient still finds in the caches when it comes back to them, last rows
// first (the memory-side cache holds 256 MiB).
constexpr int64_t kKeepBytes = 160ll << 20;
constexpr int kRatioThreads = 1024;
// Rows of a call's longest answer from which ratios are formed in a launch of their own.  (That against
// every workgroup for itself, one pair: with gradient, 64 rows of 32,000 bf16 logits 15.8 against 15.4 us,
// 128 rows 16.6 against 20.0, 1,024 rows 70 against 121; without, 64 rows 9.6 against 11.9 and 16 rows 9.4
// against 9.0.)
constexpr int kLongRows = 96;
constexpr float kLog2e = 1.44269504088896340736f;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
struct bf16_t {
    uint16_t bits;
};
// one chunk as stored
template <typename T> struct Raw;
template <> struct Raw<bf16_t> {
    u32x4 a;
};
template <> struct Raw<float> {
    u32x4 a, b;
};
// STREAM: past the caches (what will not be read again before it would be pushed out)
template <bool STREAM>
__device__ __forceinline__ u32x4 load16(const u32x4* p) {
    return STREAM ? __builtin_nontemporal_load(p) : *p;
}
template <bool STREAM>
__device__ __forceinline__ Raw<bf16_t> load_raw(const bf16_t* row, int c) {
    return {load16<STREAM>(reinterpret_cast<const u32x4*>(row) + c)};
}
template <bool STREAM>
__device__ __forceinline__ Raw<float> load_raw(const float* row, int c) {
    const u32x4* p = reinterpret_cast<const u32x4*>(row) + 2 * c;
    return {load16<STREAM>(p), load16<STREAM>(p + 1)};
}
__device__ __forceinline__ void unpack(const Raw<bf16_t>& r, float (&x)[kChunk]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(r.a[e] << 16);
        x[2 * e + 1] = __uint_as_float(r.a[e] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const Raw<float>& r, float (&x)[kChunk]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = __uint_as_float(r.a[e]);
        x[4 + e] = __uint_as_float(r.b[e]);
    }
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
    const bf16x2 v = {(__bf16)a, (__bf16)b};   // round to nearest even, once per output
    return __builtin_bit_cast(uint32_t, v);
}
// (The gradient is stored past the caches.  Through them, 389 MB of it in a step of 1,280 rows x 151,938
// logits make the next step's rows 157 us instead of 124, its own pass 139 instead of 151: the step 292, 271 so.)
__device__ __forceinline__ void store_chunk(bf16_t* row, int c, const float (&x)[kChunk]) {
    __builtin_nontemporal_store((u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])}),
                                reinterpret_cast<u32x4*>(row) + c);
}
__device__ __forceinline__ void store_chunk(float* row, int c, const float (&x)[kChunk]) {
    u32x4 a, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        a[e] = __float_as_uint(x[e]);
        b[e] = __float_as_uint(x[4 + e]);
    }
    reinterpret_cast<u32x4*>(row)[2 * c] = a;   // half of a lane's 32 bytes each: through the caches
    reinterpret_cast<u32x4*>(row)[2 * c + 1] = b;
}
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float value(const bf16_t* row, int i) { return __uint_as_float((uint32_t)row[i].bits << 16); }
__device__ __forceinline__ float value(const float* row, int i) { return row[i]; }

// Part of a row's sum: z of e^(x - m).  m is a logit that no other passes by kSlack; it follows the
// largest one lazily, which leaves most chunks without a rescaling.
constexpr float kSlack = 16.f;
struct Sum {
    float m, z;
};
__device__ __forceinline__ Sum join(Sum a, Sum b) {
    const float m = fmaxf(a.m, b.m), ref = m == -INFINITY ? 0.f : m;
    return {m, a.z * exp2_((a.m - ref) * kLog2e) + b.z * exp2_((b.m - ref) * kLog2e)};
}

// ln p(target) of a row, and what its probabilities are made from: p_v = e^(x_v - m) / z.
struct RowStat {
    double logp;
    float m, z;
};

template <typename T>
struct RowsArgs {
    const T* x[2];            // policy, reference (null: policy rows only)
    int64_t stride[2];
    const int32_t* target;
    RowStat* stat;            // [2][n] out, or null
    float* logp;              // [n] out, or null
    int32_t n, vocab;
    int32_t stream;           // policy rows before this one are streamed, and all of the reference's
};

template <typename T, int TH>
__global__ __launch_bounds__(TH) void prefer_rows_kernel(RowsArgs<T> a) {
    // the reference's rows first: the gradient then finds the policy's last rows in the caches
    const int tid = threadIdx.x, which = (int)gridDim.x > a.n && (int)blockIdx.x < a.n, row = (int)(blockIdx.x % (uint32_t)a.n);
    const int target = a.target[row];
    RowStat* stat = a.stat ? a.stat + which * a.n + row : nullptr;
    if (target < 0 || target >= a.vocab) {   // no loss at this row
        if (tid == 0) {
            if (stat) *stat = {0.0, 0.f, 0.f};
            if (a.logp) a.logp[row] = 0.f;
        }
        return;
    }
    const T* x = a.x[which] + row * a.stride[which];
    const int full = a.vocab / kChunk;
    Sum s{-INFINITY, 0.f};
    float ref = 0.f;   // m, or 0 before the first finite logit
    auto add = [&](const float (&v)[kChunk]) {
        float m = v[0];
#pragma unroll
        for (int e = 1; e < kChunk; ++e) m = fmaxf(m, v[e]);
        if (__any(m > s.m + kSlack)) {
            m = fmaxf(m, s.m);
            ref = m == -INFINITY ? 0.f : m;
            s = {m, s.z * exp2_((s.m - ref) * kLog2e)};
        }
#pragma unroll
        for (int e = 0; e < kChunk; ++e) s.z += exp2_((v[e] - ref) * kLog2e);
    };
    constexpr int kAhead = sizeof(T) == 2 ? 8 : 4;   // chunks requested at once: 64 KiB and more of a CU's waves
    auto sweep = [&](auto stream) {
        constexpr bool STREAM = decltype(stream)::value;
        int c = tid;
        for (; c + (kAhead - 1) * TH < full; c += kAhead * TH) {
            Raw<T> r[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) r[k] = load_raw<STREAM>(x, c + k * TH);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                float v[kChunk];
                unpack(r[k], v);
                add(v);
            }
        }
        for (; c < full; c += TH) {
            float v[kChunk];
            unpack(load_raw<STREAM>(x, c), v);
            add(v);
        }
    };
    if (which || row < a.stream) sweep(std::true_type{});
    else sweep(std::false_type{});
    if (tid < a.vocab - full * kChunk) s = join(s, {value(x, full * kChunk + tid), 1.f});
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s = join(s, {__shfl_xor(s.m, d), __shfl_xor(s.z, d)});
    __shared__ Sum part[TH / 64];
    if (tid % 64 == 0) part[tid / 64] = s;
    __syncthreads();
    if (tid) return;
    for (int w = 1; w < TH / 64; ++w) s = join(s, part[w]);
    const double logp = (double)(value(x, target) - s.m) - log((double)s.z);
    if (stat) *stat = {logp, s.m, s.z};
    if (a.logp) a.logp[row] = (float)logp;
}

template <typename T>
struct GradArgs {
    const T* x;
    T* grad;                  // null: no gradient
    int64_t stride;
    const RowStat* stat;      // [2][n]
    const float* ref_logp;    // [n], or null: the reference's rows are in stat
    double* sums;             // [2 pairs] ratios that prefer_ratio_kernel has formed, or null
    const int32_t* target;
    float* losses;            // [3]
    float* ratios;            // [2 pairs], or null
    int32_t n, vocab, pairs;
    int32_t stream;           // rows before this one are streamed
    float beta, smoothing;
    int32_t start[kAnswers + 1];   // first row of each answer
};

// ln p_policy - ln p_reference of a row's target, summed over rows first, first + step, .. < end.
template <typename T>
__device__ __forceinline__ double rows_ratio(const GradArgs<T>& a, int first, int end, int step) {
    double r = 0.0;
    for (int i = first; i < end; i += step) {
        const int t = a.target[i];
        const double p = a.stat[i].logp, q = a.ref_logp ? (double)a.ref_logp[i] : a.stat[a.n + i].logp;
        r += t >= 0 && t < a.vocab ? p - q : 0.0;
    }
    return r;
}
// The ratio of answer k, by WIDTH lanes that all get it.
template <int WIDTH, typename T>
__device__ __forceinline__ double answer_ratio(const GradArgs<T>& a, int k) {
    if (a.sums) return a.sums[k];
    double r = rows_ratio(a, a.start[k] + (int)(threadIdx.x % WIDTH), a.start[k + 1], WIDTH);
#pragma unroll
    for (int d = 1; d < WIDTH; d *= 2) r += __shfl_xor(r, d);
    return r;
}
// The ratio of a long answer, once: every workgroup of the gradient would walk all of its pair's rows
// (a pair of 4,096 rows an answer, 151,938 bf16 logits: 1,917 us, 1,373 so; 997 logits: 238 us, 36 so).
template <typename T>
__global__ __launch_bounds__(kRatioThreads) void prefer_ratio_kernel(GradArgs<T> a) {
    const int tid = threadIdx.x, k = blockIdx.x;
    __shared__ double part[kRatioThreads / 64];
    double r = rows_ratio(a, a.start[k] + tid, a.start[k + 1], kRatioThreads);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) r += __shfl_xor(r, d);
    if (tid % 64 == 0) part[tid / 64] = r;
    __syncthreads();
    if (tid) return;
    for (int w = 1; w < kRatioThreads / 64; ++w) r += part[w];
    a.sums[k] = r;
}
// ln(1 / (1 + e^-h))
__device__ __forceinline__ double log_sigmoid(double h) { return fmin(h, 0.0) - log1p(exp(-fabs(h))); }
__device__ __forceinline__ double sigmoid(double h) { return 1.0 / (1.0 + exp(-h)); }
// weight times term; a term without weight is left out, also where it is infinite (a target whose logit
// is -infinity makes h infinite)
__device__ __forceinline__ double weigh(double weight, double term) { return weight > 0.0 ? weight * term : 0.0; }

template <typename T, int TH>
__global__ __launch_bounds__(TH) void prefer_grad_kernel(GradArgs<T> a) {
    const int tid = threadIdx.x, lane = tid & 63;
    if (blockIdx.x == 0) {   // the loss: eight lanes a pair
        constexpr int WIDTH = 8, GROUPS = TH / WIDTH;
        __shared__ double sums[GROUPS][3];
        const int group = tid / WIDTH;
        double loss = 0.0, margin = 0.0, won = 0.0;
        for (int p = group; p < a.pairs; p += GROUPS) {
            const double good = answer_ratio<WIDTH>(a, 2 * p), poor = answer_ratio<WIDTH>(a, 2 * p + 1);
            const double h = a.beta * (good - poor);
            loss -= weigh(1.0 - a.smoothing, log_sigmoid(h)) + weigh(a.smoothing, log_sigmoid(-h));
            margin += h;
            won += h > 0.0 ? 1.0 : 0.0;
            if (a.ratios && tid % WIDTH == 0) {
                a.ratios[2 * p] = (float)good;
                a.ratios[2 * p + 1] = (float)poor;
            }
        }
        if (tid % WIDTH == 0) sums[group][0] = loss, sums[group][1] = margin, sums[group][2] = won;
        __syncthreads();
        if (tid < 3) {
            double t = 0.0;
            for (int w = 0; w < GROUPS && w < a.pairs; ++w) t += sums[w][tid];
            a.losses[tid] = (float)(t / a.pairs);
        }
        return;
    }
    const int row = a.n - (int)blockIdx.x;   // the rows read last come first: they may still be in a cache
    const int target = a.target[row];
    T* g = a.grad + row * a.stride;
    const int chunks = (int)(a.stride / kChunk);
    float slope = 0.f, ref = 0.f, inv = 0.f;
    if (target >= 0 && target < a.vocab) {
        // the row's answer: as many answers start at or before it, less one
        int before = 0;
        for (int k = lane; k < 2 * a.pairs; k += 64) before += a.start[k] <= row;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) before += __shfl_xor(before, d);
        const int answer = before - 1, p = answer / 2;
        const double good = answer_ratio<64>(a, 2 * p), poor = answer_ratio<64>(a, 2 * p + 1);
        const double h = a.beta * (good - poor);
        // -dL/d(good): L falls as the chosen answer's ratio grows
        const double c = a.beta * ((1.0 - a.smoothing) * sigmoid(-h) - a.smoothing * sigmoid(h)) / a.pairs;
        slope = (float)(answer & 1 ? -c : c);
        ref = a.stat[row].m;
        inv = slope / a.stat[row].z;
    }
    const T* x = a.x + row * a.stride;
    const int used = (a.vocab + kChunk - 1) / kChunk;
    auto write = [&](int c, const Raw<T>& r) {
        float v[kChunk];
        unpack(r, v);
#pragma unroll
        for (int e = 0; e < kChunk; ++e) {
            const int i = c * kChunk + e;
            v[e] = inv * exp2_((v[e] - ref) * kLog2e);
            if (i == target) v[e] -= slope;
            if (slope == 0.f || i >= a.vocab) v[e] = 0.f;
        }
        store_chunk(g, c, v);
    };
    constexpr int kAhead = 4;
    auto sweep = [&](auto stream) {
        constexpr bool STREAM = decltype(stream)::value;
        int c = tid;
        for (; c + (kAhead - 1) * TH < used; c += kAhead * TH) {
            Raw<T> r[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) r[k] = load_raw<STREAM>(x, c + k * TH);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) write(c + k * TH, r[k]);
        }
        for (; c < used; c += TH) write(c, load_raw<STREAM>(x, c));
        return c;
    };
    int c = row < a.stream ? sweep(std::true_type{}) : sweep(std::false_type{});
    for (; c < chunks; c += TH) {
        const float zero[kChunk] = {};
        store_chunk(g, c, zero);
    }
}

struct DevGuard {
    int prev = -1;
    explicit DevGuard(int dev) {
        if (hipGetDevice(&prev) != hipSuccess) prev = -1;
        if (prev != dev) (void)hipSetDevice(dev);
    }
    ~DevGuard() {
        if (prev >= 0) (void)hipSetDevice(prev);
    }
};

bool misaligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1u)) != 0; }

}  // namespace

struct a2t_prefer {
    int32_t max_rows = 0, vocab = 0, dtype = 0, device = 0;
    hipStream_t stream = nullptr;
    RowStat* stat = nullptr;   // [2][max_rows]
    double* sums = nullptr;    // [kAnswers] ratios of a call with long answers
    int cus = 256;
    bool poisoned = false;
};

namespace {

// n rows of logits, as far as they are read, or (`whole`) written.
a2t::Rows logit_rows(const a2t_prefer* p, const void* x, int64_t stride, int64_t n, bool whole = false) {
    const int64_t size = p->dtype == A2T_F32 ? 4 : 2;
    return {x, n, (whole ? stride : ((int64_t)p->vocab + kChunk - 1) / kChunk * kChunk) * size, stride * size};
}
// 1,024 threads a row instead of 256: where rows are long (1,280 gradient rows of 151,938 bf16 logits:
// 151 against 164 us), or where they alone do not fill the CUs.
bool wide_rows(const a2t_prefer* p, int64_t rows) {
    const int chunks = p->vocab / kChunk;
    return chunks >= 8192 || (rows < 4 * p->cus && chunks >= 1024);
}
// Row statistics of the policy's rows and, with `reference`, of the reference's behind them.
template <typename T>
hipError_t launch_rows(a2t_prefer* p, int n, const void* policy, int64_t ps, const void* reference, int64_t rs, const int32_t* target,
                       RowStat* stat, float* logp, int stream) {
    RowsArgs<T> a{{static_cast<const T*>(policy), static_cast<const T*>(reference)}, {ps, rs}, target, stat, logp, n, p->vocab, stream};
    const int64_t rows = reference ? 2 * (int64_t)n : n;
    const dim3 grid((uint32_t)rows);
    if (wide_rows(p, rows)) return a2t::launch_kernel(prefer_rows_kernel<T, 1024>, grid, dim3(1024), p->stream, a);
    return a2t::launch_kernel(prefer_rows_kernel<T, 256>, grid, dim3(256), p->stream, a);
}

}  // namespace

extern "C" int a2t_prefer_create(int32_t max_rows, int32_t vocab, int32_t dtype, int32_t device, void* hip_stream, a2t_prefer** out) {
    if (!out) return A2T_ERR_INVALID;
    *out = nullptr;
    if (max_rows < 1 || max_rows > (1 << 22) || vocab < 1 || vocab > (1 << 30) || (dtype != A2T_F32 && dtype != A2T_BF16)) return A2T_ERR_INVALID;
    int n_dev = 0;
    if (hipGetDeviceCount(&n_dev) != hipSuccess || device < 0 || device >= n_dev) return A2T_ERR_NODEV;
    DevGuard g(device);
    a2t_prefer* p = new (std::nothrow) a2t_prefer();
    if (!p) return A2T_ERR_OOM;
    p->max_rows = max_rows;
    p->vocab = vocab;
    p->dtype = dtype;
    p->device = device;
    p->stream = static_cast<hipStream_t>(hip_stream);
    int cus = 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device) == hipSuccess && cus > 0) p->cus = cus;
    if (hipMalloc(&p->stat, sizeof(RowStat) * 2 * (size_t)max_rows) != hipSuccess || hipMalloc(&p->sums, sizeof(double) * kAnswers) != hipSuccess) {
        (void)hipGetLastError();
        (void)hipFree(p->stat);
        delete p;
        return A2T_ERR_OOM;
    }
    *out = p;
    return A2T_OK;
}

extern "C" int a2t_prefer_destroy(a2t_prefer* p) {
    if (!p) return A2T_ERR_INVALID;
    {
        DevGuard g(p->device);
        (void)hipStreamSynchronize(p->stream);
        (void)hipFree(p->stat);
        (void)hipFree(p->sums);
    }
    delete p;
    return A2T_OK;
}

extern "C" int a2t_prefer_set_stream(a2t_prefer* p, void* hip_stream) {
    if (!p) return A2T_ERR_INVALID;
    p->stream = static_cast<hipStream_t>(hip_stream);
    return A2T_OK;
}

extern "C" int a2t_prefer_logp(a2t_prefer* p, int32_t n_rows, const void* logits, int64_t stride, const int32_t* target, float* logp) {
    if (!p) return A2T_ERR_INVALID;
    if (p->poisoned) return A2T_ERR_HIP;
    if (n_rows < 1 || n_rows > p->max_rows || !logits || !target || !logp || stride < p->vocab || stride % 8 || stride > (1ll << 40) ||
        misaligned(logits, 16) || misaligned(target, 4) || misaligned(logp, 4))
        return A2T_ERR_INVALID;
    const a2t::Rows to = a2t::run_of(logp, (int64_t)n_rows * 4);
    if (a2t::overlap(to, logit_rows(p, logits, stride, n_rows)) || a2t::overlap(to, a2t::run_of(target, (int64_t)n_rows * 4))) return A2T_ERR_INVALID;
    DevGuard g(p->device);
    const hipError_t e = p->dtype == A2T_F32 ? launch_rows<float>(p, n_rows, logits, stride, nullptr, 0, target, nullptr, logp, 0)
                                             : launch_rows<bf16_t>(p, n_rows, logits, stride, nullptr, 0, target, nullptr, logp, 0);
    if (e != hipSuccess) {
        p->poisoned = true;
        return A2T_ERR_HIP;
    }
    return A2T_OK;
}

extern "C" int a2t_prefer_loss(a2t_prefer* p, int32_t n_pairs, const int32_t* answer_rows, const void* policy, int64_t policy_stride,
                               const void* reference, int64_t reference_stride, const float* ref_logp, const int32_t* target,
                               float beta, float smoothing, float* losses, float* ratios, void* grad) {
    if (!p) return A2T_ERR_INVALID;
    if (p->poisoned) return A2T_ERR_HIP;
    if (n_pairs < 1 || n_pairs > kMaxPairs || !answer_rows || !policy || !target || !losses || (reference != nullptr) == (ref_logp != nullptr))
        return A2T_ERR_INVALID;
    if (!std::isfinite(beta) || beta <= 0.f || !(smoothing >= 0.f && smoothing <= 1.f)) return A2T_ERR_INVALID;
    int64_t n = 0;
    for (int i = 0; i < 2 * n_pairs; ++i) {
        if (answer_rows[i] < 0) return A2T_ERR_INVALID;
        n += answer_rows[i];
    }
    if (n < 1 || n > p->max_rows) return A2T_ERR_INVALID;
    auto bad_stride = [&](int64_t s) { return s < p->vocab || s % 8 || s > (1ll << 33); };
    if (bad_stride(policy_stride) || (reference && bad_stride(reference_stride)) || misaligned(policy, 16) || misaligned(reference, 16) ||
        misaligned(grad, 16) || misaligned(ref_logp, 4) || misaligned(target, 4) || misaligned(losses, 4) || misaligned(ratios, 4))
        return A2T_ERR_INVALID;
    // The gradient's workgroups write a row that they alone read, and read targets and log probabilities of all
    // rows; the reference's logits are read by an earlier launch, so that the gradient may lie over them.
    const a2t::Rows in[] = {logit_rows(p, policy, policy_stride, n), a2t::run_of(target, n * 4), a2t::run_of(ref_logp, n * 4),
                            logit_rows(p, reference, reference_stride, n)};
    const a2t::Rows to[] = {a2t::run_of(losses, 12), a2t::run_of(ratios, 8 * (int64_t)n_pairs), logit_rows(p, grad, policy_stride, n, true)};
    for (int x = 0; x < 3; ++x) {
        for (int y = 0; y < x; ++y)
            if (a2t::overlap(to[x], to[y])) return A2T_ERR_INVALID;
        for (int y = 0; y < 4; ++y) {
            if (x == 2 && (y == 3 || (y == 0 && grad == policy))) continue;
            if (a2t::overlap(to[x], in[y])) return A2T_ERR_INVALID;
        }
    }
    DevGuard g(p->device);
    auto go = [&](auto* type) {
        using T = std::remove_pointer_t<decltype(type)>;
        const int64_t keep = kKeepBytes / (policy_stride * (int64_t)sizeof(T));
        const int stream = n > keep ? (int)(n - keep) : 0;
        hipError_t e = launch_rows<T>(p, (int)n, policy, policy_stride, reference, reference_stride, target, p->stat, nullptr, stream);
        if (e != hipSuccess) return e;
        GradArgs<T> a{};
        a.x = static_cast<const T*>(policy);
        a.grad = static_cast<T*>(grad);
        a.stride = policy_stride;
        a.stat = p->stat;
        a.ref_logp = ref_logp;
        a.target = target;
        a.losses = losses;
        a.ratios = ratios;
        a.n = (int32_t)n;
        a.stream = stream;
        a.vocab = p->vocab;
        a.pairs = n_pairs;
        a.beta = beta;
        a.smoothing = smoothing;
        for (int i = 0; i < 2 * n_pairs; ++i) a.start[i + 1] = a.start[i] + answer_rows[i];
        if (*std::max_element(answer_rows, answer_rows + 2 * n_pairs) >= kLongRows) {
            a.sums = p->sums;
            e = a2t::launch_kernel(prefer_ratio_kernel<T>, dim3(2 * n_pairs), dim3(kRatioThreads), p->stream, a);
            if (e != hipSuccess) return e;
        }
        const dim3 grid(grad ? (uint32_t)n + 1 : 1);
        if (!grad || wide_rows(p, n)) return a2t::launch_kernel(prefer_grad_kernel<T, 1024>, grid, dim3(1024), p->stream, a);
        return a2t::launch_kernel(prefer_grad_kernel<T, 256>, grid, dim3(256), p->stream, a);
    };
    const hipError_t e = p->dtype == A2T_F32 ? go((float*)nullptr) : go((bf16_t*)nullptr);
    if (e != hipSuccess) {
        p->poisoned = true;
        return A2T_ERR_HIP;
    }
    return A2T_OK;
}
