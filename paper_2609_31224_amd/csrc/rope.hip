// Rotary encoding of packed rows of queries and keys and its gradient (gfx950).
// Public API: include/a2t.h (a2t_rope_*).
//
// Row t turns channel pairs (x, y) of its first r channels by the angle a = pos_t f_i:
//   x' = m (x cos a - y sin a),  y' = m (y cos a + x sin a)
// (the gradient by -a); the other channels are copied.  Angles are products in 64 bits,
// reduced to a fraction of a turn there; sine and cosine of the fraction are fp32.
//
// Bound: HBM, every element read and written once.  A workgroup takes a few rows: it
// evaluates their r / 2 angles once, into LDS, and then every thread turns 8 pairs at a
// time (two 16-byte chunks of bf16) of one head after the other, so that the 64-bit
// arithmetic is shared by all heads of a row.
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

constexpr int kThreads = 256;
constexpr int kMaxRows = 8;       // most rows of a workgroup
// Outputs larger than the L2 caches (32 MiB together) are stored past them (three sets of inputs in turn,
// 40 bf16 heads of 128: 5,000 rows 17.2 us against 21.2, 16,384 rows 67.8 against 71.7, 32,768 rows 132 against 136).
constexpr int64_t kStreamBytes = 32 << 20;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
struct bf16_t {
    uint16_t bits;
};

struct RopeArgs {
    double turns[64];     // f_i / (2 pi)
    const int32_t* pos;
    const void* in[2];    // queries, keys
    void* out[2];
    int64_t in_stride[2], out_stride[2];   // elements between rows
    int32_t heads0, heads;                 // heads of the queries, of both
    uint64_t inv_heads;                    // ceil(2^32 / heads)
    int32_t n, rows;                       // rows, rows of a workgroup
    int32_t part2, half;                   // r / 2; pairs (i, i + r/2) or (2i, 2i + 1)
    float m, sign;
};

// the elements of 16 bytes
__device__ __forceinline__ void load(const bf16_t* p, float (&x)[8]) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(w[e] << 16);
        x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load(const float* p, float (&x)[4]) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(w[e]);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
    const bf16x2 v = {(__bf16)a, (__bf16)b};   // round to nearest even, once per output
    return __builtin_bit_cast(uint32_t, v);
}
template <bool STREAM>
__device__ __forceinline__ void store16(void* p, const u32x4& x) {
    if (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(p));
    else *reinterpret_cast<u32x4*>(p) = x;
}
template <bool STREAM>
__device__ __forceinline__ void store(bf16_t* p, const float (&x)[8]) {
    store16<STREAM>(p, u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])});
}
template <bool STREAM>
__device__ __forceinline__ void store(float* p, const float (&x)[4]) {
    store16<STREAM>(p, u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])});
}

template <typename T, int D, bool STREAM>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
    __shared__ __align__(16) float2 s_cs[kMaxRows][D / 2];
    const int tid = threadIdx.x, row0 = blockIdx.x * a.rows, rows = min(a.rows, a.n - row0);
    for (int k = tid; k < rows * (D / 2); k += kThreads) {
        const int r = k / (D / 2), i = k % (D / 2);
        if (i >= a.part2) continue;
        double t = (double)a.pos[row0 + r] * a.turns[i];
        t -= rint(t);
        float s, c;
        sincospif(2.f * (float)t, &s, &c);
        s_cs[r][i] = make_float2(a.m * c, a.sign * a.m * s);
    }
    __syncthreads();
    // A unit is two chunks of 16 bytes, P elements each.  Lanes next to each other take chunks next to
    // each other, so that every access is whole lines.
    constexpr int P = 16 / (int)sizeof(T), U = D / (2 * P);   // units of a head
    const int u = tid % U, part = 2 * a.part2, rest = (D - part) / 2;
    const bool both = a.half && u < a.part2 / P;              // half layout: the chunks are each other's partners
    const int c0 = !a.half || both ? P * u : part + P * u - a.part2;
    const int c1 = c0 + (!a.half ? D / 2 : both ? a.part2 : rest);
    // pairs layout: each chunk has its own pairs, or none
    const bool turn0 = !a.half && c0 < part, turn1 = !a.half && c1 < part, moves = both || turn0 || turn1;
    const int all = rows * a.heads;       // heads of all rows
    constexpr int STEP = kThreads / U;
    struct Unit {
        float x[P], y[P];
        T* out;
        int row;
        bool here;
    };
    auto fetch = [&](Unit& t, int k) {
        t.here = k < all;
        if (!t.here) return;
        t.row = (int)((uint64_t)(uint32_t)k * a.inv_heads >> 32);
        const int h = k - t.row * a.heads, which = h >= a.heads0;
        const int64_t row = row0 + t.row;
        const int head = (h - (which ? a.heads0 : 0)) * D;
        const T* in = static_cast<const T*>(a.in[which]) + row * a.in_stride[which] + head;
        t.out = static_cast<T*>(a.out[which]) + row * a.out_stride[which] + head;
        if (!moves && in == t.out) t.here = false;
        load(in + c0, t.x);
        load(in + c1, t.y);
    };
    auto finish = [&](Unit& t) {
        if (!t.here) return;
        if (both) {
            float p[P], q[P];
            const float2* cs = &s_cs[t.row][P * u];
#pragma unroll
            for (int e = 0; e < P; ++e) {
                p[e] = t.x[e] * cs[e].x - t.y[e] * cs[e].y;
                q[e] = t.y[e] * cs[e].x + t.x[e] * cs[e].y;
            }
            store<STREAM>(t.out + c0, p);
            store<STREAM>(t.out + c1, q);
            return;
        }
        auto pairs = [&](float (&x)[P], const float2* cs) {
#pragma unroll
            for (int e = 0; e < P / 2; ++e) {
                const float a = x[2 * e], b = x[2 * e + 1];
                x[2 * e] = a * cs[e].x - b * cs[e].y;
                x[2 * e + 1] = b * cs[e].x + a * cs[e].y;
            }
        };
        if (turn0) pairs(t.x, &s_cs[t.row][c0 / 2]);
        if (turn1) pairs(t.y, &s_cs[t.row][c1 / 2]);
        store<STREAM>(t.out + c0, t.x);
        store<STREAM>(t.out + c1, t.y);
    };
    // a unit's loads are under way while another is finished (in place, a unit's elements are its own)
    Unit a0, a1;
    fetch(a0, tid / U);
    for (int k = tid / U; k < all; k += 2 * STEP) {
        fetch(a1, k + STEP);
        finish(a0);
        fetch(a0, k + 2 * STEP);
        finish(a1);
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

}  // namespace

struct a2t_rope {
    a2t_rope_config cfg{};
    int32_t part = 0;
    double freq[64] = {};
    double m = 1.0;
    hipStream_t stream = nullptr;
    int cus = 256;
    bool poisoned = false;
};

extern "C" int a2t_rope_create(const a2t_rope_config* cfg, void* hip_stream, a2t_rope** out) {
    if (!out) return A2T_ERR_INVALID;
    *out = nullptr;
    if (!cfg) return A2T_ERR_INVALID;
    const int D = cfg->head_dim, part = cfg->rotary_dim ? cfg->rotary_dim : D;
    const double theta = cfg->theta == 0.0 ? 1e6 : cfg->theta;
    if ((D != 64 && D != 128) || part < 16 || part > D || part % 16 || (cfg->dtype != A2T_F32 && cfg->dtype != A2T_BF16) ||
        (cfg->layout != A2T_ROPE_HALF && cfg->layout != A2T_ROPE_PAIRS) || !std::isfinite(theta) || theta <= 1.0)
        return A2T_ERR_INVALID;
    const double f = cfg->factor;
    if (cfg->scaling < A2T_ROPE_PLAIN || cfg->scaling > A2T_ROPE_YARN) return A2T_ERR_INVALID;
    if (cfg->scaling != A2T_ROPE_PLAIN && (!std::isfinite(f) || f < 1.0)) return A2T_ERR_INVALID;
    if (cfg->scaling == A2T_ROPE_YARN &&
        (cfg->trained_rows < 1 || !std::isfinite(cfg->turns_fast) || !std::isfinite(cfg->turns_slow) ||
         cfg->turns_slow <= 0.0 || cfg->turns_fast < cfg->turns_slow))
        return A2T_ERR_INVALID;
    int n_dev = 0;
    if (hipGetDeviceCount(&n_dev) != hipSuccess || cfg->device < 0 || cfg->device >= n_dev) return A2T_ERR_NODEV;
    a2t_rope* r = new (std::nothrow) a2t_rope();
    if (!r) return A2T_ERR_OOM;
    r->cfg = *cfg;
    r->part = part;
    r->stream = static_cast<hipStream_t>(hip_stream);
    int cus = 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, cfg->device) == hipSuccess && cus > 0) r->cus = cus;
    const double pi = 3.14159265358979323846;
    const double base = cfg->scaling == A2T_ROPE_NTK ? theta * std::pow(f, part / (part - 2.0)) : theta;
    // channel pair whose wavelength fits `turns` times into the trained rows
    auto pair_of = [&](double turns) { return part * std::log(cfg->trained_rows / (turns * 2 * pi)) / (2 * std::log(theta)); };
    double low = 0, high = 1;
    if (cfg->scaling == A2T_ROPE_YARN) {
        low = std::fmax(std::floor(pair_of(cfg->turns_fast)), 0.0);
        high = std::fmin(std::ceil(pair_of(cfg->turns_slow)), part - 1.0);
        r->m = 0.1 * std::log(f) + 1.0;
    }
    for (int i = 0; i < part / 2; ++i) {
        double w = std::pow(base, -2.0 * i / part);
        if (cfg->scaling == A2T_ROPE_LINEAR) w /= f;
        if (cfg->scaling == A2T_ROPE_YARN) {
            const double ramp = std::fmin(1.0, std::fmax(0.0, (i - low) / std::fmax(high - low, 1e-3)));
            w = w * (1.0 - ramp) + w / f * ramp;
        }
        r->freq[i] = w;
    }
    *out = r;
    return A2T_OK;
}

extern "C" int a2t_rope_destroy(a2t_rope* r) {
    if (!r) return A2T_ERR_INVALID;
    delete r;
    return A2T_OK;
}

extern "C" int a2t_rope_set_stream(a2t_rope* r, void* hip_stream) {
    if (!r) return A2T_ERR_INVALID;
    r->stream = static_cast<hipStream_t>(hip_stream);
    return A2T_OK;
}

extern "C" int a2t_rope_apply(a2t_rope* r, int32_t n_rows, const int32_t* pos, int32_t q_heads, const void* q, int64_t q_stride,
                              void* q_out, int64_t q_out_stride, int32_t k_heads, const void* k, int64_t k_stride, void* k_out,
                              int64_t k_out_stride, int32_t grad) {
    if (!r) return A2T_ERR_INVALID;
    if (r->poisoned) return A2T_ERR_HIP;
    const int D = r->cfg.head_dim, size = r->cfg.dtype == A2T_F32 ? 4 : 2;
    if (n_rows < 1 || n_rows > (1 << 26) || !pos || (reinterpret_cast<uintptr_t>(pos) & 3u)) return A2T_ERR_INVALID;
    if (!q) q_heads = 0;
    if (!k) k_heads = 0;
    if (q_heads < 0 || k_heads < 0 || (q && q_heads < 1) || (k && k_heads < 1) || q_heads + (int64_t)k_heads < 1 ||
        q_heads + (int64_t)k_heads > 4096)
        return A2T_ERR_INVALID;
    auto bad = [&](int heads, const void* in, int64_t is, const void* out, int64_t os) {
        if (!heads) return false;
        return !out || (((uintptr_t)in | (uintptr_t)out) & 15u) || is < (int64_t)heads * D || os < (int64_t)heads * D || is % 8 || os % 8 ||
               std::max(is, os) > (1ll << 56) / n_rows;
    };
    if (bad(q_heads, q, q_stride, q_out, q_out_stride) || bad(k_heads, k, k_stride, k_out, k_out_stride)) return A2T_ERR_INVALID;
    // an output is in place of its own input, row for row, or apart from everything: workgroups read theirs
    // at different times
    auto rows = [&](const void* p, int heads, int64_t stride) { return a2t::Rows{p, n_rows, (int64_t)heads * D * size, stride * size}; };
    const a2t::Rows in[] = {rows(q, q_heads, q_stride), rows(k, k_heads, k_stride), a2t::run_of(pos, (int64_t)n_rows * 4)};
    const a2t::Rows to[] = {rows(q ? q_out : nullptr, q_heads, q_out_stride), rows(k ? k_out : nullptr, k_heads, k_out_stride)};
    if (a2t::overlap(to[0], to[1])) return A2T_ERR_INVALID;
    for (int x = 0; x < 2; ++x)
        for (int y = 0; y < 3; ++y)
            if (!(x == y && to[x].p == in[x].p && to[x].stride == in[x].stride) && a2t::overlap(to[x], in[y])) return A2T_ERR_INVALID;
    DevGuard g(r->cfg.device);
    RopeArgs a{};
    const double two_pi = 6.28318530717958647692;
    for (int i = 0; i < r->part / 2; ++i) a.turns[i] = r->freq[i] / two_pi;
    a.pos = pos;
    a.in[0] = q, a.in[1] = k;
    a.out[0] = q_out, a.out[1] = k_out;
    a.in_stride[0] = q_stride, a.in_stride[1] = k_stride;
    a.out_stride[0] = q_out_stride, a.out_stride[1] = k_out_stride;
    a.heads0 = q_heads;
    a.heads = q_heads + k_heads;
    a.inv_heads = ((1ull << 32) + a.heads - 1) / a.heads;
    a.n = n_rows;
    a.part2 = r->part / 2;
    a.half = r->cfg.layout == A2T_ROPE_HALF;
    a.m = (float)r->m;
    a.sign = grad ? -1.f : 1.f;
    // as many rows a workgroup as leave every CU a few workgroups
    a.rows = 1;
    while (a.rows < kMaxRows && (int64_t)n_rows >= (int64_t)a.rows * 2 * 4 * r->cus) a.rows *= 2;
    const dim3 grid((n_rows + a.rows - 1) / a.rows);
    auto go = [&](auto kernel) { return a2t::launch_kernel(kernel, grid, dim3(kThreads), r->stream, a); };
    const bool stream = (int64_t)n_rows * a.heads * D * size > kStreamBytes;
    auto typed = [&](auto* type) {
        using T = std::remove_pointer_t<decltype(type)>;
        if (D == 64) return stream ? go(rope_kernel<T, 64, true>) : go(rope_kernel<T, 64, false>);
        return stream ? go(rope_kernel<T, 128, true>) : go(rope_kernel<T, 128, false>);
    };
    if ((r->cfg.dtype == A2T_F32 ? typed((float*)nullptr) : typed((bf16_t*)nullptr)) != hipSuccess) {
        r->poisoned = true;
        return A2T_ERR_HIP;
    }
    return A2T_OK;
}
