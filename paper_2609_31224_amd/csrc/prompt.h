// Internal interface of the attention over packed sequences (a2t_prompt_* of include/a2t.h):
// what the host hands to the kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace a2t {
namespace prompt {

// Most sequences of a launch (their table travels in the kernel's arguments: 3 KiB of 4).
constexpr int kMaxSeqs = 256;
// Rows of a workgroup: packed query rows (G n of a KV head) of the forward and dQ kernels, keys
// of the dK, dV kernel.
constexpr int kBlock = 128;

// The sequences of a launch, longest first, and the first block of each (blocks of a sequence
// follow each other).
template <int N>
struct SeqTable {
    int32_t count;
    int32_t block0[N];
    int32_t row0[N];
    int32_t rows[N];
};

// Keys and values as the kernels read them.  Row r of a sequence is its key r, expiring at `until`
// if that is given, unless `meta` is: then the rows are sorted (lasting keys first) and meta tells
// each one's place and the first place that does not see it.
struct KeyRows {
    const void* k;
    const void* v;
    int64_t k_stride, v_stride;   // elements between rows
    const int32_t* until;         // [rows] or null
    const int2* meta;             // [rows] (place, until) or null
    const int32_t* lasting;       // [rows] lasting keys at or before the place
    const int32_t* first;         // [rows] first passing key (in sorted order) that the place may still see
};

struct Args {
    KeyRows kv;
    const void* q;
    int64_t q_stride;
    void* o;
    const void* o_in;
    const void* d_o;
    float* lse;             // [Hq][total]
    float* delta;           // [Hq][total] sum of dO O
    void* dq;               // rows at the strides of q, k and v
    void* dk;
    void* dv;
    int64_t k_out, v_out;
    int32_t Hq, Hkv, G;
    int32_t total;          // packed rows
    uint32_t inv_g;         // ceil(2^16 / G)
    float scale, scale_log2e;
    // a block's tiles may be split over several workgroups: their fp32 sums go to `part`
    int32_t splits;
    float* part;
};

struct Shape {
    bool f32;
    int head_dim;
};

hipError_t launch_forward(const Shape& s, const Args& a, const SeqTable<kMaxSeqs>& t, int blocks, hipStream_t stream);
hipError_t launch_dq(const Shape& s, const Args& a, const SeqTable<kMaxSeqs>& t, int blocks, hipStream_t stream);
hipError_t launch_dkv(const Shape& s, const Args& a, const SeqTable<kMaxSeqs>& t, int blocks, hipStream_t stream);

// Sorts the keys of sequences for calls with `until`: lasting keys (seen by every later row of
// the sequence) first, then the passing ones, each in order.  Two launches: what a place's keys are
// (one workgroup a sequence), then the rows' copies.
struct SortArgs {
    const int32_t* until;
    const void* k;
    const void* v;
    int64_t k_stride, v_stride;   // bytes between rows
    void* k_out;                  // [rows][row_bytes]
    void* v_out;
    int32_t row_bytes;            // of all KV heads
    int2* meta;
    int32_t* lasting;
    int32_t* first;
    int32_t* reach;               // [rows] scratch: largest `until` among the passing keys up to each
};
hipError_t launch_sort(const SortArgs& a, const SeqTable<kMaxSeqs>& t, hipStream_t stream);

// Calls f with the table in the smallest of four sizes: a launch copies its arguments.
template <class F>
hipError_t by_count(const SeqTable<kMaxSeqs>& t, F&& f) {
    auto as = [&](auto size) {
        constexpr int N = decltype(size)::value;
        SeqTable<N> s{};
        s.count = t.count;
        for (int i = 0; i < N && i < t.count; ++i) s.block0[i] = t.block0[i], s.row0[i] = t.row0[i], s.rows[i] = t.rows[i];
        return f(s);
    };
    if (t.count <= 1) return as(std::integral_constant<int, 1>{});
    if (t.count <= 16) return as(std::integral_constant<int, 16>{});
    if (t.count <= 64) return as(std::integral_constant<int, 64>{});
    return f(t);
}

}  // namespace prompt
}  // namespace a2t
