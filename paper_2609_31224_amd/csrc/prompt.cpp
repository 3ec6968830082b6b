// Host side of the attention over packed sequences (a2t_prompt_* of include/a2t.h): argument
// checks, the table of sequences that a launch carries, and the launches.
#include "../../include/a2t.h"
#include "overlap.h"
#include "prompt.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdlib>
#include <new>

using namespace a2t::prompt;

namespace {
constexpr int kTileRows = 64;
constexpr int kSortRows = 10240;                 // query rows (rows x heads) of the longest sequence from which keys that expire are sorted
}  // namespace

struct a2t_prompt {
    int32_t max_rows = 0, Hq = 0, Hkv = 0, D = 0, dtype = 0, device = 0;
    double scale = 0.0;
    hipStream_t stream = nullptr;
    float* delta = nullptr;      // [Hq][rows of the call]
    float* part = nullptr;       // sums of split blocks
    int64_t part_rows = 0;       // (row, head, split) triples that fit it
    int cus = 256;
    // handles for calls with `until`: sorted copies of K and V, and what the kernels know of them
    void* k = nullptr;
    void* v = nullptr;
    int2* meta = nullptr;
    int32_t* lasting = nullptr;
    int32_t* first = nullptr;
    int32_t* reach = nullptr;
    bool until = false;
    int sort_rows = kSortRows;   // A2T_PROMPT_SORT
    int force_splits = 0;        // A2T_PROMPT_SPLITS
    bool poisoned = false;
};

namespace {

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

int env_int(const char* name, int dflt) {
    const char* v = std::getenv(name);
    return (v && *v) ? std::atoi(v) : dflt;
}

void free_prompt(a2t_prompt* p) {
    for (void* m : {(void*)p->delta, p->k, p->v, (void*)p->meta, (void*)p->lasting, (void*)p->first, (void*)p->reach, (void*)p->part})
        if (m) (void)hipFree(m);
    delete p;
}

constexpr int kSplitSeqs = 64;                   // launches of more sequences are not split
constexpr int64_t kPartRows = 1 << 18;           // most (row, head, split) triples of split sums (130 MiB of 128 dimensions)

bool misaligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1u)) != 0; }

// A call's rows, checked: 0 where something is wrong with them.
int64_t total_rows(const a2t_prompt* p, int32_t n_seqs, const int32_t* seq_rows) {
    if (n_seqs < 1 || !seq_rows) return 0;
    int64_t total = 0;
    for (int32_t i = 0; i < n_seqs; ++i) {
        if (seq_rows[i] < 0) return 0;
        total += seq_rows[i];
        if (total > p->max_rows) return 0;
    }
    return total;
}

bool bad_rows(const a2t_prompt* p, const void* x, int64_t stride, int heads) {
    return !x || misaligned(x, 16) || stride < (int64_t)heads * p->D || stride % 8 || stride > (1 << 22);
}

// A call's outputs and inputs in memory.  Every output is written while other workgroups, or a later
// launch of the call, still read the inputs: they must not touch each other, but for an output that is
// `in_place` of one operand, row for row, where whoever reads a row is who writes it (or was a launch
// before).  That holds for the operand, not for its memory: another one may be there too.
struct Memory {
    const a2t_prompt* p;
    int64_t total;
    a2t::Rows out[3], in[7];
    int outs = 0, ins = 0;
    a2t::Rows rows(const void* x, int64_t stride, int heads) const {
        const int64_t size = p->dtype == A2T_F32 ? 4 : 2;
        return {x, total, (int64_t)heads * p->D * size, stride * size};
    }
    a2t::Rows packed(const void* x) const { return rows(x, (int64_t)p->Hq * p->D, p->Hq); }
    a2t::Rows floats(const void* x, int64_t n) const { return a2t::run_of(x, n * 4); }
    // in_place[i]: the input that output i may be, or -1
    bool clash(const int (&in_place)[3]) const {
        for (int i = 0; i < outs; ++i) {
            for (int j = 0; j < i; ++j)
                if (a2t::overlap(out[i], out[j])) return true;
            for (int j = 0; j < ins; ++j) {
                if (j == in_place[i] && in[j].p == out[i].p && in[j].stride == out[i].stride) continue;
                if (a2t::overlap(out[i], in[j])) return true;
            }
        }
        return false;
    }
};

// Calls f with tables of at most kMaxSeqs sequences, longest first (the launch's last workgroups
// are short ones); sequences without rows take no part.
template <class F>
hipError_t in_tables(int32_t n_seqs, const int32_t* seq_rows, F&& f) {
    struct Seq {
        int32_t row0, rows;
    } s[kMaxSeqs];
    int32_t row0 = 0;
    for (int32_t i = 0; i < n_seqs;) {
        int count = 0;
        for (; i < n_seqs && count < kMaxSeqs; row0 += seq_rows[i++])
            if (seq_rows[i]) s[count++] = {row0, seq_rows[i]};
        if (!count) continue;
        std::sort(s, s + count, [](const Seq& a, const Seq& b) { return a.rows != b.rows ? a.rows > b.rows : a.row0 < b.row0; });
        SeqTable<kMaxSeqs> t;
        t.count = count;
        for (int k = 0; k < count; ++k) t.row0[k] = s[k].row0, t.rows[k] = s[k].rows, t.block0[k] = 0;
        const hipError_t e = f(t);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
// The first block of every sequence of `rows_of(i)` rows; the number of blocks.
template <class F>
int place_blocks(SeqTable<kMaxSeqs>& t, F&& rows_of) {
    int64_t blocks = 0;
    for (int i = 0; i < t.count; ++i) {
        t.block0[i] = (int32_t)blocks;
        blocks += (rows_of(i) + kBlock - 1) / kBlock;
    }
    return (int)blocks;
}

// Whether keys that expire are sorted first: two launches and a copy of K and V against the pairs
// that nobody sees.  (Forward and gradient with 35 % of the keys' lifetimes left, sorted against as they
// are: 32 heads on 8, 200 rows 76 against 63 us, 400 rows 95 against 99, 1,000 rows 132 against 191; 8
// heads on 2, 600 rows 68 against 62, 1,000 rows 80 against 83.)
bool sort_pays(const a2t_prompt* p, int32_t n_seqs, const int32_t* seq_rows) {
    return (int64_t)*std::max_element(seq_rows, seq_rows + n_seqs) * p->Hq >= p->sort_rows;
}

Args base_args(const a2t_prompt* p, int64_t total, const void* q, int64_t qs, const void* k, int64_t ks, const void* v, int64_t vs,
               const int32_t* until, bool sorted) {
    Args a{};
    const int64_t own = (int64_t)p->Hkv * p->D;
    a.kv = KeyRows{k, v, ks, vs, until, nullptr, nullptr, nullptr};
    if (sorted) a.kv = KeyRows{p->k, p->v, own, own, until, p->meta, p->lasting, p->first};
    a.q = q;
    a.q_stride = qs;
    a.delta = p->delta;
    a.k_out = ks;
    a.v_out = vs;
    a.Hq = p->Hq;
    a.Hkv = p->Hkv;
    a.G = p->Hq / p->Hkv;
    a.total = (int32_t)total;
    a.inv_g = (65536u + a.G - 1) / a.G;
    a.part = p->part;
    a.splits = 1;
    a.scale = (float)p->scale;
    a.scale_log2e = (float)(p->scale * 1.44269504088896340736);
    return a;
}
// What a launch's workgroups cost, us: a tile of 64 rows with `per_cu` workgroups on every CU, and a
// workgroup's beginning and end.  (Measured on sequences of 8,192 and 1,500 rows.)
struct Cost {
    double tile, start;
    int per_cu;
};
enum { kForward, kQueries, kKeys };
Cost cost_of(const a2t_prompt* p, int kernel) {
    static const Cost bf16[2][3] = {{{2.4, 3, 4}, {2.6, 3, 3}, {1.7, 4, 1}}, {{2.2, 3, 2}, {2.5, 3, 2}, {2.4, 5, 1}}};
    static const Cost f32[2][3] = {{{7, 3, 2}, {10, 3, 2}, {8.5, 4, 1}}, {{9, 4, 1}, {13, 4, 1}, {17, 5, 1}}};
    return (p->dtype == A2T_F32 ? f32 : bf16)[p->D == 128][kernel];
}
// Workgroups that each block's tiles are split over.  A launch takes about as long as its longest
// workgroup, or as all of them spread over the CUs if that is more; splits cost their sums' way to
// memory and a launch that adds them.
int splits_for(const a2t_prompt* p, const SeqTable<kMaxSeqs>& t, int kernel, int64_t total) {
    if (t.count > kSplitSeqs) return 1;
    const Cost c = cost_of(p, kernel);
    const int64_t G = p->Hq / p->Hkv, slots = (int64_t)p->cus * c.per_cu, heads = kernel == kKeys ? 2 * (int64_t)p->Hkv : p->Hq;
    int64_t wgs = 0, work = 0, longest = 0;
    for (int i = 0; i < t.count; ++i) {
        const int64_t tiles = (t.rows[i] + kTileRows - 1) / kTileRows * (kernel == kKeys ? G : 1);
        const int64_t blocks = ((kernel == kKeys ? 1 : G) * t.rows[i] + kBlock - 1) / kBlock * p->Hkv;
        wgs += blocks;
        work += blocks * (tiles + 1) / 2;
        longest = std::max(longest, tiles);
    }
    if (p->force_splits) return (int)std::max<int64_t>(1, std::min<int64_t>(p->force_splits, p->part_rows / (total * heads)));
    int best = 1;
    double least = 0.0;
    for (int s : {1, 2, 3, 4, 6, 8, 12, 16}) {
        if (s > 1 && (s > longest || s * total * heads > p->part_rows)) break;
        const double most = (double)((longest + s - 1) / s);
        const double tiles = std::max(most, (double)work / slots + 0.35 * most);   // the last ones end unevenly
        // a CU's workgroups slow each other down: alone, one takes 0.55 of a tile's time
        const double full = c.per_cu == 1 ? 1.0 : std::min(1.0, std::max(0.0, ((double)(wgs * s) / p->cus - 1.0) / (c.per_cu - 1)));
        const double join = s > 1 ? 4.0 + (double)(s * total * heads) * p->D * 8 / 8e6 : 0.0;
        const double us = tiles * c.tile * (0.55 + 0.45 * full) + c.start * ((wgs * s + slots - 1) / slots) + join;
        if (s == 1 || us < least) best = s, least = us;
    }
    return best;
}
hipError_t sort_keys(const a2t_prompt* p, const SeqTable<kMaxSeqs>& t, const int32_t* until, const void* k, int64_t ks, const void* v, int64_t vs) {
    const int size = p->dtype == A2T_F32 ? 4 : 2;
    const SortArgs s{until, k, v, ks * size, vs * size, p->k, p->v, p->Hkv * p->D * size, p->meta, p->lasting, p->first, p->reach};
    return launch_sort(s, t, p->stream);
}

}  // namespace

extern "C" int a2t_prompt_create(int32_t max_rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                                 double attn_scale, uint32_t flags, int32_t device, void* hip_stream, a2t_prompt** out) {
    if (!out) return A2T_ERR_INVALID;
    *out = nullptr;
    if (max_rows < 1 || n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > 128 ||
        n_q_heads > 4096 || max_rows > (1 << 26) || (int64_t)max_rows * n_q_heads > (1 << 29) || (head_dim != 64 && head_dim != 128) || (dtype != A2T_F32 && dtype != A2T_BF16) ||
        (flags & ~A2T_PROMPT_UNTIL) || !std::isfinite(attn_scale) || attn_scale < 0.0 || attn_scale > 1e6 ||
        (attn_scale != 0.0 && attn_scale < 1e-6))
        return A2T_ERR_INVALID;
    int n_dev = 0;
    if (hipGetDeviceCount(&n_dev) != hipSuccess || device < 0 || device >= n_dev) return A2T_ERR_NODEV;
    DevGuard g(device);
    a2t_prompt* p = new (std::nothrow) a2t_prompt();
    if (!p) return A2T_ERR_OOM;
    p->max_rows = max_rows;
    p->Hq = n_q_heads;
    p->Hkv = n_kv_heads;
    p->D = head_dim;
    p->dtype = dtype;
    p->device = device;
    p->scale = attn_scale == 0.0 ? 1.0 / std::sqrt((double)head_dim) : attn_scale;
    p->stream = static_cast<hipStream_t>(hip_stream);
    p->until = flags & A2T_PROMPT_UNTIL;
    int cus = 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device) == hipSuccess && cus > 0) p->cus = cus;
    p->sort_rows = env_int("A2T_PROMPT_SORT", kSortRows);
    p->force_splits = std::min(16, std::max(0, env_int("A2T_PROMPT_SPLITS", 0)));
    p->part_rows = std::min<int64_t>((int64_t)max_rows * n_q_heads * 16, kPartRows);
    const size_t rows = (size_t)max_rows, row = (size_t)n_kv_heads * head_dim * (dtype == A2T_F32 ? 4 : 2);
    bool ok = hipMalloc(&p->delta, rows * n_q_heads * sizeof(float)) == hipSuccess;
    ok = ok && hipMalloc(&p->part, (size_t)p->part_rows * (head_dim + 2) * sizeof(float)) == hipSuccess;
    if (p->until)
        ok = ok && hipMalloc(&p->k, rows * row) == hipSuccess && hipMalloc(&p->v, rows * row) == hipSuccess &&
             hipMalloc(&p->meta, rows * sizeof(int2)) == hipSuccess && hipMalloc(&p->lasting, rows * 4) == hipSuccess &&
             hipMalloc(&p->first, rows * 4) == hipSuccess && hipMalloc(&p->reach, rows * 4) == hipSuccess;
    if (!ok) {
        (void)hipGetLastError();
        free_prompt(p);
        return A2T_ERR_OOM;
    }
    *out = p;
    return A2T_OK;
}

extern "C" int a2t_prompt_destroy(a2t_prompt* p) {
    if (!p) return A2T_ERR_INVALID;
    DevGuard g(p->device);
    (void)hipStreamSynchronize(p->stream);
    free_prompt(p);
    return A2T_OK;
}

extern "C" int a2t_prompt_set_stream(a2t_prompt* p, void* hip_stream) {
    if (!p) return A2T_ERR_INVALID;
    p->stream = static_cast<hipStream_t>(hip_stream);
    return A2T_OK;
}

extern "C" int a2t_prompt_attn(a2t_prompt* p, int32_t n_seqs, const int32_t* seq_rows, const void* q, int64_t q_stride, const void* k,
                               int64_t k_stride, const void* v, int64_t v_stride, const int32_t* until, void* o, float* lse) {
    if (!p) return A2T_ERR_INVALID;
    if (p->poisoned) return A2T_ERR_HIP;
    const int64_t total = total_rows(p, n_seqs, seq_rows);
    if (!total || bad_rows(p, q, q_stride, p->Hq) || bad_rows(p, k, k_stride, p->Hkv) || bad_rows(p, v, v_stride, p->Hkv) || !o ||
        misaligned(o, 16) || misaligned(lse, 4) || misaligned(until, 4) || (until && !p->until))
        return A2T_ERR_INVALID;
    Memory m{p, total};
    for (const a2t::Rows& x : {m.rows(q, q_stride, p->Hq), m.rows(k, k_stride, p->Hkv), m.rows(v, v_stride, p->Hkv), m.floats(until, total)})
        m.in[m.ins++] = x;
    for (const a2t::Rows& x : {m.packed(o), m.floats(lse, total * p->Hq)}) m.out[m.outs++] = x;
    if (m.clash({0, -1, -1})) return A2T_ERR_INVALID;   // o over q: a block reads its queries before its first tile
    DevGuard g(p->device);
    const bool sorted = until && sort_pays(p, n_seqs, seq_rows);
    Args a = base_args(p, total, q, q_stride, k, k_stride, v, v_stride, until, sorted);
    a.o = o;
    a.lse = lse;
    const Shape shape{p->dtype == A2T_F32, p->D};
    const hipError_t e = in_tables(n_seqs, seq_rows, [&](SeqTable<kMaxSeqs>& t) {
        hipError_t s = sorted ? sort_keys(p, t, until, k, k_stride, v, v_stride) : hipSuccess;
        if (s != hipSuccess) return s;
        const int blocks = place_blocks(t, [&](int i) { return (int64_t)a.G * t.rows[i]; });
        a.splits = splits_for(p, t, kForward, total);
        return launch_forward(shape, a, t, blocks, p->stream);
    });
    if (e != hipSuccess) {
        p->poisoned = true;
        return A2T_ERR_HIP;
    }
    return A2T_OK;
}

extern "C" int a2t_prompt_attn_grad(a2t_prompt* p, int32_t n_seqs, const int32_t* seq_rows, const void* q, int64_t q_stride,
                                    const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* until,
                                    const void* o, const float* lse, const void* d_o, void* dq, void* dk, void* dv) {
    if (!p) return A2T_ERR_INVALID;
    if (p->poisoned) return A2T_ERR_HIP;
    const int64_t total = total_rows(p, n_seqs, seq_rows);
    if (!total || bad_rows(p, q, q_stride, p->Hq) || bad_rows(p, k, k_stride, p->Hkv) || bad_rows(p, v, v_stride, p->Hkv) || !o || !lse ||
        !d_o || !dq || !dk || !dv || misaligned(o, 16) || misaligned(lse, 4) || misaligned(d_o, 16) || misaligned(dq, 16) ||
        misaligned(dk, 16) || misaligned(dv, 16) || misaligned(until, 4) || (until && !p->until))
        return A2T_ERR_INVALID;
    Memory m{p, total};
    for (const a2t::Rows& x : {m.rows(q, q_stride, p->Hq), m.rows(k, k_stride, p->Hkv), m.rows(v, v_stride, p->Hkv), m.floats(until, total),
                               m.packed(o), m.floats(lse, total * p->Hq), m.packed(d_o)})
        m.in[m.ins++] = x;
    for (const a2t::Rows& x : {m.rows(dq, q_stride, p->Hq), m.rows(dk, k_stride, p->Hkv), m.rows(dv, v_stride, p->Hkv)}) m.out[m.outs++] = x;
    // dq over o: O is read by the rows' own blocks before their first tile; dk over k, dv over v: K and V are
    // read by all blocks of the launch for dQ, then by the keys' own alone
    if (m.clash({4, 1, 2})) return A2T_ERR_INVALID;
    DevGuard g(p->device);
    const bool sorted = until && sort_pays(p, n_seqs, seq_rows);
    Args a = base_args(p, total, q, q_stride, k, k_stride, v, v_stride, until, sorted);
    a.o_in = o;
    a.d_o = d_o;
    a.lse = const_cast<float*>(lse);
    a.dq = dq;
    a.dk = dk;
    a.dv = dv;
    const Shape shape{p->dtype == A2T_F32, p->D};
    const hipError_t e = in_tables(n_seqs, seq_rows, [&](SeqTable<kMaxSeqs>& t) {
        hipError_t s = sorted ? sort_keys(p, t, until, k, k_stride, v, v_stride) : hipSuccess;
        if (s != hipSuccess) return s;
        int blocks = place_blocks(t, [&](int i) { return (int64_t)a.G * t.rows[i]; });
        a.splits = splits_for(p, t, kQueries, total);
        s = launch_dq(shape, a, t, blocks, p->stream);
        if (s != hipSuccess) return s;
        blocks = place_blocks(t, [&](int i) { return (int64_t)t.rows[i]; });
        a.splits = splits_for(p, t, kKeys, total);
        return launch_dkv(shape, a, t, blocks, p->stream);
    });
    if (e != hipSuccess) {
        p->poisoned = true;
        return A2T_ERR_HIP;
    }
    return A2T_OK;
}
