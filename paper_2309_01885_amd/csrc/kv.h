// Layout of the 4-bit key/value cache (qe.h) and the loads and stores that its
// kernels share.
#pragma once

#include "qe_internal.h"

namespace qe {

constexpr int kKvTok = 32;            // tokens of a record
constexpr float kKvMinScale = 1.17549435e-38f;   // 2^-126
constexpr float kKvFifteenth = 1.f / 15.f;       // (rounded)

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// dim rounded up to a width that the kernels are built for; 0: not supported
__host__ __device__ constexpr int kv_dp(int dim)
{
    return dim <= 64 ? 64 : dim <= 96 ? 96 : dim <= 128 ? 128 : dim <= 192 ? 192 : dim <= 256 ? 256 : 0;
}
__host__ __device__ constexpr int kv_ng(int dp, int group) { return (dp + group - 1) / group; }

// Byte offsets inside a record of 32 tokens.
template <int DP, int GROUP> struct KvRec {
    static constexpr int NC = DP / 32;                   // words a lane takes of a key row
    static constexpr int NG = kv_ng(DP, GROUP);
    static constexpr int kKeyRow = DP / 2;
    static constexpr int kKeyWords = kKvTok * kKeyRow;
    static constexpr int kVal = kKeyWords + kKvTok * 4 * NG;
    static constexpr int kValWords = kVal + kKvTok * DP / 2;
    static constexpr int kBytes = kValWords + kKvTok * 4 * NG;
};

inline int64_t kv_record_bytes(int dp, int group) { return kKvTok * (int64_t)(dp + 8 * kv_ng(dp, group)); }

struct KvCache {
    uint8_t* pages;
    int64_t pages_count, slots;          // slots: pages_count * page
    uint32_t per;         // records of a page
    int heads, dim;
};

// Record of a slot (slot < cache.slots; fewer than 2^32 records, checked on the host).
template <int BYTES> __device__ inline uint8_t* kv_record(const KvCache& c, int64_t slot, int head)
{
    const uint32_t at = (uint32_t)(slot >> 5), page = at / c.per;
    return c.pages + (((int64_t)page * c.heads + head) * c.per + (at - page * c.per)) * BYTES;
}

// A group's scale and zero point in one word.
__device__ inline float kv_scale(uint32_t w) { return __uint_as_float(w & ~15u); }
__device__ inline float kv_zero(uint32_t w) { return (float)(w & 15u); }

// Eight consecutive channels; vec: the address is a multiple of 16 bytes.
template <class T> __device__ inline void kv_load8(const T* p, bool vec, float* x)
{
    T v[8];
    if (vec) {
        u32x4 raw[sizeof(T) / 2];
#pragma unroll
        for (int u = 0; u < (int)sizeof(T) / 2; ++u) raw[u] = reinterpret_cast<const u32x4*>(p)[u];
        __builtin_memcpy(v, raw, sizeof(v));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = p[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
}
template <class T> __device__ inline void kv_store8(T* p, bool vec, const float* x)
{
    T v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (T)x[e];
    if (vec) {
        u32x4 raw[sizeof(T) / 2];
        __builtin_memcpy(raw, v, sizeof(v));
#pragma unroll
        for (int u = 0; u < (int)sizeof(T) / 2; ++u) reinterpret_cast<u32x4*>(p)[u] = raw[u];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = v[e];
    }
}

// One attention call (qe.h); host-checked except where a comment says otherwise.
struct KvAttn {
    KvCache c;                     // c.dim: the heads' size
    const void* q;
    void* out;
    float* lse;                    // or null
    int64_t qt, qh, ot, oh;        // strides of a token and a head, in elements
    const int32_t* q_start;        // or null: max_q queries each.  Values are clamped on the device
    int64_t total, max_q, width;
    int32_t batch, heads;
    const int32_t* table;          // page numbers, checked on the device
    const int32_t* lengths;        // clamped on the device
    float scale;
    int32_t causal, window, sinks;
    const float* slopes;           // or null
    int32_t dtype, group;
    bool vec_q, vec_o;             // 16-byte accesses of q and out
    int* status;
};

// What one workgroup of kv_attn_shared's kernels does (KvUnit's fields of the same names).
struct KvItem { int32_t first, b, kvh, tile_row, rows, len, pos0, rec0, rec1, slot, ref, pad; };

// What the plan of kv_attn_shared knows of a group and of a sequence.
struct KvGroup {
    int32_t reader, first, tokens;         // the sequence whose pages are read; first row of Q, rows
    int32_t records;                       // shared records, 0: none
    int32_t tiles, splits, item;           // tiles and splits of the shared part, its first entry of list 0
    int32_t pad;
};
struct KvSequence {
    int32_t first, nq, len;                // nq < 0: rows outside of the call
    int32_t group;                         // -1: none that shares anything
    int32_t tiles, splits, item;           // of its own part, in list 1
    int32_t pad;
};
// A call of kv_attn_shared, beside its KvAttn.
struct KvShared {
    const int32_t *groups, *shared;        // groups[g] .. groups[g + 1] - 1 share shared[g] pages; checked on the device
    int32_t ngroups;
    int32_t rows[2], rows_log2[2];         // of the two lists: rows of a tile,
    int32_t fill[2], least[2];             // entries that fill the chip, records of an entry at least
    int32_t room[2];                       // entries that a list holds
    bool joint, pair;                      // both lists in one launch (equal fill); with tiles of 32 rows and of 16
    KvGroup* group;
    KvSequence* seq;
    KvItem* items[2];
    int32_t* count;
};

// What kv_extend knows of a sequence when the tokens' slots are looked up.
struct KvExtendSeq {
    int32_t old, held, start;      // tokens and pages before the call; first token of the call
    int32_t first;                 // its first wanted page's place among all that are taken; -1: none given, -2: bad arguments
};
struct KvExtend {
    const int32_t* counts;
    int32_t* table;
    int32_t* lengths;
    const int32_t* keep;           // or null
    int32_t* free;
    int32_t* free_count;
    int64_t* slots;
    int32_t* positions;
    int32_t* q_start;
    int32_t* lacking;              // or null
    int64_t batch, width, num_pages, total, page;
    int* status;
    KvExtendSeq* seqs;             // in the workspace
    int64_t* top;
};

size_t kv_extend_ws_bytes(int64_t batch);
qe_status launch_kv_extend(const KvExtend& a, void* ws, hipStream_t s);

struct KvRotation {
    const int32_t* positions;      // or null: no rotation, every query row is taken
    const float *cos, *sin;        // rows x half; null: no rotation
    int64_t rows;
    int half;                      // pairs of channels
    bool interleaved, vec;         // vec: pairs of halves, whole octets in each half
};
struct KvNorm {
    const float *q, *k;            // weights; null: no norm
    double eps, inv_dim;
    bool vec;                      // 16-byte loads of the weights
};
qe_status launch_kv_append(const void* Q, const void* K, const void* V, void* out, int dtype, const int64_t* strides, int64_t tokens,
                           int heads, const KvRotation& r, const KvNorm& n, const int64_t* slots, const KvCache& c, int group,
                           int* status, hipStream_t s);

inline void kv_attn_vec(KvAttn& a)
{
    const size_t size = a.dtype == QE_F32 ? 4 : 2;
    a.vec_q = ((uintptr_t)a.q | (uint64_t)a.qt * size | (uint64_t)a.qh * size) % 16 == 0;
    a.vec_o = ((uintptr_t)a.out | (uint64_t)a.ot * size | (uint64_t)a.oh * size) % 16 == 0;
}

size_t kv_attn_ws_bytes(int64_t batch, int64_t max_q, int heads, int kv_heads, int dim);
qe_status launch_kv_attn(const KvAttn& a, void* ws, hipStream_t s);
bool kv_attn_many(const KvAttn& a);               // whether the call takes the many-row form
size_t kv_attn_shared_ws_bytes(int64_t total, int64_t batch, int64_t max_q, int heads, int kv_heads, int dim, int64_t ngroups, bool always);
qe_status launch_kv_attn_shared(const KvAttn& a, const int32_t* groups, const int32_t* shared, int64_t ngroups, void* ws, size_t ws_bytes,
                                bool always, hipStream_t s);   // always: also where kv_attn is faster
qe_status launch_kv_write(const void* K, const void* V, int dtype, const int64_t* strides, const int64_t* slots,
                          int64_t tokens, const KvCache& c, int group, int* status, hipStream_t s);
qe_status launch_kv_read(const KvCache& c, int group, const int64_t* slots, int64_t tokens, void* K, void* V,
                         int dtype, const int64_t* strides, int* status, hipStream_t s);

// Calls f with a width and a group as types (kv_dp and the group were checked).
template <int D, int G> struct KvShape { static constexpr int DP = D, GROUP = G; };
template <int D, class F> void kv_dispatch_group(int group, F f)
{
    if (group == 32) f(KvShape<D, 32>());
    else if (group == 64 || D <= 64) f(KvShape<D, 64>());   // (a group of 128 ends with the 64 channels)
    else f(KvShape<D, D <= 64 ? 64 : 128>());
}
template <class F> void kv_dispatch(int dim, int group, F f)
{
    switch (kv_dp(dim)) {
        case 64: kv_dispatch_group<64>(group, f); break;
        case 96: kv_dispatch_group<96>(group, f); break;
        case 128: kv_dispatch_group<128>(group, f); break;
        case 192: kv_dispatch_group<192>(group, f); break;
        default: kv_dispatch_group<256>(group, f);
    }
}

}  // namespace qe
