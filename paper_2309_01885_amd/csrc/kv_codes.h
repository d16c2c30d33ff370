// What the kernels that put tokens into the 4-bit cache (kv_cache.hip, kv_append.hip) share: the chunk of tokens of
// a workgroup and the codes of a group.
#pragma once

#include "kv.h"

namespace qe {

// One workgroup per 32 entries of `slots` and head, keys and values; a thread takes 8
// channels of a token, OP threads a token: a power of two, so that a group's threads are an
// aligned stretch of a wave and its minimum and maximum a few shuffles.  (A workgroup for the
// keys and one for the values had half the bytes in flight: 409 against 351 us, write and
// read back 8 x 4096 tokens of 32 heads of 128.)
template <int DP> constexpr int kOctets = DP <= 64 ? 8 : DP <= 128 ? 16 : 32;
// Half-words of a value unit's row in LDS: 32 and padding, so that a wave's threads, which
// hold different units of few tokens, spread over the banks.
constexpr int kRowHalves = 40;

struct KvStrides { int64_t kt, kh, vt, vh; };

// The chunk of 32 tokens that a workgroup works on.  Lane l of every wave holds the slot of token l % 32,
// -1 where there is none or it lies outside of the cache.
struct Chunk {
    int64_t t0, slot;
    int head;
    bool whole;                          // the slots are one record in order
    __device__ bool open(int64_t wg, const KvCache& c, const int64_t* slots, int64_t tokens, int* status)
    {
        const int64_t chunk = wg / c.heads;
        head = (int)(wg - chunk * c.heads);
        t0 = chunk * kKvTok;
        if (t0 >= tokens) return false;
        const int l = threadIdx.x & 31;
        slot = t0 + l < tokens ? slots[t0 + l] : -1;
        if (slot >= c.slots) {
            if (status) set_status(status, QE_ERR_ARG);
            slot = -1;
        }
        const int64_t first = __shfl(slot, 0);
        whole = __all(slot >= 0 && (first & 31) == 0 && slot == first + l);
        return true;
    }
    __device__ int64_t slot_of(int t) const { return __shfl(slot, t); }
};

// Codes of 8 channels of a group, LANES threads of a wave a group; word: its scale and zero point.
template <int LANES> __device__ inline uint32_t quantize8(const float* x, uint32_t& word)
{
    float lo = 0.f, hi = 0.f;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        lo = fminf(lo, x[e]);
        hi = fmaxf(hi, x[e]);
        bad = bad || !(fabsf(x[e]) <= 3.402823466e38f);
    }
    if (bad) hi = __builtin_inff();
#pragma unroll
    for (int m = 1; m < LANES; m *= 2) {
        lo = fminf(lo, __shfl_xor(lo, m));
        hi = fmaxf(hi, __shfl_xor(hi, m));
    }
    const float range = hi - lo;
    uint32_t n8 = 0;
    word = 0x7fc00000u;                                  // a NaN scale: the group reads back as NaN
    if (range <= 3.402823466e38f) {
        word = (__float_as_uint(fmaxf(range * kKvFifteenth, kKvMinScale)) + 8u) & ~15u;
        const float inv = 1.f / __uint_as_float(word);
        const float z = fminf(fmaxf(rintf(-lo * inv), 0.f), 15.f);
        word |= (uint32_t)z;
#pragma unroll
        for (int e = 0; e < 8; ++e) n8 |= (uint32_t)fminf(fmaxf(rintf(x[e] * inv) + z, 0.f), 15.f) << (4 * e);
    }
    return n8;
}

// 16-byte accesses: base and strides (in elements) keep every octet aligned.
inline bool vec_ok(const void* p, int64_t a, int64_t b, size_t size)
{
    return ((uintptr_t)p | (uint64_t)a * size | (uint64_t)b * size) % 16 == 0;
}

}  // namespace qe
