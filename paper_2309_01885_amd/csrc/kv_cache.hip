// Writing keys and values into the 4-bit cache, and reading them back (qe.h).
//
// A group of channels x gets an asymmetric min/max grid as the weights' rows do
// (grid_minmax_kernel), in fp32:
//   lo = min(0, min x), hi = max(0, max x),
//   s = max((hi - lo) * fp32(1 / 15), 2^-126), to 20 bits of mantissa (the zero point takes the
//   other four), z = rint(-lo (1 / s)),  n = clamp(rint(x (1 / s)) + z, 0, 15).
// Every step is one correctly rounded fp32 operation, so the codes depend on the group's
// values alone.  Each value is moved once: 8 x 4096 tokens of 32 heads of 128 in fp16 are written in
// 165 us and read back in 155 (680 MB each, 4.1 to 4.4 TB/s, a plain copy reaches 4.9); 131072 tokens of 8 heads
// of 128 in bf16 are read in 170 us (4.1 TB/s).  Reading is bound by memory (vector units 53 % busy); writing as much
// by the vector units, which a cold call of that size (178 us and more) keeps busy throughout.
// A few tokens cost their launch and three dependent loads: 3 to 5 us.
#include "kv.h"

namespace qe {

namespace {

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
    __device__ bool open(const KvCache& c, const int64_t* slots, int64_t tokens, int* status)
    {
        const int64_t wg = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, chunk = wg / c.heads;
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

template <class T, int DP, int GROUP>
__global__ __launch_bounds__(256) void kv_write_kernel(const T* __restrict__ K, const T* __restrict__ V,
                                                       KvStrides st, bool vec_k, bool vec_v,
                                                       const int64_t* __restrict__ slots, int64_t tokens,
                                                       KvCache c, int* status)
{
    using R = KvRec<DP, GROUP>;
    constexpr int OP = kOctets<DP>, TPP = 256 / OP, P = OP / 8;      // tokens of a pass, passes
    constexpr int LANES = GROUP / 8 < OP ? GROUP / 8 : OP;
    __shared__ __align__(16) uint16_t tile[(DP / 4) * kRowHalves];
    Chunk ch;
    if (!ch.open(c, slots, tokens, status)) return;
    const int tid = threadIdx.x, o = tid % OP;
    float k[P][8], v[P][8];
    int64_t slot[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int t = p * TPP + tid / OP;
        slot[p] = ch.slot_of(t);
#pragma unroll
        for (int e = 0; e < 8; ++e) k[p][e] = v[p][e] = 0.f;
        if (8 * o < c.dim && slot[p] >= 0) {
            kv_load8(K + (ch.t0 + t) * st.kt + ch.head * st.kh + 8 * o, vec_k, k[p]);
            kv_load8(V + (ch.t0 + t) * st.vt + ch.head * st.vh + 8 * o, vec_v, v[p]);
        }
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int t = p * TPP + tid / OP;
        uint32_t kw, vw;
        const uint32_t k8 = quantize8<LANES>(k[p], kw), v8 = quantize8<LANES>(v[p], vw);
        if (slot[p] < 0 || 8 * o >= DP) continue;
        uint8_t* rec = kv_record<R::kBytes>(c, slot[p], ch.head);
        const int at = (int)(slot[p] & 31);
        if (o % LANES == 0) {
            reinterpret_cast<uint32_t*>(rec + R::kKeyWords)[o / LANES * kKvTok + at] = kw;
            reinterpret_cast<uint32_t*>(rec + R::kValWords)[o / LANES * kKvTok + at] = vw;
        }
        reinterpret_cast<uint32_t*>(rec + at * R::kKeyRow)[(o & 3) * R::NC + (o >> 2)] = k8;
        tile[(2 * o) * kRowHalves + t] = (uint16_t)v8;
        tile[(2 * o + 1) * kRowHalves + t] = (uint16_t)(v8 >> 16);
    }
    __syncthreads();
    if (ch.whole) {
        uint8_t* rec = kv_record<R::kBytes>(c, ch.slot_of(0), ch.head) + R::kVal;
        for (int x = tid; x < DP; x += 256)
            reinterpret_cast<u32x4*>(rec)[x] = *reinterpret_cast<const u32x4*>(tile + (x >> 2) * kRowHalves + (x & 3) * 8);
    } else if (ch.slot >= 0) {
        uint16_t* rec = reinterpret_cast<uint16_t*>(kv_record<R::kBytes>(c, ch.slot, ch.head) + R::kVal);
        for (int u = tid >> 5; u < DP / 4; u += 8) rec[u * kKvTok + (ch.slot & 31)] = tile[u * kRowHalves + (tid & 31)];
    }
}

// The eight values of a word.
template <class T> __device__ inline void put8(T* to, bool vec, uint32_t n8, uint32_t word)
{
    const float s = kv_scale(word), z = kv_zero(word);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = s * ((float)((n8 >> (4 * e)) & 15u) - z);
    kv_store8(to, vec, x);
}

template <class T, int DP, int GROUP>
__global__ __launch_bounds__(256) void kv_read_kernel(KvCache c, const int64_t* __restrict__ slots,
                                                      int64_t tokens, T* __restrict__ K, T* __restrict__ V,
                                                      KvStrides st, bool vec_k, bool vec_v, int* status)
{
    using R = KvRec<DP, GROUP>;
    constexpr int OP = kOctets<DP>, TPP = 256 / OP, P = OP / 8;
    __shared__ __align__(16) uint16_t tile[(DP / 4) * kRowHalves];
    Chunk ch;
    if (!ch.open(c, slots, tokens, status)) return;
    const int tid = threadIdx.x, o = tid % OP;
    if (ch.whole) {
        const uint8_t* rec = kv_record<R::kBytes>(c, ch.slot_of(0), ch.head) + R::kVal;
        for (int x = tid; x < DP; x += 256)
            *reinterpret_cast<u32x4*>(tile + (x >> 2) * kRowHalves + (x & 3) * 8) = reinterpret_cast<const u32x4*>(rec)[x];
    } else if (ch.slot >= 0) {
        const uint16_t* rec = reinterpret_cast<const uint16_t*>(kv_record<R::kBytes>(c, ch.slot, ch.head) + R::kVal);
        for (int u = tid >> 5; u < DP / 4; u += 8) tile[u * kRowHalves + (tid & 31)] = rec[u * kKvTok + (ch.slot & 31)];
    }
    uint32_t k8[P], kw[P], vw[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int64_t slot = ch.slot_of(p * TPP + tid / OP);
        k8[p] = kw[p] = vw[p] = 0;                       // (no such slot: a scale of 0)
        if (slot >= 0 && 8 * o < c.dim) {
            const uint8_t* rec = kv_record<R::kBytes>(c, slot, ch.head);
            const int at = (int)(slot & 31), g = 8 * o / GROUP;
            k8[p] = reinterpret_cast<const uint32_t*>(rec + at * R::kKeyRow)[(o & 3) * R::NC + (o >> 2)];
            kw[p] = reinterpret_cast<const uint32_t*>(rec + R::kKeyWords)[g * kKvTok + at];
            vw[p] = reinterpret_cast<const uint32_t*>(rec + R::kValWords)[g * kKvTok + at];
        }
    }
    const bool mine = 8 * o < c.dim;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int64_t token = ch.t0 + p * TPP + tid / OP;
        if (mine && token < tokens) put8(K + token * st.kt + ch.head * st.kh + 8 * o, vec_k, k8[p], kw[p]);
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int t = p * TPP + tid / OP;
        if (!mine || ch.t0 + t >= tokens) continue;
        // (a token without a slot has left no codes)
        const uint32_t v8 = vw[p] ? tile[(2 * o) * kRowHalves + t] | (uint32_t)tile[(2 * o + 1) * kRowHalves + t] << 16 : 0u;
        put8(V + (ch.t0 + t) * st.vt + ch.head * st.vh + 8 * o, vec_v, v8, vw[p]);
    }
}

// 16-byte accesses: base and strides (in elements) keep every octet aligned.
bool vec_ok(const void* p, int64_t a, int64_t b, size_t size)
{
    return ((uintptr_t)p | (uint64_t)a * size | (uint64_t)b * size) % 16 == 0;
}

template <class T>
qe_status write_typed(const void* K, const void* V, const KvStrides& st, const int64_t* slots, int64_t tokens,
                      const KvCache& c, int group, int* status, hipStream_t s)
{
    const dim3 grid = grid_xy(cdiv(tokens, kKvTok) * c.heads, 256);
    const bool vk = vec_ok(K, st.kt, st.kh, sizeof(T)), vv = vec_ok(V, st.vt, st.vh, sizeof(T));
    kv_dispatch(c.dim, group, [&](auto shape) {
        hipLaunchKernelGGL((kv_write_kernel<T, shape.DP, shape.GROUP>), grid, dim3(256), 0, s, (const T*)K, (const T*)V, st,
                           vk, vv, slots, tokens, c, status);
    });
    return hipGetLastError() == hipSuccess ? QE_OK : QE_ERR_HIP;
}

template <class T>
qe_status read_typed(const KvCache& c, int group, const int64_t* slots, int64_t tokens, void* K, void* V,
                     const KvStrides& st, int* status, hipStream_t s)
{
    const dim3 grid = grid_xy(cdiv(tokens, kKvTok) * c.heads, 256);
    const bool vk = vec_ok(K, st.kt, st.kh, sizeof(T)), vv = vec_ok(V, st.vt, st.vh, sizeof(T));
    kv_dispatch(c.dim, group, [&](auto shape) {
        hipLaunchKernelGGL((kv_read_kernel<T, shape.DP, shape.GROUP>), grid, dim3(256), 0, s, c, slots, tokens, (T*)K, (T*)V,
                           st, vk, vv, status);
    });
    return hipGetLastError() == hipSuccess ? QE_OK : QE_ERR_HIP;
}

}  // namespace

qe_status launch_kv_write(const void* K, const void* V, int dtype, const int64_t* strides, const int64_t* slots,
                          int64_t tokens, const KvCache& c, int group, int* status, hipStream_t s)
{
    const KvStrides st{strides[0], strides[1], strides[2], strides[3]};
    if (dtype == QE_F32) return write_typed<float>(K, V, st, slots, tokens, c, group, status, s);
    if (dtype == QE_F16) return write_typed<_Float16>(K, V, st, slots, tokens, c, group, status, s);
    return write_typed<__bf16>(K, V, st, slots, tokens, c, group, status, s);
}

qe_status launch_kv_read(const KvCache& c, int group, const int64_t* slots, int64_t tokens, void* K, void* V,
                         int dtype, const int64_t* strides, int* status, hipStream_t s)
{
    const KvStrides st{strides[0], strides[1], strides[2], strides[3]};
    if (dtype == QE_F32) return read_typed<float>(c, group, slots, tokens, K, V, st, status, s);
    if (dtype == QE_F16) return read_typed<_Float16>(c, group, slots, tokens, K, V, st, status, s);
    return read_typed<__bf16>(c, group, slots, tokens, K, V, st, status, s);
}

}  // namespace qe
