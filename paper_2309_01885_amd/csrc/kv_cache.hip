// Writing keys and values into the 4-bit cache, and reading them back (qe.h).
//
// A group of channels x gets an asymmetric min/max grid as the weights' rows do
// (grid_minmax_kernel), in fp32:
//   lo = min(0, min x), hi = max(0, max x),
//   s = max((hi - lo) / 15, 2^-126), to 20 bits of mantissa (the zero point takes the
//   other four), z = rint(-lo (1 / s)),  n = clamp(rint(x (1 / s)) + z, 0, 15).
// Every step is one correctly rounded fp32 operation, so the codes depend on the group's
// values alone.  Both kernels are bound by memory: each value is moved once.
#include "kv.h"

namespace qe {

namespace {

// One workgroup per 32 entries of `slots`, head, and K or V; a thread takes 8 channels of
// a token, OP threads a token: a power of two, so that a group's threads are an aligned
// stretch of a wave and its minimum and maximum a few shuffles.
template <int DP> constexpr int kOctets = DP <= 64 ? 8 : DP <= 128 ? 16 : 32;
// Half-words of a value unit's row in LDS: 32 and padding, so that a wave's threads, which
// hold different units of few tokens, spread over the banks.
constexpr int kRowHalves = 40;

struct KvStrides { int64_t kt, kh, vt, vh; };

// The slot of the chunk's token t; -1 where there is none or it lies outside of the cache.
__device__ inline int64_t slot_of(const int64_t* slots, int64_t token, int64_t tokens, int64_t limit, int* status)
{
    if (token >= tokens) return -1;
    const int64_t s = slots[token];
    if (s >= limit) {
        if (status) set_status(status, QE_ERR_ARG);
        return -1;
    }
    return s < 0 ? -1 : s;
}

template <class T, int DP, int GROUP>
__global__ __launch_bounds__(256) void kv_write_kernel(const T* __restrict__ K, const T* __restrict__ V,
                                                       KvStrides st, bool vec_k, bool vec_v,
                                                       const int64_t* __restrict__ slots, int64_t tokens,
                                                       KvCache c, int* status)
{
    using R = KvRec<DP, GROUP>;
    constexpr int OP = kOctets<DP>, TPP = 256 / OP;      // tokens of a pass
    constexpr int LANES = GROUP / 8 < OP ? GROUP / 8 : OP;
    __shared__ __align__(16) uint16_t tile[(DP / 4) * kRowHalves];
    __shared__ int64_t slot[kKvTok];
    const int64_t wg = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t chunk = wg / (2 * c.heads);
    const int64_t t0 = chunk * kKvTok;
    if (t0 >= tokens) return;
    const int hk = (int)(wg - chunk * (2 * c.heads)), head = hk % c.heads;
    const bool value = hk >= c.heads;
    const int tid = threadIdx.x;
    if (tid < kKvTok) slot[tid] = slot_of(slots, t0 + tid, tokens, c.slots, status);
    __syncthreads();
    // the 32 slots are one record in order
    const bool whole = __syncthreads_and((slot[0] & 31) == 0 && slot[0] >= 0 && slot[tid & 31] == slot[0] + (tid & 31));

    const T* src = value ? V + head * st.vh : K + head * st.kh;
    const int64_t stride = value ? st.vt : st.kt;
    const bool vec = value ? vec_v : vec_k;
    const int o = tid % OP;
    float x[OP / 8][8];
#pragma unroll
    for (int p = 0; p < OP / 8; ++p) {
        const int t = p * TPP + tid / OP;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[p][e] = 0.f;
        if (8 * o < c.dim && slot[t] >= 0) kv_load8(src + (t0 + t) * stride + 8 * o, vec, x[p]);
    }
#pragma unroll
    for (int p = 0; p < OP / 8; ++p) {
        const int t = p * TPP + tid / OP;
        float lo = 0.f, hi = 0.f;
        bool bad = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            lo = fminf(lo, x[p][e]);
            hi = fmaxf(hi, x[p][e]);
            bad = bad || !(fabsf(x[p][e]) <= 3.402823466e38f);
        }
        if (bad) hi = __builtin_inff();
#pragma unroll
        for (int m = 1; m < LANES; m *= 2) {
            lo = fminf(lo, __shfl_xor(lo, m));
            hi = fmaxf(hi, __shfl_xor(hi, m));
        }
        const float range = hi - lo;
        uint32_t n8 = 0, word = 0x7fc00000u;             // a NaN scale: the group reads back as NaN
        if (range <= 3.402823466e38f) {
            word = (__float_as_uint(fmaxf(range / 15.f, kKvMinScale)) + 8u) & ~15u;
            const float inv = 1.f / __uint_as_float(word);
            const float z = fminf(fmaxf(rintf(-lo * inv), 0.f), 15.f);
            word |= (uint32_t)z;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                n8 |= (uint32_t)fminf(fmaxf(rintf(x[p][e] * inv) + z, 0.f), 15.f) << (4 * e);
        }
        if (slot[t] < 0 || 8 * o >= DP) continue;
        uint8_t* rec = kv_record<R::kBytes>(c, slot[t], head);
        const int at = (int)(slot[t] & 31);
        if (o % LANES == 0)
            reinterpret_cast<uint32_t*>(rec + (value ? R::kValWords : R::kKeyWords))[o / LANES * kKvTok + at] = word;
        if (!value)
            reinterpret_cast<uint32_t*>(rec + at * R::kKeyRow)[(o & 3) * R::NC + (o >> 2)] = n8;
        else {
            tile[(2 * o) * kRowHalves + t] = (uint16_t)n8;
            tile[(2 * o + 1) * kRowHalves + t] = (uint16_t)(n8 >> 16);
        }
    }
    if (!value) return;
    __syncthreads();
    if (whole) {
        uint8_t* rec = kv_record<R::kBytes>(c, slot[0], head) + R::kVal;
        for (int v = tid; v < DP; v += 256)
            reinterpret_cast<u32x4*>(rec)[v] = *reinterpret_cast<const u32x4*>(tile + (v >> 2) * kRowHalves + (v & 3) * 8);
        return;
    }
    const int t = tid & 31;
    if (slot[t] < 0) return;
    uint16_t* rec = reinterpret_cast<uint16_t*>(kv_record<R::kBytes>(c, slot[t], head) + R::kVal);
    for (int u = tid >> 5; u < DP / 4; u += 8) rec[u * kKvTok + (slot[t] & 31)] = tile[u * kRowHalves + t];
}

template <class T, int DP, int GROUP>
__global__ __launch_bounds__(256) void kv_read_kernel(KvCache c, const int64_t* __restrict__ slots,
                                                      int64_t tokens, T* __restrict__ K, T* __restrict__ V,
                                                      KvStrides st, bool vec_k, bool vec_v, int* status)
{
    using R = KvRec<DP, GROUP>;
    constexpr int OP = kOctets<DP>, TPP = 256 / OP;
    __shared__ __align__(16) uint16_t tile[(DP / 4) * kRowHalves];
    __shared__ int64_t slot[kKvTok];
    const int64_t wg = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t chunk = wg / (2 * c.heads);
    const int64_t t0 = chunk * kKvTok;
    if (t0 >= tokens) return;
    const int hk = (int)(wg - chunk * (2 * c.heads)), head = hk % c.heads;
    const bool value = hk >= c.heads;
    const int tid = threadIdx.x;
    if (tid < kKvTok) slot[tid] = slot_of(slots, t0 + tid, tokens, c.slots, status);
    __syncthreads();
    if (value) {
        const bool whole = __syncthreads_and((slot[0] & 31) == 0 && slot[0] >= 0 && slot[tid & 31] == slot[0] + (tid & 31));
        if (whole) {
            const uint8_t* rec = kv_record<R::kBytes>(c, slot[0], head) + R::kVal;
            for (int v = tid; v < DP; v += 256)
                *reinterpret_cast<u32x4*>(tile + (v >> 2) * kRowHalves + (v & 3) * 8) = reinterpret_cast<const u32x4*>(rec)[v];
        } else if (slot[tid & 31] >= 0) {
            const int t = tid & 31;
            const uint16_t* rec = reinterpret_cast<const uint16_t*>(kv_record<R::kBytes>(c, slot[t], head) + R::kVal);
            for (int u = tid >> 5; u < DP / 4; u += 8) tile[u * kRowHalves + t] = rec[u * kKvTok + (slot[t] & 31)];
        }
        __syncthreads();
    }
    T* dst = value ? V + head * st.vh : K + head * st.kh;
    const int64_t stride = value ? st.vt : st.kt;
    const bool vec = value ? vec_v : vec_k;
    const int o = tid % OP;
    if (8 * o >= c.dim) return;
#pragma unroll
    for (int p = 0; p < OP / 8; ++p) {
        const int t = p * TPP + tid / OP;
        if (t0 + t >= tokens) continue;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;
        if (slot[t] >= 0) {
            const uint8_t* rec = kv_record<R::kBytes>(c, slot[t], head);
            const int at = (int)(slot[t] & 31);
            const uint32_t w = reinterpret_cast<const uint32_t*>(rec + (value ? R::kValWords : R::kKeyWords))[8 * o / GROUP * kKvTok + at];
            const uint32_t n8 = value ? tile[(2 * o) * kRowHalves + t] | (uint32_t)tile[(2 * o + 1) * kRowHalves + t] << 16
                                      : reinterpret_cast<const uint32_t*>(rec + at * R::kKeyRow)[(o & 3) * R::NC + (o >> 2)];
            const float s = kv_scale(w), z = kv_zero(w);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = s * ((float)((n8 >> (4 * e)) & 15u) - z);
        }
        kv_store8(dst + (t0 + t) * stride + 8 * o, vec, x);
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
    const dim3 grid = grid_xy(cdiv(tokens, kKvTok) * 2 * c.heads, 256);
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
    const dim3 grid = grid_xy(cdiv(tokens, kKvTok) * 2 * c.heads, 256);
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
