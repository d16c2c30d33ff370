// Attention over the 4-bit key/value cache (qe.h).
#include "kv.h"

namespace qe {

namespace {

// Sum or maximum over the 256 threads of a workgroup.
template <bool MAX> __device__ inline float wg_reduce(float x, float* part)
{
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const float y = __shfl_xor(x, m);
        x = MAX ? fmaxf(x, y) : x + y;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    return MAX ? fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])) : part[0] + part[1] + part[2] + part[3];
}

__device__ inline float load_elem(const void* p, int dtype, int64_t i)
{
    return dtype == QE_F32 ? static_cast<const float*>(p)[i]
         : dtype == QE_F16 ? (float)static_cast<const _Float16*>(p)[i] : (float)static_cast<const __bf16*>(p)[i];
}
__device__ inline void store_elem(void* p, int dtype, int64_t i, float x)
{
    if (dtype == QE_F32) static_cast<float*>(p)[i] = x;
    else if (dtype == QE_F16) static_cast<_Float16*>(p)[i] = (_Float16)x;
    else static_cast<__bf16*>(p)[i] = (__bf16)x;
}

// One workgroup per (sequence, query, head): a thread scores one of 256 tokens, then
// takes one channel of the weighted sum.
template <int DP, int GROUP> __global__ __launch_bounds__(256) void kv_attn_kernel(KvAttn a)
{
    using R = KvRec<DP, GROUP>;
    __shared__ float qs[DP], ps[256], part[4];
    const int64_t wg = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int head = (int)(wg % a.heads);
    const int64_t r = wg / a.heads, b = r / a.max_q, i = r - b * a.max_q;
    if (b >= a.batch) return;
    const int tid = threadIdx.x;
    int64_t first = b * a.max_q, nq = a.max_q;
    if (a.q_start) {
        first = a.q_start[b];
        nq = (int64_t)a.q_start[b + 1] - first;
        if (first < 0 || nq < 0 || nq > a.max_q || first + nq > a.total) {
            if (tid == 0) set_status(a.status, QE_ERR_ARG);
            first = first < 0 ? 0 : first;
            nq = min(min(nq, a.max_q), a.total - first);
        }
    }
    if (i >= nq) return;
    const int page = (int)a.c.per * kKvTok;
    int64_t len = a.lengths[b];
    if (len < 0 || len > a.width * page) {
        if (tid == 0) set_status(a.status, QE_ERR_ARG);
        len = len < 0 ? 0 : a.width * page;
    }
    const int64_t pos = len - nq + i;
    const int64_t end = a.causal ? min(len, pos + 1) : len;
    const int64_t begin = a.window ? max((int64_t)0, pos - a.window + 1) : 0;
    const int kvh = head / (a.heads / a.c.heads);
    if (tid < DP) qs[tid] = tid < a.c.dim ? load_elem(a.q, a.dtype, (first + i) * a.qt + head * a.qh + tid) * a.scale : 0.f;
    const float slope = a.slopes ? a.slopes[head] : 0.f;
    float top = -__builtin_inff(), mass = 0.f, acc = 0.f;
    __syncthreads();
    for (int64_t t0 = begin & ~(int64_t)31; t0 < end; t0 += 256) {
        const int64_t t = t0 + tid;
        float s = -__builtin_inff();
        if (t >= begin && t < end) {
            const int64_t id = a.table[b * a.width + t / page];
            if (id < 0 || id >= a.c.slots / page) set_status(a.status, QE_ERR_ARG);
            else {
                const uint8_t* rec = kv_record<R::kBytes>(a.c, id * page + t % page, kvh);
                const uint32_t* row = reinterpret_cast<const uint32_t*>(rec + (t & 31) * R::kKeyRow);
                const uint32_t* words = reinterpret_cast<const uint32_t*>(rec + R::kKeyWords) + (t & 31);
                s = 0.f;
                for (int o = 0; o < DP / 8; ++o) {
                    const uint32_t n8 = row[(o & 3) * R::NC + (o >> 2)], w = words[8 * o / GROUP * kKvTok];
                    for (int e = 0; e < 8; ++e)
                        s += kv_scale(w) * ((float)((n8 >> (4 * e)) & 15u) - kv_zero(w)) * qs[8 * o + e];
                }
                s += slope * (float)(t - pos);
            }
        }
        const float m = fmaxf(top, wg_reduce<true>(s, part));
        const float p = s == -__builtin_inff() ? 0.f : expf(s - m);
        const float f = top == -__builtin_inff() ? 0.f : expf(top - m);
        ps[tid] = p;
        mass = mass * f + wg_reduce<false>(p, part);
        acc *= f;
        top = m;
        if (tid < DP)
            for (int64_t u = t0; u < min(end, t0 + 256); u += 1) {
                const float pu = ps[u - t0];
                const int64_t id = a.table[b * a.width + u / page];
                if (u < begin || id < 0 || id >= a.c.slots / page) continue;
                const uint8_t* rec = kv_record<R::kBytes>(a.c, id * page + u % page, kvh);
                const uint32_t n = reinterpret_cast<const uint16_t*>(rec + R::kVal)[tid / 4 * kKvTok + (u & 31)] >> (4 * (tid & 3)) & 15u;
                const uint32_t w = reinterpret_cast<const uint32_t*>(rec + R::kValWords)[tid / GROUP * kKvTok + (u & 31)];
                acc += pu * (kv_scale(w) * ((float)n - kv_zero(w)));
            }
        __syncthreads();
    }
    if (tid < a.c.dim) store_elem(a.out, a.dtype, (first + i) * a.ot + head * a.oh + tid, mass == 0.f ? 0.f : acc / mass);
    if (a.lse && tid == 0) a.lse[(first + i) * a.heads + head] = mass == 0.f ? -__builtin_inff() : top + logf(mass);
}

}  // namespace

size_t kv_attn_ws_bytes(int64_t batch, int64_t max_q, int heads, int kv_heads, int dim) { return kStatusBytes; }

qe_status launch_kv_attn(const KvAttn& a, void* ws, hipStream_t s)
{
    const dim3 grid = grid_xy((int64_t)a.batch * a.max_q * a.heads, 256);
    kv_dispatch(a.c.dim, a.group, [&](auto shape) {
        hipLaunchKernelGGL((kv_attn_kernel<shape.DP, shape.GROUP>), grid, dim3(256), 0, s, a);
    });
    return hipGetLastError() == hipSuccess ? QE_OK : QE_ERR_HIP;
}

}  // namespace qe
