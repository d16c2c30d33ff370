// Norm of each head's query and key, rotation by their positions, and the write into the 4-bit cache, in one pass (qe.h).
//
// Every step is one correctly rounded fp32 operation (the compiler must not fuse them), so that the codes, which are
// integers, are a function of the row's values alone; the norm's sum of squares and its root are in 64 bits, where no order
// of the sum shows after the rounding to fp32:
//   r = fp32(1 / sqrt(sum x^2 / dim + eps)), y = fp32(fp32(x r) w),
//   a' = fp32(fp32(a c) - fp32(b s)), b' = fp32(fp32(b c) + fp32(a s)).
// A thread has 8 channels of a row, 8 to 32 lanes of a wave a row; a channel's partner in the rotation comes
// through the row's own stretch of LDS, where any number of rotated channels is right.
// The first workgroups take 32 tokens' keys and values of a head each, as the plain write does; the others 32 query
// rows in the order of memory.
#include "kv_codes.h"

namespace qe {

namespace {

struct KvAppend {
    int64_t qt, qh, kt, kh, vt, vh, ot, oh;
    int64_t tokens, kv_wgs;
    int heads;
    bool vec_q, vec_k, vec_v, vec_o;
    KvRotation r;
    KvNorm n;
    int* status;
};

// Position of a token: -1 where it has none, or one past the tables.
__device__ inline int64_t position_of(const KvAppend& a, int64_t token)
{
    if (!a.r.positions || token >= a.tokens) return token < a.tokens ? 0 : -1;
    const int64_t p = a.r.positions[token];
    if (p >= a.r.rows && a.r.cos) {
        if (a.status) set_status(a.status, QE_ERR_ARG);
        return -1;
    }
    return p;
}

// A row's 8 channels from 8 o on, normed.  OP lanes a row.
template <int OP> __device__ inline void norm8(float (&x)[8], const float* w, int o, int dim, double eps)
{
#pragma clang fp contract(off)
    double ss = 0.;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = __builtin_fma((double)x[e], (double)x[e], ss);
#pragma unroll
    for (int m = 1; m < OP; m *= 2) ss += __shfl_xor(ss, m);
    const float r = (float)(1. / __builtin_sqrt(ss / (double)dim + eps));
    if (8 * o >= dim) return;
    float g[8];
    kv_load8(w + 8 * o, false, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float y = x[e] * r;
        x[e] = y * g[e];
    }
}

// The same, rotated.  at: the row's OP * 8 floats of LDS, used by its lanes alone.
template <int OP> __device__ inline void rotate8(float (&x)[8], const KvRotation& r, int64_t pos, int o, float* at)
{
#pragma clang fp contract(off)
    const float* cos = r.cos + pos * r.half;
    const float* sin = r.sin + pos * r.half;
    if (r.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 4 * o + e;
            if (i >= r.half) continue;
            const float c = cos[i], s = sin[i], a = x[2 * e], b = x[2 * e + 1];
            const float ac = a * c, bs = b * s, bc = b * c, as = a * s;
            x[2 * e] = ac - bs;
            x[2 * e + 1] = bc + as;
        }
        return;
    }
    // (LDS serves a wave in order)
#pragma unroll
    for (int e = 0; e < 8; e += 4) *reinterpret_cast<f32x4*>(at + 8 * o + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int d = 8 * o + e;
        if (d >= 2 * r.half) continue;
        const bool low = d < r.half;
        const int i = low ? d : d - r.half;
        const float c = cos[i], s = sin[i], other = at[low ? d + r.half : i];
        const float own = x[e] * c, far = other * s;
        x[e] = low ? own - far : own + far;
    }
    __builtin_amdgcn_wave_barrier();
}

template <class T, int DP, int GROUP>
__global__ __launch_bounds__(256) void kv_append_kernel(const T* Q, const T* __restrict__ K, const T* __restrict__ V, T* out,
                                                        const int64_t* __restrict__ slots, KvCache c, KvAppend a)
{
    using R = KvRec<DP, GROUP>;
    constexpr int OP = kOctets<DP>, TPP = 256 / OP, P = OP / 8;      // rows of a pass, passes
    constexpr int LANES = GROUP / 8 < OP ? GROUP / 8 : OP;
    __shared__ __align__(16) uint16_t tile[(DP / 4) * kRowHalves];
    __shared__ __align__(16) float turn[TPP][OP * 8 + 4];
    const int64_t wg = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int tid = threadIdx.x, o = tid % OP, row = tid / OP;
    if (wg >= a.kv_wgs) {
        const int64_t rows = a.tokens * a.heads, r0 = (wg - a.kv_wgs) * kKvTok;
        float x[P][8];
        int64_t pos[P], token[P];
        int head[P];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int64_t at = r0 + p * TPP + row;
            token[p] = at / a.heads;
            head[p] = (int)(at - token[p] * a.heads);
            pos[p] = at < rows ? position_of(a, token[p]) : -1;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[p][e] = 0.f;
            if (8 * o < c.dim && pos[p] >= 0) kv_load8(Q + token[p] * a.qt + head[p] * a.qh + 8 * o, a.vec_q, x[p]);
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (a.n.q) norm8<OP>(x[p], a.n.q, o, c.dim, a.n.eps);
            if (a.r.cos) rotate8<OP>(x[p], a.r, max(pos[p], (int64_t)0), o, turn[row]);
            if (8 * o < c.dim && pos[p] >= 0) kv_store8(out + token[p] * a.ot + head[p] * a.oh + 8 * o, a.vec_o, x[p]);
        }
        return;
    }
    Chunk ch;
    if (!ch.open(wg, c, slots, a.tokens, a.status)) return;
    float k[P][8], v[P][8];
    int64_t slot[P], pos[P];
    // (a token without a position is not written: its slot is taken as none)
    if (a.r.positions) {
        const int64_t t = ch.t0 + (tid & 31);
        if (position_of(a, t) < 0) ch.slot = -1;
        ch.whole = __all(ch.slot >= 0) && ch.whole;
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int t = p * TPP + row;
        slot[p] = ch.slot_of(t);
        pos[p] = a.r.positions && slot[p] >= 0 ? a.r.positions[ch.t0 + t] : 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) k[p][e] = v[p][e] = 0.f;
        if (8 * o < c.dim && slot[p] >= 0) {
            kv_load8(K + (ch.t0 + t) * a.kt + ch.head * a.kh + 8 * o, a.vec_k, k[p]);
            kv_load8(V + (ch.t0 + t) * a.vt + ch.head * a.vh + 8 * o, a.vec_v, v[p]);
        }
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int t = p * TPP + row;
        if (a.n.k) norm8<OP>(k[p], a.n.k, o, c.dim, a.n.eps);
        if (a.r.cos) rotate8<OP>(k[p], a.r, pos[p], o, turn[row]);
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

template <class T>
qe_status append_typed(const void* Q, const void* K, const void* V, void* out, KvAppend a, const int64_t* slots, const KvCache& c,
                       int group, hipStream_t s)
{
    a.vec_q = vec_ok(Q, a.qt, a.qh, sizeof(T));
    a.vec_k = vec_ok(K, a.kt, a.kh, sizeof(T));
    a.vec_v = vec_ok(V, a.vt, a.vh, sizeof(T));
    a.vec_o = vec_ok(out, a.ot, a.oh, sizeof(T));
    a.kv_wgs = cdiv(a.tokens, kKvTok) * c.heads;
    const dim3 grid = grid_xy(a.kv_wgs + cdiv(a.tokens * a.heads, kKvTok), 256);
    kv_dispatch(c.dim, group, [&](auto shape) {
        hipLaunchKernelGGL((kv_append_kernel<T, shape.DP, shape.GROUP>), grid, dim3(256), 0, s, (const T*)Q, (const T*)K, (const T*)V,
                           (T*)out, slots, c, a);
    });
    return hipGetLastError() == hipSuccess ? QE_OK : QE_ERR_HIP;
}

}  // namespace

qe_status launch_kv_append(const void* Q, const void* K, const void* V, void* out, int dtype, const int64_t* strides, int64_t tokens,
                           int heads, const KvRotation& r, const KvNorm& n, const int64_t* slots, const KvCache& c, int group,
                           int* status, hipStream_t s)
{
    KvAppend a{};
    a.qt = strides[0];
    a.qh = strides[1];
    a.kt = strides[2];
    a.kh = strides[3];
    a.vt = strides[4];
    a.vh = strides[5];
    a.ot = strides[6];
    a.oh = strides[7];
    a.tokens = tokens;
    a.heads = heads;
    a.r = r;
    a.n = n;
    a.status = status;
    if (dtype == QE_F32) return append_typed<float>(Q, K, V, out, a, slots, c, group, s);
    if (dtype == QE_F16) return append_typed<_Float16>(Q, K, V, out, a, slots, c, group, s);
    return append_typed<__bf16>(Q, K, V, out, a, slots, c, group, s);
}

}  // namespace qe
