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
    bool narrow;                   // query rows are counted in 32 bits
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

// The sum over the OP lanes of a row, in all of them: inside 16 lanes by permutations that the vector units do themselves.
template <int CTRL> __device__ inline double moved(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)u, CTRL, 0xf, 0xf, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(u >> 32), CTRL, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int OP> __device__ inline double row_sum(double x)
{
    x += moved<0xB1>(x);                                 // lanes 1 0 3 2 of four
    x += moved<0x4E>(x);                                 // lanes 2 3 0 1 of four
    x += moved<0x141>(x);                                // eight lanes, mirrored
    if (OP >= 16) x += moved<0x140>(x);                  // sixteen lanes, mirrored
    if (OP == 32) x += __shfl_xor(x, 16);
    return x;
}

// 1 / sqrt(x) to a few units of fp64's last place: two steps of a third-order iteration on the hardware's estimate; 0, infinity
// and NaN as the estimate has them.
__device__ inline double root_inverse(double x)
{
    const double y0 = __builtin_amdgcn_rsq(x);
    double y = y0;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const double e = __builtin_fma(-x * y, y, 1.);
        y = __builtin_fma(y * e, __builtin_fma(e, 0.375, 0.5), y);
    }
    return y == y ? y : y0;
}

// A row's 8 channels, normed with their weights w.  OP lanes a row, zeros in those that have no channel.
template <int OP> __device__ inline void norm8(float (&x)[8], const float (&w)[8], const KvNorm& n)
{
#pragma clang fp contract(off)
    double ss = 0.;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = __builtin_fma((double)x[e], (double)x[e], ss);
    const float r = (float)root_inverse(row_sum<OP>(ss) * n.inv_dim + n.eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float y = x[e] * r;
        x[e] = y * w[e];
    }
}

// The cosines and sines of a row's 8 channels from 8 o on, where they lie aligned and beside each other (r.vec): with pairs of
// halves those of channel e in c[e], the sine's sign that of its product; else those of pair e in c[e], e < 4.
struct Turn { float c[8], s[8]; };
__device__ inline void turn_of(Turn& t, const KvRotation& r, int64_t pos, int o)
{
    if (!r.vec || 8 * o >= 2 * r.half) return;
    const int i = r.interleaved ? 4 * o : 8 * o < r.half ? 8 * o : 8 * o - r.half;
    const float sign = !r.interleaved && 8 * o < r.half ? -1.f : 1.f;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        if (y == 1 && r.interleaved) break;
        const f32x4 c = *reinterpret_cast<const f32x4*>(r.cos + pos * r.half + i + 4 * y);
        const f32x4 s = *reinterpret_cast<const f32x4*>(r.sin + pos * r.half + i + 4 * y);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            t.c[4 * y + e] = c[e];
            t.s[4 * y + e] = sign * s[e];
        }
    }
}

// A row's 8 channels, rotated.  at: the row's OP * 8 floats of LDS, used by its lanes (of one wave) alone.
template <int OP> __device__ inline void rotate8(float (&x)[8], const Turn& t, const KvRotation& r, int64_t pos, int o, float* at)
{
#pragma clang fp contract(off)
    if (r.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 4 * o + e;
            if (i >= r.half) continue;
            const float c = r.vec ? t.c[e] : r.cos[pos * r.half + i], s = r.vec ? t.s[e] : r.sin[pos * r.half + i];
            const float a = x[2 * e], b = x[2 * e + 1], ac = a * c, bs = b * s, bc = b * c, as = a * s;
            x[2 * e] = ac - bs;
            x[2 * e + 1] = bc + as;
        }
        return;
    }
    // (LDS serves a wave in order)
#pragma unroll
    for (int e = 0; e < 8; e += 4) *reinterpret_cast<f32x4*>(at + 8 * o + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
    __builtin_amdgcn_wave_barrier();
    if (r.vec) {
        if (8 * o < 2 * r.half) {
            const float* from = at + (8 * o < r.half ? 8 * o + r.half : 8 * o - r.half);
            const f32x4 a = *reinterpret_cast<const f32x4*>(from), b = *reinterpret_cast<const f32x4*>(from + 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float own = x[e] * t.c[e], far = (e < 4 ? a[e] : b[e - 4]) * t.s[e];
                x[e] = own + far;
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int d = 8 * o + e;
            if (d >= 2 * r.half) continue;
            const bool low = d < r.half;
            const int i = low ? d : d - r.half;
            const float c = r.cos[pos * r.half + i], s = r.sin[pos * r.half + i], other = at[low ? d + r.half : i];
            const float own = x[e] * c, far = other * s;
            x[e] = low ? own - far : own + far;
        }
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
    const bool mine = 8 * o < c.dim, query = wg >= a.kv_wgs;
    float w[8] = {};
    if (const float* from = query ? a.n.q : a.n.k; from && mine) kv_load8(from + 8 * o, a.n.vec, w);
    Turn t[P] = {};
    if (query) {
        const int64_t rows = a.tokens * a.heads, r0 = (wg - a.kv_wgs) * kKvTok;
        float x[P][8];
        int64_t pos[P], token[P];
        int head[P];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int64_t at = r0 + p * TPP + row;
            token[p] = a.narrow ? (int64_t)((uint32_t)at / (uint32_t)a.heads) : at / a.heads;
            head[p] = (int)(at - token[p] * a.heads);
            pos[p] = at < rows ? position_of(a, token[p]) : -1;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[p][e] = 0.f;
            if (mine && at < rows) kv_load8(Q + token[p] * a.qt + head[p] * a.qh + 8 * o, a.vec_q, x[p]);
        }
        if (a.r.cos) {
#pragma unroll
            for (int p = 0; p < P; ++p) turn_of(t[p], a.r, max(pos[p], (int64_t)0), o);
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (a.n.q) norm8<OP>(x[p], w, a.n);
            if (a.r.cos) rotate8<OP>(x[p], t[p], a.r, max(pos[p], (int64_t)0), o, turn[row]);
            if (mine && pos[p] >= 0) kv_store8(out + token[p] * a.ot + head[p] * a.oh + 8 * o, a.vec_o, x[p]);
        }
        return;
    }
    Chunk ch;
    if (!ch.open(wg, c, slots, a.tokens, a.status)) return;
    float k[P][8], v[P][8];
    int64_t slot[P], pos[P];
    // (a token without a position is not written: its slot is taken as none)
    int64_t at_lane = 0;
    if (a.r.positions) {
        at_lane = position_of(a, ch.t0 + (tid & 31));
        if (at_lane < 0) ch.slot = -1;
        ch.whole = __all(ch.slot >= 0) && ch.whole;
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int i = p * TPP + row;
        slot[p] = ch.slot_of(i);
        pos[p] = max((int64_t)0, (int64_t)__shfl(at_lane, i));
#pragma unroll
        for (int e = 0; e < 8; ++e) k[p][e] = v[p][e] = 0.f;
        if (mine && slot[p] >= 0) {
            kv_load8(K + (ch.t0 + i) * a.kt + ch.head * a.kh + 8 * o, a.vec_k, k[p]);
            kv_load8(V + (ch.t0 + i) * a.vt + ch.head * a.vh + 8 * o, a.vec_v, v[p]);
        }
    }
    if (a.r.cos) {
#pragma unroll
        for (int p = 0; p < P; ++p) turn_of(t[p], a.r, pos[p], o);
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int i = p * TPP + row;
        if (a.n.k) norm8<OP>(k[p], w, a.n);
        if (a.r.cos) rotate8<OP>(k[p], t[p], a.r, pos[p], o, turn[row]);
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
        tile[(2 * o) * kRowHalves + i] = (uint16_t)v8;
        tile[(2 * o + 1) * kRowHalves + i] = (uint16_t)(v8 >> 16);
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
    a.n.inv_dim = 1. / c.dim;
    a.n.vec = ((uintptr_t)n.q | (uintptr_t)n.k) % 16 == 0;
    a.r.vec = ((uintptr_t)r.cos | (uintptr_t)r.sin) % 16 == 0 && r.half % (r.interleaved ? 4 : 8) == 0;
    a.narrow = tokens * heads < (int64_t(1) << 31);
    a.status = status;
    if (dtype == QE_F32) return append_typed<float>(Q, K, V, out, a, slots, c, group, s);
    if (dtype == QE_F16) return append_typed<_Float16>(Q, K, V, out, a, slots, c, group, s);
    return append_typed<__bf16>(Q, K, V, out, a, slots, c, group, s);
}

}  // namespace qe
