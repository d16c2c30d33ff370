// Norm of each head's query and key, rotation by their positions, and the write into the 4-bit cache, in one pass (qe.h).
//
// Every step is one correctly rounded fp32 operation (the compiler must not fuse them), so that the codes, which are
// integers, are a function of the row's values alone; the norm's sum of squares and its root are in 64 bits, where another order
// of the sum or another root differs by some 2^-50 and moves the rounding to fp32 in one row of about 2^25:
//   r = fp32(1 / sqrt(sum x^2 / dim + eps)), y = fp32(fp32(x r) w),
//   a' = fp32(fp32(a c) - fp32(b s)), b' = fp32(fp32(b c) + fp32(a s)).
// A channel's partner in the rotation comes through the row's own stretch of LDS, where any number of rotated channels is
// right.  The first workgroups take 32 tokens' keys and values of a head each, as the plain write does (a thread
// has 8 channels of a row), the others queries.
//
// What bounds it: 16384 tokens of 32 + 8 + 8 heads of 128 in bf16, all channels rotated, take 84 us for 371 MB,
// 4.4 TB/s (a plain copy moves 4.9 to 5.1), with the vector units 65 % busy; without norm and rotation 76 us.  With the
// queries as the keys are, 8 channels a thread and a workgroup per 32 rows, the norm's sum through LDS and its weights
// and cosines a word a load, it took 234; wide loads and sums inside the vector units made it 149.  A few tokens
// cost their launch and three dependent loads: 5.6 us up to 64 tokens, 8 at 1024.
#include "kv_codes.h"

namespace qe {

namespace {

struct KvAppend {
    int64_t qt, qh, kt, kh, vt, vh, ot, oh;
    int64_t tokens, kv_wgs;
    int heads;
    bool vec_q, vec_k, vec_v, vec_o;
    int head_run, head_groups;     // heads that a workgroup goes through
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
    if (OP >= 8) x += moved<0x141>(x);                   // eight lanes, mirrored
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

// N channels of a row, normed with their weights w.  OP lanes a row, zeros in those that have no channel.
template <int OP, int N> __device__ inline void norm(float (&x)[N], const float (&w)[N], const KvNorm& n)
{
#pragma clang fp contract(off)
    double ss = 0.;
#pragma unroll
    for (int e = 0; e < N; ++e) ss = __builtin_fma((double)x[e], (double)x[e], ss);
    const float r = (float)root_inverse(row_sum<OP>(ss) * n.inv_dim + n.eps);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float y = x[e] * r;
        x[e] = y * w[e];
    }
}

// The cosines and sines of a row's 8 channels from 8 o on: with pairs of halves those of channel e in c[e], the sine with the
// sign of its product; else those of pair e in c[e], e < 4.  (Read once for all heads of a token; from rows that are
// aligned to 4 bytes alone, 16 at a time where they are pairs of an octet.)
struct Turn { float c[8], s[8]; };
typedef float f32x4a4 __attribute__((ext_vector_type(4), aligned(4)));
__device__ inline void turn_of(Turn& t, const KvRotation& r, int64_t pos, int o)
{
    const float *cos = r.cos + pos * r.half, *sin = r.sin + pos * r.half;
    if (8 * o >= 2 * r.half) return;
    auto four = [&](int y, int i, float sign) {
        const f32x4 c = *reinterpret_cast<const f32x4a4*>(cos + i), s = *reinterpret_cast<const f32x4a4*>(sin + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            t.c[4 * y + e] = c[e];
            t.s[4 * y + e] = sign * s[e];
        }
    };
    if (r.interleaved) {
        if (4 * o + 4 <= r.half) {
            four(0, 4 * o, 1.f);
            return;
        }
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (4 * o + e < r.half) {
                t.c[e] = cos[4 * o + e];
                t.s[e] = sin[4 * o + e];
            }
    } else if (r.vec) {
        const int i = 8 * o < r.half ? 8 * o : 8 * o - r.half;
        four(0, i, 8 * o < r.half ? -1.f : 1.f);
        four(1, i + 4, 8 * o < r.half ? -1.f : 1.f);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int d = 8 * o + e, i = d < r.half ? d : d - r.half;
            if (d >= 2 * r.half) continue;
            t.c[e] = cos[i];
            t.s[e] = d < r.half ? -sin[i] : sin[i];
        }
    }
}

// N octets of a row, o + n step, rotated.  at: the row's floats of LDS, used by its lanes (of one wave) alone.  here: the
// lane has channels.
template <int N> __device__ inline void rotate(float (&x)[8 * N], const Turn (&t)[N], const KvRotation& r, int o, int step, bool here, float* at)
{
#pragma clang fp contract(off)
    if (r.interleaved) {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = x[8 * n + 2 * e], b = x[8 * n + 2 * e + 1], c = t[n].c[e], s = t[n].s[e];
                const float ac = a * c, bs = b * s, bc = b * c, as = a * s;
                const bool turned = 4 * (o + n * step) + e < r.half;
                x[8 * n + 2 * e] = turned ? ac - bs : a;
                x[8 * n + 2 * e + 1] = turned ? bc + as : b;
            }
        return;
    }
    // (LDS serves a wave in order)
    if (here) {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < 8; e += 4) *reinterpret_cast<f32x4*>(at + 8 * (o + n * step) + e) = f32x4{x[8 * n + e], x[8 * n + e + 1], x[8 * n + e + 2], x[8 * n + e + 3]};
    }
    __builtin_amdgcn_wave_barrier();
    if (here) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int d0 = 8 * (o + n * step);
            if (d0 >= 2 * r.half) continue;
            float other[8];
            if (r.vec) {
                const float* from = at + (d0 < r.half ? d0 + r.half : d0 - r.half);
                const f32x4 a = *reinterpret_cast<const f32x4*>(from), b = *reinterpret_cast<const f32x4*>(from + 4);
#pragma unroll
                for (int e = 0; e < 8; ++e) other[e] = e < 4 ? a[e] : b[e - 4];
            } else {
                // (past the rotated channels: any of the row's)
#pragma unroll
                for (int e = 0; e < 8; ++e) other[e] = at[d0 + e < r.half ? d0 + e + r.half : d0 + e - r.half];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float own = x[8 * n + e] * t[n].c[e], far = other[e] * t[n].s[e];
                x[8 * n + e] = d0 + e < 2 * r.half ? own + far : x[8 * n + e];
            }
        }
    }
    __builtin_amdgcn_wave_barrier();
}

// Eight channels as they lie in memory.
template <class T> struct Raw8 {
    u32x4 at[sizeof(T) / 2];
    __device__ void load(const T* p, bool vec)
    {
        if (vec) {
#pragma unroll
            for (int u = 0; u < (int)sizeof(T) / 2; ++u) at[u] = reinterpret_cast<const u32x4*>(p)[u];
        } else {
            T v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = p[e];
            __builtin_memcpy(at, v, sizeof(v));
        }
    }
    __device__ void get(float* x) const
    {
        T v[8];
        __builtin_memcpy(v, at, sizeof(v));
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
    }
};

// The queries of some tokens and heads.  A lane has two octets of a token's channels, o and o + step, half as many lanes a row
// as for the keys: the norm's sum and root, which every lane of a row forms, are shared by twice the channels, and where all
// channels are rotated by halves the partners lie in one lane.  It goes through its heads with one set of
// cosines and sines, the next head's loads on the way.
template <class T, int DP>
__device__ inline void kv_queries(const T* Q, T* out, int dim, const KvAppend& a, int64_t wg, float* turn)
{
#pragma clang fp contract(off)
    constexpr int OQ = kOctets<DP> / 2, ROWS = 256 / OQ;
    const int64_t chunk = wg / a.head_groups;
    const int h0 = (int)(wg - chunk * a.head_groups) * a.head_run, h1 = min(h0 + a.head_run, a.heads);
    const int tid = threadIdx.x, o = tid % OQ, row = tid / OQ;
    const int step = (dim / 8 + 1) / 2;
    const int64_t token = chunk * ROWS + row;
    const int64_t pos = token < a.tokens ? position_of(a, token) : -1;
    const bool here[2] = {pos >= 0 && o < step, pos >= 0 && 8 * (o + step) < dim && o < step};
    const int at[2] = {8 * o, 8 * (o + step)};
    const T* from = Q + token * a.qt + h0 * a.qh;
    T* to = out + token * a.ot + h0 * a.oh;
    Raw8<T> next[2] = {};
    float w[16] = {};
#pragma unroll
    for (int y = 0; y < 2; ++y)
        if (here[y] && h0 < h1) next[y].load(from + at[y], a.vec_q);
    if (a.n.q) {
#pragma unroll
        for (int y = 0; y < 2; ++y)
            if (here[y]) kv_load8(a.n.q + at[y], a.n.vec, w + 8 * y);
    }
    // by halves, all of an even number of octets: channel e of the one octet and of the other are a pair
    const bool paired = a.r.vec && !a.r.interleaved && 2 * a.r.half == dim;
    Turn t[2] = {};
    if (a.r.cos && pos >= 0 && o < step) {
        turn_of(t[0], a.r, pos, o);
        if (!paired) turn_of(t[1], a.r, pos, o + step);
    }
    float* const mine = turn + row * (kOctets<DP> * 8 + 8);
    for (int h = h0; h < h1; ++h) {
        float x[16];
#pragma unroll
        for (int y = 0; y < 2; ++y) next[y].get(x + 8 * y);
        from += a.qh;
        if (h + 1 < h1) {
#pragma unroll
            for (int y = 0; y < 2; ++y)
                if (here[y]) next[y].load(from + at[y], a.vec_q);
        }
        if (a.n.q) norm<OQ>(x, w, a.n);
        if (paired) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // (t[0].s is the sine with the sign of the first of a pair)
                const float ac = x[e] * t[0].c[e], bs = x[8 + e] * t[0].s[e], bc = x[8 + e] * t[0].c[e], as = x[e] * t[0].s[e];
                x[e] = ac + bs;
                x[8 + e] = bc - as;
            }
        } else if (a.r.cos) {
            rotate<2>(x, t, a.r, o, step, o < step, mine);
        }
#pragma unroll
        for (int y = 0; y < 2; ++y)
            if (here[y]) kv_store8(to + at[y], a.vec_o, x + 8 * y);
        to += a.oh;
    }
}

template <class T, int DP, int GROUP>
__global__ __launch_bounds__(256, sizeof(T) == 4 ? 3 : 4) void kv_append_kernel(const T* Q, const T* __restrict__ K, const T* __restrict__ V, T* out,
                                                        const int64_t* __restrict__ slots, KvCache c, KvAppend a)
{
    using R = KvRec<DP, GROUP>;
    constexpr int OP = kOctets<DP>, TPP = 256 / OP, P = OP / 8;      // rows of a pass, passes
    constexpr int LANES = GROUP / 8 < OP ? GROUP / 8 : OP;
    __shared__ __align__(16) uint16_t tile[(DP / 4) * kRowHalves];
    __shared__ __align__(16) float turn[TPP][2 * (OP * 8 + 8)];      // (the queries have twice the rows)
    const int64_t wg = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int tid = threadIdx.x, o = tid % OP, row = tid / OP;
    const bool mine = 8 * o < c.dim;
    if (wg >= a.kv_wgs) {
        kv_queries<T, DP>(Q, out, c.dim, a, wg - a.kv_wgs, &turn[0][0]);
        return;
    }
    float w[8] = {};
    if (a.n.k && mine) kv_load8(a.n.k + 8 * o, a.n.vec, w);
    Chunk ch;
    if (!ch.open(wg, c, slots, a.tokens, a.status)) return;
    Raw8<T> k[P] = {}, v[P] = {};
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
        if (mine && slot[p] >= 0) {
            k[p].load(K + (ch.t0 + i) * a.kt + ch.head * a.kh + 8 * o, a.vec_k);
            v[p].load(V + (ch.t0 + i) * a.vt + ch.head * a.vh + 8 * o, a.vec_v);
        }
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int i = p * TPP + row;
        Turn t[1] = {};
        if (a.r.cos) turn_of(t[0], a.r, pos[p], o);
        float x[8], y[8];
        k[p].get(x);
        v[p].get(y);
        if (a.n.k) norm<OP>(x, w, a.n);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = mine ? x[e] : 0.f;        // (0 times an infinite root)
        if (a.r.cos) rotate<1>(x, t, a.r, o, 0, true, turn[row]);
        uint32_t kw, vw;
        const uint32_t k8 = quantize8<LANES>(x, kw), v8 = quantize8<LANES>(y, vw);
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
    kv_dispatch(c.dim, group, [&](auto shape) {
        // Heads that a workgroup goes through: as many as leave two workgroups for a compute unit, four at most.  32 heads of
        // 128, us with 1, 2, 4 and 8: 256 tokens 6.2, 6.2, 6.2, 8.9; 1024 8.7, 7.8, 8.0, 11.5; 2048 15.6, 13.6, 13.1,
        // 14.8; 16384 105, 88, 84, 87.
        const int64_t chunks = cdiv(a.tokens, 512 / kOctets<shape.DP>);
        a.head_run = (int)std::max<int64_t>(1, std::min<int64_t>(4, chunks * a.heads / 512));
        a.head_groups = (int)cdiv(a.heads, a.head_run);
        const dim3 grid = grid_xy(a.kv_wgs + chunks * a.head_groups, 256);
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
    a.r.vec = !r.interleaved && r.half % 8 == 0;
    a.status = status;
    if (dtype == QE_F32) return append_typed<float>(Q, K, V, out, a, slots, c, group, s);
    if (dtype == QE_F16) return append_typed<_Float16>(Q, K, V, out, a, slots, c, group, s);
    return append_typed<__bf16>(Q, K, V, out, a, slots, c, group, s);
}

}  // namespace qe
