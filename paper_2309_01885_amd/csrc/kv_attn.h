// The attention kernel over the 4-bit cache, for one width (instantiated by kv_attn_*.hip).
//
//   S^T = K Q^T on v_mfma_f32_16x16x32_f16 (A: 16 tokens x 32 channels of codes, B: query rows),
//   P = exp2(S - m) with a running maximum, O^T += V^T P^T (A: 16 channels x 32 tokens).
// The scales stay outside of the products: S_t = s_t sum_d q'_d (n_td - z_t) with q' the query
// scaled by a power of two, O_d = sum_t (p_t s'_t) (n_td - z_t).
// A code becomes the exact fp16 number n - z: 1024 + n by its bits, less 1024 + z, nine
// instructions for a word of eight.  (Codes as they are, subnormals n 2^-24, would take five, but
// the matrix cores align products by exponent and lose a subnormal's leading zeros: 2^-17 of
// the sums' size, which showed in the scores.)
// C of the first product (lane l: query l % 16, tokens by l / 16) is B of the second without a
// move between lanes: token 8 (l / 16) + 4 h + r is row 4 (l / 16) + r of half h.
#pragma once

#include "kv.h"

namespace qe {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2a8 __attribute__((ext_vector_type(2), aligned(8)));
typedef uint32_t u32x3a4 __attribute__((ext_vector_type(3), aligned(4)));

constexpr int kKvWaves = 4;                 // waves of a workgroup
constexpr float kKvInf = __builtin_inff();
constexpr float kLog2e = 1.44269504088896341f;

// How a call is cut into workgroups.  A unit is a tile of `rows` query rows (row = query *
// heads per key head + head in the group) of one sequence and key head; each unit has
// nsplit workgroups along the tokens, whose results kv_join_kernel joins.
struct KvPlan {
    int64_t row_tiles;                      // units of a sequence and key head
    int nsplit, rows;
    float* part;                            // nsplit > 1: (unit, split, row, DP) sums relative to the maximum
    float* stat;                            // (unit, split, row, 2): maximum (log2) and mass
};

// What a workgroup works on; the join recomputes it.
struct KvUnit {
    int64_t first, pos0, len;               // first row of Q, position of query 0, cached tokens
    int nq, rec0, rec1, splits;             // queries; records that any row of the unit sees; splits in use
};

// Records a split has at least (a workgroup's waves take them in turn).
constexpr int kKvMinRecords = 4;

__device__ inline KvUnit kv_unit(const KvAttn& a, const KvPlan& p, int64_t b, int64_t tile, bool report)
{
    KvUnit u;
    bool bad = false;
    u.first = b * a.max_q;
    int64_t nq = a.max_q;
    if (a.q_start) {
        u.first = a.q_start[b];
        nq = (int64_t)a.q_start[b + 1] - u.first;
        bad = u.first < 0 || nq < 0 || nq > a.max_q || u.first + nq > a.total;
        u.first = u.first < 0 ? 0 : u.first;
        nq = min(min(nq, a.max_q), a.total - u.first);
    }
    const int64_t room = a.width * (int64_t)a.c.per * kKvTok;
    u.len = a.lengths[b];
    bad = bad || u.len < 0 || u.len > room;
    u.len = u.len < 0 ? 0 : min(u.len, room);
    if (bad && report) set_status(a.status, QE_ERR_ARG);
    u.nq = nq < 0 ? 0 : (int)nq;
    u.pos0 = u.len - u.nq;
    // the rows of the unit are queries i0 .. i1
    const int per = a.heads / a.c.heads;
    const int64_t i0 = tile * p.rows / per, i1 = min((int64_t)u.nq, (tile * p.rows + p.rows + per - 1) / per) - 1;
    int64_t end = a.causal ? min(u.len, u.pos0 + i1 + 1) : u.len;
    int64_t begin = a.window ? max((int64_t)0, u.pos0 + i0 - a.window + 1) : 0;
    if (i0 >= u.nq || end < begin) end = begin = 0;
    u.rec0 = (int)(begin / kKvTok);
    u.rec1 = (int)((end + kKvTok - 1) / kKvTok);
    u.splits = max(1, min(p.nsplit, (u.rec1 - u.rec0) / kKvMinRecords));
    return u;
}

__device__ inline float kv_q_elem(const KvAttn& a, int64_t at)
{
    return a.dtype == QE_F32 ? static_cast<const float*>(a.q)[at]
         : a.dtype == QE_F16 ? (float)static_cast<const _Float16*>(a.q)[at] : (float)static_cast<const __bf16*>(a.q)[at];
}
__device__ inline void kv_q8(const KvAttn& a, int64_t at, float* x)
{
    if (a.dtype == QE_F32) kv_load8(static_cast<const float*>(a.q) + at, a.vec_q, x);
    else if (a.dtype == QE_F16) kv_load8(static_cast<const _Float16*>(a.q) + at, a.vec_q, x);
    else kv_load8(static_cast<const __bf16*>(a.q) + at, a.vec_q, x);
}
__device__ inline void kv_out(const KvAttn& a, int64_t at, float x)
{
    if (a.dtype == QE_F32) static_cast<float*>(a.out)[at] = x;
    else if (a.dtype == QE_F16) static_cast<_Float16*>(a.out)[at] = (_Float16)x;
    else static_cast<__bf16*>(a.out)[at] = (__bf16)x;
}

// A pair of codes of a word (nibbles k and k + 4 of w >> 4 k') less their zero points: `high`: the
// codes in bits 4-7, times 16.  minus: a pair of -(1024 + z), or of -(1024 + 16 z).
__device__ inline uint32_t kv_code_pair(uint32_t w, bool high, uint32_t minus)
{
    const uint32_t n = (w & (high ? 0x00F000F0u : 0x000F000Fu)) | 0x64006400u;
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, n) + __builtin_bit_cast(f16x2, minus));
}

// N consecutive words at an address that is a multiple of 4 N bytes up to 16 (N = 3: of 4).
template <int N> __device__ inline void kv_words(const uint8_t* p, uint32_t* w)
{
    if constexpr (N == 3) {
        const u32x3a4 v = *reinterpret_cast<const u32x3a4*>(p);
        w[0] = v[0];
        w[1] = v[1];
        w[2] = v[2];
    } else if constexpr (N % 4 == 0) {
#pragma unroll
        for (int u = 0; u < N; u += 4) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(p + 4 * u);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[u + e] = v[e];
        }
    } else {
#pragma unroll
        for (int u = 0; u < N; u += 2) {
            const u32x2a8 v = *reinterpret_cast<const u32x2a8*>(p + 4 * u);
            w[u] = v[0];
            w[u + 1] = v[1];
        }
    }
}

__device__ inline f16x8 kv_frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const u32x4 v = {a, b, c, d};
    return __builtin_bit_cast(f16x8, v);
}
__device__ inline uint32_t kv_pack(float a, float b)
{
    const f16x2 v = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ inline f32x4 kv_mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

__device__ inline float kv_max4(float x)    // over the four lanes of a query
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float kv_sum4(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// NT tiles of 16 query rows per wave.  ROWS: the workgroup's waves have rows of their own
// and see the same tokens; else they share the rows and take the records in turn.
// PARTS: fp16 parts of a query and of a probability (2 for fp32 calls).
template <int DP, int GROUP, int NT, int PARTS, bool ROWS>
__global__ __launch_bounds__(256, 2) void kv_attn_kernel(KvAttn a, KvPlan plan)
{
    using R = KvRec<DP, GROUP>;
    constexpr int NC = R::NC, NG = R::NG;
    constexpr int CPG = GROUP / 32;                      // 32-channel products of a key group
    // products of a record's values: a lane's unit is 4 channels; groups of 32 pair two
    // classes of 8 units, wider ones one class of 16
    constexpr bool kHalf = GROUP == 32;
    constexpr int UT = kHalf ? DP / 32 : (DP + 63) / 64; // unit tiles
    constexpr int CL = kHalf ? 2 : 4;                    // channel classes of a unit tile
    const int64_t wg = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int split = (int)(wg % plan.nsplit);
    const int64_t unit = wg / plan.nsplit, bh = unit / plan.row_tiles, tile = unit - bh * plan.row_tiles;
    const int64_t b = bh / a.c.heads;
    if (b >= a.batch) return;
    const int kvh = (int)(bh - b * a.c.heads);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i = tid & 15, j = (tid & 63) >> 4;
    const KvUnit u = kv_unit(a, plan, b, tile, tid == 0 && split == 0 && tile == 0 && kvh == 0);
    if (split >= u.splits) return;
    const int per = a.heads / a.c.heads;
    const int64_t rows = (int64_t)u.nq * per;
    const int64_t row0 = tile * plan.rows + (ROWS ? wave * (16 * NT) : 0);
    if ((ROWS ? row0 : tile * plan.rows) >= rows) return;

    // ---- the query rows: scaled by 2^e to a largest element in [2^14, 2^15), rounded to fp16
    f16x8 q[PARTS][NT][NC];
    float cq[NT], slope[NT];
    int64_t lo[NT], hi[NT];                              // the tokens that the lane's row sees
    int64_t all_lo = 0, all_hi = u.len;                  // that every row of the wave sees
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int64_t row = row0 + 16 * n + i;
        const bool have = row < rows;
        const int qi = have ? (int)(row / per) : 0, head = kvh * per + (have ? (int)(row - (int64_t)qi * per) : 0);
        float x[NC][8];
        float top = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[c][e] = 0.f;
            const int d = 8 * (4 * c + j);
            if (have && d < a.c.dim) kv_q8(a, (u.first + qi) * a.qt + head * a.qh + d, x[c]);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[c][e]));
        }
        top = kv_max4(top);
        // (a row of zeros, NaN or infinities keeps its values)
        const int e2 = top > 0.f && top <= 3.402823466e38f ? max(-100, min(100, 15 - (int)((__float_as_uint(top) >> 23) - 126))) : 0;
        const float mul = __uint_as_float((uint32_t)(127 + e2) << 23) * (a.scale < 0.f ? -1.f : 1.f);
        cq[n] = fabsf(a.scale) * kLog2e * __uint_as_float((uint32_t)(127 - e2) << 23);
        slope[n] = a.slopes && have ? a.slopes[head] * kLog2e : 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            // (channels 1, 3, 5, 7 meet codes in bits 4-7, 16 times as large)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[c][e] *= mul;
            uint32_t h[4], m[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const float f = p & 1 ? 0.0625f : 1.f;
                const _Float16 h0 = (_Float16)(x[c][p] * f), h1 = (_Float16)(x[c][p + 4] * f);
                const f16x2 hv = {h0, h1};
                h[p] = __builtin_bit_cast(uint32_t, hv);
                if constexpr (PARTS == 2) {
                    const _Float16 m0 = (_Float16)(x[c][p] * f - (float)h0), m1 = (_Float16)(x[c][p + 4] * f - (float)h1);
                    const f16x2 mv = {m0, m1};
                    m[p] = __builtin_bit_cast(uint32_t, mv);
                }
            }
            q[0][n][c] = kv_frag(h[0], h[1], h[2], h[3]);
            if constexpr (PARTS == 2) q[1][n][c] = kv_frag(m[0], m[1], m[2], m[3]);
        }
        const int64_t pos = u.pos0 + qi;
        hi[n] = !have ? u.len : a.causal ? min(u.len, pos + 1) : u.len;
        lo[n] = have && a.window ? pos - a.window + 1 : 0;
    }
    int64_t any_lo = 0, any_hi = u.len;                  // that some row of the wave sees
    if (a.causal) {
        // the first and the last row of the wave bound the others
        const int64_t last = min(rows, row0 + 16 * NT) - 1;
        all_hi = min(u.len, u.pos0 + row0 / per + 1);
        any_hi = min(u.len, u.pos0 + last / per + 1);
        if (a.window) {
            all_lo = u.pos0 + last / per - a.window + 1;
            any_lo = u.pos0 + row0 / per - a.window + 1;
        }
    }

    // ---- the sums
    f32x4 o[UT][CL][NT];
    float top[NT], mass[NT];
    float limit[NG], norm[NG];                           // largest value scale allowed; 2^10 / its power of two
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int t = 0; t < UT; ++t)
#pragma unroll
            for (int c = 0; c < CL; ++c) o[t][c][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        top[n] = -kKvInf;
        mass[n] = 0.f;
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        limit[g] = 0.f;
        norm[g] = 1.f;
    }

    const int count = u.rec1 - u.rec0;
    const int r0 = u.rec0 + (int)((int64_t)count * split / u.splits), r1 = u.rec0 + (int)((int64_t)count * (split + 1) / u.splits);
    const int64_t pages = a.c.slots / ((int64_t)a.c.per * kKvTok);
    for (int r = r0 + (ROWS ? 0 : wave); r < r1; r += ROWS ? 1 : kKvWaves) {
        const int64_t t0 = (int64_t)r * kKvTok;
        if (ROWS && (t0 >= any_hi || t0 + kKvTok <= any_lo)) continue;
        const uint32_t pg = (uint32_t)r / a.c.per;
        const int64_t id = a.table[b * a.width + pg];
        if (id < 0 || id >= pages) {
            set_status(a.status, QE_ERR_ARG);
            continue;
        }
        const uint8_t* rec = a.c.pages + ((id * a.c.heads + kvh) * a.c.per + ((uint32_t)r - pg * a.c.per)) * R::kBytes;
        uint32_t kraw[2][NC], vraw[UT][4], kw[NG][8], vw[NG][8];
#pragma unroll
        for (int h = 0; h < 2; ++h) kv_words<NC>(rec + (8 * (i >> 2) + 4 * h + (i & 3)) * R::kKeyRow + j * (4 * NC), kraw[h]);
#pragma unroll
        for (int g = 0; g < NG; ++g) kv_words<8>(rec + R::kKeyWords + g * (4 * kKvTok) + 32 * j, kw[g]);
#pragma unroll
        for (int t = 0; t < UT; ++t) {
            int unit4 = kHalf ? 8 * t + (i & 7) : 16 * t + i;
            if (DP % 64 != 0 && !kHalf) unit4 = min(unit4, DP / 4 - 1);      // (the lanes past the last unit give nothing)
            kv_words<4>(rec + R::kVal + unit4 * (2 * kKvTok) + 16 * j, vraw[t]);
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) kv_words<8>(rec + R::kValWords + g * (4 * kKvTok) + 32 * j, vw[g]);

        uint32_t kz[2][NG];                              // zero points of the tokens whose codes the lane holds
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int g = 0; g < NG; ++g)
                kz[h][g] = reinterpret_cast<const uint32_t*>(rec + R::kKeyWords)[g * kKvTok + 8 * (i >> 2) + 4 * h + (i & 3)] & 15u;

        // ---- scores
        float s[NT][8];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            f32x4 acc[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) acc[n][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = g * CPG; c < (g + 1) * CPG && c < NC; ++c)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t w = kraw[h][c], w8 = w >> 8;
                    const uint32_t lo = kz[h][g] * 0x10001u | 0xE400E400u, hi = kz[h][g] * 0x100010u | 0xE400E400u;
                    const f16x8 f = kv_frag(kv_code_pair(w, false, lo), kv_code_pair(w, true, hi),
                                            kv_code_pair(w8, false, lo), kv_code_pair(w8, true, hi));
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) acc[n][h] = kv_mfma(f, q[p][n][c], acc[n][h]);
                }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float sc = kv_scale(kw[g][e]), v = acc[n][e >> 2][e & 3];
                    s[n][e] = g == 0 ? sc * v : fmaf(sc, v, s[n][e]);
                }
        }

        // ---- probabilities
        const bool masked = t0 + kKvTok > all_hi || t0 < all_lo;
        uint32_t seen = 0xffu;                           // tokens of the lane that lie before the sequence's end
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float c = cq[n];
            if (a.slopes) {
                const float base = slope[n] * (float)(int)(t0 + 8 * j - (hi[n] - 1));
#pragma unroll
                for (int e = 0; e < 8; ++e) s[n][e] = fmaf(s[n][e], c, fmaf(slope[n], (float)e, base));
                c = 1.f;
            }
            uint32_t vis = 0xffu;
            float big;
            if (masked) {
                big = -kKvInf;
                vis = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t t = t0 + 8 * j + e;
                    const bool see = t >= lo[n] && t < hi[n];
                    vis |= (see ? 1u : 0u) << e;
                    big = see ? fmaxf(big, s[n][e]) : big;
                }
            } else {
                big = fmaxf(fmaxf(fmaxf(s[n][0], s[n][1]), fmaxf(s[n][2], s[n][3])), fmaxf(fmaxf(s[n][4], s[n][5]), fmaxf(s[n][6], s[n][7])));
            }
            big *= c;
            // the maximum moves only when it has to: probabilities reach 2^4 before
            if (__any(big > top[n] + 4.f)) {
                const float m = kv_max4(fmaxf(top[n], big));
                const float f = m == top[n] ? 1.f : __builtin_amdgcn_exp2f(top[n] - m);
                top[n] = m;
                mass[n] *= f;
#pragma unroll
                for (int t = 0; t < UT; ++t)
#pragma unroll
                    for (int k = 0; k < CL; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[t][k][n][e] *= f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) s[n][e] = __builtin_amdgcn_exp2f(fmaf(s[n][e], c, -top[n]));
            if (masked) {
#pragma unroll
                for (int e = 0; e < 8; ++e) s[n][e] = vis >> e & 1u ? s[n][e] : 0.f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) mass[n] += s[n][e];
        }
        if (t0 + kKvTok > u.len) {
            // words past the sequence's end are anything: no scale of theirs may meet a 0
#pragma unroll
            for (int e = 0; e < 8; ++e) seen &= t0 + 8 * j + e < u.len ? ~0u : ~(1u << e);
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int e = 0; e < 8; ++e) vw[g][e] = seen >> e & 1u ? vw[g][e] : 0u;
        }

        // ---- weighted sum of the values
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            float sv[8];
            float big = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sv[e] = kv_scale(vw[g][e]);
                big = fmaxf(big, sv[e]);
            }
            // p s' stays below 2^15: s' is the scale over the largest one's power of two, times 2^10
            if (__any(big > limit[g])) {
                big = kv_max4(big);
                big = fmaxf(big, __shfl_xor(big, 1));
                const uint32_t ex = max(__float_as_uint(big) >> 23, 20u);
                limit[g] = __uint_as_float(ex << 23 | 0x7fffffu);
                const float to = __uint_as_float((264u - ex) << 23), f = to / norm[g];
                norm[g] = to;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int t = 0; t < UT; ++t)
                        if ((kHalf ? 32 * t : 64 * t) / GROUP == g)
#pragma unroll
                            for (int k = 0; k < CL; ++k)
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[t][k][n][e] *= f;
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sv[e] *= norm[g];
            f16x8 pr[PARTS][NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                uint32_t h[4], m[4];
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    float x0 = s[n][2 * p] * sv[2 * p], x1 = s[n][2 * p + 1] * sv[2 * p + 1];
                    if (masked) {                        // (a NaN scale of a token that the row does not see)
                        x0 = s[n][2 * p] == 0.f ? 0.f : x0;
                        x1 = s[n][2 * p + 1] == 0.f ? 0.f : x1;
                    }
                    h[p] = kv_pack(x0, x1);
                    if constexpr (PARTS == 2) {
                        const f16x2 hv = __builtin_bit_cast(f16x2, h[p]);
                        m[p] = kv_pack(x0 - (float)hv[0], x1 - (float)hv[1]);
                    }
                }
                pr[0][n] = kv_frag(h[0], h[1], h[2], h[3]);
                if constexpr (PARTS == 2) pr[1][n] = kv_frag(m[0], m[1], m[2], m[3]);
            }
            uint32_t z[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) z[p] = __builtin_amdgcn_perm(vw[g][2 * p + 1], vw[g][2 * p], 0x05040100u) & 0x000F000Fu;
#pragma unroll
            for (int t = 0; t < UT; ++t) {
                if ((kHalf ? 32 * t : 64 * t) / GROUP != g) continue;
                uint32_t w[4];
#pragma unroll
                for (int p = 0; p < 4; ++p) w[p] = kHalf ? vraw[t][p] >> (i & 8) : vraw[t][p];
#pragma unroll
                for (int k = 0; k < CL; ++k) {
                    uint32_t v[4];
#pragma unroll
                    for (int p = 0; p < 4; ++p)
                        v[p] = kv_code_pair(w[p] >> (k >= 2 ? 8 : 0), k & 1, (k & 1 ? z[p] << 4 : z[p]) | 0xE400E400u);
                    const f16x8 f = kv_frag(v[0], v[1], v[2], v[3]);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) o[t][k][n] = kv_mfma(f, pr[p][n], o[t][k][n]);
                }
            }
        }
    }

    // ---- to plain sums relative to the maximum: o[t][k][n][e] is channel `channel(t, k, 4 j + e)`
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        mass[n] = kv_sum4(mass[n]);
#pragma unroll
        for (int t = 0; t < UT; ++t) {
            const int g = (kHalf ? 32 * t : 64 * t) / GROUP;
            const float f = 1.f / norm[g];
#pragma unroll
            for (int k = 0; k < CL; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[t][k][n][e] *= k & 1 ? 0.0625f * f : f;
        }
    }

    if constexpr (!ROWS) {
        // join the waves: every wave to the common maximum, then sums over the waves through LDS
        __shared__ float wtop[kKvWaves][16 * NT], wmass[kKvWaves][16 * NT];
        __shared__ float acc[kKvWaves][16 * NT][DP + 1];
#pragma unroll
        for (int n = 0; n < NT; ++n)
            if (j == 0) {
                wtop[wave][16 * n + i] = top[n];
                wmass[wave][16 * n + i] = mass[n];
            }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float m = wtop[0][16 * n + i];
#pragma unroll
            for (int w = 1; w < kKvWaves; ++w) m = fmaxf(m, wtop[w][16 * n + i]);
            const float f = m == top[n] ? 1.f : __builtin_amdgcn_exp2f(top[n] - m);
#pragma unroll
            for (int t = 0; t < UT; ++t)
#pragma unroll
                for (int k = 0; k < CL; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int rho = 4 * j + e;
                        const int d = kHalf ? 32 * t + 4 * (rho & 7) + k + 2 * (rho >> 3) : 64 * t + 4 * rho + k;
                        if (DP % 64 == 0 || kHalf || d < DP) acc[wave][16 * n + i][d] = o[t][k][n][e] * f;
                    }
        }
        __syncthreads();
        for (int at = tid; at < 16 * NT * DP; at += 256) {
            const int rr = at / DP, d = at - rr * DP;
            const int64_t row = row0 + rr;
            if (row >= rows) break;
            float m = -kKvInf, l = 0.f, x = 0.f;
#pragma unroll
            for (int w = 0; w < kKvWaves; ++w) m = fmaxf(m, wtop[w][rr]);
#pragma unroll
            for (int w = 0; w < kKvWaves; ++w) {
                l += wtop[w][rr] == m ? wmass[w][rr] : wmass[w][rr] * __builtin_amdgcn_exp2f(wtop[w][rr] - m);
                x += acc[w][rr][d];
            }
            if (u.splits > 1) {
                const int64_t slot = (unit * plan.nsplit + split) * plan.rows + rr;
                plan.part[slot * DP + d] = x;
                if (d == 0) {
                    plan.stat[2 * slot] = m;
                    plan.stat[2 * slot + 1] = l;
                }
            } else {
                const int64_t qi = row / per;
                const int head = kvh * per + (int)(row - qi * per);
                if (d < a.c.dim) kv_out(a, (u.first + qi) * a.ot + head * a.oh + d, l == 0.f ? 0.f : x / l);
                if (a.lse && d == 0) a.lse[(u.first + qi) * a.heads + head] = l == 0.f ? -kKvInf : (m + __builtin_amdgcn_logf(l)) / kLog2e;
            }
        }
    } else {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int64_t row = row0 + 16 * n + i;
            if (row >= rows) continue;
            const int64_t qi = row / per;
            const int head = kvh * per + (int)(row - qi * per);
            const int64_t slot = (unit * plan.nsplit + split) * plan.rows + (row - tile * plan.rows);
            const float inv = mass[n] == 0.f ? 0.f : 1.f / mass[n];
#pragma unroll
            for (int t = 0; t < UT; ++t)
#pragma unroll
                for (int k = 0; k < CL; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int rho = 4 * j + e;
                        const int d = kHalf ? 32 * t + 4 * (rho & 7) + k + 2 * (rho >> 3) : 64 * t + 4 * rho + k;
                        if (u.splits > 1) {
                            if (DP % 64 == 0 || kHalf || d < DP) plan.part[slot * DP + d] = o[t][k][n][e];
                        } else if (d < a.c.dim)
                            kv_out(a, (u.first + qi) * a.ot + head * a.oh + d, mass[n] == 0.f ? 0.f : o[t][k][n][e] * inv);
                    }
            if (j == 0) {
                if (u.splits > 1) {
                    plan.stat[2 * slot] = top[n];
                    plan.stat[2 * slot + 1] = mass[n];
                } else if (a.lse)
                    a.lse[(u.first + qi) * a.heads + head] = mass[n] == 0.f ? -kKvInf : (top[n] + __builtin_amdgcn_logf(mass[n])) / kLog2e;
            }
        }
    }
}

// Joins the splits of a row: one wave per row.
template <int DP> __global__ __launch_bounds__(256) void kv_join_kernel(KvAttn a, KvPlan plan)
{
    const int64_t at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int64_t unit = at / plan.rows, rr = at - unit * plan.rows, bh = unit / plan.row_tiles, tile = unit - bh * plan.row_tiles;
    const int64_t b = bh / a.c.heads;
    if (b >= a.batch) return;
    const int kvh = (int)(bh - b * a.c.heads), per = a.heads / a.c.heads;
    const KvUnit u = kv_unit(a, plan, b, tile, false);
    const int64_t row = tile * plan.rows + rr;
    if (u.splits <= 1 || row >= (int64_t)u.nq * per) return;
    const int64_t slot = unit * plan.nsplit * plan.rows + rr;
    float m = -kKvInf;
    for (int s = lane; s < u.splits; s += 64) m = fmaxf(m, plan.stat[2 * (slot + (int64_t)s * plan.rows)]);
#pragma unroll
    for (int x = 1; x < 64; x *= 2) m = fmaxf(m, __shfl_xor(m, x));
    float l = 0.f, x[DP / 64 + (DP % 64 != 0)] = {};
    for (int s = 0; s < u.splits; ++s) {
        const int64_t k = slot + (int64_t)s * plan.rows;
        const float t = plan.stat[2 * k], f = t == m ? 1.f : __builtin_amdgcn_exp2f(t - m);
        l = fmaf(plan.stat[2 * k + 1], f, l);
#pragma unroll
        for (int c = 0; c < (DP + 63) / 64; ++c)
            if (DP % 64 == 0 || 64 * c + lane < DP) x[c] = fmaf(plan.part[k * DP + 64 * c + lane], f, x[c]);
    }
    const int64_t qi = row / per;
    const int head = kvh * per + (int)(row - qi * per);
#pragma unroll
    for (int c = 0; c < (DP + 63) / 64; ++c)
        if (64 * c + lane < a.c.dim) kv_out(a, (u.first + qi) * a.ot + head * a.oh + 64 * c + lane, l == 0.f ? 0.f : x[c] / l);
    if (a.lse && lane == 0) a.lse[(u.first + qi) * a.heads + head] = l == 0.f ? -kKvInf : (m + __builtin_amdgcn_logf(l)) / kLog2e;
}

// The form of a call: rows of a wave in tiles of 16, and whether waves have rows of their own.
struct KvForm { int nt; bool rows; };

template <int DP, int GROUP, int NT, int PARTS, bool ROWS>
void kv_attn_start(const KvAttn& a, const KvPlan& plan, dim3 grid, hipStream_t s)
{
    hipLaunchKernelGGL((kv_attn_kernel<DP, GROUP, NT, PARTS, ROWS>), grid, dim3(256), 0, s, a, plan);
}

// Query tiles of a wave in the ROWS form: what the registers hold.
template <int DP, int PARTS> constexpr int kRowsNT = DP <= 128 ? (PARTS == 1 ? 2 : 1) : 1;

template <int DP> void kv_attn_width(const KvAttn& a, const KvPlan& plan, KvForm form, dim3 grid, hipStream_t s)
{
    kv_dispatch_group<DP>(a.group, [&](auto shape) {
        constexpr int G = decltype(shape)::GROUP;
        if (a.dtype == QE_F32) {
            if (form.rows) kv_attn_start<DP, G, kRowsNT<DP, 2>, 2, true>(a, plan, grid, s);
            else kv_attn_start<DP, G, 1, 2, false>(a, plan, grid, s);
        } else {
            if (form.rows) kv_attn_start<DP, G, kRowsNT<DP, 1>, 1, true>(a, plan, grid, s);
            else if (form.nt == 1) kv_attn_start<DP, G, 1, 1, false>(a, plan, grid, s);
            else kv_attn_start<DP, G, 2, 1, false>(a, plan, grid, s);
        }
    });
    if (plan.nsplit > 1) {
        const int64_t rows = (int64_t)a.batch * a.c.heads * plan.row_tiles * plan.rows;
        hipLaunchKernelGGL(kv_join_kernel<DP>, grid_xy(cdiv(rows, 4), 256), dim3(256), 0, s, a, plan);
    }
}

}  // namespace qe
