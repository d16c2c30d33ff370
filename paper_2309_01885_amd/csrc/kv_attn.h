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
//
// What bounds it: one new token of a sequence reads the cache once (dim + 8 groups bytes a token and
// key head); 2 x 262144 tokens of 8 heads of 128 take 112 us, 5.1 TB/s of reads, where a plain copy moves
// 4.9 (read and written).  Chunks wait for vector instructions most: 2048 queries over 16384 tokens of 32
// heads take 671 to 695 us, 741 to 768 TFLOP/s, with the vector units 62 % busy, the matrix cores 30 %,
// and no more than two waves a SIMD to overlap them.
// (A matrix product of fp16 numbers in memory reaches 1140 TFLOP/s here, and has neither an
// exponential a score nor codes to convert.)
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
constexpr float kKvUnit = 120.f, kKvLag = 60.f;   // of KvSums: the largest exponent of unit; what a maximum may lag behind

// How a call is cut into workgroups.  A unit is a tile of `rows` query rows (row = query *
// heads per key head + head in the group) of one sequence and key head; each unit has
// nsplit workgroups along the tokens, whose results a second launch joins.
struct KvPlan {
    int64_t row_tiles, units;               // units of a sequence and key head; of the call
    int nsplit, rows, rows_log2, per;       // per: heads of a key head
    float* part;                            // nsplit > 1: (unit, split, row, DP) sums divided by the split's mass
    float* stat;                            // (unit, split, row, 2): a mass f 2^(e + kKvJoinLog2) as e and f
};

// What a workgroup works on; the join recomputes it.
struct KvUnit {
    int64_t first, pos0;                    // first row of Q, position of query 0
    int b, kvh, per, tile_row, rows;        // per: heads of a key head; the unit's first row; rows of the sequence
    int len, rec0, rec1, splits;            // cached tokens; records that some row sees; splits in use

    // records [from(s), from(s + 1)) are split s's
    __device__ int from(int split) const
    {
        const uint32_t n = rec1 - rec0, q = n / (uint32_t)splits;
        return rec0 + (int)(q * split + min((uint32_t)split, n - q * splits));
    }
};

// Records a split has at least (a workgroup's waves take them in turn), and from which splitting gains
// more than the join costs (a record takes a wave about 1.3 us, the join with its launch 6 us).
constexpr int kKvMinRecords = 4, kKvSplitFrom = 20;
constexpr int kKvFewSplits = 8;
// Masses reach the join as f 2^(e + kKvJoinLog2), f in [2^-12, 2^-11): neither the sum of as many of them as there
// are splits (kFill doubled at most) nor that of the parts that they weigh overflows.
constexpr int kKvJoinLog2 = 12;

// A value that is the same for the whole workgroup and not written by the kernel: a scalar load.
__device__ inline int kv_scalar(const int32_t* p) { return *(const __attribute__((address_space(4))) int32_t*)p; }

// (Divisions are of 32 bits: units and the rows of a sequence are fewer than 2^31, checked on the
// host, and one of 64 bits takes 130 instructions.)
__device__ inline KvUnit kv_unit(const KvAttn& a, const KvPlan& p, uint32_t unit, bool report)
{
    KvUnit u;
    const uint32_t bh = unit / (uint32_t)p.row_tiles, tile = unit - bh * (uint32_t)p.row_tiles;
    u.b = (int)(bh / (uint32_t)a.c.heads);
    u.kvh = (int)(bh - (uint32_t)u.b * a.c.heads);
    u.per = p.per;
    bool bad = false;
    u.first = u.b * a.max_q;
    int64_t nq = a.max_q;
    if (a.q_start) {
        u.first = kv_scalar(a.q_start + u.b);
        nq = (int64_t)kv_scalar(a.q_start + u.b + 1) - u.first;
        bad = u.first < 0 || nq < 0 || nq > a.max_q || u.first + nq > a.total;
        u.first = u.first < 0 ? 0 : u.first;
        nq = max((int64_t)0, min(min(nq, a.max_q), a.total - u.first));
    }
    const int64_t room = a.width * (int64_t)a.c.per * kKvTok;
    int64_t len = kv_scalar(a.lengths + u.b);
    bad = bad || len < 0 || len > room;
    len = len < 0 ? 0 : min(len, room);
    if (bad && report && tile == 0 && u.kvh == 0) set_status(a.status, QE_ERR_ARG);
    u.len = (int)len;
    u.pos0 = len - nq;
    u.rows = (int)(nq * u.per);
    const int64_t r0 = (int64_t)tile * p.rows;
    u.tile_row = (int)min(r0, (int64_t)u.rows);
    // the unit's queries i0 .. i1
    const uint32_t i0 = (uint32_t)u.tile_row / (uint32_t)u.per;
    const int64_t i1 = min(nq, (int64_t)(((uint32_t)u.tile_row + p.rows + u.per - 1) / (uint32_t)u.per)) - 1;
    int64_t end = a.causal ? min(len, u.pos0 + i1 + 1) : len;
    const int64_t begin = a.window ? max((int64_t)0, u.pos0 + i0 - a.window + 1) : 0;
    if (r0 >= u.rows || end < begin) end = begin;
    u.rec0 = (int)(begin / kKvTok);
    u.rec1 = end > begin ? (int)((end + kKvTok - 1) / kKvTok) : u.rec0;
    const int records = u.rec1 - u.rec0;
    u.splits = records < kKvSplitFrom ? 1 : min(p.nsplit, records / kKvMinRecords);
    return u;
}

// Eight channels of out.  (Fp32 calls are the kernels with PARTS == 2.)
template <int PARTS> __device__ inline void kv_out8(const KvAttn& a, int64_t at, const float* x)
{
    if constexpr (PARTS == 2) kv_store8(static_cast<float*>(a.out) + at, a.vec_o, x);
    else if (a.dtype == QE_F16) kv_store8(static_cast<_Float16*>(a.out) + at, a.vec_o, x);
    else kv_store8(static_cast<__bf16*>(a.out) + at, a.vec_o, x);
}
__device__ inline void kv_out(const KvAttn& a, int64_t at, float x)
{
    if (a.dtype == QE_F32) static_cast<float*>(a.out)[at] = x;
    else if (a.dtype == QE_F16) static_cast<_Float16*>(a.out)[at] = (_Float16)x;
    else static_cast<__bf16*>(a.out)[at] = (__bf16)x;
}
// Constants in registers: an instruction takes no two literals, and "and, or" is one instruction
// with both of them in registers.
struct KvBits {
    uint32_t low = 0x000F000Fu, high = 0x00F000F0u, n = 0x64006400u, z = 0xE400E400u;
    __device__ KvBits()
    {
        asm("" : "+s"(low), "+s"(high));
        asm("" : "+v"(n), "+v"(z));
    }
};
// A pair of codes of a word (nibbles k and k + 4 of w >> 4 k') less their zero points: mask: low, or
// high for the codes in bits 4-7, times 16.  minus: a pair of -(1024 + z), or of -(1024 + 16 z).
__device__ inline uint32_t kv_code_pair(uint32_t w, uint32_t mask, uint32_t minus, const KvBits& bits)
{
    const uint32_t n = (w & mask) | bits.n;
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

// Over the four lanes of a query, 16 apart.  The swap instructions exchange rows of 16 (or halves of 32) lanes of two
// copies of x, after which the two hold a lane's own value and its partner's.  (With exchanges through
// LDS one token over 500 of 8 key heads took 9.4 us, with these 9.1.)
__device__ inline float kv_swap(float x, int by, float& other)
{
    const uint32_t u = __float_as_uint(x);
    const auto r = by == 16 ? __builtin_amdgcn_permlane16_swap(u, u, false, false) : __builtin_amdgcn_permlane32_swap(u, u, false, false);
    other = __uint_as_float(r[1]);
    return __uint_as_float(r[0]);
}
__device__ inline float kv_max4(float x)
{
    float y;
    x = kv_swap(x, 16, y);
    x = fmaxf(x, y);
    x = kv_swap(x, 32, y);
    return fmaxf(x, y);
}
__device__ inline float kv_sum4(float x)
{
    float y;
    x = kv_swap(x, 16, y);
    x += y;
    x = kv_swap(x, 32, y);
    return x + y;
}

// Channels a lane's words are made of.  A key word is an octet: row `token`, octet 4 c + j.  A
// value word is a unit of 4 channels of two tokens; a unit tile is 16 units (one channel
// class of theirs is a product's 16 rows), with groups of 32 it is 8 (two classes are).
template <int DP, int GROUP> struct KvTiles {
    using R = KvRec<DP, GROUP>;
    static constexpr int NC = R::NC, NG = R::NG;
    static constexpr int CPG = GROUP / 32;                       // 32-channel products of a key group
    static constexpr bool kHalf = GROUP == 32;
    static constexpr int UT = kHalf ? DP / 32 : (DP + 63) / 64;  // unit tiles
    static constexpr int CL = kHalf ? 2 : 4;                     // classes of a unit tile
    // token (of the record) whose key row is row i of half h
    __device__ static int key_token(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }
    __device__ static int unit(int t, int i)
    {
        const int u = kHalf ? 8 * t + (i & 7) : 16 * t + i;
        return DP % 64 == 0 || kHalf ? u : min(u, DP / 4 - 1);   // (rows past the last unit give channels past DP)
    }
    static constexpr int group_of(int t) { return (kHalf ? 32 * t : 64 * t) / GROUP; }
    // row r of unit tile t, class k is channel 64 t + 4 r + k; with groups of 32, 32 t + 4 (r & 7) + k + 2 (r >> 3)
    static constexpr int kWidth = DP;
    static constexpr bool kWhole = DP % 64 == 0 || kHalf;        // every one of them is below DP
};

// The zero points of a key row as the pairs kv_code_pair takes, and of two tokens' value words.
__device__ inline void kv_key_zero(uint32_t word, uint32_t& lo, uint32_t& hi, const KvBits& bits)
{
    const uint32_t z = word & 15u, z2 = z << 16 | z;
    lo = z2 | bits.z;
    hi = z2 << 4 | bits.z;
}
__device__ inline void kv_value_zero(uint32_t w0, uint32_t w1, uint32_t& lo, uint32_t& hi, const KvBits& bits)
{
    const uint32_t w = __builtin_amdgcn_perm(w1, w0, 0x05040100u);
    lo = (w & bits.low) | bits.z;
    hi = ((w << 4) & bits.high) | bits.z;
}
__device__ inline f16x8 kv_key_frag(uint32_t w, uint32_t lo, uint32_t hi, const KvBits& bits)
{
    const uint32_t w8 = w >> 8;
    return kv_frag(kv_code_pair(w, bits.low, lo, bits), kv_code_pair(w, bits.high, hi, bits),
                   kv_code_pair(w8, bits.low, lo, bits), kv_code_pair(w8, bits.high, hi, bits));
}
// The largest; NaNs are passed over.
__device__ inline float kv_max8(const float (&x)[8])
{
    return fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(x[0], x[1]), x[2]), x[3]), x[4]), x[5]), x[6]), x[7]);
}

// A wave's query rows, 16 a tile, and what they see.
template <int NC, int NT, int PARTS> struct KvRows {
    f16x8 q[PARTS][NT][NC];
    float c[NT], slope[NT];                 // score of a product: c s + slope (t - pos), in powers of two
    int lo[NT], hi[NT];                     // the tokens that the lane's row sees
    int all_lo, all_hi;                     // that every row of the wave sees

    // A row is scaled by 2^e to a largest element in [2^14, 2^15) and rounded to fp16.
    __device__ void load(const KvAttn& a, const KvUnit& u, int row0)
    {
        const int i = threadIdx.x & 15, j = (threadIdx.x & 63) >> 4;
        // all loads first (each with its conversion would wait for the one before)
        constexpr int E = PARTS == 2 ? 4 : 2;                // bytes of a channel
        u32x4 raw[NT][NC][E / 2];
        int qi[NT], head[NT];
        const char* at[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int row = min(row0 + 16 * n + i, u.rows - 1);
            qi[n] = row / u.per;
            head[n] = u.kvh * u.per + row - qi[n] * u.per;
            at[n] = static_cast<const char*>(a.q) + ((u.first + qi[n]) * a.qt + head[n] * a.qh) * E;
        }
        if (a.vec_q) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int k = 0; k < NC; ++k)
#pragma unroll
                    for (int y = 0; y < E / 2; ++y)
                        raw[n][k][y] = reinterpret_cast<const u32x4*>(at[n] + min(8 * (4 * k + j), a.c.dim - 8) * E)[y];
        } else {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int k = 0; k < NC; ++k)
#pragma unroll
                    for (int y = 0; y < E / 2; ++y)
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const char* from = at[n] + min(8 * (4 * k + j), a.c.dim - 8) * E + 16 * y + 4 * w;
                            if constexpr (PARTS == 2) raw[n][k][y][w] = *reinterpret_cast<const uint32_t*>(from);
                            else raw[n][k][y][w] = *reinterpret_cast<const uint16_t*>(from) | (uint32_t)*reinterpret_cast<const uint16_t*>(from + 2) << 16;
                        }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const bool have = row0 + 16 * n + i < u.rows;
            float x[NC][8], top = 0.f;
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                const uint32_t in = have && 8 * (4 * k + j) < a.c.dim ? ~0u : 0u;
#pragma unroll
                for (int y = 0; y < E / 2; ++y)
#pragma unroll
                    for (int w = 0; w < 4; ++w) raw[n][k][y][w] &= in;
            }
            auto take = [&](auto channel) {
#pragma unroll
                for (int k = 0; k < NC; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        x[k][e] = channel(k, e);
                        top = fmaxf(top, fabsf(x[k][e]));
                    }
            };
            if constexpr (PARTS == 2) take([&](int k, int e) { return __uint_as_float(raw[n][k][e / 4][e % 4]); });
            else if (a.dtype == QE_BF16) take([&](int k, int e) { return __uint_as_float(e & 1 ? raw[n][k][0][e / 2] & 0xffff0000u : raw[n][k][0][e / 2] << 16); });
            else take([&](int k, int e) { return (float)__builtin_bit_cast(f16x2, (uint32_t)raw[n][k][0][e / 2])[e & 1]; });
            top = kv_max4(top);
            // (a row of zeros, NaN or infinities keeps its values)
            const int e2 = top > 0.f && top <= 3.402823466e38f ? max(-100, min(100, 141 - (int)(__float_as_uint(top) >> 23))) : 0;
            const float mul = __uint_as_float((uint32_t)(127 + e2) << 23) * (a.scale < 0.f ? -1.f : 1.f);
            c[n] = fmaxf(fabsf(a.scale) * kLog2e * __uint_as_float((uint32_t)(127 - e2) << 23), 1e-37f);   // (0 times -inf)
            slope[n] = a.slopes && have ? a.slopes[head[n]] * kLog2e : 0.f;
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                uint32_t h[4], m[4];
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    // (channels 1, 3, 5, 7 meet 16 times their codes)
                    const float f = p & 1 ? 0.0625f * mul : mul, x0 = x[k][p] * f, x1 = x[k][p + 4] * f;
                    const f16x2 hv = {(_Float16)x0, (_Float16)x1};
                    h[p] = __builtin_bit_cast(uint32_t, hv);
                    if constexpr (PARTS == 2) m[p] = kv_pack(x0 - (float)hv[0], x1 - (float)hv[1]);
                }
                q[0][n][k] = kv_frag(h[0], h[1], h[2], h[3]);
                if constexpr (PARTS == 2) q[1][n][k] = kv_frag(m[0], m[1], m[2], m[3]);
            }
            const int64_t pos = u.pos0 + qi[n];
            hi[n] = have && a.causal ? (int)max((int64_t)0, pos + 1) : u.len;
            lo[n] = have && a.window ? (int)max((int64_t)0, pos - a.window + 1) : 0;
        }
        all_lo = 0;
        all_hi = u.len;
        if (a.causal) {
            // the first and the last row bound the others
            const int64_t p0 = u.pos0 + row0 / u.per, p1 = u.pos0 + (min(u.rows, row0 + 16 * NT) - 1) / u.per;
            all_hi = (int)max((int64_t)0, p0 + 1);
            if (a.window) all_lo = (int)max((int64_t)0, p1 - a.window + 1);
        }
    }
    __device__ bool masked(int t0) const { return t0 > all_hi - kKvTok || t0 < all_lo; }
};

// The running softmax and the weighted sums of a wave's rows, o[t][k][n][e]: class k, row 4 j + e of tile t.
// A probability is p = 2^(score - top), top an integer that the row's scores pass by kKvLag at most.  The fp16
// weights of a row and channel group are p s' 2^e (unit: 2^e).  e is the row's and the group's own, so that
// what other rows see and other channels hold takes no bits from them: when it is set, the largest product so
// far lies in [2^10, 2^12); it is lowered where a product could pass fp16's range.  When top moves by d, e follows by d
// and the sums stay as they are, up to e = kKvUnit (value scales below 2^-109 lose bits); what p times unit can be is
// finite, so that it is 0 for a token that the row does not see, whatever its scale.  Factors are powers of two.
// (One exponent for a wave, from the value scales of all tokens read, was faster: 648 against 682 us, 2048
// queries over 16384 tokens of 32 heads of 128, 32 against 37 with five fp32 chunks and slopes.  But a row lost
// its bits to a large value that it does not see: 3e-5 of an fp32 result to one 2^20 times the others, all
// of it from 2^37 times on.)
template <class T, int NT> struct KvSums {
    static constexpr int UT = T::UT, CL = T::CL, NG = T::NG;
    f32x4 o[UT][CL][NT];
    float top[NT], mass[NT], unit[NT][NG];

    __device__ void clear()
    {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int t = 0; t < UT; ++t)
#pragma unroll
                for (int k = 0; k < CL; ++k) o[t][k][n] = f32x4{0.f, 0.f, 0.f, 0.f};
            top[n] = -kKvInf;
            mass[n] = 0.f;
#pragma unroll
            for (int g = 0; g < NG; ++g) unit[n][g] = 1.f;
        }
    }
    __device__ static float exponent(float x) { return (float)((int)(__float_as_uint(x) >> 23) - 127); }
    // Moves the maxima and the units where a row's maximum (at: a lane's, in powers of two) or a weight (big: a lane's
    // largest value scales, seen or not: the products themselves are compared only then) is out of range.
    // s c: the scores.
    template <int KR, class F> __device__ void move(const float (&at)[NT], const float (&c)[NT], const float (&big)[NG], const float (&s)[KR][NT][8], F scales)
    {
        bool out = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float p = __builtin_amdgcn_exp2f(at[n] - top[n]);          // (NaN: nothing seen so far, nor here)
            out = out || at[n] > top[n] + kKvLag;
#pragma unroll
            for (int g = 0; g < NG; ++g) out = out || p * unit[n][g] * big[g] > 65000.f;
        }
        if (!__any(out)) return;
        float y[NT][NG];                                                     // the largest products of the records, 127 more than their logarithms
#pragma unroll
        for (int g = 0; g < NG; ++g) {
#pragma unroll
            for (int n = 0; n < NT; ++n) y[n][g] = -kKvInf;
#pragma unroll
            for (int r = 0; r < KR; ++r) {
                float sv[8];
                scales(r, g, sv);
#pragma unroll
                for (int x = 0; x < 8; ++x)
#pragma unroll
                    for (int n = 0; n < NT; ++n)                             // (a number's bits are its logarithm, to 0.09, plus 127)
                        y[n][g] = fmaxf(y[n][g], fmaf(s[r][n][x], c[n], (float)(int)__float_as_uint(sv[x]) * 0x1p-23f));
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float m = __builtin_ceilf(kv_max4(fmaxf(top[n], at[n])));
            const bool first = top[n] == -kKvInf;
            const float d = m == top[n] ? 0.f : m - top[n];
            mass[n] *= __builtin_amdgcn_exp2f(-d);
            top[n] = m;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const float keep = first ? kKvUnit : exponent(unit[n][g]) + d;
                const float e = fminf(fminf(keep, kKvUnit), __builtin_ceilf(137.f - (kv_max4(y[n][g]) - m)));
                const float f = first ? 1.f : __builtin_amdgcn_exp2f(e - keep);
                unit[n][g] = __uint_as_float((uint32_t)((int)fmaxf(e, -kKvUnit) + 127) << 23);
#pragma unroll
                for (int t = 0; t < UT; ++t) {
                    if (T::group_of(t) != g) continue;
#pragma unroll
                    for (int k = 0; k < CL; ++k)
#pragma unroll
                        for (int x = 0; x < 4; ++x) o[t][k][n][x] *= f;
                }
            }
        }
    }
    // Where some row does not see a token (its score s is -inf), a NaN scale of that token would meet a
    // probability of 0.  Such scales are to be taken as 0 (the result), and the sums of the rows and
    // groups that do see one become NaN here.
    template <int KR, class F> __device__ bool meet_nans(const float (&s)[KR][NT][8], F scales)
    {
        float sum = 0.f;
#pragma unroll
        for (int y = 0; y < KR; ++y)
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                float sv[8];
                scales(y, g, sv);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += sv[e];
            }
        if (!__any(sum != sum)) return false;
#pragma unroll 1
        for (int g = 0; g < NG; ++g) {
            float met[NT] = {};
#pragma unroll
            for (int y = 0; y < KR; ++y) {
                float sv[8];
                scales(y, g, sv);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 8; ++e) met[n] = s[y][n][e] != -kKvInf && sv[e] != sv[e] ? 1.f : met[n];
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float add = kv_max4(met[n]) == 0.f ? 0.f : __builtin_nanf("");
#pragma unroll
                for (int t = 0; t < UT; ++t)
#pragma unroll
                    for (int k = 0; k < CL; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[t][k][n][e] += T::group_of(t) == g ? add : 0.f;
            }
        }
        return true;
    }
    // s: the products times their key scales, of KR records that start at tokens t0; on return the probabilities
    // (0 where the row does not see the token).  masked: some row does not see all of them.  scales(y, g, x) gives
    // the lane's value scales; clear() is called if NaNs among them are to be taken as 0.
    template <int KR, int NC, int PARTS, class F, class C>
    __device__ void weigh(float (&s)[KR][NT][8], const KvRows<NC, NT, PARTS>& r, bool slopes, const int (&t0)[KR], bool masked, F scales, C clear)
    {
        float big[NG];
#pragma unroll
        for (int y = 0; y < KR; ++y)
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                float sv[8];
                scales(y, g, sv);
                big[g] = y == 0 ? kv_max8(sv) : fmaxf(big[g], kv_max8(sv));
            }
        float at[NT], c[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            c[n] = r.c[n];
            at[n] = kv_max8(s[0][n]);
#pragma unroll
            for (int y = 1; y < KR; ++y) at[n] = fmaxf(at[n], kv_max8(s[y][n]));
            at[n] *= c[n];
        }
        if (masked || slopes) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                at[n] = -kKvInf;
#pragma unroll
                for (int y = 0; y < KR; ++y) {
                    const int t = t0[y] + 8 * ((threadIdx.x & 63) >> 4);
                    const float base = r.slope[n] * (float)(t - (r.hi[n] - 1));
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        s[y][n][e] = fmaf(s[y][n][e], c[n], fmaf(r.slope[n], (float)e, base));
                        s[y][n][e] = t + e >= r.lo[n] && t + e < r.hi[n] ? s[y][n][e] : -kKvInf;
                    }
                    at[n] = fmaxf(at[n], kv_max8(s[y][n]));
                }
                c[n] = 1.f;
            }
            if (masked && meet_nans<KR>(s, scales)) clear();
        }
        move<KR>(at, c, big, s, scales);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float off = top[n] == -kKvInf ? 0.f : -top[n];            // (nothing seen so far: every s is -inf)
#pragma unroll
            for (int y = 0; y < KR; ++y) {
                float (&x)[8] = s[y][n];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(x[e], c[n], off));
                mass[n] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
            }
        }
    }
    // The products' fp16 weights p s' of a group.
    template <int PARTS> __device__ void weights(const float (&s)[NT][8], int g, const float (&sv)[8], f16x8 (&pr)[PARTS][NT]) const
    {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            uint32_t h[4], m[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                float x0 = s[n][2 * p] * unit[n][g] * sv[2 * p], x1 = s[n][2 * p + 1] * unit[n][g] * sv[2 * p + 1];
                // (one rounded product for both parts: fused into the first part's conversion only, it made
                // the parts miss each other by a step of fp16 once in some thousand)
                if (PARTS == 2) asm("" : "+v"(x0), "+v"(x1));
                h[p] = kv_pack(x0, x1);
                if constexpr (PARTS == 2) {
                    const f16x2 hv = __builtin_bit_cast(f16x2, h[p]);
                    m[p] = kv_pack(x0 - (float)hv[0], x1 - (float)hv[1]);
                }
            }
            pr[0][n] = kv_frag(h[0], h[1], h[2], h[3]);
            if constexpr (PARTS == 2) pr[1][n] = kv_frag(m[0], m[1], m[2], m[3]);
        }
    }
    // Keeps every sum in one place from record to record (the compiler copied half of them otherwise).
    __device__ void pin()
    {
#pragma unroll
        for (int t = 0; t < UT; ++t)
#pragma unroll
            for (int k = 0; k < CL; ++k)
#pragma unroll
                for (int n = 0; n < NT; ++n) asm("" : "+v"(o[t][k][n]));
    }
    // Calls f with the channel and the values, times `by` (relative to top), of each octet of channels of tile n that ends
    // up in this lane.
    template <class F> __device__ void octets(int n, float moved, float by, F f)
    {
        const int j = (threadIdx.x & 63) >> 4;
        float to[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) to[g] = __builtin_amdgcn_exp2f(moved - exponent(unit[n][g])) * by;
#pragma unroll
        for (int t = 0; t < UT; ++t) {
            const float of = to[T::group_of(t)];
            float x[8];
            if constexpr (T::kHalf) {
                // rows 0 .. 7 (lanes j < 2) hold classes 0 and 1 of a unit, rows 8 .. 15 classes 2 and 3
                const bool up = j >= 2;
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float own = up ? o[t][k][n][2 + e] : o[t][k][n][e], give = up ? o[t][k][n][e] : o[t][k][n][2 + e];
                        const float got = __shfl_xor(give, 32);
                        x[4 * e + k] = (up ? got : own) * of;
                        x[4 * e + 2 + k] = (up ? own : got) * of;
                    }
                f(32 * t + 16 * (j & 1) + (up ? 8 : 0), x);
            } else {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[4 * e + k] = o[t][k][n][2 * y + e] * of;
                    const int d = 64 * t + 16 * j + 8 * y;
                    if (T::kWhole || d < T::kWidth) f(d, x);
                }
            }
        }
    }
    // after the last record: plain sums (odd classes were 16 times as large), the rows' masses
    __device__ void finish()
    {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            mass[n] = kv_sum4(mass[n]);
#pragma unroll
            for (int t = 0; t < UT; ++t)
#pragma unroll
                for (int k = 1; k < CL; k += 2)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[t][k][n][e] *= 0.0625f;
        }
    }
};

// A lane's value scales of KR records.  Up to two of a lane's sets of eight are kept in registers; more are read from LDS
// where they are used (held, they were 64 registers with eight groups).
template <int KR, int NG> struct KvScales {
    static constexpr bool kKept = KR * NG <= 2;
    float s[kKept ? KR : 1][kKept ? NG : 1][8];
    const float* at[kKept ? 1 : KR];                             // group 0's; the others' are `step` floats apart
    int step;
    bool nans;

    __device__ static void read(const float* p, float (&x)[8])
    {
        const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < 4 ? a[e] : b[e - 4];
    }
    template <class F> __device__ void load(F from)
    {
        nans = false;
        if constexpr (kKept) {
#pragma unroll
            for (int y = 0; y < KR; ++y)
#pragma unroll
                for (int g = 0; g < NG; ++g) read(from(y, g), s[y][g]);
        } else {
            step = (int)(from(0, 1) - from(0, 0));
#pragma unroll
            for (int y = 0; y < KR; ++y) at[y] = from(y, 0);
        }
    }
    __device__ void get(int y, int g, float (&x)[8]) const
    {
        if constexpr (kKept) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = NG == 1 ? s[y][0][e] : g == 0 ? s[y][0][e] : s[y][NG - 1][e];
        } else {
            read(at[y] + g * step, x);
            if (nans) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = x[e] != x[e] ? 0.f : x[e];
            }
        }
    }
    __device__ void clear()
    {
        nans = true;
        if constexpr (kKept) {
#pragma unroll
            for (int y = 0; y < KR; ++y)
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[y][g][e] = s[y][g][e] != s[y][g][e] ? 0.f : s[y][g][e];
        }
    }
};

__device__ inline float kv_lse(float top, float mass) { return mass == 0.f ? -kKvInf : (top + __builtin_amdgcn_logf(mass)) / kLog2e; }

// ---------------------------------------------------------------- few rows
// Four waves share 16 NT rows (the matrix instruction's tile: a single token's heads of a key head are rows of
// it) and take the unit's records in turn, so that a record is read by one wave and one wave's loads
// wait while the others work; the waves' sums meet in LDS, the splits' in a second launch.  Two tiles
// where rows and tokens are many: a record's conversion, half of the vector instructions, is shared.
// 64 sequences of 2048 to 8192 tokens, 29 query heads on one of 64 channels, take 81 to 88 us with the join, from
// run to run, for 40 us of bytes at a copy's rate: the vector units are 60 % busy, the matrix cores
// 11 %, and the rest is waits of few waves.
//
// Workgroups of a CU that the registers are to allow.  Never one: beyond 256 registers the compiler
// keeps the sums in accumulation registers and was seen to read one back after the last matrix
// instruction of a loop without the wait that it needs.
constexpr int kv_few_occupancy(int dp, int group, int nt, int parts)
{
    if (dp == 64) return nt == 1 ? 4 : 3;
    if (dp <= 128 && nt == 1) return group == 128 && parts == 1 ? 4 : group >= 64 ? 3 : 2;
    return 2;
}

template <int DP, int GROUP, int NT, int PARTS>
__global__ __launch_bounds__(256, kv_few_occupancy(DP, GROUP, NT, PARTS)) void kv_few_kernel(KvAttn a, KvPlan plan)
{
    using R = KvRec<DP, GROUP>;
    using T = KvTiles<DP, GROUP>;
    constexpr int NC = T::NC, NG = T::NG, UT = T::UT, CL = T::CL;
    const uint32_t unit = blockIdx.x / (uint32_t)plan.nsplit;
    const int split = (int)(blockIdx.x - unit * plan.nsplit);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i = tid & 15, j = (tid & 63) >> 4;
    const KvUnit u = kv_unit(a, plan, unit, tid == 0 && split == 0);
    if (split >= u.splits || u.tile_row >= u.rows) return;
    const int r1 = u.from(split + 1);
    int r = u.from(split) + wave;

    // A record's codes, and a word of each group: a key's (lanes 0 .. 31) or a value's.  The keys' registers
    // are free once the scores are there and take the next record's keys; the values' likewise after
    // the weighted sum.  The words' scales and zero points reach the lanes that need them through the
    // wave's part of LDS.  (Read from memory by each of those lanes they took 18 registers a group and
    // 32 more instructions.)
    struct Words {
        float s[NG][64];                                         // scales
        uint16_t lo[NG][64], hi[NG][64];                         // -(1024 + z), -(1024 + 16 z) in fp16
    };
    constexpr int kRow = DP + 4;                                 // floats of a row (16-byte aligned, spread over the banks)
    __shared__ __align__(16) union {
        Words words[kKvWaves];
        float acc[kKvWaves][16 * NT][kRow];
    } shared;
    Words& held = shared.words[wave];
    const int lane = tid & 63;
    const KvBits bits;
    uint32_t k[2][NC], v[UT][4], word[NG];
    const int64_t pages = a.c.pages_count;
    const int32_t* table = a.table + u.b * a.width;
    const int per = (int)a.c.per;
    int pg = (uint32_t)r / (uint32_t)per, rem = r - pg * per;
    int id = r < r1 ? table[pg] : 0;
    const uint8_t* rec = a.c.pages;
    bool here = false;                                           // whether the record is there (else any other is read, and not used)
    // The address of record r, whose page number was read before; reads the one after it.
    auto find = [&](int r) {
        int page = __builtin_amdgcn_readfirstlane(id);
        here = page >= 0 && page < pages;
        if (!here) {
            set_status(a.status, QE_ERR_ARG);
            page = 0;
        }
        rec = a.c.pages + (((int64_t)page * a.c.heads + u.kvh) * per + rem) * R::kBytes;
        rem += kKvWaves;
        while (rem >= per) {
            rem -= per;
            ++pg;
        }
        if (r + kKvWaves < r1) id = table[pg];            // (in a vector register until it is needed: a wait for it now would be one for all loads)
    };
    auto keys = [&] {
#pragma unroll
        for (int g = 0; g < NG; ++g)
            word[g] = *reinterpret_cast<const uint32_t*>(rec + (uint32_t)((lane < 32 ? R::kKeyWords : R::kValWords) + g * (4 * kKvTok) + 4 * (lane & 31)));
#pragma unroll
        for (int h = 0; h < 2; ++h) kv_words<NC>(rec + (uint32_t)(T::key_token(i, h) * R::kKeyRow + j * (4 * NC)), k[h]);
    };
    auto values = [&] {
#pragma unroll
        for (int t = 0; t < UT; ++t) kv_words<4>(rec + (uint32_t)(R::kVal + T::unit(t, i) * (2 * kKvTok) + 16 * j), v[t]);
    };
    // (LDS serves a wave in order: what was read before is not overwritten.)
    auto hold = [&](int t0) {
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            // words past the sequence's end are anything: no value scale of theirs may meet a 0
            held.s[g][lane] = lane >= 32 && t0 > u.len - 1 - (lane & 31) ? 0.f : kv_scale(word[g]);
            held.lo[g][lane] = (uint16_t)(0xE400u | (word[g] & 15u));
            held.hi[g][lane] = (uint16_t)(0xE400u | (word[g] & 15u) << 4);
        }
        __builtin_amdgcn_wave_barrier();
    };
    auto first_token = [&](int r) { return here ? r * kKvTok : 0x7fffff00; };    // (of no record: past every sequence's end)
    if (r < r1) {
        find(r);
        keys();
        values();
    }
    KvRows<NC, NT, PARTS> rows;
    rows.load(a, u, u.tile_row);
    KvSums<T, NT> sums;
    sums.clear();

    int t0 = first_token(r);
    if (r < r1) hold(t0);
    for (; r < r1; r += kKvWaves) {
        const bool masked = rows.masked(t0), more = r + kKvWaves < r1;
        const int at[1] = {t0};
        float s[1][NT][8];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            f32x4 acc[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) acc[n][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t l = held.lo[g][T::key_token(i, h)], x = held.hi[g][T::key_token(i, h)], lo = l << 16 | l, hi = x << 16 | x;
#pragma unroll
                for (int c = g * T::CPG; c < (g + 1) * T::CPG && c < NC; ++c) {
                    const f16x8 f = kv_key_frag(k[h][c], lo, hi, bits);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) acc[n][h] = kv_mfma(f, rows.q[p][n][c], acc[n][h]);
                }
            }
            const f32x4 s0 = *reinterpret_cast<const f32x4*>(&held.s[g][8 * j]), s1 = *reinterpret_cast<const f32x4*>(&held.s[g][8 * j + 4]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float sc = e < 4 ? s0[e] : s1[e - 4];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float x = acc[n][e >> 2][e & 3];
                    s[0][n][e] = g == 0 ? sc * x : fmaf(sc, x, s[0][n][e]);
                }
            }
        }
        if (more) {
            find(r + kKvWaves);
            keys();
        }
        KvScales<1, NG> sv;
        sv.load([&](int, int g) { return &held.s[g][32 + 8 * j]; });
        sums.template weigh<1>(s, rows, a.slopes != nullptr, at, masked, [&](int y, int g, float (&x)[8]) { sv.get(y, g, x); }, [&] { sv.clear(); });
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            f16x8 pr[PARTS][NT];
            float x[8];
            sv.get(0, g, x);
            sums.template weights<PARTS>(s[0], g, x, pr);
            const u32x4 lo = *reinterpret_cast<const u32x4*>(&held.lo[g][32 + 8 * j]), hi = *reinterpret_cast<const u32x4*>(&held.hi[g][32 + 8 * j]);
#pragma unroll
            for (int t = 0; t < UT; ++t) {
                if (T::group_of(t) != g) continue;
                uint32_t w[4];
#pragma unroll
                for (int p = 0; p < 4; ++p) w[p] = T::kHalf ? v[t][p] >> (i & 8) : v[t][p];
#pragma unroll
                for (int c = 0; c < CL; ++c) {
                    uint32_t pair[4];
#pragma unroll
                    for (int p = 0; p < 4; ++p) pair[p] = kv_code_pair(w[p] >> (c >= 2 ? 8 : 0), c & 1 ? bits.high : bits.low, c & 1 ? hi[p] : lo[p], bits);
                    const f16x8 f = kv_frag(pair[0], pair[1], pair[2], pair[3]);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) sums.o[t][c][n] = kv_mfma(f, pr[p][n], sums.o[t][c][n]);
                }
            }
        }
        if (more) {
            values();
            t0 = first_token(r + kKvWaves);
            hold(t0);
        }
        sums.pin();
    }
    sums.finish();

    // every wave to the common maximum, divided by the common mass (sums of large values would pass the
    // largest number before it), then sums over the waves
    __shared__ float wtop[kKvWaves][16 * NT], wmass[kKvWaves][16 * NT], rtop[16 * NT], rmass[16 * NT];
    auto& acc = shared.acc;                                      // (written after a barrier that ends the use of the words)
#pragma unroll
    for (int n = 0; n < NT; ++n)
        if (j == 0) {
            wtop[wave][16 * n + i] = sums.top[n];
            wmass[wave][16 * n + i] = sums.mass[n];
        }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float m = -kKvInf, l = 0.f;
#pragma unroll
        for (int w = 0; w < kKvWaves; ++w) m = fmaxf(m, wtop[w][16 * n + i]);
#pragma unroll
        for (int w = 0; w < kKvWaves; ++w) {
            const float t = wtop[w][16 * n + i];
            l = fmaf(t == m ? 1.f : __builtin_amdgcn_exp2f(t - m), wmass[w][16 * n + i], l);
        }
        if (wave == 0 && j == 0) {
            rtop[16 * n + i] = m;
            rmass[16 * n + i] = l;
        }
        sums.octets(n, m == sums.top[n] ? 0.f : sums.top[n] - m, l == 0.f ? 0.f : 1.f / l, [&](int d, const float* x) {
#pragma unroll
            for (int y = 0; y < 8; y += 4) *reinterpret_cast<f32x4*>(&acc[wave][16 * n + i][d + y]) = f32x4{x[y], x[y + 1], x[y + 2], x[y + 3]};
        });
    }
    __syncthreads();
    for (int x = tid; x < 16 * NT * (DP / 8); x += 256) {
        const int rr = x / (DP / 8), d = 8 * (x - rr * (DP / 8)), row = u.tile_row + rr;
        if (row >= u.rows) break;
        f32x4 sum[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const f32x4 s0 = *reinterpret_cast<const f32x4*>(&acc[0][rr][d + 4 * y]), s1 = *reinterpret_cast<const f32x4*>(&acc[1][rr][d + 4 * y]);
            const f32x4 s2 = *reinterpret_cast<const f32x4*>(&acc[2][rr][d + 4 * y]), s3 = *reinterpret_cast<const f32x4*>(&acc[3][rr][d + 4 * y]);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[y][e] = (s0[e] + s1[e]) + (s2[e] + s3[e]);
        }
        const float m = rtop[rr], l = rmass[rr];
        if (u.splits > 1) {
            const int64_t slot = ((int64_t)unit * plan.nsplit + split) * plan.rows + rr;
#pragma unroll
            for (int y = 0; y < 2; ++y) *reinterpret_cast<f32x4*>(plan.part + slot * DP + d + 4 * y) = sum[y];
            if (d == 0) {
                const int e = (int)(__float_as_uint(l) >> 23) - 127;      // (of no mass: m is -inf)
                plan.stat[2 * slot] = m + (float)e;
                plan.stat[2 * slot + 1] = l * __uint_as_float((uint32_t)(127 - kKvJoinLog2 - e) << 23);
            }
        } else {
            const int qi = row / u.per, head = u.kvh * u.per + row - qi * u.per;
            float out[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] = sum[e >> 2][e & 3];
            if (d < a.c.dim) kv_out8<PARTS>(a, (u.first + qi) * a.ot + head * a.oh + d, out);
            if (a.lse && d == 0) a.lse[(u.first + qi) * a.heads + head] = kv_lse(m, l);
        }
    }
}

// ---------------------------------------------------------------- many rows
// Every wave has 16 NT rows of its own and the workgroup goes through the records together, KR at a
// time.  (Two records where LDS and registers hold them: one barrier for twice the work.)
// Codes are turned into fp16 once, by kKvWaves / KR waves a record, and reach the others
// through LDS as the products' operands (1 KB each, in lane order); while a stage is multiplied,
// the next is converted and the one after it is on its way.  A stage is straight code, also where a
// wave's rows see none of it and past the last record: conversion and first products, then
// exponentials and second products can overlap.  2048 queries over 16384 tokens of 32 heads of 128:
// 682 us; with every wave converting its own (the few-row form) 831.
constexpr int kv_stage_records(int dp) { return dp <= 128 ? 2 : 1; }

template <int DP, int GROUP, int NT, int PARTS>
__global__ __launch_bounds__(256, 2) void kv_many_kernel(KvAttn a, KvPlan plan)
{
    using R = KvRec<DP, GROUP>;
    using T = KvTiles<DP, GROUP>;
    constexpr int NC = T::NC, NG = T::NG, UT = T::UT, CL = T::CL;
    constexpr int KR = kv_stage_records(DP), W = kKvWaves / KR;  // records of a stage, waves that convert one
    // Records whose exponentials are taken together: all of a stage, where the registers hold them.  Two tiles
    // of two groups spill (2048 queries of 32 heads of 128 in groups of 64 over 8192 tokens: 547 us
    // together, 450 one by one; 96 channels over 4096 226 / 228; groups of 128 over 16384 696 / 737, 64
    // channels in groups of 64 over 8192 273 / 296).
    constexpr int KW = NG == 2 && NT == 2 && DP > 64 ? 1 : KR;
    constexpr int CW = KR == 2 ? NC : (NC + 1) / 2;              // key products a wave converts
    constexpr int VW = T::kHalf ? (UT + 1) / 2 : UT, VK = KR;    // unit tiles and classes
    constexpr int SW = KR == 2 ? (NG + 1) / 2 : (NG + 3) / 4;    // scales a lane converts
    constexpr int SG = SW * (KR == 2 ? 2 : 4);
    struct Stage {
        f16x8 k[KR][2][NC][64], v[KR][UT][CL][64];
        float ks[KR][SG][kKvTok], vs[KR][SG][kKvTok];            // (groups past NG: what lanes without a group write)
        int at[KR];                                              // the records' first tokens
    };
    __shared__ Stage stage[2];
    // workgroups of an XCD (every eighth) get a contiguous stretch of units: rows of the same keys
    // share its L2
    const uint32_t wg = blockIdx.x, q8 = gridDim.x / 8, r8 = gridDim.x % 8, x8 = wg & 7;
    const uint32_t unit = x8 * q8 + min(x8, r8) + (wg >> 3);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int i = tid & 15, j = lane >> 4;
    const KvUnit u = kv_unit(a, plan, unit, tid == 0);
    if (u.tile_row >= u.rows) return;
    const int r0 = u.rec0, r1 = u.rec1;
    const int row0 = u.tile_row + wave * (16 * NT);

    // what the wave converts: of record `part` of a stage, key half kh from channel block kc on, value
    // classes vk .. of the unit tiles vt, vt + 2, .. (groups of 32) or all
    const int part = wave / W, q = wave % W;
    const int kh = q & 1, kc = KR == 2 ? 0 : (q >> 1) * CW;
    const int vk = T::kHalf ? (KR == 2 ? 0 : q & 1) : KR == 2 ? 2 * (q & 1) : q;
    const int vt = T::kHalf ? (KR == 2 ? q & 1 : q >> 1) : 0;
    const KvBits bits;
    const uint32_t vmask = vk & 1 ? bits.high : bits.low, vshift = vk & 1 ? 4 : 0;   // (KR == 1)
    const int token = T::key_token(i, kh);
    constexpr int VG = T::kHalf ? VW : NG;                       // value groups whose zero points the wave needs
    uint32_t k[CW], kz[CW], v[VW][4], vw[VG][8], word[SW];

    const int64_t pages = a.c.pages_count;
    const int32_t* table = a.table + u.b * a.width;
    const int per = (int)a.c.per;
    // the wave's record of the next stage to be loaded, its page's place in the table and its place in the page
    int next = max(0, min(r0 + part, r1 - 1)), pg = (uint32_t)next / (uint32_t)per, rem = next - pg * per;
    int id = r0 < r1 ? table[pg] : 0;
    bool here = false;                                           // whether the record is there (else any other is read, and not used)
    // Starts the loads of the wave's share of the next stage, whose page number was read before, and reads
    // the one after it.  Past the last record it is loaded again.
    auto start = [&] {
        int page = __builtin_amdgcn_readfirstlane(id);
        here = page >= 0 && page < pages;
        if (!here) {
            if (lane == 0) set_status(a.status, QE_ERR_ARG);
            page = 0;
        }
        const uint8_t* rec = a.c.pages + (((int64_t)page * a.c.heads + u.kvh) * per + rem) * R::kBytes;
        kv_words<CW>(rec + (uint32_t)(token * R::kKeyRow + j * (4 * NC)) + 4 * kc, k);
#pragma unroll
        for (int x = 0; x < CW; ++x)
            kz[x] = *reinterpret_cast<const uint32_t*>(rec + (uint32_t)(R::kKeyWords + min((kc + x) / T::CPG, NG - 1) * (4 * kKvTok) + 4 * token));
#pragma unroll
        for (int x = 0; x < VG; ++x)
            kv_words<8>(rec + (uint32_t)(R::kValWords + (T::kHalf ? min(vt + 2 * x, NG - 1) : x) * (4 * kKvTok) + 32 * j), vw[x]);
#pragma unroll
        for (int x = 0; x < VW; ++x)
            kv_words<4>(rec + (uint32_t)(R::kVal + T::unit(T::kHalf ? min(vt + 2 * x, UT - 1) : x, i) * (2 * kKvTok) + 16 * j), v[x]);
#pragma unroll
        for (int x = 0; x < SW; ++x) {
            const bool key = KR == 2 ? kh == 0 : lane < 32;
            const int g = KR == 2 ? min((lane >> 5) + 2 * x, NG - 1) : min(q + 4 * x, NG - 1);
            word[x] = *reinterpret_cast<const uint32_t*>(rec + (uint32_t)((key ? R::kKeyWords : R::kValWords) + g * (4 * kKvTok) + 4 * (lane & 31)));
        }
        const int step = min(KR, r1 - 1 - next);
        next += step;
        rem += step;
        while (rem >= per) {
            rem -= per;
            ++pg;
        }
        id = table[pg];                                   // (in a vector register until it is needed: a wait for it now would be one for all loads)
    };
    // r: the first record of the stage
    auto convert = [&](Stage& st, int r) {
#pragma unroll
        for (int x = 0; x < CW; ++x) {
            if (KR == 1 && NC % 2 != 0 && kc + x >= NC) continue;
            uint32_t lo, hi;
            kv_key_zero(kz[x], lo, hi, bits);
            st.k[part][kh][kc + x][lane] = kv_key_frag(k[x], lo, hi, bits);
        }
#pragma unroll
        for (int x = 0; x < VW; ++x) {
            const int t = T::kHalf ? vt + 2 * x : x;
            if (T::kHalf && UT % 2 != 0 && t >= UT) continue;
            uint32_t f[VK][4];
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const uint32_t w0 = vw[T::kHalf ? x : T::group_of(x)][2 * p], w1 = vw[T::kHalf ? x : T::group_of(x)][2 * p + 1];
                const uint32_t w = v[x][p] >> (T::kHalf ? i & 8 : vk & 2 ? 8 : 0);
                if constexpr (KR == 2) {
                    uint32_t lo, hi;
                    kv_value_zero(w0, w1, lo, hi, bits);
                    f[0][p] = kv_code_pair(w, bits.low, lo, bits);
                    f[1][p] = kv_code_pair(w, bits.high, hi, bits);
                } else {
                    const uint32_t z = ((__builtin_amdgcn_perm(w1, w0, 0x05040100u) << vshift) & vmask) | bits.z;
                    f[0][p] = kv_code_pair(w, vmask, z, bits);
                }
            }
#pragma unroll
            for (int y = 0; y < VK; ++y) st.v[part][t][vk + y][lane] = kv_frag(f[y][0], f[y][1], f[y][2], f[y][3]);
        }
#pragma unroll
        for (int x = 0; x < SW; ++x) {
            const bool key = KR == 2 ? kh == 0 : lane < 32;
            const int g = KR == 2 ? (lane >> 5) + 2 * x : q + 4 * x;
            float sc = kv_scale(word[x]);
            // (words past the sequence's end, or of a record that is not there, are anything: no scale of theirs may meet a 0)
            sc = !key && (!here || (r + part) * kKvTok + (lane & 31) >= u.len) ? 0.f : sc;
            (key ? st.ks : st.vs)[part][g][lane & 31] = sc;
        }
        // (past the last record, or on a page that is not there: past every sequence's end)
        st.at[part] = here && r + part < r1 ? (r + part) * kKvTok : 0x7fffff00;
    };

    if (r0 < r1) start();
    KvRows<NC, NT, PARTS> rows;
    rows.load(a, u, min(row0, u.rows - 1));
    KvSums<T, NT> sums;
    sums.clear();
    if (r0 < r1) {
        convert(stage[0], r0);
        start();
    }
    __syncthreads();
    for (int r = r0, b = 0; r < r1; r += KR, b ^= 1) {
        convert(stage[b ^ 1], r + KR);
        const Stage& st = stage[b];
#pragma unroll
        for (int y0 = 0; y0 < KR; y0 += KW) {
            float s[KW][NT][8];
            int t0[KW];
            bool masked = false;
#pragma unroll
            for (int y = 0; y < KW; ++y) {
                t0[y] = __builtin_amdgcn_readfirstlane(st.at[y0 + y]);
                masked = masked || rows.masked(t0[y]);
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    f32x4 acc[NT][2];
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int h = 0; h < 2; ++h) acc[n][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = g * T::CPG; c < (g + 1) * T::CPG && c < NC; ++c)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const f16x8 f = st.k[y0 + y][h][c][lane];
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int p = 0; p < PARTS; ++p) acc[n][h] = kv_mfma(f, rows.q[p][n][c], acc[n][h]);
                        }
                    const f32x4 s0 = *reinterpret_cast<const f32x4*>(&st.ks[y0 + y][g][8 * j]), s1 = *reinterpret_cast<const f32x4*>(&st.ks[y0 + y][g][8 * j + 4]);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float sc = e < 4 ? s0[e] : s1[e - 4], x = acc[n][e >> 2][e & 3];
                            s[y][n][e] = g == 0 ? sc * x : fmaf(sc, x, s[y][n][e]);
                        }
                }
            }
            if (y0 == 0) start();
            KvScales<KW, NG> sv;
            sv.load([&](int y, int g) { return &st.vs[y0 + y][g][8 * j]; });
            sums.template weigh<KW>(s, rows, a.slopes != nullptr, t0, masked, [&](int y, int g, float (&x)[8]) { sv.get(y, g, x); }, [&] { sv.clear(); });
#pragma unroll
            for (int y = 0; y < KW; ++y)
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    f16x8 pr[PARTS][NT];
                    float x[8];
                    sv.get(y, g, x);
                    sums.template weights<PARTS>(s[y], g, x, pr);
#pragma unroll
                    for (int t = 0; t < UT; ++t) {
                        if (T::group_of(t) != g) continue;
#pragma unroll
                        for (int c = 0; c < CL; ++c) {
                            const f16x8 f = st.v[y0 + y][t][c][lane];
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int p = 0; p < PARTS; ++p) sums.o[t][c][n] = kv_mfma(f, pr[p][n], sums.o[t][c][n]);
                        }
                    }
                }
        }
        sums.pin();
        __syncthreads();
    }
    if (row0 >= u.rows) return;
    sums.finish();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = row0 + 16 * n + i, qi = row / u.per, head = u.kvh * u.per + row - qi * u.per;
        sums.octets(n, 0.f, sums.mass[n] == 0.f ? 0.f : 1.f / sums.mass[n], [&](int d, const float* x) {
            if (row < u.rows && d < a.c.dim) kv_out8<PARTS>(a, (u.first + qi) * a.ot + head * a.oh + d, x);
        });
        if (row < u.rows && j == 0 && a.lse) a.lse[(u.first + qi) * a.heads + head] = kv_lse(sums.top[n], sums.mass[n]);
    }
}

// Joins the splits of a row: one workgroup a row, whose waves take the splits in turn.
template <int DP> __global__ __launch_bounds__(256) void kv_join_kernel(KvAttn a, KvPlan plan)
{
    constexpr int C = (DP + 63) / 64;
    __shared__ float sum[kKvWaves][DP], mass[kKvWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t at = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (at >= plan.units * plan.rows) return;
    // (plan.rows is a power of two)
    const uint32_t unit = (uint32_t)(at >> plan.rows_log2);
    const int rr = (int)(at & (plan.rows - 1));
    const KvUnit u = kv_unit(a, plan, unit, false);
    const int row = u.tile_row + rr;
    if (u.splits <= 1 || row >= u.rows) return;
    const int64_t slot = (int64_t)unit * plan.nsplit * plan.rows + rr;
    float m = -kKvInf;
    for (int s = lane; s < u.splits; s += 64) m = fmaxf(m, plan.stat[2 * (slot + (int64_t)s * plan.rows)]);
#pragma unroll
    for (int x = 1; x < 64; x *= 2) m = fmaxf(m, __shfl_xor(m, x));
    float l = 0.f, x[C] = {};
#pragma unroll 4
    for (int s = wave; s < u.splits; s += kKvWaves) {
        const int64_t k = slot + (int64_t)s * plan.rows;
        const float t = plan.stat[2 * k], f = plan.stat[2 * k + 1] * (t == m ? 1.f : __builtin_amdgcn_exp2f(t - m));
        l += f;
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (DP % 64 == 0 || 64 * c + lane < DP) x[c] = fmaf(plan.part[k * DP + 64 * c + lane], f, x[c]);
    }
    const int qi = row / u.per, head = u.kvh * u.per + row - qi * u.per;
#pragma unroll
    for (int c = 0; c < C; ++c)
        if (DP % 64 == 0 || 64 * c + lane < DP) sum[wave][64 * c + lane] = x[c];
    if (lane == 0) mass[wave] = l;
    __syncthreads();
    l = (mass[0] + mass[1]) + (mass[2] + mass[3]);
    if (tid < a.c.dim)
        kv_out(a, (u.first + qi) * a.ot + head * a.oh + tid,
               l == 0.f ? 0.f : ((sum[0][tid] + sum[1][tid]) + (sum[2][tid] + sum[3][tid])) / l);
    if (a.lse && tid == 0) a.lse[(u.first + qi) * a.heads + head] = kv_lse(m + kKvJoinLog2, l);
}

// The same for few splits (kKvFewSplits at most) of many rows: one workgroup a unit, a thread 8 channels of a row,
// four splits on the way at a time.
template <int DP> __global__ __launch_bounds__(256) void kv_join_unit_kernel(KvAttn a, KvPlan plan)
{
    const uint32_t unit = blockIdx.x;
    const KvUnit u = kv_unit(a, plan, unit, false);
    if (u.splits <= 1) return;
    const float2* const stat = reinterpret_cast<const float2*>(plan.stat);
    for (int x = threadIdx.x; x < plan.rows * (DP / 8); x += 256) {
        const int rr = x / (DP / 8), d = 8 * (x - rr * (DP / 8)), row = u.tile_row + rr;
        if (row >= u.rows) break;
        const int64_t slot = (int64_t)unit * plan.nsplit * plan.rows + rr;
        auto place = [&](int s) { return slot + (int64_t)min(s, u.splits - 1) * plan.rows; };
        float2 st[kKvFewSplits];
        float m = -kKvInf, l = 0.f;
#pragma unroll
        for (int s = 0; s < kKvFewSplits; ++s) st[s] = stat[place(s)];
#pragma unroll
        for (int s = 0; s < kKvFewSplits; ++s) m = fmaxf(m, st[s].x);
        f32x4 sum[2] = {};
#pragma unroll
        for (int s0 = 0; s0 < kKvFewSplits; s0 += 4) {
            if (s0 >= u.splits) break;
            f32x4 part[4][2];
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int y = 0; y < 2; ++y) part[s][y] = *reinterpret_cast<const f32x4*>(plan.part + place(s0 + s) * DP + d + 4 * y);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if (s0 + s >= u.splits) break;
                const float f = st[s0 + s].y * (st[s0 + s].x == m ? 1.f : __builtin_amdgcn_exp2f(st[s0 + s].x - m));
                l += f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e >> 2][e & 3] = fmaf(part[s][e >> 2][e & 3], f, sum[e >> 2][e & 3]);
            }
        }
        const int qi = row / u.per, head = u.kvh * u.per + row - qi * u.per;
        const int64_t to = (u.first + qi) * a.ot + head * a.oh + d;
        float out[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = l == 0.f ? 0.f : sum[e >> 2][e & 3] / l;
        if (d < a.c.dim) {
            if (a.dtype == QE_F32) kv_out8<2>(a, to, out);
            else kv_out8<1>(a, to, out);
        }
        if (a.lse && d == 0) a.lse[(u.first + qi) * a.heads + head] = kv_lse(m + kKvJoinLog2, l);
    }
}

// The form of a call: many rows or few, and a wave's tiles of 16 rows.
struct KvForm { bool many; int nt; };

// Tiles of a wave with many rows, and of a unit with few at most: what the registers hold.
constexpr int kv_many_nt(int dp, int group, bool f32) { return dp <= 128 && !f32 && (group > 32 || dp == 64) ? 2 : 1; }
constexpr int kv_few_nt(int dp, int group, bool f32) { return dp <= 128 && !f32 && (group > 32 || dp < 128) ? 2 : 1; }

template <int DP> void kv_attn_width(const KvAttn& a, const KvPlan& plan, KvForm form, dim3 grid, hipStream_t s)
{
    kv_dispatch_group<DP>(a.group, [&](auto shape) {
        constexpr int G = decltype(shape)::GROUP;
        if (a.dtype == QE_F32) {
            if (form.many) hipLaunchKernelGGL((kv_many_kernel<DP, G, kv_many_nt(DP, G, true), 2>), grid, dim3(256), 0, s, a, plan);
            else hipLaunchKernelGGL((kv_few_kernel<DP, G, 1, 2>), grid, dim3(256), 0, s, a, plan);
        } else if (form.many) {
            hipLaunchKernelGGL((kv_many_kernel<DP, G, kv_many_nt(DP, G, false), 1>), grid, dim3(256), 0, s, a, plan);
        } else if (form.nt == 1) {
            hipLaunchKernelGGL((kv_few_kernel<DP, G, 1, 1>), grid, dim3(256), 0, s, a, plan);
        } else {
            hipLaunchKernelGGL((kv_few_kernel<DP, G, kv_few_nt(DP, G, false), 1>), grid, dim3(256), 0, s, a, plan);
        }
    });
    if (plan.nsplit > kKvFewSplits)
        hipLaunchKernelGGL((kv_join_kernel<DP>), grid_xy(plan.units * plan.rows, 256), dim3(256), 0, s, a, plan);
    else if (plan.nsplit > 1)
        hipLaunchKernelGGL((kv_join_unit_kernel<DP>), dim3((unsigned)plan.units), dim3(256), 0, s, a, plan);
}

}  // namespace qe
