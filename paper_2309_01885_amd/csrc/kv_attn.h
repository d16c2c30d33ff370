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
    const KvItem* items[2];                 // kKvListed: two lists of what the workgroups do, the first wgs0 of them the first list,
    const int32_t* count;                   // and how long the lists are
    int wgs0;
};

// What a kernel's workgroups work on: every (unit, split) of a call; the same where first tokens stay visible beside a
// window; or the entries of two lists, whose results are always joined by another launch.
// First tokens cost their records alone: a unit's records are the first tokens' and the window's, counted through, so
// that splits and both forms are the plain call's.  2048 queries of 32 heads on 8 of 128 channels at the end of 32768 tokens,
// a window of 4096 and 128 first tokens: 193 us, 733 TFLOP/s, the rate of a plain chunk; one token of 64 sequences, 71 heads
// on one of 64 channels, 4000 and 100 tokens: 31 us, of which 11 are what any call with a join takes; vector units 40 % busy.
enum KvMode { kKvPlain, kKvSinks, kKvListed };

// What a workgroup works on; the join recomputes it.
struct KvUnit {
    int64_t first, pos0;                    // first row of Q, position of query 0
    int b, kvh, per, tile_row, rows;        // per: heads of a key head; the unit's first row; rows of the sequence
    int len, rec0, rec1, splits;            // cached tokens; records that some row sees; splits in use
    int gap, skip;                          // kKvSinks: records from the gap on are `skip` further behind
    int ref, slot;                          // kKvListed: what slopes count from (-1: the row's position); first row of its results

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

// Record r of a unit.
template <KvMode MODE> __device__ inline int kv_place(const KvUnit& u, int r) { return MODE == kKvSinks && r >= u.gap ? r + u.skip : r; }

// (Divisions are of 32 bits: units and the rows of a sequence are fewer than 2^31, checked on the
// host, and one of 64 bits takes 130 instructions.)
template <KvMode MODE> __device__ inline KvUnit kv_unit(const KvAttn& a, const KvPlan& p, uint32_t unit, bool report)
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
    if constexpr (MODE == kKvSinks) {
        // the first tokens' records, then the window's; where they meet, everything in between
        u.gap = min(u.rec0, (int)((min((int64_t)a.sinks, end) + kKvTok - 1) / kKvTok));
        if (r0 >= u.rows) u.gap = 0;
        u.skip = u.rec0 - u.gap;
        u.rec1 -= u.skip;
        u.rec0 = 0;
        if (r0 >= u.rows) u.rec1 = 0;
    }
    const int records = u.rec1 - u.rec0;
    u.splits = records < kKvSplitFrom ? 1 : min(p.nsplit, records / kKvMinRecords);
    return u;
}

// A workgroup's entry of the lists.  Consecutive entries go to one XCD (every eighth workgroup): tiles of
// the same records share its L2.  False: there is none.
__device__ inline bool kv_listed(const KvPlan& p, KvUnit& u)
{
    const bool second = (int)blockIdx.x >= p.wgs0;
    const uint32_t wg = second ? blockIdx.x - p.wgs0 : blockIdx.x, n = kv_scalar(p.count + (second ? 1 : 0));
    const uint32_t x8 = wg & 7, at = x8 * (n / 8) + min(x8, n % 8) + (wg >> 3);
    if (wg >> 3 >= n / 8 + (x8 < n % 8 ? 1 : 0)) return false;
    const int32_t* it = reinterpret_cast<const int32_t*>((second ? p.items[1] : p.items[0]) + at);
    u.first = kv_scalar(it);
    u.b = kv_scalar(it + 1);
    u.kvh = kv_scalar(it + 2);
    u.tile_row = kv_scalar(it + 3);
    u.rows = kv_scalar(it + 4);
    u.len = kv_scalar(it + 5);
    u.pos0 = kv_scalar(it + 6);
    u.rec0 = kv_scalar(it + 7);
    u.rec1 = kv_scalar(it + 8);
    u.slot = kv_scalar(it + 9);
    u.ref = kv_scalar(it + 10);
    u.per = p.per;
    u.splits = 1;
    return u.tile_row < u.rows;
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
template <int NC, int NT, int PARTS, KvMode MODE> struct KvRows {
    f16x8 q[PARTS][NT][NC];
    float c[NT], slope[NT];                 // score of a product: c s + slope (t - pos), in powers of two
    int lo[NT], hi[NT];                     // the tokens that the lane's row sees
    int all_lo, all_hi;                     // that every row of the wave sees
    int sinks, ref;                         // kKvSinks: first tokens that every row sees, whatever lo is; KvUnit::ref

    // A row is scaled by 2^e to a largest element in [2^14, 2^15) and rounded to fp16.
    __device__ void load(const KvAttn& a, const KvUnit& u, int row0)
    {
        const int i = threadIdx.x & 15, j = (threadIdx.x & 63) >> 4;
        // (a shared part's rows see all of it, and have no positions in it)
        const bool causal = a.causal && (MODE != kKvListed || u.ref < 0);
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
            hi[n] = have && causal ? (int)max((int64_t)0, pos + 1) : u.len;
            lo[n] = have && a.window ? (int)max((int64_t)0, pos - a.window + 1) : 0;
        }
        all_lo = 0;
        all_hi = u.len;
        if constexpr (MODE == kKvSinks) sinks = a.sinks;
        if constexpr (MODE == kKvListed) ref = u.ref;
        if (causal) {
            // the first and the last row bound the others
            const int64_t p0 = u.pos0 + row0 / u.per, p1 = u.pos0 + (min(u.rows, row0 + 16 * NT) - 1) / u.per;
            all_hi = (int)max((int64_t)0, p0 + 1);
            if (a.window) all_lo = (int)max((int64_t)0, p1 - a.window + 1);
        }
    }
    __device__ bool masked(int t0) const { return t0 > all_hi - kKvTok || (t0 < all_lo && (MODE != kKvSinks || t0 > sinks - kKvTok)); }
    static constexpr bool kSinks = MODE == kKvSinks;
    __device__ int from(int n) const { return MODE == kKvListed && ref >= 0 ? ref : hi[n] - 1; }
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
    template <int KR, class ROWS, class F, class C>
    __device__ void weigh(float (&s)[KR][NT][8], const ROWS& r, bool slopes, const int (&t0)[KR], bool masked, F scales, C clear)
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
                    const float base = r.slope[n] * (float)(t - r.from(n));
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        s[y][n][e] = fmaf(s[y][n][e], c[n], fmaf(r.slope[n], (float)e, base));
                        s[y][n][e] = (t + e >= r.lo[n] || (ROWS::kSinks && t + e < r.sinks)) && t + e < r.hi[n] ? s[y][n][e] : -kKvInf;
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

// What a few-row workgroup keeps in LDS: its waves' words, later their sums and the rows' maxima and masses.
template <int DP, int GROUP, int NT> struct KvFewLds {
    static constexpr int NG = KvTiles<DP, GROUP>::NG;
    struct Words {
        float s[NG][64];                                         // scales
        uint16_t lo[NG][64], hi[NG][64];                         // -(1024 + z), -(1024 + 16 z) in fp16
    };
    static constexpr int kRow = DP + 4;                          // floats of a row (16-byte aligned, spread over the banks)
    __align__(16) union {
        Words words[kKvWaves];
        float acc[kKvWaves][16 * NT][kRow];
    };
    float wtop[kKvWaves][16 * NT], wmass[kKvWaves][16 * NT], rtop[16 * NT], rmass[16 * NT];
};

template <int DP, int GROUP, int NT, int PARTS>
__global__ __launch_bounds__(256, kv_few_occupancy(DP, GROUP, NT, PARTS)) void kv_few_kernel(KvAttn a, KvPlan plan)
{
    constexpr KvMode MODE = kKvPlain;
    __shared__ KvFewLds<DP, GROUP, NT> lds;
#include "kv_attn_few.h"
}
// (The bodies are included: as inlined functions of the kernels' arguments they took other registers, and one instance in
// groups of 32 spilled 27 instead of 10, another 11 instead of none.)
template <int DP, int GROUP, int NT, int PARTS, KvMode MODE>
__global__ __launch_bounds__(256, kv_few_occupancy(DP, GROUP, NT, PARTS)) void kv_few_mode_kernel(KvAttn a, KvPlan plan)
{
    __shared__ KvFewLds<DP, GROUP, NT> lds;
#include "kv_attn_few.h"
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
    constexpr KvMode MODE = kKvPlain;
#include "kv_attn_many.h"
}
template <int DP, int GROUP, int NT, int PARTS, KvMode MODE>
__global__ __launch_bounds__(256, 2) void kv_many_mode_kernel(KvAttn a, KvPlan plan)
{
#include "kv_attn_many.h"
}

// Joins the splits of a row: one workgroup a row, whose waves take the splits in turn.
template <int DP, KvMode MODE> __global__ __launch_bounds__(256) void kv_join_kernel(KvAttn a, KvPlan plan)
{
    constexpr int C = (DP + 63) / 64;
    __shared__ float sum[kKvWaves][DP], mass[kKvWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t at = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (at >= plan.units * plan.rows) return;
    // (plan.rows is a power of two)
    const uint32_t unit = (uint32_t)(at >> plan.rows_log2);
    const int rr = (int)(at & (plan.rows - 1));
    const KvUnit u = kv_unit<MODE>(a, plan, unit, false);
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
template <int DP, KvMode MODE> __global__ __launch_bounds__(256) void kv_join_unit_kernel(KvAttn a, KvPlan plan)
{
    const uint32_t unit = blockIdx.x;
    const KvUnit u = kv_unit<MODE>(a, plan, unit, false);
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

template <int DP, KvMode MODE> void kv_join_launch(const KvAttn& a, const KvPlan& plan, hipStream_t s)
{
    if (plan.nsplit > kKvFewSplits)
        hipLaunchKernelGGL((kv_join_kernel<DP, MODE>), grid_xy(plan.units * plan.rows, 256), dim3(256), 0, s, a, plan);
    else if (plan.nsplit > 1)
        hipLaunchKernelGGL((kv_join_unit_kernel<DP, MODE>), dim3((unsigned)plan.units), dim3(256), 0, s, a, plan);
}

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
    kv_join_launch<DP, kKvPlain>(a, plan, s);
}

}  // namespace qe
