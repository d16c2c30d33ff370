// The attention kernels' other modes (kv_attn.h), for one width (instantiated by kv_attn_modes_*.hip), and the join of
// the lists' results.
#pragma once

#include "kv_attn.h"

namespace qe {

template <int DP, KvMode MODE> void kv_mode_launch(const KvAttn& a, const KvPlan& plan, KvForm form, dim3 grid, hipStream_t s)
{
    kv_dispatch_group<DP>(a.group, [&](auto shape) {
        constexpr int G = decltype(shape)::GROUP;
        if (a.dtype == QE_F32) {
            if (form.many) hipLaunchKernelGGL((kv_many_mode_kernel<DP, G, kv_many_nt(DP, G, true), 2, MODE>), grid, dim3(256), 0, s, a, plan);
            else hipLaunchKernelGGL((kv_few_mode_kernel<DP, G, 1, 2, MODE>), grid, dim3(256), 0, s, a, plan);
        } else if (form.many) {
            hipLaunchKernelGGL((kv_many_mode_kernel<DP, G, kv_many_nt(DP, G, false), 1, MODE>), grid, dim3(256), 0, s, a, plan);
        } else if (form.nt == 1) {
            hipLaunchKernelGGL((kv_few_mode_kernel<DP, G, 1, 1, MODE>), grid, dim3(256), 0, s, a, plan);
        } else {
            hipLaunchKernelGGL((kv_few_mode_kernel<DP, G, kv_few_nt(DP, G, false), 1, MODE>), grid, dim3(256), 0, s, a, plan);
        }
    });
}

// Both lists at once where the shared part's tiles have 32 rows and the own part's 16: the short own parts fill what the
// others leave.
template <int DP, int GROUP> union KvPairLds {
    KvFewLds<DP, GROUP, 2> shared;
    KvFewLds<DP, GROUP, 1> own;
};
template <int DP, int GROUP>
__global__ __launch_bounds__(256, kv_few_occupancy(DP, GROUP, 2, 1)) void kv_pair_kernel(KvAttn a, KvPlan plan)
{
    constexpr KvMode MODE = kKvListed;
    constexpr int PARTS = 1;
    __shared__ KvPairLds<DP, GROUP> both;
    if ((int)blockIdx.x < plan.wgs0) {
        constexpr int NT = 2;
        auto& lds = both.shared;
#include "kv_attn_few.h"
    } else {
        constexpr int NT = 1;
        auto& lds = both.own;
#include "kv_attn_few.h"
    }
}
// Joins what the lists' entries found for a row: the parts of the group's shared records, then those of the sequence's
// own.  A thread has 8 channels of a row and every SUB-th of its parts.
template <int DP, int SUB> __global__ __launch_bounds__(256) void kv_shared_join_kernel(KvAttn a, KvPlan plan, KvShared sh, uint32_t tiles)
{
    constexpr int OCT = DP / 8, LANES = 256 / SUB, ROWS = LANES / OCT;
    __shared__ __align__(16) float part[SUB > 1 ? SUB : 1][SUB > 1 ? ROWS * OCT : 1][12];
    const uint32_t bh = blockIdx.x / tiles, tile = blockIdx.x - bh * tiles;
    const int b = (int)(bh / (uint32_t)a.c.heads), kvh = (int)(bh - (uint32_t)b * a.c.heads);
    const int32_t* sq = reinterpret_cast<const int32_t*>(sh.seq + b);
    const int first = kv_scalar(sq), nq = kv_scalar(sq + 1), len = kv_scalar(sq + 2), g = kv_scalar(sq + 3);
    const int own_tiles = kv_scalar(sq + 4), own = kv_scalar(sq + 5), own_item = kv_scalar(sq + 6);
    const int rows = max(nq, 0) * plan.per;
    if ((int)(tile * ROWS) >= rows) return;
    int records = 0, shared = 0, shared_tiles = 0, shared_item = 0, before = 0;
    if (g >= 0) {
        const int32_t* gr = reinterpret_cast<const int32_t*>(sh.group + g);
        before = (first - kv_scalar(gr + 1)) * plan.per;
        records = kv_scalar(gr + 3);
        shared_tiles = kv_scalar(gr + 4);
        shared = kv_scalar(gr + 5);
        shared_item = kv_scalar(gr + 6);
    }
    const int sub = threadIdx.x / LANES, x = threadIdx.x - sub * LANES, rr = x / OCT, d = 8 * (x - rr * OCT);
    const int row = (int)tile * ROWS + rr;
    const bool mine = rr < ROWS && row < rows;
    const int qi = row / plan.per, head = kvh * plan.per + row - qi * plan.per;
    const int all = mine ? shared + own : 0;
    const int at_a = before + row;
    const int64_t from_a = (int64_t)(shared_item + (kvh * shared_tiles + (at_a >> sh.rows_log2[0])) * shared) * sh.rows[0] + (at_a & (sh.rows[0] - 1));
    const int64_t from_b = (int64_t)sh.room[0] * sh.rows[0] + (int64_t)(own_item + (kvh * own_tiles + (row >> sh.rows_log2[1])) * own) * sh.rows[1] + (row & (sh.rows[1] - 1));
    // (the shared parts' slopes count from their last token)
    const float shift = mine && a.slopes && shared ? a.slopes[head] * kLog2e * (float)(records * kKvTok - 1 - (len - nq + qi)) : 0.f;
    auto place = [&](int s) { return s < shared ? from_a + (int64_t)s * sh.rows[0] : from_b + (int64_t)(s - shared) * sh.rows[1]; };
    const float2* const stat = reinterpret_cast<const float2*>(plan.stat);
    float m = -kKvInf, l = 0.f;
#pragma unroll 4
    for (int s = sub; s < all; s += SUB) m = fmaxf(m, stat[place(s)].x + (s < shared ? shift : 0.f));
    f32x4 sum[2] = {};
#pragma unroll 4
    for (int s = sub; s < all; s += SUB) {
        const int64_t k = place(s);
        const float2 st = stat[k];
        const float t = st.x + (s < shared ? shift : 0.f), f = st.y * (t == m ? 1.f : __builtin_amdgcn_exp2f(t - m));
        const f32x4 p0 = *reinterpret_cast<const f32x4*>(plan.part + k * DP + d), p1 = *reinterpret_cast<const f32x4*>(plan.part + k * DP + d + 4);
        l += f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sum[0][e] = fmaf(p0[e], f, sum[0][e]);
            sum[1][e] = fmaf(p1[e], f, sum[1][e]);
        }
    }
    if constexpr (SUB > 1) {
        if (rr < ROWS) {
            float* to = part[sub][x];
            *reinterpret_cast<f32x4*>(to) = sum[0];
            *reinterpret_cast<f32x4*>(to + 4) = sum[1];
            to[8] = m;
            to[9] = l;
        }
        __syncthreads();
        if (sub > 0) return;
#pragma unroll
        for (int y = 1; y < SUB; ++y) m = fmaxf(m, rr < ROWS ? part[y][x][8] : m);
        float f = rr < ROWS && part[0][x][8] != m ? __builtin_amdgcn_exp2f(part[0][x][8] - m) : 1.f;
        l *= f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e >> 2][e & 3] *= f;
        if (rr >= ROWS) return;
#pragma unroll
        for (int y = 1; y < SUB; ++y) {
            const float* p = part[y][x];
            f = p[8] != m ? __builtin_amdgcn_exp2f(p[8] - m) : 1.f;
            l = fmaf(p[9], f, l);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e >> 2][e & 3] = fmaf(p[e], f, sum[e >> 2][e & 3]);
        }
    }
    if (!mine) return;
    float out[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = l == 0.f ? 0.f : sum[e >> 2][e & 3] / l;
    if (d < a.c.dim) {
        const int64_t to = (first + (int64_t)qi) * a.ot + head * a.oh + d;
        if (a.dtype == QE_F32) kv_out8<2>(a, to, out);
        else kv_out8<1>(a, to, out);
    }
    if (a.lse && d == 0) a.lse[(first + (int64_t)qi) * a.heads + head] = kv_lse(m + kKvJoinLog2, l);
}

template <int DP> void kv_sinks_width(const KvAttn& a, const KvPlan& plan, KvForm form, dim3 grid, hipStream_t s)
{
    kv_mode_launch<DP, kKvSinks>(a, plan, form, grid, s);
    kv_join_launch<DP, kKvSinks>(a, plan, s);
}

// Both lists in one launch where they have one form, and the join.
template <int DP> void kv_listed_width(const KvAttn& a, const KvPlan& plan, const KvShared& sh, KvForm shared, KvForm own, hipStream_t s)
{
    KvPlan p = plan;
    const dim3 all((unsigned)(sh.room[0] + sh.room[1]));
    if (sh.pair) {
        kv_dispatch_group<DP>(a.group, [&](auto shape) {
            constexpr int G = decltype(shape)::GROUP;
            if constexpr (kv_few_nt(DP, G, false) == 2) hipLaunchKernelGGL((kv_pair_kernel<DP, G>), all, dim3(256), 0, s, a, p);
        });
    } else if (sh.joint) {
        kv_mode_launch<DP, kKvListed>(a, p, own, all, s);
    } else {
        kv_mode_launch<DP, kKvListed>(a, p, shared, dim3((unsigned)sh.room[0]), s);
        p.wgs0 = 0;
        kv_mode_launch<DP, kKvListed>(a, p, own, dim3((unsigned)sh.room[1]), s);
    }
    constexpr int few = 256 / 4 / (DP / 8), many = 256 / (DP / 8);
    const int64_t rows = a.max_q * plan.per;
    const int64_t tiles = cdiv(rows, rows <= few ? few : many);
    const dim3 grid((unsigned)(a.batch * a.c.heads * tiles));
    if (rows <= few) hipLaunchKernelGGL((kv_shared_join_kernel<DP, 4>), grid, dim3(256), 0, s, a, plan, sh, (uint32_t)tiles);
    else hipLaunchKernelGGL((kv_shared_join_kernel<DP, 1>), grid, dim3(256), 0, s, a, plan, sh, (uint32_t)tiles);
}

}  // namespace qe
