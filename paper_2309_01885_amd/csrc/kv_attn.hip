// How an attention call over the 4-bit cache is cut into workgroups.
#include "kv_attn_modes.h"

namespace qe {

extern template void kv_attn_width<64>(const KvAttn&, const KvPlan&, KvForm, dim3, hipStream_t);
extern template void kv_sinks_width<64>(const KvAttn&, const KvPlan&, KvForm, dim3, hipStream_t);
extern template void kv_attn_width<96>(const KvAttn&, const KvPlan&, KvForm, dim3, hipStream_t);
extern template void kv_sinks_width<96>(const KvAttn&, const KvPlan&, KvForm, dim3, hipStream_t);
extern template void kv_attn_width<128>(const KvAttn&, const KvPlan&, KvForm, dim3, hipStream_t);
extern template void kv_sinks_width<128>(const KvAttn&, const KvPlan&, KvForm, dim3, hipStream_t);
extern template void kv_attn_width<192>(const KvAttn&, const KvPlan&, KvForm, dim3, hipStream_t);
extern template void kv_sinks_width<192>(const KvAttn&, const KvPlan&, KvForm, dim3, hipStream_t);
extern template void kv_attn_width<256>(const KvAttn&, const KvPlan&, KvForm, dim3, hipStream_t);
extern template void kv_sinks_width<256>(const KvAttn&, const KvPlan&, KvForm, dim3, hipStream_t);

namespace {

// Workgroups of the many-row form from which it is taken: two of a CU.  Below that the few-row form is
// faster, since its workgroups are smaller and share a row's tokens.  128 queries over 2048 tokens, bf16, us of the many /
// the few at 256, 384 and 512 workgroups of the many: 64 channels in groups of 64 57 / 52, 81 / 72, 83 / 89; 96 in 64 94 / 85,
// 126 / 119, 131 / 157; 128 in 128 74 / 75, 103 / 110, 110 / 149; in 64 97 / 89, 132 / 134, 138 / 177; in 32 87 / 84,
// 110 / 121, 115 / 161; 192 in 64 122 / 90, 146 / 125, 149 / 166; in 32 164 / 125, 201 / 180, 205 / 239; 256 in 128 115 / 95,
// 147 / 139, 153 / 183; in 64 148 / 109, 189 / 159, 204 / 206.  fp32, 128 in 64: 89 / 74 at 256, 117 / 130 at 512.
// 256 channels in groups of 32 do not fit the few-row form's registers: at 128, 160 and 256 workgroups 375 / 234,
// 373 / 403, 376 / 463 (fp32 at 128, 192 and 256 477 / 261, 481 / 481, 499 / 527).
constexpr int64_t kManyRows = 128, kManyFill = 512, kManyFillWide = 160;
// Workgroups of the few-row form that fill the chip, three of a CU.  Units that are more than half of that would not be
// split; they are, in two or three, where each has kSplitLong records (8192 tokens) or more: the last ones, or the
// long ones, are not left to the end.  29 query heads on one of 64 channels, us with 768 / 1536 workgroups:
// 8192 tokens (2048 to 8192): 128 units 36 / 46 (32 / 41), 256 59 / 64 (50 / 51), 400 106 / 90 (91 / 73), 512 107 / 107
// (93 / 88), 640 136 / 128 (106 / 102), 768 139 / 150 (116 / 119); 4096 tokens (1024 to 4096): 448 54 / 61 (49 / 47),
// 512 58 / 64 (48 / 52); 16384 tokens (4096 to 16384): 400 196 / 156 (173 / 125), 640 263 / 233 (198 / 180).
constexpr int64_t kFill = 768, kSplitLong = 256;
// Records (32 tokens of one head for one unit) from which the few-row form takes 32 rows a unit
// instead of 16: a record's codes are then converted for twice the rows, but by half as many workgroups.
// 29 heads on one, 16 against 32 rows, in us: 128 channels in groups of 64, 256 units of 64 records 45 / 52, 512 of 64 65 /
// 72, 1024 of 32 65 / 57, 256 of 256 118 / 114; in groups of 128, 256 of 64 37 / 47, 256 of 256 100 / 101; 64 channels:
// 21 of 63 14 / 16, 64 of 256 30 / 32, 512 of 256 99 / 85; groups of 32: 64 channels, 256 of 256 90 / 79, 96 channels 122 / 119;
// 128 channels in groups of 32 spill: 176 / 281, and keep 16 (kv_few_nt).
constexpr int64_t kWideFrom = 32768;

KvForm form_of(int64_t heads, int64_t rows, int64_t records, int dp, int group, bool f32)
{
    const int nt = kv_many_nt(dp, group, f32);
    if (rows >= kManyRows && heads * cdiv(rows, 16 * nt * kKvWaves) >= (dp == 8 * group ? kManyFillWide : kManyFill)) return {true, nt};
    return {false, rows <= 16 || kv_few_nt(dp, group, f32) == 1 || heads * cdiv(rows, 32) < cdiv(kWideFrom, std::max<int64_t>(records, 1)) ? 1 : 2};
}

// Splits along the tokens: as many as fill the chip, each of at least kKvMinRecords records.
int splits_of(KvForm form, int64_t units, int64_t records)
{
    if (form.many || records < kKvSplitFrom) return 1;
    const int64_t fill = units > kFill / 2 && units < kFill && records >= kSplitLong ? 2 * kFill : kFill;
    return (int)std::max<int64_t>(1, std::min(fill / std::max<int64_t>(units, 1), records / kKvMinRecords));
}

struct Sizes {
    KvForm form;
    int rows;
    int64_t row_tiles, units;
};

Sizes sizes_of(int64_t batch, int64_t max_q, int heads, int kv_heads, int dim, int group, int64_t records, bool f32)
{
    Sizes z;
    const int64_t rows = max_q * (heads / kv_heads);
    z.form = form_of(batch * kv_heads, rows, records, kv_dp(dim), group, f32);
    z.rows = 16 * z.form.nt * (z.form.many ? kKvWaves : 1);
    z.row_tiles = cdiv(rows, z.rows);
    z.units = batch * kv_heads * z.row_tiles;
    return z;
}

size_t part_floats(const Sizes& z, int dp, int nsplit) { return (size_t)z.units * nsplit * z.rows * dp; }
size_t stat_floats(const Sizes& z, int nsplit) { return (size_t)z.units * nsplit * z.rows * 2; }

}  // namespace

size_t kv_attn_ws_bytes(int64_t batch, int64_t max_q, int heads, int kv_heads, int dim)
{
    size_t need = 0;
    // (The many-row form has no splits, and a group of 32 only takes it earlier: a group of 128 needs the
    // most.  With few records units have 16 rows, with many 32; fp32 calls have 16.)
    for (int64_t records : {(int64_t)1, (int64_t)INT32_MAX}) {
        for (int f32 = 0; f32 < 2; ++f32) {
            const Sizes z = sizes_of(batch, max_q, heads, kv_heads, dim, 128, records, f32 != 0);
            const int nsplit = splits_of(z.form, z.units, INT32_MAX);
            if (nsplit > 1)
                need = std::max(need, align256(part_floats(z, kv_dp(dim), nsplit) * 4) + align256(stat_floats(z, nsplit) * 4));
        }
    }
    return kStatusBytes + need;
}

bool kv_attn_many(const KvAttn& a)
{
    return sizes_of(a.batch, a.max_q, a.heads, a.c.heads, a.c.dim, a.group, a.width * a.c.per, a.dtype == QE_F32).form.many;
}

qe_status launch_kv_attn(const KvAttn& call, void* ws, hipStream_t s)
{
    KvAttn a = call;
    const int dp = kv_dp(a.c.dim);
    kv_attn_vec(a);
    int64_t records = a.width * a.c.per;
    if (a.window) records = std::min<int64_t>(records, (a.window + a.max_q) / kKvTok + 2 + cdiv(a.sinks, kKvTok));
    else a.sinks = 0;                                      // (every token is visible)
    const Sizes z = sizes_of(a.batch, a.max_q, a.heads, a.c.heads, a.c.dim, a.group, records, a.dtype == QE_F32);
    KvPlan plan{};
    plan.row_tiles = z.row_tiles;
    plan.units = z.units;
    plan.per = a.heads / a.c.heads;
    plan.rows_log2 = __builtin_ctz((unsigned)z.rows);
    plan.rows = z.rows;
    plan.nsplit = splits_of(z.form, z.units, records);
    plan.part = reinterpret_cast<float*>(static_cast<char*>(ws) + kStatusBytes);
    plan.stat = reinterpret_cast<float*>(reinterpret_cast<char*>(plan.part) + align256(part_floats(z, dp, plan.nsplit) * 4));
    const dim3 grid((unsigned)(z.units * plan.nsplit));
    auto width = [&](auto dp) {
        if (a.sinks) kv_sinks_width<dp>(a, plan, z.form, grid, s);
        else kv_attn_width<dp>(a, plan, z.form, grid, s);
    };
    switch (dp) {
        case 64: width(std::integral_constant<int, 64>()); break;
        case 96: width(std::integral_constant<int, 96>()); break;
        case 128: width(std::integral_constant<int, 128>()); break;
        case 192: width(std::integral_constant<int, 192>()); break;
        default: width(std::integral_constant<int, 256>());
    }
    return hipGetLastError() == hipSuccess ? QE_OK : QE_ERR_HIP;
}

}  // namespace qe
