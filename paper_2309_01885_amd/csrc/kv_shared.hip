// Attention of sequences that start with the same pages (qe.h): the lists of work.
//
// A softmax over two sets of tokens is the two sets' softmaxes weighed by their masses, so the tokens that a group of
// sequences shares can be taken for all of its queries at once: its rows (every query and head of a key head) are
// one stretch of Q and fill the matrix instructions' tiles, and a shared record is read once for a tile instead of
// once for a sequence.  Shared are the records that every query of the group sees whole; so no row of that part
// is masked, and what a sequence has behind them is its own part, with every mask that kv_attn has.
// Both parts are cut into entries of lists, along the tokens in pieces of one size, which only the device knows the
// lengths for: one workgroup writes the lists, the attention kernels take an entry a workgroup, a last launch joins.
//
// What bounds it: one token of 64 sequences behind 8192 shared tokens and 256 to 1024 of their own, 32 heads on 8 of 128
// channels in bf16, takes 50 to 52 us (kv_attn 103, though the shared records come from a cache there): 7 for the lists, 6 for the
// join, and the entries' vector instructions (units 50 % busy over the launch, near their limit while the shared entries
// run); behind 32768 tokens 97 us (kv_attn 344).
#include "kv_attn_modes.h"
#include "kv_scan.h"

#include <algorithm>

namespace qe {

extern template void kv_listed_width<64>(const KvAttn&, const KvPlan&, const KvShared&, KvForm, KvForm, hipStream_t);
extern template void kv_listed_width<96>(const KvAttn&, const KvPlan&, const KvShared&, KvForm, KvForm, hipStream_t);
extern template void kv_listed_width<128>(const KvAttn&, const KvPlan&, const KvShared&, KvForm, KvForm, hipStream_t);
extern template void kv_listed_width<192>(const KvAttn&, const KvPlan&, const KvShared&, KvForm, KvForm, hipStream_t);
extern template void kv_listed_width<256>(const KvAttn&, const KvPlan&, const KvShared&, KvForm, KvForm, hipStream_t);

namespace {

// Rows of a call that the lists take (all heads of a key head; so that rows and what is added to them stay ints).
constexpr int32_t kMostRows = 1 << 29;
constexpr int kMaxGroups = kScanThreads;                 // a thread a group

__device__ inline int32_t div_up(int32_t a, int32_t b) { return (int32_t)(((uint32_t)a + (uint32_t)b - 1) / (uint32_t)b); }

// Pieces of about `size` (or up to twice that) that n records are cut into: no more in all than the sizes were made for.
__device__ inline int32_t pieces(int32_t n, int32_t size) { return n == 0 ? 0 : max(n / size, 1); }
// The first record of piece k of m.
__device__ inline int32_t piece(int32_t n, int32_t m, int32_t k)
{
    const uint32_t q = (uint32_t)n / (uint32_t)m;
    return (int32_t)(q * (uint32_t)k + min((uint32_t)k, (uint32_t)n - q * (uint32_t)m));
}

// A thread has a group, and a stretch of sequences.  What one needs of the other goes through LDS; the entries are written
// last.  64 sequences: 7 us, of which the sums take two, the first loads and the entries one each.
__global__ __launch_bounds__(kScanThreads) void kv_shared_plan_kernel(KvAttn a, KvShared sh)
{
    __shared__ ScanLds<2> lds;
    __shared__ ScanLds<2> lds2;
    __shared__ int32_t bound[kMaxGroups + 1];            // first sequences
    __shared__ int32_t sees[kMaxGroups], first[kMaxGroups], active[kMaxGroups], records[kMaxGroups], item[kMaxGroups + 1];
    __shared__ int32_t reader[kMaxGroups];               // the first sequence with queries: its row of the table names the shared pages
    __shared__ unsigned long long tokens[kMaxGroups];
    __shared__ KvGroup group[kMaxGroups];
    __shared__ KvSequence seq[kScanThreads];              // (of more sequences than threads: in memory alone)
    __shared__ int wrong, end_b;
    const int tid = threadIdx.x, threads = blockDim.x, per = a.heads / a.c.heads;
    const int64_t room = a.width * (int64_t)a.c.per * kKvTok;
    const int64_t run = (a.batch + threads - 1) / threads, b0 = min((int64_t)tid * run, (int64_t)a.batch), b1 = min(b0 + run, (int64_t)a.batch);
    const int ngroups = sh.ngroups;
    int32_t shared_pages = 0;
    if (tid == 0) {
        wrong = 0;
        end_b = 0x7fffffff;
    }
    if (tid <= ngroups) bound[tid] = sh.groups[tid];
    if (tid == 0 && threads == ngroups) bound[ngroups] = sh.groups[ngroups];
    if (tid < ngroups) {
        shared_pages = sh.shared[tid];
        sees[tid] = 0x7fffffff;
        reader[tid] = 0x7fffffff;
        first[tid] = 0;
        active[tid] = 0;
        tokens[tid] = 0;
    }
    // the thread's sequences: one in registers, more in memory
    KvSequence mine = {};
    auto get = [&](int64_t b) { return run == 1 ? mine : sh.seq[b]; };
    auto put = [&](int64_t b, const KvSequence& s) {
        if (run == 1) mine = s;
        else sh.seq[b] = s;
    };
    for (int64_t b = b0; b < b1; ++b) {
        KvSequence s = {};
        int64_t at = b * a.max_q, nq = a.max_q;
        const int64_t len = a.lengths[b];
        bool bad = len < 0 || len > room;
        if (a.q_start) {
            at = a.q_start[b];
            nq = (int64_t)a.q_start[b + 1] - at;
            if (at < 0 || nq < 0 || nq > a.max_q || at + nq > a.total) {
                bad = true;
                at = 0;
                nq = -1;
            }
        }
        if (bad) set_status(a.status, QE_ERR_ARG);
        s.first = (int32_t)at;
        s.nq = (int32_t)nq;
        s.len = (int32_t)max((int64_t)0, min(len, room));
        s.tiles = nq > 0 ? (s.nq * per + sh.rows[1] - 1) >> sh.rows_log2[1] : 0;
        put(b, s);
    }
    __syncthreads();
    if (tid < ngroups && (bound[tid] < 0 || bound[tid + 1] < bound[tid] || bound[tid + 1] > a.batch)) wrong = 1;
    // what all queries of a group see
    for (int64_t b = b0; b < b1; ++b) {
        KvSequence s = get(b);
        const int g = s.group = b < bound[0] || b >= bound[ngroups] ? -1 : (int)last_at_most(bound, ngroups, b);
        put(b, s);
        if (g < 0) continue;
        if (b == bound[g]) first[g] = s.first;
        if (s.nq < 0) atomicMin(&sees[g], 0);            // (its rows are not where the group's are)
        if (s.nq <= 0) continue;
        atomicMin(&sees[g], max(0, a.causal ? (int32_t)max((int64_t)s.len - s.nq + 1, (int64_t)0) : s.len));
        atomicMin(&reader[g], (int32_t)b);
        atomicAdd(&active[g], 1);
        atomicAdd(&tokens[g], (unsigned long long)s.nq);
    }
    __syncthreads();
    const bool none = wrong != 0;
    if (none && tid == 0) set_status(a.status, QE_ERR_ARG);
    KvGroup gr = {};
    if (tid < ngroups) {
        if (shared_pages < 0 || shared_pages > a.width) set_status(a.status, QE_ERR_ARG);
        const int64_t most = max((int64_t)0, min((int64_t)shared_pages, a.width)) * a.c.per;
        const bool gains = !none && active[tid] > 1 && tokens[tid] <= (unsigned long long)a.total;
        gr.reader = reader[tid];
        gr.first = first[tid];
        gr.tokens = gains ? (int32_t)tokens[tid] : 0;
        gr.records = gains ? (int32_t)min(most, (int64_t)(sees[tid] / kKvTok)) : 0;
        gr.tiles = gr.records ? (gr.tokens * per + sh.rows[0] - 1) >> sh.rows_log2[0] : 0;
        records[tid] = gr.records;
    }
    __syncthreads();

    // the sizes of the lists' entries: what fills the chip; once more without sharing where the first list would overflow (rows
    // that several groups claim, with a bad q_start between them)
    int64_t all[2], at[2], own[2];
    int32_t size[2], items_a;
    bool share = !none;                                  // (gr.records is 0 where none)
    auto own_records = [&](const KvSequence& s) { return max(0, div_up(s.len, kKvTok) - (s.group >= 0 ? records[s.group] : 0)); };
    for (;;) {
        at[0] = (int64_t)gr.tiles * gr.records;
        at[1] = 0;
        for (int64_t b = b0; b < b1; ++b) {
            KvSequence s = get(b);
            if (s.group >= 0 && !(share && records[s.group])) s.group = -1;
            at[1] += (int64_t)s.tiles * own_records(s);
            put(b, s);
        }
        scan_add(at, lds, all);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            // In one launch, long shared entries start first and short own ones fill the rest of the chip: a record of 32 shared
            // rows then counts as 4 of 5 parts of a record of 16 own ones (both wait more than they compute), as 8 where the own part
            // is a small rest.  us with 4 / 8, one query each of 32 heads on 8 of 128: 64 sequences behind 8192 tokens (1.6 times
            // the own records) 50.8 / 54.2, 16 behind 4096 (0.8) 24.4 / 25.4, 8 behind 16384 (3.2) 30.9 / 32.9, 64 behind 32768
            // (6.4) 107 / 96.
            const int64_t shared_weight = !sh.pair ? 5 : all[0] > 5 * all[1] ? 8 : 4;
            const int64_t work = sh.joint ? all[0] * shared_weight + all[1] * 5 : 5 * all[y];
            const double by = 1. / (double)(sh.fill[y] * (sh.joint && y == 0 ? shared_weight : 5));
            size[y] = max(sh.least[y], (int32_t)fmin(2147483647., ceil((double)(work * a.c.heads) * by)));
        }
        gr.splits = pieces(gr.records, size[0]);
        own[0] = at[0] = (int64_t)gr.tiles * gr.splits * a.c.heads;
        at[1] = 0;
        for (int64_t b = b0; b < b1; ++b) {
            KvSequence s = get(b);
            s.splits = s.tiles ? pieces(own_records(s), size[1]) : 0;
            at[1] += (int64_t)s.tiles * s.splits * a.c.heads;
            put(b, s);
        }
        own[1] = at[1];
        scan_add(at, lds2, all);
        items_a = (int32_t)all[0];
        if (all[0] <= sh.room[0]) break;
        if (tid == 0) set_status(a.status, QE_ERR_ARG);
        share = false;
        gr.records = gr.tiles = 0;
        __syncthreads();
    }
    if (tid < ngroups) {
        gr.item = (int32_t)(at[0] - own[0]);
        item[tid] = gr.item;
        group[tid] = gr;
    }
    int64_t next = at[1] - own[1];
    for (int64_t b = b0; b < b1; ++b) {
        KvSequence s = get(b);
        s.item = (int32_t)min(next, (int64_t)sh.room[1]);
        next += (int64_t)s.tiles * s.splits * a.c.heads;
        if (next > sh.room[1]) {
            // (rows that several sequences claim, with a bad q_start between them: the last of these get nothing)
            set_status(a.status, QE_ERR_ARG);
            atomicMin(&end_b, s.item);
            s.nq = -1;
            s.splits = 0;
        }
        put(b, s);
        if (run == 1) seq[tid] = s;
    }
    __syncthreads();
    const int32_t items_b = (int32_t)min(all[1], (int64_t)end_b);
    if (tid == 0) {
        sh.count[0] = items_a;
        sh.count[1] = items_b;
    }
    for (int32_t i = tid; i < items_a; i += threads) {
        const KvGroup q = group[last_at_most(item, ngroups, i)];
        // tiles of the same records side by side
        const uint32_t n = (uint32_t)(i - q.item), tile = n % (uint32_t)q.tiles, rest = n / (uint32_t)q.tiles;
        const int32_t split = (int32_t)(rest % (uint32_t)q.splits), kvh = (int32_t)(rest / (uint32_t)q.splits);
        KvItem it = {};
        it.first = q.first;
        it.b = q.reader;
        it.kvh = kvh;
        it.tile_row = (int32_t)tile * sh.rows[0];
        it.rows = q.tokens * per;
        it.len = q.records * kKvTok;
        it.rec0 = piece(q.records, q.splits, split);
        it.rec1 = piece(q.records, q.splits, split + 1);
        it.slot = (q.item + (kvh * q.tiles + (int32_t)tile) * q.splits + split) * sh.rows[0];
        it.ref = it.len - 1;
        sh.items[0][i] = it;
    }
    // a thread a sequence and key head
    for (int64_t p = tid; p < (int64_t)a.batch * a.c.heads; p += threads) {
        const uint32_t b = (uint32_t)p / (uint32_t)a.c.heads;
        const int32_t kvh = (int32_t)((uint32_t)p - b * (uint32_t)a.c.heads);
        const KvSequence q = run == 1 ? seq[b] : sh.seq[b];
        if (q.nq <= 0 || q.splits == 0) continue;
        const int32_t from = q.group >= 0 ? records[q.group] : 0, count = div_up(q.len, kKvTok) - from;
        KvItem* to = sh.items[1] + q.item + kvh * q.tiles * q.splits;
        KvItem it = {};
        it.first = q.first;
        it.b = (int32_t)b;
        it.kvh = kvh;
        it.rows = q.nq * per;
        it.len = q.len;
        it.pos0 = q.len - q.nq;
        it.ref = -1;
        const int32_t slot = sh.room[0] * sh.rows[0] + (q.item + kvh * q.tiles * q.splits) * sh.rows[1];
        for (int32_t split = 0; split < q.splits; ++split) {
            const int32_t r0 = from + piece(count, q.splits, split), r1 = from + piece(count, q.splits, split + 1);
            for (int32_t tile = 0; tile < q.tiles; ++tile) {
                it.tile_row = tile * sh.rows[1];
                it.rec0 = r0;
                it.rec1 = r1;
                if (a.causal && q.tiles > 1) {
                    // (what the tile's last row does not see)
                    const int32_t last = (min(it.rows, it.tile_row + sh.rows[1]) - 1) / per, end = max(0, it.pos0 + last + 1);
                    it.rec1 = max(r0, min(r1, div_up(end, kKvTok)));
                }
                it.slot = slot + (tile * q.splits + split) * sh.rows[1];
                *to++ = it;
            }
        }
    }
    // (what the join reads; before the barrier, everything would wait for these stores)
    if (tid < ngroups) sh.group[tid] = gr;
    if (run == 1 && b0 < b1) sh.seq[b0] = mine;
}

struct Lists {
    KvForm form[2];
    KvShared sh;
    int64_t slots;                                       // rows of partial results
};

// Rows, and records of its tiles, from which a part takes the many-row form: entries of 48 records on 512 workgroups.  Shorter
// ones lose to its start and the 64 KB of results that an entry writes.  One query each, us of the few rows' form / the
// many's: 64 sequences behind 8192 tokens, 32 heads on 8 of 128 channels (8 records an entry) 54 / 69, behind 32768 (32) 96 /
// 110; 32 behind 8192, 232 heads on 8 of 64 (29) 56 / 74; 7 queries of 48 behind 8192 to 16384 in five groups, 58 heads on 2
// of 64 (94) 118 / 111; chunks of 256 of 4 behind 8192, 32 heads on 8 of 128 (136) 199 / 145.
constexpr int64_t kManyRows = 128, kManyRecords = 48 * 512;
// Records of 16-row tiles that sharing has to save before it is taken: what its two more launches cost.  One query each, us of
// kv_attn / the lists: 4 sequences behind 1000 tokens, 20 heads on 5 of 80, fp32 (saves 1000) 13.8 / 20.1; 32 heads on 8 of
// 128: 16 behind 4096 (15000) 25.4 / 25.4, 8 behind 16384 (26000) 35.6 / 32.9, 64 behind 8192 (106000) 103 / 54.
// The host knows the table's width alone, and takes sequences and prefixes to fill it.  Where they do not, the lists lose: in a table for
// 131072 tokens, 8 of 500 tokens behind 64 12.0 / 18.9, 64 of 500 behind 64 18.3 / 35.1, 64 of 4000 behind 64 66 / 83, behind 3840
// 54 / 51; 8 of 16584 behind 16384 34.2 / 30.7.
constexpr int64_t kSaves = 20000;

// The forms of the shared and the own part, and the sizes of their lists.
Lists lists_of(int64_t total, int64_t batch, int64_t max_q, int heads, int kv_heads, int dim, int group, bool f32, int64_t ngroups,
               int64_t records)
{
    Lists z{};
    const int dp = kv_dp(dim), per = heads / kv_heads;
    const int64_t rows = total * per, group_rows = rows / std::max<int64_t>(ngroups, 1), own_rows = max_q * per;
    const int many = kv_many_nt(dp, group, f32), few = kv_few_nt(dp, group, f32);
    const int64_t many_units = kv_heads * cdiv(rows, 16 * many * kKvWaves);
    const bool long_rows = group_rows >= kManyRows && many_units * std::min<int64_t>(records, 1 << 24) >= kManyRecords;
    z.form[0] = long_rows ? KvForm{true, many} : KvForm{false, group_rows > 16 ? few : 1};
    z.form[1] = own_rows >= kManyRows ? KvForm{true, many} : KvForm{false, own_rows > 16 ? few : 1};
    const bool pair = z.sh.pair = !z.form[0].many && !z.form[1].many && z.form[0].nt > z.form[1].nt;
    z.sh.joint = pair || (z.form[0].many == z.form[1].many && z.form[0].nt == z.form[1].nt);
    int64_t units[2];
    for (int y = 0; y < 2; ++y) {
        const KvForm form = pair ? z.form[0] : z.form[y];
        z.sh.rows[y] = 16 * z.form[y].nt * (z.form[y].many ? kKvWaves : 1);
        z.sh.rows_log2[y] = __builtin_ctz((unsigned)z.sh.rows[y]);
        z.sh.fill[y] = 256 * (form.many ? 2 : kv_few_occupancy(dp, dp <= 64 ? std::min(group, 64) : group, form.nt, f32 ? 2 : 1));
        z.sh.least[y] = kKvMinRecords;
        units[y] = kv_heads * (cdiv(rows, z.sh.rows[y]) + (y == 0 ? ngroups : batch));
    }
    units[1] = std::min(units[1], kv_heads * batch * cdiv(own_rows, z.sh.rows[1]));
    z.slots = 0;
    for (int y = 0; y < 2; ++y) {
        const int64_t n = cdiv(units[y] + z.sh.fill[y], 8) * 8;
        z.slots += n * z.sh.rows[y];
        z.sh.room[y] = (int32_t)std::min<int64_t>(n, INT32_MAX);
    }
    z.sh.ngroups = (int32_t)ngroups;
    return z;
}

// Where the lists, the partial results or the join's workgroups (of 8 rows at least) pass 32-bit numbers, or nothing can be
// shared, the call is kv_attn's.
bool listed(const Lists& z, int64_t total, int64_t batch, int64_t max_q, int heads, int kv_heads)
{
    const int64_t per = heads / kv_heads, most = int64_t(1) << 23;
    return batch > 1 && z.sh.ngroups > 0 && z.sh.ngroups <= kMaxGroups && total * per < kMostRows && z.slots < (int64_t(1) << 31) &&
           (int64_t)z.sh.room[0] + z.sh.room[1] < most && batch * kv_heads * cdiv(max_q * per, 8) < most;
}

// Whether sharing can gain what its launches cost.  (Where a sequence's rows fill tiles by themselves it saves no tile, but
// the lists' many-row form has splits, and kv_attn's does not.)
bool gains(const Lists& z, const KvAttn& a)
{
    const int64_t per = a.heads / a.c.heads, records = a.width * a.c.per, groups = z.sh.ngroups;
    if (z.form[0].many && !kv_attn_many(a)) return true;
    const int64_t tiles = a.batch * cdiv(a.max_q * per, 16) - groups * cdiv(a.total * per, 16 * groups);
    return tiles > 0 && tiles * a.c.heads >= cdiv(kSaves, std::max<int64_t>(records, 1));
}

struct Layout {
    size_t group, seq, items[2], count, part, stat, end;
};
Layout layout_of(const Lists& z, int64_t batch, int dp)
{
    Layout l;
    size_t at = kStatusBytes;
    auto take = [&](size_t bytes) {
        const size_t from = at;
        at += align256(bytes);
        return from;
    };
    l.group = take(z.sh.ngroups * sizeof(KvGroup));
    l.seq = take(batch * sizeof(KvSequence));
    for (int y = 0; y < 2; ++y) l.items[y] = take(z.sh.room[y] * sizeof(KvItem));
    l.count = take(2 * sizeof(int32_t));
    l.part = take((size_t)z.slots * dp * sizeof(float));
    l.stat = take((size_t)z.slots * 2 * sizeof(float));
    l.end = at;
    return l;
}

}  // namespace

// (always: of the lists, also where kv_attn itself would be taken whatever the table's width.)
size_t kv_attn_shared_ws_bytes(int64_t total, int64_t batch, int64_t max_q, int heads, int kv_heads, int dim, int64_t ngroups, bool always)
{
    size_t need = kv_attn_ws_bytes(batch, max_q, heads, kv_heads, dim);
    KvAttn a{};
    a.total = total;
    a.batch = (int32_t)std::min<int64_t>(batch, INT32_MAX);
    a.max_q = max_q;
    a.heads = heads;
    a.c.heads = kv_heads;
    a.c.dim = dim;
    a.c.per = 1;
    a.width = INT32_MAX;                                 // (a wider table makes sharing gain more)
    for (int group : {32, 64, 128})
        for (int f32 = 0; f32 < 2; ++f32) {
            a.group = group;
            a.dtype = f32 ? QE_F32 : QE_BF16;
            for (int64_t records : {(int64_t)1, a.width}) {
                const Lists z = lists_of(total, batch, max_q, heads, kv_heads, dim, group, f32 != 0, ngroups, records);
                if (!listed(z, total, batch, max_q, heads, kv_heads)) continue;
                const Lists wide = lists_of(total, batch, max_q, heads, kv_heads, dim, group, f32 != 0, ngroups, a.width);
                if (always || gains(wide, a)) need = std::max(need, layout_of(z, batch, kv_dp(dim)).end);
            }
        }
    return need;
}

// (The workspace is checked for what this call takes: the size for any group, type and width, as the caller has asked for it, is a
// dozen lists' layouts, 2 us.)
qe_status launch_kv_attn_shared(const KvAttn& call, const int32_t* groups, const int32_t* shared, int64_t ngroups, void* ws, size_t ws_bytes,
                                bool always, hipStream_t s)
{
    KvAttn a = call;
    const int dp = kv_dp(a.c.dim);
    Lists z = lists_of(a.total, a.batch, a.max_q, a.heads, a.c.heads, a.c.dim, a.group, a.dtype == QE_F32, ngroups, a.width * a.c.per);
    if (!listed(z, a.total, a.batch, a.max_q, a.heads, a.c.heads) || !(always || gains(z, a))) {
        if (ws_bytes < kv_attn_ws_bytes(a.batch, a.max_q, a.heads, a.c.heads, a.c.dim)) return QE_ERR_WORKSPACE;
        return launch_kv_attn(a, ws, s);
    }
    const Layout l = layout_of(z, a.batch, dp);
    if (ws_bytes < l.end) return QE_ERR_WORKSPACE;
    kv_attn_vec(a);
    char* const base = static_cast<char*>(ws);
    KvShared& sh = z.sh;
    sh.groups = groups;
    sh.shared = shared;
    sh.group = reinterpret_cast<KvGroup*>(base + l.group);
    sh.seq = reinterpret_cast<KvSequence*>(base + l.seq);
    for (int y = 0; y < 2; ++y) sh.items[y] = reinterpret_cast<KvItem*>(base + l.items[y]);
    sh.count = reinterpret_cast<int32_t*>(base + l.count);
    KvPlan plan{};
    plan.per = a.heads / a.c.heads;
    plan.nsplit = 1;
    plan.part = reinterpret_cast<float*>(base + l.part);
    plan.stat = reinterpret_cast<float*>(base + l.stat);
    for (int y = 0; y < 2; ++y) plan.items[y] = sh.items[y];
    plan.count = sh.count;
    plan.wgs0 = sh.room[0];
    hipLaunchKernelGGL(kv_shared_plan_kernel, dim3(1), dim3(scan_threads(std::max<int64_t>({a.batch, ngroups, 512}))), 0, s, a, sh);
    switch (dp) {
        case 64: kv_listed_width<64>(a, plan, sh, z.form[0], z.form[1], s); break;
        case 96: kv_listed_width<96>(a, plan, sh, z.form[0], z.form[1], s); break;
        case 128: kv_listed_width<128>(a, plan, sh, z.form[0], z.form[1], s); break;
        case 192: kv_listed_width<192>(a, plan, sh, z.form[0], z.form[1], s); break;
        default: kv_listed_width<256>(a, plan, sh, z.form[0], z.form[1], s);
    }
    return hipGetLastError() == hipSuccess ? QE_OK : QE_ERR_HIP;
}

}  // namespace qe
