// Attention of sequences that start with the same pages (qe.h): the lists of work.
//
// A softmax over two sets of tokens is the two sets' softmaxes weighed by their masses, so the tokens that a group of
// sequences shares can be taken for all of its queries at once: its rows (every query and head of a key head) are
// one stretch of Q and fill the matrix instructions' tiles, and a shared record is read once for a tile instead of
// once for a sequence.  Shared are the records that every query of the group sees whole; so no row of that part
// is masked, and what a sequence has behind them is its own part, with every mask that kv_attn has.
// Both parts are cut into entries of lists, along the tokens in pieces of one size, which only the device knows the
// lengths for: one workgroup writes the lists, the attention kernels take an entry a workgroup, a last launch joins.
#include "kv_attn_modes.h"
#include "kv_scan.h"

namespace qe {

extern template void kv_listed_width<64>(const KvAttn&, const KvPlan&, const KvShared&, KvForm, KvForm, hipStream_t);
extern template void kv_listed_width<96>(const KvAttn&, const KvPlan&, const KvShared&, KvForm, KvForm, hipStream_t);
extern template void kv_listed_width<128>(const KvAttn&, const KvPlan&, const KvShared&, KvForm, KvForm, hipStream_t);
extern template void kv_listed_width<192>(const KvAttn&, const KvPlan&, const KvShared&, KvForm, KvForm, hipStream_t);
extern template void kv_listed_width<256>(const KvAttn&, const KvPlan&, const KvShared&, KvForm, KvForm, hipStream_t);

namespace {

// Position of query 0 of a shared part: behind every token (and so that a position stays an int).
constexpr int32_t kBehind = 1 << 29;
constexpr int kNear = 4096;                              // lists whose starts are searched in LDS

__device__ inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Entries: splits of n records in pieces of about `size`, at most as many as the lists were made for.
__device__ inline int32_t splits_of(int64_t n, int64_t size) { return n == 0 ? 0 : (int32_t)max(n / size, (int64_t)1); }

__global__ __launch_bounds__(kScanThreads) void kv_shared_plan_kernel(KvAttn a, KvShared sh)
{
    __shared__ int64_t part[3][kScanThreads / 64];
    __shared__ int32_t start[kNear + 1];
    __shared__ int wrong_groups;
    const int tid = threadIdx.x, lane = tid & 63, per = a.heads / a.c.heads;
    const int64_t width = a.width, room = width * (int64_t)a.c.per * kKvTok;
    if (tid == 0) wrong_groups = 0;
    __syncthreads();
    // the sequences
    for (int64_t b = tid; b < a.batch; b += kScanThreads) {
        int64_t first = b * a.max_q, nq = a.max_q, len = a.lengths[b];
        bool bad = len < 0 || len > room;
        KvSequence s = {};
        if (a.q_start) {
            first = a.q_start[b];
            nq = (int64_t)a.q_start[b + 1] - first;
            if (first < 0 || nq < 0 || nq > a.max_q || first + nq > a.total) {
                bad = true;
                first = 0;
                nq = -1;
            }
        }
        if (bad) set_status(a.status, QE_ERR_ARG);
        s.first = (int32_t)first;
        s.nq = (int32_t)nq;
        s.len = (int32_t)max((int64_t)0, min(len, room));
        s.group = -1;
        sh.seq[b] = s;
    }
    for (int g = tid; g < sh.ngroups; g += kScanThreads) {
        const int32_t s0 = sh.groups[g], s1 = sh.groups[g + 1], n = sh.shared[g];
        if (s0 < 0 || s1 < s0 || s1 > a.batch) wrong_groups = 1;
        if (n < 0 || n > width) set_status(a.status, QE_ERR_ARG);
    }
    __syncthreads();
    if (wrong_groups && tid == 0) set_status(a.status, QE_ERR_ARG);
    const int ngroups = wrong_groups ? 0 : sh.ngroups;

    // the groups, a wave each: the records that all of their queries see
    for (int g = tid >> 6; g < ngroups; g += kScanThreads / 64) {
        const int32_t s0 = sh.groups[g], s1 = sh.groups[g + 1];
        int64_t sees = max(0, min(sh.shared[g], (int32_t)min(width, (int64_t)0x7fffffff))) * (int64_t)a.c.per * kKvTok;
        int64_t tokens = 0;
        int active = 0;
        for (int64_t b = s0 + lane; b < s1; b += 64) {
            const KvSequence s = sh.seq[b];
            if (s.nq < 0) sees = 0;                      // (its rows are not where the group's are)
            if (s.nq <= 0) continue;
            sees = min(sees, max((int64_t)0, a.causal ? (int64_t)s.len - s.nq + 1 : (int64_t)s.len));
            tokens += s.nq;
            ++active;
        }
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            sees = min(sees, __shfl_xor(sees, m));
            tokens += __shfl_xor(tokens, m);
            active += __shfl_xor(active, m);
        }
        KvGroup gr = {};
        gr.first_seq = s0;
        gr.tokens = (int32_t)min(tokens, a.total);
        gr.records = active < 2 || tokens > a.total ? 0 : (int32_t)(sees / kKvTok);
        gr.tiles = gr.records ? (int32_t)div_up((int64_t)gr.tokens * per, sh.rows[0]) : 0;
        if (s0 < s1) gr.first = sh.seq[s0].first;
        if (lane == 0) sh.group[g] = gr;
        if (gr.records)
            for (int64_t b = s0 + lane; b < s1; b += 64) sh.seq[b].group = g;
    }
    __syncthreads();

    // a piece's size: what fills the chip
    int64_t work[2] = {0, 0}, all[2], size[2];
    for (int g = tid; g < ngroups; g += kScanThreads) work[0] += (int64_t)sh.group[g].tiles * sh.group[g].records;
    for (int64_t b = tid; b < a.batch; b += kScanThreads) {
        const KvSequence s = sh.seq[b];
        const int64_t own = div_up(s.len, kKvTok) - (s.group >= 0 ? sh.group[s.group].records : 0);
        work[1] += div_up((int64_t)max(s.nq, 0) * per, sh.rows[1]) * max(own, (int64_t)0);
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        scan_add(work[y], part[y], all[y]);
        size[y] = max((int64_t)sh.least[y], div_up(all[y] * a.c.heads, sh.fill[y]));
    }

    // where the entries lie
    int64_t next = 0, sum;
    for (int64_t g0 = 0; g0 < ngroups; g0 += kScanThreads) {
        const int64_t g = g0 + tid;
        KvGroup gr = {};
        if (g < ngroups) gr = sh.group[g];
        gr.splits = splits_of(gr.records, size[0]);
        const int64_t n = (int64_t)gr.tiles * gr.splits * a.c.heads;
        __syncthreads();
        const int64_t end = next + scan_add(n, part[0], sum);
        gr.item = (int32_t)min(end - n, (int64_t)sh.room[0]);
        if (g < ngroups) {
            sh.group[g] = gr;
            if (g <= kNear) start[g] = gr.item;
        }
        next += sum;
    }
    __syncthreads();
    // (rows that several groups claim, with a bad q_start between them, can be more than the list holds: then nothing is shared)
    const bool fits = next <= sh.room[0];
    const int64_t items_a = fits ? next : 0;
    if (!fits) {
        if (tid == 0) set_status(a.status, QE_ERR_ARG);
        for (int64_t b = tid; b < a.batch; b += kScanThreads) sh.seq[b].group = -1;
    }
    for (int64_t i = tid; i < items_a; i += kScanThreads) {
        int64_t g;
        if (ngroups <= kNear) {
            g = last_at_most(start, ngroups, i);
        } else {
            int64_t lo = 0, hi = ngroups;
            while (hi - lo > 1) {
                const int64_t mid = (lo + hi) >> 1;
                if (sh.group[mid].item <= i) lo = mid;
                else hi = mid;
            }
            g = lo;
        }
        const KvGroup gr = sh.group[g];
        // tiles of the same records side by side
        const uint32_t at = (uint32_t)(i - gr.item), tile = at % (uint32_t)gr.tiles, rest = at / (uint32_t)gr.tiles;
        const uint32_t split = rest % (uint32_t)gr.splits, kvh = rest / (uint32_t)gr.splits;
        KvItem it = {};
        it.first = gr.first;
        it.b = gr.first_seq;
        it.kvh = (int32_t)kvh;
        it.tile_row = (int32_t)(tile * sh.rows[0]);
        it.rows = gr.tokens * per;
        it.len = gr.records * kKvTok;
        it.pos0 = kBehind;
        it.rec0 = (int32_t)((int64_t)gr.records * split / gr.splits);
        it.rec1 = (int32_t)((int64_t)gr.records * (split + 1) / gr.splits);
        it.slot = (int32_t)((gr.item + (kvh * gr.tiles + tile) * gr.splits + split) * sh.rows[0]);
        it.ref = it.len - 1;
        sh.items[0][i] = it;
    }
    __syncthreads();
    next = 0;
    for (int64_t b0 = 0; b0 < a.batch; b0 += kScanThreads) {
        const int64_t b = b0 + tid;
        KvSequence s = {};
        int64_t own = 0;
        if (b < a.batch) {
            s = sh.seq[b];
            own = max((int64_t)0, div_up(s.len, kKvTok) - (s.group >= 0 ? sh.group[s.group].records : 0));
        }
        s.tiles = (int32_t)div_up((int64_t)max(s.nq, 0) * per, sh.rows[1]);
        s.splits = s.tiles ? splits_of(own, size[1]) : 0;
        const int64_t n = (int64_t)s.tiles * s.splits * a.c.heads;
        __syncthreads();
        const int64_t end = next + scan_add(n, part[0], sum);
        s.item = (int32_t)min(end - n, (int64_t)sh.room[1]);
        if (b < a.batch) {
            if (end > sh.room[1]) {
                // (rows that several sequences claim, with a bad q_start between them: the last of these get nothing)
                set_status(a.status, QE_ERR_ARG);
                s.nq = -1;
                s.splits = 0;
            }
            sh.seq[b] = s;
            if (b <= kNear) start[b] = s.item;
        }
        next += sum;
    }
    __syncthreads();
    const int64_t items_b = min(next, (int64_t)sh.room[1]);
    for (int64_t i = tid; i < items_b; i += kScanThreads) {
        int64_t b;
        if (a.batch <= kNear) {
            b = last_at_most(start, a.batch, i);
        } else {
            int64_t lo = 0, hi = a.batch;
            while (hi - lo > 1) {
                const int64_t mid = (lo + hi) >> 1;
                if (sh.seq[mid].item <= i) lo = mid;
                else hi = mid;
            }
            b = lo;
        }
        const KvSequence s = sh.seq[b];
        KvItem it = {};
        if (s.splits > 0) {
            const uint32_t at = (uint32_t)(i - s.item), tile = at % (uint32_t)s.tiles, rest = at / (uint32_t)s.tiles;
            const uint32_t split = rest % (uint32_t)s.splits, kvh = rest / (uint32_t)s.splits;
            const int32_t from = s.group >= 0 ? sh.group[s.group].records : 0, n = (int32_t)div_up(s.len, kKvTok) - from;
            it.first = s.first;
            it.b = (int32_t)b;
            it.kvh = (int32_t)kvh;
            it.tile_row = (int32_t)(tile * sh.rows[1]);
            it.rows = s.nq * per;
            it.len = s.len;
            it.pos0 = s.len - s.nq;
            it.rec0 = from + (int32_t)((int64_t)n * split / s.splits);
            it.rec1 = from + (int32_t)((int64_t)n * (split + 1) / s.splits);
            if (a.causal) {
                // (what the tile's last row does not see)
                const int32_t last = (min(it.rows, it.tile_row + sh.rows[1]) - 1) / per, end = max(0, it.pos0 + last + 1);
                it.rec1 = max(it.rec0, min(it.rec1, (end + kKvTok - 1) / kKvTok));
            }
            it.slot = sh.room[0] * sh.rows[0] + (int32_t)((s.item + (kvh * s.tiles + tile) * s.splits + split) * sh.rows[1]);
            it.ref = -1;
        }
        sh.items[1][i] = it;
    }
    if (tid == 0) {
        sh.count[0] = (int32_t)items_a;
        sh.count[1] = (int32_t)items_b;
    }
}

struct Lists {
    KvForm form[2];
    KvShared sh;
    int64_t slots;                                       // rows of partial results
};

// The forms of the shared and the own part, and the sizes of their lists.
Lists lists_of(int64_t total, int64_t batch, int64_t max_q, int heads, int kv_heads, int dim, int group, bool f32, int64_t ngroups)
{
    Lists z{};
    const int dp = kv_dp(dim), per = heads / kv_heads;
    const int64_t rows = total * per, group_rows = rows / std::max<int64_t>(ngroups, 1), own_rows = max_q * per;
    const int many = kv_many_nt(dp, group, f32), few = kv_few_nt(dp, group, f32);
    z.form[0] = group_rows >= 64 ? KvForm{true, many} : KvForm{false, group_rows > 16 ? few : 1};
    z.form[1] = KvForm{false, own_rows > 16 ? few : 1};
    int64_t units[2];
    for (int y = 0; y < 2; ++y) {
        z.sh.rows[y] = 16 * z.form[y].nt * (z.form[y].many ? kKvWaves : 1);
        z.sh.fill[y] = z.form[y].many ? 512 : 768;
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

// Where the lists and the partial results do not fit 32-bit numbers, or nothing can be shared, the call is kv_attn's.
bool listed(const Lists& z, int64_t batch, int64_t rows)
{
    return batch > 1 && z.sh.ngroups > 0 && rows < kBehind && z.slots < (int64_t(1) << 31) && (int64_t)z.sh.room[0] + z.sh.room[1] < (int64_t(1) << 23);
}

// Whether sharing can gain what its launches cost.
bool gains(const KvAttn&) { return true; }

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

size_t kv_attn_shared_ws_bytes(int64_t total, int64_t batch, int64_t max_q, int heads, int kv_heads, int dim, int64_t ngroups)
{
    size_t need = kv_attn_ws_bytes(batch, max_q, heads, kv_heads, dim);
    for (int group : {32, 64, 128})
        for (int f32 = 0; f32 < 2; ++f32) {
            const Lists z = lists_of(total, batch, max_q, heads, kv_heads, dim, group, f32 != 0, ngroups);
            if (listed(z, batch, total * (heads / kv_heads))) need = std::max(need, layout_of(z, batch, kv_dp(dim)).end);
        }
    return need;
}

qe_status launch_kv_attn_shared(const KvAttn& call, const int32_t* groups, const int32_t* shared, int64_t ngroups, void* ws, bool always, hipStream_t s)
{
    KvAttn a = call;
    const int dp = kv_dp(a.c.dim);
    Lists z = lists_of(a.total, a.batch, a.max_q, a.heads, a.c.heads, a.c.dim, a.group, a.dtype == QE_F32, ngroups);
    if (!listed(z, a.batch, a.total * (a.heads / a.c.heads)) || !(always || gains(a))) return launch_kv_attn(a, ws, s);
    kv_attn_vec(a);
    const Layout l = layout_of(z, a.batch, dp);
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
    hipLaunchKernelGGL(kv_shared_plan_kernel, dim3(1), dim3(kScanThreads), 0, s, a, sh);
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
