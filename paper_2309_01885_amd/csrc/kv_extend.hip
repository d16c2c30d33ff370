// Pages and slots of a step of many sequences (qe.h).
//
// With exclusive sums over the sequences in their order (G: pages that go back, N: pages wanted, q: tokens) everything
// has its place at once: page r of those that go back lies at place top - 1 - r of the stack, top = free + sum G,
// page r of those that are taken comes from place top - 1 - r, and token i of the call belongs to the last b with
// q_b <= i.  Since the sums of N grow, the sequences that get their pages are those up to the first that does not.
//
// One workgroup does the sums (a thread a stretch of sequences) and the pages that go back; the tokens' slots, and with
// them the pages that are taken (each by the token that is first on it), are a thread a token.
//
// What bounds it is latency: a launch and three dependent loads, 2.7 to 3.3 us for a token of one sequence, 5 us for a step of 257
// sequences or 64 prompts of 2048 tokens, and 4 us for the launch that places the tokens of larger calls.
#include "kv_scan.h"

namespace qe {

namespace {

struct Change {
    int64_t tokens;
    int32_t old, now, held, want, give, need;
    bool wrong;
};

__device__ inline Change change_of(const KvExtend& a, int64_t b, bool report)
{
    Change c;
    const int64_t room = a.width * a.page;
    const int64_t count = a.counts[b];
    int64_t old = a.lengths[b], keep = a.keep ? a.keep[b] : 0;
    c.wrong = old < 0 || old > room || keep < 0 || keep > a.width;
    c.tokens = max(count, (int64_t)0);
    const int64_t now = max(old + count, (int64_t)0);
    c.wrong = c.wrong || now > min(room, (int64_t)0x7fffffff);
    if (c.wrong && report) set_status(a.status, QE_ERR_ARG);
    c.old = (int32_t)old;
    c.now = (int32_t)(c.wrong ? old : now);
    c.held = c.want = 0;
    if (!c.wrong) {
        // (32 bits: lengths are)
        c.held = max((int32_t)(((uint32_t)old + (uint32_t)a.page - 1) / (uint32_t)a.page), (int32_t)keep);
        c.want = max((int32_t)(((uint32_t)now + (uint32_t)a.page - 1) / (uint32_t)a.page), (int32_t)keep);
    }
    c.give = max(c.held - c.want, 0);
    c.need = max(c.want - c.held, 0);
    return c;
}

// The sequence of token i: the last b with q_start[b] <= i (batch where it is none's).
template <class I> __device__ inline int64_t sequence_of(const I* q_start, int64_t batch, int64_t i)
{
    return last_at_most(q_start, batch + 1, i);
}

__device__ inline void place(const KvExtend& a, int64_t i, int64_t b, const KvExtendSeq* seqs, int64_t start, int64_t top)
{
    int64_t slot = -1;
    int32_t pos = -1;
    if (b < a.batch) {
        const KvExtendSeq s = seqs[b];
        const int64_t at = s.old + (i - start);
        pos = (int32_t)min(at, (int64_t)0x7fffffff);
        if (s.first >= 0) {
            const uint32_t j = (uint32_t)at / (uint32_t)a.page, in = (uint32_t)at - j * (uint32_t)a.page;
            int32_t page;
            if ((int32_t)j < s.held) {
                page = a.table[b * a.width + j];
            } else {
                // (a stack that would pass its end has lost what lies there)
                const int64_t from = top - 1 - (s.first + (int64_t)((int32_t)j - s.held));
                page = from < a.num_pages ? a.free[from] : -1;
                if (in == 0) a.table[b * a.width + j] = page;
            }
            if (page >= 0 && page < a.num_pages) slot = (int64_t)page * a.page + in;
            else set_status(a.status, QE_ERR_ARG);
        } else {
            pos = s.first == -1 ? pos : -1;
        }
    }
    a.slots[i] = slot;
    a.positions[i] = pos;
}

__global__ __launch_bounds__(kScanThreads) void kv_extend_kernel(KvExtend a, bool fill)
{
    __shared__ ScanLds<3> lds;
    __shared__ int64_t wave_taken[kScanThreads / 64];
    __shared__ int32_t start[kScanThreads + 1];
    __shared__ KvExtendSeq seqs[kScanThreads];
    __shared__ int2 back[kScanThreads];                  // pages that go back before a sequence's, and the first of its own
    const int tid = threadIdx.x, lane = tid & 63, threads = blockDim.x;
    const int64_t per = (a.batch + threads - 1) / threads;
    const int64_t b0 = min(tid * per, a.batch), b1 = min(b0 + per, a.batch);
    int64_t free_count = *a.free_count;
    int64_t sum[3] = {0, 0, 0}, own[3], all[3];          // tokens, pages that go back, pages wanted
    Change c = {};
    for (int64_t b = b0; b < b1; ++b) {
        c = change_of(a, b, true);
        sum[0] += c.tokens;
        sum[1] += c.give;
        sum[2] += c.need;
    }
#pragma unroll
    for (int n = 0; n < 3; ++n) own[n] = sum[n];
    scan_add(sum, lds, all);
    int64_t token = sum[0] - own[0], given = sum[1] - own[1], needed = sum[2] - own[2];
    const bool bad = free_count < 0 || free_count > a.num_pages;
    free_count = max((int64_t)0, min(free_count, a.num_pages));
    const int64_t top = free_count + all[1], have = min(top, a.num_pages);
    if (tid == 0 && (bad || top > a.num_pages || all[0] > a.total)) set_status(a.status, QE_ERR_ARG);

    // pages that go back: a thread a page; of more sequences than threads a wave's together, a sequence after the other
    if (all[1] > 0 && per == 1 && all[1] <= 0x7fffffff) {
        back[tid] = make_int2((int32_t)given, c.want);
        __syncthreads();
        for (int32_t r = tid; r < (int32_t)all[1]; r += threads) {
            int lo = 0, hi = (int)a.batch;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (back[mid].x <= r) lo = mid;
                else hi = mid;
            }
            int32_t* const page = a.table + lo * a.width + back[lo].y + (r - back[lo].x);
            if (top - 1 - r < a.num_pages) a.free[top - 1 - r] = *page;
            *page = -1;
        }
    } else {
        for (int64_t n = 0; all[1] > 0 && n < per; ++n) {
            const int64_t b = b0 + n;
            if (per > 1 && b < b1) c = change_of(a, b, false);
            const int32_t mine = b < b1 ? c.give : 0;
            uint64_t left = __ballot(mine > 0);
            while (left) {
                const int l = __builtin_ctzll(left);
                left &= left - 1;
                int32_t* const row = a.table + __shfl(b, l) * a.width + __shfl(c.want, l);
                const int64_t at = top - 1 - __shfl(given, l);
                const int32_t count = __shfl(mine, l);
                for (int32_t j = lane; j < count; j += 64) {
                    if (at - j < a.num_pages) a.free[at - j] = row[j];
                    row[j] = -1;
                }
            }
            given += mine;
        }
    }

    // who gets the pages
    int64_t taken = 0;
    for (int64_t b = b0; b < b1; ++b) {
        if (per > 1) c = change_of(a, b, false);
        const int64_t end = token + c.tokens, last = needed + c.need;
        // (past the rows of this call nothing is written: the sequence stays as it is, its tokens are nobody's.  One without rows
        // is none of those, whatever came before it: its pages may have gone back already)
        const bool got = !c.wrong && (c.need == 0 || last <= have) && (c.tokens == 0 || end <= a.total);
        KvExtendSeq s;
        s.old = c.old;
        s.held = c.held;
        s.first = got ? (int32_t)min(needed, (int64_t)0x7fffffff) : c.wrong ? -2 : -1;
        if (got && c.need) taken = last;
        s.start = (int32_t)min(token, a.total);
        a.q_start[b] = s.start;
        if (got) a.lengths[b] = c.now;
        if (fill) {
            seqs[b] = s;
            start[b] = s.start;
        } else {
            a.seqs[b] = s;
        }
        token = end;
        needed = last;
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) taken = max(taken, __shfl_xor(taken, m));
    if (lane == 0) wave_taken[tid >> 6] = taken;
    if (tid == 0 && fill) start[a.batch] = (int32_t)min(all[0], a.total);
    __syncthreads();                                     // (also: the pages that go back are there)
    if (tid == 0) {
        for (int w = 1; w < threads / 64; ++w) taken = max(taken, wave_taken[w]);
        a.q_start[a.batch] = (int32_t)min(all[0], a.total);
        if (a.lacking) *a.lacking = (int32_t)min(max(all[2] - have, (int64_t)0), (int64_t)0x7fffffff);
        *a.free_count = (int32_t)(have - taken);
        if (!fill) *a.top = top;
    }
    if (!fill) return;
    for (int64_t i = tid; i < a.total; i += threads) {
        const int64_t b = sequence_of(start, a.batch, i);
        place(a, i, b, seqs, b < a.batch ? start[b] : 0, top);
    }
}

// The tokens of larger calls.
constexpr int kFillTokens = 256, kFillStarts = 4096;
__global__ __launch_bounds__(kFillTokens) void kv_fill_kernel(KvExtend a)
{
    __shared__ int32_t start[kFillStarts + 1];
    const bool near = a.batch <= kFillStarts;
    if (near) {
        for (int64_t b = threadIdx.x; b <= a.batch; b += kFillTokens) start[b] = a.q_start[b];
        __syncthreads();
    }
    const int64_t top = *a.top, i = (int64_t)blockIdx.x * kFillTokens + threadIdx.x;
    if (i >= a.total) return;
    const int64_t b = near ? sequence_of(start, a.batch, i) : sequence_of(a.q_start, a.batch, i);
    place(a, i, b, a.seqs, b < a.batch ? (near ? start[b] : a.q_start[b]) : 0, top);
}

// Calls of at most this many tokens (and a sequence a thread) are one launch.  us of a call and its undoing, as one launch / two:
// one sequence, 1024 tokens 8.0 / 9.1, 2048 8.6 / 9.2, 4096 10.1 / 10.0, 8192 12.9 / 10.3; 16 sequences, 1568 9.2 / 9.5, 3136 11.1 /
// 10.5; 1000 sequences, 1000 12.4 / 15.3, 2000 13.5 / 15.9, 3500 15.8 / 15.7.
constexpr int64_t kFillInPlace = 2048;

}  // namespace

size_t kv_extend_ws_bytes(int64_t batch) { return 2 * kStatusBytes + align256(batch * sizeof(KvExtendSeq)); }

qe_status launch_kv_extend(const KvExtend& call, void* ws, hipStream_t s)
{
    KvExtend a = call;
    a.top = reinterpret_cast<int64_t*>(static_cast<char*>(ws) + kStatusBytes);
    a.seqs = reinterpret_cast<KvExtendSeq*>(static_cast<char*>(ws) + 2 * kStatusBytes);
    const bool fill = a.batch <= kScanThreads && a.total <= kFillInPlace;
    hipLaunchKernelGGL(kv_extend_kernel, dim3(1), dim3(scan_threads(std::max(std::min(a.batch * a.width, a.batch + kScanThreads), fill ? a.total : 0))), 0, s, a, fill);
    if (!fill && a.total > 0) hipLaunchKernelGGL(kv_fill_kernel, dim3((unsigned)cdiv(a.total, kFillTokens)), dim3(kFillTokens), 0, s, a);
    return hipGetLastError() == hipSuccess ? QE_OK : QE_ERR_HIP;
}

}  // namespace qe
