// Pages and slots of a step of many sequences (qe.h).
//
// With exclusive sums over the sequences in their order (G: pages that go back, N: pages wanted, q: tokens) everything
// has its place at once: page r of those that go back lies at place top - 1 - r of the stack, top = free + sum G,
// page r of those that are taken comes from place top - 1 - r, and token i of the call belongs to the last b with
// q_b <= i.  Since the sums of N grow, the sequences that get their pages are those up to the first that does not.
//
// One workgroup does the sums (a thread a stretch of sequences) and the pages that go back; the tokens' slots, and with
// them the pages that are taken (each by the token that is first on it), are a thread a token.
#include "kv_scan.h"

namespace qe {

namespace {

struct Change {
    int64_t tokens, give, need;
    int32_t old, now, held, want, keep;
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
    c.keep = (int32_t)keep;
    c.held = c.want = 0;
    if (!c.wrong) {
        c.held = (int32_t)max((old + a.page - 1) / a.page, keep);
        c.want = (int32_t)max((now + a.page - 1) / a.page, keep);
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
    __shared__ int64_t part[4][kScanThreads / 64];
    __shared__ int32_t start[kScanThreads + 1];
    __shared__ KvExtendSeq seqs[kScanThreads];
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t per = (a.batch + kScanThreads - 1) / kScanThreads;
    const int64_t b0 = min(tid * per, a.batch), b1 = min(b0 + per, a.batch);
    int64_t tokens = 0, give = 0, need = 0;
    Change c = {};
    for (int64_t b = b0; b < b1; ++b) {
        c = change_of(a, b, true);
        tokens += c.tokens;
        give += c.give;
        need += c.need;
    }
    int64_t all_tokens, all_give, all_need;
    int64_t token = scan_add(tokens, part[0], all_tokens) - tokens;
    int64_t given = scan_add(give, part[1], all_give) - give;
    int64_t needed = scan_add(need, part[2], all_need) - need;
    int64_t held_free = *a.free_count;
    const bool bad = held_free < 0 || held_free > a.num_pages;
    held_free = max((int64_t)0, min(held_free, a.num_pages));
    const int64_t top = held_free + all_give, have = min(top, a.num_pages);
    if (tid == 0 && (bad || top > a.num_pages || all_tokens > a.total)) set_status(a.status, QE_ERR_ARG);

    // pages that go back: a wave moves its threads' pages together, a sequence after the other
    for (int64_t n = 0; n < per; ++n) {
        const int64_t b = b0 + n;
        if (per > 1 && b < b1) c = change_of(a, b, false);
        const int64_t mine = b < b1 ? c.give : 0;
        uint64_t left = __ballot(mine > 0);
        while (left) {
            const int l = __builtin_ctzll(left);
            left &= left - 1;
            const int64_t row = __shfl(b, l) * a.width, rank = __shfl(given, l), from = __shfl(c.want, l), count = __shfl(mine, l);
            for (int64_t j = lane; j < count; j += 64) {
                const int64_t at = top - 1 - (rank + j);
                if (at < a.num_pages) a.free[at] = a.table[row + from + j];
                a.table[row + from + j] = -1;
            }
        }
        given += mine;
    }

    // who gets the pages
    int64_t taken = 0;
    for (int64_t b = b0; b < b1; ++b) {
        if (per > 1) c = change_of(a, b, false);
        const int64_t end = token + c.tokens, last = needed + c.need;
        // (past the rows of this call nothing is written: the sequence stays as it is, its tokens are nobody's)
        const bool got = !c.wrong && (c.need == 0 || last <= have) && end <= a.total;
        KvExtendSeq s;
        s.old = c.old;
        s.held = c.held;
        s.first = got ? (int32_t)min(needed, (int64_t)0x7fffffff) : c.wrong ? -2 : -1;
        if (got) taken = max(taken, c.need ? last : 0);
        const int32_t from = (int32_t)min(token, a.total);
        s.start = from;
        a.q_start[b] = from;
        if (got) a.lengths[b] = c.now;
        if (fill) {
            seqs[b] = s;
            start[b] = from;
        } else {
            a.seqs[b] = s;
        }
        token = end;
        needed = last;
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) taken = max(taken, __shfl_xor(taken, m));
    if (lane == 0) part[3][tid >> 6] = taken;
    __syncthreads();                                     // (also: every thread has read free_count, and the pages that go back are there)
    if (tid == 0) {
#pragma unroll
        for (int w = 0; w < kScanThreads / 64; ++w) taken = max(taken, part[3][w]);
        const int32_t end = (int32_t)min(all_tokens, a.total);
        a.q_start[a.batch] = end;
        start[fill ? a.batch : 0] = end;
        if (a.lacking) *a.lacking = (int32_t)min(max(all_need - have, (int64_t)0), (int64_t)0x7fffffff);
        *a.free_count = (int32_t)(have - taken);
        if (!fill) *a.top = top;
    }
    if (!fill) return;
    __syncthreads();
    for (int64_t i = tid; i < a.total; i += kScanThreads) {
        const int64_t b = sequence_of(start, a.batch, i);
        place(a, i, b, seqs, b < a.batch ? start[b] : 0, top);
    }
}

// The tokens of larger calls: 1024 a workgroup.
constexpr int kFillTokens = 1024, kFillStarts = 4096;
__global__ __launch_bounds__(256) void kv_fill_kernel(KvExtend a)
{
    __shared__ int32_t start[kFillStarts + 1];
    const bool near = a.batch <= kFillStarts;
    if (near) {
        for (int64_t b = threadIdx.x; b <= a.batch; b += 256) start[b] = a.q_start[b];
        __syncthreads();
    }
    const int64_t top = *a.top, first = (int64_t)blockIdx.x * kFillTokens;
#pragma unroll
    for (int n = 0; n < kFillTokens / 256; ++n) {
        const int64_t i = first + 256 * n + threadIdx.x;
        if (i >= a.total) return;
        const int64_t b = near ? sequence_of(start, a.batch, i) : sequence_of(a.q_start, a.batch, i);
        place(a, i, b, a.seqs, b < a.batch ? (near ? start[b] : a.q_start[b]) : 0, top);
    }
}

// Calls of at most this many tokens (and a sequence a thread) are one launch.
constexpr int64_t kFillInPlace = 2048;

}  // namespace

size_t kv_extend_ws_bytes(int64_t batch) { return 2 * kStatusBytes + align256(batch * sizeof(KvExtendSeq)); }

qe_status launch_kv_extend(const KvExtend& call, void* ws, hipStream_t s)
{
    KvExtend a = call;
    a.top = reinterpret_cast<int64_t*>(static_cast<char*>(ws) + kStatusBytes);
    a.seqs = reinterpret_cast<KvExtendSeq*>(static_cast<char*>(ws) + 2 * kStatusBytes);
    const bool fill = a.batch <= kScanThreads && a.total <= kFillInPlace;
    hipLaunchKernelGGL(kv_extend_kernel, dim3(1), dim3(kScanThreads), 0, s, a, fill);
    if (!fill && a.total > 0) hipLaunchKernelGGL(kv_fill_kernel, dim3((unsigned)cdiv(a.total, kFillTokens)), dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? QE_OK : QE_ERR_HIP;
}

}  // namespace qe
