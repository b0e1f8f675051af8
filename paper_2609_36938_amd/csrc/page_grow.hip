// Page tables and slot maps from the sessions' lengths.
//
// Session b holds the pages of its history entries, ceil(H_b / page_size), and
// needs ceil(C_b / page_size).  The new ones come off a free list in session
// order, so session b's first is entry head + sum over the sessions before it.
// One launch: every block sums the sessions before its rows by itself (8 bytes
// a session, from L2), scans the ones that its rows belong to, and gives each
// row its slot.  Every new page begins with exactly one appended entry, whose
// thread writes the table; the pages that other threads look up in the table
// are the history's, which no thread writes.  So no block waits for another.
#include "janus_device.hpp"
#include "janus_host.hpp"

namespace janus {

constexpr int GROW_THREADS = 256;  // rows of a block, and sessions scanned at a time

struct Growth {
    int had, fresh;  // pages of the history, pages to take
};
JANUS_DEV Growth growth(int M, int N, int es, int page_shift)
{
    // (rounded up without a sum: entries and pages may be near 2^31)
    auto pages = [&](int n) { return (n >> page_shift) + ((n & ((1 << page_shift) - 1)) != 0); };
    const int had = pages(entries_of(M, es));
    return {had, pages(entries_of(M + N, es)) - had};
}

// Sum over the block; every thread gets it.
JANUS_DEV int block_sum(int v, int *red)
{
    const int wave = threadIdx.x >> 6;
    v = __builtin_amdgcn_readlane(wave_sum_scan(v), 63);
    __syncthreads();
    red[wave] = v;
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3];
}

__global__ __launch_bounds__(GROW_THREADS) void page_grow(
    const int32_t *__restrict__ q_start, const int32_t *__restrict__ hist_len, int num_seqs, int es, int total_q,
    int page_shift, const int32_t *__restrict__ free_list, int free_len, const int32_t *__restrict__ free_head,
    int32_t *table, int pt_ld, int64_t *__restrict__ slots, int32_t *__restrict__ counts)
{
    __shared__ int sQ[GROW_THREADS], sM[GROW_THREADS], sHad[GROW_THREADS], sFirst[GROW_THREADS];
    __shared__ int red[GROW_THREADS / kWave];
    static_assert(GROW_THREADS == 4 * kWave, "block_sum adds four waves");
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r0 = blockIdx.x * GROW_THREADS, r1 = r0 + min(GROW_THREADS, total_q - r0);
    const bool live = tid < r1 - r0;
    const int row = live ? r0 + tid : 0;
    const int head = free_head ? *free_head : 0;
    int next = head;  // free list entry of the first page of the sessions scanned next
    int s0 = 0;       // first of them
    if (num_seqs > GROW_THREADS && blockIdx.x > 0) {
        // sessions that end before this block's rows: how many, and their pages
        int before = 0, pages = 0;
        for (int s = tid; s < num_seqs; s += GROW_THREADS) {
            const int a = q_start[s], e = q_start[s + 1];
            if (e <= r0) {
                ++before;
                pages += growth(hist_len[s], e - a, es, page_shift).fresh;
            }
        }
        s0 = block_sum(before, red);
        next += block_sum(pages, red);
    }
    int64_t slot = -1;
    bool open = live;  // no session found yet
    for (; s0 < num_seqs; s0 += GROW_THREADS) {
        const int s = s0 + tid;
        int a = 0x7fffffff, e = 0x7fffffff, M = 0;
        Growth g = {0, 0};
        if (s < num_seqs) {
            a = q_start[s];
            e = q_start[s + 1];
            M = hist_len[s];
            g = growth(M, e - a, es, page_shift);
        }
        const int incl = wave_sum_scan(g.fresh);
        __syncthreads();  // the last sessions' arrays are read
        if (lane == 63)
            red[wave] = incl;
        sQ[tid] = a;
        sM[tid] = M;
        sHad[tid] = g.had;
        __syncthreads();
        int below = next;
        for (int w = 0; w < wave; ++w)
            below += red[w];
        sFirst[tid] = below + incl - g.fresh;
        next += red[0] + red[1] + red[2] + red[3];
        __syncthreads();
        const int n = min(GROW_THREADS, num_seqs - s0);
        const int end = q_start[s0 + n];
        if (open && row < end) {
            open = false;
            int lo = 0, hi = n - 1;  // the last session that starts at or before the row
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (sQ[mid] <= row)
                    lo = mid;
                else
                    hi = mid - 1;
            }
            const int tokens = sM[lo] + (row - sQ[lo]) + 1;  // of the session up to this one
            const int entry = entries_of(tokens, es) - 1;
            if ((tokens & ((1 << es) - 1)) == 0) {
                const int j = entry >> page_shift, in = entry & ((1 << page_shift) - 1);
                int32_t *cell = table + (int64_t)(s0 + lo) * pt_ld + j;
                int page = -1;
                if (j < sHad[lo]) {
                    page = *cell;
                } else {
                    const int at = sFirst[lo] + (j - sHad[lo]);
                    if (at >= 0 && at < free_len)
                        page = free_list[at];
                    if (in == 0 && page >= 0)
                        *cell = page;
                }
                if (page >= 0)
                    slot = ((int64_t)page << page_shift) + in;
            }
        }
        if (end >= r1)
            break;  // (uniform) the later sessions have no row here
    }
    if (live)
        slots[row] = slot;
    // the last block has seen every session that appends
    if (blockIdx.x == gridDim.x - 1 && tid == 0) {
        const int want = next - head, left = max(0, free_len - head), taken = min(want, left);
        counts[0] = taken;
        counts[1] = head + taken;
        counts[2] = want - taken;
    }
}

}  // namespace janus

using namespace janus;

extern "C" int janus_page_grow(const janus_batch *b, int page_size, const int32_t *free_list, int free_len,
                               const int32_t *free_head, int32_t *page_table, int pt_ld, int64_t *slots,
                               int32_t *counts, void *stream)
{
    if (!batch_ok(b) || !pow2(page_size) || free_len < 0 || (free_len > 0 && !free_list) || !page_table || !slots ||
        !counts || !table_covers(b, pt_ld, page_size) || (free_head >= counts && free_head < counts + 3))
        return JANUS_ERR_INVALID_ARG;
    hipLaunchKernelGGL(page_grow, dim3(b->total_q > 0 ? ceil_div(b->total_q, GROW_THREADS) : 1), dim3(GROW_THREADS),
                       0, as_stream(stream), b->q_start, b->hist_len, b->num_seqs, b->entry_shift, b->total_q,
                       __builtin_ctz((unsigned)page_size), free_list, free_len, free_head, page_table, pt_ld, slots,
                       counts);
    return launch_status();
}
