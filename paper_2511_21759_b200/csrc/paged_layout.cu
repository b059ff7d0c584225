// Block tables and slot maps of a forward, from its requests' lengths.
//
// A request of len tokens holds ceil(len / page) pages, the front entries of its table row.  n = n_pages - sum(held) pages
// are free, the front entries of the free list.  The pages given back (requests in order, then pages in order) go behind
// them, the pages taken come from the end: page j that is taken (requests in order, then pages in order) is entry
// n + G - 1 - j of that list.  Every table entry, free-list entry and row follows from prefix sums over the requests, so
// every block forms the sums for itself and takes its share of the rows: one launch, no order between blocks.  What is
// read (the first n free entries, the tails given back) and what is written (new tails, free entries from n on) never
// meet.
//
// Bound by latency: a chain of loads, three scans and a search.  Lengths that do not fit (negative, longer than a table
// row, more pages than there are, rows behind the length) change no table: there are no rows then, and the status word
// says why.
#include "paged.cuh"

namespace odb {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = kPagedMaxSeqs / kThreads;   // requests of a thread

struct Sums {
    int row0[kPagedMaxSeqs + 1], take0[kPagedMaxSeqs + 1], give0[kPagedMaxSeqs + 1];
    int held[kPagedMaxSeqs], need[kPagedMaxSeqs];
    long long warp_sum[32];
    int bad;
};

__global__ void __launch_bounds__(kThreads) paged_layout_kernel(const PagedLayoutArgs a) {
    __shared__ Sums sm;
    const int tid = threadIdx.x;
    pdl_launch_dependents();
    if (tid == 0) sm.bad = 0;
    __syncthreads();
    pdl_wait();

    const long long P = 1ll << a.page_shift, longest = static_cast<long long>(a.table_stride) << a.page_shift;
    const int per = (a.n_seqs + kThreads - 1) / kThreads, s0 = min(tid * per, a.n_seqs), s1 = min(s0 + per, a.n_seqs);
    long long rows = 0, take = 0, give = 0, held_all = 0;
    bool bad_arg = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int s = s0 + i;
        if (i >= per || s >= s1) break;
        const long long before = a.len_before[s], after = a.len_after[s], first = a.first[s], count = a.count[s];
        if (before < 0 || before > longest || after < 0 || after > longest || count < 0 || first < 0 || (count > 0 && first + count > after)) {
            bad_arg = true;
            break;
        }
        const long long held = (before + P - 1) >> a.page_shift, need = (after + P - 1) >> a.page_shift;
        sm.held[s] = static_cast<int>(held);
        sm.need[s] = static_cast<int>(need);
        rows += count;
        take += max(0ll, need - held);
        give += max(0ll, held - need);
        held_all += held;
    }
    if (bad_arg) atomicExch(&sm.bad, ODB_ERR_ARG);
    long long all_rows, all_take, all_give, all_held;
    long long row0 = paged_block_scan<kThreads>(rows, sm.warp_sum, all_rows);
    long long take0 = paged_block_scan<kThreads>(take, sm.warp_sum, all_take);
    long long give0 = paged_block_scan<kThreads>(give, sm.warp_sum, all_give);
    paged_block_scan<kThreads>(held_all, sm.warp_sum, all_held);
    int bad = sm.bad;
    if (!bad && (all_held > a.n_pages || all_held + all_take - all_give > a.n_pages)) bad = ODB_ERR_WORKSPACE;
    if (!bad && all_rows > a.max_rows) bad = ODB_ERR_SHAPE;
    if (bad) {
        if (blockIdx.x == 0 && tid == 0) atomicExch(a.status, bad);
        all_rows = all_take = all_give = 0;
    }
    for (int s = s0; s < s1; ++s) {
        if (bad) {
            sm.row0[s] = 0;
        } else {
            sm.row0[s] = static_cast<int>(row0);
            sm.take0[s] = static_cast<int>(take0);
            sm.give0[s] = static_cast<int>(give0);
            const int held = sm.held[s], need = sm.need[s];
            row0 += a.count[s];
            take0 += max(0, need - held);
            give0 += max(0, held - need);
        }
        if (blockIdx.x == 0) a.row_start[s] = sm.row0[s];
    }
    const int n_rows = static_cast<int>(all_rows), T = static_cast<int>(all_take), G = static_cast<int>(all_give);
    const int n_free = a.n_pages - static_cast<int>(bad ? 0 : all_held);
    if (tid == 0) {
        sm.row0[a.n_seqs] = n_rows;
        sm.take0[a.n_seqs] = T;
        sm.give0[a.n_seqs] = G;
        if (blockIdx.x == 0) a.row_start[a.n_seqs] = n_rows;
    }
    __syncthreads();

    auto entry = [&](int s, int i) { return a.table + static_cast<size_t>(s) * a.table_stride + i; };
    auto given = [&](int g) {                     // page g that is given back
        const int s = paged_upper(sm.give0, a.n_seqs + 1, g);
        return *entry(s, sm.need[s] + g - sm.give0[s]);
    };
    auto taken = [&](int j) {                     // page j that is taken
        const int i = n_free + G - 1 - j;
        return i < n_free ? a.free_pages[i] : given(i - n_free);
    };
    const int step = gridDim.x * kThreads, t0 = blockIdx.x * kThreads + tid;
    for (int r = t0; r < a.max_rows; r += step) {
        int seq = -1, pos = -1, slot = -1;
        if (r < n_rows) {
            seq = paged_upper(sm.row0, a.n_seqs + 1, r);
            pos = a.first[seq] + r - sm.row0[seq];
            const int i = pos >> a.page_shift;
            const int page = i < sm.held[seq] ? *entry(seq, i) : taken(sm.take0[seq] + i - sm.held[seq]);
            if (page >= 0 && page < a.n_pages) slot = (page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
            else atomicExch(a.status, ODB_ERR_STATE);   // the table or the free list is not one that these lengths go with
        }
        a.row_seq[r] = seq;
        a.row_pos[r] = pos;
        a.row_slot[r] = slot;
    }
    for (int j = t0; j < T; j += step) {
        const int s = paged_upper(sm.take0, a.n_seqs + 1, j);
        *entry(s, sm.held[s] + j - sm.take0[s]) = taken(j);
    }
    for (int g = t0; g < G - T; g += step) a.free_pages[n_free + g] = given(g);
}

}  // namespace

cudaError_t launch_paged_layout(const PagedLayoutArgs& a, cudaStream_t st) {
    const int blocks = (a.max_rows + kThreads - 1) / kThreads;
    return launch_kernel(paged_layout_kernel, dim3(blocks < 1 ? 1 : blocks > 296 ? 296 : blocks), dim3(kThreads), 0, st, a);
}

}  // namespace odb
