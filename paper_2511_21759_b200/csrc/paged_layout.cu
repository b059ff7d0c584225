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
// Bound by latency: a chain of loads, one scan of four sums and a search; 16 requests take 3.5 us a call among others, 1000
// requests, long prompts among them, 9.7 us.  Over a pool of 8 bits the scales of the pages taken become the smallest, a block to a page, all
// layers (32 layers of 8 heads: 48 requests that take a page each 2.8 -> 3.5 us in a graph, a prompt of 4096 rows 2.5 -> 3.2, of 16 x 2000 6.0).
// Lengths that do not fit (negative, longer than a table
// row, more pages than there are, rows behind the length) change no table: there are no rows then, and the status word
// says why.
#include "paged.cuh"

namespace odb {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = kPagedMaxSeqs / kThreads;   // requests of a thread
constexpr int kScaleBlocks = 148;                // blocks at least, over a pool of 8 bits: pages may be taken for many more rows than the forward has

struct Sums {
    int row0[kPagedMaxSeqs + 1], take0[kPagedMaxSeqs + 1], give0[kPagedMaxSeqs + 1];
    int held[kPagedMaxSeqs], need[kPagedMaxSeqs];
    long long warp_sum[kThreads / 32][4];
    int bad;
};

// exclusive sums of four numbers over the block at once; every thread gets the totals
__device__ __forceinline__ void scan4(long long (&v)[4], long long (*warp_sum)[4], long long (&total)[4]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = v[k];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const long long y = __shfl_up_sync(0xffffffffu, x[k], d);
            if (lane >= d) x[k] += y;
        }
    if (lane == 31)
#pragma unroll
        for (int k = 0; k < 4; ++k) warp_sum[warp][k] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        long long before = 0;
        total[k] = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) {
            const long long t = warp_sum[w][k];
            if (w < warp) before += t;
            total[k] += t;
        }
        v[k] = before + x[k] - v[k];
    }
}

__global__ void __launch_bounds__(kThreads) paged_layout_kernel(const PagedLayoutArgs a) {
    __shared__ Sums sm;
    const int tid = threadIdx.x;
    pdl_launch_dependents();
    if (tid == 0) sm.bad = 0;
    __syncthreads();
    pdl_wait();

    const long long P = 1ll << a.page_shift, longest = static_cast<long long>(a.table_stride) << a.page_shift;
    const int per = (a.n_seqs + kThreads - 1) / kThreads, s0 = min(tid * per, a.n_seqs), s1 = min(s0 + per, a.n_seqs);
    long long at[4] = {0, 0, 0, 0}, all[4];        // rows, pages taken, pages given, pages held
    bool bad_arg = false;
    int counts[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        counts[i] = 0;
        const int s = s0 + i;
        if (i < per && s < s1) {
            const long long before = a.len_before[s], after = a.len_after[s], first = a.first[s], count = a.count[s];
            if (before < 0 || before > longest || after < 0 || after > longest || count < 0 || first < 0 || (count > 0 && first + count > after)) {
                bad_arg = true;
            } else {
                const long long held = (before + P - 1) >> a.page_shift, need = (after + P - 1) >> a.page_shift;
                sm.held[s] = static_cast<int>(held);
                sm.need[s] = static_cast<int>(need);
                counts[i] = static_cast<int>(count);
                at[0] += count;
                at[1] += max(0ll, need - held);
                at[2] += max(0ll, held - need);
                at[3] += held;
            }
        }
    }
    if (bad_arg) atomicExch(&sm.bad, ODB_ERR_ARG);
    scan4(at, sm.warp_sum, all);
    int bad = sm.bad;
    if (!bad && (all[3] > a.n_pages || all[3] + all[1] - all[2] > a.n_pages)) bad = ODB_ERR_WORKSPACE;
    if (!bad && all[0] > a.max_rows) bad = ODB_ERR_SHAPE;
    if (bad) {
        if (blockIdx.x == 0 && tid == 0) atomicExch(a.status, bad);
        all[0] = all[1] = all[2] = 0;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int s = s0 + i;
        if (i < per && s < s1) {
            sm.row0[s] = bad ? 0 : static_cast<int>(at[0]);
            if (!bad) {
                sm.take0[s] = static_cast<int>(at[1]);
                sm.give0[s] = static_cast<int>(at[2]);
                const int held = sm.held[s], need = sm.need[s];
                at[0] += counts[i];
                at[1] += max(0, need - held);
                at[2] += max(0, held - need);
            }
            if (blockIdx.x == 0) a.row_start[s] = sm.row0[s];
        }
    }
    const int n_rows = static_cast<int>(all[0]), T = static_cast<int>(all[1]), G = static_cast<int>(all[2]);
    const int n_free = a.n_pages - static_cast<int>(bad ? 0 : all[3]);
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
#pragma unroll 4
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
    if (a.scales) {
        // a block to a page: its scales become the smallest, under which what is left there of others counts as nothing
        const float least = __uint_as_float(static_cast<uint32_t>(kPagedLowExp + 127) << 23);
        for (int j = blockIdx.x; j < T; j += gridDim.x) {
            const int page = taken(j);
            if (page < 0 || page >= a.n_pages) continue;
            for (int i = tid; i < a.parts * a.page_scales; i += kThreads) {
                const int part = i / a.page_scales;
                a.scales[(static_cast<size_t>(part) * a.n_pages + page) * a.page_scales + (i - part * a.page_scales)] = least;
            }
        }
    }
}

}  // namespace

cudaError_t launch_paged_layout(const PagedLayoutArgs& a, cudaStream_t st) {
    const int rows = (a.max_rows + kThreads - 1) / kThreads, least = a.scales ? kScaleBlocks : 1, blocks = rows < least ? least : rows;
    return launch_kernel(paged_layout_kernel, dim3(blocks > 296 ? 296 : blocks), dim3(kThreads), 0, st, a);
}

}  // namespace odb
