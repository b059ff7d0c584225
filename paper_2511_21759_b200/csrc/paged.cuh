// Declarations shared by the paged-cache translation units: the handle, the launchers' arguments and the walk over the
// attention's work, which the kernels of few and of many rows have in common.
#pragma once

#include <cuda_fp16.h>

#include "attention_tc.cuh"

namespace odb {

constexpr int kPagedMaxSeqs = 1024;        // requests of one forward
constexpr int kPagedMaxCtas = 1216;        // CTAs of an attention launch, at most: four waves of two on each of the 148 SMs
constexpr int kPagedPartRows = 304 * 128;  // rows that the workspace holds of all CTAs' first or last items, whatever the kernel
constexpr int kPagedMaxParts = 2;          // unfinished segments a CTA leaves behind: of its first item and of its last
constexpr int kPagedUnlimited = 1 << 30;   // a window side without limit; lengths and positions stay below it

// ---- layout (paged_layout.cu) ----
struct PagedLayoutArgs {
    const int32_t *len_before, *len_after, *first, *count;
    int32_t *table, *free_pages;
    int32_t *row_start, *row_seq, *row_pos, *row_slot;
    int n_seqs, max_rows, page_shift, n_pages, table_stride;
    int* status;
    float* scales;                                        // [parts][n_pages][page_scales], null: a pool of bf16
    int parts, page_scales;                               // K and V of every layer; scales of a page in one of them
};
cudaError_t launch_paged_layout(const PagedLayoutArgs& a, cudaStream_t st);

// ---- norm, rotation and store (paged_store.cu) ----
struct PagedStoreArgs {
    const __nv_bfloat16 *q, *k, *v;
    long long q_stride, k_stride, v_stride, out_stride;   // elements from row to row
    __nv_bfloat16* q_out;
    const float *q_gain, *k_gain;                         // null: no norm
    const unsigned long long* turns;                      // fractions of a turn per position, [rot / 2]
    float magnitude, eps;
    const int32_t *row_pos, *row_slot;
    __nv_bfloat16 *k_pool, *v_pool;                       // this layer's
    int rows, H, KV, HD, rot, interleaved, page_shift, n_pages;
};
cudaError_t launch_paged_store(const PagedStoreArgs& a, cudaStream_t st);

// ---- pools of 8 bits: e4m3 and a scale, a power of two, for each block of 16 positions of a head (paged_e4m3_store.cu) ----
constexpr int kPagedBlock = ODB_PAGED_SCALE_BLOCK;
constexpr int kPagedLowExp = ODB_PAGED_LEAST_SCALE, kPagedHighExp = 119;   // of scales: what the codes stand for is then a number of bf16
struct PagedE4m3StoreArgs {
    PagedStoreArgs rows;                                  // KV = 0: as units it has those of q
    const int32_t *row_seq, *len;
    unsigned char *k_pool, *v_pool;                       // this layer's
    float *k_scales, *v_scales;
    int KV, n_seqs, window, heads;                        // window: rows in which a warp looks for the beginnings of blocks, 1 or 16; heads: of a unit
};
cudaError_t launch_paged_e4m3_store(const PagedE4m3StoreArgs& a, cudaStream_t st);

// ---- rows back from the pool (paged_load.cu) ----
struct PagedLoadArgs {
    const unsigned char *k_pool, *v_pool;                 // this layer's: codes, or bf16 where there are no scales
    const float *k_scales, *v_scales;
    const int32_t* row_slot;
    __nv_bfloat16 *k_out, *v_out;
    long long k_stride, v_stride;
    int rows, KV, HD, page_shift, n_pages;
    int per_row, block_rows;                              // pieces of 8 values of a row, K and V; rows of a block (the launcher's)
};
cudaError_t launch_paged_load(PagedLoadArgs a, cudaStream_t st);

// ---- attention (paged_attention.cu) ----
// n / d for 0 <= n < 2^31 by a product: with l = ceil(log2 d) and m = floor(2^(31 + l) / d) + 1, which fits 32 bits, n m 2^-(31 + l)
// exceeds n / d by less than 1 / d (Granlund and Montgomery, PLDI 1994).
struct PagedDiv {
    unsigned int mul, shift;
    __host__ static PagedDiv by(unsigned int d) {
        unsigned int l = 0;
        while ((1ull << l) < d) ++l;
        return PagedDiv{static_cast<unsigned int>((1ull << (31 + l)) / d + (d == 1 ? 0 : 1)), 31 + l};
    }
#ifdef __CUDACC__
    __device__ __forceinline__ int operator()(int n) const {
        return static_cast<int>((static_cast<unsigned long long>(static_cast<unsigned int>(n)) * mul) >> shift);
    }
#endif
};

// An item that begins in a CTA and ends in CTA `last_cta`: its rows, or none.
struct PagedShared {
    int row0, head, first_idx, rows, last_cta;
};

struct PagedAttnArgs {
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    float* lse;                                           // null: not wanted
    long long q_stride, out_stride;
    const int32_t *table, *len, *first, *row_start;
    int n_seqs, max_rows, H, KV, G, page_shift, n_pages, table_stride;
    const unsigned short* pool;                           // bf16 [pool_rows][hd]
    int k_row0, v_row0, pool_rows;                        // rows of hd values of the whole pool: this layer's K, its V, all of them
    int left, right, sinks;
    float scale_log2;                                     // softmax scale x log2(e)
    int* status;
    unsigned int* arrivals;                               // [kPagedMaxCtas], zero between launches
    float* part_o;                                        // [ctas][2][part_rows][HD]; many rows: [ctas][2][Q tile][HD / 4][128 rows][4]
    float* part_ml;                                       // [ctas][2][part_rows][2]
    int negate;                                           // many rows: the scale's sign, which scale_log2 no longer has
    int at_once;                                          // CTAs that run at one time
    int part_rows;                                        // rows of a tile
    struct PagedShared* shared;                           // [kPagedMaxCtas], of the last launch that adds up in a kernel of its own
    PagedDiv by_group, by_rows, by_once;                  // divisions by G, by the packed rows of an item, by at_once
    int tile_rows, tile_tokens;                           // many rows: packed rows of an item, query rows of a Q tile
    const float* scales;                                  // pools of 8 bits: [pool_rows / 16]
};
// the pool's two maps: boxes of whole rows, and of 64 values of a row
struct PagedMaps {
    CUtensorMap rows, atoms;
};
// The kernel of an attention over n_seqs requests with max_rows rows together, `longest` positions in a table row: 0 the few rows', 1 or 2
// Q tiles of the many rows', -1: none, its sums would pass 32 bits.  max_new: rows of the longest request, a hint; 0: not known.
int paged_attention_kernel_of(int n_seqs, int max_rows, int max_new, int group, int kv_heads, long long longest, long long out_stride);
cudaError_t launch_paged_attention(PagedAttnArgs a, const PagedMaps& maps, int hd, int q_tiles, int sms, cudaStream_t st);
// many packed rows on the tensor cores (paged_attention_tc.cu); q_tiles: Q tiles of 128 rows a CTA takes
cudaError_t launch_paged_attention_tc(PagedAttnArgs a, const PagedMaps& maps, int hd, int q_tiles, int sms, cudaStream_t st);
constexpr int kPagedTcMaxGroup = 128;   // heads of a group that fit a Q tile
constexpr int kPagedTcItem = 3;         // key tiles that an item costs the many rows' kernel beside its own
size_t paged_part_bytes(int hd);

// ---- attention over a pool of 8 bits (paged_e4m3_attention.cu) ----
// The kernel: 8 or 16, the packed rows of the few rows' items; 1, the many rows' over the codes; 2, that of bf16 with two Q tiles, over a copy of
// the pages (room: there is memory for one); -1: none, its sums would pass 32 bits.
int paged_e4m3_attention_kernel_of(int n_seqs, int max_rows, int max_new, int group, int kv_heads, long long longest, long long out_stride, bool room);
cudaError_t launch_paged_e4m3_attention_tc(PagedAttnArgs a, const CUtensorMap& map, int hd, int sms, cudaStream_t st);
cudaError_t launch_paged_e4m3_attention(PagedAttnArgs a, const CUtensorMap& map, int hd, int kernel, int sms, cudaStream_t st);
// The pages that an attention's rows see, as bf16 in their places of one layer's K and V (paged_load.cu).
cudaError_t launch_paged_expand(const PagedAttnArgs& a, __nv_bfloat16* layer, int layer_rows, int hd, cudaStream_t st);

#ifdef __CUDACC__
// ---------------------------------------------------------------------------------------
// The attention's work.  An item is one tile of up to a.tile_rows packed rows (row i of a request and query head g of the
// group: packed row i * G + g) of one K/V head; its keys are cut into tiles of KT positions.  All key tiles of all
// items in the order head, request, row tile, key tile are one line, which is divided evenly over the CTAs: whatever
// the lengths, every CTA gets the same share.  An item's first key tile has E units in front of it that stand for what
// an item costs beside its tiles (fetching Q, writing results): a share that ends among them leaves the item to the next.
// ---------------------------------------------------------------------------------------

struct PagedSeq {
    int row0, n, first, len, n_rt;
    __device__ __forceinline__ void tiles(const PagedAttnArgs& a) { n_rt = a.by_rows(n * a.G + a.tile_rows - 1); }
};

__device__ __forceinline__ PagedSeq paged_seq(const PagedAttnArgs& a, int s) {
    PagedSeq q;
    const int r0 = min(max(a.row_start[s], 0), a.max_rows), r1 = min(a.row_start[s + 1], a.max_rows);
    q.row0 = r0;
    q.n = max(r1 - r0, 0);
    q.first = min(max(a.first[s], -kPagedUnlimited), kPagedUnlimited - 1);
    // the table bounds the keys whatever the length says (its rows hold fewer than 2^30 positions)
    q.len = min(max(a.len[s], 0), a.table_stride << a.page_shift);
    q.tiles(a);
    return q;
}

// Rows follow one another within those of the call.  Every sum below, the launcher's grid and the count of an item's parts rest on it:
// requests whose rows overlap may have more work than the grid has CTAs for, and the item that is cut at its end would wait for parts
// that nobody brings, in this launch and in the next ones.
__device__ __forceinline__ bool paged_rows_follow(const PagedAttnArgs& a, int s) {
    const int r0 = a.row_start[s], r1 = a.row_start[s + 1];
    return 0 <= r0 && r0 <= r1 && r1 <= a.max_rows;
}

// The length is one that the table has entries for (where not, it is cut, and the status word says so).
__device__ __forceinline__ bool paged_length_fits(const PagedAttnArgs& a, int s) {
    const int len = a.len[s];
    return 0 <= len && len <= a.table_stride << a.page_shift;
}

// The key tiles of a row tile: `sink_tiles` from the front, the others from tile `first_tile` on; `n` of them, at least
// one (an item without a visible key still writes its rows).  Positions from `hi` on are seen by no row, nor are those
// of [sinks, lo).
struct PagedKeys {
    int lo, hi, sink_tiles, first_tile, n;
    __device__ __forceinline__ int tile(int t) const { return t < sink_tiles ? t : first_tile + t - sink_tiles; }
};

template <int KT>
__device__ __forceinline__ PagedKeys paged_keys(const PagedAttnArgs& a, const PagedSeq& q, int rt) {
    const int i0 = a.by_group(rt * a.tile_rows), i1 = min(q.n - 1, a.by_group(rt * a.tile_rows + a.tile_rows - 1));
    PagedKeys k;
    // first + i + right + 1 stays below 2^30 + 2^30 + rows and may pass 2^31: as unsigned it does not wrap
    k.hi = max(0, q.first + i1 < 0 ? q.first + i1 + a.right + 1
                                   : static_cast<int>(min(static_cast<unsigned>(q.len), static_cast<unsigned>(q.first + i1) + a.right + 1u)));
    k.hi = min(k.hi, q.len);
    k.lo = max(0, min(k.hi, q.first + i0 - a.left));
    const int end = (k.hi + KT - 1) / KT;
    k.first_tile = k.lo < k.hi ? k.lo / KT : end;
    k.sink_tiles = min((min(a.sinks, k.hi) + KT - 1) / KT, k.first_tile);
    k.n = max(1, k.sink_tiles + end - k.first_tile);
    return k;
}

// The line's division: `waves` times as many CTAs as run at one time, of shares that grow smaller from wave to wave (the sizes are
// of each wave's CTAs; a line that ends early leaves the later ones without work).
constexpr int kPagedWaves = 4;
struct PagedShares {
    int size[kPagedWaves], at_once;
    __device__ __forceinline__ void divide(int total, int waves, int min_units, int full_units, const PagedDiv& by_once) {
        // 45, 27, 17 and 11 of a hundred: see the launcher of the few rows' kernel
        constexpr int kPart[kPagedWaves] = {115, 69, 44, 28};
        const int most = by_once(total + at_once - 1), least = max(min_units, min(full_units, most));
        int left = total;
#pragma unroll
        for (int w = 0; w < kPagedWaves; ++w) {
            const int all = by_once(left + at_once - 1);
            const int part = w + 1 < waves ? static_cast<int>(static_cast<unsigned>(most) * kPart[w] / 256) + 1 : all;
            size[w] = max(min(part, all), least);
            left -= min(left, size[w] * at_once);
        }
    }
    __device__ __forceinline__ long long begin(int cta) const {
        long long u = 0;
        int i = cta;
#pragma unroll
        for (int w = 0; w < kPagedWaves; ++w) {
            const int n = min(i, at_once);
            u += static_cast<long long>(n) * size[w];
            i -= n;
        }
        return i > 0 ? 0x7fffffffffffll : u;
    }
    __device__ __forceinline__ int owner(int u) const {
        int cta = 0;
#pragma unroll
        for (int w = 0; w < kPagedWaves; ++w) {
            const long long all = static_cast<long long>(size[w]) * at_once;
            if (u < all || w + 1 == kPagedWaves) return cta + u / size[w];
            u -= static_cast<int>(all);
            cta += at_once;
        }
        return cta;
    }
};

// Where a CTA's share of the line begins: `off` units into an item; units [u0, u1).
struct PagedStart {
    int head, seq, rt, off;
    int u0, u1;
    PagedShares shares;
};

constexpr int kPagedEntries = 1024;   // sums of units kept while a CTA finds its start
struct PagedScratch {
    int4 seq[kPagedMaxSeqs];          // a request's row0, n, first, len
    int rt0[kPagedMaxSeqs + 1];       // row tiles before a request
    int sum[kPagedEntries + 1];       // units before a group of row tiles
    long long warp_sum[32];
};

// exclusive sum over the block; every thread gets the total
template <int THREADS, typename T>
__device__ __forceinline__ T paged_block_scan(T v, long long* sums, T& total) {
    T* warp_sum = reinterpret_cast<T*>(sums);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    T x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();                  // the previous scan's sums have been read
    if (lane == 31) warp_sum[warp] = x;
    __syncthreads();
    T before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        const T t = warp_sum[w];
        if (w < warp) before += t;
        all += t;
    }
    total = all;
    return before + x - v;
}

__device__ __forceinline__ int paged_upper(const int* v, int n, int x) {   // the last i of [0, n) with v[i] <= x; v[0] <= x
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (v[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// WARPS: for kernels of few rows, whose requests have a row tile each (the others only lose by the question: blocks of 32 rows
// 47.9 -> 49.0 us).  Called by all THREADS threads of the block; false: there is nothing for this CTA to do.
// waves: CTAs of the grid for each of the a.at_once that run at one time.  min_units: what a CTA takes at least (more than E);
// full_units: what it takes at least as long as those have work.
// The launcher's bounds on rows, requests and keys keep every sum below 2^31, as long as the requests' rows follow one another; where
// they do not, the call has no work and the status word says so.
template <int THREADS, int KT, int E, bool WARPS>
__device__ bool paged_find_start(const PagedAttnArgs& a, PagedScratch& sc, int waves, int min_units, int full_units, PagedStart& st) {
    const int tid = threadIdx.x;
    auto kept = [&](int s) {          // the request's numbers, loaded once
        const int4 v = sc.seq[s];
        PagedSeq q{v.x, v.y, v.z, v.w, 0};
        q.tiles(a);
        return q;
    };
    auto share = [&](int per_head, int& rem) {   // this CTA's part of the line, and its place within a head's
        const int total = per_head * a.KV;
        st.shares.at_once = a.at_once;
        st.shares.divide(total, waves, min_units, full_units, a.by_once);
        const long long u0 = st.shares.begin(blockIdx.x), u1 = st.shares.begin(blockIdx.x + 1);
        if (u0 >= total) return false;
        st.u0 = static_cast<int>(u0);
        st.u1 = static_cast<int>(min(u1, static_cast<long long>(total)));
        st.head = st.u0 / per_head;
        rem = st.u0 - st.head * per_head;
        return true;
    };
    // Few requests of one row tile each: every warp by itself, a request a lane, without a barrier (577 keys 9.5 -> 9.2 us).
    if (WARPS && a.n_seqs <= 32) {
        const int s = tid & 31;
        int units = 0, n_rt = 0, rem;
        bool wrong = false;
        if (s < a.n_seqs) {
            const PagedSeq q = paged_seq(a, s);
            wrong = !paged_rows_follow(a, s);
            if (blockIdx.x == 0 && tid < 32 && !paged_length_fits(a, s)) atomicExch(a.status, ODB_ERR_ARG);
            n_rt = q.n_rt;
            if (n_rt > 0) units = paged_keys<KT>(a, q, 0).n + E;
        }
        if (!__any_sync(0xffffffffu, n_rt > 1 || wrong)) {
            int sum = units;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, sum, d);
                if (s >= d) sum += x;
            }
            const int per_head = __shfl_sync(0xffffffffu, sum, 31);
            if (per_head == 0 || !share(per_head, rem)) return false;
            st.seq = __ffs(__ballot_sync(0xffffffffu, sum > rem)) - 1;
            st.rt = 0;
            st.off = rem - __shfl_sync(0xffffffffu, sum - units, st.seq);
            return true;
        }
    }
    const int per_s = (a.n_seqs + THREADS - 1) / THREADS, s0 = min(tid * per_s, a.n_seqs), s1 = min(s0 + per_s, a.n_seqs);
    int n_rt, mine_rt = 0, units = 0, rem;
    bool several = false, wrong = false;
#pragma unroll 4
    for (int s = s0; s < s1; ++s) {
        const PagedSeq q = paged_seq(a, s);
        wrong = wrong || !paged_rows_follow(a, s);
        if (blockIdx.x == 0 && !paged_length_fits(a, s)) atomicExch(a.status, ODB_ERR_ARG);
        sc.seq[s] = make_int4(q.row0, q.n, q.first, q.len);
        mine_rt += q.n_rt;
        several = several || q.n_rt > 1;
        sc.sum[s] = units;
        if (q.n_rt > 0) units += paged_keys<KT>(a, q, 0).n + E;
    }
    if (!__syncthreads_or(several || wrong)) {   // no request has more than a row tile (single tokens, short blocks): sums over the requests do
        int per_head;
        const int before = paged_block_scan<THREADS>(units, sc.warp_sum, per_head);
        if (per_head == 0) return false;
        for (int s = s0; s < s1; ++s) sc.sum[s] += before;
        if (!share(per_head, rem)) return false;
        __syncthreads();
        st.seq = paged_upper(sc.sum, a.n_seqs, rem);
        st.rt = 0;
        st.off = rem - sc.sum[st.seq];
        __syncthreads();                // the scratch may be overwritten now
        return true;
    }
    {
        // where a request's rows do not follow, its thread's sum is out of the range of any that may be
        long long all;
        int at = static_cast<int>(paged_block_scan<THREADS>(wrong ? 1ll << 40 : static_cast<long long>(mine_rt), sc.warp_sum, all));
        if (all >> 40) {
            if (blockIdx.x == 0 && tid == 0) atomicExch(a.status, ODB_ERR_ARG);
            return false;
        }
        n_rt = static_cast<int>(all);
        for (int s = s0; s < s1; ++s) {
            sc.rt0[s] = at;
            at += kept(s).n_rt;
        }
        if (tid == 0) sc.rt0[a.n_seqs] = n_rt;
    }
    __syncthreads();
    const int group = (n_rt + kPagedEntries - 1) / kPagedEntries, entries = group == 1 ? n_rt : (n_rt + group - 1) / group;
    int per_head;
    {
        const int per = (entries + THREADS - 1) / THREADS, e0 = min(tid * per, entries), e1 = min(e0 + per, entries);
        int mine = 0;
        if (e0 < e1) {
            int s = paged_upper(sc.rt0, a.n_seqs + 1, e0 * group);
            PagedSeq q = kept(s);
            int rt = e0 * group - sc.rt0[s];
            for (int e = e0; e < e1; ++e) {
                sc.sum[e] = mine;
                for (int j = e * group; j < min((e + 1) * group, n_rt); ++j, ++rt) {
                    while (rt >= q.n_rt) { q = kept(++s); rt = 0; }
                    mine += paged_keys<KT>(a, q, rt).n + E;
                }
            }
        }
        const int before = paged_block_scan<THREADS>(mine, sc.warp_sum, per_head);
        for (int e = e0; e < e1; ++e) sc.sum[e] += before;
        __syncthreads();
    }
    if (!share(per_head, rem)) return false;
    const int e = paged_upper(sc.sum, entries, rem);
    const int j = e * group;
    int left = rem - sc.sum[e];
    st.seq = paged_upper(sc.rt0, a.n_seqs + 1, j);
    PagedSeq q = kept(st.seq);
    st.rt = j - sc.rt0[st.seq];
    for (;;) {
        while (st.rt >= q.n_rt) { q = kept(++st.seq); st.rt = 0; }
        const int n = paged_keys<KT>(a, q, st.rt).n + E;
        if (left < n) break;
        left -= n;
        ++st.rt;
    }
    st.off = left;
    __syncthreads();                  // the scratch may be overwritten now
    return true;
}

// The items of a CTA's share, one after the other.
template <int KT, int E>
struct PagedWalk {
    const PagedAttnArgs& a;
    PagedSeq q;
    PagedKeys k;
    int head, seq, rt;
    int t0, t1;                      // this CTA's key tiles of the item
    int begin;                       // the unit of the item's first key tile
    int u1;
    const PagedShares& shares;

    __device__ __forceinline__ PagedWalk(const PagedAttnArgs& args, const PagedStart& st)
        : a(args), head(st.head), seq(st.seq), rt(st.rt), begin(st.u0 - st.off + E), u1(st.u1), shares(st.shares) {
        q = paged_seq(a, seq);
        k = paged_keys<KT>(a, q, rt);
        t0 = max(0, st.off - E);
        t1 = min(k.n, u1 - begin);
    }
    // to the next item; false: the share has ended
    __device__ __forceinline__ bool next() {
        begin += k.n + E;
        if (begin >= u1) return false;
        ++rt;
        while (rt >= q.n_rt) {
            rt = 0;
            if (++seq == a.n_seqs) { seq = 0; ++head; }
            q = paged_seq(a, seq);
        }
        k = paged_keys<KT>(a, q, rt);
        t0 = 0;
        t1 = min(k.n, u1 - begin);
        return true;
    }
    __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == k.n; }
    // the CTAs that share the item
    __device__ __forceinline__ int first_cta() const { return shares.owner(begin); }
    __device__ __forceinline__ int last_cta() const { return shares.owner(begin + k.n - 1); }
};

// The pages of a request as a warp sees them: 32 entries of its table row at a time, one a lane.  Every lane calls row() with the
// same position and gets the pool row of it (of head 0 behind `base`, the layer's K or V); of a page that is none, the row
// behind the pool, which reads as zeros.  ASK: that is an error where some row of the request sees one of the page's positions (pages in
// front of a window may be gone), which is asked when the entries are loaded - once for K and V, of V in the many rows' kernel, whose K
// is the first that everybody waits for.  TOGETHER: the warp comes together right behind the question (the code that the compiler makes
// of it: 577 keys 9.2 us with, 9.5 without; a prompt of 4096 rows 140.4 with, 139.5 without, 139 if nobody asks).
struct PagedPages {
    int seq = -1, first = 0, entry = 0;
    template <bool ASK, bool TOGETHER = false>
    __device__ __forceinline__ int row(const PagedAttnArgs& a, const PagedSeq& q, int s, int head, int pos, int base) {
        const int p = pos >> a.page_shift;
        if (s != seq || p < first || p >= first + 32) {
            seq = s;
            first = p;
            const int mine = p + static_cast<int>(threadIdx.x & 31);
            entry = -1;
            if (mine < a.table_stride) {
                entry = a.table[static_cast<size_t>(s) * a.table_stride + mine];
                if (ASK && __builtin_expect(static_cast<unsigned>(entry) >= static_cast<unsigned>(a.n_pages), 0)) {
                    const long long from = static_cast<long long>(mine) << a.page_shift, lo = static_cast<long long>(q.first) - a.left,
                                    hi = min(static_cast<long long>(q.len), static_cast<long long>(q.first) + q.n + a.right);
                    if (from < hi && (from < a.sinks || min(from + (1 << a.page_shift), hi) > lo)) atomicExch(a.status, ODB_ERR_STATE);
                }
            }
            if (TOGETHER) __syncwarp();
        }
        return at(a, head, pos, base, __shfl_sync(0xffffffffu, entry, p - first));
    }
    // Position pos + more of each lane, of those that `wanted` says (others get the row behind the pool): at most 64 positions from pos on,
    // which is a multiple of them, so that their pages are among the 32 entries with pos's.
    template <bool ASK>
    __device__ __forceinline__ int rows(const PagedAttnArgs& a, const PagedSeq& q, int s, int head, int pos, int more, bool wanted, int base) {
        row<ASK, true>(a, q, s, head, pos, base);
        const int p = pos + more, i = (p >> a.page_shift) - first, page = __shfl_sync(0xffffffffu, entry, i & 31);
        return wanted && i < 32 ? at(a, head, p, base, page) : a.pool_rows;
    }
    __device__ __forceinline__ static int at(const PagedAttnArgs& a, int head, int pos, int base, int page) {
        return page >= 0 && page < a.n_pages ? base + ((page * a.KV + head) << a.page_shift) + (pos & ((1 << a.page_shift) - 1)) : a.pool_rows;
    }
};

// One lane of a converged warp.  TMA copies and MMAs take their operands from uniform registers: behind elect, with operands that
// every lane has, they follow one another without a detour (behind `lane == 0` an MMA took 110 cycles to issue, and one of
// 128 x 64 x 16 runs for 51).
__device__ __forceinline__ bool paged_elect() {
    uint32_t x;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(x));
    return x != 0;
}

// 2^(m - M) with M the larger of the two; a side that has seen nothing counts nothing
__device__ __forceinline__ float paged_weight(float m, float M) { return m == -INFINITY ? 0.f : ex2_approx(m - M); }
// log-sum-exp of a row from its shift in the log2 domain and its sum
__device__ __forceinline__ float paged_lse(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f; }
__device__ __forceinline__ uint32_t paged_bf16x2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ uint32_t paged_f16x2(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// A CTA's place for its part of an item that other CTAs share: parts [CTA][first or last item][row of the tile].
__device__ __forceinline__ size_t paged_part(const PagedAttnArgs& a, int cta, bool begins) {
    return (static_cast<size_t>(cta) * kPagedMaxParts + (begins ? 1 : 0)) * a.part_rows;
}
// The parts of RB rows of an item that begins in CTA c0, added up in the order of the CTAs: 32 parts' maxima and sums at once, one a
// lane, then their outputs, 16 loads in flight.
template <int HD, int RB>
struct PagedSum {
    static constexpr int V = HD / 32, CU = 16 / RB;  // dims of a lane; parts at once
    float M[RB], L[RB], acc[RB][V];

    __device__ __forceinline__ void load(const float* p, float (&x)[V]) const {
        if constexpr (V == 4) {
            const float4 t = __ldcg(reinterpret_cast<const float4*>(p));
            x[0] = t.x; x[1] = t.y; x[2] = t.z; x[3] = t.w;
        } else {
            const float2 t = __ldcg(reinterpret_cast<const float2*>(p));
            x[0] = t.x; x[1] = t.y;
        }
    }
    // rows r0, r0 + step ..; those behind the last repeat it
    __device__ __forceinline__ void rows(const PagedAttnArgs& a, int c0, int c1, int r0, int step, int n_rows) {
        const int lane = threadIdx.x & 31;
        int r[RB];
#pragma unroll
        for (int k = 0; k < RB; ++k) {
            r[k] = min(r0 + k * step, n_rows - 1);
            M[k] = -INFINITY;
            L[k] = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) acc[k][j] = 0.f;
        }
        for (int c = c0; c <= c1; c += 32) {
            const int n = min(32, c1 + 1 - c), mine = c + min(lane, n - 1);
            float2 ml[RB];
            float w[RB];
#pragma unroll
            for (int k = 0; k < RB; ++k) ml[k] = __ldcg(reinterpret_cast<const float2*>(a.part_ml + (paged_part(a, mine, mine == c0) + r[k]) * 2));
#pragma unroll
            for (int k = 0; k < RB; ++k) {
                float top = ml[k].x;
#pragma unroll
                for (int d = 16; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                top = fmaxf(top, M[k]);
                w[k] = lane < n ? paged_weight(ml[k].x, top) : 0.f;
                const float f = paged_weight(M[k], top);
                float l = w[k] * ml[k].y;
#pragma unroll
                for (int d = 16; d >= 1; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
                M[k] = top;
                L[k] = L[k] * f + l;
#pragma unroll
                for (int j = 0; j < V; ++j) acc[k][j] *= f;
            }
            for (int u0 = 0; u0 < n; u0 += CU) {
                float x[CU][RB][V];
#pragma unroll
                for (int u = 0; u < CU; ++u) {
                    const int cta = c + min(u0 + u, n - 1);
                    const float* part = a.part_o + paged_part(a, cta, cta == c0) * HD + lane * V;
#pragma unroll
                    for (int k = 0; k < RB; ++k) load(part + r[k] * HD, x[u][k]);
                }
#pragma unroll
                for (int u = 0; u < CU; ++u) {
#pragma unroll
                    for (int k = 0; k < RB; ++k) {
                        const float e = __shfl_sync(0xffffffffu, w[k], (u0 + u) & 31);   // zero behind the last
                        if (u0 + u < n)
#pragma unroll
                            for (int j = 0; j < V; ++j) acc[k][j] += e * x[u][k][j];
                    }
                }
            }
        }
    }
    // output of row k, packed row idx of the request whose rows begin at row0
    __device__ __forceinline__ void write(const PagedAttnArgs& a, int k, int row0, int head, int idx) const {
        const int lane = threadIdx.x & 31, i = a.by_group(idx), h = head * a.G + idx - i * a.G;
        const size_t row = static_cast<size_t>(row0 + i);
        const float inv = L[k] == 0.f ? 0.f : 1.0f / L[k];
        uint32_t* op = reinterpret_cast<uint32_t*>(a.out + row * a.out_stride + h * HD + lane * V);
#pragma unroll
        for (int j = 0; j < V; j += 2) op[j / 2] = paged_bf16x2(acc[k][j] * inv, acc[k][j + 1] * inv);
        if (a.lse && lane == 0) a.lse[row * a.H + h] = paged_lse(M[k], L[k]);
    }
};

#endif

}  // namespace odb
