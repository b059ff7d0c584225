// Declarations shared by the paged-cache translation units: the handle, the launchers' arguments and the walk over the
// attention's work, which the kernels of few and of many rows have in common.
#pragma once

#include "odb_internal.cuh"

namespace odb {

constexpr int kPagedMaxSeqs = 1024;        // requests of one forward
constexpr int kPagedMaxCtas = 304;         // CTAs of an attention launch, at most: two on each of the 148 SMs and a few
constexpr int kPagedPartRows = 128;         // rows of a part with two CTAs on an SM; twice that with one
constexpr int kPagedMaxParts = 2;          // unfinished segments a CTA leaves behind: of its first item and of its last
constexpr int kPagedUnlimited = 1 << 30;   // a window side without limit; lengths and positions stay below it

// ---- layout (paged_layout.cu) ----
struct PagedLayoutArgs {
    const int32_t *len_before, *len_after, *first, *count;
    int32_t *table, *free_pages;
    int32_t *row_start, *row_seq, *row_pos, *row_slot;
    int n_seqs, max_rows, page_shift, n_pages, table_stride;
    int* status;
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

// ---- attention (paged_attention.cu) ----
struct PagedAttnArgs {
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    float* lse;                                           // null: not wanted
    long long q_stride, out_stride;
    const int32_t *table, *len, *first, *row_start;
    int n_seqs, max_rows, H, KV, G, page_shift, n_pages, table_stride;
    int k_row0, v_row0, pool_rows;                        // rows of hd values of the whole pool: this layer's K, its V, all of them
    int left, right, sinks;
    float scale_log2;                                     // softmax scale x log2(e)
    int* status;
    unsigned int* arrivals;                               // [kPagedMaxCtas], zero between launches
    float* part_o;                                        // [ctas][2][part_rows][HD]
    float* part_ml;                                       // [ctas][2][part_rows][2]
    int part_rows;                                        // rows of a tile
    int tile_rows, tile_tokens;                           // many rows: packed rows of an item, query rows of a Q tile
};
// the pool's two maps: boxes of whole rows, and of 64 values of a row
struct PagedMaps {
    CUtensorMap rows, atoms;
};
// max_new: rows of the longest request; a hint that picks the kernel
cudaError_t launch_paged_attention(PagedAttnArgs a, const PagedMaps& maps, int hd, int max_new, int sms, cudaStream_t st);
// many packed rows on the tensor cores (paged_attention_tc.cu); q_tiles: Q tiles of 128 rows a CTA takes
cudaError_t launch_paged_attention_tc(PagedAttnArgs a, const PagedMaps& maps, int hd, int q_tiles, int sms, cudaStream_t st);
constexpr int kPagedTcMaxGroup = 128;   // heads of a group that fit a Q tile
size_t paged_part_bytes(int hd);

#ifdef __CUDACC__
// ---------------------------------------------------------------------------------------
// The attention's work.  An item is one tile of up to `rows` packed rows (row i of a request and query head g of the
// group: packed row i * G + g) of one K/V head; its keys are cut into tiles of KT positions.  All key tiles of all
// items in the order head, request, row tile, key tile are one line, which is divided evenly over the CTAs: whatever
// the lengths, every CTA gets the same number of key tiles.
// ---------------------------------------------------------------------------------------

struct PagedSeq {
    int row0, n, first, len, n_rt;
};

__device__ __forceinline__ PagedSeq paged_seq(const PagedAttnArgs& a, int s, int rows) {
    PagedSeq q;
    const int r0 = min(max(a.row_start[s], 0), a.max_rows), r1 = min(a.row_start[s + 1], a.max_rows);
    q.row0 = r0;
    q.n = max(r1 - r0, 0);
    q.first = min(max(a.first[s], -kPagedUnlimited), kPagedUnlimited - 1);
    // the table bounds the keys whatever the length says
    q.len = static_cast<int>(min(static_cast<long long>(max(a.len[s], 0)), static_cast<long long>(a.table_stride) << a.page_shift));
    q.n_rt = static_cast<int>((static_cast<unsigned>(q.n) * static_cast<unsigned>(a.G) + rows - 1) / static_cast<unsigned>(rows));
    return q;
}

// The key tiles of a row tile: `sink_tiles` from the front, the others from tile `first_tile` on; `n` of them, at least
// one (an item without a visible key still writes its rows).  Positions from `hi` on are seen by no row, nor are those
// of [sinks, lo).
struct PagedKeys {
    int lo, hi, sink_tiles, first_tile, n;
    __device__ __forceinline__ int tile(int t) const { return t < sink_tiles ? t : first_tile + t - sink_tiles; }
};

template <int KT>
__device__ __forceinline__ PagedKeys paged_keys(const PagedAttnArgs& a, const PagedSeq& q, int rt, int rows) {
    const int i0 = rt * rows / a.G, i1 = min(q.n - 1, (rt * rows + rows - 1) / a.G);
    PagedKeys k;
    k.hi = static_cast<int>(max(0ll, min(static_cast<long long>(q.len), static_cast<long long>(q.first) + i1 + a.right + 1)));
    k.lo = static_cast<int>(max(0ll, min(static_cast<long long>(k.hi), static_cast<long long>(q.first) + i0 - a.left)));
    const int end = (k.hi + KT - 1) / KT;
    k.first_tile = k.lo < k.hi ? k.lo / KT : end;
    k.sink_tiles = min((min(a.sinks, k.hi) + KT - 1) / KT, k.first_tile);
    k.n = max(1, k.sink_tiles + end - k.first_tile);
    return k;
}

// Where a CTA's share of the line begins.
struct PagedStart {
    int head, seq, rt, tile;         // the item, and the key tile inside it
    long long u0, u1;                // its units [u0, u1) of
    long long total;                 // this many, divided over
    int ctas;                        // this many CTAs
};

constexpr int kPagedEntries = 1024;   // sums of key tiles kept while a CTA finds its start
struct PagedScratch {
    int rt0[kPagedMaxSeqs + 1];       // row tiles before a request
    int sum[kPagedEntries + 1];       // key tiles before a group of row tiles
    long long warp_sum[32];
};

// exclusive sum over the block; every thread gets the total
template <int THREADS>
__device__ __forceinline__ long long paged_block_scan(long long v, long long* warp_sum, long long& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();                  // the previous scan's sums have been read
    if (lane == 31) warp_sum[warp] = x;
    __syncthreads();
    long long before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        const long long t = warp_sum[w];
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

// Called by all THREADS threads of the block; false: there is nothing for this CTA to do.
// min_units: key tiles a CTA takes at least where there are fewer than the grid could share.
template <int THREADS, int KT>
__device__ bool paged_find_start(const PagedAttnArgs& a, int rows, PagedScratch& sc, int min_units, PagedStart& st) {
    const int tid = threadIdx.x;
    long long total;
    {
        const int per = (a.n_seqs + THREADS - 1) / THREADS, s0 = min(tid * per, a.n_seqs), s1 = min(s0 + per, a.n_seqs);
        long long mine = 0;
        for (int s = s0; s < s1; ++s) mine += paged_seq(a, s, rows).n_rt;
        long long at = paged_block_scan<THREADS>(mine, sc.warp_sum, total);
        for (int s = s0; s < s1; ++s) {
            sc.rt0[s] = static_cast<int>(at);
            at += paged_seq(a, s, rows).n_rt;
        }
        if (tid == 0) sc.rt0[a.n_seqs] = static_cast<int>(total);
    }
    const int n_rt = static_cast<int>(total);      // rows x group fits: max_rows * H < 2^31
    if (n_rt == 0) return false;
    __syncthreads();
    const int group = (n_rt + kPagedEntries - 1) / kPagedEntries, entries = (n_rt + group - 1) / group;
    {
        const int per = (entries + THREADS - 1) / THREADS, e0 = min(tid * per, entries), e1 = min(e0 + per, entries);
        long long mine = 0;
        if (e0 < e1) {
            int s = paged_upper(sc.rt0, a.n_seqs + 1, e0 * group);
            PagedSeq q = paged_seq(a, s, rows);
            int rt = e0 * group - sc.rt0[s];
            for (int e = e0; e < e1; ++e) {
                sc.sum[e] = static_cast<int>(mine);
                for (int j = e * group; j < min((e + 1) * group, n_rt); ++j, ++rt) {
                    while (rt >= q.n_rt) { q = paged_seq(a, ++s, rows); rt = 0; }
                    mine += paged_keys<KT>(a, q, rt, rows).n;
                }
            }
        }
        const long long before = paged_block_scan<THREADS>(mine, sc.warp_sum, total);
        for (int e = e0; e < e1; ++e) sc.sum[e] += static_cast<int>(before);
        __syncthreads();
    }
    // total key tiles of one head fit 31 bits: at most 2^31 / KT a row tile's keys and 2^31 packed rows would not, but the
    // launcher bounds rows x keys
    const long long per_head = total;
    st.total = per_head * a.KV;
    st.ctas = static_cast<int>(max(1ll, min(static_cast<long long>(gridDim.x), st.total / min_units)));
    if (static_cast<int>(blockIdx.x) >= st.ctas) return false;
    st.u0 = st.total * blockIdx.x / st.ctas;
    st.u1 = st.total * (blockIdx.x + 1) / st.ctas;
    st.head = static_cast<int>(st.u0 / per_head);
    const int rem = static_cast<int>(st.u0 - st.head * per_head);
    const int e = paged_upper(sc.sum, entries, rem);
    int j = e * group, left = rem - sc.sum[e];
    st.seq = paged_upper(sc.rt0, a.n_seqs + 1, j);
    PagedSeq q = paged_seq(a, st.seq, rows);
    st.rt = j - sc.rt0[st.seq];
    for (;;) {
        while (st.rt >= q.n_rt) { q = paged_seq(a, ++st.seq, rows); st.rt = 0; }
        const int n = paged_keys<KT>(a, q, st.rt, rows).n;
        if (left < n) break;
        left -= n;
        ++st.rt;
    }
    st.tile = left;
    __syncthreads();                  // the scratch may be overwritten now
    return st.u1 > st.u0;
}

// The items of a CTA's share, one after the other.
template <int KT>
struct PagedWalk {
    const PagedAttnArgs& a;
    const int rows;
    PagedSeq q;
    PagedKeys k;
    int head, seq, rt;
    int t0, t1;                      // this CTA's key tiles of the item
    long long u, u1;                 // units left: [u, u1) from t0 on

    __device__ __forceinline__ PagedWalk(const PagedAttnArgs& args, const PagedStart& st, int tile_rows)
        : a(args), rows(tile_rows), head(st.head), seq(st.seq), rt(st.rt), t0(st.tile), u(st.u0), u1(st.u1) {
        q = paged_seq(a, seq, rows);
        k = paged_keys<KT>(a, q, rt, rows);
        t1 = static_cast<int>(min(static_cast<long long>(k.n), t0 + (u1 - u)));
    }
    __device__ __forceinline__ long long item_begin() const { return u - t0; }
    // to the next item; false: the share has ended
    __device__ __forceinline__ bool next() {
        u += t1 - t0;
        if (u >= u1) return false;
        ++rt;
        while (rt >= q.n_rt) {
            rt = 0;
            if (++seq == a.n_seqs) { seq = 0; ++head; }
            q = paged_seq(a, seq, rows);
        }
        k = paged_keys<KT>(a, q, rt, rows);
        t0 = 0;
        t1 = static_cast<int>(min(static_cast<long long>(k.n), u1 - u));
        return true;
    }
};

// 2^x for x <= 0 on the special-function unit (flushes to zero far below zero, which is the wanted value)
__device__ __forceinline__ float paged_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 2^(m - M) with M the larger of the two; a side that has seen nothing counts nothing
__device__ __forceinline__ float paged_weight(float m, float M) { return m == -INFINITY ? 0.f : paged_ex2(m - M); }
// log-sum-exp of a row from its shift in the log2 domain and its sum
__device__ __forceinline__ float paged_lse(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f; }
__device__ __forceinline__ uint32_t paged_bf16x2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// A CTA's place for its part of an item that other CTAs share: parts [CTA][first or last item][row of the tile].
__device__ __forceinline__ size_t paged_part(const PagedAttnArgs& a, int cta, bool begins) {
    return (static_cast<size_t>(cta) * kPagedMaxParts + (begins ? 1 : 0)) * a.part_rows;
}
// Rows of an item's parts, which CTAs c0 .. c1 have written, added up in the order of the CTAs with a running maximum: RB rows
// of a warp at a time, so that their loads are in flight together.
template <int HD, int RB>
__device__ __forceinline__ void paged_merge_rows(const PagedAttnArgs& a, int row0, int head, int first_idx, int rows, int c0, int c1, int r0, int step) {
    constexpr int V = HD / 32;                       // dims of a lane
    const int lane = threadIdx.x & 31;
    float M[RB], L[RB], acc[RB][V];
#pragma unroll
    for (int k = 0; k < RB; ++k) {
        M[k] = -INFINITY;
        L[k] = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) acc[k][j] = 0.f;
    }
    constexpr int CU = 8 / RB;                       // parts in flight
    for (int c = c0; c <= c1; c += CU) {
        float2 ml[CU][RB];
        float x[CU][RB][V];
#pragma unroll
        for (int u = 0; u < CU; ++u)
#pragma unroll
            for (int k = 0; k < RB; ++k) {
                const size_t slot = paged_part(a, min(c + u, c1), c + u == c0) + min(r0 + k * step, rows - 1);
                ml[u][k] = __ldcg(reinterpret_cast<const float2*>(a.part_ml + slot * 2));
                const float* po = a.part_o + slot * HD + lane * V;
                if constexpr (V == 4) {
                    const float4 t = __ldcg(reinterpret_cast<const float4*>(po));
                    x[u][k][0] = t.x; x[u][k][1] = t.y; x[u][k][2] = t.z; x[u][k][3] = t.w;
                } else {
                    const float2 t = __ldcg(reinterpret_cast<const float2*>(po));
                    x[u][k][0] = t.x; x[u][k][1] = t.y;
                }
            }
#pragma unroll
        for (int u = 0; u < CU; ++u) {
            if (c + u > c1) break;
#pragma unroll
            for (int k = 0; k < RB; ++k) {
                const float m = fmaxf(M[k], ml[u][k].x), f = paged_weight(M[k], m), e = paged_weight(ml[u][k].x, m);
                M[k] = m;
                L[k] = L[k] * f + ml[u][k].y * e;
#pragma unroll
                for (int j = 0; j < V; ++j) acc[k][j] = acc[k][j] * f + x[u][k][j] * e;
            }
        }
    }
#pragma unroll
    for (int k = 0; k < RB; ++k) {
        const int r = r0 + k * step;
        if (r >= rows) break;
        const int idx = first_idx + r, i = idx / a.G, h = head * a.G + idx - i * a.G;
        const size_t row = static_cast<size_t>(row0 + i);
        const float inv = L[k] == 0.f ? 0.f : 1.0f / L[k];
        uint32_t* op = reinterpret_cast<uint32_t*>(a.out + row * a.out_stride + h * HD + lane * V);
#pragma unroll
        for (int j = 0; j < V; j += 2) op[j / 2] = paged_bf16x2(acc[k][j] * inv, acc[k][j + 1] * inv);
        if (a.lse && lane == 0) a.lse[row * a.H + h] = paged_lse(M[k], L[k]);
    }
}
template <int HD>
__device__ __forceinline__ void paged_merge(const PagedAttnArgs& a, int row0, int head, int first_idx, int rows, int c0, int c1, int warp, int warps) {
    if (rows > 4 * warps)
        for (int r = warp; r < rows; r += 8 * warps) paged_merge_rows<HD, 8>(a, row0, head, first_idx, rows, c0, c1, r, warps);
    else
        for (int r = warp; r < rows; r += warps) paged_merge_rows<HD, 1>(a, row0, head, first_idx, rows, c0, c1, r, warps);
}

// the CTA whose share holds unit u
__device__ __forceinline__ int paged_owner(long long u, long long total, int ctas) {
    return static_cast<int>(((u + 1) * ctas - 1) / total);
}
#endif

}  // namespace odb
