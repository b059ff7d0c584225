// Rows back from the pool, by their slots, as bf16: out = code * scale, which a scale of 2^-100 .. 2^119 leaves exact (a code's three
// bits, and 2^-9 * 2^-100 is no less than the smallest number of bf16); of a pool of bf16 the values themselves.
//
// A thread takes 8 values of a head, a warp's threads lie side by side along a row: a store fills whole sectors (with 16 values, two stores to
// a sector each, 16 x 32 rows of 32 heads 6.9 us instead of 4.9 in a graph).  Four of them are in flight at once.
//
// What bounds it: HBM, the writes of bf16 beside the reads of codes.  16 requests of 3000 to 8192 positions, 8 heads of 128, take 103 us,
// 554 MB at 0.82 of the copy rate (113 with streaming stores, 122 with eight in flight); 25771 rows 31.5 to 34.7; 48 rows 2.4 in a graph.  Over a pool
// of bf16 the 16 requests take 115 us for 743 MB, 0.98 of the copy rate, 25771 rows 35, 577 rows 2.7.
#include <type_traits>

#include "paged_e4m3.cuh"

namespace odb {

namespace {

constexpr int kThreads = 256, kAtOnce = 4, kCopied = 2;   // loads in flight of a thread: of the load's, of the copy's, which has eight blocks on an SM

// 8 codes as bf16
__device__ __forceinline__ uint4 expand8(const uint2& codes, float scale) {
    const uint32_t c[2] = {codes.x, codes.y};
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = f32x2_of(static_cast<unsigned short>(c[i / 2] >> 16 * (i & 1)));
        w[i] = paged_bf16x2(f.x * scale, f.y * scale);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int HD, bool E4M3>
__global__ void __launch_bounds__(kThreads) paged_load_kernel(const PagedLoadArgs p, const PagedDiv by_row) {
    typedef typename std::conditional<E4M3, uint2, uint4>::type Piece;
    constexpr int kPieces = HD / 8;                             // of a head
    pdl_launch_dependents();
    pdl_wait();
    const int r0 = blockIdx.x * p.block_rows, all = min(p.block_rows, p.rows - r0) * p.per_row, half = p.per_row / 2;
    for (int u0 = threadIdx.x; u0 < all; u0 += kThreads * kAtOnce) {
        Piece v[kAtOnce];
        float scale[kAtOnce];
        __nv_bfloat16* out[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int u = u0 + k * kThreads;
            out[k] = nullptr;
            if (u >= all) continue;
            const int row = by_row(u), x = u - row * p.per_row;
            const bool is_v = x >= half;
            const int head = (is_v ? x - half : x) / kPieces, piece = x % kPieces, r = r0 + row;
            const int slot = p.row_slot[r], page = slot >> p.page_shift;
            if (slot < 0 || page >= p.n_pages) continue;
            const size_t at = ((static_cast<size_t>(page) * p.KV + head) << p.page_shift) + (slot & ((1 << p.page_shift) - 1));
            v[k] = *reinterpret_cast<const Piece*>((is_v ? p.v_pool : p.k_pool) + (at * HD + piece * 8) * (E4M3 ? 1 : 2));
            if (E4M3) scale[k] = (is_v ? p.v_scales : p.k_scales)[at / kPagedBlock];
            out[k] = (is_v ? p.v_out + r * p.v_stride : p.k_out + r * p.k_stride) + head * HD + piece * 8;
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            if (!out[k]) continue;
            if constexpr (E4M3) *reinterpret_cast<uint4*>(out[k]) = expand8(v[k], scale[k]);
            else *reinterpret_cast<uint4*>(out[k]) = v[k];
        }
    }
}

// The pages that the attention's rows see, one head of K or V a block at a time, from their codes into the same places of a pool of one layer
// in bf16, which the attention's kernel for pools of bf16 then reads: for prompts, whose row tiles would otherwise each turn the same codes
// into operands.  The reads are ordinary loads: a block is resident while the store in front of it still writes the pool, and the loads for
// memory that is constant promise nothing about what is written in a kernel's lifetime, be it in front of its wait.  A prompt of 4096 rows, 8 heads
// of 128, takes 9.4 us, four requests of 900 to 1536 rows with 32 heads 24 (as a loop of one load at a time 11.7 and 32).
template <int HD>
__global__ void __launch_bounds__(kThreads, 8) paged_expand_kernel(const PagedAttnArgs a, __nv_bfloat16* layer, const int layer_rows) {
    pdl_launch_dependents();
    pdl_wait();
    const int s = blockIdx.y, head = blockIdx.z % a.KV;
    const bool is_v = static_cast<int>(blockIdx.z) >= a.KV;
    const PagedSeq q = paged_seq(a, s);
    if (q.n == 0) return;
    const long long top = min(static_cast<long long>(q.len), static_cast<long long>(q.first) + q.n + a.right), low = static_cast<long long>(q.first) - a.left;
    for (long long p = blockIdx.x; p << a.page_shift < top; p += gridDim.x) {
        const long long from = p << a.page_shift;
        if (from + (1 << a.page_shift) <= low && from >= a.sinks) continue;
        const int page = a.table[static_cast<size_t>(s) * a.table_stride + p];
        if (page < 0 || page >= a.n_pages) continue;
        const size_t row = static_cast<size_t>(page * a.KV + head) << a.page_shift, at = row + (is_v ? a.v_row0 : a.k_row0);
        const uint2* src = reinterpret_cast<const uint2*>(reinterpret_cast<const unsigned char*>(a.pool) + at * HD);
        const float* scale = a.scales + at / kPagedBlock;
        uint4* dst = reinterpret_cast<uint4*>(layer + (row + (is_v ? layer_rows : 0)) * HD);
        const int all = (HD / 8) << a.page_shift;
        for (int i0 = threadIdx.x; i0 < all; i0 += kThreads * kCopied) {
            uint2 codes[kCopied];
            float by[kCopied];
#pragma unroll
            for (int k = 0; k < kCopied; ++k) {
                const int i = i0 + k * kThreads;
                if (i >= all) break;
                codes[k] = src[i];
                by[k] = scale[i / (2 * HD)];                    // 16 positions of HD / 8 pieces each have a scale
            }
#pragma unroll
            for (int k = 0; k < kCopied; ++k) {
                const int i = i0 + k * kThreads;
                if (i < all) dst[i] = expand8(codes[k], by[k]);
            }
        }
    }
}

template <int HD, bool E4M3>
cudaError_t launch(PagedLoadArgs a, cudaStream_t st) {
    a.per_row = 2 * a.KV * (HD / 8);
    a.block_rows = a.per_row >= kThreads * kAtOnce ? 1 : kThreads * kAtOnce / a.per_row;
    return launch_kernel(paged_load_kernel<HD, E4M3>, dim3((a.rows + a.block_rows - 1) / a.block_rows), dim3(kThreads), 0, st, a, PagedDiv::by(a.per_row));
}

}  // namespace

cudaError_t launch_paged_load(PagedLoadArgs a, cudaStream_t st) {
    if (a.k_scales) return a.HD == 128 ? launch<128, true>(a, st) : launch<64, true>(a, st);
    return a.HD == 128 ? launch<128, false>(a, st) : launch<64, false>(a, st);
}

cudaError_t launch_paged_expand(const PagedAttnArgs& a, __nv_bfloat16* layer, int layer_rows, int hd, cudaStream_t st) {
    // some 4096 blocks, whatever the requests
    const long long others = static_cast<long long>(a.n_seqs) * 2 * a.KV, stripes = (4096 + others - 1) / others;
    const dim3 grid(static_cast<unsigned>(stripes < a.table_stride ? stripes : a.table_stride), a.n_seqs, 2 * a.KV);
    return hd == 128 ? launch_kernel(paged_expand_kernel<128>, grid, dim3(kThreads), 0, st, a, layer, layer_rows)
                     : launch_kernel(paged_expand_kernel<64>, grid, dim3(kThreads), 0, st, a, layer, layer_rows);
}

}  // namespace odb
