// Norm, rotation and store for a pool of 8 bits: queries as for a pool of bf16 (formulas: paged_store.cu), keys and values as e4m3
// under a scale for each block of 16 positions, one K/V head, K or V.
//
//   e = the smallest integer with max |x| <= 448 * 2^e over the finite values that the call writes of the block
//   e = max(e, the block's exponent before) where the block keeps positions: those below len_after that the call does not write
//   code = e4m3(x * 2^-e), to the nearest even; not finite: NaN.   Kept codes: e4m3(code * 2^(before - e)).   scale = 2^e
//
// with x in fp32 straight from norm and rotation: one rounding, by at most 2^-4 of x or 2^-10 of the scale.  The scale is a power of
// two: e4m3 has the same step relative to a value whatever the exponent, so that a scale that fits the largest value more closely gains
// nothing but for the few values below 2^-6 of it; and what a code stands for is a number of bf16, kept codes of 2^-6 and more change
// their exponent without a rounding, and x * 2^-e has none.
//
// Four warps take a block of K or of V, four rows each, HD / 8 threads a row, each the places that the
// store of bf16 gives it, and `heads` heads one after the other, the next one's rows in flight while the one before is turned: the block's
// sines, its table and its slots are found once.  Blocks begin where a row's request or block differs from the row's before it: every warp
// looks for them among `window` rows, with all their maps in one load.  Units of q as in the store of bf16, behind the blocks.
//
// What bounds it: a refresh of 16 requests of 1200 to 1999 rows, 32 + 8 heads of 128, reads 317 MB and writes 264 with q, 88 us at the copy
// rate; it takes 111 us, 63 of them for q and 48 for K and V (75 with a warp to a block and head).  A thread holds two rows' values,
// angles and loads in flight: the registers limit the warps of an SM, and seven CTAs of four (72 registers; up to 20 bytes spilled in some
// forms) take 111 us where six (80, none spilled) take 121, at 16 x 32 rows 11.1 and 11.2.  48 tokens take 4.3 us in a graph, a
// launch and three dependent reads (map, table, row).
#include "paged_rows.cuh"

#include "paged_e4m3.cuh"

namespace odb {

namespace {

constexpr int kWarps = 4;                                     // of a block of positions
constexpr int kThreads = 32 * kWarps;

// codes of four values; those that are not finite become NaN
__device__ __forceinline__ uint32_t codes4(f2 u, f2 v, f2 by) {
    const f2 zero = pair(0.f, 0.f);
    const float2 a = floats(fma(u, zero, mul(u, by))), b = floats(fma(v, zero, mul(v, by)));
    return e4m3x2_of(a.x, a.y) | static_cast<uint32_t>(e4m3x2_of(b.x, b.y)) << 16;
}
__device__ __forceinline__ float finite_max(float top, f2 x) {
    const float2 y = floats(fma(x, pair(0.f, 0.f), x));     // an infinity becomes NaN, which fmaxf passes over
    return fmaxf(top, fmaxf(fabsf(y.x), fabsf(y.y)));
}

// V: the blocks are of V
template <int HD, bool INTER, bool ALL, bool V>
__device__ __forceinline__ void block_unit(const PagedE4m3StoreArgs& p, int w, int head0) {
    constexpr int kLanes = HD / 8, kAtOnce = kThreads / kLanes, kSteps = kPagedBlock / kAtOnce;
    constexpr unsigned kFull = 0xffffffffu;
    const PagedStoreArgs& rows = p.rows;
    const int lane = threadIdx.x & 31, l = lane % kLanes, sub = threadIdx.x / kLanes;
    __shared__ float tops[2][kWarps];
    int turn = 0;
    const int heads = min(p.heads, p.KV - head0);
    // lane i: row r0 + i, the one in front of the window first
    const int r0 = w * p.window - 1;
    int seq = -1, pos = -1, slot = -1;
    if (r0 + lane >= 0 && r0 + lane < rows.rows) {
        seq = p.row_seq[r0 + lane];
        pos = rows.row_pos[r0 + lane];
        slot = rows.row_slot[r0 + lane];
    }
    const bool known = pos >= 0 && seq >= 0 && seq < p.n_seqs;
    const int mine = known ? pos / kPagedBlock : -1;
    const int seq_before = __shfl_up_sync(kFull, seq, 1), mine_before = __shfl_up_sync(kFull, mine, 1);
    const unsigned same = __ballot_sync(kFull, lane > 0 && known && mine == mine_before && seq == seq_before);
    unsigned begins = __ballot_sync(kFull, known && lane > 0 && lane <= p.window) & ~same;
    const int to_end = known ? min(max(p.len[seq], 0), 0x7fffffff - kPagedBlock) - (pos & ~(kPagedBlock - 1)) : 0;   // what the request has from the block's first position on
    // the slot of the block's first position, -1 where the row has none
    const int first = known && slot >= 0 && slot >> rows.page_shift < rows.n_pages && !((slot ^ pos) % kPagedBlock) ? slot & ~(kPagedBlock - 1) : -1;

    const bool turned = !V && (ALL || l < rows.rot / 8);
    const int ca = V || (turned && !INTER) ? 4 * l : 8 * l,
              cb = V ? HD / 2 + 4 * l : turned && !INTER ? (ALL ? HD : rows.rot) / 2 + 4 * l : 8 * l + 4;
    StoreTurn<INTER> t;
    f2 cosines[kSteps][2], sines[kSteps][2];                    // of a thread's rows
    const bool normed = !V && rows.k_gain;
    if (normed) t.gains(rows.k_gain, ca, cb);

    while (begins) {
        const int a = __ffs(begins) - 1;
        begins &= begins - 1;
        // its rows are lanes a .. a + n - 1; those with a slot in the same place of the pool are written
        const int n = min(kPagedBlock, __ffs(~(same >> 1 >> a)));
        const bool in = lane >= a && lane < a + n && first >= 0;
        const unsigned any = __ballot_sync(kFull, in);
        if (!any) continue;
        const int f = __ffs(any) - 1, base = __shfl_sync(kFull, first, f), live = __shfl_sync(kFull, to_end, f);
        const unsigned stored = __ballot_sync(kFull, in && first == base);
        const unsigned written = __reduce_or_sync(kFull, (stored >> lane) & 1u ? 1u << pos % kPagedBlock : 0u);
        const unsigned kept = ((1u << min(max(live, 0), kPagedBlock)) - 1u) & ~written;
        const int page = base >> rows.page_shift;
        const unsigned at = (static_cast<unsigned>(page * p.KV + head0) << rows.page_shift) + (base & ((1 << rows.page_shift) - 1));   // row of the layer's pool: below 2^31

        const long long stride = V ? rows.v_stride : rows.k_stride;
        const __nv_bfloat16* src = (V ? rows.v : rows.k) + (r0 + a + sub) * stride + head0 * HD;
        uint2 va[kSteps], vb[kSteps];
        auto load = [&]() {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                va[i] = vb[i] = make_uint2(0u, 0u);
                if ((stored >> a >> (i * kAtOnce + sub)) & 1u) {
                    va[i] = *reinterpret_cast<const uint2*>(src + i * kAtOnce * stride + ca);
                    vb[i] = *reinterpret_cast<const uint2*>(src + i * kAtOnce * stride + cb);
                }
            }
            src += HD;
        };
        load();
        if (!V) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                t.angles(rows, __shfl_sync(kFull, pos, min(a + i * kAtOnce + sub, 31)), l, turned);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    cosines[i][k] = t.c[k];
                    sines[i][k] = t.s[k];
                }
            }
        }
#pragma unroll 1
        for (int h = 0; h < heads; ++h) {
            const unsigned row = at + (static_cast<unsigned>(h) << rows.page_shift);
            unsigned char* dst = (V ? p.v_pool : p.k_pool) + static_cast<size_t>(row) * HD;
            float* scale = (V ? p.v_scales : p.k_scales) + row / kPagedBlock;
            const int before = kept ? e4m3_exponent(*scale) : kPagedLowExp;
            f2 x[kSteps][4];
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                f2 u[2], v[2];
                if (V) widen<false>(va[i], vb[i], u, v);
                else widen<INTER>(va[i], vb[i], u, v);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    x[i][k] = u[k];
                    x[i][2 + k] = v[k];
                }
            }
            if (h + 1 < heads) load();                          // the next head's rows while these are at work
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                f2 u[2] = {x[i][0], x[i][1]}, v[2] = {x[i][2], x[i][3]};
                if (!V) {
                    if (normed) t.template norm<HD>(u, v, rows.eps, kFull);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        t.c[k] = cosines[i][k];
                        t.s[k] = sines[i][k];
                        t.ms[k] = sines[i][k] ^ 0x8000000080000000ull;      // both signs turned: registers are what limits the warps of an SM
                    }
                    t.turn(u, v, turned);
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    x[i][k] = u[k];
                    x[i][2 + k] = v[k];
                    top = finite_max(finite_max(top, u[k]), v[k]);
                }
            }
            top = __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(top)));
            if (lane == 0) tops[turn][threadIdx.x >> 5] = top;
            __syncthreads();                                    // all have the block's exponent from before, too
#pragma unroll
            for (int i = 0; i < kWarps; ++i) top = fmaxf(top, tops[turn][i]);
            turn ^= 1;
            const int e = max(e4m3_exponent_for(top), before);
            const float by = exp2_int(-e);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int off = __shfl_sync(kFull, pos, min(a + i * kAtOnce + sub, 31)) % kPagedBlock;
                if (!((stored >> a >> (i * kAtOnce + sub)) & 1u)) continue;
                f2 u0 = x[i][0], u1 = x[i][1], v0 = x[i][2], v1 = x[i][3];
                if (INTER && !V) {                           // the pairs back in their places
                    const float2 a0 = floats(u0), a1 = floats(u1), b0 = floats(v0), b1 = floats(v1);
                    u0 = pair(a0.x, b0.x); u1 = pair(a0.y, b0.y);
                    v0 = pair(a1.x, b1.x); v1 = pair(a1.y, b1.y);
                }
                *reinterpret_cast<uint32_t*>(dst + off * HD + ca) = codes4(u0, u1, pair(by, by));
                *reinterpret_cast<uint32_t*>(dst + off * HD + cb) = codes4(v0, v1, pair(by, by));
            }
            if (kept && e > before) {                           // the scale has grown: what stays is rounded again under it
                const float down = exp2_int(max(before - e, -126));
#pragma unroll 1
                for (int i = 0; i < kSteps; ++i) {
                    const int off = i * kAtOnce + sub;
                    if (!((kept >> off) & 1u)) continue;
                    uint2* c = reinterpret_cast<uint2*>(dst + off * HD + 8 * l);
                    const uint2 old = *c;
                    *c = make_uint2(e4m3x4_times(old.x, down), e4m3x4_times(old.y, down));
                }
            }
            if (threadIdx.x == 0) *scale = exp2_int(e);
        }
    }
}

template <int HD, bool INTER, bool ALL>
__global__ void __launch_bounds__(kThreads, 7) paged_e4m3_store_kernel(const PagedE4m3StoreArgs p, const int blocks) {
    pdl_launch_dependents();
    pdl_wait();
    if (static_cast<int>(blockIdx.x) < blocks) {
        const int groups = (p.KV + p.heads - 1) / p.heads, w = blockIdx.x / (2 * groups), part = blockIdx.x - w * 2 * groups;
        if (part < groups) block_unit<HD, INTER, ALL, false>(p, w, part * p.heads);
        else block_unit<HD, INTER, ALL, true>(p, w, (part - groups) * p.heads);
    } else {
        constexpr int kLanes = HD / 8;
        store_unit<HD, INTER, ALL>(p.rows, static_cast<long long>(blockIdx.x - blocks) * (kThreads / kLanes) + threadIdx.x / kLanes);
    }
}

template <int HD, bool INTER, bool ALL>
cudaError_t launch(const PagedE4m3StoreArgs& a, cudaStream_t st) {
    const int blocks = (a.rows.rows + a.window - 1) / a.window * 2 * ((a.KV + a.heads - 1) / a.heads);
    const long long q_units = static_cast<long long>(a.rows.rows) * ((a.rows.H + kStoreHeads - 1) / kStoreHeads), per = kThreads / (HD / 8);
    return launch_kernel(paged_e4m3_store_kernel<HD, INTER, ALL>, dim3(static_cast<unsigned>(blocks + (q_units + per - 1) / per)), dim3(kThreads), 0, st, a,
                         blocks);
}

}  // namespace

cudaError_t launch_paged_e4m3_store(const PagedE4m3StoreArgs& a, cudaStream_t st) {
    const bool all = a.rows.rot == a.rows.HD;
    if (a.rows.interleaved) {
        if (a.rows.HD == 128) return all ? launch<128, true, true>(a, st) : launch<128, true, false>(a, st);
        return all ? launch<64, true, true>(a, st) : launch<64, true, false>(a, st);
    }
    if (a.rows.HD == 128) return all ? launch<128, false, true>(a, st) : launch<128, false, false>(a, st);
    return all ? launch<64, false, true>(a, st) : launch<64, false, false>(a, st);
}

}  // namespace odb
