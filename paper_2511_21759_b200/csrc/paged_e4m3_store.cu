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
// A warp takes a block and one head of K or of V: HD / 8 threads a row, each the places that the store of bf16 gives it, all 16 rows'
// loads in flight before the largest value is known.  Blocks begin where a row's request or block differs from the row's before it: a warp
// looks for them among `window` rows (16 where requests have that many on average, otherwise 1), with all their maps in one load.
// Units of q as in the store of bf16.
#include "paged_rows.cuh"

#include "paged_e4m3.cuh"

namespace odb {

namespace {

constexpr int kThreads = 64;

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

template <int HD, bool INTER, bool ALL>
__device__ __forceinline__ void block_unit(const PagedE4m3StoreArgs& p, int unit) {
    constexpr int kLanes = HD / 8, kAtOnce = 32 / kLanes, kSteps = kPagedBlock / kAtOnce;
    constexpr unsigned kFull = 0xffffffffu;
    const PagedStoreArgs& rows = p.rows;
    const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes;
    const int w = unit / (2 * p.KV), part = unit - w * 2 * p.KV;
    const bool is_v = part >= p.KV;
    const int head = is_v ? part - p.KV : part;
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
    const int within = pos % kPagedBlock;
    const bool has_slot = known && slot >= 0 && slot >> rows.page_shift < rows.n_pages && slot % kPagedBlock == within;

    const bool turned = !is_v && (ALL || l < rows.rot / 8);
    const int ca = is_v || (turned && !INTER) ? 4 * l : 8 * l,
              cb = is_v ? HD / 2 + 4 * l : turned && !INTER ? (ALL ? HD : rows.rot) / 2 + 4 * l : 8 * l + 4;
    StoreTurn<INTER> t;
    const bool normed = !is_v && rows.k_gain;
    if (normed) t.gains(rows.k_gain, ca, cb);

    while (begins) {
        const int a = __ffs(begins) - 1;
        begins &= begins - 1;
        // its rows are lanes a .. a + n - 1; those with a slot in the same place of the pool are written
        const int n = min(kPagedBlock, __ffs(~(same >> 1 >> a)));
        const bool in = lane >= a && lane < a + n && has_slot;
        const unsigned any = __ballot_sync(kFull, in);
        if (!any) continue;
        const int f = __ffs(any) - 1, base = __shfl_sync(kFull, slot - within, f), from = __shfl_sync(kFull, pos - within, f), s = __shfl_sync(kFull, seq, f);
        const unsigned stored = __ballot_sync(kFull, in && slot - within == base);
        const unsigned written = __reduce_or_sync(kFull, (stored >> lane) & 1u ? 1u << within : 0u);
        const int live = min(max(p.len[s], 0), 0x7fffffff - kPagedBlock) - from;
        const unsigned kept = ((1u << min(max(live, 0), kPagedBlock)) - 1u) & ~written;
        const int page = base >> rows.page_shift;
        const size_t at = ((static_cast<size_t>(page) * p.KV + head) << rows.page_shift) + (base & ((1 << rows.page_shift) - 1));
        unsigned char* dst = (is_v ? p.v_pool : p.k_pool) + at * HD;
        float* scale = (is_v ? p.v_scales : p.k_scales) + at / kPagedBlock;
        const int before = kept ? e4m3_exponent(*scale) : kPagedLowExp;

        const __nv_bfloat16* src = is_v ? rows.v + (r0 + a) * rows.v_stride + head * HD : rows.k + (r0 + a) * rows.k_stride + head * HD;
        const long long stride = is_v ? rows.v_stride : rows.k_stride;
        uint2 va[kSteps], vb[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int j = i * kAtOnce + sub;
            va[i] = vb[i] = make_uint2(0u, 0u);
            if ((stored >> a >> j) & 1u) {
                va[i] = *reinterpret_cast<const uint2*>(src + j * stride + ca);
                vb[i] = *reinterpret_cast<const uint2*>(src + j * stride + cb);
            }
        }
        f2 x[kSteps][4];
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            f2 u[2], v[2];
            if (is_v) {
                widen<false>(va[i], vb[i], u, v);
            } else {
                widen<INTER>(va[i], vb[i], u, v);
                if (normed) t.template norm<HD>(u, v, rows.eps, kFull);
                t.angles(rows, __shfl_sync(kFull, pos, min(a + i * kAtOnce + sub, 31)), l, turned);
                t.turn(u, v, turned);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                x[i][k] = u[k];
                x[i][2 + k] = v[k];
                top = finite_max(finite_max(top, u[k]), v[k]);
            }
        }
        const int e = max(e4m3_exponent_for(__uint_as_float(__reduce_max_sync(kFull, __float_as_uint(top)))), before);
        const float by = exp2_int(-e);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int off = __shfl_sync(kFull, within, min(a + i * kAtOnce + sub, 31));
            if (!((stored >> a >> (i * kAtOnce + sub)) & 1u)) continue;
            f2 u0 = x[i][0], u1 = x[i][1], v0 = x[i][2], v1 = x[i][3];
            if (INTER && !is_v) {                               // the pairs back in their places
                const float2 a0 = floats(u0), a1 = floats(u1), b0 = floats(v0), b1 = floats(v1);
                u0 = pair(a0.x, b0.x); u1 = pair(a0.y, b0.y);
                v0 = pair(a1.x, b1.x); v1 = pair(a1.y, b1.y);
            }
            *reinterpret_cast<uint32_t*>(dst + off * HD + ca) = codes4(u0, u1, pair(by, by));
            *reinterpret_cast<uint32_t*>(dst + off * HD + cb) = codes4(v0, v1, pair(by, by));
        }
        if (kept && e > before) {                               // the scale has grown: what stays is rounded again under it
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
        if (lane == 0) *scale = exp2_int(e);
    }
}

template <int HD, bool INTER, bool ALL>
__global__ void __launch_bounds__(kThreads) paged_e4m3_store_kernel(const PagedE4m3StoreArgs p, const int blocks, const int units) {
    pdl_launch_dependents();
    pdl_wait();
    if (static_cast<int>(blockIdx.x) < blocks) {
        const int unit = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
        if (unit < units) block_unit<HD, INTER, ALL>(p, unit);
    } else {
        constexpr int kLanes = HD / 8;
        store_unit<HD, INTER, ALL>(p.rows, static_cast<long long>(blockIdx.x - blocks) * (kThreads / kLanes) + threadIdx.x / kLanes);
    }
}

template <int HD, bool INTER, bool ALL>
cudaError_t launch(const PagedE4m3StoreArgs& a, cudaStream_t st) {
    const int units = (a.rows.rows + a.window - 1) / a.window * 2 * a.KV, blocks = (units + kThreads / 32 - 1) / (kThreads / 32);
    const long long q_units = static_cast<long long>(a.rows.rows) * ((a.rows.H + kStoreHeads - 1) / kStoreHeads), per = kThreads / (HD / 8);
    return launch_kernel(paged_e4m3_store_kernel<HD, INTER, ALL>, dim3(static_cast<unsigned>(blocks + (q_units + per - 1) / per)), dim3(kThreads), 0, st, a,
                         blocks, units);
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
