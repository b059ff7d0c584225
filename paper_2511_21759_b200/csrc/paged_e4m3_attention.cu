// Attention over a pool of 8 bits: few packed rows (query rows x heads of a group), or little work.  Formulas, masks and the division
// of the work: paged_attention.cu, paged.cuh; K and V of a position are code * scale, the scale that of its block of 16 positions.
//
// Both products run on f16 (mma.sync m16n8k16): a code is a number of f16, so a tile leaves shared memory as it came and two codes
// become a word of an operand by one instruction; scales stay outside.  The operand of 16 rows is K's and V's, that of 8 Q's and P's:
// S^T = K Q^T is 16 keys x 8 packed rows, O^T = V^T P^T 16 dims x 8 packed rows.  The other way round 4 packed rows, a token of a group
// of four heads, fill a quarter of each product and of the softmax.  NR: 8 or 16 packed rows an item, whose products share the codes.
//   S: a row of Q is brought into 1 .. 2 by a power of two first (f16 keeps 2^-25 of its largest value; the sums of products are fp32);
//      the scores are multiplied by that power, the softmax scale and the block's scale, all at once.
//   P V: beside the running maximum m of a row's scores x stands g, so that m + g + 15 is the running maximum of x + log2(V's scale).  The
//      weights that multiply codes are 2^(x - m + log2(scale) - g) <= 2^15, in f16: off by up to 2^-11 of themselves, or 2^-40 of the
//      row's largest.  The 15 are for contexts in which one key takes most (with weights up to 1 all that are 2^-25 of the largest
//      vanished, up to 2^-8 of the sum of 131072 keys, and all of the output where the one key's V is zero).  The sum takes them in fp32, block
//      by block, times 2^(g - log2(scale)): whatever the scales, the largest product of a weight and a scale keeps its precision.  (g and
//      not the maximum itself, which would lose the scales in large scores' last bits.)
// A warp multiplies 16 positions of a tile of 64: a block, with one scale of K and one of V.
//
// Places in a fragment are the dims that they have in memory: of 16 dims a lane has the four that ldmatrix gives it as one word, the same
// four of Q; V's words (transposed by pairs of bytes) hold two keys of two dims, the even ones for rows 0 .. 7 of the product and the odd
// ones for rows 8 .. 15.  P's fragments are S's, turned 8 x 8 at a time (movmatrix).
//
// What bounds it: the codes' way from memory.  A token of 48 requests of up to 8192 keys (32 + 8 heads of 128, 454 MB) takes 83 to 90 us from card
// to card, 0.77 to 0.83 of the copy rate, of two of up to 131072 keys 90 to 96, 0.81 to 0.86; the rest is the CTAs' start, their last tiles and the meeting of parts (one wave of
// CTAs with equal shares; the four waves that pays for bf16 took 89.8, half the bytes leave half the time to hide a start in).  A loader
// warp issues a box a page and a copy of scales a block, whose number a tile was the bound while K and V had a barrier each (153 us).  Three
// CTAs an SM with four stages of K and V 83.4, four CTAs with three stages 89.8; with items of 16, whose registers leave two CTAs, seven.
// 577 keys take 8.3 us: the latency of a launch, three dependent reads, two tiles and the parts.
#include "paged_e4m3.cuh"

namespace odb {

namespace {

constexpr int kItem = 1;                    // key tiles that an item costs beside its own
constexpr int kMinUnits = 2;                // units of a CTA, at least
constexpr int kKT = 64;                     // keys per tile
constexpr int kFewRows = 32;                // packed rows of the longest request, up to which few rows' kernel takes them
constexpr int kSmallUnits = 2304;           // up to here few rows' kernel for any number of rows
constexpr int kCopiedRows = 384;            // packed rows of the longest request above which requests that are alike take a copy in bf16
constexpr int kManyRows = 1024;             // packed rows a request, on average, from which the copy is right whatever the longest
constexpr int kMmaWarps = 4;                // 16 keys of a tile each
constexpr int kThreads = 32 * (kMmaWarps + 1);
constexpr int kBlocks = kKT / kPagedBlock;  // of a tile
constexpr float kRoom = 15.f;               // log2 of the largest weight, whose f16 ends below 2^16
template <int NR> constexpr int kCtas = NR == 8 ? 3 : 2;                    // of an SM
template <int HD> constexpr uint32_t kTileBytes = kKT * HD;                 // K or V of a tile
template <int HD, int NR> constexpr int kStages = HD == 128 ? (NR == 8 ? 4 : 7) : (NR == 8 ? 8 : 13);   // K and V tiles on the way or in use

template <int HD, int NR>
struct Shared {
    uint64_t full[kStages<HD, NR>], empty[kStages<HD, NR>];
    float scale[kStages<HD, NR>][2][kBlocks];   // of K's blocks, of V's
    float ml[kMmaWarps][NR][2];
    int last, abort;
};
template <int HD, int NR> constexpr uint32_t kSmem = kStages<HD, NR> * 2 * kTileBytes<HD> + (sizeof(Shared<HD, NR>) + 127) / 128 * 128;
template <int HD, int NR> constexpr bool kFits = kCtas<NR> * (kSmem<HD, NR> + 1024) <= 228 * 1024;
static_assert(kFits<128, 8> && kFits<64, 8> && kFits<128, 16> && kFits<64, 16>, "the CTAs share an SM");

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_warps_barrier() { asm volatile("bar.sync 1, %0;" ::"r"(32 * kMmaWarps) : "memory"); }
// over the lanes that hold a packed row's keys
__device__ __forceinline__ float row_max(float x) {
#pragma unroll
    for (int d = 4; d <= 16; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
    return x;
}
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
    for (int d = 4; d <= 16; d <<= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    return x;
}
// an 8 x 8 matrix of a warp, turned
__device__ __forceinline__ uint32_t turned(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
template <int HD, int NR>
__global__ void __launch_bounds__(kThreads, kCtas<NR>) paged_e4m3_attention_kernel(const __grid_constant__ CUtensorMap tm, const PagedAttnArgs a) {
    constexpr int KW = kKT / kMmaWarps;                         // keys of a warp
    static_assert(KW == kPagedBlock, "a warp's keys have one scale");
    constexpr int NG = NR / 8, NE = 2 * NG, NC = HD / 16;       // groups of eight packed rows; rows of a thread; chunks of 16 dims
    constexpr int S = kStages<HD, NR>;
    constexpr uint32_t kT = kTileBytes<HD>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* smem = smem_raw;
    const uint32_t tiles = smem_u32(smem);                      // [stage][K, V]
    auto* sh = reinterpret_cast<Shared<HD, NR>*>(smem + S * 2 * kT);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    volatile int* cta_abort = &sh->abort;

    if ((smem_u32(smem_raw) & 1023u) != 0) {                    // the swizzled tiles need 1024-byte alignment
        if (tid == 0) atomicExch(a.status, ODB_ERR_CUDA);
        pdl_wait();
        return;
    }
    if (tid == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm)) : "memory");
        for (int i = 0; i < S; ++i) {
            mbar_init(&sh->full[i], 1 + 2 * kBlocks);           // the tiles, and the lanes that copy their scales
            mbar_init(&sh->empty[i], kMmaWarps);
        }
        sh->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_launch_dependents();
    pdl_wait();
    // the ring's memory holds the sums until the start is found
    static_assert(sizeof(PagedScratch) <= S * 2 * kT, "the scratch fits the rings");
    PagedStart start;
    const bool any = paged_find_start<kThreads, kKT, kItem, true>(a, *reinterpret_cast<PagedScratch*>(smem), 1, kMinUnits, 0, start);
    if (!any) return;                                           // block-uniform
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the scratch's writes before the copies that take its place
    __syncthreads();

    PagedWalk<kKT, kItem> w(a, start);
    const int box_shift = min(a.page_shift, 6), box = 1 << box_shift;   // rows of a copy
    int stage = 0;
    uint32_t phase = 0;
    auto next_stage = [&]() {
        if (++stage == S) { stage = 0; phase ^= 1u; }
    };

    if (warp == kMmaWarps) {
        // ================= loader: lane i finds the rows of block i of a tile =================
        bool ok = true;
        int issued = 0;
        PagedPages pages;
        do {
            for (int t = w.t0; t < w.t1; ++t) {
                const int k0 = w.k.tile(t) * kKT;
                const int boxes = max(0, (min(kKT, w.k.hi - k0) + box - 1) >> box_shift), n_blocks = boxes << box_shift >> 4;
                const int b = lane & (kBlocks - 1);
                const int row = pages.rows<true>(a, w.q, w.seq, w.head, k0, b * kPagedBlock, b < n_blocks, a.k_row0);
                const bool there = row < a.pool_rows;
                if (issued >= S) ok = __all_sync(0xffffffffu, mbar_wait_bounded(&sh->empty[stage], phase ^ 1u, cta_abort, a.status));
                if (!ok) break;
                const uint32_t s = __shfl_sync(0xffffffffu, stage, 0), to = tiles + s * 2 * kT;
                uint64_t* full = &sh->full[s];
                if (paged_elect()) mbar_expect_tx(full, static_cast<uint32_t>(boxes) * box * HD * 2);
                __syncwarp();
                for (int c = 0; c < boxes; ++c) {
                    const int r = __shfl_sync(0xffffffffu, row, c << box_shift >> 4);
                    if (paged_elect()) {
                        tma_codes(to + c * box * HD, &tm, full, r);
                        tma_codes(to + kT + c * box * HD, &tm, full, r < a.pool_rows ? r + a.v_row0 - a.k_row0 : r);
                    }
                    __syncwarp();
                }
                if (lane < 2 * kBlocks) {                       // K's scales, then V's; a page that is none reads as zeros
                    float* scale = &sh->scale[s][0][lane];
                    if (b < n_blocks && !there) {
                        *scale = 1.f;
                        mbar_arrive(full);                      // a copy's arrival would not wait for this lane's own write
                    } else {
                        if (b < n_blocks) copy4(smem_u32(scale), a.scales + (row + (lane < kBlocks ? 0 : a.v_row0 - a.k_row0)) / kPagedBlock);
                        copies_arrive(full);
                    }
                }
                __syncwarp();
                next_stage();
                ++issued;
            }
        } while (ok && w.next());
        if (!ok) {   // copies in flight land before the memory goes away
            const long long t0 = clock64();
            for (int j = max(0, issued - S); j < issued; ++j)
                while (!mbar_try_wait_parity(&sh->full[j % S], static_cast<uint32_t>(j / S) & 1u) && clock64() - t0 < kWaitLimitCycles / 8) {
                }
        }
        return;
    }

    // ================= the products =================
    // This thread's packed rows of the tile, e = 0 .. NE - 1, in the fragments of scores and outputs.
    auto row_of = [&](int e) { return 8 * (e >> 1) + 2 * (lane & 3) + (e & 1); };
    // chunk ch of 16 bytes of key c of a tile
    auto chunk_at = [&](int c, int ch) -> uint32_t {
        return HD == 128 ? static_cast<uint32_t>(c * 128 + ((ch ^ (c & 7)) << 4)) : static_cast<uint32_t>(c * 64 + ((ch ^ (c >> 1 & 3)) << 4));
    };
    do {
        const int rows = min(NR, w.q.n * a.G - w.rt * NR);      // packed rows of this item
        uint32_t qf[NG][NC][2];
        int pos[NE];
        float unit[NE];                                         // what a score's product is multiplied by, but for K's scale
#pragma unroll
        for (int n = 0; n < NG; ++n) {
            const int idx = w.rt * NR + min(8 * n + (lane >> 2), rows - 1), i = a.by_group(idx);   // rows behind the last repeat it
            const __nv_bfloat16* qp = a.q + static_cast<size_t>(w.q.row0 + i) * a.q_stride + (w.head * a.G + idx - i * a.G) * HD + (lane & 3) * 4;
            uint2 x[NC];
            uint32_t top = 0;
#pragma unroll
            for (int c = 0; c < NC; ++c) x[c] = *reinterpret_cast<const uint2*>(qp + c * 16);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                top = max(top, max(x[c].x & 0x7fffu, x[c].x >> 16 & 0x7fffu));
                top = max(top, max(x[c].y & 0x7fffu, x[c].y >> 16 & 0x7fffu));
            }
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int ex = q_exponent(top);
            const float by = exp2_int(-ex), mine = exp2_int(ex) * a.scale_log2;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                qf[n][c][0] = paged_f16x2(__uint_as_float(x[c].x << 16) * by, __uint_as_float(x[c].x & 0xffff0000u) * by);
                qf[n][c][1] = paged_f16x2(__uint_as_float(x[c].y << 16) * by, __uint_as_float(x[c].y & 0xffff0000u) * by);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                unit[2 * n + j] = __shfl_sync(0xffffffffu, mine, (2 * (lane & 3) + j) * 4);
                pos[2 * n + j] = w.q.first + a.by_group(w.rt * NR + min(row_of(2 * n + j), rows - 1));
            }
        }
        const bool final = w.whole();
        const int c0 = final ? 0 : w.first_cta(), c1 = final ? 0 : w.last_cta();   // while K is on its way
        const int idx_last = w.rt * NR + rows - 1;
        const int p_min = w.q.first + a.by_group(w.rt * NR), p_max = w.q.first + a.by_group(idx_last);
        // keys from all_lo on and below all_hi are seen by all rows of the item
        const int all_hi = static_cast<int>(max(0ll, min(static_cast<long long>(w.q.len), static_cast<long long>(p_min) + a.right + 1)));
        const int all_lo = static_cast<int>(max(-1ll, static_cast<long long>(p_max) - a.left));
        // of 16 dims dims 2 (lane / 4) and the next one, each of two rows
        float o[NG][NC][4], m[NE], g[NE], l[NE];
#pragma unroll
        for (int e = 0; e < NE; ++e) {
            m[e] = g[e] = -INFINITY;
            l[e] = 0.f;
        }
#pragma unroll
        for (int n = 0; n < NG; ++n)
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[n][c][j] = 0.f;

        for (int t = w.t0; t < w.t1; ++t) {
            const int k0 = w.k.tile(t) * kKT + warp * KW;         // this warp's first key
            // Behind an expired wait the warp goes on through the tiles without their products: it must not be missing at a barrier.
            const bool ok = __all_sync(0xffffffffu, mbar_wait_bounded(&sh->full[stage], phase, cta_abort, a.status));
            const uint32_t sk = tiles + stage * 2 * kT, sv = sk + kT;
            const bool any_key = k0 < w.k.hi && (k0 + KW > w.k.lo || k0 < a.sinks);   // some row of the item sees some key
            if (ok && any_key) {
                const bool whole = k0 + KW <= all_hi && (k0 >= all_lo || k0 + KW <= a.sinks);
                if (!whole) {
                    // V in places that a row does not see: zero where no row sees it, by the element where it is NaN
                    constexpr int kChunks = KW * HD / 16 / 32;  // 16-byte chunks of a lane
                    bool nan = false;
#pragma unroll
                    for (int i = 0; i < kChunks; ++i) {
                        const int c16 = i * 32 + lane, kc = c16 / NC, ch = c16 % NC, key = k0 + kc;
                        const uint32_t ad = sv + chunk_at(warp * KW + kc, ch);
                        uint32_t v[4];
                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(ad) : "memory");
                        const bool out = key >= w.k.hi || (key < w.k.lo && key >= a.sinks);
                        if (out)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(ad), "r"(0) : "memory");
                        else
                            nan = nan || odd_codes(v[0]) || odd_codes(v[1]) || odd_codes(v[2]) || odd_codes(v[3]);
                    }
                    nan = __any_sync(0xffffffffu, nan);
                    __syncwarp();                  // all have looked
                    if (nan) {
#pragma unroll 1
                        for (int kc = 0; kc < KW; ++kc) {       // rare: NaN in V, seen by some of the rows
                            const int key = k0 + kc;
                            bool seen[NE];
#pragma unroll
                            for (int e = 0; e < NE; ++e) seen[e] = key < w.q.len && key - a.right <= pos[e] && (key + a.left >= pos[e] || key < a.sinks);
#pragma unroll
                            for (int c = 0; c < NC; ++c) {
                                unsigned short v;
                                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(sv + chunk_at(warp * KW + kc, c) + (lane >> 2) * 2) : "memory");
#pragma unroll
                                for (int d = 0; d < 2; ++d)
                                    if ((v >> 8 * d & 0x7f) == 0x7f)
#pragma unroll
                                        for (int e = 0; e < NE; ++e)
                                            if (seen[e]) o[e >> 1][c][2 * d + (e & 1)] = __uint_as_float(0x7fffffffu);
                            }
                        }
                        __syncwarp();
#pragma unroll 1
                        for (int i = 0; i < KW * HD / 4 / 32; ++i) {
                            const int c4 = i * 32 + lane, kc = c4 / (HD / 4), dd = c4 % (HD / 4);
                            const uint32_t ad = sv + chunk_at(warp * KW + kc, dd >> 2) + (dd & 3) * 4;
                            uint32_t v;
                            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(ad) : "memory");
                            asm volatile("st.shared.b32 [%0], %1;" ::"r"(ad), "r"(without_nan(v)) : "memory");
                        }
                        __syncwarp();
                    }
                    __syncwarp();
                }
                uint32_t kx[NC / 2][4], vx[NC / 2][4];          // both tiles' words at once: V's become f16 while the scores are on their way
#pragma unroll
                for (int c = 0; c < NC / 2; ++c)                // keys 0 .. 7 of chunk 2 c and the next, then keys 8 .. 15
                    ldsm4(sk + chunk_at(warp * KW + (lane & 7) + ((lane >> 4) << 3), 2 * c + (lane >> 3 & 1)), kx[c]);
#pragma unroll
                for (int c = 0; c < NC / 2; ++c)                // keys 0 .. 7 and 8 .. 15 of chunk 2 c, then of the next
                    ldsm4_t(sv + chunk_at(warp * KW + (lane & 15), 2 * c + (lane >> 4)), vx[c]);
                float s[NG][4], odd[NG][4];                     // keys lane / 4 and 8 behind it, each of two rows; every other step in sums of its own
#pragma unroll
                for (int n = 0; n < NG; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[n][j] = odd[n][j] = 0.f;
#pragma unroll
                for (int c = 0; c < NC / 2; ++c)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t ka[4] = {low_codes(kx[c][h]), low_codes(kx[c][2 + h]), high_codes(kx[c][h]), high_codes(kx[c][2 + h])};
#pragma unroll
                        for (int n = 0; n < NG; ++n) mma(h ? odd[n] : s[n], ka, qf[n][2 * c + h][0], qf[n][2 * c + h][1]);
                    }
                const float ks = sh->scale[stage][0][warp];
                const float log_vs = static_cast<float>(static_cast<int>(__float_as_uint(sh->scale[stage][1][warp]) >> 23) - 127);
                float top[NE];
#pragma unroll
                for (int e = 0; e < NE; ++e) {
                    float* x = &s[e >> 1][e & 1];               // x[0], x[2]
                    const float by = finite_factor(unit[e] * ks);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        x[2 * h] = __fmul_rn(x[2 * h] + odd[e >> 1][2 * h + (e & 1)], by);   // rounded as the maximum is
                        if (!whole) {
                            const int key = k0 + h * 8 + (lane >> 2);
                            const bool seen = key < w.q.len && key - a.right <= pos[e] && (key + a.left >= pos[e] || key < a.sinks);
                            x[2 * h] = seen ? x[2 * h] : -INFINITY;
                        }
                    }
                    top[e] = row_max(fmaxf(x[0], x[2]));
                }
                float factor[NE], shift[NE], more[NE];
                bool rare = false;                              // O has to be rescaled
#pragma unroll
                for (int e = 0; e < NE; ++e) {
                    factor[e] = 1.f;
                    shift[e] = more[e] = 0.f;
                    const float mn = fmaxf(m[e], top[e]);
                    if (mn == -INFINITY) continue;              // the row has seen no key
                    const float before = m[e] - mn + g[e], gn = fmaxf(before, top[e] - mn + (log_vs - kRoom));
                    l[e] *= ex2_approx(m[e] - mn);
                    factor[e] = ex2_approx(before - gn);
                    shift[e] = mn;
                    more[e] = log_vs - gn;
                    m[e] = mn;
                    g[e] = gn;
                    rare = rare || before != gn;
                }
                float sum[NE];
#pragma unroll
                for (int e = 0; e < NE; ++e) {
                    float* x = &s[e >> 1][e & 1];
                    const float y0 = x[0] - shift[e], y1 = x[2] - shift[e];
                    x[0] = ex2_approx(y0 + more[e]);
                    x[2] = ex2_approx(y1 + more[e]);
                    // weights that a far larger scale elsewhere lets vanish still count in the sum
                    sum[e] = more[e] < -60.f ? ex2_approx(y0) + ex2_approx(y1) : (x[0] + x[2]) * ex2_approx(-more[e]);
                }
#pragma unroll
                for (int e = 0; e < NE; ++e) l[e] += sum[e];
                uint32_t p[NG][2];
#pragma unroll
                for (int n = 0; n < NG; ++n)
#pragma unroll
                    for (int h = 0; h < 2; ++h) p[n][h] = turned(paged_f16x2(s[n][2 * h], s[n][2 * h + 1]));
                if (__any_sync(0xffffffffu, rare)) {
#pragma unroll
                    for (int n = 0; n < NG; ++n)
#pragma unroll
                        for (int c = 0; c < NC; ++c)
#pragma unroll
                            for (int j = 0; j < 4; ++j) o[n][c][j] *= factor[2 * n + (j & 1)];
                }
#pragma unroll
                for (int c = 0; c < NC / 2; ++c)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {               // a word: two keys of an even dim, then of the odd one
                        const uint32_t y = __byte_perm(vx[c][2 * h], 0, 0x3120), z = __byte_perm(vx[c][2 * h + 1], 0, 0x3120);
                        const uint32_t va[4] = {low_codes(y), high_codes(y), low_codes(z), high_codes(z)};
#pragma unroll
                        for (int n = 0; n < NG; ++n) mma(o[n][2 * c + h], va, p[n][0], p[n][1]);
                    }
                if (!whole) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // this warp's writes to V before the next copy into it
            }
            if (t + 1 == w.t1) break;                 // the item's last V tile stays: its place is where the warps meet
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->empty[stage]);
            next_stage();
        }

        // ---- the warps that share the rows meet ----
#pragma unroll
        for (int e = 0; e < NE; ++e) l[e] = row_sum(l[e]);
        {
            if (lane < 4) {
#pragma unroll
                for (int e = 0; e < NE; ++e) {
                    sh->ml[warp][row_of(e)][0] = m[e];
                    sh->ml[warp][row_of(e)][1] = l[e];
                }
            }
            mma_warps_barrier();                                // all have read the last V tile
            float* merge = reinterpret_cast<float*>(smem + stage * 2 * kT + kT);
            static_assert(kMmaWarps / 2 * 8 * HD * 4 <= kT, "half the warps' outputs of eight rows fit a tile");
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                float M = -INFINITY, L = 0.f;
#pragma unroll
                for (int i = 0; i < kMmaWarps; ++i) M = fmaxf(M, sh->ml[i][row_of(e)][0]);
#pragma unroll
                for (int i = 0; i < kMmaWarps; ++i) {
                    const float* x = sh->ml[i][row_of(e)];
                    L += paged_weight(x[0], M) * x[1];
                }
                const float f = g[e] == -INFINITY ? 0.f : ex2_approx(m[e] - M + (g[e] + kRoom)) * 0x1p-15f;   // from here on in units of 2^M, without scales
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    o[e >> 1][c][e & 1] *= f;
                    o[e >> 1][c][2 + (e & 1)] *= f;
                }
                m[e] = M;
                l[e] = L;
            }
#pragma unroll
            for (int n = 0; n < NG; ++n) {
                if (8 * n >= rows) break;
#pragma unroll
                for (int half = kMmaWarps / 2; half >= 1; half >>= 1) {  // the upper half of the warps hands over to the lower
                    float* mb = merge + (warp % half) * NC * 4 * 32 + lane;
                    if (warp >= half && warp < 2 * half) {
#pragma unroll
                        for (int c = 0; c < NC; ++c)
#pragma unroll
                            for (int j = 0; j < 4; ++j) mb[(c * 4 + j) * 32] = o[n][c][j];
                    }
                    mma_warps_barrier();
                    if (warp < half) {
#pragma unroll
                        for (int c = 0; c < NC; ++c)
#pragma unroll
                            for (int j = 0; j < 4; ++j) o[n][c][j] += mb[(c * 4 + j) * 32];
                    }
                    mma_warps_barrier();
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->empty[stage]);
            next_stage();
        }

        // ---- results, or this CTA's part of them ----
        const size_t part = paged_part(a, blockIdx.x, w.t0 == 0);
        if (warp == 0) {
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                const int r = row_of(e);
                if (r >= rows) continue;
                if (final) {
                    const int idx = w.rt * NR + r, i = a.by_group(idx), head = w.head * a.G + idx - i * a.G;
                    const size_t row = static_cast<size_t>(w.q.row0 + i);
                    const float inv = l[e] == 0.f ? 0.f : 1.0f / l[e];
                    __nv_bfloat16* op = a.out + row * a.out_stride + head * HD + (lane >> 2) * 2;
#pragma unroll
                    for (int c = 0; c < NC; ++c)
                        *reinterpret_cast<uint32_t*>(op + c * 16) = paged_bf16x2(o[e >> 1][c][e & 1] * inv, o[e >> 1][c][2 + (e & 1)] * inv);
                    if (a.lse && lane < 4) a.lse[row * a.H + head] = paged_lse(m[e], l[e]);
                } else {
                    float* op = a.part_o + (part + r) * HD + (lane >> 2) * 2;
#pragma unroll
                    for (int c = 0; c < NC; ++c) *reinterpret_cast<float2*>(op + c * 16) = make_float2(o[e >> 1][c][e & 1], o[e >> 1][c][2 + (e & 1)]);
                    if (lane < 4) *reinterpret_cast<float2*>(a.part_ml + (part + r) * 2) = make_float2(m[e], l[e]);
                }
            }
        }
        if (!final) {
            mma_warps_barrier();
            if (tid == 0) {
                // releases what the barrier has put in front of it, and acquires what the other CTAs have released
                unsigned before;
                asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(a.arrivals + c0) : "memory");
                const bool last = before == static_cast<unsigned>(c1 - c0);
                if (last) a.arrivals[c0] = 0;                    // for the next launch; an item is counted at the CTA it begins in
                sh->last = last;
            }
            mma_warps_barrier();
            if (sh->last) {
                auto add_up = [&](auto sum) {
                    constexpr int RB = sizeof(sum.M) / sizeof(float);
                    if (warp >= rows) return;
                    sum.rows(a, c0, c1, warp, kMmaWarps, rows);
#pragma unroll
                    for (int k = 0; k < RB; ++k)
                        if (warp + k * kMmaWarps < rows) sum.write(a, k, w.q.row0, w.head, w.rt * NR + warp + k * kMmaWarps);
                };
                if (rows <= kMmaWarps) add_up(PagedSum<HD, 1>{});
                else if (NR == 8 || rows <= 2 * kMmaWarps) add_up(PagedSum<HD, 2>{});
                else add_up(PagedSum<HD, 4>{});
                mma_warps_barrier();                             // sh->last has been read by all
            }
        }
    } while (w.next());
}

template <int HD, int NR>
cudaError_t launch(PagedAttnArgs a, const CUtensorMap& tmap, int sms, cudaStream_t st) {
    static std::atomic<unsigned long long> attr_done{0};
    cudaError_t e = set_smem_limit_once(attr_done, paged_e4m3_attention_kernel<HD, NR>, static_cast<int>(kSmem<HD, NR>));
    if (e != cudaSuccess) return e;
    a.tile_rows = NR;
    a.by_rows = PagedDiv::by(NR);
    a.part_rows = NR;
    a.at_once = kCtas<NR> * sms;
    a.by_once = PagedDiv::by(a.at_once);
    // one wave of CTAs with equal shares; no more than the table's width leaves work for
    const long long tiles = (static_cast<long long>(a.table_stride) << a.page_shift) / kKT + 1 + kItem,
                    most = (static_cast<long long>(a.max_rows) * a.G / NR + a.n_seqs) * a.KV * tiles / kMinUnits + 1;
    static_assert(kPagedMaxCtas * 16 <= kPagedPartRows, "parts");
    const int grid = static_cast<int>(most < a.at_once ? most : a.at_once);
    return launch_kernel(paged_e4m3_attention_kernel<HD, NR>, dim3(grid), dim3(kThreads), kSmem<HD, NR>, st, tmap, a);
}

}  // namespace

// Which kernel (8, 16: few rows' for items of so many; 1: one Q tile of the tensor cores; 2: the copy in bf16), by the packed rows of the
// longest request and by the work, as for a pool of bf16 (paged_attention_kernel_of).  Both sides, 8 K/V heads of 128, in us:
//   items of 8 or 16 rows: tokens of 16 requests x 8192 keys, groups of 8 heads: 33 | 43, of 12: 52 | 46; 20 packed rows, 4096 keys: 73 | 78,
//     32 rows: 90 | 80 (a third item of 8 costs less than a second of 16 does)
//   kFewRows, 16 requests, 4096 keys: 32 packed rows 80 | 92 on the tensor cores, 48 rows 112 | 92
//   kSmallUnits, blocks of 32 rows x group 4: 1536 units (4 requests of 256 keys) 12.5 | 23.4, 2304 (2 of 1024) 22.7 | 24.8, 4608 (4 of 1024)
//     31 | 26
//   kCopiedRows, 16 requests, 4096 keys: 384 packed rows 247 | 287 with the copy, 512 rows 321 | 291, 1024 rows 616 | 463
// The copy wants the requests alike, for all pages are copied, those of single tokens too.  Alike is what the kernel over bf16 calls so (the
// longest up to three times the mean), where that costs no copy: a prompt beside one or two tokens counts, and where they have long contexts
// the copy is the slower side.  A chunk of 512 rows at 4096 keys x group 4, copy | tensor cores over codes (those with more tokens take the
// latter): beside one token of 32768 keys 112 | 116, beside two 172 | 145; beside one of 131072 keys 310 | 220, beside two 557 | 324.
// Head dim 64 takes the same limits, none of which was looked for there; the copy against the codes: a refresh of 4 x 900 - 1536 rows, 32 K/V
// heads, 82 | 167, the chunk beside a token of 32768 keys 82 | 100, of 131072 205 | 186.
int paged_e4m3_attention_kernel_of(int n_seqs, int max_rows, int max_new, int group, int kv_heads, long long longest, long long out_stride, bool room) {
    const long long all = static_cast<long long>(max_rows) * group, mean = (max_rows + n_seqs - 1ll) / n_seqs * group,
                    mine = max_new > 0 ? static_cast<long long>(max_new) * group : mean, tiles = longest / kKT + 1;
    // units of all items together and what is added to them on the way, with rows that follow one another
    auto fits = [&](int tile_rows, int item) {
        return (static_cast<double>(all / tile_rows) + n_seqs) * kv_heads * static_cast<double>(tiles + item) < 2147483648.0 - 65536;
    };
    const int few = (mine <= 8 || (mine > 16 && mine <= 24)) && fits(8, kItem) ? 8 : fits(16, kItem) ? 16 : -1;
    if (group <= kPagedTcMaxGroup && out_stride <= 1ll << 27) {
        const int tile = kPagedTcMaxGroup / group * group;
        const double units = static_cast<double>((all + 15ll * n_seqs) / 16) * kv_heads * static_cast<double>(tiles + kItem);
        if ((mine > kFewRows && units > kSmallUnits) || few < 0) {
            const bool alike = max_new > 0 ? static_cast<long long>(max_new) * n_seqs <= 3ll * max_rows : n_seqs == 1 || mean >= kManyRows;
            if (room && ((mine > kCopiedRows && alike) || !fits(tile, kPagedTcItem)) && fits(2 * tile, kPagedTcItem)) return 2;
            return fits(tile, kPagedTcItem) ? 1 : few;
        }
    }
    return few;
}

cudaError_t launch_paged_e4m3_attention(PagedAttnArgs a, const CUtensorMap& map, int hd, int kernel, int sms, cudaStream_t st) {
    if (sms < 1 || 2 * sms * 128 > kPagedPartRows || 3 * sms > kPagedMaxCtas) return cudaErrorInvalidValue;   // the workspace's size
    a.by_group = PagedDiv::by(a.G);
    if (kernel == 8) return hd == 128 ? launch<128, 8>(a, map, sms, st) : launch<64, 8>(a, map, sms, st);
    if (kernel == 16) return hd == 128 ? launch<128, 16>(a, map, sms, st) : launch<64, 16>(a, map, sms, st);
    return launch_paged_e4m3_attention_tc(a, map, hd, sms, st);
}

}  // namespace odb
