// Attention over a pool of 8 bits: few packed rows (query rows x heads of a group), or little work.  Formulas, masks and the division
// of the work: paged_attention.cu, paged.cuh; K and V of a position are code * scale, the scale that of its block of 16 positions.
//
// Both products run on f16 (mma.sync m16n8k16): a code is a number of f16, so a tile leaves shared memory as it came and two codes
// become a word of an operand by one instruction; scales stay outside.
//   S: a row of Q is brought into 1 .. 2 by a power of two first (f16 keeps 2^-25 of its largest value; the sums of products are fp32);
//      the scores are multiplied by that power, the softmax scale and the block's scale, all at once.
//   P V: beside the running maximum m of a row's scores x stands g, so that m + g is the running maximum of x + log2(V's scale).  The
//      weights that multiply codes are 2^(x - m + log2(scale) - g) <= 1, in f16 (up to 2^-11 of themselves, or 2^-25 of the row's
//      largest), the sum's 2^(x - m), in fp32: whatever the scales, the largest product of a weight and a scale keeps its precision.
//      (g and not the maximum itself, which would lose the scales in large scores' last bits.)
// A warp multiplies 16 positions of a tile of 64: one block, one scale of K and one of V.
//
// Places in a fragment are the dims that they have in memory: of 16 dims a lane has the four that ldmatrix gives it as one word, the same
// four of Q; V's words (transposed by pairs of bytes) hold two keys of two dims, of which the even and the odd ones go to products of
// their own, and the output's fragments are again four dims in a row.
#include "paged_e4m3.cuh"

namespace odb {

namespace {

constexpr int kKT = 64;                    // keys per tile
constexpr int kItem = 1;                    // key tiles that an item costs beside its own
constexpr int kMinUnits = 2, kFullUnits = 24;   // units of a CTA, at least; where all places on the SMs have work
constexpr int kRows = 16;                   // packed rows of an item
constexpr int kMmaWarps = 4;
constexpr int kThreads = 32 * (kMmaWarps + 1);
template <int HD> constexpr int kSlots = HD == 128 ? 7 : 13;                // K tiles on the way or in use, and V tiles
template <int HD> constexpr uint32_t kTileBytes = kKT * HD;                 // K or V of a tile

template <int S>
struct Barriers {
    uint64_t k_full[S], v_full[S], k_empty[S], v_empty[S];
    float ml[kMmaWarps][16][2];
    float k_scale[S][4], v_scale[S][4];     // of the tile's blocks
    int last, abort;
};
template <int HD> constexpr uint32_t kSmem = 2 * kSlots<HD> * kTileBytes<HD> + (sizeof(Barriers<kSlots<HD>>) + 127) / 128 * 128;
static_assert(2 * (kSmem<128> + 1024) <= 228 * 1024 && 2 * (kSmem<64> + 1024) <= 228 * 1024, "two CTAs share an SM");

// a box of rows of the pool
__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* tmap, uint64_t* bar, int row) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_u32(bar)), "r"(0), "r"(row)
                 : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
// an arrival once this thread's copies so far have landed; counted among the barrier's
__device__ __forceinline__ void copies_arrive(uint64_t* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
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
__device__ __forceinline__ float quad_max(float x) {
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
    return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
}
__device__ __forceinline__ float quad_sum(float x) {
    x += __shfl_xor_sync(0xffffffffu, x, 1);
    return x + __shfl_xor_sync(0xffffffffu, x, 2);
}
__device__ __forceinline__ uint32_t f16x2(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t low_codes(uint32_t w) { return f16x2_of(static_cast<unsigned short>(w)); }
__device__ __forceinline__ uint32_t high_codes(uint32_t w) { return f16x2_of(static_cast<unsigned short>(w >> 16)); }
// some code of the four is NaN: 0x7f + 1 carries into the sign's place
__device__ __forceinline__ bool odd_codes(uint32_t four) { return ((four & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

template <int HD>
__global__ void __launch_bounds__(kThreads, 2) paged_e4m3_attention_kernel(const __grid_constant__ CUtensorMap tm, const PagedAttnArgs a) {
    constexpr int KW = kKT / kMmaWarps;                         // keys of a warp: a block of the scales
    static_assert(KW == kPagedBlock, "a warp's keys have one scale");
    constexpr int kS = kSlots<HD>, ND = HD / 8;
    constexpr uint32_t kT = kTileBytes<HD>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* smem = smem_raw;
    const uint32_t k_tiles = smem_u32(smem), v_tiles = k_tiles + kS * kT;
    auto* sh = reinterpret_cast<Barriers<kS>*>(smem + 2 * kS * kT);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    volatile int* cta_abort = &sh->abort;

    if ((smem_u32(smem_raw) & 1023u) != 0) {                    // the swizzled tiles need 1024-byte alignment
        if (tid == 0) atomicExch(a.status, ODB_ERR_CUDA);
        pdl_wait();
        return;
    }
    if (tid == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm)) : "memory");
        for (int i = 0; i < kS; ++i) {
            mbar_init(&sh->k_full[i], 1 + 4);                   // the tile, and the lanes that copy its scales
            mbar_init(&sh->v_full[i], 1 + 4);
            mbar_init(&sh->k_empty[i], kMmaWarps);
            mbar_init(&sh->v_empty[i], kMmaWarps);
        }
        sh->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_launch_dependents();
    pdl_wait();
    // the ring's memory holds the sums until the start is found
    static_assert(sizeof(PagedScratch) <= 2 * kSlots<64> * kTileBytes<64>, "the scratch fits the rings");
    PagedStart start;
    const bool any = paged_find_start<kThreads, kKT, kItem, true>(a, *reinterpret_cast<PagedScratch*>(smem), kPagedWaves, kMinUnits, kFullUnits, start);
    if (!any) return;                                           // block-uniform
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the scratch's writes before the copies that take its place
    __syncthreads();

    PagedWalk<kKT, kItem> w(a, start);
    const int box_shift = min(a.page_shift, 6), box = 1 << box_shift;   // rows of a copy
    struct Ring {
        int slot = 0;
        uint32_t phase = 0;
        __device__ __forceinline__ void next() {
            if (++slot == kS) { slot = 0; phase ^= 1u; }
        }
    } kr, vr;

    if (warp == kMmaWarps) {
        // ================= loader =================
        bool ok = true;
        int issued = 0;
        PagedPages pages;
        do {
            for (int t = w.t0; t < w.t1 && ok; ++t) {
                const int k0 = w.k.tile(t) << 6;
                const int boxes = max(0, (min(kKT, w.k.hi - k0) + box - 1) >> box_shift);
                const uint32_t bytes = static_cast<uint32_t>(boxes) * box * HD;
                auto load = [&](Ring& r, uint64_t* empty, uint64_t* full, uint32_t tiles, float (*scales)[4], int base) {
                    if (issued >= kS) ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(&empty[r.slot], r.phase ^ 1u, cta_abort, a.status));
                    if (!ok) return;
                    const uint32_t slot = __shfl_sync(0xffffffffu, r.slot, 0), to = tiles + slot * kT;
                    if (paged_elect()) mbar_expect_tx(&full[slot], bytes);
                    __syncwarp();
                    for (int c = 0; c < boxes; ++c) {
                        const int row = pages.row<true, true>(a, w.q, w.seq, w.head, k0 + (c << box_shift), base);
                        if (paged_elect()) tma_rows(to + c * box * HD, &tm, &full[slot], row);
                        __syncwarp();
                        const int b = lane - (c << box_shift >> 4);                   // block of the box
                        if (lane < 4 && b >= 0 && b < box >> 4) {
                            if (row < a.pool_rows) copy4(smem_u32(&scales[slot][lane]), a.scales + (row >> 4) + b);
                            else scales[slot][lane] = 1.f;                            // a page that is none reads as zeros
                        }
                    }
                    if (lane < 4) copies_arrive(&full[slot]);
                    __syncwarp();
                    r.next();
                };
                load(kr, sh->k_empty, sh->k_full, k_tiles, sh->k_scale, a.k_row0);
                load(vr, sh->v_empty, sh->v_full, v_tiles, sh->v_scale, a.v_row0);
                if (!ok) break;
                ++issued;
            }
        } while (ok && w.next());
        if (!ok) {   // copies in flight land before the memory goes away
            const long long t0 = clock64();
            auto land = [&](uint64_t* full) {
                for (int j = max(0, issued + 1 - kS); j <= issued; ++j)   // the last one may have a K tile only
                    while (!mbar_try_wait_parity(&full[j % kS], static_cast<uint32_t>(j / kS) & 1u) && clock64() - t0 < kWaitLimitCycles / 8) {
                    }
            };
            land(sh->k_full);
            land(sh->v_full);
        }
        return;
    }

    // ================= the products =================
    const int r_lo = lane >> 2;                     // this thread's rows of the tile: r_lo and r_lo + 8
    // chunk ch of 16 bytes of key c of a tile
    auto chunk_at = [&](int c, int ch) -> uint32_t {
        return HD == 128 ? static_cast<uint32_t>(c * 128 + ((ch ^ (c & 7)) << 4)) : static_cast<uint32_t>(c * 64 + ((ch ^ (c >> 1 & 3)) << 4));
    };
    do {
        const int rows = min(kRows, w.q.n * a.G - w.rt * kRows);  // packed rows of this item
        uint32_t qf[HD / 16][4];
        int pos[2];
        size_t at[2];                                           // row of q, out and lse, in heads
        float unit[2];                                          // what a score's product is multiplied by, but for K's scale
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = min(r_lo + 8 * e, rows - 1), idx = w.rt * kRows + r, i = a.by_group(idx);   // rows behind the last repeat it
            pos[e] = w.q.first + i;
            at[e] = static_cast<size_t>(w.q.row0 + i);
            const __nv_bfloat16* qp = a.q + at[e] * a.q_stride + (w.head * a.G + idx - i * a.G) * HD + (lane & 3) * 4;
            uint2 x[HD / 16];
            uint32_t top = 0;
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) x[kk] = *reinterpret_cast<const uint2*>(qp + kk * 16);
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) {
                top = max(top, max(x[kk].x & 0x7fffu, x[kk].x >> 16 & 0x7fffu));
                top = max(top, max(x[kk].y & 0x7fffu, x[kk].y >> 16 & 0x7fffu));
            }
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int ex = min(max(static_cast<int>(top >> 7) - 127, -126), 126);     // an infinity stays one
            const float by = exp2_int(-ex);
            unit[e] = exp2_int(ex) * a.scale_log2;
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) {
                qf[kk][e] = f16x2(__uint_as_float(x[kk].x << 16) * by, __uint_as_float(x[kk].x & 0xffff0000u) * by);
                qf[kk][2 + e] = f16x2(__uint_as_float(x[kk].y << 16) * by, __uint_as_float(x[kk].y & 0xffff0000u) * by);
            }
        }
        const bool final = w.whole();
        const int c0 = final ? 0 : w.first_cta(), c1 = final ? 0 : w.last_cta();   // while K is on its way
        const int idx_last = w.rt * kRows + rows - 1;
        const int p_min = w.q.first + a.by_group(w.rt * kRows), p_max = w.q.first + a.by_group(idx_last);
        // keys from all_lo on and below all_hi are seen by all rows of the item
        const int all_hi = static_cast<int>(max(0ll, min(static_cast<long long>(w.q.len), static_cast<long long>(p_min) + a.right + 1)));
        const int all_lo = static_cast<int>(max(-1ll, static_cast<long long>(p_max) - a.left));
        float o[ND][4];                                         // o[2 c], o[2 c + 1]: the even and the odd dims of 16 c ..
        float m[2] = {-INFINITY, -INFINITY}, g[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[d][j] = 0.f;

        for (int t = w.t0; t < w.t1; ++t) {
            const int k0 = (w.k.tile(t) << 6) + warp * KW;        // this warp's first key
            // Behind an expired wait the warp goes on through the tiles without their products: it must not be missing at a barrier.
            bool ok = __all_sync(0xffffffffu, mbar_wait_bounded(&sh->k_full[kr.slot], kr.phase, cta_abort, a.status));
            bool k_read = false;
            auto k_done = [&]() {                               // K's place is free again before the softmax
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh->k_empty[kr.slot]);
                kr.next();
                k_read = true;
            };
            const uint32_t sk = k_tiles + kr.slot * kT, sv = v_tiles + vr.slot * kT;
            const bool any_key = k0 < w.k.hi && (k0 + KW > w.k.lo || k0 < a.sinks);   // some row of the item sees some key
            if (ok && any_key) {
                float s[2][4], odd[2][4];                       // every other step in sums of its own: half as long a chain of products
#pragma unroll
                for (int nb = 0; nb < 2; ++nb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[nb][j] = odd[nb][j] = 0.f;
                const int key_k = warp * KW + (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
                for (int kk = 0; kk < HD / 16; kk += 2) {
                    uint32_t b[4];                              // keys 0 .. 7 of dims 16 kk .. and the next 16, then keys 8 .. 15
                    ldsm4(sk + chunk_at(key_k, kk + (lane >> 3 & 1)), b);
                    mma(s[0], qf[kk], low_codes(b[0]), high_codes(b[0]));
                    mma(s[1], qf[kk], low_codes(b[2]), high_codes(b[2]));
                    mma(odd[0], qf[kk + 1], low_codes(b[1]), high_codes(b[1]));
                    mma(odd[1], qf[kk + 1], low_codes(b[3]), high_codes(b[3]));
                }
                const float ks = sh->k_scale[kr.slot][warp];
                k_done();
                const bool whole = k0 + KW <= all_hi && (k0 >= all_lo || k0 + KW <= a.sinks);
                float top[2] = {-INFINITY, -INFINITY};
                const float by[2] = {unit[0] * ks, unit[1] * ks};
#pragma unroll
                for (int nb = 0; nb < 2; ++nb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float x = (s[nb][j] + odd[nb][j]) * by[j >> 1];
                        if (!whole) {
                            const int key = k0 + nb * 8 + (lane & 3) * 2 + (j & 1), p = pos[j >> 1];
                            const bool seen = key < w.q.len && key - a.right <= p && (key + a.left >= p || key < a.sinks);
                            x = seen ? x : -INFINITY;
                        }
                        s[nb][j] = x;
                        top[j >> 1] = fmaxf(top[j >> 1], x);
                    }
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(&sh->v_full[vr.slot], vr.phase, cta_abort, a.status));
                const float log_vs = static_cast<float>(static_cast<int>(__float_as_uint(sh->v_scale[vr.slot][warp]) >> 23) - 127);
                float factor[2] = {1.f, 1.f}, shift[2] = {0.f, 0.f}, more[2] = {0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float mt = quad_max(top[e]), mn = fmaxf(m[e], mt);
                    if (mn == -INFINITY) continue;              // the row has seen no key
                    const float before = m[e] - mn + g[e], gn = fmaxf(before, mt - mn + log_vs);
                    l[e] *= ex2_approx(m[e] - mn);
                    factor[e] = ex2_approx(before - gn);
                    shift[e] = mn;
                    more[e] = log_vs - gn;
                    m[e] = mn;
                    g[e] = gn;
                }
                uint32_t p[2][2];
                const bool two = __any_sync(0xffffffffu, more[0] != 0.f || more[1] != 0.f);
#pragma unroll
                for (int nb = 0; nb < 2; ++nb) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float x = s[nb][j] - shift[j >> 1], weight = ex2_approx(x);
                        l[j >> 1] += weight;
                        s[nb][j] = two ? ex2_approx(x + more[j >> 1]) : weight;
                    }
                    p[nb][0] = f16x2(s[nb][0], s[nb][1]);
                    p[nb][1] = f16x2(s[nb][2], s[nb][3]);
                }
                if (__any_sync(0xffffffffu, factor[0] != 1.f || factor[1] != 1.f)) {
#pragma unroll
                    for (int d = 0; d < ND; ++d)
#pragma unroll
                        for (int j = 0; j < 4; ++j) o[d][j] *= factor[j >> 1];
                }
                if (!whole) {
                    // V in places that a row does not see: zero where no row sees it, by the element where it is NaN
                    constexpr int kChunks = KW * HD / 16 / 32;  // 16-byte chunks of a lane
                    bool nan = false;
#pragma unroll
                    for (int i = 0; i < kChunks; ++i) {
                        const int c16 = i * 32 + lane, kc = c16 / (HD / 16), ch = c16 % (HD / 16), key = k0 + kc;
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
                            bool seen[2];
#pragma unroll
                            for (int e = 0; e < 2; ++e) seen[e] = key < w.q.len && key - a.right <= pos[e] && (key + a.left >= pos[e] || key < a.sinks);
#pragma unroll
                            for (int c = 0; c < HD / 16; ++c) {
                                uint32_t v;                     // dims 16 c + 4 (lane & 3) ..: o[2 c][0], o[2 c + 1][0], o[2 c][1], o[2 c + 1][1]
                                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(sv + chunk_at(warp * KW + kc, c) + (lane & 3) * 4) : "memory");
                                if (odd_codes(v))
#pragma unroll
                                    for (int i = 0; i < 4; ++i)
                                        if ((v >> 8 * i & 0x7fu) == 0x7fu)
#pragma unroll
                                            for (int e = 0; e < 2; ++e)
                                                if (seen[e]) o[2 * c + (i & 1)][2 * e + (i >> 1)] = __uint_as_float(0x7fffffffu);
                            }
                        }
                        __syncwarp();
#pragma unroll 1
                        for (int i = 0; i < KW * HD / 4 / 32; ++i) {
                            const int c4 = i * 32 + lane, kc = c4 / (HD / 4), dd = c4 % (HD / 4);
                            const uint32_t ad = sv + chunk_at(warp * KW + kc, dd >> 2) + (dd & 3) * 4;
                            uint32_t v;
                            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(ad) : "memory");
#pragma unroll
                            for (int b = 0; b < 4; ++b)
                                if ((v >> 8 * b & 0x7fu) == 0x7fu) v &= ~(0xffu << 8 * b);
                            asm volatile("st.shared.b32 [%0], %1;" ::"r"(ad), "r"(v) : "memory");
                        }
                        __syncwarp();
                    }
                    __syncwarp();
                }
                const uint32_t pa[4] = {p[0][0], p[0][1], p[1][0], p[1][1]};
                const int key_v = warp * KW + (lane & 15);
#pragma unroll
                for (int c = 0; c < HD / 16; c += 2) {
                    uint32_t b[4];                              // keys 0 .. 7 and 8 .. 15 of dims 16 c .., then of the next 16
                    ldsm4_t(sv + chunk_at(key_v, c + (lane >> 4)), b);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {               // a word: two keys of an even dim, then of the odd one
                        const uint32_t x = __byte_perm(b[2 * h], 0, 0x3120), y = __byte_perm(b[2 * h + 1], 0, 0x3120);
                        mma(o[2 * (c + h)], pa, low_codes(x), low_codes(y));
                        mma(o[2 * (c + h) + 1], pa, high_codes(x), high_codes(y));
                    }
                }
                if (!whole) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // this warp's writes to V before the next copy into it
            }
            if (!k_read) {                                      // nothing to multiply: in step with the loader all the same
                k_done();
                mbar_wait_bounded(&sh->v_full[vr.slot], vr.phase, cta_abort, a.status);
            }
            if (t + 1 == w.t1) break;                 // the item's last V tile stays: its place is where the warps meet
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->v_empty[vr.slot]);
            vr.next();
        }

        // ---- the warps that share the rows meet ----
#pragma unroll
        for (int e = 0; e < 2; ++e) l[e] = quad_sum(l[e]);
        {
            if ((lane & 3) == 0) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    sh->ml[warp][(lane >> 2) + 8 * e][0] = m[e];
                    sh->ml[warp][(lane >> 2) + 8 * e][1] = l[e];
                }
            }
            mma_warps_barrier();                                // all have read the last V tile
            const bool upper = rows > 8;                        // rows from 8 on
            float* merge = reinterpret_cast<float*>(smem + (kS + vr.slot) * kT);
            static_assert(2 * 8 * HD * 4 <= kT, "two warps' outputs of eight rows fit a tile");
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float M = -INFINITY, L = 0.f;
#pragma unroll
                for (int i = 0; i < kMmaWarps; ++i) M = fmaxf(M, sh->ml[i][(lane >> 2) + 8 * e][0]);
#pragma unroll
                for (int i = 0; i < kMmaWarps; ++i) {
                    const float* x = sh->ml[i][(lane >> 2) + 8 * e];
                    L += paged_weight(x[0], M) * x[1];
                }
                const float f = g[e] == -INFINITY ? 0.f : ex2_approx(m[e] - M + g[e]);   // from here on in units of 2^M, without scales
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    o[d][2 * e] *= f;
                    o[d][2 * e + 1] *= f;
                }
                m[e] = M;
                l[e] = L;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (e == 1 && !upper) break;
#pragma unroll
                for (int half = kMmaWarps / 2; half >= 1; half >>= 1) {   // the upper half of the warps hands over to the lower
                    float* mb = merge + (warp % half) * ND * 2 * 32 + lane;
                    if (warp >= half && warp < 2 * half) {
#pragma unroll
                        for (int d = 0; d < ND; ++d)
#pragma unroll
                            for (int j = 0; j < 2; ++j) mb[(d * 2 + j) * 32] = o[d][2 * e + j];
                    }
                    mma_warps_barrier();
                    if (warp < half) {
#pragma unroll
                        for (int d = 0; d < ND; ++d)
#pragma unroll
                            for (int j = 0; j < 2; ++j) o[d][2 * e + j] += mb[(d * 2 + j) * 32];
                    }
                    mma_warps_barrier();
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->v_empty[vr.slot]);
            vr.next();
        }

        // ---- results, or this CTA's part of them ----
        const size_t part = paged_part(a, blockIdx.x, w.t0 == 0);
        if (warp == 0) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = r_lo + 8 * e;
                if (r >= rows) continue;
                if (final) {
                    const int idx = w.rt * kRows + r, head = w.head * a.G + idx - a.by_group(idx) * a.G;
                    const float inv = l[e] == 0.f ? 0.f : 1.0f / l[e];
                    __nv_bfloat16* op = a.out + at[e] * a.out_stride + head * HD + (lane & 3) * 4;
#pragma unroll
                    for (int c = 0; c < HD / 16; ++c)
                        *reinterpret_cast<uint2*>(op + c * 16) = make_uint2(paged_bf16x2(o[2 * c][2 * e] * inv, o[2 * c + 1][2 * e] * inv),
                                                                            paged_bf16x2(o[2 * c][2 * e + 1] * inv, o[2 * c + 1][2 * e + 1] * inv));
                    if (a.lse && (lane & 3) == 0) a.lse[at[e] * a.H + head] = paged_lse(m[e], l[e]);
                } else {
                    float* op = a.part_o + (part + r) * HD + (lane & 3) * 4;
#pragma unroll
                    for (int c = 0; c < HD / 16; ++c)
                        *reinterpret_cast<float4*>(op + c * 16) = make_float4(o[2 * c][2 * e], o[2 * c + 1][2 * e], o[2 * c][2 * e + 1], o[2 * c + 1][2 * e + 1]);
                    if ((lane & 3) == 0) *reinterpret_cast<float2*>(a.part_ml + (part + r) * 2) = make_float2(m[e], l[e]);
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
                        if (warp + k * kMmaWarps < rows) sum.write(a, k, w.q.row0, w.head, w.rt * kRows + warp + k * kMmaWarps);
                };
                if (rows <= kMmaWarps) add_up(PagedSum<HD, 1>{});
                else if (rows <= 2 * kMmaWarps) add_up(PagedSum<HD, 2>{});
                else add_up(PagedSum<HD, 4>{});
                mma_warps_barrier();                             // sh->last has been read by all
            }
        }
    } while (w.next());
}

template <int HD>
cudaError_t launch(PagedAttnArgs a, const CUtensorMap& tmap, int sms, cudaStream_t st) {
    static std::atomic<unsigned long long> attr_done{0};
    cudaError_t e = set_smem_limit_once(attr_done, paged_e4m3_attention_kernel<HD>, static_cast<int>(kSmem<HD>));
    if (e != cudaSuccess) return e;
    a.tile_rows = kRows;
    a.by_rows = PagedDiv::by(kRows);
    a.part_rows = kRows;
    a.at_once = 2 * sms;
    a.by_once = PagedDiv::by(a.at_once);
    // four waves of CTAs, as for a pool of bf16; no more than the table's width leaves work for
    const long long tiles = (static_cast<long long>(a.table_stride) << a.page_shift) / kKT + 1 + kItem,
                    most = (static_cast<long long>(a.max_rows) * a.G / kRows + a.n_seqs) * a.KV * tiles / kMinUnits + 1;
    static_assert(kPagedMaxCtas * kRows <= kPagedPartRows, "parts");
    const int grid = static_cast<int>(most < kPagedWaves * a.at_once ? most : kPagedWaves * a.at_once);
    return launch_kernel(paged_e4m3_attention_kernel<HD>, dim3(grid), dim3(kThreads), kSmem<HD>, st, tmap, a);
}

}  // namespace

int paged_e4m3_attention_kernel_of(int n_seqs, int max_rows, int, int group, int kv_heads, long long longest, long long) {
    const long long all = static_cast<long long>(max_rows) * group, tiles = longest / kKT + 1;
    return (static_cast<double>(all / kRows) + n_seqs) * kv_heads * static_cast<double>(tiles + kItem) < 2147483648.0 - 65536 ? 0 : -1;
}

cudaError_t launch_paged_e4m3_attention(PagedAttnArgs a, const CUtensorMap& map, int hd, int, int sms, cudaStream_t st) {
    if (sms < 1 || 2 * sms * 128 > kPagedPartRows || kPagedWaves * 2 * sms > kPagedMaxCtas) return cudaErrorInvalidValue;   // the workspace's size
    a.by_group = PagedDiv::by(a.G);
    return hd == 128 ? launch<128>(a, map, sms, st) : launch<64>(a, map, sms, st);
}

}  // namespace odb
