// Attention of the rows of each request over its pages of the K/V pool: few packed rows (query rows x heads of a group), or little work.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = 2^(s_j - m),  s_j = log2(e) * scale * q.k_j,  lse = ln 2 * (m + log2 sum_j p_j)
//
// over the visible keys j < len, j <= pos + right, (j >= pos - left or j < sinks).  One pass over the keys with the running
// maximum m and sum in fp32; P is rounded to bf16 for the second product (the sum keeps the unrounded values: the rounding's
// relative error of up to 2^-8 per key is independent from key to key and ends below the output's own rounding).
//
// Work: see paged.cuh; items of 16 packed rows, key tiles of 64 positions.  One warp loads (TMA, a box per page of a tile, 128-byte
// swizzle, rings of K and of V tiles with a full and an empty barrier each), four warps multiply (mma.sync m16n8k16), 16 keys of a
// tile each with a running maximum, sum and output of their own, which meet in the last V tile's place when the item ends.  An item
// that several CTAs share leaves unnormalised parts in the workspace; the CTA that arrives last adds them up in the order of the
// CTAs, whoever it is: the same bits every time.
//
// Bound by HBM where there is work for all SMs (a pool read once; the products of 16 rows take a third of a tile's time): one token
// of 48 requests, 905 MB, 152 us = 6.0 TB/s, of two of 131072 keys, 1.02 GB, 167 us = 6.1 TB/s; the rest is the start (a microsecond to
// find the share, two until the first tile is there), the parts and the slowest SMs' tail.  Small calls are bound by latency: one token
// of 577 keys 9.2 us, 16 requests with a window of 4096 keys of 64 (67 MB) 21 us.
//
// Rows of V behind the last visible key are whatever the page held before: their P is zero, but zero times an infinity or NaN
// there is not, so they are set to zero in shared memory first.  A key that some rows of the tile see and others do not is
// treated by the element: V's values that are not finite are taken out of the tile and given to the rows that see them.
#include "paged.cuh"

namespace odb {

namespace {

constexpr int kKT = 64;                    // keys per tile
constexpr int kItem = 1;                    // key tiles that an item costs beside its own
constexpr int kMinUnits = 2, kFullUnits = 24;   // units of a CTA, at least; where all places on the SMs have work
constexpr int kRows = 16;                   // packed rows of an item
constexpr int kSmallUnits = 1024;           // up to here few rows' kernel for any number of rows
constexpr int kManyRows = 1024;             // packed rows a request, on average, from which two Q tiles are right whatever the longest
constexpr int kMmaWarps = 4;
constexpr int kThreads = 32 * (kMmaWarps + 1);
template <int HD> constexpr int kKSlots = HD == 128 ? 3 : 7;                // K tiles on the way or in use
template <int HD> constexpr int kVSlots = HD == 128 ? 4 : 7;
template <int HD> constexpr uint32_t kTileBytes = kKT * HD * 2;            // K or V of a tile
template <int HD> constexpr uint32_t kSmem = (kKSlots<HD> + kVSlots<HD>) * kTileBytes<HD> + 1024;
static_assert(2 * (kSmem<128> + 1024) <= 228 * 1024 && 2 * (kSmem<64> + 1024) <= 228 * 1024, "two CTAs share an SM");

struct Barriers {
    uint64_t k_full[8], v_full[8], k_empty[8], v_empty[8];
    float ml[kMmaWarps][16][2];
    int last, abort;
};
static_assert(sizeof(Barriers) <= 1024, "the barriers end inside the allocation");

// a box of rows of the pool: all head dims of a row, 64 at a time
__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* tmap, uint64_t* bar, int row) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_u32(bar)), "r"(0), "r"(row), "r"(0)
        : "memory");
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
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
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
__device__ __forceinline__ bool odd_bf16(uint32_t two) {   // one of the two is an infinity or NaN
    return (two & 0x7f80u) == 0x7f80u || (two & 0x7f800000u) == 0x7f800000u;
}

template <int HD>
__global__ void __launch_bounds__(kThreads, 2) paged_attention_kernel(const __grid_constant__ CUtensorMap tm, const PagedAttnArgs a) {
    constexpr int KW = kKT / kMmaWarps;                         // keys of a warp
    constexpr int kAtoms = HD / 64, NS = KW / 8, ND = HD / 8;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* smem = smem_raw;
    constexpr int KS = kKSlots<HD>, VS = kVSlots<HD>;
    const uint32_t k_tiles = smem_u32(smem), v_tiles = k_tiles + KS * kTileBytes<HD>;
    Barriers* sh = reinterpret_cast<Barriers*>(smem + (KS + VS) * kTileBytes<HD>);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    volatile int* cta_abort = &sh->abort;

    if ((smem_u32(smem_raw) & 1023u) != 0) {                    // the swizzled tiles need 1024-byte alignment
        if (tid == 0) atomicExch(a.status, ODB_ERR_CUDA);
        pdl_wait();
        return;
    }
    if (tid == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm)) : "memory");
        for (int i = 0; i < KS; ++i) {
            mbar_init(&sh->k_full[i], 1);
            mbar_init(&sh->k_empty[i], kMmaWarps);
        }
        for (int i = 0; i < VS; ++i) {
            mbar_init(&sh->v_full[i], 1);
            mbar_init(&sh->v_empty[i], kMmaWarps);
        }
        sh->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_launch_dependents();
    pdl_wait();
    // the ring's memory holds the sums until the start is found
    static_assert(sizeof(PagedScratch) <= kSmem<64> - 1024, "the scratch fits the rings");
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
        __device__ __forceinline__ void next(int slots) {
            if (++slot == slots) { slot = 0; phase ^= 1u; }
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
                const uint32_t bytes = static_cast<uint32_t>(boxes) * box * HD * 2;
                auto load = [&](Ring& r, int slots, uint64_t* empty, uint64_t* full, uint32_t tiles, int base) {
                    if (issued >= slots) ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(&empty[r.slot], r.phase ^ 1u, cta_abort, a.status));
                    if (!ok) return;
                    const uint32_t slot = __shfl_sync(0xffffffffu, r.slot, 0), to = tiles + slot * kTileBytes<HD>;
                    if (paged_elect()) mbar_expect_tx(&full[slot], bytes);
                    __syncwarp();
                    for (int c = 0; c < boxes; ++c) {
                        const int row = pages.row<true, true>(a, w.q, w.seq, w.head, k0 + (c << box_shift), base);
                        if (paged_elect()) tma_rows(to + c * box * HD * 2, &tm, &full[slot], row);
                        __syncwarp();
                    }
                    r.next(slots);
                };
                load(kr, KS, sh->k_empty, sh->k_full, k_tiles, a.k_row0);
                load(vr, VS, sh->v_empty, sh->v_full, v_tiles, a.v_row0);
                if (!ok) break;
                ++issued;
            }
        } while (ok && w.next());
        if (!ok) {   // copies in flight land before the memory goes away
            const long long t0 = clock64();
            auto land = [&](uint64_t* full, int slots) {
                for (int j = max(0, issued + 1 - slots); j <= issued; ++j)   // the last one may have a K tile only
                    while (!mbar_try_wait_parity(&full[j % slots], static_cast<uint32_t>(j / slots) & 1u) && clock64() - t0 < kWaitLimitCycles / 8) {
                    }
            };
            land(sh->k_full, KS);
            land(sh->v_full, VS);
        }
        return;
    }

    // ================= the products =================
    const int r_lo = lane >> 2;                     // this thread's rows of the tile: r_lo and r_lo + 8
    do {
        const int rows = min(kRows, w.q.n * a.G - w.rt * kRows);  // packed rows of this item
        uint32_t qf[HD / 16][4];
        int pos[2];
        size_t at[2];                                           // row of q, out and lse, in heads
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = min(r_lo + 8 * e, rows - 1), idx = w.rt * kRows + r, i = a.by_group(idx);   // rows behind the last repeat it
            pos[e] = w.q.first + i;
            at[e] = static_cast<size_t>(w.q.row0 + i);
            const __nv_bfloat16* qp = a.q + at[e] * a.q_stride + (w.head * a.G + idx - i * a.G) * HD + (lane & 3) * 2;
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) {
                qf[kk][e] = *reinterpret_cast<const uint32_t*>(qp + kk * 16);
                qf[kk][2 + e] = *reinterpret_cast<const uint32_t*>(qp + kk * 16 + 8);
            }
        }
        const bool final = w.whole();
        const int c0 = final ? 0 : w.first_cta(), c1 = final ? 0 : w.last_cta();   // while K is on its way
        const int idx_last = w.rt * kRows + rows - 1;
        const int p_min = w.q.first + a.by_group(w.rt * kRows), p_max = w.q.first + a.by_group(idx_last);
        // keys from all_lo on and below all_hi are seen by all rows of the item
        const int all_hi = static_cast<int>(max(0ll, min(static_cast<long long>(w.q.len), static_cast<long long>(p_min) + a.right + 1)));
        const int all_lo = static_cast<int>(max(-1ll, static_cast<long long>(p_max) - a.left));
        float o[ND][4];
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
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
                kr.next(KS);
                k_read = true;
            };
            const uint32_t sk = k_tiles + kr.slot * kTileBytes<HD>, sv = v_tiles + vr.slot * kTileBytes<HD>;
            // key c of the tile, atom h: box (c >> box_shift), then [atom][row of the box][128 bytes]
            auto key_at = [&](int c, int h) -> uint32_t {
                return static_cast<uint32_t>((((c >> box_shift) * kAtoms + h) << box_shift) + (c & (box - 1))) * 128u;
            };
            const bool any_key = k0 < w.k.hi && (k0 + KW > w.k.lo || k0 < a.sinks);   // some row of the item sees some key
            if (ok && any_key) {
                float s[NS][4];
#pragma unroll
                for (int nb = 0; nb < NS; ++nb) s[nb][0] = s[nb][1] = s[nb][2] = s[nb][3] = 0.f;
                const uint32_t sw = static_cast<uint32_t>(lane & 7) << 4;
#pragma unroll
                for (int nb = 0; nb < NS; nb += 2) {
                    const int c = warp * KW + nb * 8 + (lane & 7) + ((lane >> 4) << 3);
                    float odd[2][4] = {};                       // every other step in sums of its own: half as long a chain of products
#pragma unroll
                    for (int kk = 0; kk < HD / 16; ++kk) {
                        uint32_t b[4];
                        ldsm4(sk + key_at(c, kk >> 2) + (((kk & 3) * 32 + ((lane >> 3) & 1) * 16) ^ sw), b);
                        if (NS == 2 && (kk & 1)) {
                            mma(odd[0], qf[kk], b[0], b[1]);
                            mma(odd[1], qf[kk], b[2], b[3]);
                        } else {
                            mma(s[nb], qf[kk], b[0], b[1]);
                            mma(s[nb + 1], qf[kk], b[2], b[3]);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[nb][j] += odd[0][j];
                        s[nb + 1][j] += odd[1][j];
                    }
                }
                k_done();
                const bool whole = k0 + KW <= all_hi && (k0 >= all_lo || k0 + KW <= a.sinks);
                float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int nb = 0; nb < NS; ++nb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float x = s[nb][j] * a.scale_log2;
                        if (!whole) {
                            const int key = k0 + nb * 8 + (lane & 3) * 2 + (j & 1), p = pos[j >> 1];
                            const bool seen = key < w.q.len && key - a.right <= p && (key + a.left >= p || key < a.sinks);
                            x = seen ? x : -INFINITY;
                        }
                        s[nb][j] = x;
                        top[j >> 1] = fmaxf(top[j >> 1], x);
                    }
                float factor[2], shift[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float mn = fmaxf(m[e], quad_max(top[e]));
                    shift[e] = mn == -INFINITY ? 0.f : mn;
                    factor[e] = paged_weight(m[e], shift[e]);
                    m[e] = mn;
                }
                float sum[2] = {0.f, 0.f};
                uint32_t p[NS][2];
#pragma unroll
                for (int nb = 0; nb < NS; ++nb) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[nb][j] = ex2_approx(s[nb][j] - shift[j >> 1]);
                        sum[j >> 1] += s[nb][j];
                    }
                    p[nb][0] = paged_bf16x2(s[nb][0], s[nb][1]);
                    p[nb][1] = paged_bf16x2(s[nb][2], s[nb][3]);
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) l[e] = l[e] * factor[e] + sum[e];
                if (__any_sync(0xffffffffu, factor[0] != 1.f || factor[1] != 1.f)) {
#pragma unroll
                    for (int d = 0; d < ND; ++d)
#pragma unroll
                        for (int j = 0; j < 4; ++j) o[d][j] *= factor[j >> 1];
                }
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(&sh->v_full[vr.slot], vr.phase, cta_abort, a.status));
                if (!whole) {
                    // V in places that a row does not see: zero where no row sees it, by the element where it is not finite
                    constexpr int kChunks = KW * HD / 8 / 32;   // 16-byte chunks of a lane
                    bool odd = false;
#pragma unroll 4
                    for (int i = 0; i < kChunks; ++i) {
                        const int c16 = i * 32 + lane, c = warp * KW + c16 / (HD / 8), ch = c16 % (HD / 8);
                        const int key = k0 + c16 / (HD / 8);
                        const uint32_t ad = sv + key_at(c, ch >> 3) + (((ch & 7) ^ (c & 7)) << 4);
                        uint32_t v[4];
                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(ad) : "memory");
                        const bool out = key >= w.k.hi || (key < w.k.lo && key >= a.sinks);
                        if (out)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(ad), "r"(0) : "memory");
                        else
                            odd = odd || odd_bf16(v[0]) || odd_bf16(v[1]) || odd_bf16(v[2]) || odd_bf16(v[3]);
                    }
                    odd = __any_sync(0xffffffffu, odd);
                    __syncwarp();                  // all have looked
                    if (odd) {
#pragma unroll 1
                        for (int kc = 0; kc < KW; ++kc) {       // rare: an infinity or NaN in V, seen by some of the rows
                            const int key = k0 + kc, c = warp * KW + kc;
                            float pr[2];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {       // P of this thread's rows and this key, from the lane that has it
                                float x = 0.f;
#pragma unroll
                                for (int nb = 0; nb < NS; ++nb)
#pragma unroll
                                    for (int j = 0; j < 2; ++j)
                                        if (nb == kc >> 3 && j == (kc & 1)) x = s[nb][e * 2 + j];
                                pr[e] = __shfl_sync(0xffffffffu, x, (lane & ~3) | ((kc & 7) >> 1));
                            }
#pragma unroll
                            for (int d = 0; d < ND; ++d) {
                                const int ch = d;
                                const uint32_t ad = sv + key_at(c, ch >> 3) + (((ch & 7) ^ (c & 7)) << 4) + (lane & 3) * 4;
                                uint32_t v;
                                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(ad) : "memory");
                                if (odd_bf16(v)) {
                                    const float v0 = __uint_as_float(v << 16), v1 = __uint_as_float(v & 0xffff0000u);
#pragma unroll
                                    for (int e = 0; e < 2; ++e) {
                                        const bool seen = key < w.q.len && key - a.right <= pos[e] && (key + a.left >= pos[e] || key < a.sinks);
                                        if (seen && !isfinite(v0)) o[d][e * 2] += pr[e] * v0;
                                        if (seen && !isfinite(v1)) o[d][e * 2 + 1] += pr[e] * v1;
                                    }
                                }
                            }
                        }
                        __syncwarp();
#pragma unroll 1
                        for (int i = 0; i < KW * HD / 2 / 32; ++i) {
                            const int c2 = i * 32 + lane, kc = c2 / (HD / 2), dd = c2 % (HD / 2), c = warp * KW + kc;
                            const uint32_t ad = sv + key_at(c, dd >> 5) + ((((dd >> 2) & 7) ^ (c & 7)) << 4) + (dd & 3) * 4;
                            uint32_t v;
                            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(ad) : "memory");
                            if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
                            if ((v & 0x7f800000u) == 0x7f800000u) v &= 0xffffu;
                            asm volatile("st.shared.b32 [%0], %1;" ::"r"(ad), "r"(v) : "memory");
                        }
                        __syncwarp();
                    }
                    __syncwarp();
                }
#pragma unroll
                for (int kb = 0; kb < KW / 16; ++kb) {
                    const uint32_t pa[4] = {p[2 * kb][0], p[2 * kb][1], p[2 * kb + 1][0], p[2 * kb + 1][1]};
                    const int c = warp * KW + kb * 16 + (lane & 15);
#pragma unroll
                    for (int d = 0; d < ND; d += 2) {
                        uint32_t b[4];
                        ldsm4_t(sv + key_at(c, d >> 3) + ((((d & 7) + (lane >> 4)) * 16) ^ sw), b);
                        mma(o[d], pa, b[0], b[1]);
                        mma(o[d + 1], pa, b[2], b[3]);
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
            vr.next(VS);
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
            float* merge = reinterpret_cast<float*>(smem + (KS + vr.slot) * kTileBytes<HD>);
            static_assert(2 * 16 * HD * 4 <= kTileBytes<HD>, "two warps' outputs fit a tile");
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float M = -INFINITY, L = 0.f;
#pragma unroll
                for (int g = 0; g < kMmaWarps; ++g) M = fmaxf(M, sh->ml[g][(lane >> 2) + 8 * e][0]);
#pragma unroll
                for (int g = 0; g < kMmaWarps; ++g) {
                    const float* x = sh->ml[g][(lane >> 2) + 8 * e];
                    L += paged_weight(x[0], M) * x[1];
                }
                const float f = paged_weight(m[e], M);
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    o[d][2 * e] *= f;
                    o[d][2 * e + 1] *= f;
                }
                m[e] = M;
                l[e] = L;
            }
#pragma unroll
            for (int half = kMmaWarps / 2; half >= 1; half >>= 1) {   // the upper half of the warps hands over to the lower
                float* mb = merge + (warp % half) * ND * 4 * 32 + lane;
                if (warp >= half && warp < 2 * half) {
#pragma unroll
                    for (int d = 0; d < ND; ++d)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (j < 2 || upper) mb[(d * 4 + j) * 32] = o[d][j];
                }
                mma_warps_barrier();
                if (warp < half) {
#pragma unroll
                    for (int d = 0; d < ND; ++d)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (j < 2 || upper) o[d][j] += mb[(d * 4 + j) * 32];
                }
                mma_warps_barrier();
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->v_empty[vr.slot]);
            vr.next(VS);
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
                    __nv_bfloat16* op = a.out + at[e] * a.out_stride + head * HD + (lane & 3) * 2;
#pragma unroll
                    for (int d = 0; d < ND; ++d) *reinterpret_cast<uint32_t*>(op + d * 8) = paged_bf16x2(o[d][2 * e] * inv, o[d][2 * e + 1] * inv);
                    if (a.lse && (lane & 3) == 0) a.lse[at[e] * a.H + head] = paged_lse(m[e], l[e]);
                } else {
                    float* op = a.part_o + (part + r) * HD + (lane & 3) * 2;
#pragma unroll
                    for (int d = 0; d < ND; ++d) *reinterpret_cast<float2*>(op + d * 8) = make_float2(o[d][2 * e], o[d][2 * e + 1]);
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
    cudaError_t e = set_smem_limit_once(attr_done, paged_attention_kernel<HD>, static_cast<int>(kSmem<HD>));
    if (e != cudaSuccess) return e;
    a.tile_rows = kRows;
    a.by_rows = PagedDiv::by(kRows);
    a.part_rows = kRows;
    a.at_once = 2 * sms;
    a.by_once = PagedDiv::by(a.at_once);
    // Under a full memory system some SMs run a third slower than others, and so does the second CTA of an SM: of one share for each
    // place the last ended a third behind the mean.  So four waves of CTAs, taken by whichever place is free, of shares that grow
    // smaller to the end.  No more CTAs than the table's width leaves work for.
    const long long tiles = (static_cast<long long>(a.table_stride) << a.page_shift) / kKT + 1 + kItem,
                    most = (static_cast<long long>(a.max_rows) * a.G / kRows + a.n_seqs) * a.KV * tiles / kMinUnits + 1;
    static_assert(kPagedMaxCtas * kRows <= kPagedPartRows, "parts");
    const int grid = static_cast<int>(most < kPagedWaves * a.at_once ? most : kPagedWaves * a.at_once);
    return launch_kernel(paged_attention_kernel<HD>, dim3(grid), dim3(kThreads), kSmem<HD>, st, tmap, a);
}

}  // namespace

size_t paged_part_bytes(int hd) { return static_cast<size_t>(kPagedMaxParts) * kPagedPartRows * (hd + 2) * sizeof(float); }

// Which kernel: by the work, then by the packed rows of the longest request.  Up to kSmallUnits key tiles of items of 16 packed rows (an
// item's start counted as one), as far as the table's width bounds them, mma.sync without a second launch is faster,
// however many rows: us, it / tensor cores with one Q tile, head dim 128: 192 units 12.6 / 16.0, 544 13.6 / 16.2, 1024 15.8 / 18.3, 1088
// 17.2 / 17.0, 1536 18.9 / 19.2, 2112 22 / 18, 4352 31 / 18; head dim 64: 192 10.7 / 12.7, 528 12.1 / 14.2, 1088 14.3 / 13.9, 2112 19 / 15.
// Above, 8 K/V heads of 128, one Q tile / two behind it:
//   4 packed rows, 1 request of 577 keys 9.1 / 17 / 20, 16 of up to 600 15 / 19 / 26, 16 of up to 4096 46 / 47 / 68, 2 of 131072
//   168 / 165 / 235;   16 rows, 1 of 577 11 / 19 / -, 16 of up to 4096 49 / 48 / 67
//   32 packed rows, 16 requests of up to 4096 keys 77 / 47 / 62, of up to 600 25 / 19 / 23
//   128 packed rows, 16 requests of up to 4096 - / 52 / 62;   192: - / 75 / 65;   256: - / 82 / 70;   a causal prompt of 4096 rows - / 162 / 142
// Two Q tiles take requests that are alike, the longest up to three times the mean: beside a prompt of 2048 rows 47 single tokens of up
// to 8192 keys leave the second one empty, and two CTAs on an SM hide more: - / 169 / 220 (head dim 64: 127 / 173); 512 rows and 8 tokens
// 50 / 63; 4096 rows and 8 tokens 180 / 172.
// Where the longest is not known (max_new 0) the mean stands for it, and a mean says nothing of the mixture: of 1024 packed rows and
// more on average two Q tiles are right for alike and unlike ones (4 of 1024 rows 127 / 113, 4096 rows and 15 tokens 198 / 197, 2 of
// 2048 and 16 tokens, 916, 127 / 129), of fewer they gain a tenth where requests are alike and lose a third where they are not (16 of
// 128 rows 95 / 83; 2048 rows and 47 tokens 177 / 237, 512 and 15 61 / 75; head dim 64 the same).
int paged_attention_kernel_of(int n_seqs, int max_rows, int max_new, int group, int kv_heads, long long longest, long long out_stride) {
    const long long all = static_cast<long long>(max_rows) * group, mean = (max_rows + n_seqs - 1ll) / n_seqs * group,
                    mine = max_new > 0 ? static_cast<long long>(max_new) * group : mean, tiles = longest / kKT + 1;
    // units of all items together and what is added to them on the way, with rows that follow one another
    auto fits = [&](int tile_rows, int item) {
        return (static_cast<double>(all / tile_rows) + n_seqs) * kv_heads * static_cast<double>(tiles + item) < 2147483648.0 - 65536;
    };
    const bool few_fit = fits(kRows, kItem);
    // the many rows' kernel keeps a row's place within its Q tile in 32 bits, in units of 8 elements
    if (group <= kPagedTcMaxGroup && out_stride <= 1ll << 27) {
        const int tile = kPagedTcMaxGroup / group * group;
        const double units = static_cast<double>((all + (kRows - 1ll) * n_seqs) / kRows) * kv_heads * static_cast<double>(tiles + kItem);
        if ((mine > kRows && units > kSmallUnits) || !few_fit) {
            const bool alike = max_new > 0 ? static_cast<long long>(max_new) * n_seqs <= 3ll * max_rows : n_seqs == 1 || mean >= kManyRows;
            const int q_tiles = mine > 128 && alike ? 2 : 1;
            if (fits(q_tiles * tile, kPagedTcItem)) return q_tiles;
            return fits(2 * tile, kPagedTcItem) ? 2 : -1;
        }
    }
    return few_fit ? 0 : -1;
}

cudaError_t launch_paged_attention(PagedAttnArgs a, const PagedMaps& maps, int hd, int q_tiles, int sms, cudaStream_t st) {
    if (sms < 1 || 2 * sms * 128 > kPagedPartRows || kPagedWaves * 2 * sms > kPagedMaxCtas) return cudaErrorInvalidValue;   // the workspace's size
    a.by_group = PagedDiv::by(a.G);
    if (q_tiles > 0) return launch_paged_attention_tc(a, maps, hd, q_tiles, sms, st);
    return hd == 128 ? launch<128>(a, maps.rows, sms, st) : launch<64>(a, maps.rows, sms, st);
}

}  // namespace odb
