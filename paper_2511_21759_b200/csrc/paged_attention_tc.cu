// Attention of the rows of each request over its pages: many packed rows, on the tcgen05 tensor cores (formulas, masks and the
// division of the work: paged_attention.cu, paged.cuh).
//
// An item is QT Q tiles of up to 128 packed rows (floor(128 / group) query rows x the heads of a group) of one K/V head; a CTA
// walks its share of the line of key tiles of 64 positions, item after item.  QT = 1: two CTAs on an SM; QT = 2 (requests of more
// than 128 packed rows): one CTA whose two Q tiles share every K and V tile, which halves what comes from L2.
//
// Per key tile and Q tile: S = Q K^T is a 128 x 64 x HD group of MMAs into TMEM; thread r of the Q tile's four softmax warps owns
// TMEM lane r = packed row r, so a row's maximum and sum never leave the thread.  The row's shift M is an integer in the log2
// domain and moves only when a tile's maximum exceeds it by more than 4; O (in TMEM) and the sum are then multiplied by an exact
// power of two.  P = exp2(S - M) < 16, rounded to bf16 (the sum keeps the unrounded values), takes S's place in TMEM as the A
// operand of O += P V, with V taken MN-major from its [key][dim] tile.  One thread loads (TMA boxes of a page's rows x 64 values,
// which land in the canonical swizzled layout whatever the page size), one issues the MMAs, all meet through mbarriers with
// bounded waits; on expiry ODB_ERR_TIMEOUT is recorded and every role runs through its remaining barriers and ends.
//
// Rows of V that no row of the item sees are set to zero in shared memory; values of V that are not finite at keys that only some
// rows see are taken out of the tile and added to O of the rows that see them, one TMEM column at a time.
#include "attention_tc.cuh"
#include "paged.cuh"

namespace odb {

namespace {

constexpr int kTQ = 128;   // packed rows of a Q tile (MMA M)
constexpr int kKT = 64;    // keys of a tile
template <int QT> constexpr int kThreads = 32 * (4 * QT + 2);
template <int HD> constexpr uint32_t kQBytes = kTQ * HD * 2;
template <int HD> constexpr uint32_t kTileBytes = kKT * HD * 2;
template <int HD, int QT> constexpr int kSlots = HD == 128 ? (QT == 1 ? 5 : 10) : (QT == 1 ? 10 : 16);
template <int HD, int QT> constexpr uint32_t kSmem = QT * kQBytes<HD> + kSlots<HD, QT> * kTileBytes<HD> + 512;
template <int HD> constexpr int kBufs = HD == 128 ? 2 : 3;   // S / P buffers of a Q tile: 256 columns, of which O takes HD
constexpr uint32_t kCols = 256;
constexpr uint32_t kPatch = 4096;                            // per softmax warp, in the Q tile: 32 rows x 128 bytes of output

struct alignas(8) Shared {
    uint64_t q_full;             // the item's Q tiles landed                     (loader -> MMA)
    uint64_t full[16];           // K or V tile landed in the ring's slot         (loader -> MMA, softmax)
    uint64_t empty[16];          // the MMAs have read the slot                   (MMA -> loader)
    uint64_t s_full[2][3];       // S of Q tile g into buffer i has completed     (MMA -> softmax)
    uint64_t p_full[2][3];       // P has taken its place                         (softmax -> MMA, 4 arrivals)
    uint64_t pv_done[2][2];      // O += P V of an even / odd tile has completed  (MMA -> MMA, softmax)
    uint64_t o_full[2];          // the item's last one has                       (MMA -> softmax)
    uint64_t item_done;          // O and the Q tiles may be overwritten          (softmax -> loader, MMA, 4 QT arrivals)
    uint32_t tmem_base;
    int abort, last, keep_o[2];
};
static_assert(sizeof(Shared) <= 512, "the barriers end inside the allocation");

// whether any softmax thread of the CTA says so
template <int QT>
__device__ __forceinline__ bool softmax_any(bool x) {
    int r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %1, 0;\n\t"
        "barrier.cta.red.or.pred q, 1, %2, p;\n\t"
        "selp.b32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"(static_cast<int>(x)), "r"(128 * QT)
        : "memory");
    return r != 0;
}
// One lane of a converged warp.  The MMA and TMA instructions take their operands from uniform registers: behind elect, with
// operands that every lane has, they follow one another without a detour (behind `lane == 0` an MMA took 110 cycles to issue, and
// one of 128 x 64 x 16 runs for 32).
__device__ __forceinline__ bool elect_one() {
    uint32_t x;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(x));
    return x != 0;
}
template <int QT>
__device__ __forceinline__ void softmax_barrier() { asm volatile("bar.sync 1, %0;" ::"r"(128 * QT) : "memory"); }

__device__ __forceinline__ void tma_box_3d(uint32_t dst, const CUtensorMap* tmap, uint64_t* bar, int c0, int c1, int c2) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}
// one TMEM column of a warp's lanes
__device__ __forceinline__ uint32_t tmem_ld1(uint32_t taddr) {
    uint32_t v;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n\ttcgen05.wait::ld.sync.aligned;" : "=r"(v) : "r"(taddr) : "memory");
    return v;
}
__device__ __forceinline__ void tmem_st1(uint32_t taddr, uint32_t v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};\n\ttcgen05.wait::st.sync.aligned;" ::"r"(taddr), "r"(v) : "memory");
}
__device__ __forceinline__ bool not_finite(uint32_t bf) { return (bf & 0x7f80u) == 0x7f80u; }

template <int HD, int QT>
__global__ void __launch_bounds__(kThreads<QT>, QT == 1 ? 2 : 1)
    paged_attention_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_kv, const PagedAttnArgs a) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    constexpr int kRing = kSlots<HD, QT>, kB = kBufs<HD>, kFirst = kB - 1, kAtoms = HD / 64;
    constexpr uint32_t kT = kTileBytes<HD>;
    constexpr int kSoftmaxWarps = 4 * QT;
    uint8_t* sQ = smem_raw;
    uint8_t* ring = sQ + QT * kQBytes<HD>;
    Shared* sh = reinterpret_cast<Shared*>(ring + kRing * kT);
    static_assert(kRing <= 16 && kB * kKT + HD <= static_cast<int>(kCols) && 4 * kPatch <= kQBytes<HD>, "ring, TMEM columns, patches");
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    volatile int* cta_abort = &sh->abort;

    if ((smem_u32(smem_raw) & 1023u) != 0) {                // the swizzled tiles need 1024-byte alignment
        if (tid == 0) atomicExch(a.status, ODB_ERR_CUDA);
        pdl_wait();
        return;
    }
    if (tid == 0) {
        mbar_init(&sh->q_full, 1);
        for (int i = 0; i < kRing; ++i) {
            mbar_init(&sh->full[i], 1);
            mbar_init(&sh->empty[i], 1);
        }
        for (int g = 0; g < QT; ++g) {
            for (int b = 0; b < kB; ++b) {
                mbar_init(&sh->s_full[g][b], 1);
                mbar_init(&sh->p_full[g][b], 4);
            }
            for (int i = 0; i < 2; ++i) mbar_init(&sh->pv_done[g][i], 1);
            mbar_init(&sh->o_full[g], 1);
            sh->keep_o[g] = 0;
        }
        mbar_init(&sh->item_done, kSoftmaxWarps);
        sh->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kSoftmaxWarps) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)), "r"(QT * kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_launch_dependents();                                // behind the TMEM allocation
    pdl_wait();

    PagedStart start;
    static_assert(sizeof(PagedScratch) <= kQBytes<64>, "the scratch fits a Q tile");
    const bool any = paged_find_start<kThreads<QT>, kKT>(a, a.tile_rows, *reinterpret_cast<PagedScratch*>(sQ), 2, start);
    proxy_fence();                                          // the scratch's writes before the copies that take its place
    __syncthreads();

    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait_bounded(bar, parity, cta_abort, a.status); };
    const uint32_t tmem = __shfl_sync(0xffffffffu, sh->tmem_base, 0);                    // per Q tile 256 columns: kB x 64 of S or P, then O
    auto tmem_o = [&](int g) { return tmem + g * kCols + kCols - HD; };

    if (any && warp == kSoftmaxWarps + 1) {
        // ================= loader =================
        PagedWalk<kKT> w(a, start, a.tile_rows);
        const int box_shift = min(a.page_shift, 6), box = 1 << box_shift, boxes_all = kKT >> box_shift;
        bool ok = true;
        uint32_t item = 0, issued = 0;
        int slot = 0;
        uint32_t ph = 1;                                         // a slot's first load waits for nothing
        do {
            const int n = w.t1 - w.t0, n_loads = 2 * n, q_at = min(n_loads, kRing);
            // Load i: K(0) .. K(kFirst - 1), then K(t + kFirst), V(t) by turns, then the last V (the order of the MMAs).
            const int head_k = min(kFirst, n), turns = 2 * (n - head_k);
            for (int i = 0; i <= n_loads && ok; ++i) {
                if (i == q_at) {                                 // Q behind the first K and V tiles: they need no Q to be let in
                    if (item > 0) ok = wait(&sh->item_done, (item - 1) & 1u);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    const uint32_t bytes = static_cast<uint32_t>(a.tile_tokens) * a.G * 128;
                    if (lane == 0) mbar_expect_tx(&sh->q_full, QT * kAtoms * bytes);
                    __syncwarp();
                    if (lane < QT * kAtoms) {
                        const int g = lane / kAtoms, at = lane % kAtoms;
                        tma_box_3d(smem_u32(sQ) + g * kQBytes<HD> + at * kTQ * 128, &tm_q, &sh->q_full, 64 * at, w.head * a.G,
                                   w.q.row0 + (w.rt * QT + g) * a.tile_tokens);
                    }
                }
                if (i == n_loads) break;
                int tile = i;
                bool v = false;
                if (i >= head_k) {
                    const int j = i - head_k;
                    v = j >= turns || (j & 1);
                    tile = j >= turns ? j - turns / 2 : (j >> 1) + (v ? 0 : kFirst);
                }
                const int k0 = w.k.tile(w.t0 + tile) << 6;
                const int sub = lane / kAtoms, at = lane % kAtoms;
                const bool mine = sub < boxes_all && k0 + (sub << box_shift) < w.k.hi;
                const int boxes = __popc(__ballot_sync(0xffffffffu, mine));
                int row = a.pool_rows;                           // behind the pool: zeros
                if (mine) {
                    const int pos = k0 + (sub << box_shift);
                    const int page = a.table[static_cast<size_t>(w.seq) * a.table_stride + (pos >> a.page_shift)];
                    if (page >= 0 && page < a.n_pages)
                        row = (v ? a.v_row0 : a.k_row0) + ((page * a.KV + w.head) << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
                }
                if (issued >= kRing) {
                    ok = __all_sync(0xffffffffu, wait(&sh->empty[slot], ph));
                    if (!ok) break;
                }
                const uint32_t sl = __shfl_sync(0xffffffffu, slot, 0), dst = smem_u32(ring) + sl * kT;
                if (elect_one()) mbar_expect_tx(&sh->full[sl], static_cast<uint32_t>(boxes) * box * 128);
                __syncwarp();
                for (int c = 0; c < boxes; ++c) {
                    const int row_c = __shfl_sync(0xffffffffu, row, c), at_c = c % kAtoms, sub_c = c / kAtoms;
                    if (elect_one()) tma_box_3d(dst + at_c * kKT * 128 + sub_c * box * 128, &tm_kv, &sh->full[sl], 0, row_c, at_c);
                    __syncwarp();
                }
                ++issued;
                if (++slot == kRing) { slot = 0; ph ^= 1u; }
            }
            ++item;
        } while (ok && w.next());
        if (*cta_abort && lane == 0) {   // copies in flight land before the CTA's shared memory goes away
            const long long t0 = clock64();
            auto land = [&](uint64_t* bar, uint32_t parity) {
                while (!mbar_try_wait_parity(bar, parity) && clock64() - t0 < kWaitLimitCycles / 8) {
                }
            };
            land(&sh->q_full, (item - 1) & 1u);
            for (uint32_t j = issued > kRing ? issued - kRing : 0; j < issued; ++j) land(&sh->full[j % kRing], (j / kRing) & 1u);
        }
    } else if (any && warp == kSoftmaxWarps) {
        // ================= MMA issuer: the whole warp walks and waits, one lane issues =================
        PagedWalk<kKT> w(a, start, a.tile_rows);
        constexpr uint32_t idesc_s = instr_desc(kTQ, kKT, 0), idesc_o = instr_desc(kTQ, HD, 1);
        const uint64_t q_desc = desc_k_major(smem_u32(sQ)), ring_k = desc_k_major(smem_u32(ring)), ring_v = desc_mn_major(smem_u32(ring), kKT * 128);
        bool ok = true;
        uint32_t item = 0, done = 0;                             // key tiles of the items before
        int slot = 0;
        uint32_t ph = 0;
        auto uniform = [](uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); };
        auto all_wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
        auto next_slot = [&]() {
            if (++slot == kRing) { slot = 0; ph ^= 1u; }
        };
        do {
            const int n = w.t1 - w.t0;
            if (item > 0) ok = all_wait(&sh->item_done, (item - 1) & 1u);   // O read; with it every MMA of the item has completed
            if (ok) ok = all_wait(&sh->q_full, item & 1u);
            // S of the item's tile t, for every Q tile: its buffer's P has been multiplied
            auto issue_s = [&](int t) {
                if (!all_wait(&sh->full[slot], ph)) return false;
                const uint32_t gt = done + t, b = uniform(gt % kB), sl = uniform(slot);
                const uint64_t k_desc = ring_k + sl * (kT >> 4);
#pragma unroll
                for (int g = 0; g < QT; ++g) {
                    if (t >= kB) {
                        const uint32_t pv = gt - kB;
                        if (!all_wait(&sh->pv_done[g][pv & 1u], (pv >> 1) & 1u)) return false;
                    }
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < HD / 16; ++kk) {
                            const uint32_t atom = kk >> 2, within = (kk & 3) * 32;
                            umma(tmem + g * kCols + b * kKT, q_desc + ((g * kQBytes<HD> + atom * (kTQ * 128) + within) >> 4),
                                 k_desc + ((atom * (kKT * 128) + within) >> 4), idesc_s, kk > 0 ? 1u : 0u);
                        }
                        umma_commit(&sh->s_full[g][b]);
                        if (g == QT - 1) umma_commit(&sh->empty[sl]);
                    }
                    __syncwarp();
                }
                next_slot();
                return true;
            };
            for (int t = 0; t < kFirst && t < n && ok; ++t) ok = issue_s(t);
            for (int t = 0; t < n && ok; ++t) {
                if (t + kFirst < n) ok = issue_s(t + kFirst);
                if (ok) ok = all_wait(&sh->full[slot], ph);
                const uint32_t gt = done + t, b = uniform(gt % kB), sl = uniform(slot), last = t + 1 == n;
                const uint64_t v_desc = ring_v + sl * (kT >> 4);
#pragma unroll
                for (int g = 0; g < QT; ++g) {
                    if (ok) ok = all_wait(&sh->p_full[g][b], (gt / kB) & 1u);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t keep = uniform(t > 0 || *const_cast<volatile int*>(&sh->keep_o[g]) ? 1u : 0u);
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < kKT / 16; ++kk)
                            umma_ts(tmem_o(g), tmem + g * kCols + b * kKT + kk * 8, v_desc + kk * (2048 >> 4), idesc_o, kk > 0 ? 1u : keep);
                        umma_commit(&sh->pv_done[g][gt & 1u]);
                        if (last) umma_commit(&sh->o_full[g]);
                        if (g == QT - 1) umma_commit(&sh->empty[sl]);
                    }
                    __syncwarp();
                }
                if (ok) next_slot();
            }
            done += n;
            ++item;
        } while (ok && w.next());
    } else if (any) {
        // ================= softmax: thread r of Q tile g = packed row r = TMEM lane r =================
        PagedWalk<kKT> w(a, start, a.tile_rows);
        const int g = warp >> 2, gw = warp & 3, r = tid & 127;
        const uint32_t lane_base = static_cast<uint32_t>(gw * 32) << 16;   // this warp's TMEM lanes
        const uint32_t s_base = tmem + g * kCols + lane_base, o_base = tmem_o(g) + lane_base;
        const int rows_g = a.tile_tokens * a.G;                  // packed rows of a Q tile
        constexpr float kSlack = 4.0f;
        const uint64_t scale2 = pack2f(a.scale_log2, a.scale_log2);
        bool ok = true;
        uint32_t item = 0, done = 0, loads = 0;                  // key tiles and loads of the items before
        do {
            const int n = w.t1 - w.t0, head_k = min(kFirst, n);
            const int tok0 = (w.rt * QT + g) * a.tile_tokens;    // the Q tile's first query row
            const int pos = w.q.first + tok0 + min(r, rows_g - 1) / a.G;
            const int p_lo = w.q.first + tok0, p_hi = p_lo + a.tile_tokens - 1;
            float M_row = -INFINITY, l_row = 0.f;
            for (int t = 0; t < n; ++t) {
                const uint32_t gt = done + t, b = gt % kB;
                const uint32_t ts = s_base + b * kKT;
                const int k0 = w.k.tile(w.t0 + t) << 6;
                // seen by every row of the Q tile / tiles with rows of V that need care, the same for all Q tiles of the item
                const bool whole = k0 + kKT <= min(static_cast<long long>(w.q.len), static_cast<long long>(p_lo) + a.right + 1) &&
                                   (k0 >= p_hi - a.left || k0 + kKT <= a.sinks);
                const int item_lo = w.q.first + w.rt * QT * a.tile_tokens, item_hi = item_lo + QT * a.tile_tokens - 1;
                const bool whole_item = QT == 1 ? whole
                    : k0 + kKT <= min(static_cast<long long>(w.q.len), static_cast<long long>(item_lo) + a.right + 1) &&
                          (k0 >= item_hi - a.left || k0 + kKT <= a.sinks);
                ok = __all_sync(0xffffffffu, wait(&sh->s_full[g][b], (gt / kB) & 1u));
                tc_fence_after();
                uint32_t sv[64];                                         // the row's scores
                tmem_ld64(ts, sv);
                unsigned long long mask = ~0ull;                         // the keys of the tile that the row sees
                if (!whole) {
                    auto below = [](long long x) { return x >= 64 ? ~0ull : x <= 0 ? 0ull : (1ull << x) - 1ull; };
                    mask = below(min(static_cast<long long>(w.q.len), static_cast<long long>(pos) + a.right + 1) - k0) &
                           (~below(static_cast<long long>(pos) - a.left - k0) | below(static_cast<long long>(a.sinks) - k0));
#pragma unroll
                    for (int j = 0; j < 64; ++j)
                        if (!((mask >> j) & 1ull)) sv[j] = 0xff800000u;
                }
                float m0 = __uint_as_float(sv[0]), m1 = __uint_as_float(sv[32]);   // largest visible score of the tile
#pragma unroll
                for (int j = 1; j < 31; j += 2) {
                    m0 = max3(m0, __uint_as_float(sv[j]), __uint_as_float(sv[j + 1]));
                    m1 = max3(m1, __uint_as_float(sv[32 + j]), __uint_as_float(sv[33 + j]));
                }
                m0 = max3(m0, m1, __uint_as_float(sv[31]));
                m0 = fmaxf(m0, __uint_as_float(sv[63]));
                if (a.scale_log2 < 0.f) {                                // a negative scale turns the order around
                    m0 = INFINITY;
#pragma unroll
                    for (int j = 0; j < 64; ++j)
                        if ((mask >> j) & 1ull) m0 = fminf(m0, __uint_as_float(sv[j]));
                        else sv[j] = 0x7f800000u;                        // times the scale: minus infinity
                }
                float factor = 1.0f;                                     // what O and the row sum so far are multiplied by
                const float mt_log2 = mask ? m0 * a.scale_log2 : -INFINITY;
                if (mt_log2 > M_row + kSlack) {                          // also the first visible key (M_row = -inf)
                    const float M_new = ceilf(mt_log2);
                    if (M_row != -INFINITY) factor = exp2f(M_row - M_new);   // an exact power of two
                    M_row = M_new;
                }
                // The exponentials take a score's exact product with the scale, the shift comes from the rounded one: from 2^22 on
                // they lie up to 0.25 and more apart, and the scores are rounded first.
                const bool far = fabsf(mt_log2) >= 0x1p22f && mt_log2 != -INFINITY;
                bool rescale = false;
                uint64_t mult2 = scale2;
                if (__any_sync(0xffffffffu, factor != 1.0f || far)) {
                    rescale = __any_sync(0xffffffffu, factor != 1.0f);
                    if (__any_sync(0xffffffffu, far)) {
#pragma unroll
                        for (int j = 0; j < 64; ++j) sv[j] = __float_as_uint(__uint_as_float(sv[j]) * a.scale_log2);
                        mult2 = pack2f(1.0f, 1.0f);
                    }
                }
                const float m_log2 = M_row == -INFINITY ? 0.f : M_row;   // a row that has seen no key: every P is 0
                const uint64_t shift2 = pack2f(-m_log2, -m_log2);
                uint64_t sum[2] = {0ull, 0ull};
                uint32_t pb[32];                                         // the row's P: 64 keys as bf16 pairs
#pragma unroll
                for (int u = 0; u < 32; ++u) {
                    const float2 x = unpack2f(fma2(pack2u(sv[2 * u], sv[2 * u + 1]), mult2, shift2));
                    const float p0 = ex2_approx(x.x), p1 = ex2_approx(x.y);
                    sum[u & 1] = add2(sum[u & 1], pack2f(p0, p1));
                    pb[u] = paged_bf16x2(p0, p1);
                }
                tmem_st32(ts, pb);
                const float2 s0 = unpack2f(add2(sum[0], sum[1]));
                bool odd = false;
                uint32_t vt = 0;
                if (!whole_item) {
                    // V in places that a row does not see, once it has landed (its place in the loader's order: behind K(t + kFirst)).
                    // The parity is not ambiguous: the load before it in this slot is a K or V tile multiplied before S(t) was, the one
                    // behind it waits for P V(t).
                    const uint32_t i = loads + (t < n - head_k ? head_k + 2 * t + 1 : n + t), slot = i % kRing;
                    ok = __all_sync(0xffffffffu, wait(&sh->full[slot], (i / kRing) & 1u)) && ok;
                    vt = smem_u32(ring) + slot * kT;
#pragma unroll
                    for (int at = 0; at < kAtoms; ++at)
                        for (uint32_t off = tid * 16; off < kKT * 128; off += 128 * QT * 16) {
                            const int key = k0 + (off >> 7);
                            uint32_t v[4];
                            if (key >= w.k.hi || (key < w.k.lo && key >= a.sinks)) {
                                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(vt + at * kKT * 128 + off), "r"(0) : "memory");
                            } else {
                                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(vt + at * kKT * 128 + off) : "memory");
#pragma unroll
                                for (int j = 0; j < 4; ++j) odd = odd || not_finite(v[j]) || not_finite(v[j] >> 16);
                            }
                        }
                    proxy_fence();
                }
                if (rescale || !whole_item) {
                    // P V(t - 1) has been added to O.  The parity is not ambiguous: S(t) was issued behind P V(t - kB), so P V(t - 3),
                    // which the same barrier counts, has completed; P V(t + 1) cannot have, it is behind this P.
                    if (t > 0) ok = __all_sync(0xffffffffu, wait(&sh->pv_done[g][(gt - 1) & 1u], ((gt - 1) >> 1) & 1u)) && ok;
                    tc_fence_after();
                }
                if (rescale && t > 0) {                                  // warp-uniform; rows that keep their shift multiply by 1
#pragma unroll 1
                    for (int c = 0; c < HD / 32; ++c) {
                        uint32_t v[32];
                        tmem_ld32(o_base + c * 32, v);
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * factor);
                        tmem_st32(o_base + c * 32, v);
                    }
                }
                bool given = false;                                      // values of V are added to O here
                if (!whole_item) {
                    given = softmax_any<QT>(odd);                        // all have looked and cleared: they share the V tile
                    if (given) {                                         // rare
                        tmem_wait_st();
                        if (t == 0) {
                            uint32_t z[32];
#pragma unroll
                            for (int j = 0; j < 32; ++j) z[j] = 0u;
#pragma unroll 1
                            for (int c = 0; c < HD / 32; ++c) tmem_st32(o_base + c * 32, z);
                            tmem_wait_st();
                        }
#pragma unroll 1
                        for (int e = 0; e < kKT * HD; ++e) {
                            const int key = e / HD, d = e % HD;
                            unsigned short bits;
                            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(bits)
                                         : "r"(vt + (d >> 6) * kKT * 128 + key * 128 + ((((d >> 3) & 7) ^ (key & 7)) << 4) + (d & 7) * 2) : "memory");
                            if (!not_finite(bits)) continue;             // the same for all lanes
                            const uint32_t p2 = tmem_ld1(ts + key / 2);
                            const float p = __uint_as_float(key & 1 ? p2 & 0xffff0000u : p2 << 16), o = __uint_as_float(tmem_ld1(o_base + d));
                            tmem_st1(o_base + d, __float_as_uint((mask >> key) & 1ull ? o + p * __uint_as_float(static_cast<uint32_t>(bits) << 16) : o));
                        }
                        softmax_barrier<QT>();
#pragma unroll 1
                        for (uint32_t off = tid * 2; off < kT; off += 128 * QT * 2) {
                            unsigned short bits;
                            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(bits) : "r"(vt + off) : "memory");
                            if (not_finite(bits)) asm volatile("st.shared.u16 [%0], %1;" ::"r"(vt + off), "h"(static_cast<unsigned short>(0)) : "memory");
                        }
                        proxy_fence();
                        softmax_barrier<QT>();
                    }
                }
                if (t == 0 && r == 0) sh->keep_o[g] = given;
                l_row = l_row * factor + (s0.x + s0.y);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh->p_full[g][b]);
            }
            done += n;
            loads += 2 * n;
            const float m_log2 = M_row == -INFINITY ? 0.f : M_row;      // the shift the row's sum and output carry
            ok = __all_sync(0xffffffffu, wait(&sh->o_full[g], item & 1u)) && ok;
            tc_fence_after();
            const int row_w = gw * 32;                                   // the warp's first row of the Q tile
            const int left = min(rows_g, (w.q.n - tok0) * a.G) - row_w;   // rows of the Q tile from there on (may be negative)
            const uint32_t patch = smem_u32(sQ) + g * kQBytes<HD> + gw * kPatch;   // every MMA that reads this Q tile has completed
            const bool final = w.t0 == 0 && w.t1 == w.k.n;
            if (final) {
                int at[8];                                               // head of rows lane / 8, lane / 8 + 4 .. of the warp, from the Q tile's first
#pragma unroll
                for (int it = 0; it < 8; ++it) {
                    const int idx = row_w + it * 4 + (lane >> 3), i = idx / a.G;
                    at[it] = i * static_cast<int>(a.out_stride / 8) + (idx - i * a.G) * (HD / 8);
                }
                uint4* out = reinterpret_cast<uint4*>(a.out + static_cast<size_t>(w.q.row0 + tok0) * a.out_stride + w.head * a.G * HD);
                const float inv = l_row == 0.f ? 0.f : 1.0f / l_row;
                if (a.lse && lane < left) {
                    const int idx = row_w + lane, i = idx / a.G;
                    a.lse[static_cast<size_t>(w.q.row0 + tok0 + i) * a.H + w.head * a.G + idx - i * a.G] = paged_lse(m_log2, l_row);
                }
#pragma unroll 1
                for (int c = 0; c < HD / 64; ++c) {
                    uint32_t v[64], x[32];
                    tmem_ld64(o_base + c * 64, v);
#pragma unroll
                    for (int j = 0; j < 32; ++j) x[j] = paged_bf16x2(__uint_as_float(v[2 * j]) * inv, __uint_as_float(v[2 * j + 1]) * inv);
                    if (l_row == 0.f)                                    // no visible key: whatever O holds
#pragma unroll
                        for (int j = 0; j < 32; ++j) x[j] = 0u;
                    turn_rows(patch, lane, x, [&](int rr, int ch, const uint4& y) {
                        if (rr < left) out[at[rr >> 2] + c * 8 + ch] = y;
                    });
                }
            } else {
                const size_t pr = paged_part(a, blockIdx.x, w.t0 == 0) + g * rows_g + row_w;
                if (lane < left) *reinterpret_cast<float2*>(a.part_ml + (pr + lane) * 2) = make_float2(m_log2, l_row);
#pragma unroll 1
                for (int c = 0; c < HD / 32; ++c) {
                    uint32_t v[32];
                    tmem_ld32(o_base + c * 32, v);
                    if (l_row == 0.f)
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = 0u;
                    turn_rows(patch, lane, v, [&](int rr, int ch, const uint4& y) {
                        if (rr < left) *reinterpret_cast<uint4*>(a.part_o + (pr + rr) * HD + c * 32 + ch * 4) = y;
                    });
                }
            }
            proxy_fence();                                               // the patches before the next Q
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->item_done);
            if (!final) {
                __threadfence();
                softmax_barrier<QT>();
                const long long ub = w.item_begin();
                const int c0 = paged_owner(ub, start.total, start.ctas), c1 = paged_owner(ub + w.k.n - 1, start.total, start.ctas);
                if (tid == 0) {
                    const bool last = atomicAdd(a.arrivals + c0, 1u) == static_cast<unsigned>(c1 - c0);
                    if (last) a.arrivals[c0] = 0;                        // for the next launch; an item is counted at the CTA it begins in
                    __threadfence();
                    sh->last = last;
                }
                softmax_barrier<QT>();
                if (sh->last)
                    paged_merge<HD>(a, w.q.row0, w.head, w.rt * a.tile_rows, min(a.tile_rows, w.q.n * a.G - w.rt * a.tile_rows), c0, c1, warp, kSoftmaxWarps);
                softmax_barrier<QT>();                                   // sh->last has been read by all
            }
            ++item;
        } while (w.next());
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kSoftmaxWarps) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(QT * kCols) : "memory");
    }
}

template <int HD, int QT>
cudaError_t launch(const PagedAttnArgs& a, const CUtensorMap& tm_q, const CUtensorMap& tm_kv, int sms, cudaStream_t st) {
    static std::atomic<unsigned long long> attr_done{0};
    const cudaError_t e = set_smem_limit_once(attr_done, paged_attention_tc_kernel<HD, QT>, static_cast<int>(kSmem<HD, QT>));
    if (e != cudaSuccess) return e;
    return launch_kernel(paged_attention_tc_kernel<HD, QT>, dim3(QT == 1 ? 2 * sms : sms), dim3(kThreads<QT>), kSmem<HD, QT>, st, tm_q, tm_kv, a);
}

}  // namespace

cudaError_t launch_paged_attention_tc(PagedAttnArgs a, const PagedMaps& maps, int hd, int q_tiles, int sms, cudaStream_t st) {
    a.tile_tokens = kTQ / a.G;
    a.tile_rows = q_tiles * a.tile_tokens * a.G;
    a.part_rows = q_tiles * kPagedPartRows;
    CUtensorMap tm_q;
    const cudaError_t e = make_group_tmap(&tm_q, a.q, a.max_rows, a.q_stride, a.H, hd, a.G, a.tile_tokens);
    if (e != cudaSuccess) return e;
    if (q_tiles == 1) return hd == 128 ? launch<128, 1>(a, tm_q, maps.atoms, sms, st) : launch<64, 1>(a, tm_q, maps.atoms, sms, st);
    return hd == 128 ? launch<128, 2>(a, tm_q, maps.atoms, sms, st) : launch<64, 2>(a, tm_q, maps.atoms, sms, st);
}

}  // namespace odb
