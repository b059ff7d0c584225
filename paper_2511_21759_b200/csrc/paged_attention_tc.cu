// Attention of the rows of each request over its pages: many packed rows, on the tcgen05 tensor cores (formulas, masks and the
// division of the work: paged_attention.cu, paged.cuh).
//
// An item is QT Q tiles of up to 128 packed rows (floor(128 / group) query rows x the heads of a group) of one K/V head; a CTA
// walks its share of the line of key tiles of 64 positions, item after item.  QT = 1: two CTAs on an SM; QT = 2 (requests of more
// than 128 packed rows): one CTA whose two Q tiles share every K and V tile, which halves what comes from L2.
//
// Per key tile and Q tile: S = Q K^T is a 128 x 64 x HD group of MMAs into TMEM; thread r of the Q tile's four softmax warps owns
// TMEM lane r = packed row r, so a row's maximum and sum never leave the thread.  The row's shift M is an integer in the log2
// domain and moves only when a tile's maximum exceeds it by more than 8; O (in TMEM) and the sum are then multiplied by an exact
// power of two (with 4 a row of every warp still moved now and then, some 1000 cycles for both Q tiles: a prompt 151 us, with 8 141).
// P = exp2(S - M) < 256, rounded to bf16 (up to 2^-8 of itself a key, independent from key to key; the sum keeps the unrounded
// values), takes S's place in TMEM as the A operand of O += P V, with V taken MN-major from its [key][dim] tile.  A warp loads K and Q
// (TMA boxes of a page's rows x 64 values, which land in the canonical swizzled layout whatever the page size) and one V (a single
// warp both where two CTAs share the SM's registers), a warp a Q tile issues its MMAs, all meet through mbarriers with bounded waits;
// on expiry ODB_ERR_TIMEOUT is recorded and every role runs through its remaining barriers and ends.  A finished Q tile leaves by TMA
// from its Q's place; the parts of an item that several CTAs share are added up by a kernel of their own.
//
// Rows of V that no row of the item sees are set to zero in shared memory by their loader; so are values of V that are not finite at
// keys that only some rows see, and the softmax warps add those, from the pool, to O of the rows that see them, one TMEM column at a
// time.
//
// Measured, 32 query and 8 K/V heads of 128: a causal prompt of 4096 rows 140 us = 985 TFLOP/s of its visible pairs (0.58 of what a
// large matrix product reaches); blocks of 32 rows of 16 requests of up to 4096 keys 45 us = 3.7 TB/s; 4 requests of some 1300 rows, 32
// K/V heads, 140 us.  Called without a pause the large ones run into the card's 1000 W, at 1.6 GHz: 160 - 166 and 166 - 176 us.  A tile of both Q
// tiles takes some 1700 cycles: the products alone 1374 (51 cycles for 128 x 64 x 16, which shared memory bounds, 72 for 128 x 128 x
// 16), the exponentials 1024, a softmax warp's own chain from one score tile to the next some 1500.  An item costs 3 tiles beside its
// own, the start 4 us, the parts' kernel 7 us.
#include "paged_attention_tc.cuh"

namespace odb {

namespace {

template <int QT> constexpr int kLoaders = QT;   // one warp for K and V, or one each (one CTA's registers have room for a twelfth warp, two CTAs' not for two more)
template <int QT> constexpr int kThreads = 32 * (5 * QT + kLoaders<QT>);   // four softmax warps and an MMA warp a Q tile
// Q buffers: with two the next item's Q tiles and first scores are there when an item ends; the larger Q tiles of two CTAs on an SM
// leave no room for it.  K and V tiles in rings of their own.
template <int HD, int QT> constexpr int kQBufs = HD == 128 && QT == 1 ? 1 : 2;
template <int HD, int QT> constexpr int kKSlots = HD == 128 ? 3 : (QT == 1 ? 5 : 8);
template <int HD, int QT> constexpr int kVSlots = HD == 128 ? (QT == 1 ? 2 : 3) : (QT == 1 ? 5 : 8);
template <int HD, int QT>
constexpr uint32_t kSmem = kQBufs<HD, QT> * QT * kQBytes<HD> + (kKSlots<HD, QT> + kVSlots<HD, QT>) * kTileBytes<HD> + 1024;

struct alignas(8) Shared {
    uint64_t q_full[2];                // an item's Q tiles landed in the buffer          (loader -> MMA)
    uint64_t k_full[8], v_full[8];     // K or V tile landed in the ring's slot           (loader -> MMA; V -> its loader)
    uint64_t v_seen[8];                // V at keys that not all rows see has been looked at (loader -> softmax)
    uint64_t k_empty[8], v_empty[8];   // the MMAs have read the slot                     (MMA -> loader, QT arrivals)
    uint64_t s_full[2][3];             // S of Q tile g into buffer i has completed       (MMA -> softmax)
    uint64_t p_full[2][3];             // P has taken its place                           (softmax -> MMA, 4 arrivals)
    uint64_t pv_done[2][2];            // O += P V of an even / odd tile has completed    (MMA -> MMA, softmax)
    uint64_t o_full[2];                // the item's last one has                         (MMA -> softmax)
    uint64_t item_done[2];             // the Q buffer may be overwritten                 (softmax -> loader, 4 QT arrivals)
    uint32_t tmem_base;
    int abort, keep_o[2];
    int odd[8];                        // V in the slot has values that are not finite where only some rows see them
};
static_assert(sizeof(Shared) <= 1024, "the barriers end inside the allocation");

template <int HD_, int QT_>
struct Tc {
    static constexpr int HD = HD_, QT = QT_, NQ = kQBufs<HD, QT>, KS = kKSlots<HD, QT>, VS = kVSlots<HD, QT>;
    static constexpr bool kCodes = false;
    using Shared = odb::Shared;
    static __device__ __forceinline__ uint64_t* q_ready(Shared* sh, int) { return sh->q_full; }
    // V of the slot has been looked at; it has values that are not finite where only some rows see them; one of them (0: finite)
    static __device__ __forceinline__ uint64_t* v_seen(Shared* sh, uint32_t slot) { return &sh->v_seen[slot]; }
    static __device__ __forceinline__ bool odd(Shared* sh, uint32_t slot) { return *const_cast<volatile int*>(&sh->odd[slot]) != 0; }
    static __device__ __forceinline__ float odd_value(const PagedAttnArgs& a, int row, int d) {
        const uint32_t bits = a.pool[static_cast<size_t>(row) * HD + d];
        return not_finite(bits) ? __uint_as_float(bits << 16) : 0.f;
    }
};

template <int HD, int QT>
__global__ void __launch_bounds__(kThreads<QT>, QT == 1 ? 2 : 1)
    paged_attention_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_rows,
                              const __grid_constant__ CUtensorMap tm_atoms, const __grid_constant__ CUtensorMap tm_out, const PagedAttnArgs a) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    constexpr int NQ = kQBufs<HD, QT>, KS = kKSlots<HD, QT>, VS = kVSlots<HD, QT>, kB = kBufs<HD>, kFirst = kB - 1, kAtoms = HD / 64;
    constexpr uint32_t kT = kTileBytes<HD>;
    constexpr int kSoftmaxWarps = 4 * QT;
    uint8_t* sQ = smem_raw;                                  // [buffer][Q tile]
    uint8_t* sK = sQ + NQ * QT * kQBytes<HD>;
    uint8_t* sV = sK + KS * kT;
    Shared* sh = reinterpret_cast<Shared*>(sV + VS * kT);
    static_assert(KS <= 8 && VS <= 8 && kB * kKT + HD <= static_cast<int>(kCols) && 4 * kPatch <= kQBytes<HD>, "rings, TMEM columns, patches");
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    volatile int* cta_abort = &sh->abort;

    if ((smem_u32(smem_raw) & 1023u) != 0) {                // the swizzled tiles need 1024-byte alignment
        if (tid == 0) atomicExch(a.status, ODB_ERR_CUDA);
        pdl_wait();
        return;
    }
    if (tid == 0) {
        tma_prefetch_map(&tm_q);
        tma_prefetch_map(a.page_shift >= 6 ? &tm_rows : &tm_atoms);
        for (int i = 0; i < NQ; ++i) {
            mbar_init(&sh->q_full[i], 1);
            mbar_init(&sh->item_done[i], kSoftmaxWarps);
        }
        for (int i = 0; i < KS; ++i) {
            mbar_init(&sh->k_full[i], 1);
            mbar_init(&sh->k_empty[i], QT);
        }
        for (int i = 0; i < VS; ++i) {
            mbar_init(&sh->v_full[i], 1);
            mbar_init(&sh->v_seen[i], 1);
            mbar_init(&sh->v_empty[i], QT);
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
        sh->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kSoftmaxWarps) {
        __syncwarp();
        tmem_alloc(&sh->tmem_base, QT * kCols);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_launch_dependents();                                // behind the TMEM allocation
    pdl_wait();

    PagedStart start;
    static_assert(sizeof(PagedScratch) <= kSmem<64, 1> - 1024, "the scratch fits the tiles");
    const bool any = paged_find_start<kThreads<QT>, kKT, kItem, false>(a, *reinterpret_cast<PagedScratch*>(sQ), 1, kItem + 2, 0, start);
    proxy_fence();                                          // the scratch's writes before the copies that take its place
    __syncthreads();

    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait_bounded(bar, parity, cta_abort, a.status); };
    const uint32_t tmem = __shfl_sync(0xffffffffu, sh->tmem_base, 0);

    if (tid == 0) a.shared[blockIdx.x].rows = 0;            // thread 0 writes it again where an item begins here and ends elsewhere

    if (any && warp >= kSoftmaxWarps + QT) {
        // ================= loaders =================
        // K tiles, with Q before its item's first tile or (one Q buffer) where the item in front has ended, and V tiles; each walks
        // the share by itself.  A single warp takes them by turns, K kFirst tiles ahead.
        const int box_shift = min(a.page_shift, 6), box = 1 << box_shift;
        bool ok = true;
        auto all_wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
        struct Tiles {
            PagedWalk<kKT, kItem> w;
            PagedPages pages;
            int t, base, slots;
            uint32_t slot = 0, ph = 1, issued = 0, at;
            uint64_t *full, *empty;
            bool have = true;
        };
        Tiles k{PagedWalk<kKT, kItem>(a, start)}, v{PagedWalk<kKT, kItem>(a, start)};
        k.t = v.t = k.w.t0;
        k.base = a.k_row0; v.base = a.v_row0;
        k.slots = KS; v.slots = VS;
        k.at = __shfl_sync(0xffffffffu, smem_u32(sK), 0); v.at = __shfl_sync(0xffffffffu, smem_u32(sV), 0);
        k.full = sh->k_full; k.empty = sh->k_empty;
        v.full = sh->v_full; v.empty = sh->v_empty;
        // V in places that a row does not see: zero where no row sees it, and values that are not finite where some do, which the softmax
        // warps add to O of the rows that see them.  Here, once the tile has landed: nobody waits for it on the way.
        auto look = [&](const Tiles& x, int k0) {
            if (!SeenByAll(a, x.w.q, x.w.rt * QT * a.tile_tokens, QT * a.tile_tokens).tile(a, k0)) {
                ok = all_wait(&x.full[x.slot], x.ph ^ 1u);
                if (!ok) return;
                const uint32_t vt = x.at + x.slot * kT;
                uint32_t top = 0;                               // largest magnitudes of both halves of the words
#pragma unroll 8
                for (uint32_t off = lane * 16; off < kT; off += 512) {
                    const int key = k0 + ((off >> 7) & (kKT - 1));
                    const bool hidden = key >= x.w.k.hi || (key < x.w.k.lo && key >= a.sinks);
                    uint32_t v[4];
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(vt + off) : "memory");
                    uint32_t m = 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) m = max_u16x2(m, v[j] & 0x7fff7fffu);
                    if (hidden) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(vt + off), "r"(0) : "memory");
                    else top = max_u16x2(top, m);
                }
                const bool odd = __any_sync(0xffffffffu, not_finite(top) || not_finite(top >> 16));
                if (odd) {                                      // rare
#pragma unroll 1
                    for (uint32_t off = lane * 2; off < kT; off += 64) {
                        unsigned short bits;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(bits) : "r"(vt + off) : "memory");
                        if (not_finite(bits)) asm volatile("st.shared.u16 [%0], %1;" ::"r"(vt + off), "h"(static_cast<unsigned short>(0)) : "memory");
                    }
                }
                if (lane == 0) *const_cast<volatile int*>(&sh->odd[x.slot]) = odd;
                proxy_fence();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->v_seen[x.slot]);
            __syncwarp();
        };
        // pages of 64 rows and more: a copy a tile; smaller ones: a copy per page and 64 values, in their places of the operand layout
        auto load = [&](Tiles& x, auto ask) {
            if (!ok || !x.have) return;
            const int k0 = x.w.k.tile(x.t) << 6, keys = min(kKT, x.w.k.hi - k0);
            const int row = x.pages.template row<decltype(ask)::value>(a, x.w.q, x.w.seq, x.w.head, k0, x.base);
            if (x.issued >= static_cast<uint32_t>(x.slots)) ok = all_wait(&x.empty[x.slot], x.ph);
            if (!ok) return;
            const uint32_t dst = x.at + x.slot * kT;
            uint64_t* bar = &x.full[x.slot];
            if (box == kKT) {
                if (paged_elect()) {
                    mbar_expect_tx(bar, keys > 0 ? kT : 0u);
                    if (keys > 0) tma_box_3d(dst, &tm_rows, bar, 0, row, 0);
                }
                __syncwarp();
            } else {
                const int boxes = max(0, (keys + box - 1) >> box_shift);
                if (paged_elect()) mbar_expect_tx(bar, static_cast<uint32_t>(boxes) * box * HD * 2);
                __syncwarp();
                for (int c = 0; c < boxes; ++c) {
                    const int row_c = x.pages.template row<decltype(ask)::value>(a, x.w.q, x.w.seq, x.w.head, k0 + (c << box_shift), x.base);
                    if (paged_elect()) {
#pragma unroll
                        for (int at = 0; at < kAtoms; ++at) tma_box_3d(dst + at * kKT * 128 + c * box * 128, &tm_atoms, bar, 0, row_c, at);
                    }
                    __syncwarp();
                }
            }
            if (x.full == sh->v_full) look(x, k0);
            ++x.issued;
            if (++x.slot == static_cast<uint32_t>(x.slots)) { x.slot = 0; x.ph ^= 1u; }
            if (++x.t == x.w.t1) {
                x.have = x.w.next();
                x.t = x.w.t0;
            }
        };
        uint32_t nq = 0;
        auto load_q = [&](const PagedWalk<kKT, kItem>& w) {
            const uint32_t buf = nq % NQ;
            if (nq >= NQ) ok = ok && all_wait(&sh->item_done[buf], (nq / NQ - 1) & 1u);
            if (!ok) return;
            const uint32_t dst = __shfl_sync(0xffffffffu, smem_u32(sQ) + buf * QT * kQBytes<HD>, 0);
            const int row = w.q.row0 + w.rt * QT * a.tile_tokens;
            if (paged_elect()) {
                mbar_expect_tx(&sh->q_full[buf], QT * kAtoms * static_cast<uint32_t>(a.tile_tokens) * a.G * 128);
#pragma unroll
                for (int g = 0; g < QT; ++g)
#pragma unroll
                    for (int at = 0; at < kAtoms; ++at)
                        tma_box_3d(dst + g * kQBytes<HD> + at * kTQ * 128, &tm_q, &sh->q_full[buf], 64 * at, w.head * a.G, row + g * a.tile_tokens);
            }
            __syncwarp();
            ++nq;
        };
        if (kLoaders<QT> == 2) {
            static_assert(kLoaders<QT> == 1 || NQ == 2, "K waits for its item's Q buffer, V does not");
            if (warp == kSoftmaxWarps + QT)
                while (ok && k.have) {
                    if (k.t == k.w.t0) load_q(k.w);
                    load(k, std::false_type());
                }
            else
                while (ok && v.have) load(v, std::true_type());
        } else {
            PagedWalk<kKT, kItem> wq(a, start);
            bool have_q = true;
            auto next_q = [&]() {
                if (!have_q) return;
                load_q(wq);
                have_q = wq.next();
            };
            for (int i = 0; i < kFirst; ++i) load(k, std::false_type());
            if (NQ == 2) next_q();
            while (ok && v.have) {
                if (NQ == 1 && v.t == v.w.t0) next_q();
                // behind the item's third tile: the epilogue in front of it, which frees the buffer, is on its way by then
                const bool then_q = NQ == 2 && v.t == min(v.w.t0 + 2, v.w.t1 - 1);
                load(k, std::false_type());
                load(v, std::true_type());
                if (then_q) next_q();
            }
        }
        if (*cta_abort && lane == 0) {   // copies in flight land before the CTA's shared memory goes away
            const long long t0 = clock64();
            auto land = [&](uint64_t* bars, uint32_t n, uint32_t slots) {
                for (uint32_t j = n > slots ? n - slots : 0; j < n; ++j)
                    while (!mbar_try_wait_parity(&bars[j % slots], (j / slots) & 1u) && clock64() - t0 < kWaitLimitCycles / 8) {
                    }
            };
            land(sh->q_full, nq, NQ);
            land(sh->k_full, k.issued, KS);
            land(sh->v_full, v.issued, VS);
        }
    } else if (any && warp >= kSoftmaxWarps) {
        paged_tc_mma<Tc<HD, QT>>(a, start, sh, sQ, sK, sV, tmem, warp - kSoftmaxWarps);
    } else if (any) {
        paged_tc_softmax<Tc<HD, QT>>(a, start, tm_out, sh, sQ, tmem);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kSoftmaxWarps) {
        __syncwarp();
        tc_fence_after();
        tmem_free(tmem, QT * kCols);
    }
}

template <int HD, int QT>
cudaError_t launch(const PagedAttnArgs& a, const CUtensorMap& tm_q, const CUtensorMap& tm_out, const PagedMaps& maps, cudaStream_t st) {
    static std::atomic<unsigned long long> attr_done{0};
    cudaError_t e = set_smem_limit_once(attr_done, paged_attention_tc_kernel<HD, QT>, static_cast<int>(kSmem<HD, QT>));
    if (e != cudaSuccess) return e;
    const dim3 grid(a.at_once);
    e = launch_kernel(paged_attention_tc_kernel<HD, QT>, grid, dim3(kThreads<QT>), kSmem<HD, QT>, st, tm_q, maps.rows, maps.atoms, tm_out, a);
    if (e != cudaSuccess) return e;
    return launch_kernel(paged_merge_kernel<HD>, dim3(grid.x, QT * HD / kMergeDims), dim3(kTQ), 0, st, a);
}

}  // namespace

cudaError_t launch_paged_attention_tc(PagedAttnArgs a, const PagedMaps& maps, int hd, int q_tiles, int sms, cudaStream_t st) {
    CUtensorMap tm_q, tm_out;
    const cudaError_t e = paged_tc_args(a, hd, q_tiles, sms, &tm_q, &tm_out);
    if (e != cudaSuccess) return e;
    if (q_tiles == 1) return hd == 128 ? launch<128, 1>(a, tm_q, tm_out, maps, st) : launch<64, 1>(a, tm_q, tm_out, maps, st);
    return hd == 128 ? launch<128, 2>(a, tm_q, tm_out, maps, st) : launch<64, 2>(a, tm_q, tm_out, maps, st);
}

}  // namespace odb
