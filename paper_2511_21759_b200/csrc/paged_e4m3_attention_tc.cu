// Attention over a pool of 8 bits: many packed rows, on the tcgen05 tensor cores.  Formulas, masks, the division of the work, products,
// softmax and results: paged_attention_tc.cu, whose kernel this is behind the K and V tiles in shared memory; K and V of a position are
// code * scale, numbers of bf16.
//
// An item is one Q tile, and every item writes its K and V tiles as operands for itself: this kernel is for requests of one row tile
// (block steps) and for mixtures; prompts, whose row tiles would all do that again, take the pool's bf16 copy where there is memory for it
// (paged_load.cu).
//
// Both products are f16: a code is a number of f16, and one instruction makes an operand's word of two codes (as bf16 with its scale a code
// took five times the work, and the converters were what the kernel waited for: blocks of 32 rows 92 us instead of 67).  TMA brings codes
// into staging tiles, and converter warps write them into the places of the operands' canonical layout.  Scales stay outside, as in the
// kernel of few rows:
//   S: each softmax thread brings its row of Q into 1 .. 2 by a power of two, as f16, before the item's first product; a score is
//      multiplied by that power, the softmax scale and its block's.
//   P V: the weights that multiply codes are 2^(x - M + log2(V's scale) - G), with M + G, both whole numbers, moved as the shift of bf16
//      is, by the largest x + log2 of a tile (apart, so that large scores do not lose the scales), whose weight is then 2^6 to 2^7 and
//      later ones' up to 2^15; in f16, off by up to 2^-11 of themselves or 2^-31 of the row's largest (with weights of 1 for the largest
//      it was 2^-24, and thousands of keys beside one that takes most lost a tenth and more of their part).  The sum takes them block by
//      block over V's scale, so that sum and output move together (the sum's unit is 2^(M + G + kRoom), the output's 2^(M + G)), and the
//      rest is as for bf16.  Where V's scales are beyond 2^+-40 weights may vanish that count in the sum, which then has exponentials of
//      its own.
// The converters also do what the loader of bf16 does with V at keys that not all rows see: zeros where no row sees them, and NaN is
// kept for the softmax warps.
//
// Registers: the softmax warps take 160, all others 96 of the 128 that a thread is launched with.
#include "paged_attention_tc.cuh"
#include "paged_e4m3.cuh"

namespace odb {

namespace {

constexpr int kThreads = 256;                               // four softmax warps; an MMA warp, the loader, a converter of K and one of V
constexpr int kLaunchRegs = 128, kSoftmaxRegs = 160, kOtherRegs = 96;   // as many warpgroups of the one as of the other
static_assert(kSoftmaxRegs + kOtherRegs <= 2 * kLaunchRegs, "the split fits what the block was launched with");
template <int HD> constexpr int kQBufs = HD == 128 ? 1 : 2;
template <int HD> constexpr int kKSlots = HD == 128 ? 1 : 3;                                // K tiles as operands
template <int HD> constexpr int kVSlots = HD == 128 ? 2 : 3;                                // V tiles
template <int HD> constexpr int kStaging = HD == 128 ? 2 : 3;                               // tiles of codes, of K and of V
template <int HD> constexpr uint32_t kCodeBytes = kKT * HD;
template <int HD>
constexpr uint32_t kSmem = kQBufs<HD> * kQBytes<HD> + (kKSlots<HD> + kVSlots<HD>) * kTileBytes<HD> + 2 * kStaging<HD> * kCodeBytes<HD> + 1024;
static_assert(2 * (kSmem<128> + 1024) <= 228 * 1024 && 2 * (kSmem<64> + 1024) <= 228 * 1024, "two CTAs share an SM");

constexpr int kBlocks = kKT / kPagedBlock;   // of a tile
constexpr int kAhead = 8;                    // a tile of K is converted less than that many tiles ahead of the softmax: kBufs - 1 scores, the slots of K

struct alignas(16) SharedE4m3 {
    uint64_t q_full[2];                // an item's Q tiles landed in the buffer          (loader -> MMA)
    uint64_t q_ready[2];               // the Q tile in the buffer is f16                 (softmax -> MMA, 4 arrivals)
    uint64_t st_full[2][3];            // a tile of codes of K, with all scales, / V landed (loader -> converters)
    uint64_t st_empty[2][3];           // the converters have read it                     (converters -> loader)
    uint64_t k_full[3], v_full[3];     // K or V tile written, V looked at                (converters -> MMA; V -> softmax)
    uint64_t k_empty[3], v_empty[3];   // the MMAs have read the slot                     (MMA -> converters)
    uint64_t s_full[1][3];             // S into buffer i has completed       (MMA -> softmax)
    uint64_t p_full[1][3];             // P has taken its place                           (softmax -> MMA, 4 arrivals)
    uint64_t pv_done[1][2];            // O += P V of an even / odd tile has completed    (MMA -> MMA, softmax)
    uint64_t o_full[1];                // the item's last one has                         (MMA -> softmax)
    uint64_t item_done[2];             // the Q buffer may be overwritten                 (softmax -> loader, 4 arrivals)
    uint32_t tmem_base;
    int abort, keep_o[1];
    float scale[3][2][kBlocks];        // of a staging tile's blocks of K, of V
    alignas(16) float scales[kAhead][3][kBlocks];   // of the tiles at work: K's scale, log2 of V's, 2^-kRoom / V's (converter of K -> softmax)
    int wide[kAhead];                  // some log2 of V's scales is beyond +-40
    int odd[3];                        // V in the slot has NaN where only some rows see it
};
static_assert(sizeof(SharedE4m3) <= 1024, "the barriers end inside the allocation");

template <int HD_>
struct TcE4m3 {
    static constexpr int HD = HD_, QT = 1, NQ = kQBufs<HD>, KS = kKSlots<HD>, VS = kVSlots<HD>;
    static constexpr bool kCodes = true;
    using Shared = SharedE4m3;
    static __device__ __forceinline__ uint64_t* q_ready(Shared* sh, int) { return sh->q_ready; }
    // The thread's row of the item's Q tile as f16 in 1 .. 2: what its scores are multiplied by.
    template <int ROWS, class Wait>
    static __device__ __forceinline__ float own_q(Shared* sh, uint8_t* sQ, uint32_t item, int r, bool& ok, Wait& wait) {
        const uint32_t buf = item % NQ, row = smem_u32(sQ) + buf * kQBytes<HD> + r * 128;
        ok = __all_sync(0xffffffffu, wait(&sh->q_full[buf], (item / NQ) & 1u)) && ok;
        auto at = [&](int c) { return row + (c >> 3) * (ROWS * 128) + (((c & 7) ^ (r & 7)) << 4); };
        uint32_t x[HD / 8][4], top = 0;
#pragma unroll
        for (int c = 0; c < HD / 8; ++c)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[c][0]), "=r"(x[c][1]), "=r"(x[c][2]), "=r"(x[c][3]) : "r"(at(c)) : "memory");
#pragma unroll
        for (int c = 0; c < HD / 8; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) top = max_u16x2(top, x[c][j] & 0x7fff7fffu);
        top = max(top & 0xffffu, top >> 16);
        const int ex = q_exponent(top);
        const float by = exp2_int(-ex);
#pragma unroll
        for (int c = 0; c < HD / 8; ++c) {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[c][j] = paged_f16x2(__uint_as_float(x[c][j] << 16) * by, __uint_as_float(x[c][j] & 0xffff0000u) * by);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at(c)), "r"(x[c][0]), "r"(x[c][1]), "r"(x[c][2]), "r"(x[c][3]) : "memory");
        }
        proxy_fence();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(&sh->q_ready[buf]);
        return exp2_int(ex);
    }
    // The scales of tile n's blocks; whether V's are wide.
    static __device__ __forceinline__ bool scales(Shared* sh, uint32_t n, float (&k)[kBlocks], float (&log_v)[kBlocks], float (&by_v)[kBlocks]) {
        const float4* s = reinterpret_cast<const float4*>(sh->scales[n % kAhead]);
        const float4 x = s[0], y = s[1], z = s[2];
        k[0] = x.x; k[1] = x.y; k[2] = x.z; k[3] = x.w;
        log_v[0] = y.x; log_v[1] = y.y; log_v[2] = y.z; log_v[3] = y.w;
        by_v[0] = z.x; by_v[1] = z.y; by_v[2] = z.z; by_v[3] = z.w;
        return sh->wide[n % kAhead] != 0;
    }
    // V of the slot has been looked at; it has NaN where only some rows see it; whether this is one (0: it is not)
    static __device__ __forceinline__ uint64_t* v_seen(Shared* sh, uint32_t slot) { return &sh->v_full[slot]; }
    static __device__ __forceinline__ bool odd(Shared* sh, uint32_t slot) { return *const_cast<volatile int*>(&sh->odd[slot]) != 0; }
    static __device__ __forceinline__ float odd_value(const PagedAttnArgs& a, int row, int d) {
        const unsigned char code = reinterpret_cast<const unsigned char*>(a.pool)[static_cast<size_t>(row) * HD + d];
        return (code & 0x7f) == 0x7f ? __uint_as_float(0x7fffffffu) : 0.f;
    }
};

template <int HD>
__global__ void __launch_bounds__(kThreads, 2)
    paged_e4m3_attention_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_codes,
                                   const __grid_constant__ CUtensorMap tm_out, const PagedAttnArgs a) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    using T = TcE4m3<HD>;
    constexpr int NQ = T::NQ, KS = T::KS, VS = T::VS, ST = kStaging<HD>, kFirst = kBufs<HD> - 1, kAtoms = HD / 64;
    constexpr uint32_t kT = kTileBytes<HD>, kC = kCodeBytes<HD>;
    constexpr int kSoftmaxWarps = 4, kLoader = 5, kConvK = 6;
    uint8_t* sQ = smem_raw;
    uint8_t* sK = sQ + NQ * kQBytes<HD>;
    uint8_t* sV = sK + KS * kT;
    uint8_t* sC = sV + VS * kT;                              // [K, V][tile]
    SharedE4m3* sh = reinterpret_cast<SharedE4m3*>(sC + 2 * ST * kC);
    static_assert(VS >= kBufs<HD>, "the tile before in a slot of V has been multiplied when the softmax asks for this one");
    static_assert(kBufs<HD> - 1 + KS < kAhead, "a tile's scales stay until the softmax has read them");
    static_assert(KS <= 3 && VS <= 3 && ST <= 3 && kBufs<HD> * kKT + HD <= static_cast<int>(kCols) && 4 * kPatch <= kQBytes<HD>, "rings, TMEM columns, patches");
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    volatile int* cta_abort = &sh->abort;

    if ((smem_u32(smem_raw) & 1023u) != 0) {                // the swizzled tiles need 1024-byte alignment
        if (tid == 0) atomicExch(a.status, ODB_ERR_CUDA);
        pdl_wait();
        return;
    }
    if (tid == 0) {
        tma_prefetch_map(&tm_q);
        tma_prefetch_map(&tm_codes);
        for (int i = 0; i < NQ; ++i) {
            mbar_init(&sh->q_full[i], 1);
            mbar_init(&sh->item_done[i], kSoftmaxWarps);
        }
        for (int i = 0; i < 2 * ST; ++i) {
            mbar_init(&sh->st_full[i & 1][i >> 1], i & 1 ? 1 : 1 + 2 * kBlocks);   // the tile, and the lanes that copy scales
            mbar_init(&sh->st_empty[i & 1][i >> 1], 1);
        }
        for (int i = 0; i < KS; ++i) {
            mbar_init(&sh->k_full[i], 1);
            mbar_init(&sh->k_empty[i], 1);
        }
        for (int i = 0; i < VS; ++i) {
            mbar_init(&sh->v_full[i], 1);
            mbar_init(&sh->v_empty[i], 1);
        }
        for (int b = 0; b < kBufs<HD>; ++b) {
            mbar_init(&sh->s_full[0][b], 1);
            mbar_init(&sh->p_full[0][b], 4);
        }
        for (int i = 0; i < 2; ++i) mbar_init(&sh->pv_done[0][i], 1);
        mbar_init(&sh->o_full[0], 1);
        for (int i = 0; i < NQ; ++i) mbar_init(&sh->q_ready[i], 4);
        sh->keep_o[0] = 0;
        sh->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kSoftmaxWarps) paged_tc_alloc(&sh->tmem_base, kCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_launch_dependents();                                // behind the TMEM allocation
    pdl_wait();

    PagedStart start;
    static_assert(sizeof(PagedScratch) <= kSmem<64> - 1024, "the scratch fits the tiles");
    const bool any = paged_find_start<kThreads, kKT, kItem, false>(a, *reinterpret_cast<PagedScratch*>(sQ), 1, kItem + 2, 0, start);
    proxy_fence();                                          // the scratch's writes before the copies that take its place
    __syncthreads();

    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait_bounded(bar, parity, cta_abort, a.status); };
    auto all_wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
    const uint32_t tmem = __shfl_sync(0xffffffffu, sh->tmem_base, 0);
    if (tid == 0) a.shared[blockIdx.x].rows = 0;            // thread 0 writes it again where an item begins here and ends elsewhere
    // K or V tiles of the share, and the staging ring that they go through
    struct Tiles {
        PagedWalk<kKT, kItem> w;
        int t;
        uint32_t slot = 0, ph = 0, n = 0;
        bool have = true;
        __device__ __forceinline__ Tiles(const PagedAttnArgs& args, const PagedStart& st) : w(args, st), t(w.t0) {}
        __device__ __forceinline__ void next() {
            ++n;
            if (++slot == static_cast<uint32_t>(ST)) { slot = 0; ph ^= 1u; }
            if (++t == w.t1) {
                have = w.next();
                t = w.t0;
            }
        }
    };

    if (!any) {
        // nothing to do for this CTA
    } else if (warp < kSoftmaxWarps) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        paged_tc_softmax<T>(a, start, tm_out, sh, sQ, tmem);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp < kLoader) {
            paged_tc_mma<T>(a, start, sh, sQ, sK, sV, tmem, warp - kSoftmaxWarps);
        } else if (warp == kLoader) {
            // ================= loader: codes and scales; Q before its item's first tile or (one Q buffer) where the item in front has ended
            const int box_shift = min(a.page_shift, 6), box = 1 << box_shift;
            bool ok = true;
            Tiles k(a, start), v(a, start);
            PagedPages k_pages, v_pages;
            uint32_t nq = 0;
            const uint32_t codes = __shfl_sync(0xffffffffu, smem_u32(sC), 0);
            auto load = [&](Tiles& x, PagedPages& pages, auto is_v) {
                constexpr int V = decltype(is_v)::value;
                if (!ok || !x.have) return;
                const int k0 = x.w.k.tile(x.t) << 6, b = lane & (kBlocks - 1);
                const int boxes = max(0, (min(kKT, x.w.k.hi - k0) + box - 1) >> box_shift), n_blocks = boxes << box_shift >> 4;
                const int row = pages.rows<V != 0>(a, x.w.q, x.w.seq, x.w.head, k0, b * kPagedBlock, b < n_blocks, V ? a.v_row0 : a.k_row0);
                if (x.n >= static_cast<uint32_t>(ST)) ok = all_wait(&sh->st_empty[V][x.slot], x.ph ^ 1u);
                if (!ok) return;
                uint64_t* full = &sh->st_full[V][x.slot];
                if (paged_elect()) mbar_expect_tx(full, static_cast<uint32_t>(boxes) * box * HD);
                __syncwarp();
                for (int c = 0; c < boxes; ++c) {
                    const int r = __shfl_sync(0xffffffffu, row, c << box_shift >> 4);
                    if (paged_elect()) tma_codes(codes + (V * ST + x.slot) * kC + c * box * HD, &tm_codes, full, r);
                    __syncwarp();
                }
                if (!V && lane < 2 * kBlocks) {              // K's scales, then V's; a page that is none reads as zeros
                    float* scale = &sh->scale[x.slot][0][lane];
                    if (b < n_blocks && row >= a.pool_rows) {
                        *scale = 1.f;
                        mbar_arrive(full);                   // a copy's arrival would not wait for this lane's own write
                    } else {
                        if (b < n_blocks) copy4(smem_u32(scale), a.scales + (row + (lane < kBlocks ? 0 : a.v_row0 - a.k_row0)) / kPagedBlock);
                        copies_arrive(full);
                    }
                }
                __syncwarp();
                x.next();
            };
            PagedWalk<kKT, kItem> wq(a, start);
            bool have_q = true;
            auto next_q = [&]() {
                if (!have_q) return;
                const uint32_t buf = nq % NQ;
                if (nq >= NQ) ok = ok && all_wait(&sh->item_done[buf], (nq / NQ - 1) & 1u);
                if (!ok) return;
                const uint32_t dst = __shfl_sync(0xffffffffu, smem_u32(sQ) + buf * kQBytes<HD>, 0);
                const int row = wq.q.row0 + wq.rt * a.tile_tokens;
                if (paged_elect()) {
                    mbar_expect_tx(&sh->q_full[buf], kAtoms * static_cast<uint32_t>(a.tile_tokens) * a.G * 128);
#pragma unroll
                    for (int at = 0; at < kAtoms; ++at) tma_box_3d(dst + at * kTQ * 128, &tm_q, &sh->q_full[buf], 64 * at, wq.head * a.G, row);
                }
                __syncwarp();
                ++nq;
                have_q = wq.next();
            };
            for (int i = 0; i < kFirst; ++i) load(k, k_pages, std::false_type());
            if (NQ == 2) next_q();
            while (ok && v.have) {
                if (NQ == 1 && v.t == v.w.t0) next_q();
                // behind the item's third tile: the epilogue in front of it, which frees the buffer, is on its way by then
                const bool then_q = NQ == 2 && v.t == min(v.w.t0 + 2, v.w.t1 - 1);
                load(k, k_pages, std::false_type());
                load(v, v_pages, std::true_type());
                if (then_q) next_q();
            }
            if (*cta_abort && lane == 0) {   // copies in flight land before the CTA's shared memory goes away
                const long long t0 = clock64();
                auto land = [&](uint64_t* bars, uint32_t n, uint32_t slots) {
                    for (uint32_t j = n > slots ? n - slots : 0; j < n; ++j)
                        while (!mbar_try_wait_parity(&bars[j % slots], (j / slots) & 1u) && clock64() - t0 < kWaitLimitCycles / 8) {
                        }
                };
                land(sh->q_full, nq, NQ);
                land(sh->st_full[0], k.n, ST);
                land(sh->st_full[1], v.n, ST);
            }
        } else {
            // ================= converters of K and of V =================
            constexpr int kPieces = HD / 16, kSteps = kKT * kPieces / 32;
            // Of eight lanes at a time, which 16 bytes a lane take together, four have neighbouring pieces of key k and four those of key k ^ 5 (head
            // dim 64: k ^ 1): by the swizzles their loads and their stores meet all banks.  Steps 0 and 1 take four each of eight keys.
            const int piece = HD == 128 ? (lane & 3) + (lane >> 3 & 1) * 4 : lane & 3, atom = piece >> 2;
            auto key_of = [&](int step) { return HD == 128 ? (step >> 1) * 8 + (((lane >> 4) + 2 * (step & 1)) ^ (5 * (lane >> 2 & 1))) : step * 8 + (lane >> 2); };
            auto convert = [&](uint8_t* tiles, uint64_t* full, uint64_t* empty, auto is_v) {
                constexpr int V = decltype(is_v)::value, SL = V ? VS : KS;
                Tiles x(a, start);
                uint32_t slot = 0, empty_ph = 1;
                while (x.have) {
                    const int k0 = x.w.k.tile(x.t) << 6;
                    const bool care = V && !SeenByAll(a, x.w.q, x.w.rt * a.tile_tokens, a.tile_tokens).tile(a, k0);
                    bool ok = all_wait(&sh->st_full[V][x.slot], x.ph);
                    if (ok && x.n >= static_cast<uint32_t>(SL)) ok = all_wait(&empty[slot], empty_ph);
                    if (!ok) break;
                    const uint32_t from = smem_u32(sC) + (V * ST + x.slot) * kC, to = smem_u32(tiles) + slot * kT + atom * kKT * 128;
                    auto code_at = [&](int key) -> uint32_t {
                        return HD == 128 ? from + key * 128 + ((piece ^ (key & 7)) << 4) : from + key * 64 + ((piece ^ (key >> 1 & 3)) << 4);
                    };
                    auto hidden = [&](int key) { return care && (k0 + key >= x.w.k.hi || (k0 + key < x.w.k.lo && k0 + key >= a.sinks)); };
                    if (!V) {                      // the tile's scales to the softmax warps
                        const int first = k0 + (lane & (kBlocks - 1)) * kPagedBlock;
                        const bool unseen = first >= x.w.k.hi || (first + kPagedBlock <= x.w.k.lo && first >= a.sinks);   // by all rows of the item
                        const int e = unseen ? 0 : e4m3_exponent((&sh->scale[x.slot][0][0])[lane & (2 * kBlocks - 1)]);
                        float* s = &sh->scales[x.n % kAhead][0][0];
                        if (lane < kBlocks) s[lane] = exp2_int(e);
                        else if (lane < 2 * kBlocks) {
                            s[lane] = static_cast<float>(e);
                            s[lane + kBlocks] = exp2_int(-e - static_cast<int>(kRoom));
                        }
                        const bool wide = __any_sync(0xffffffffu, lane >= kBlocks && lane < 2 * kBlocks && (e < -40 || e > 40));
                        if (lane == 0) sh->wide[x.n % kAhead] = wide;
                    }
                    bool nan = false;
                    // few instructions, in a loop that is not unrolled far: what the softmax warps beside it run has to stay in the instruction cache
#pragma unroll 1
                    for (int step = 0; step < kSteps; ++step) {
                        const int key = key_of(step);
                        uint32_t w[4];
                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(code_at(key)) : "memory");
                        if (care) {
                            const bool out = hidden(key);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                if (out) w[j] = 0u;
                                nan = nan || odd_codes(w[j]);             // rare: the softmax warps give it to the rows that see it
                                w[j] = without_nan(w[j]);
                            }
                        }
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + key * 128 + ((((piece & 3) * 2 + h) ^ (key & 7)) << 4)),
                                         "r"(low_codes(w[2 * h])), "r"(high_codes(w[2 * h])), "r"(low_codes(w[2 * h + 1])), "r"(high_codes(w[2 * h + 1]))
                                         : "memory");
                    }
                    nan = __any_sync(0xffffffffu, nan);
                    if (care && lane == 0) *const_cast<volatile int*>(&sh->odd[slot]) = nan;
                    proxy_fence();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(&full[slot]);
                        mbar_arrive(&sh->st_empty[V][x.slot]);
                    }
                    __syncwarp();
                    if (++slot == static_cast<uint32_t>(SL)) { slot = 0; empty_ph ^= 1u; }
                    x.next();
                }
            };
            if (warp == kConvK) convert(sK, sh->k_full, sh->k_empty, std::false_type());
            else convert(sV, sh->v_full, sh->v_empty, std::true_type());
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kSoftmaxWarps) {
        __syncwarp();
        tc_fence_after();
        tmem_free(tmem, kCols);
    }
}

template <int HD>
cudaError_t launch(const PagedAttnArgs& a, const CUtensorMap& tm_q, const CUtensorMap& tm_out, const CUtensorMap& map, cudaStream_t st) {
    static std::atomic<unsigned long long> attr_done{0};
    cudaError_t e = set_smem_limit_once(attr_done, paged_e4m3_attention_tc_kernel<HD>, static_cast<int>(kSmem<HD>));
    if (e != cudaSuccess) return e;
    static std::atomic<int> regs{0};
    if (regs.load(std::memory_order_relaxed) != kLaunchRegs) {   // with fewer the softmax warps would wait for the others' without end
        cudaFuncAttributes f;
        e = cudaFuncGetAttributes(&f, paged_e4m3_attention_tc_kernel<HD>);
        if (e != cudaSuccess) return e;
        if (f.numRegs != kLaunchRegs) return cudaErrorInvalidConfiguration;
        regs.store(f.numRegs, std::memory_order_relaxed);
    }
    const dim3 grid(a.at_once);
    e = launch_kernel(paged_e4m3_attention_tc_kernel<HD>, grid, dim3(kThreads), kSmem<HD>, st, tm_q, map, tm_out, a);
    if (e != cudaSuccess) return e;
    return launch_kernel(paged_merge_kernel<HD>, dim3(grid.x, HD / kMergeDims), dim3(kTQ), 0, st, a);
}

}  // namespace

cudaError_t launch_paged_e4m3_attention_tc(PagedAttnArgs a, const CUtensorMap& map, int hd, int sms, cudaStream_t st) {
    CUtensorMap tm_q, tm_out;
    const cudaError_t e = paged_tc_args(a, hd, 1, sms, &tm_q, &tm_out);
    if (e != cudaSuccess) return e;
    return hd == 128 ? launch<128>(a, tm_q, tm_out, map, st) : launch<64>(a, tm_q, tm_out, map, st);
}

}  // namespace odb
