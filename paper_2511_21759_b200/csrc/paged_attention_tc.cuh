// Attention of many packed rows on the tcgen05 tensor cores: what the kernels over pools of bf16 and of 8 bits have in common, which is all
// behind the K and V tiles in shared memory (formulas and figures: paged_attention_tc.cu).
#pragma once

#include "paged.cuh"

namespace odb {

namespace {

constexpr int kTQ = 128;   // packed rows of a Q tile (MMA M)
constexpr int kKT = 64;    // keys of a tile
constexpr int kItem = kPagedTcItem;
template <int HD> constexpr uint32_t kQBytes = kTQ * HD * 2;
template <int HD> constexpr uint32_t kTileBytes = kKT * HD * 2;             // K or V of a tile, as the products take it
template <int HD> constexpr int kBufs = HD == 128 ? 2 : 3;   // S / P buffers of a Q tile: 256 columns, of which O takes HD
constexpr uint32_t kCols = 256;
// kCodes: a tile that moves the shift has weights up to 2^kRoom, those behind it up to 2^(kRoom + kSlack), where f16 ends below 2^16, so that few
// are too small for f16.  The row's sum stands without it, over 2^kRoom: where V's scales are the smallest it is near the end of fp32.
constexpr float kSlack = 8.0f, kRoom = 7.0f;
constexpr uint32_t kPatch = 4096;                            // per softmax warp, in the Q tile: 32 rows x 128 bytes of output

// The launch's numbers and the maps of Q and of the outputs.
inline cudaError_t paged_tc_args(PagedAttnArgs& a, int hd, int q_tiles, int sms, CUtensorMap* tm_q, CUtensorMap* tm_out) {
    a.negate = a.scale_log2 < 0.f;                           // the softmax takes the largest score for the largest exponent
    a.scale_log2 = fabsf(a.scale_log2);
    a.tile_tokens = kTQ / a.G;
    a.tile_rows = q_tiles * a.tile_tokens * a.G;
    a.by_rows = PagedDiv::by(a.tile_rows);
    a.at_once = q_tiles == 1 ? 2 * sms : sms;
    a.by_once = PagedDiv::by(a.at_once);
    a.part_rows = q_tiles * kTQ;
    const cudaError_t e = make_group_tmap(tm_q, a.q, a.max_rows, a.q_stride, a.H, hd, a.G, a.tile_tokens);
    return e != cudaSuccess ? e : make_group_tmap(tm_out, a.out, a.max_rows, a.out_stride, a.H, hd, a.G, a.tile_tokens);
}

// Columns of tensor memory, by one warp; the successor is let go behind it.
__device__ __forceinline__ void paged_tc_alloc(uint32_t* base, uint32_t columns) {
    __syncwarp();
    tmem_alloc(base, columns);
}

// per Q tile 256 columns of TMEM: kBufs x 64 of S or P, then O
template <int HD>
__device__ __forceinline__ uint32_t paged_tc_o(uint32_t tmem, int g) { return tmem + g * kCols + kCols - HD; }

__device__ __forceinline__ void tma_box_3d(uint32_t dst, const CUtensorMap* tmap, uint64_t* bar, int c0, int c1, int c2) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}
__device__ __forceinline__ void tma_store_box_3d(const CUtensorMap* tmap, uint32_t src, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(reinterpret_cast<uint64_t>(tmap)), "r"(src),
                 "r"(c0), "r"(c1), "r"(c2)
                 : "memory");
}
__device__ __forceinline__ void tma_prefetch_map(const CUtensorMap* tmap) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(tmap)) : "memory");
}
// The products with descriptors as their low words (address, and what stands below bit 32) and the high word that all tiles here
// share: one 32-bit addition from product to product.
__device__ __forceinline__ void umma_lo(uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "mov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n\t}" ::"r"(tmem_d),
        "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void umma_ts_lo(uint32_t tmem_d, uint32_t tmem_a, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\t"
        "mov.b64 b, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}" ::"r"(tmem_d),
        "r"(tmem_a), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void commit_at(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// whether the phase has completed for all lanes of a converged warp
__device__ __forceinline__ bool try_all(uint32_t bar, uint32_t parity) {
    uint32_t x;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "vote.sync.all.pred p, p, 0xffffffff;\n\t"
        "selp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(x)
        : "r"(bar), "r"(parity)
        : "memory");
    return x != 0;
}

// 64 TMEM columns asked for, and (with whatever else was asked for) there
__device__ __forceinline__ void tmem_ask64(uint32_t taddr, uint32_t (&v)[64]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
        "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
        "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
          "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
          "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31]), "=r"(v[32]),
          "=r"(v[33]), "=r"(v[34]), "=r"(v[35]), "=r"(v[36]), "=r"(v[37]), "=r"(v[38]), "=r"(v[39]), "=r"(v[40]),
          "=r"(v[41]), "=r"(v[42]), "=r"(v[43]), "=r"(v[44]), "=r"(v[45]), "=r"(v[46]), "=r"(v[47]), "=r"(v[48]),
          "=r"(v[49]), "=r"(v[50]), "=r"(v[51]), "=r"(v[52]), "=r"(v[53]), "=r"(v[54]), "=r"(v[55]), "=r"(v[56]),
          "=r"(v[57]), "=r"(v[58]), "=r"(v[59]), "=r"(v[60]), "=r"(v[61]), "=r"(v[62]), "=r"(v[63])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_got64(uint32_t (&v)[64]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int j = 0; j < 64; ++j) asm volatile("" : "+r"(v[j]));       // no use of them moves in front of the wait
}
__device__ __forceinline__ void tmem_ld16_now(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr)
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
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Keys from lo on and below hi are seen by all of the query rows tok .. tok + n - 1 of a request.
struct SeenByAll {
    int lo, hi;
    __device__ __forceinline__ SeenByAll(const PagedAttnArgs& a, const PagedSeq& q, int tok, int n)
        : lo(static_cast<int>(max(-1ll, static_cast<long long>(q.first) + tok + n - 1 - a.left))),
          hi(static_cast<int>(max(0ll, min(static_cast<long long>(q.len), static_cast<long long>(q.first) + tok + a.right + 1)))) {}
    // the tile from k0 on
    __device__ __forceinline__ bool tile(const PagedAttnArgs& a, int k0) const { return k0 + kKT <= hi && (k0 >= lo || k0 + kKT <= a.sinks); }
};

// Turns of the two Q tiles' softmax warps gw: Q tile 0 first.
__device__ __forceinline__ void turn_begin(int g, int gw) { asm volatile("bar.sync %0, 64;" ::"r"(2 + 4 * g + gw) : "memory"); }
__device__ __forceinline__ void turn_end(int g, int gw) { asm volatile("bar.arrive %0, 64;" ::"r"(2 + 4 * (g ^ 1) + gw) : "memory"); }

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
        "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}

// The MMAs of Q tile g: the whole warp walks and waits, one lane issues.
// T: HD, QT; NQ Q buffers, KS and VS places of the K and V rings, and the barriers' struct; kCodes: the operands are f16 (paged_e4m3_attention_tc.cu).
template <class T>
__device__ __forceinline__ void paged_tc_mma(const PagedAttnArgs& a, const PagedStart& start, typename T::Shared* sh, const uint8_t* sQ, const uint8_t* sK,
                                             const uint8_t* sV, uint32_t tmem, int g) {
    constexpr int HD = T::HD, QT = T::QT, NQ = T::NQ, KS = T::KS, VS = T::VS, kB = kBufs<HD>, kFirst = kB - 1;
    constexpr uint32_t kT = kTileBytes<HD>;
    volatile int* cta_abort = &sh->abort;
    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait_bounded(bar, parity, cta_abort, a.status); };
    // S of tile i + kFirst, P V of tile i by turns; with two Q buffers into the next item, so that its first scores are ready when
    // the softmax warps have written the one in front of it.  (P of an item's first tile says that O has been read.)
    PagedWalk<kKT, kItem> ws(a, start), wv(a, start);
    constexpr int kItems = T::kCodes ? 1 : NQ;               // kCodes: the next item's Q becomes f16 when this one has been written
    constexpr uint32_t kTypes = T::kCodes ? ~((7u << 7) | (7u << 10)) : ~0u;               // f16: both types zero
    const uint32_t idesc_s = (instr_desc(kTQ, kKT, 0) & kTypes) | (a.negate ? 1u << 13 : 0u);   // bit 13: the product's A is taken with its sign turned
    constexpr uint32_t idesc_o = instr_desc(kTQ, HD, 1) & kTypes;
    const uint32_t cols = tmem + g * kCols;
    const uint32_t q_lo = static_cast<uint32_t>(desc_k_major(smem_u32(sQ) + g * kQBytes<HD>)), k_lo = static_cast<uint32_t>(desc_k_major(smem_u32(sK))),
                   v_lo = static_cast<uint32_t>(desc_mn_major(smem_u32(sV), kKT * 128));
    const uint32_t hi = static_cast<uint32_t>(desc_k_major(0) >> 32);    // desc_mn_major's too
    const uint32_t bars = smem_u32(sh);
    auto bar_of = [&](const uint64_t* first, uint32_t i) { return bars + static_cast<uint32_t>(reinterpret_cast<const char*>(first) - reinterpret_cast<const char*>(sh)) + i * 8; };
    // Places and phases are counted along: what a tile takes here is what bounds the whole where products and exponentials overlap.
    bool ok = true, have_s = true;
    int s_ahead = 0, i_ahead = 0;                            // S issued beyond P V, items beyond P V's that the next S is
    int ts = ws.t0;
    uint32_t k_slot = 0, k_ph = 0, s_buf = 0, q_buf = 0, q_ph = 0;
    uint32_t v_slot = 0, v_ph = 0, p_buf = 0, p_ph = 0;
    uint32_t pv_bar = 1, pv_ph = 1;                          // of the last P V: barrier and phase
    auto all_wait = [&](uint64_t* first, uint32_t i, uint32_t parity) {
        if (!try_all(bar_of(first, i), parity)) ok = __all_sync(0xffffffffu, wait(first + i, parity));
    };
    auto issue_s = [&](bool first_pv) {
        const uint32_t q = q_lo + q_buf * (QT * kQBytes<HD> >> 4), k = k_lo + k_slot * (kT >> 4), d = cols + s_buf * kKT;
        const uint32_t full = bar_of(sh->s_full[g], s_buf), empty = bar_of(sh->k_empty, k_slot);
        if (ts == ws.t0) all_wait(T::q_ready(sh, g), q_buf, q_ph);
        if (ok) all_wait(sh->k_full, k_slot, k_ph);
        // the last P V has been done, and with it the one that read P in this S's place
        if (ok && !first_pv) all_wait(sh->pv_done[g], pv_bar, pv_ph);
        if (!ok) return;
        tc_fence_after();
        if (paged_elect()) {
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) {
                const uint32_t atom = kk >> 2, within = (kk & 3) * 32;
                umma_lo(d, q + ((atom * (kTQ * 128) + within) >> 4), k + ((atom * (kKT * 128) + within) >> 4), hi, idesc_s, kk > 0 ? 1u : 0u);
            }
            commit_at(full);
            commit_at(empty);
        }
        __syncwarp();
        ++s_ahead;
        if (++k_slot == KS) { k_slot = 0; k_ph ^= 1u; }
        if (++s_buf == kB) s_buf = 0;
        if (++ts == ws.t1) {
            have_s = ws.next();
            ts = ws.t0;
            ++i_ahead;
            if (++q_buf == NQ) { q_buf = 0; q_ph ^= 1u; }
        }
    };
    bool first_pv = true;
    do {
        const int n = wv.t1 - wv.t0;
        for (int t = 0; t < n && ok; ++t) {
            while (ok && have_s && s_ahead <= kFirst && i_ahead < kItems) issue_s(first_pv);
            const uint32_t v = v_lo + v_slot * (kT >> 4), o = paged_tc_o<HD>(tmem, g), pa = cols + p_buf * kKT;
            pv_bar ^= 1u;
            if (pv_bar == 0) pv_ph ^= 1u;
            const uint32_t done_bar = bar_of(sh->pv_done[g], pv_bar), empty = bar_of(sh->v_empty, v_slot), o_bar = bar_of(sh->o_full, g);
            if (ok) all_wait(sh->v_full, v_slot, v_ph);
            if (ok) all_wait(sh->p_full[g], p_buf, p_ph);
            if (!ok) break;
            tc_fence_after();
            const uint32_t keep = t > 0 ? 1u : __shfl_sync(0xffffffffu, *const_cast<volatile int*>(&sh->keep_o[g]), 0);
            if (paged_elect()) {
#pragma unroll
                for (int kk = 0; kk < kKT / 16; ++kk) umma_ts_lo(o, pa + kk * 8, v + kk * (2048 >> 4), hi, idesc_o, kk > 0 ? 1u : keep);
                commit_at(done_bar);
                commit_at(empty);
                if (t + 1 == n) commit_at(o_bar);
            }
            __syncwarp();
            first_pv = false;
            --s_ahead;
            if (++v_slot == VS) { v_slot = 0; v_ph ^= 1u; }
            if (++p_buf == kB) { p_buf = 0; p_ph ^= 1u; }
        }
        --i_ahead;
    } while (ok && wv.next());
}

// The softmax of a Q tile: thread r of Q tile g = packed row r = TMEM lane r.
template <class T>
__device__ __forceinline__ void paged_tc_softmax(const PagedAttnArgs& a, const PagedStart& start, const CUtensorMap& tm_out, typename T::Shared* sh, uint8_t* sQ,
                                                 uint32_t tmem) {
    constexpr int HD = T::HD, QT = T::QT, NQ = T::NQ, VS = T::VS, kB = kBufs<HD>, kAtoms = HD / 64;
    volatile int* cta_abort = &sh->abort;
    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait_bounded(bar, parity, cta_abort, a.status); };
    PagedWalk<kKT, kItem> w(a, start);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), g = warp >> 2, gw = warp & 3, r = tid & 127;
    const uint32_t lane_base = static_cast<uint32_t>(gw * 32) << 16;   // this warp's TMEM lanes
    const uint32_t s_base = tmem + g * kCols + lane_base, o_base = paged_tc_o<HD>(tmem, g) + lane_base;
    const int rows_g = a.tile_tokens * a.G;                  // packed rows of a Q tile
    float scale = a.scale_log2;                              // of the row's scores
    bool ok = true;
    uint32_t item = 0, done = 0;                             // key tiles of the items before
    bool storing = false;                                    // the last item's output is on its way from the Q tile's place
    auto q_free = [&]() {                                    // it has left that place
        if (!storing) return;
        if (lane == 0) {
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            mbar_arrive(&sh->item_done[(item - 1) % NQ]);
        }
        __syncwarp();
        storing = false;
    };
    if (QT == 2 && g == 1) turn_end(1, gw);
    do {
        const int n = w.t1 - w.t0;
        const int tok0 = (w.rt * QT + g) * a.tile_tokens;    // the Q tile's first query row
        const int pos = w.q.first + tok0 + a.by_group(min(r, rows_g - 1));
        const SeenByAll by_tile(a, w.q, tok0, a.tile_tokens), by_item(a, w.q, w.rt * QT * a.tile_tokens, QT * a.tile_tokens);
        const int left = min(rows_g, (w.q.n - tok0) * a.G);          // rows of the Q tile (may be negative); others hold anything
        const bool mine = r < left;
        if constexpr (T::kCodes) scale = a.scale_log2 * T::template own_q<kTQ>(sh, sQ, item, r, ok, wait);
        float M_row = -INFINITY, l_row = 0.f, G_row = 0.f;           // the row's shift, M (kCodes: M + G), and its sum (kCodes: over 2^kRoom)
        uint32_t sv[64];                                             // the row's scores of the tile at hand
        auto ask = [&](int t) {                                      // for those of tile t, once they are there
            const uint32_t gt = done + t, b = gt % kB;
            if (!try_all(smem_u32(&sh->s_full[g][b]), (gt / kB) & 1u)) ok = __all_sync(0xffffffffu, wait(&sh->s_full[g][b], (gt / kB) & 1u)) && ok;
            tc_fence_after();
            tmem_ask64(s_base + b * kKT, sv);
        };
        // One tile.  care: some row of the item does not see all of its keys.
        auto tile = [&](bool care, int t, int k0) {
            const uint32_t gt = done + t, b = gt % kB;
            const uint32_t ts = s_base + b * kKT;
            tmem_got64(sv);
            unsigned long long mask = ~0ull;                         // the keys of the tile that the row sees
            if (care && !by_tile.tile(a, k0)) {
                auto below = [](long long x) { return x >= 64 ? ~0ull : x <= 0 ? 0ull : (1ull << x) - 1ull; };
                mask = below(min(static_cast<long long>(w.q.len), static_cast<long long>(pos) + a.right + 1) - k0) &
                       (~below(static_cast<long long>(pos) - a.left - k0) | below(static_cast<long long>(a.sinks) - k0));
#pragma unroll
                for (int j = 0; j < 64; ++j)
                    if (!((mask >> j) & 1ull)) sv[j] = 0xff800000u;
            }
            float mx[4];                                             // largest visible score of the tile, in four chains
            float mul[4], up[4], weight[4];                          // kCodes: of the tile's blocks: K's scale and the row's, log2 of V's, and 2^-kRoom / V's
            bool wide = false;                                       // V's scales lie far from 1: see the sum
            if constexpr (T::kCodes) {
                wide = T::scales(sh, gt, mul, up, weight);
#pragma unroll
                for (int c = 0; c < 4; ++c) mul[c] = fminf(fmaxf(mul[c] * scale, 0x1p-126f), 0x1.fffffep127f);   // not zero: masked scores stay what they are; finite: scores of zero do
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                mx[c] = __uint_as_float(sv[16 * c]);
#pragma unroll
                for (int j = 1; j < 15; j += 2) mx[c] = max3(mx[c], __uint_as_float(sv[16 * c + j]), __uint_as_float(sv[16 * c + j + 1]));
            }
            // Whether the shift has to move, for a tile that exceeds it by more than kSlack or holds the first visible key.
            // The exponentials take a score's exact product with the scale, the shift comes from the rounded one: from 2^22 on
            // they lie up to 0.25 and more apart, and the scores are rounded first (in products of their own, here and below).
            bool far, move;
            float M_new;
            if constexpr (T::kCodes) {
                float most = -INFINITY, exceeds = -INFINITY;
                const float M = M_row == -INFINITY ? 0.f : M_row;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    mx[c] = __fmul_rn(fmaxf(mx[c], __uint_as_float(sv[16 * c + 15])), mul[c]);
                    most = fmaxf(most, mx[c]);
                    exceeds = fmaxf(exceeds, mx[c] - M + up[c]);
                }
                const bool seen = mine && mask && most != -INFINITY;
                far = seen && fabsf(most) >= 0x1p22f;
                move = seen && (M_row == -INFINITY || exceeds > G_row + (kSlack + kRoom) || most > M_row + 60.f);
                M_new = fmaxf(M_row, ceilf(most));
            } else {
                float m0 = fmaxf(max3(mx[0], mx[1], __uint_as_float(sv[15])), max3(mx[2], mx[3], __uint_as_float(sv[31])));
                m0 = max3(m0, __uint_as_float(sv[47]), __uint_as_float(sv[63]));
                const float mt_log2 = mine && mask ? m0 * scale : -INFINITY;   // rows that are none turn nothing for the warp's others
                far = fabsf(mt_log2) >= 0x1p22f && mt_log2 != -INFINITY;
                move = mt_log2 > M_row + kSlack;                     // also the first visible key (M_row = -inf)
                M_new = ceilf(mt_log2);
            }
            uint64_t mult2[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) mult2[c] = T::kCodes ? pack2f(mul[c], mul[c]) : pack2f(scale, scale);
            float factor = 1.0f;                                     // what O and the row sum so far are multiplied by
            bool rescale = false, rounded = false;                   // rounded: the scores stand as x, kCodes: as x - M
            if (__builtin_expect(__any_sync(0xffffffffu, move || far), 0)) {
                if (move) {
                    float G_new = 0.f;
                    if constexpr (T::kCodes) {
                        G_new = mx[0] - M_new + up[0];
#pragma unroll
                        for (int c = 1; c < 4; ++c) G_new = fmaxf(G_new, mx[c] - M_new + up[c]);
                        G_new = ceilf(G_new) - kRoom;
                        if (M_row != -INFINITY) G_new = fmaxf(G_new, M_row - M_new + G_row);   // M + G never falls
                    }
                    if (M_row != -INFINITY) factor = exp2f(M_row - M_new + (G_row - G_new));   // an exact power of two
                    M_row = M_new;
                    G_row = G_new;
                }
                rescale = __any_sync(0xffffffffu, factor != 1.0f);
                rounded = __any_sync(0xffffffffu, far);
                if (rounded) {
#pragma unroll
                    for (int j = 0; j < 64; ++j)
                        sv[j] = __float_as_uint(T::kCodes ? __fmul_rn(__uint_as_float(sv[j]), mul[j / 16]) - (M_row == -INFINITY ? 0.f : M_row) : __uint_as_float(sv[j]) * scale);
#pragma unroll
                    for (int c = 0; c < 4; ++c) mult2[c] = pack2f(1.0f, 1.0f);
                }
                if (rescale && t > 0) {                              // warp-uniform; rows that keep their shift multiply by 1
                    // P V(t - 1) has been added to O.  The parity is not ambiguous: S(t) was issued behind P V(t - kB), so P V(t - 3),
                    // which the same barrier counts, has completed; P V(t + 1) cannot have, it is behind this P.
                    ok = __all_sync(0xffffffffu, wait(&sh->pv_done[g][(gt - 1) & 1u], ((gt - 1) >> 1) & 1u)) && ok;
                    tc_fence_after();
                    l_row *= factor;
#pragma unroll 1
                    for (int c = 0; c < HD / 16; ++c) {
                        uint32_t v[16];
                        tmem_ld16_now(o_base + c * 16, v);
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * factor);
                        tmem_st16(o_base + c * 16, v);
                    }
                }
            }
            const float m_log2 = M_row == -INFINITY ? 0.f : M_row;   // a row that has seen no key: every P is 0
            uint64_t shift2[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float shift = T::kCodes ? up[c] - G_row - (rounded ? 0.f : m_log2) : -m_log2;
                shift2[c] = pack2f(shift, shift);
            }
            uint64_t sum[4] = {0ull, 0ull, 0ull, 0ull};
            // The two softmax warps of a scheduler take turns at the exponentials: left alone they fall into step, share the
            // special-function unit for twice as long and leave it idle together for the rest of the tile.
            if (QT == 2) turn_begin(g, gw);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t pb[16];                                     // P of 32 keys as pairs
#pragma unroll
                for (int u = 0; u < 16; ++u) {
                    const int c = 2 * half + u / 8, chain = T::kCodes ? c : u & 3;
                    const float2 x = unpack2f(fma2(pack2u(sv[32 * half + 2 * u], sv[32 * half + 2 * u + 1]), mult2[c], shift2[c]));
                    const float p0 = ex2_approx(x.x), p1 = ex2_approx(x.y);
                    sum[chain] = add2(sum[chain], pack2f(p0, p1));
                    pb[u] = T::kCodes ? paged_f16x2(p0, p1) : paged_bf16x2(p0, p1);
                }
                tmem_st16(ts + 16 * half, pb);
            }
            if (QT == 2) turn_end(g, gw);
            if constexpr (T::kCodes) {
                if (__builtin_expect(wide, 0)) {                                // weights that a scale lets vanish still count in the sum
                    float all = 0.f;
#pragma unroll
                    for (int j = 0; j < 64; ++j) all += ex2_approx(__uint_as_float(sv[j]) * unpack2f(mult2[j / 16]).x - (rounded ? 0.f : m_log2));
                    l_row += all * exp2f(-G_row - kRoom);
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const float2 s0 = unpack2f(sum[c]);
                        l_row += (s0.x + s0.y) * weight[c];
                    }
                }
            } else {
                const float2 s0 = unpack2f(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])));
                l_row += s0.x + s0.y;
            }
            if (care) {
                // The parity is not ambiguous: the tile before it in this slot was multiplied before S(t) was, the one behind it waits
                // for P V(t).
                const uint32_t slot = gt % VS;
                ok = __all_sync(0xffffffffu, wait(T::v_seen(sh, slot), (gt / VS) & 1u)) && ok;
                if (ok && T::odd(sh, slot)) {   // rare: values of V, from the pool, are added to O here
                    if (t > 0) ok = __all_sync(0xffffffffu, wait(&sh->pv_done[g][(gt - 1) & 1u], ((gt - 1) >> 1) & 1u)) && ok;
                    tc_fence_after();
                    tmem_wait_st();
                    if (t == 0) {
                        uint32_t z[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) z[j] = 0u;
#pragma unroll 1
                        for (int c = 0; c < HD / 16; ++c) tmem_st16(o_base + c * 16, z);
                        tmem_wait_st();
                    }
                    PagedPages pages;
#pragma unroll 1
                    for (int e = 0; e < kKT; ++e) {
                        const int key = k0 + e;
                        if (key >= w.k.hi || (key < w.k.lo && key >= a.sinks)) continue;
                        const int row = pages.template row<false>(a, w.q, w.seq, w.head, key, a.v_row0);
                        if (row >= a.pool_rows) continue;
                        const uint32_t p2 = tmem_ld1(ts + e / 2);
                        const float p = __uint_as_float(e & 1 ? p2 & 0xffff0000u : p2 << 16);
#pragma unroll 1
                        for (int d = 0; d < HD; ++d) {
                            const float v = T::odd_value(a, row, d);
                            if (v == 0.f) continue;                      // the same for all lanes
                            const float o = __uint_as_float(tmem_ld1(o_base + d));
                            tmem_st1(o_base + d, __float_as_uint((mask >> e) & 1ull ? o + p * v : o));
                        }
                    }
                    if (t == 0 && r == 0) sh->keep_o[g] = 1;
                }
            }
            // The next scores are asked for before P is waited for: one latency instead of two.  They depend on P of the tile before
            // this one only.
            if (t + 1 < n) ask(t + 1);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->p_full[g][b]);
        };
        if (r == 0) sh->keep_o[g] = 0;
        ask(0);
        for (int t = 0; t < n; ++t) {
            const int k0 = w.k.tile(w.t0 + t) << 6;
            tile(!by_item.tile(a, k0), t, k0);
            if (t == 0) q_free();
        }
        done += n;
        const float m_log2 = M_row == -INFINITY ? 0.f : M_row;      // the shift the row's sum and output carry
        ok = __all_sync(0xffffffffu, wait(&sh->o_full[g], item & 1u)) && ok;
        tc_fence_after();
        const int row_w = gw * 32;                                   // the warp's first row of the Q tile
        const uint32_t place = smem_u32(sQ) + ((item % NQ) * QT + g) * kQBytes<HD>;   // every MMA that reads this Q tile has completed
        const uint32_t patch = place + gw * kPatch;
        const bool final = w.whole();
        const float inv = l_row == 0.f ? 0.f : (T::kCodes ? exp2f(-kRoom) : 1.0f) / l_row;
        if (final && a.lse && row_w + lane < left) {
            const int idx = row_w + lane, i = a.by_group(idx);
            a.lse[static_cast<size_t>(w.q.row0 + tok0 + i) * a.H + w.head * a.G + idx - i * a.G] = paged_lse(m_log2, T::kCodes ? l_row * exp2f(G_row + kRoom) : l_row);   // the logarithm of a number near 1 where one key takes most
        }
        // 64 values of the row as pairs of bf16
        auto result = [&](int c, uint32_t (&x)[32]) {
            uint32_t v[64];
            tmem_ld64(o_base + c * 64, v);
#pragma unroll
            for (int j = 0; j < 32; ++j) x[j] = paged_bf16x2(__uint_as_float(v[2 * j]) * inv, __uint_as_float(v[2 * j + 1]) * inv);
            if (l_row == 0.f)                                        // no visible key: whatever O holds
#pragma unroll
                for (int j = 0; j < 32; ++j) x[j] = 0u;
        };
        if (final && left == rows_g) {                               // a Q tile without gaps: stored as it was loaded
#pragma unroll 1
            for (int c = 0; c < HD / 64; ++c) {
                uint32_t x[32];
                result(c, x);
#pragma unroll
                for (int ch = 0; ch < 8; ++ch)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(place + c * kTQ * 128 + r * 128 + ((ch ^ (r & 7)) << 4)), "r"(x[4 * ch]),
                                 "r"(x[4 * ch + 1]), "r"(x[4 * ch + 2]), "r"(x[4 * ch + 3])
                                 : "memory");
            }
            proxy_fence();
            asm volatile("bar.sync %0, 128;" ::"r"(10 + g) : "memory");
            if (gw == 0 && lane == 0) {
#pragma unroll
                for (int c = 0; c < kAtoms; ++c) tma_store_box_3d(&tm_out, place + c * kTQ * 128, 64 * c, w.head * a.G, w.q.row0 + tok0);
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
            storing = gw == 0;
        } else if (final) {
            int at[8];                                               // head of rows lane / 8, lane / 8 + 4 .. of the warp, from the Q tile's first
#pragma unroll
            for (int it = 0; it < 8; ++it) {
                const int idx = row_w + it * 4 + (lane >> 3), i = a.by_group(idx);
                at[it] = i * static_cast<int>(a.out_stride / 8) + (idx - i * a.G) * (HD / 8);
            }
            uint4* out = reinterpret_cast<uint4*>(a.out + static_cast<size_t>(w.q.row0 + tok0) * a.out_stride + w.head * a.G * HD);
#pragma unroll 1
            for (int c = 0; c < HD / 64; ++c) {
                uint32_t x[32];
                result(c, x);
                turn_rows(patch, lane, x, [&](int rr, int ch, const uint4& y) {
                    if (row_w + rr < left) out[at[rr >> 2] + c * 8 + ch] = y;
                });
            }
        } else {
            // [16 bytes of a row][row]: a warp's store is 512 bytes in one piece, and so is a load of the kernel that adds up
            const size_t part = paged_part(a, blockIdx.x, w.t0 == 0) + g * kTQ;
            float* po = a.part_o + part * HD + r * 4;
            const float unit = T::kCodes ? exp2f(G_row) : 1.f;       // a part's unit is 2^M
            if (r < left) *reinterpret_cast<float2*>(a.part_ml + (part + r) * 2) = make_float2(M_row, T::kCodes ? l_row * exp2f(G_row + kRoom) : l_row);
#pragma unroll 1
            for (int c = 0; c < HD / 32; ++c) {
                uint32_t v[32];
                tmem_ld32(o_base + c * 32, v);
                if (T::kCodes)
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * unit);
                if (l_row == 0.f)
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = 0u;
                if (r < left)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *reinterpret_cast<uint4*>(po + (c * 8 + j) * kTQ * 4) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            }
        }
        proxy_fence();                                               // the patches before the next Q
        tc_fence_before();
        __syncwarp();
        if (!storing && lane == 0) mbar_arrive(&sh->item_done[item % NQ]);
        if (!final && w.t0 == 0 && tid == 0) {
            PagedShared& d = a.shared[blockIdx.x];
            d.row0 = w.q.row0;
            d.head = w.head;
            d.first_idx = w.rt * a.tile_rows;
            d.last_cta = w.last_cta();
            d.rows = min(a.tile_rows, w.q.n * a.G - w.rt * a.tile_rows);
        }
        ++item;
        if (NQ == 1) q_free();                               // the next item's Q tile has no other place
    } while (w.next());
    if (gw == 0 && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    if (QT == 2 && g == 0) turn_begin(0, gw);                // the other's last word
}

// Adds up the parts of the items that several CTAs share, in the order of the CTAs with a running maximum: a thread takes kMergeDims
// values of a row, a block the rows of a Q tile, four parts in flight.  Most items have two or three parts: with eight in flight the
// registers leave half as many blocks on an SM (blocks of 32 rows 48.2 us, a prompt of 4096 rows 153.7; with four 46.4 and 150.3; with
// two 45.9 and 149.3, but twice the latency of items of many parts).
constexpr int kMergeDims = 8, kMergeParts = 4;
template <int HD>
__global__ void __launch_bounds__(kTQ, 8) paged_merge_kernel(const PagedAttnArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    const PagedShared d = a.shared[blockIdx.x];
    const int g = blockIdx.y / (HD / kMergeDims), dim0 = blockIdx.y % (HD / kMergeDims) * kMergeDims, r = threadIdx.x;
    const int rows_g = a.tile_tokens * a.G, at = g * rows_g + r;
    if (r >= rows_g || at >= d.rows) return;
    float M = -INFINITY, L = 0.f, acc[kMergeDims];
#pragma unroll
    for (int j = 0; j < kMergeDims; ++j) acc[j] = 0.f;
    for (int c = blockIdx.x; c <= d.last_cta; c += kMergeParts) {
        float2 ml[kMergeParts];
        float4 x[kMergeParts][kMergeDims / 4];
#pragma unroll
        for (int u = 0; u < kMergeParts; ++u) {
            if (c + u > d.last_cta) break;
            const size_t part = paged_part(a, c + u, c + u == static_cast<int>(blockIdx.x)) + g * kTQ;
            ml[u] = __ldcg(reinterpret_cast<const float2*>(a.part_ml + (part + r) * 2));
#pragma unroll
            for (int j = 0; j < kMergeDims / 4; ++j) x[u][j] = __ldcg(reinterpret_cast<const float4*>(a.part_o + part * HD + ((dim0 / 4 + j) * kTQ + r) * 4));
        }
#pragma unroll
        for (int u = 0; u < kMergeParts; ++u) {
            if (c + u > d.last_cta) break;
            const float top = fmaxf(M, ml[u].x), f = paged_weight(M, top), e = paged_weight(ml[u].x, top);
            M = top;
            L = L * f + ml[u].y * e;
#pragma unroll
            for (int j = 0; j < kMergeDims / 4; ++j) {
                acc[4 * j] = acc[4 * j] * f + x[u][j].x * e;
                acc[4 * j + 1] = acc[4 * j + 1] * f + x[u][j].y * e;
                acc[4 * j + 2] = acc[4 * j + 2] * f + x[u][j].z * e;
                acc[4 * j + 3] = acc[4 * j + 3] * f + x[u][j].w * e;
            }
        }
    }
    const int idx = d.first_idx + at, i = a.by_group(idx), h = d.head * a.G + idx - i * a.G;
    const size_t row = static_cast<size_t>(d.row0 + i);
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    uint32_t o[kMergeDims / 2];
#pragma unroll
    for (int j = 0; j < kMergeDims / 2; ++j) o[j] = paged_bf16x2(acc[2 * j] * inv, acc[2 * j + 1] * inv);
    static_assert(kMergeDims == 8, "a store of 16 bytes");
    *reinterpret_cast<uint4*>(a.out + row * a.out_stride + h * HD + dim0) = make_uint4(o[0], o[1], o[2], o[3]);
    if (a.lse && dim0 == 0) a.lse[row * a.H + h] = paged_lse(M, L);
}

}  // namespace

}  // namespace odb
