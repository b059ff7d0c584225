// What the stores of the paged cache have in common: a thread's part of a head, its norm and its rotation (formulas: paged_store.cu).
#pragma once

#include "paged.cuh"

namespace odb {

namespace {

constexpr int kStoreHeads = 8;                                // heads of a unit

typedef unsigned long long f2;                                // two floats
__device__ __forceinline__ f2 pair(float a, float b) {
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 floats(f2 x) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}
__device__ __forceinline__ f2 mul(f2 a, f2 b) {
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 fma(f2 a, f2 b, f2 c) {
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float low(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float high(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf16x2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Sine and cosine of two angles of t / 2^32 turns.  The nearest quarter turn is taken off in integers, which leaves |x| <= pi / 4;
// there the Taylor polynomials up to x^9 and x^8 end within 2e-9 and 3e-8.  (A quarter of the instructions of the library's call,
// which for eight heads a thread were 40 % of all.)
__device__ __forceinline__ void sincos_turns(uint32_t t0, uint32_t t1, float (&sn)[2], float (&cs)[2]) {
    const uint32_t q0 = t0 + 0x20000000u, q1 = t1 + 0x20000000u;   // the quarter in the two highest bits
    constexpr float kUnit = 1.4629180792671596e-9f;                // 2 pi / 2^32
    const f2 x = mul(pair(static_cast<float>(static_cast<int>(t0 - (q0 & 0xc0000000u))), static_cast<float>(static_cast<int>(t1 - (q1 & 0xc0000000u)))),
                     pair(kUnit, kUnit));
    auto both = [](float v) { return pair(v, v); };
    const f2 z = mul(x, x);
    const f2 s = fma(mul(x, z), fma(z, fma(z, fma(z, both(1.f / 362880.f), both(-1.f / 5040.f)), both(1.f / 120.f)), both(-1.f / 6.f)), x);
    const f2 c = fma(z, fma(z, fma(z, fma(z, both(1.f / 40320.f), both(-1.f / 720.f)), both(1.f / 24.f)), both(-0.5f)), both(1.f));
    const float2 sf = floats(s), cf = floats(c);
    auto place = [](uint32_t q, float s0, float c0, float& so, float& co) {   // quarters 0 .. 3: (s, c), (c, -s), (-s, -c), (-c, s)
        const bool swap = q & 0x40000000u;
        const float a = swap ? c0 : s0, b = swap ? s0 : c0;
        so = __uint_as_float(__float_as_uint(a) ^ (q & 0x80000000u));
        co = __uint_as_float(__float_as_uint(b) ^ ((q + 0x40000000u) & 0x80000000u));
    };
    place(q0, sf.x, cf.x, sn[0], cs[0]);
    place(q1, sf.y, cf.y, sn[1], cs[1]);
}

// Four pairs (a_j, b_j) of a thread from its two chunks' words, and back.
template <bool INTER>
__device__ __forceinline__ void widen(uint2 va, uint2 vb, f2 (&a)[2], f2 (&b)[2]) {
    if (INTER) {
        a[0] = pair(low(va.x), low(va.y)); b[0] = pair(high(va.x), high(va.y));
        a[1] = pair(low(vb.x), low(vb.y)); b[1] = pair(high(vb.x), high(vb.y));
    } else {
        a[0] = pair(low(va.x), high(va.x)); a[1] = pair(low(va.y), high(va.y));
        b[0] = pair(low(vb.x), high(vb.x)); b[1] = pair(low(vb.y), high(vb.y));
    }
}
template <bool INTER>
__device__ __forceinline__ void narrow(const f2 (&a)[2], const f2 (&b)[2], uint2& va, uint2& vb) {
    const float2 a0 = floats(a[0]), a1 = floats(a[1]), b0 = floats(b[0]), b1 = floats(b[1]);
    if (INTER) {
        va = make_uint2(bf16x2(a0.x, b0.x), bf16x2(a0.y, b0.y));
        vb = make_uint2(bf16x2(a1.x, b1.x), bf16x2(a1.y, b1.y));
    } else {
        va = make_uint2(bf16x2(a0.x, a0.y), bf16x2(a1.x, a1.y));
        vb = make_uint2(bf16x2(b0.x, b0.y), bf16x2(b1.x, b1.y));
    }
}

// A thread's four pairs of every head: cosines and sines of the row's angles, and the gains.
template <bool INTER>
struct StoreTurn {
    f2 c[2], s[2], ms[2], ga[2], gb[2];

    __device__ __forceinline__ void angles(const PagedStoreArgs& p, int pos, int l, bool turned) {
        c[0] = c[1] = s[0] = s[1] = ms[0] = ms[1] = pair(0.f, 0.f);
        if (!turned) return;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const ulonglong2 f = *reinterpret_cast<const ulonglong2*>(p.turns + 4 * l + 2 * j);
            const long long at = pos;
            float sn[2], cs[2];
            sincos_turns(static_cast<uint32_t>(f.x * static_cast<unsigned long long>(at) >> 32), static_cast<uint32_t>(f.y * static_cast<unsigned long long>(at) >> 32), sn, cs);
            c[j] = pair(cs[0] * p.magnitude, cs[1] * p.magnitude);
            s[j] = pair(sn[0] * p.magnitude, sn[1] * p.magnitude);
            ms[j] = pair(-sn[0] * p.magnitude, -sn[1] * p.magnitude);
        }
    }
    __device__ __forceinline__ void gains(const float* gain, int ca, int cb) {
        const float4 u = *reinterpret_cast<const float4*>(gain + ca), v = *reinterpret_cast<const float4*>(gain + cb);
        if (INTER) {
            ga[0] = pair(u.x, u.z); gb[0] = pair(u.y, u.w);
            ga[1] = pair(v.x, v.z); gb[1] = pair(v.y, v.w);
        } else {
            ga[0] = pair(u.x, u.y); ga[1] = pair(u.z, u.w);
            gb[0] = pair(v.x, v.y); gb[1] = pair(v.z, v.w);
        }
    }
    template <int HD>
    __device__ __forceinline__ void norm(f2 (&a)[2], f2 (&b)[2], float eps, unsigned mask) const {
        const float2 sq = floats(fma(a[0], a[0], fma(a[1], a[1], fma(b[0], b[0], mul(b[1], b[1])))));
        float ss = sq.x + sq.y;
#pragma unroll
        for (int d = HD / 16; d >= 1; d >>= 1) ss += __shfl_xor_sync(mask, ss, d);
        const float r = rsqrtf(ss * (1.0f / HD) + eps);             // within 2 ulp
        const f2 rr = pair(r, r);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            a[j] = mul(mul(a[j], rr), ga[j]);
            b[j] = mul(mul(b[j], rr), gb[j]);
        }
    }
    __device__ __forceinline__ void turn(f2 (&a)[2], f2 (&b)[2], bool turned) const {
#pragma unroll
        for (int j = 0; j < 2; ++j) {                           // values behind rot pass: by cosine 1 and sine 0 an infinity would make NaN of its partner
            const f2 u = fma(a[j], c[j], mul(b[j], ms[j])), v = fma(b[j], c[j], mul(a[j], s[j]));
            a[j] = turned ? u : a[j];
            b[j] = turned ? v : b[j];
        }
    }
};

// A unit: a row and up to kStoreHeads heads of one kind, by HD / 8 threads of a warp that lie together; called by whole warps.
template <int HD, bool INTER, bool ALL>
__device__ __forceinline__ void store_unit(const PagedStoreArgs& p, long long unit) {
    constexpr int kLanes = HD / 8, kHeads = kStoreHeads;      // threads of a unit
    const int q_units = (p.H + kHeads - 1) / kHeads, k_units = (p.KV + kHeads - 1) / kHeads, units = q_units + 2 * k_units;
    const int l = threadIdx.x % kLanes;
    const bool any = unit < static_cast<long long>(p.rows) * units;
    const int row = p.rows * units < 0x7fffffff ? static_cast<int>(static_cast<unsigned>(unit) / static_cast<unsigned>(units)) : static_cast<int>(unit / units);
    const int part = static_cast<int>(unit - static_cast<long long>(row) * units);
    const bool is_q = part < q_units, is_v = part >= q_units + k_units;
    const float* gain = is_q ? p.q_gain : p.k_gain;
    // the lanes that will form sums of squares: those of a warp's other units (values, heads without a gain, none) are not waited for
    const unsigned mask = __ballot_sync(0xffffffffu, any && !is_v && gain);
    if (!any) return;
    const int h0 = (is_q ? part : is_v ? part - q_units - k_units : part - q_units) * kHeads, n = min(kHeads, (is_q ? p.H : p.KV) - h0);
    const int pos = p.row_pos[row], slot = p.row_slot[row] | pos >> 31;   // without a position no slot
    const int page = slot >> p.page_shift, off = slot & ((1 << p.page_shift) - 1);
    const bool stored = is_q ? pos >= 0 : slot >= 0 && page < p.n_pages;
    // from head to head: HD values in q, a page's rows in the pool
    const size_t step = is_q ? HD : static_cast<size_t>(HD) << p.page_shift;
    __nv_bfloat16* dst = is_q ? p.q_out + row * p.out_stride + h0 * HD
                              : (is_v ? p.v_pool : p.k_pool) + (((static_cast<size_t>(page) * p.KV + h0) << p.page_shift) + off) * HD;

    if (is_v) {
        const __nv_bfloat16* src = p.v + row * p.v_stride + h0 * HD + 4 * l;
        uint2 v[kHeads][2];
#pragma unroll
        for (int i = 0; i < kHeads; ++i)
            if (i < n) {
                v[i][0] = *reinterpret_cast<const uint2*>(src + i * HD);
                v[i][1] = *reinterpret_cast<const uint2*>(src + i * HD + HD / 2);
            }
        if (!stored) return;
#pragma unroll
        for (int i = 0; i < kHeads; ++i)
            if (i < n) {
                *reinterpret_cast<uint2*>(dst + i * step + 4 * l) = v[i][0];
                *reinterpret_cast<uint2*>(dst + i * step + 4 * l + HD / 2) = v[i][1];
            }
        return;
    }
    const bool turned = ALL || l < p.rot / 8;
    const int ca = turned && !INTER ? 4 * l : 8 * l, cb = turned && !INTER ? (ALL ? HD : p.rot) / 2 + 4 * l : 8 * l + 4;
    const __nv_bfloat16* src = (is_q ? p.q + row * p.q_stride : p.k + row * p.k_stride) + h0 * HD;
    uint2 va[kHeads], vb[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        va[i] = vb[i] = make_uint2(0u, 0u);
        if (i < n) {
            va[i] = *reinterpret_cast<const uint2*>(src + i * HD + ca);
            vb[i] = *reinterpret_cast<const uint2*>(src + i * HD + cb);
        }
    }
    StoreTurn<INTER> t;
    t.angles(p, pos, l, turned);
    if (gain) t.gains(gain, ca, cb);
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        f2 a[2], b[2];
        widen<INTER>(va[i], vb[i], a, b);
        if (gain) t.template norm<HD>(a, b, p.eps, mask);
        t.turn(a, b, turned);
        if (i < n && stored) {
            uint2 x, y;
            narrow<INTER>(a, b, x, y);
            *reinterpret_cast<uint2*>(dst + i * step + ca) = x;
            *reinterpret_cast<uint2*>(dst + i * step + cb) = y;
        }
    }
}

}  // namespace

}  // namespace odb
