// Norm of every query and key head, rotation by the row's position, keys and values into their slots of the pool: one pass.
//
//   y = x / sqrt(mean(x^2) + eps) * gain          over the head's HD values (q and k; null gain: y = x)
//   (y_a, y_b) -> magnitude * (y_a cos t - y_b sin t, y_b cos t + y_a sin t)    for the pairs of the first `rot` values
//
// in fp32, rounded once.  The angle of pair i is position x frequency; the frequencies come as 64-bit fractions of a turn
// per position, so that the integer product's upper half is the angle with its whole turns already gone: exact to 2^-32 of
// a turn at every position (fp32 position x frequency is off by 4e-3 rad at position 131072).
//
// HD / 8 threads take a head, each two chunks of four values that hold four whole pairs (values 4 l .. and rot / 2 + 4 l ..,
// or 8 l .. of interleaved pairs; behind `rot` the next ones), so no value changes threads but for the sum of squares.  A
// thread takes the same place of HG heads: one set of sines for all of them, and HG pairs of loads in flight.  Bound by
// HBM: every value read and written once.
#include "paged.cuh"

namespace odb {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float4 widen(uint2 v) {
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
}
__device__ __forceinline__ uint2 narrow(float4 v) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
    const float x = a * c - b * s;
    b = b * c + a * s;
    a = x;
}

template <int HD, int HG>
__global__ void __launch_bounds__(kThreads) paged_store_kernel(const PagedStoreArgs p) {
    constexpr int kLanes = HD / 8;                            // threads of a head
    pdl_launch_dependents();
    pdl_wait();
    const int n_heads = p.H + 2 * p.KV, groups = (n_heads + HG - 1) / HG;
    const int l = threadIdx.x % kLanes;
    // chunk places
    const int rot_lanes = p.rot / 8;
    const bool turned = l < rot_lanes;
    const int ca = turned ? (p.interleaved ? 8 * l : 4 * l) : 8 * l;
    const int cb = turned ? (p.interleaved ? 8 * l + 4 : p.rot / 2 + 4 * l) : 8 * l + 4;

    const long long units = static_cast<long long>(p.rows) * groups;
    const long long unit = static_cast<long long>(blockIdx.x) * (kThreads / kLanes) + threadIdx.x / kLanes;
    const unsigned mask = __ballot_sync(0xffffffffu, unit < units);   // a head's lanes are in one warp
    if (unit >= units) return;
    const int row = static_cast<int>(unit / groups), grp = static_cast<int>(unit - static_cast<long long>(row) * groups);
    const int pos = p.row_pos[row], slot = p.row_slot[row];

    uint2 va[HG], vb[HG];
#pragma unroll
    for (int i = 0; i < HG; ++i) {
        const int h = grp + i * groups;
        va[i] = vb[i] = make_uint2(0u, 0u);
        if (h < n_heads) {
            const __nv_bfloat16* src = h < p.H ? p.q + row * p.q_stride + h * HD
                                     : h < p.H + p.KV ? p.k + row * p.k_stride + (h - p.H) * HD
                                                      : p.v + row * p.v_stride + (h - p.H - p.KV) * HD;
            va[i] = *reinterpret_cast<const uint2*>(src + ca);
            vb[i] = *reinterpret_cast<const uint2*>(src + cb);
        }
    }
    float c[4], s[4];
    if (turned) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned long long t = p.turns[4 * l + j] * static_cast<unsigned long long>(static_cast<long long>(pos));
            sincospif(static_cast<float>(static_cast<int>(t >> 32)) * 0x1p-31f, &s[j], &c[j]);
            s[j] *= p.magnitude;
            c[j] *= p.magnitude;
        }
    }
    const bool row_ok = pos >= 0, slot_ok = slot >= 0 && (slot >> p.page_shift) < p.n_pages;
    const int page = slot >> p.page_shift, off = slot & ((1 << p.page_shift) - 1);
#pragma unroll
    for (int i = 0; i < HG; ++i) {
        const int h = grp + i * groups;
        const bool have = h < n_heads, is_q = h < p.H, is_v = h >= p.H + p.KV;
        const float* gain = is_q ? p.q_gain : p.k_gain;
        float4 x = widen(va[i]), y = widen(vb[i]);
        if (p.q_gain || p.k_gain) {                           // uniform
            float ss = x.x * x.x + x.y * x.y + x.z * x.z + x.w * x.w + y.x * y.x + y.y * y.y + y.z * y.z + y.w * y.w;
#pragma unroll
            for (int d = kLanes / 2; d >= 1; d >>= 1) ss += __shfl_xor_sync(mask, ss, d);
            if (have && !is_v && gain) {
                const float r = 1.0f / sqrtf(ss * (1.0f / HD) + p.eps);
                const float4 ga = *reinterpret_cast<const float4*>(gain + ca), gb = *reinterpret_cast<const float4*>(gain + cb);
                x = make_float4(x.x * r * ga.x, x.y * r * ga.y, x.z * r * ga.z, x.w * r * ga.w);
                y = make_float4(y.x * r * gb.x, y.y * r * gb.y, y.z * r * gb.z, y.w * r * gb.w);
            }
        }
        if (!have) continue;
        if (turned && !is_v) {
            if (p.interleaved) {
                turn(x.x, x.y, c[0], s[0]);
                turn(x.z, x.w, c[1], s[1]);
                turn(y.x, y.y, c[2], s[2]);
                turn(y.z, y.w, c[3], s[3]);
            } else {
                turn(x.x, y.x, c[0], s[0]);
                turn(x.y, y.y, c[1], s[1]);
                turn(x.z, y.z, c[2], s[2]);
                turn(x.w, y.w, c[3], s[3]);
            }
        }
        __nv_bfloat16* dst;
        if (is_q) {
            if (!row_ok) continue;
            dst = p.q_out + row * p.out_stride + h * HD;
        } else {
            if (!slot_ok) continue;
            const int kh = is_v ? h - p.H - p.KV : h - p.H;
            dst = (is_v ? p.v_pool : p.k_pool) + (((static_cast<size_t>(page) * p.KV + kh) << p.page_shift) + off) * HD;
        }
        if (is_v) {
            *reinterpret_cast<uint2*>(dst + ca) = va[i];
            *reinterpret_cast<uint2*>(dst + cb) = vb[i];
        } else {
            *reinterpret_cast<uint2*>(dst + ca) = narrow(x);
            *reinterpret_cast<uint2*>(dst + cb) = narrow(y);
        }
    }
}

template <int HD, int HG>
cudaError_t launch(const PagedStoreArgs& a, cudaStream_t st) {
    const long long groups = (a.H + 2 * a.KV + HG - 1) / HG, units = a.rows * groups, per = kThreads / (HD / 8);
    return launch_kernel(paged_store_kernel<HD, HG>, dim3(static_cast<unsigned>((units + per - 1) / per)), dim3(kThreads), 0, st, a);
}

}  // namespace

cudaError_t launch_paged_store(const PagedStoreArgs& a, cudaStream_t st) {
    return a.HD == 128 ? launch<128, 4>(a, st) : launch<64, 4>(a, st);
}

}  // namespace odb
