// Norm of every query and key head, rotation by the row's position, keys and values into their slots of the pool: one pass.
//
//   y = x / sqrt(mean(x^2) + eps) * gain          over the head's HD values (q and k; null gain: y = x)
//   (y_a, y_b) -> magnitude * (y_a cos t - y_b sin t, y_b cos t + y_a sin t)    for the pairs of the first `rot` values
//
// in fp32, rounded once.  The angle of pair i is position x frequency; the frequencies come as 64-bit fractions of a turn
// per position, so that the integer product's upper half is the angle with its whole turns already gone: exact to 2^-32 of
// a turn (fp32 position x frequency is off by 4e-3 rad at position 131072) up to positions of some 10^7, from where on the rounding of
// the frequencies themselves, which are computed as doubles, is more than that.
//
// A unit is a row and up to 8 heads of one kind (q, k or v); HD / 8 threads take it, each the same place of all its heads: two chunks
// of four values that hold four whole pairs (values 4 l .. and rot / 2 + 4 l .., or 8 l .. of interleaved pairs; behind `rot` the
// next ones, which pass), so that no value changes threads but for the sum of squares, the sines are computed once and all
// heads' loads are in flight together.  Arithmetic on pairs of floats (f32x2).
// Every value is read and written once: HBM is the bound.  25568 rows of 32 + 2 x 8 heads of 128 (628 MB) take 106 us = 5.9 TB/s, with
// half of each head turned 111.  Whole heads have an instance of their own (ALL): in the one that asks every lane they take 112.
// With the kinds mixed in a unit of four heads and single floats it was the issue slots: 241 instructions a head and warp, 164 us; in
// blocks of 128 threads and more 118 us.  8 or 512 rows are the call's cost on the host, 13 us with three slices of a projection.
#include "paged_rows.cuh"

namespace odb {

namespace {

constexpr int kThreads = 64;
constexpr int kHeads = kStoreHeads;                           // heads of a unit

template <int HD, bool INTER, bool ALL>
__global__ void __launch_bounds__(kThreads, 14) paged_store_kernel(const PagedStoreArgs p) {
    constexpr int kLanes = HD / 8;
    pdl_launch_dependents();
    pdl_wait();
    store_unit<HD, INTER, ALL>(p, static_cast<long long>(blockIdx.x) * (kThreads / kLanes) + threadIdx.x / kLanes);
}

template <int HD, bool INTER, bool ALL>
cudaError_t launch(const PagedStoreArgs& a, cudaStream_t st) {
    const long long units = static_cast<long long>(a.rows) * ((a.H + kHeads - 1) / kHeads + 2 * ((a.KV + kHeads - 1) / kHeads)), per = kThreads / (HD / 8);
    return launch_kernel(paged_store_kernel<HD, INTER, ALL>, dim3(static_cast<unsigned>((units + per - 1) / per)), dim3(kThreads), 0, st, a);
}

}  // namespace

cudaError_t launch_paged_store(const PagedStoreArgs& a, cudaStream_t st) {
    const bool all = a.rot == a.HD;
    if (a.interleaved) {
        if (a.HD == 128) return all ? launch<128, true, true>(a, st) : launch<128, true, false>(a, st);
        return all ? launch<64, true, true>(a, st) : launch<64, true, false>(a, st);
    }
    if (a.HD == 128) return all ? launch<128, false, true>(a, st) : launch<128, false, false>(a, st);
    return all ? launch<64, false, true>(a, st) : launch<64, false, false>(a, st);
}

}  // namespace odb
