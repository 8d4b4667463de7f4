// Ring-step kernels on the fp32 matrix cores (f32_tiles.h) and which launches take them.
#include "f32_tiles.h"

namespace sa {

namespace {

// Both in one launch (KEYS and QUERIES): workgroups 0 .. n_dkdv - 1 own keys, the others queries.
// They share nothing but the inputs; where neither fills the chip they run beside each other, and
// a step is one launch less.  At 256 columns each by itself, with a register budget of its own (fp32: queries spill 149 registers and
// keys 24 where two wavefronts share a walk, 21 and 26 where not).  Packed sequences take both in one launch there too (packed_f32.hip).
template <typename T, int DP, int SPLIT, bool KEYS, bool QUERIES>
__global__ void __launch_bounds__(64 * WAVES, DP > 64 ? 1 : 2)
bwd_f32_kernel(StepArgs p, int n_tiles, int n_dkdv) {
    __shared__ __attribute__((aligned(16))) float lds[tile_floats<SPLIT, DP>()];
    __shared__ float stats[KEYS ? 2 * tile_rows(SPLIT) : 1];        // LSE | delta of a tile's queries
    __shared__ uint32_t masks[WAVES];
    if (KEYS && (!QUERIES || (int)blockIdx.x < n_dkdv))
        bwd_dkdv<T, DP, SPLIT>(p, n_tiles, (int)blockIdx.x, lds, stats, masks);
    else if (QUERIES) bwd_dq<T, DP, SPLIT>(p, n_tiles, (int)blockIdx.x - (KEYS ? n_dkdv : 0), lds, masks);
}

// ----------------------------------------------------------------- dispatch
template <typename T, int DP, int SPLIT>
hipError_t run_fwd(const StepArgs& a, hipStream_t st) {
    const int rows = 32 * (WAVES / SPLIT), n_tiles = (a.c + rows - 1) / rows;
    hipLaunchKernelGGL((fwd_f32_kernel<T, DP, SPLIT>), dim3((unsigned)n_tiles * a.n_q * a.B * a.H), dim3(64 * WAVES),
                       0, st, a, n_tiles);
    return hipGetLastError();
}
template <typename T, int DP, int SPLIT>
hipError_t run_bwd(const StepArgs& a, hipStream_t st) {
    const int rows = 32 * (WAVES / SPLIT), n_tiles = (a.c + rows - 1) / rows;
    const int n_dkdv = n_tiles * a.n_kv * a.B * a.H_kv * (DP > 128 ? 2 : 1), n_dq = n_tiles * a.n_q * a.B * a.H;
    const dim3 block(64 * WAVES);
    if constexpr (DP <= 128) {
        hipLaunchKernelGGL((bwd_f32_kernel<T, DP, SPLIT, true, true>), dim3((unsigned)(n_dkdv + n_dq)), block, 0, st, a,
                           n_tiles, n_dkdv);
    } else {
        hipLaunchKernelGGL((bwd_f32_kernel<T, DP, SPLIT, false, true>), dim3((unsigned)n_dq), block, 0, st, a, n_tiles,
                           0);
        if (hipError_t e = hipGetLastError()) return e;
        hipLaunchKernelGGL((bwd_f32_kernel<T, DP, SPLIT, true, false>), dim3((unsigned)n_dkdv), block, 0, st, a,
                           n_tiles, n_dkdv);
    }
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t run(const StepArgs& a, bool backward, hipStream_t st) {
    constexpr int MOST = DP > 128 ? 2 : 4;          // what 160 KiB of LDS hold
    const bool split = few_row_tiles(a, backward);
    if (backward) return split ? run_bwd<T, DP, MOST>(a, st) : run_bwd<T, DP, 1>(a, st);
    return split ? run_fwd<T, DP, MOST>(a, st) : run_fwd<T, DP, 1>(a, st);
}
hipError_t run(const StepArgs& a, int dtype, bool backward, hipStream_t st) {
    if (dtype == SA_F32) return run<float, 256>(a, backward, st);
    if (a.d <= 32) return run<__hip_bfloat16, 32>(a, backward, st);
    if (a.d <= 64) return run<__hip_bfloat16, 64>(a, backward, st);
    if (a.d <= 128) return run<__hip_bfloat16, 128>(a, backward, st);
    return run<__hip_bfloat16, 256>(a, backward, st);
}
// fp32 launches of few row tiles
template <int DP>
hipError_t run_few(const StepArgs& a, bool backward, hipStream_t st) {
    return backward ? run_bwd<float, DP, 4>(a, st) : run_fwd<float, DP, 4>(a, st);
}
hipError_t launch_f32_storage(const StepArgs& a, bool backward, hipStream_t st) {
    const F32Route route = f32_route(a, backward);
    if (route == F32_SPLIT) return launch_f32x3_split(a, backward, st);
    if (route != F32_INSTRUCTION) return launch_f32x3(a, backward, route == F32_TERMS_ALONE, st);
    return a.d <= 32 ? run_few<32>(a, backward, st) : a.d <= 64 ? run_few<64>(a, backward, st) : run_few<128>(a, backward, st);
}

}  // namespace

hipError_t launch_fwd_f32(const StepArgs& a, int dtype, hipStream_t st) {
    if (few_rows_wanted(a, dtype, false)) return launch_few_rows(a, dtype, false, st);
    if (dtype == SA_F32 && a.d <= 128) return launch_f32_storage(a, false, st);
    if (short_exact_wanted(a, dtype, false)) return launch_short_exact(a, false, st);
    return run(a, dtype, false, st);
}
hipError_t launch_bwd_f32(const StepArgs& a, int dtype, hipStream_t st) {
    if (few_rows_wanted(a, dtype, true)) return launch_few_rows(a, dtype, true, st);
    if (dtype == SA_F32 && a.d <= 128) return launch_f32_storage(a, true, st);
    if (short_exact_wanted(a, dtype, true)) return launch_short_exact(a, true, st);
    return run(a, dtype, true, st);
}

}  // namespace sa
