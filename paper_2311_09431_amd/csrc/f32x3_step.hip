// Ring-step kernels for fp32 operands on the bf16 matrix cores (f32x3_tiles.h): their launches.
#include "f32x3_tiles.h"

namespace sa {

namespace {

template <int DP, int WAVES>
hipError_t run_fwd(const StepArgs& a, hipStream_t st) {
    const int rows = 32 * WAVES, n_tiles = (a.c + rows - 1) / rows;
    hipLaunchKernelGGL((fwd_f32x3_kernel<DP, WAVES>), dim3((unsigned)n_tiles * a.n_q * a.B * a.H), dim3(64 * WAVES), 0, st,
                       a, n_tiles);
    return hipGetLastError();
}
template <int DP>
hipError_t run_alone(const StepArgs& a, hipStream_t st) {
    const int rows = 32 * ALONE, n_tiles = (a.c + rows - 1) / rows;
    const int n_dkdv = n_tiles * a.n_kv * a.B * a.H_kv, n_dq = n_tiles * a.n_q * a.B * a.H;
    hipLaunchKernelGGL((bwd_f32x3_alone_kernel<DP>), dim3((unsigned)(n_dkdv + n_dq)), dim3(64 * ALONE), 0, st, a, n_tiles,
                       n_dkdv);
    return hipGetLastError();
}
template <int DP>
hipError_t run(const StepArgs& a, bool backward, hipStream_t st) {
    const int rows = 32 * GROUPS, n_tiles = (a.c + rows - 1) / rows;
    if (!backward) return (int64_t)n_tiles * a.n_q * a.B * a.H >= 512 ? run_fwd<DP, 8>(a, st) : run_fwd<DP, 4>(a, st);
    const int n_dkdv = n_tiles * a.n_kv * a.B * a.H_kv, n_dq = n_tiles * a.n_q * a.B * a.H;
    // one device's queries against more than two shards (d 64: 3 of 2048 tokens, 8 heads, 617 -> 501 us, 4 of 512, 32
    // heads, 215 -> 156; two of 512, 32 heads, d 128, 176 -> 201)
    const bool keys_first = 2 * (int64_t)a.n_q * (a.H / a.H_kv) >= a.n_kv;
    hipLaunchKernelGGL((bwd_f32x3_kernel<DP>), dim3((unsigned)(n_dkdv + n_dq)), dim3(64 * 2 * GROUPS), 0, st, a, n_tiles,
                       keys_first ? n_dkdv : n_dq, keys_first);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_f32x3(const StepArgs& a, bool backward, bool alone, hipStream_t st) {
    if (alone) return run_alone<128>(a, st);
    return a.d <= 64 ? run<64>(a, backward, st) : run<128>(a, backward, st);
}

}  // namespace sa
