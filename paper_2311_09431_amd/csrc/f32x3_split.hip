// Ring-step kernels for fp32 operands in workgroups of 32 rows (f32x3_split_tiles.h): their launches.
#include "f32x3_split_tiles.h"

namespace sa {

namespace {

// Both in one launch (they share nothing but the inputs).
template <int DP>
__global__ void __launch_bounds__(64 * WAVES_OF<DP>, WAVES_OF<DP> / 4)
bwd_f32x3_split_kernel(StepArgs p, int n_tiles, BothKinds kinds) {
    __shared__ __attribute__((aligned(1024))) char lds[STAGES_BYTES<DP> + 2 * OWN_BYTES<DP>];
    __shared__ __attribute__((aligned(1024))) char stats[WAVES_OF<DP> * STAT_BYTES];
    __shared__ __attribute__((aligned(16))) uint32_t masks[4 * WAVES_OF<DP>];          // (RowsToRedo)
    int linear = (int)blockIdx.x;
    if (owns_keys(kinds, linear)) bwd_dkdv<DP>(p, n_tiles, linear, lds, stats, masks);
    else bwd_dq<DP>(p, n_tiles, linear, lds, masks);
}

template <int DP>
hipError_t run(const StepArgs& a, bool backward, hipStream_t st) {
    const int n_tiles = (a.c + OWN - 1) / OWN;
    const int n_dkdv = n_tiles * a.n_kv * a.B * a.H_kv, n_dq = n_tiles * a.n_q * a.B * a.H;
    const dim3 block(64 * WAVES_OF<DP>);
    if (backward)
        hipLaunchKernelGGL((bwd_f32x3_split_kernel<DP>), dim3((unsigned)(n_dkdv + n_dq)), block, 0, st, a, n_tiles,
                           both_kinds(a, n_dkdv, n_dq, 1.25));
    else hipLaunchKernelGGL((fwd_f32x3_split_kernel<DP>), dim3((unsigned)n_dq), block, 0, st, a, n_tiles);
    return hipGetLastError();
}

}  // namespace

bool f32x3_split_supported(const StepArgs& a, bool backward) {
    // both sides' rows come through descriptors with 32-bit byte offsets, up to 32 rows behind the block's last sub-tile
    const int64_t widest = a.stride_s > a.kv_stride_s ? a.stride_s : a.kv_stride_s;
    if (((int64_t)(a.c + 31) / 32 * 32 + OWN) * 4 * widest + 4 * a.d + 4096 >= (int64_t(1) << 31)) return false;
    // HIP takes fewer than 2^32 threads a launch.  (One beyond it, in parts, would be faster here than in 128-row
    // workgroups; nothing near such sizes has been measured.)
    const int64_t tiles = (a.c + OWN - 1) / OWN, owners = (int64_t)a.n_q * a.B * a.H + (backward ? (int64_t)a.n_kv * a.B * a.H_kv : 0);
    return a.d <= TD && tiles * owners * 64 * (a.d <= 64 ? WAVES_OF<64> : WAVES_OF<128>) < (int64_t(1) << 32);
}

hipError_t launch_f32x3_split(const StepArgs& a, bool backward, hipStream_t st) {
    if (a.d <= 32) return run<32>(a, backward, st);
    return a.d <= 64 ? run<64>(a, backward, st) : run<128>(a, backward, st);
}

}  // namespace sa
