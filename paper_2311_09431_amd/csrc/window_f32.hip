// Attention with a window (window.h) and its gradient, fp32 storage, on the fp32 matrix cores (f32_tiles.h).
#include "f32_tiles.h"

namespace sa {

namespace {

// workgroups 0 .. n_dkdv - 1 own keys, the others queries
template <int DP, int SPLIT>
__global__ void __launch_bounds__(64 * WAVES, DP > 64 ? 1 : 2)
window_bwd_f32_kernel(WindowArgs p, int n_dkdv) {
    constexpr int ROWS = 32 * WAVES / SPLIT;
    __shared__ __attribute__((aligned(16))) float lds[tile_floats<SPLIT, DP>()];
    __shared__ float stats[2 * tile_rows(SPLIT)];                   // LSE | delta of a tile's queries
    __shared__ uint32_t masks[WAVES];
    const int heads = p.H_kv * (DP > 128 ? 2 : 1);
    int n_tiles, rank, head;
    if ((int)blockIdx.x < n_dkdv) {
        if (!enter_sequence<false, ROWS>(p, (int)blockIdx.x, heads, n_tiles, rank, head)) return;
        bwd_dkdv<float, DP, SPLIT, true, WindowArgs>(p, n_tiles, rank * heads + head, lds, stats, masks);
    } else {
        if (!enter_sequence<true, ROWS>(p, (int)blockIdx.x - n_dkdv, p.H, n_tiles, rank, head)) return;
        bwd_dq<float, DP, SPLIT, true, WindowArgs>(p, n_tiles, rank * p.H + head, lds, masks);
    }
}

template <int DP, int SPLIT>
hipError_t run(WindowArgs p, bool backward, hipStream_t st) {
    p.n_ranks = (int)most_tiles(p, 32 * WAVES / SPLIT);
    const unsigned n_dkdv = (unsigned)p.n_ranks * p.H_kv * (DP > 128 ? 2 : 1), n_dq = (unsigned)p.n_ranks * p.H;
    if (backward) hipLaunchKernelGGL((window_bwd_f32_kernel<DP, SPLIT>), dim3(n_dkdv + n_dq), dim3(64 * WAVES), 0, st, p, (int)n_dkdv);
    else hipLaunchKernelGGL((fwd_f32_kernel<float, DP, SPLIT, WindowArgs>), dim3(n_dq), dim3(64 * WAVES), 0, st, p, 0);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_window_f32(WindowArgs p, bool backward, hipStream_t st) {
    if (backward)
        if (hipError_t e = launch_packed_delta(p, SA_F32, st)) return e;
    p.by_rank = true;
    if (p.d > 128) return run<256, 2>(p, backward, st);
    if (p.d <= 32) return run<32, 4>(p, backward, st);
    return run<128, 4>(p, backward, st);
}

}  // namespace sa
