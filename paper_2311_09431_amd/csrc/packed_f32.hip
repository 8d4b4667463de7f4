// Causal attention of packed sequences and its gradient, fp32 storage, on the fp32 matrix cores: the ring step's workgroups
// (f32_tiles.h), each on one 128-row tile of one sequence (packed.h).
#include "f32_tiles.h"

namespace sa {

namespace {

// workgroups 0 .. n_dkdv - 1 own keys, the others queries; at 256 columns each kind in a launch of its own
template <int DP, bool KEYS, bool QUERIES>
__global__ void __launch_bounds__(64 * WAVES, DP > 64 ? 1 : 2)
packed_bwd_f32_kernel(PackedArgs p, int n_dkdv) {
    __shared__ __attribute__((aligned(16))) float lds[tile_floats<1, DP>()];
    __shared__ float stats[KEYS ? 2 * tile_rows(1) : 1];
    __shared__ uint32_t masks[WAVES];
    const int heads = p.H_kv * (DP > 128 ? 2 : 1);
    int n_tiles, rank, head;
    if (KEYS && (!QUERIES || (int)blockIdx.x < n_dkdv)) {
        if (!enter_sequence<false>(p, (int)blockIdx.x, heads, n_tiles, rank, head)) return;
        bwd_dkdv<float, DP, 1, true>(p, n_tiles, rank * heads + head, lds, stats, masks);
    } else if (QUERIES) {
        if (!enter_sequence<true>(p, (int)blockIdx.x - (KEYS ? n_dkdv : 0), p.H, n_tiles, rank, head)) return;
        bwd_dq<float, DP, 1, true>(p, n_tiles, rank * p.H + head, lds, masks);
    }
}

template <int DP>
hipError_t fwd(const PackedArgs& p, hipStream_t st) {
    hipLaunchKernelGGL((fwd_f32_kernel<float, DP, 1, PackedArgs>), dim3((unsigned)p.n_ranks * p.H), dim3(64 * WAVES), 0, st, p, 0);
    return hipGetLastError();
}
template <int DP>
hipError_t bwd(const PackedArgs& p, hipStream_t st) {
    const unsigned n_dkdv = (unsigned)p.n_ranks * p.H_kv * (DP > 128 ? 2 : 1), n_dq = (unsigned)p.n_ranks * p.H;
    const dim3 block(64 * WAVES);
    if constexpr (DP <= 128) {
        hipLaunchKernelGGL((packed_bwd_f32_kernel<DP, true, true>), dim3(n_dkdv + n_dq), block, 0, st, p, (int)n_dkdv);
    } else {
        hipLaunchKernelGGL((packed_bwd_f32_kernel<DP, false, true>), dim3(n_dq), block, 0, st, p, 0);
        if (hipError_t e = hipGetLastError()) return e;
        hipLaunchKernelGGL((packed_bwd_f32_kernel<DP, true, false>), dim3(n_dkdv), block, 0, st, p, (int)n_dkdv);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_f32(PackedArgs p, bool backward, hipStream_t st) {
    p.by_rank = true;
    if (p.d <= 32) return backward ? bwd<32>(p, st) : fwd<32>(p, st);
    if (p.d <= 64) return backward ? bwd<64>(p, st) : fwd<64>(p, st);
    if (p.d <= 128) return backward ? bwd<128>(p, st) : fwd<128>(p, st);
    return backward ? bwd<256>(p, st) : fwd<256>(p, st);
}

}  // namespace sa
