// dK and dV of packed sequences, in launches of few tiles dQ too, bf16, 65 to 128 columns: the workgroups of bwd_ring_tiles.h, each on one 128-row tile of one
// sequence (packed.h).
#include "bwd_ring_tiles.h"
#include "packed.h"

namespace sa {

namespace {

template <int DP, bool PART>
__global__ void __launch_bounds__(256, 1)
packed_dkdv_ring_kernel(PackedArgs p) {
    __shared__ __attribute__((aligned(1024))) char lds[SLOTS * SLOT<DP>];
    __shared__ __attribute__((aligned(16))) float stat[STAT_FLOATS];
    int n_tiles, rank, head;
    if (!enter_sequence<false, BM>(p, (int)blockIdx.x, p.H_kv, n_tiles, rank, head)) return;
    dkdv_ring<DP, PART, false, true>(p, n_tiles, rank * p.H_kv + head, lds, stat);
}

// Both kinds of workgroups in a launch, delta formed by one in front of it.
template <int DP, bool PART>
__global__ void __launch_bounds__(256, 1)
packed_both_ring_kernel(PackedArgs p, PlacedKinds kinds) {
    __shared__ __attribute__((aligned(1024))) char lds[SLOTS * SLOT<DP>];
    __shared__ __attribute__((aligned(16))) float stat[STAT_FLOATS];
    int linear = (int)blockIdx.x, n_tiles, rank, head;
    const int keys = __builtin_amdgcn_readfirstlane(owns_keys(kinds, linear));
    linear = __builtin_amdgcn_readfirstlane(linear);        // (both kept scalar)
    if (keys) {
        if (!enter_sequence<false, BM>(p, linear, p.H_kv, n_tiles, rank, head)) return;
        dkdv_ring<DP, PART, false, true>(p, n_tiles, rank * p.H_kv + head, lds, stat);
    } else {
        if (!enter_sequence<true, BM>(p, linear, p.H, n_tiles, rank, head)) return;
        dq_ring<DP, PART, true>(p, n_tiles, rank * p.H + head, lds);
    }
}

template <int DP, bool PART>
hipError_t launch(const PackedArgs& p, bool both, hipStream_t st) {
    if (both) {
        const int n_dkdv = p.n_ranks * p.H_kv, n_dq = p.n_ranks * p.H;
        const PlacedKinds kinds = placed_kinds(p, n_dkdv, n_dq, packed_ratio(p));
        hipLaunchKernelGGL((packed_both_ring_kernel<DP, PART>), dim3((unsigned)(n_dkdv + n_dq)), dim3(256), 0, st, p, kinds);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((packed_dkdv_ring_kernel<DP, PART>), dim3((unsigned)p.n_ranks * p.H_kv), dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_bwd_ring(const PackedArgs& p, bool both, hipStream_t st) {
    const bool part = p.d % 8 != 0;
    if (p.d <= 112) return part ? launch<112, true>(p, both, st) : launch<112, false>(p, both, st);
    return part ? launch<128, true>(p, both, st) : launch<128, false>(p, both, st);
}

}  // namespace sa
