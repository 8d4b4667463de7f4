// dK and dV of packed sequences, bf16, 65 to 128 columns: the workgroups of bwd_ring_tiles.h, each on one 128-row tile of one
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

template <int DP, bool PART>
hipError_t launch(const PackedArgs& p, hipStream_t st) {
    hipLaunchKernelGGL((packed_dkdv_ring_kernel<DP, PART>), dim3((unsigned)p.n_ranks * p.H_kv), dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_bwd_ring(const PackedArgs& p, hipStream_t st) {
    const bool part = p.d % 8 != 0;
    if (p.d <= 112) return part ? launch<112, true>(p, st) : launch<112, false>(p, st);
    return part ? launch<128, true>(p, st) : launch<128, false>(p, st);
}

}  // namespace sa
