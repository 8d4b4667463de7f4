// Causal attention of packed sequences and its gradient, fp32 storage in three bf16 terms: the ring step's workgroups of 32 rows
// (f32x3_split_tiles.h), each on one tile of one sequence (packed.h).  Where there are few, whose walks are what takes time: 5 sequences of up to
// 777 rows, 16 heads on 8, d 64, backward 91 us (128-row workgroups 135, the fp32 instruction 127).
#include "f32x3_split_tiles.h"

namespace sa {

namespace {

// workgroups 0 .. n_dkdv - 1 own keys, the others queries
template <int DP>
__global__ void __launch_bounds__(64 * WAVES_OF<DP>, WAVES_OF<DP> / 4)
packed_bwd_f32x3_split_kernel(PackedArgs p, int n_dkdv) {
    __shared__ __attribute__((aligned(1024))) char lds[STAGES_BYTES<DP> + 2 * OWN_BYTES<DP>];
    __shared__ __attribute__((aligned(1024))) char stats[WAVES_OF<DP> * STAT_BYTES];
    __shared__ __attribute__((aligned(16))) uint32_t masks[4 * WAVES_OF<DP>];          // (RowsToRedo)
    int n_tiles, rank, head;
    if ((int)blockIdx.x < n_dkdv) {
        if (!enter_sequence<false, OWN>(p, (int)blockIdx.x, p.H_kv, n_tiles, rank, head)) return;
        bwd_dkdv<DP, true>(p, n_tiles, rank * p.H_kv + head, lds, stats, masks);
    } else {
        if (!enter_sequence<true, OWN>(p, (int)blockIdx.x - n_dkdv, p.H, n_tiles, rank, head)) return;
        bwd_dq<DP, true>(p, n_tiles, rank * p.H + head, lds, masks);
    }
}

template <int DP>
hipError_t run(PackedArgs p, bool backward, hipStream_t st) {
    p.n_ranks = (int)most_tiles(p, OWN);
    const unsigned n_dkdv = (unsigned)p.n_ranks * p.H_kv, n_dq = (unsigned)p.n_ranks * p.H;
    const dim3 block(64 * WAVES_OF<DP>);
    if (backward) hipLaunchKernelGGL((packed_bwd_f32x3_split_kernel<DP>), dim3(n_dkdv + n_dq), block, 0, st, p, (int)n_dkdv);
    else hipLaunchKernelGGL((fwd_f32x3_split_kernel<DP, PackedArgs>), dim3(n_dq), block, 0, st, p, 0);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_f32x3_split(PackedArgs p, bool backward, hipStream_t st) {
    if (p.d <= 32) return run<32>(p, backward, st);
    return p.d <= 64 ? run<64>(p, backward, st) : run<128>(p, backward, st);
}

}  // namespace sa
