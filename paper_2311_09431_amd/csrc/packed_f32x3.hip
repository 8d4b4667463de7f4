// Causal attention of packed sequences and its gradient, fp32 storage in three bf16 terms: the ring step's workgroups of 128 rows and
// more (f32x3_tiles.h), each on one tile of one sequence (packed.h).  Bound by the longest walk or, in launches that fill the chip, the
// splitting of rows into terms: 16 sequences of up to 1000 rows, 16 heads on 8, forward, d 128, 215 us, 120 TFLOP/s of allowed pairs (32-row
// workgroups of three-term products 421, the fp32 instruction 543), d 64 112, 116 (209, 223).  At 128 columns registers are spilled: 36 in the backward (148
// bytes of scratch a lane), 11 (44 bytes) in the forward of 256 rows.
#include "f32x3_tiles.h"

namespace sa {

namespace {

// workgroups 0 .. n_dkdv - 1 own keys, the others queries
template <int DP>
__global__ void __launch_bounds__(64 * 2 * GROUPS, 2)
packed_bwd_f32x3_kernel(PackedArgs p, int n_dkdv) {
    constexpr int ROWS = 32 * GROUPS;
    __shared__ __attribute__((aligned(1024))) char lds[2 * BUFFER];
    __shared__ __attribute__((aligned(1024))) char tiles[EXCHANGED];
    __shared__ float stats[2 * 3 * TILE];          // [buffer][LSE hi | LSE lo | delta][row]
    __shared__ uint32_t masks[6 * GROUPS];
    int n_tiles, rank, head;
    if ((int)blockIdx.x < n_dkdv) {
        if (!enter_sequence<false, ROWS>(p, (int)blockIdx.x, p.H_kv, n_tiles, rank, head)) return;
        bwd_dkdv<DP, true>(p, n_tiles, rank * p.H_kv + head, lds, tiles, stats, masks);
    } else {
        if (!enter_sequence<true, ROWS>(p, (int)blockIdx.x - n_dkdv, p.H, n_tiles, rank, head)) return;
        bwd_dq<DP, true>(p, n_tiles, rank * p.H + head, lds, tiles, masks);
    }
}

template <int DP, int WAVES>
hipError_t run_fwd(PackedArgs p, hipStream_t st) {
    p.n_ranks = (int)most_tiles(p, 32 * WAVES);
    hipLaunchKernelGGL((fwd_f32x3_kernel<DP, WAVES, PackedArgs>), dim3((unsigned)p.n_ranks * p.H), dim3(64 * WAVES), 0, st, p, 0);
    return hipGetLastError();
}
template <int DP>
hipError_t run(PackedArgs p, bool backward, hipStream_t st) {
    p.n_ranks = (int)most_tiles(p, 32 * GROUPS);
    if (!backward) return (int64_t)p.n_ranks * p.H >= 512 ? run_fwd<DP, 8>(p, st) : run_fwd<DP, 4>(p, st);
    const unsigned n_dkdv = (unsigned)p.n_ranks * p.H_kv, n_dq = (unsigned)p.n_ranks * p.H;
    hipLaunchKernelGGL((packed_bwd_f32x3_kernel<DP>), dim3(n_dkdv + n_dq), dim3(64 * 2 * GROUPS), 0, st, p, (int)n_dkdv);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_f32x3(PackedArgs p, bool backward, hipStream_t st) {
    return p.d <= 64 ? run<64>(p, backward, st) : run<128>(p, backward, st);
}

}  // namespace sa
