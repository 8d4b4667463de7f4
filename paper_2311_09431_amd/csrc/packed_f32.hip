// Causal attention of packed sequences and its gradient, fp32 storage: which kernels play a launch, and those on the fp32 matrix
// cores, the ring step's workgroups (f32_tiles.h), each on one tile of one sequence (packed.h).
//
// Up to 128 columns three kinds of kernels compete, as for a ring step, by the times that are put together there (f32_route.hip): the longest walk is
// that of a sequence of max_len rows, the load that of as many rows in sequences a quarter of the way from the mean to the longest (the lengths
// themselves are on the device).  Over 428 launches of 1 to 64 sequences of up to 32 to 4096 rows, d 64 and 128, forward and backward, what is picked
// takes 0.03 to 0.6 % more than the best kind; with one length for both, halfway, 0.6 to 1.3 %: 5 of up to 777 rows, 16 heads on 4, d 64, forward
// 53 : 43 us, 8 of up to 2000, 4 heads, backward 166 : 148, 5 of up to 777, 32 on 8, d 128, backward 506 : 373.
// Sequences of one 32-row tile leave the wavefronts that share a walk without one: never those kernels, and up to 64 columns the fp32
// instruction in launches of any size.  64 of up to 32 rows, 16 heads, d 32, forward 11 us on the fp32 instruction, 23 there, whole pass 53, 81; d
// 128, in terms 43, 60, 152, 256.
#include <math.h>

#include <algorithm>

#include "f32_tiles.h"

namespace sa {

namespace {

// workgroups 0 .. n_dkdv - 1 own keys, the others queries.  In a launch each at 256 columns, whole training pass, us, together : apart: 4 sequences
// of up to 1084 rows, 2 heads on 1, 776 : 1055, 16 heads 1705 : 1795, 3 of up to 500, 4 heads, 253 : 392, 8 of up to 1000, 32 on 8, 3232 : 3648.
// (There it spills 182 registers, 528 bytes of scratch a lane, with two wavefronts to a walk and 52, 116 bytes, with one.)
template <int DP, int SPLIT>
__global__ void __launch_bounds__(64 * WAVES, DP > 64 ? 1 : 2)
packed_bwd_f32_kernel(PackedArgs p, int n_dkdv) {
    constexpr int ROWS = 32 * WAVES / SPLIT;
    __shared__ __attribute__((aligned(16))) float lds[tile_floats<SPLIT, DP>()];
    __shared__ float stats[2 * tile_rows(SPLIT)];                   // LSE | delta of a tile's queries
    __shared__ uint32_t masks[WAVES];
    const int heads = p.H_kv * (DP > 128 ? 2 : 1);
    int n_tiles, rank, head;
    if ((int)blockIdx.x < n_dkdv) {
        if (!enter_sequence<false, ROWS>(p, (int)blockIdx.x, heads, n_tiles, rank, head)) return;
        bwd_dkdv<float, DP, SPLIT, true>(p, n_tiles, rank * heads + head, lds, stats, masks);
    } else {
        if (!enter_sequence<true, ROWS>(p, (int)blockIdx.x - n_dkdv, p.H, n_tiles, rank, head)) return;
        bwd_dq<float, DP, SPLIT, true>(p, n_tiles, rank * p.H + head, lds, masks);
    }
}

template <int DP, int SPLIT>
hipError_t run_fwd(PackedArgs p, hipStream_t st) {
    p.n_ranks = (int)most_tiles(p, 32 * WAVES / SPLIT);
    hipLaunchKernelGGL((fwd_f32_kernel<float, DP, SPLIT, PackedArgs>), dim3((unsigned)p.n_ranks * p.H), dim3(64 * WAVES), 0, st, p, 0);
    return hipGetLastError();
}
template <int DP, int SPLIT>
hipError_t run(PackedArgs p, bool backward, hipStream_t st) {
    if (!backward) return run_fwd<DP, SPLIT>(p, st);
    p.n_ranks = (int)most_tiles(p, 32 * WAVES / SPLIT);
    const unsigned n_dkdv = (unsigned)p.n_ranks * p.H_kv * (DP > 128 ? 2 : 1), n_dq = (unsigned)p.n_ranks * p.H;
    hipLaunchKernelGGL((packed_bwd_f32_kernel<DP, SPLIT>), dim3(n_dkdv + n_dq), dim3(64 * WAVES), 0, st, p, (int)n_dkdv);
    return hipGetLastError();
}

// a launch like p's of sequences of one length; blocks: how many of those
StepArgs like_equal_ones(const PackedArgs& p, double& blocks) {
    const int64_t mean = std::min((int64_t)p.max_len, ((int64_t)p.rows + p.n_seq - 1) / p.n_seq);
    StepArgs like = p;
    like.c = (int)((3 * mean + p.max_len + 2) / 4);
    blocks = std::max(1., (double)p.rows / like.c);
    return like;
}
}  // namespace

F32Route packed_f32_route(const PackedArgs& p, bool backward) {
    double blocks;
    const StepArgs like = like_equal_ones(p, blocks);
    StepArgs longest = p;
    longest.c = p.max_len;
    const F32Route route = f32_packed_route(like, p.max_len, blocks, most_tiles(p, 128) * p.H >= 512, backward);
    return route == F32_SPLIT && !f32x3_split_supported(longest, backward) ? F32_TERMS : route;
}
bool packed_f32_few(const PackedArgs& p, bool backward) {
    double blocks;
    StepArgs like = like_equal_ones(p, blocks);
    like.B = (int)ceil(blocks);
    return few_row_tiles(like, backward);
}

hipError_t launch_packed_f32(PackedArgs p, bool backward, hipStream_t st) {
    if (backward)
        if (hipError_t e = launch_packed_delta(p, SA_F32, st)) return e;
    p.by_rank = true;
    if (p.d > 128) return packed_f32_few(p, backward) ? run<256, 2>(p, backward, st) : run<256, 1>(p, backward, st);
    const F32Route route = packed_f32_route(p, backward);
    if (route == F32_SPLIT) return launch_packed_f32x3_split(p, backward, st);
    if (route != F32_INSTRUCTION) return launch_packed_f32x3(p, backward, st);
    if (p.d > 32 && p.d <= 64) return run_fwd<64, 4>(p, st);         // (forward: f32_packed_route)
    return p.d <= 32 ? run<32, 4>(p, backward, st) : run<128, 4>(p, backward, st);
}

}  // namespace sa
