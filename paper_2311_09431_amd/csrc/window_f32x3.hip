// Attention with a window (window.h) and its gradient, fp32 storage in three bf16 terms: the workgroups of 128 rows and more (f32x3_tiles.h).
// Streamed tiles are of 32 rows, and a wavefront's 32 rows leave out those of which they see nothing.  Bound by the number of such tiles, each between
// barriers, more than by products: 5 sequences of up to 777 rows, 16 heads on 8, 100 columns, window 100, forward 41 us (matrix cores 12 % busy),
// gradient 111 (15 %, 55 % of cycles in waits), 105 keys a row seen of 288 walked over.  (The gradient's kernel of 65 to 128 columns spills 39 registers.)
#include "f32x3_tiles.h"

namespace sa {

namespace {

// workgroups 0 .. n_dkdv - 1 own keys, the others queries
template <int DP>
__global__ void __launch_bounds__(64 * 2 * GROUPS, 2)
window_bwd_f32x3_kernel(WindowArgs p, int n_dkdv) {
    constexpr int ROWS = 32 * GROUPS;
    __shared__ __attribute__((aligned(1024))) char lds[2 * BUFFER];
    __shared__ __attribute__((aligned(1024))) char tiles[EXCHANGED];
    __shared__ float stats[2 * 3 * TILE];          // [buffer][LSE hi | LSE lo | delta][row]
    __shared__ uint32_t masks[6 * GROUPS];
    int n_tiles, rank, head, seq;
    if ((int)blockIdx.x < n_dkdv) {
        if (!enter_sequence<false, ROWS>(p, (int)blockIdx.x, p.H_kv, n_tiles, rank, head, &seq)) return;
        p.slot = find_slot(p, seq, rank * ROWS);
        bwd_dkdv<DP, true, WindowArgs>(p, n_tiles, rank * p.H_kv + head, lds, tiles, stats, masks);
    } else {
        if (!enter_sequence<true, ROWS>(p, (int)blockIdx.x - n_dkdv, p.H, n_tiles, rank, head)) return;
        bwd_dq<DP, true, WindowArgs>(p, n_tiles, rank * p.H + head, lds, tiles, masks);
    }
}

template <int DP, int WAVES>
hipError_t run_fwd(WindowArgs p, hipStream_t st) {
    p.n_ranks = (int)most_tiles(p, 32 * WAVES);
    hipLaunchKernelGGL((fwd_f32x3_kernel<DP, WAVES, WindowArgs>), dim3((unsigned)p.n_ranks * p.H), dim3(64 * WAVES), 0, st, p, 0);
    return hipGetLastError();
}
template <int DP>
hipError_t run(WindowArgs p, bool backward, hipStream_t st) {
    p.n_ranks = (int)most_tiles(p, 32 * GROUPS);
    if (!backward) return run_fwd<DP, 4>(p, st);
    const unsigned n_dkdv = (unsigned)p.n_ranks * p.H_kv, n_dq = (unsigned)p.n_ranks * p.H;
    hipLaunchKernelGGL((window_bwd_f32x3_kernel<DP>), dim3(n_dkdv + n_dq), dim3(64 * 2 * GROUPS), 0, st, p, (int)n_dkdv);
    if (hipError_t e = hipGetLastError()) return e;
    return launch_window_far(p, SA_F32, st);
}

}  // namespace

hipError_t launch_window_f32x3(WindowArgs p, bool backward, hipStream_t st) {
    return p.d <= 64 ? run<64>(p, backward, st) : run<128>(p, backward, st);
}

}  // namespace sa
