// Gradient of attention with a window (window.h), bf16: the packed sequences' workgroups of 128 rows (bwd_tiles.h).  The query-owning ones come first
// and form delta = rowsum(dO * O) of their rows for both.  With P_ab = exp(scale q_a k_b - LSE_a), dS = P (dO V^T - delta): dQ = scale dS K, dK = scale
// dS^T Q, dV = P^T dO over the pairs that are seen.  P and dS meet dO, Q and K rounded to one bf16 term, as the causal kernels': 0.0024 from 64
// bits, 0.0017 of it the results' own rounding.  Bound by the products, as the causal kernels: 2 sequences of up to 16384 rows, 16 heads on 8, 128
// columns, window 2048, dQ 495 us (matrix cores 59 % busy), dK and dV 720 to 760 (43 %, one wavefront a SIMD), the first keys' far rows 52 and
// joining them 17.  (First keys walked to the sequence's end: forward and gradient 2079 us, not 1600.)
#include "bwd_tiles.h"

namespace sa {

namespace {

template <int DP, bool PART>
__global__ void __launch_bounds__(256, DP > 128 ? 1 : 2)
window_dq_kernel(WindowArgs p) {
    __shared__ __attribute__((aligned(1024))) char lds0[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds1[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds2[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds3[tile_bytes(DP) * halves_of(DP)];
    int n_tiles, rank, head;
    if (!enter_sequence<true, BM>(p, (int)blockIdx.x, p.H, n_tiles, rank, head)) return;
    bwd_dq<true, WALK_TRI, DP, PART, false, true, true, WindowArgs>(p, n_tiles, rank * p.H + head, lds0, lds1, lds2, lds3);
}

template <int DP, bool PART>
__global__ void __launch_bounds__(256, DP == 32 ? 2 : 1)
window_dkdv_kernel(WindowArgs p) {
    __shared__ __attribute__((aligned(1024))) char lds0[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds1[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds2[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds3[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(16))) float stat[KV_STAT_FLOATS];
    const int heads = p.H_kv * halves_of(DP);
    int n_tiles, rank, head, seq;
    if (!enter_sequence<false, BM>(p, (int)blockIdx.x, heads, n_tiles, rank, head, &seq)) return;
    p.slot = find_slot(p, seq, rank * BM);
    bwd_dkdv<WALK_RING, true, DP, PART, false, true, WindowArgs>(p, n_tiles, rank * heads + head, lds0, lds1, lds2, lds3, stat);
}

template <int DP, bool PART>
hipError_t launch(WindowArgs p, hipStream_t st) {
    p.n_ranks = (int)most_tiles(p, BM);
    p.by_rank = true;
    hipLaunchKernelGGL((window_dq_kernel<DP, PART>), dim3((unsigned)p.n_ranks * p.H), dim3(256), 0, st, p);
    if (hipError_t e = hipGetLastError()) return e;
    hipLaunchKernelGGL((window_dkdv_kernel<DP, PART>), dim3((unsigned)p.n_ranks * p.H_kv * halves_of(DP)), dim3(256), 0, st, p);
    if (hipError_t e = hipGetLastError()) return e;
    return launch_window_far(p, SA_BF16, st);
}

}  // namespace

hipError_t launch_window_bwd(WindowArgs p, hipStream_t st) {
    if (window_bwd_split_wanted(p)) return launch_window_bwd_split(p, st);
    const bool part = p.d % 8 != 0;
    if (p.d > 128) return part ? launch<256, true>(p, st) : launch<256, false>(p, st);
    if (p.d <= 32 && !part) return launch<32, false>(p, st);
    if (p.d <= 64) return part ? launch<64, true>(p, st) : launch<64, false>(p, st);
    if (p.d <= 112) return part ? launch<112, true>(p, st) : launch<112, false>(p, st);
    return part ? launch<128, true>(p, st) : launch<128, false>(p, st);
}

}  // namespace sa
