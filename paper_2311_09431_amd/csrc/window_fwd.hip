// Attention with a window (window.h), forward, bf16: the packed sequences' workgroups of 128 rows (fwd_tiles.h).
//
// O_a = sum_b exp(scale q_a k_b - LSE_a) v_b over the keys that row a sees.  Weights meet V rounded to one bf16 term, as the causal kernel's: 0.0020 from
// 64 bits, 0.0017 of it the result's own rounding.  Bound by the products, as that one: a row's window of W keys costs W + 128 of them on average, W + 256 with first
// keys, for which a tile of 128 is walked over, at the causal kernel's rate: 32768 rows, 16 heads on 8, 128 columns, window 4096, 947 to 1050 us by the card, matrix
// cores 60 % busy, up to 1.09 PFLOP/s of the pairs that are seen.  Tiles with pairs that are not seen go through loops of their own: both kinds in one loop, behind a branch,
// spilled 39 registers (dQ's: 128).
#include "fwd_tiles.h"

namespace sa {

namespace {

template <int DP, bool PART>
hipError_t launch(const WindowArgs& p, hipStream_t st) {
    hipLaunchKernelGGL((fwd_mfma_kernel<true, WALK_TRI, DP, PART, false, false, WindowArgs>), dim3((unsigned)p.n_ranks * p.H), dim3(64 * NW), 0, st, p, 0);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_window_fwd(WindowArgs p, hipStream_t st) {
    if (const int waves = window_split_waves(p)) return launch_window_split(p, waves, st);
    p.n_ranks = (int)most_tiles(p, BM);
    p.by_rank = true;
    const bool part = p.d % 8 != 0;
    if (p.d > 128) return part ? launch<256, true>(p, st) : launch<256, false>(p, st);
    if (p.d <= 32 && !part) return launch<32, false>(p, st);
    if (p.d <= 64) return part ? launch<64, true>(p, st) : launch<64, false>(p, st);
    if (p.d <= 112) return part ? launch<112, true>(p, st) : launch<112, false>(p, st);
    return part ? launch<128, true>(p, st) : launch<128, false>(p, st);
}

}  // namespace sa
