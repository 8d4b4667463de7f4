// Attention with a window (window.h), forward, bf16: the packed sequences' workgroups of 128 rows (fwd_tiles.h).
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
