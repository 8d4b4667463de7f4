// Attention with a window (window.h) and its gradient, fp32 storage, on the fp32 matrix cores (f32_tiles.h): above 128 columns.  Up to
// 128 by three bf16 terms a number (window_f32x3.hip, packed_f32x3_split.hip).  Bound by walks that few workgroups take, each key-owning one a group's
// heads in turn, with scores formed for either half of the columns: 3 sequences of up to 265 rows, 8 heads on 1, 256 columns, window 100, forward 58, gradient 582 us.  (The
// gradient's kernel spills 113 registers, the forward's 21.)
#include "f32_tiles.h"

namespace sa {

namespace {

// workgroups 0 .. n_dkdv - 1 own keys, the others queries
template <int DP, int SPLIT>
__global__ void __launch_bounds__(64 * WAVES, DP > 64 ? 1 : 2)
window_bwd_f32_kernel(WindowArgs p, int n_dkdv) {
    constexpr int ROWS = 32 * WAVES / SPLIT;
    __shared__ __attribute__((aligned(16))) float lds[tile_floats<SPLIT, DP>()];
    __shared__ float stats[2 * tile_rows(SPLIT)];                   // LSE | delta of a tile's queries
    __shared__ uint32_t masks[WAVES];
    const int heads = p.H_kv * (DP > 128 ? 2 : 1);
    int n_tiles, rank, head, seq;
    if ((int)blockIdx.x < n_dkdv) {
        if (!enter_sequence<false, ROWS>(p, (int)blockIdx.x, heads, n_tiles, rank, head, &seq)) return;
        p.slot = find_slot(p, seq, rank * ROWS);
        bwd_dkdv<float, DP, SPLIT, true, WindowArgs>(p, n_tiles, rank * heads + head, lds, stats, masks);
    } else {
        if (!enter_sequence<true, ROWS>(p, (int)blockIdx.x - n_dkdv, p.H, n_tiles, rank, head)) return;
        bwd_dq<float, DP, SPLIT, true, WindowArgs>(p, n_tiles, rank * p.H + head, lds, masks);
    }
}

template <int DP, int SPLIT>
hipError_t run(WindowArgs p, bool backward, hipStream_t st) {
    p.n_ranks = (int)most_tiles(p, 32 * WAVES / SPLIT);
    const unsigned n_dkdv = (unsigned)p.n_ranks * p.H_kv * (DP > 128 ? 2 : 1), n_dq = (unsigned)p.n_ranks * p.H;
    if (backward) {
        hipLaunchKernelGGL((window_bwd_f32_kernel<DP, SPLIT>), dim3(n_dkdv + n_dq), dim3(64 * WAVES), 0, st, p, (int)n_dkdv);
        if (hipError_t e = hipGetLastError()) return e;
        return launch_window_far(p, SA_F32, st);
    }
    hipLaunchKernelGGL((fwd_f32_kernel<float, DP, SPLIT, WindowArgs>), dim3(n_dq), dim3(64 * WAVES), 0, st, p, 0);
    return hipGetLastError();
}

}  // namespace

// Up to 128 columns in three bf16 terms, launches of few tiles (of 128 rows, as many as there can be, of all heads) by workgroups of 32 rows.  us, fp32
// instruction : 32 rows : 128 rows, forward and gradient.  d 128: a sequence of 4000 rows, 2 heads on 1, window 2000 (64 tiles) 140, 416 : 72, 255 :
// 242, 728; of 200, one head, 22, 37 : 18, 39 : 27, 49; but of 1000, 16 heads, 128 (144) 59, 160 : 43, 158 : 40, 91; of 4000, 8 heads, 1000 (264)
// 303, 754 : 172, 532 : 139, 378; 5 of up to 777, 16 heads on 8, 100 (d 100) 85, 209 : 71, 191 : 42, 141.  d 64: 2 of up to 1000, 2 heads, 300 (32)
// 37, 60 : 12, 34 : 39, 59; 2000, 4 heads, 200 (68) 30, 86 : 13, 48 : 33, 55; but 5 of up to 777, 16 heads on 8, 100, 82, 193 : 37, 93 : 27, 75.
// (Of the gradient those of all key/value heads, 128 : 32 rows: 2 of 625, 16 heads on 2, 100 (22 tiles) 393 : 170; 5 of 454, 8 on 1, d 96, window 2 (22) 262 : 132; 2 of
// 2000, 16 on 2, 500 (66) 900 : 602; 1000, 64 on 8, 100 (64) 415 : 384; d 64, 2 of 1000, 32 on 4, 100 (68) 184 : 140; d 32, 4 of 777, 8 on 2, 100 (56) 109 : 61.)
// (Forward, longer walks, 128 : 32 rows: d 32, 2 of up to 2768 rows, 4 heads, 2395, 182 : 38; 3000, 16 heads, 1000 (400) 156 : 73; 4000, 8 heads, 300 (264) 39 : 32; d 64, 3000, 16
// heads, 1000 159 : 119; 4 of up to 2000, 8 heads, 800, 72 : 41; but 8000, 4 heads, 500 (252) 55 : 60.)
static bool few_tiles(const WindowArgs& p, bool backward) {
    StepArgs longest = p;
    longest.c = p.max_len;
    longest.B = 1;
    const bool fits = most_tiles(p, 32) * p.H * 64 * 8 * 2 < (int64_t(1) << 32);
    if (!fits || !f32x3_split_supported(longest, backward)) return false;
    const int64_t tiles = most_tiles(p, 128), reach = (int64_t)p.window + 32 + p.sinks, walk = p.max_len < reach ? p.max_len : reach;
    if (!backward && p.d <= 64 && tiles * p.H <= 512 && walk >= (p.d <= 32 ? 300 : 800)) return true;
    return tiles * (backward ? p.H_kv : p.H) <= 96;
}

hipError_t launch_window_f32(WindowArgs p, bool backward, hipStream_t st) {
    if (backward)
        if (hipError_t e = launch_packed_delta(p, SA_F32, st)) return e;
    p.by_rank = true;
    if (p.d <= 128) return few_tiles(p, backward) ? launch_window_f32x3_split(p, backward, st) : launch_window_f32x3(p, backward, st);
    return run<256, 2>(p, backward, st);
}

}  // namespace sa
