// Causal attention of packed sequences and its gradient, bf16, launches of few tiles: the ring step's workgroups of 32 rows
// (split_tiles.h), each on one tile of one sequence (packed.h).  Bound by the length of a walk, which several wavefronts share.  Those
// with a window too (window.h).
#include "split_tiles.h"

namespace sa {

namespace {

// workgroups 0 .. n_dkdv - 1 own keys, the others queries
template <int DP, bool PART>
__global__ void __launch_bounds__(64 * BWD_WAVES, DP <= 64 ? 2 : 1)
packed_bwd_split_kernel(PackedArgs p, int n_dkdv) {
    __shared__ __attribute__((aligned(1024))) char lds[BWD_WAVES * 2 * STAGE_BYTES<DP> + 2 * SUB_BYTES<DP>];
    __shared__ __attribute__((aligned(1024))) char stats[BWD_WAVES * 2 * STAT_BYTES];
    __shared__ uint32_t masks[BWD_WAVES];
    int n_tiles, rank, head;
    if ((int)blockIdx.x < n_dkdv) {
        if (!enter_sequence<false, OWN>(p, (int)blockIdx.x, p.H_kv, n_tiles, rank, head)) return;
        bwd_dkdv<DP, PART, false, true>(p, n_tiles, rank * p.H_kv + head, lds, stats, masks);
    } else {
        if (!enter_sequence<true, OWN>(p, (int)blockIdx.x - n_dkdv, p.H, n_tiles, rank, head)) return;
        bwd_dq<DP, PART, false, true>(p, n_tiles, rank * p.H + head, lds, stats, masks);
    }
}

template <int DP, bool PART>
hipError_t run(PackedArgs p, bool backward, hipStream_t st) {
    p.n_ranks = (int)most_tiles(p, OWN);
    p.by_rank = true;
    const unsigned n_dkdv = (unsigned)p.n_ranks * p.H_kv, n_dq = (unsigned)p.n_ranks * p.H;
    if (backward) hipLaunchKernelGGL((packed_bwd_split_kernel<DP, PART>), dim3(n_dkdv + n_dq), dim3(64 * BWD_WAVES), 0, st, p, (int)n_dkdv);
    else hipLaunchKernelGGL((fwd_split_kernel<DP, PART, false, false, PackedArgs>), dim3(n_dq), dim3(64 * FWD_WAVES), 0, st, p, 0);
    return hipGetLastError();
}

}  // namespace

// By 128-row tiles (as many as there can be) of all query heads, and of all key/value heads in the backward.  us, 128-row kernels : these.
// Forward, d 128: 3 sequences of up to 300 rows, 8 heads (48 tiles) 10.4 : 8.8, 2048, 8 heads (128) 34 : 25, 4 of up to 4096, 2 heads (144)
// 60 : 35, 1000, 16 heads (128) 21 : 20, but 16 of up to 300, 4 heads (136) 10.8 : 13.5, 5 of up to 200, 16 heads (144) 9.9 : 14.6; 8192, 4 heads
// (256) 114 : 106, but 4096, 8 heads (256) 62 : 66; 5 of up to 777, 4 heads (68) 18 : 11, 8 heads (136) 18 : 17.  d 64 likewise.
// Backward, those kernels in one launch or two (packed_bwd.hip), the better, whole pass: d 128, 2000, 6 of up to, 16 heads on 2 (122) 426 : 312, 2
// of up to 4096, 32 heads on 4 (184) 899 : 848, 4 of up to 2000, 6 heads (144) 82 : 77, but 16 of up to 128, 8 heads (128) 27 : 34, 3000, 6
// heads (144) 120 : 122, 4 of up to 3000, 32 on 4 (212) 724 : 763; below 96 tiles to 0.5.  d 64, 16 of up to 1000, 32 on 4 (328) 290 : 256, 8 of up
// to 2000, 8 heads (480) 105 : 97, but 16 of up to 128, 16 heads (256) 27 : 31, d 32 22 : 27.
bool packed_split_wanted(const PackedArgs& p, bool backward) {
    // requests behind a walk's end name up to 32 rows behind the last sub-tile: their offsets must not wrap into the sequence
    const int64_t widest = p.stride_s > p.kv_stride_s ? p.stride_s : p.kv_stride_s;
    if (p.d > TD || ((int64_t)(p.max_len + 127) / 128 * 128 + OWN) * 2 * widest + 2 * p.d >= (int64_t(1) << 31)) return false;
    // HIP takes fewer than 2^32 threads a launch: the backward's rule goes by key/value heads, of which each may have thousands of query heads
    if (most_tiles(p, OWN) * (p.H + (backward ? p.H_kv : 0)) * 64 * (backward ? BWD_WAVES : FWD_WAVES) >= (int64_t(1) << 32)) return false;
    const int64_t tiles = most_tiles(p, 128) * (backward ? p.H_kv : p.H);
    if (!backward) return tiles <= 80 || (tiles <= 144 && p.max_len >= 700) || (tiles <= 256 && p.max_len >= 8192);
    if (p.d <= 64) return tiles <= (p.max_len >= 1000 ? 512 : p.max_len <= 64 || p.max_len > 128 ? 320 : 160);
    const int64_t walk = (int64_t)p.max_len * (p.H / p.H_kv);
    return tiles <= (walk >= 12000 ? 184 : walk >= 2000 ? 152 : 96);
}

// offsets and threads fit their bits, as packed_split_wanted has it
static bool in_reach(const WindowArgs& p) {
    const int64_t widest = p.stride_s > p.kv_stride_s ? p.stride_s : p.kv_stride_s;
    return p.d <= TD && ((int64_t)(p.max_len + 127) / 128 * 128 + OWN) * 2 * widest + 2 * p.d < (int64_t(1) << 31) &&
           most_tiles(p, OWN) * (p.H + p.H_kv) * 64 * 4 < (int64_t(1) << 32);
}

// With a window, forward: four wavefronts a workgroup, or two, for walks that are no longer than the window.  Wavefronts of a workgroup (0: the
// 128-row kernels), by 128-row tiles of all heads and by keys a walk goes over.  A small launch is latency, that of code read for the first time too:
// 14 KB here, of which a tile passes all, 61 KB there.  us, 128-row : two wavefronts : four (: eight), first tokens 4.
// d 128: 300 rows, 8 heads, window 64 (24 tiles) 17.0 : 8.0 : 7.4 : 7.9; 4096, 2 heads, 1024 (66) 29.8 : 17.2 : 14.1 : 13.7; 2000, 8 heads, 500
// (136) 25.7 : 15.6 : 13.3 : 20.5; 4096, 4 heads, 2048 (132) 43 : 33 : 26 : 33; 2 of 2000, 8 heads, 500 (264) 26.3 : 24.0 : 23.3, but 4096, 8 heads,
// 1024 (264) 30.9 : 35.6 : 32.3, 4 of 1000, 16 heads, 128 (576) 25.3 : 27.4 : 34.6; 100 of 20, 16 heads (1856) 32.9 : 17.7 : 23.2.
// d 64: 5 of 200, 16 heads, 64 (208) 11.8 : 8.6 : 8.7 : 17.2; 4 of 1000, 16 heads, 512 (576) 20.8 : 20.1 : 24.5; 8 of 1000, 16 heads, 200 (1136)
// 34.4 : 28.3 : 41.5, but 32 of 256, 32 heads, 64 (over 3000) 37.8 : 42.0 : 65.0.
int window_split_waves(const WindowArgs& p) {
    if (!in_reach(p)) return 0;
    const int64_t tiles = most_tiles(p, 128) * p.H, reach = (int64_t)p.window + OWN + p.sinks, walk = p.max_len < reach ? p.max_len : reach;
    if (tiles <= 144) return 4;
    if (p.max_len <= OWN) return 2;
    return (p.d <= 64 ? tiles <= 1600 && tiles * walk <= 320000 : tiles * walk <= 160000) ? 2 : 0;
}
template <int DP, bool PART>
static hipError_t run_window(const WindowArgs& p, int waves, hipStream_t st) {
    const dim3 grid((unsigned)p.n_ranks * p.H), block(64 * waves);
    if (waves == 2) hipLaunchKernelGGL((fwd_split_kernel<DP, PART, false, false, WindowArgs, 2>), grid, block, 0, st, p, 0);
    else hipLaunchKernelGGL((fwd_split_kernel<DP, PART, false, false, WindowArgs, 4>), grid, block, 0, st, p, 0);
    return hipGetLastError();
}
// The gradient, by four wavefronts, where there are few tiles of all key/value heads.  us, 128-row : these, whole call, first tokens 4.  d 128: 300 rows, 8 heads,
// window 64 (24 tiles) 41 : 15; 8192, one head, 4096 (65) 225 : 90; 2 of 2000, 16 heads on 2, 500 (66) 278 : 177; 4 of 2000, 64 on 1, 500 (66) 2106 : 1290; 1000, 16
// on 8, 200 (64) 83 : 54; 2000, 8 heads, 500 (128) 78 : 63; but 4 of 1000, 32 on 4, 128 (140) 200 : 222; 2500, 8 heads, 128 (160) 60 : 66; 4096, 8
// heads, 1024 (264) 101 : 132.  d 64: 1000, 16 on 8, 200 (64) 65 : 36; 8 of 500, 16 on 2, 64 (78) 82 : 39; 4 of 1000, 6 heads, 128 (210) 53 : 30; 12 of 200,
// 8 heads, 64 (240) 26.6 : 25.0; but 4 of 1000, 16 on 8, 256 (280) 69 : 74; 4000, 16 heads, 64 (512) 73 : 80.
template <int DP, bool PART>
__global__ void __launch_bounds__(64 * BWD_WAVES, DP <= 64 ? 2 : 1)
window_bwd_split_kernel(WindowArgs p, int n_dkdv) {
    __shared__ __attribute__((aligned(1024))) char lds[BWD_WAVES * 2 * STAGE_BYTES<DP> + 2 * SUB_BYTES<DP>];
    __shared__ __attribute__((aligned(1024))) char stats[BWD_WAVES * 2 * STAT_BYTES];
    __shared__ uint32_t masks[2 * BWD_WAVES];
    int n_tiles, rank, head, seq;
    if ((int)blockIdx.x < n_dkdv) {
        if (!enter_sequence<false, OWN>(p, (int)blockIdx.x, p.H_kv, n_tiles, rank, head, &seq)) return;
        p.slot = find_slot(p, seq, rank * OWN);
        bwd_dkdv<DP, PART, false, true, WindowArgs>(p, n_tiles, rank * p.H_kv + head, lds, stats, masks);
    } else {
        if (!enter_sequence<true, OWN>(p, (int)blockIdx.x - n_dkdv, p.H, n_tiles, rank, head)) return;
        bwd_dq<DP, PART, false, true, WindowArgs>(p, n_tiles, rank * p.H + head, lds, stats, masks);
    }
}
template <int DP, bool PART>
static hipError_t run_window_bwd(const WindowArgs& p, hipStream_t st) {
    const unsigned n_dkdv = (unsigned)p.n_ranks * p.H_kv, n_dq = (unsigned)p.n_ranks * p.H;
    hipLaunchKernelGGL((window_bwd_split_kernel<DP, PART>), dim3(n_dkdv + n_dq), dim3(64 * BWD_WAVES), 0, st, p, (int)n_dkdv);
    return hipGetLastError();
}
bool window_bwd_split_wanted(const WindowArgs& p) {
    return in_reach(p) && most_tiles(p, 128) * p.H_kv <= (p.d <= 64 ? 240 : 128);
}
hipError_t launch_window_bwd_split(WindowArgs p, hipStream_t st) {
    if (hipError_t e = launch_packed_delta(p, SA_BF16, st)) return e;
    p.n_ranks = (int)most_tiles(p, OWN);
    p.by_rank = true;
    const bool part = p.d % 8 != 0;
    hipError_t e;
    if (p.d <= 32 && !part) e = run_window_bwd<32, false>(p, st);
    else if (p.d <= 64) e = part ? run_window_bwd<64, true>(p, st) : run_window_bwd<64, false>(p, st);
    else if (p.d <= 112) e = part ? run_window_bwd<112, true>(p, st) : run_window_bwd<112, false>(p, st);
    else e = part ? run_window_bwd<128, true>(p, st) : run_window_bwd<128, false>(p, st);
    return e != hipSuccess ? e : launch_window_far(p, SA_BF16, st);
}
hipError_t launch_window_split(WindowArgs p, int waves, hipStream_t st) {
    p.n_ranks = (int)most_tiles(p, OWN);
    p.by_rank = true;
    const bool part = p.d % 8 != 0;
    if (p.d <= 32 && !part) return run_window<32, false>(p, waves, st);
    if (p.d <= 64) return part ? run_window<64, true>(p, waves, st) : run_window<64, false>(p, waves, st);
    if (p.d <= 112) return part ? run_window<112, true>(p, waves, st) : run_window<112, false>(p, waves, st);
    return part ? run_window<128, true>(p, waves, st) : run_window<128, false>(p, waves, st);
}

hipError_t launch_packed_split(PackedArgs p, bool backward, hipStream_t st) {
    if (backward)
        if (hipError_t e = launch_packed_delta(p, SA_BF16, st)) return e;
    const bool part = p.d % 8 != 0;
    if (p.d <= 32 && !part) return run<32, false>(p, backward, st);
    if (p.d <= 64) return part ? run<64, true>(p, backward, st) : run<64, false>(p, backward, st);
    if (p.d <= 112) return part ? run<112, true>(p, backward, st) : run<112, false>(p, backward, st);
    return part ? run<128, true>(p, backward, st) : run<128, false>(p, backward, st);
}

}  // namespace sa
