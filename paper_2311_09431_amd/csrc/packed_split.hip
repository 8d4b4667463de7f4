// Causal attention of packed sequences and its gradient, bf16, launches of few tiles: the ring step's workgroups of 32 rows
// (split_tiles.h), each on one tile of one sequence (packed.h).  Bound by the length of a walk, which several wavefronts share.
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
