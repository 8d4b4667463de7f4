// Forward ring step on the matrix cores: which launches take the kernel of fwd_tiles.h, and how they are ordered.
#include "fwd_tiles.h"

namespace sa {

bool fwd_mfma_supported(const StepArgs& a, int dtype) {
    // the tile loads address a shard through a buffer descriptor with 32-bit byte offsets:
    // the last row of its last (possibly partial) tile pair must end below 2^31 bytes from
    // its first
    const int64_t rows = (int64_t)(a.c + BM - 1) / BM * BM;
    // one workgroup per (128-row tile, device, batch, head) in a 1-D grid
    if (rows / BM * a.B * a.H * a.n_q >= (int64_t(1) << 31)) return false;
    // head dimensions above 128 (two 128-column halves) in whole 16-byte chunks only
    if (a.d > 2 * D || (a.d > D && a.d % 8)) return false;
    return dtype == SA_BF16 && a.d % 4 == 0 && a.c >= BM &&
           rows * 2 * a.kv_stride_s + 2 * a.d < (int64_t(1) << 31);
}

// Query-owning workgroups by ranks (decode_block), us, groups : ranks.  Above 128 columns walks over a striped ring's shards
// gain up to 1536: 64 heads of 4 x 1024, d 256, 686 : 717, of 4 x 1000 675 : 693.  Many heads of few tiles have their groups'
// tails short already and too much K and V in flight for the L2: triangular steps, d 64, 512 heads of 384 rows 33.1 : 36.6,
// 512 of 640 61.6 : 69.7, 256 of 512 30.2 : 30.4, 256 of 768 45.3 : 44.0; d 128, 384 of 256 34.8 : 39.7, 256 of 1024 135 : 152,
// 256 of 512 49.6 : 50.0, 160 of 1024 .97; d 100, 848 of 384 113 : 146, 320 of 1024 153 : 180, 192 of 1024 86.6 : 84.1; d 256,
// 680 of 384 259 : 286, 256 of 384 81 : 88, 256 of 512 145 : 138.  32 columns computed: 1280 of 256 30.0 : 32.1, 512 of 256 .94.
bool fwd_by_rank(const StepArgs& a) {
    const int64_t ranks = (int64_t)((a.c + BM - 1) / BM) * a.n_q, heads = (int64_t)a.B * a.H;
    const bool ring = a.layout == SA_STRIPED && a.n_kv > 1;
    if (!by_rank(uneven(a), ranks * heads, a.d > 128 ? ring ? 6 * N_CU : MOST_BY_RANK<256, true> : a.d > 112 ? MOST_BY_RANK<128, true> : MOST_BY_RANK<64, true>)) return false;
    if (a.d <= 32 && a.d % 8 == 0) return heads <= 768;
    return ranks >= 4 && heads <= (a.d <= 64 ? 256 : a.d <= 128 ? 192 : 512);
}

namespace {
bool one_block(const StepArgs& a) { return a.n_q == 1 && a.n_kv == 1 && !a.fresh; }
template <int WALK, int DP, bool PART, bool BY_RANK = false>
void launch_fwd_walk(const StepArgs& a, hipStream_t st, dim3 grid, dim3 block, int n_qtiles) {
    if constexpr (WALK != WALK_FULL && !BY_RANK)
        if (fwd_by_rank(a)) return launch_fwd_walk<WALK, DP, PART, true>(a, st, grid, block, n_qtiles);
    // Up to 64 columns three workgroups fit a compute unit; uneven work that they would hold all (or
    // nearly all) at once is balanced better by two, so LDS is asked for that keeps the third out: 640
    // workgroups 96 -> 77 us, 768 96 -> 84, 1024 183 -> 173, but 1536 242 -> 260.
    const unsigned wgs = grid.x, keep_out = DP <= 64 && uneven(a) && wgs > 2 * N_CU && wgs <= 4 * N_CU ? 24576 : 0;
    if (a.c % BM) hipLaunchKernelGGL((fwd_mfma_kernel<true, WALK, DP, PART, BY_RANK>), grid, block, keep_out, st, a, n_qtiles);
    else hipLaunchKernelGGL((fwd_mfma_kernel<false, WALK, DP, PART, BY_RANK>), grid, block, keep_out, st, a, n_qtiles);
}
template <int DP, bool PART>
void launch_fwd_variant(const StepArgs& a, hipStream_t st, dim3 grid, dim3 block, int n_qtiles) {
    if (!one_block(a)) launch_fwd_walk<WALK_RING, DP, PART>(a, st, grid, block, n_qtiles);
    else if (block_kind(a.q_dev, a.kv_dev, a.layout) == MASK_FULL)
        launch_fwd_walk<WALK_FULL, DP, PART>(a, st, grid, block, n_qtiles);
    else launch_fwd_walk<WALK_TRI, DP, PART>(a, st, grid, block, n_qtiles);
}
template <int DP>
void launch_fwd_rope(const StepArgs& a, hipStream_t st, dim3 grid, dim3 block, int n_qtiles) {
    if (block_kind(a.q_dev, a.kv_dev, a.layout) == MASK_FULL)
        hipLaunchKernelGGL((fwd_mfma_kernel<false, WALK_FULL, DP, false, false, true>), grid, block, 0, st, a, n_qtiles);
    else if (fwd_by_rank(a))
        hipLaunchKernelGGL((fwd_mfma_kernel<false, WALK_TRI, DP, false, true, true>), grid, block, 0, st, a, n_qtiles);
    else
        hipLaunchKernelGGL((fwd_mfma_kernel<false, WALK_TRI, DP, false, false, true>), grid, block, 0, st, a, n_qtiles);
}
}  // namespace

// fused query rotation: head dimension 64, 128 or 256 (both halves of a rotation pair in one
// lane) and block sizes that are a multiple of 128
bool fwd_mfma_rope_supported(const StepArgs& a, int dtype) {
    return fwd_mfma_supported(a, dtype) && (a.d == 64 || a.d == 128 || a.d == 256) && a.c % BM == 0;
}

hipError_t launch_fwd_mfma(const StepArgs& a, hipStream_t st) {
    const int n_qtiles = (a.c + BM - 1) / BM;
    const dim3 grid((unsigned)n_qtiles * a.n_q * a.B * a.H), block(64 * NW);
    const bool part = a.d % 8 != 0;
    if (a.q_pos) {
        if (a.d == 64) launch_fwd_rope<64>(a, st, grid, block, n_qtiles);
        else if (a.d == 128) launch_fwd_rope<128>(a, st, grid, block, n_qtiles);
        else launch_fwd_rope<256>(a, st, grid, block, n_qtiles);
    } else if (a.d > 128) {
        launch_fwd_variant<256, false>(a, st, grid, block, n_qtiles);
    } else if (a.d <= 32 && !part) {
        launch_fwd_variant<32, false>(a, st, grid, block, n_qtiles);
    } else if (a.d <= 64) {
        if (part) launch_fwd_variant<64, true>(a, st, grid, block, n_qtiles);
        else launch_fwd_variant<64, false>(a, st, grid, block, n_qtiles);
    } else if (a.d <= 112) {
        if (part) launch_fwd_variant<112, true>(a, st, grid, block, n_qtiles);
        else launch_fwd_variant<112, false>(a, st, grid, block, n_qtiles);
    } else {
        if (part) launch_fwd_variant<128, true>(a, st, grid, block, n_qtiles);
        else launch_fwd_variant<128, false>(a, st, grid, block, n_qtiles);
    }
    return hipGetLastError();
}

}  // namespace sa
