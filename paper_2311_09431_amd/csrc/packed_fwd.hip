// Causal attention of packed sequences, forward, bf16: the ring step's workgroups (fwd_tiles.h), each on one 128-row tile of
// one sequence (packed.h).
//
// A launch has a workgroup for every tile that the sequences can have, rows / 128 + n_seq of them a head, whatever the offsets
// say (they are on the device); those behind the last tile end at once.
//
// Bound as the ring step's forward is, by the products and the exponentials beside them.  By the card, 8 sequences of up to 4096 rows, 32 heads on 8, d 128, 538
// to 577 us, 0.94 to 1.0 PFLOP/s of allowed pairs, 2 of 16384, 8 heads, 912 to 997 us, 1.1 to 1.2; of the pairs computed, diagonal tiles whole and
// rows behind a sequence's end too, the former are 93 %.
//
// A probability is rounded to one bf16 before it meets V, as in the ring step (row sums are of the unrounded ones): a second term would be half as many
// products again in the kernel that products bound.  O is 0.0020 from 64 bits (2-norm, relative), of which its own rounding is 0.0016.
#include "fwd_tiles.h"

namespace sa {

namespace {

template <int DP, bool PART>
hipError_t launch(const PackedArgs& p, hipStream_t st) {
    hipLaunchKernelGGL((fwd_mfma_kernel<true, WALK_TRI, DP, PART, false, false, PackedArgs>), dim3((unsigned)p.n_ranks * p.H),
                       dim3(64 * NW), 0, st, p, 0);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_fwd(PackedArgs p, hipStream_t st) {
    if (packed_split_wanted(p, false)) return launch_packed_split(p, false, st);
    p.n_ranks = (int)most_tiles(p, BM);
    p.by_rank = by_rank_wanted(p);
    const bool part = p.d % 8 != 0;
    if (p.d > 128) return part ? launch<256, true>(p, st) : launch<256, false>(p, st);
    if (p.d <= 32 && !part) return launch<32, false>(p, st);
    if (p.d <= 64) return part ? launch<64, true>(p, st) : launch<64, false>(p, st);
    if (p.d <= 112) return part ? launch<112, true>(p, st) : launch<112, false>(p, st);
    return part ? launch<128, true>(p, st) : launch<128, false>(p, st);
}

}  // namespace sa
