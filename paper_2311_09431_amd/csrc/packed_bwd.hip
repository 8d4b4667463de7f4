// Gradient of causal attention over packed sequences, bf16: the ring step's workgroups (bwd_tiles.h; dK and dV at 65 to 128 columns:
// packed_bwd_ring.hip), each on one 128-row tile of one sequence (packed.h).  The query-owning ones come first and form delta =
// rowsum(dO * O) of their rows for both.
//
// Bound as the ring step's backward is, by products and the vector work beside them: 6 sequences of up to 4096 rows, 32 heads, d 100, dQ 0.67 and
// dK, dV 1.01 ms beside 0.49 forward, whole training pass 2.19 to 2.28 (by the card).  delta comes from O as it was stored, dS meets K and Q as bf16 (a second
// term would cost a third more products): gradients are 0.0025 to 0.0032 from 64 bits (2-norm, relative), their own rounding 0.0017.
#include "bwd_tiles.h"
#include "packed.h"

namespace sa {

namespace {

template <int DP, bool PART>
__global__ void __launch_bounds__(256, DP > 128 ? 1 : 2)
packed_dq_kernel(PackedArgs p) {
    __shared__ __attribute__((aligned(1024))) char lds0[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds1[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds2[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds3[tile_bytes(DP) * halves_of(DP)];
    int n_tiles, rank, head;
    if (!enter_sequence<true, BM>(p, (int)blockIdx.x, p.H, n_tiles, rank, head)) return;
    bwd_dq<true, WALK_TRI, DP, PART, false, true>(p, n_tiles, rank * p.H + head, lds0, lds1, lds2, lds3);
}

// up to 64 columns and above 128
// WAVES: wavefronts a SIMD that the register budget is cut for; at 64 columns two spill 141 registers (296 bytes of scratch a lane).
template <int DP, bool PART, int WAVES>
__global__ void __launch_bounds__(256, WAVES)
packed_dkdv_kernel(PackedArgs p) {
    __shared__ __attribute__((aligned(1024))) char lds0[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds1[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds2[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds3[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(16))) float stat[KV_STAT_FLOATS];
    const int heads = p.H_kv * halves_of(DP);
    int n_tiles, rank, head;
    if (!enter_sequence<false, BM>(p, (int)blockIdx.x, heads, n_tiles, rank, head)) return;
    bwd_dkdv<WALK_RING, true, DP, PART, false, true>(p, n_tiles, rank * heads + head, lds0, lds1, lds2, lds3, stat);
}

// Both kinds of workgroups in a launch, delta formed by one in front of it.  Above 128 columns (65 to 128: packed_bwd_ring.hip).
template <int DP, bool PART>
__global__ void __launch_bounds__(256, 1)
packed_both_kernel(PackedArgs p, PlacedKinds kinds) {
    __shared__ __attribute__((aligned(1024))) char lds0[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds1[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds2[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds3[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(16))) float stat[KV_STAT_FLOATS];
    int linear = (int)blockIdx.x, n_tiles, rank, head;
    const int keys = __builtin_amdgcn_readfirstlane(owns_keys(kinds, linear)), heads = keys ? p.H_kv * halves_of(DP) : p.H;
    linear = __builtin_amdgcn_readfirstlane(linear);        // (both kept scalar)
    if (keys) {
        if (!enter_sequence<false, BM>(p, linear, heads, n_tiles, rank, head)) return;
        bwd_dkdv<WALK_RING, true, DP, PART, false, true>(p, n_tiles, rank * heads + head, lds0, lds1, lds2, lds3, stat);
    } else {
        if (!enter_sequence<true, BM>(p, linear, heads, n_tiles, rank, head)) return;
        bwd_dq<true, WALK_TRI, DP, PART, false, true, false>(p, n_tiles, rank * heads + head, lds0, lds1, lds2, lds3);
    }
}

}  // namespace

// At 64 columns two wavefronts a SIMD are faster where many long walks hide each other's latency, whole training pass, us, one : two:
// 2 x 8192 rows, 32 heads, 2506 : 2296, 8192, 16 heads, 688 : 677; but 6 of up to 4096, 16 heads, 713 : 717, 16 of up to 1000, 32
// heads, 294 : 341, 4 of up to 500, 16 heads, 41 : 52, and with four query heads to a key/value head 8192, 32 heads, 1305 : 1415.
bool packed_two_wavefronts(const PackedArgs& p) { return p.H == p.H_kv && p.max_len >= 8192 && (int64_t)p.n_ranks * p.H_kv > 2 * N_CU; }

// Above 128 columns workgroups with all of them from 160 tiles on, whole training pass, d 256, us, halves : all: 4 of up to 500, 16 heads,
// 110 : 104, 8 of up to 1000 267 : 219, 6 of up to 4096, 8 heads, 1568 : 1273; but (fewer tiles) 2 of up to 1000, 4 heads, 140 : 153, 8 of up
// to 1000, 16 heads on 4, 308 : 342.
bool packed_all_columns(const PackedArgs& p) { return (int64_t)p.n_ranks * p.H_kv > 5 * N_CU / 8; }

// Both kinds of workgroups in one launch, by 128-row tiles (as many as there can be) of all key/value heads: few of them leave the chip half empty
// while the first kind ends.  Over 570 launches of 1 to 64 sequences of up to 64 to 8192 rows the rules here and in packed_split_wanted take 0.3 %
// more than the best choice, two launches always 17 % above 128 columns and 5 % below.  Whole training pass, us, one : two.  d 128: 1536, 16
// heads (192 tiles) 80 : 110, 4096, 8 heads (256) 196 : 244, 8 of up to 2000, 8 heads (480) 132 : 146, but 2048, 32 heads (512) 196 : 189; 4 of
// up to 4096, 32 heads on 8, (560) 1018 : 965, 6 of up to 1000, 64 on 8 (288) 389 : 407.  d 256: 1000 or 8192 rows, 1 to 4 heads 0.7,
// 4096, 8 heads (256) 453 : 502, but 12 heads (384) 628 : 574; 8 of up to 2000, 32 on 4 (240) 1000 : 1417.  A walk of one tile leaves little
// to fill: d 128, 16 of up to 128, 32 on 8, 59 : 53, 40 of up to 64, 32 on 8, 91 : 76, d 256, 64 of up to 64, 16 on 4, 166 : 118; 8 heads of
// their own 27 : 34.  Up to 64 columns these are packed_split.hip's launches: of 334, one launch here was the fastest by 5 % in 13.
bool packed_one_launch(const PackedArgs& p) {
    const int64_t tiles = (int64_t)p.n_ranks * p.H_kv;
    const bool own = p.H == p.H_kv;
    if (p.max_len <= BM) return tiles <= (own ? 192 : p.d > 128 ? 64 : 0);
    return tiles <= (own ? p.d > 128 ? 280 : 512 : 352);
}

namespace {

template <int DP, bool PART>
hipError_t launch_dkdv(const PackedArgs& p, hipStream_t st, int64_t n) {
    if constexpr (DP <= 64) {
        if (DP == 32 || packed_two_wavefronts(p)) {
            hipLaunchKernelGGL((packed_dkdv_kernel<DP, PART, 2>), dim3((unsigned)n), dim3(256), 0, st, p);
            return hipGetLastError();
        }
    }
    if constexpr (DP == 256 && !PART) {
        if (packed_all_columns(p)) return launch_packed_dkdv_wide(p, (unsigned)(n / 2), st);
    }
    if constexpr (DP != 32) hipLaunchKernelGGL((packed_dkdv_kernel<DP, PART, 1>), dim3((unsigned)n), dim3(256), 0, st, p);
    return hipGetLastError();
}

template <int DP, bool PART>
hipError_t launch(PackedArgs p, hipStream_t st) {
    p.n_ranks = (int)most_tiles(p, BM);
    const int64_t n_dq = (int64_t)p.n_ranks * p.H, n_dkdv = (int64_t)p.n_ranks * p.H_kv * halves_of(DP);
    p.by_rank = by_rank_wanted(p);
    if constexpr (DP > 64) {
        if (packed_one_launch(p)) {
            if (hipError_t e = launch_packed_delta(p, SA_BF16, st)) return e;
            if constexpr (DP <= 128) return launch_packed_bwd_ring(p, true, st);
            else {
                const PlacedKinds kinds = placed_kinds(p, n_dkdv, n_dq, packed_ratio(p));
                hipLaunchKernelGGL((packed_both_kernel<DP, PART>), dim3((unsigned)(n_dkdv + n_dq)), dim3(256), 0, st, p, kinds);
                return hipGetLastError();
            }
        }
    }
    hipLaunchKernelGGL((packed_dq_kernel<DP, PART>), dim3((unsigned)n_dq), dim3(256), 0, st, p);
    if (hipError_t e = hipGetLastError()) return e;
    if constexpr (DP == 112 || DP == 128) return launch_packed_bwd_ring(p, false, st);
    else return launch_dkdv<DP, PART>(p, st, n_dkdv);
}

}  // namespace

hipError_t launch_packed_bwd(const PackedArgs& p, hipStream_t st) {
    if (packed_split_wanted(p, true)) return launch_packed_split(p, true, st);
    const bool part = p.d % 8 != 0;
    if (p.d > 128) return part ? launch<256, true>(p, st) : launch<256, false>(p, st);
    if (p.d <= 32 && !part) return launch<32, false>(p, st);
    if (p.d <= 64) return part ? launch<64, true>(p, st) : launch<64, false>(p, st);
    if (p.d <= 112) return part ? launch<112, true>(p, st) : launch<112, false>(p, st);
    return part ? launch<128, true>(p, st) : launch<128, false>(p, st);
}

}  // namespace sa
