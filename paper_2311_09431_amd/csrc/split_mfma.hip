// Ring step for launches of few workgroups (split_tiles.h), bf16: the kernels' launches, and which launches they are.
#include "split_tiles.h"

namespace sa {

namespace {

// Both in one launch (they share nothing but the inputs).
template <int DP, bool PART, bool EXACT>
__global__ void __launch_bounds__(64 * BWD_WAVES, DP <= 64 ? 2 : 1)
bwd_split_kernel(StepArgs p, int n_tiles, BothKinds kinds) {
    __shared__ __attribute__((aligned(1024))) char lds[BWD_WAVES * 2 * STAGE_BYTES<DP> + 2 * SUB_BYTES<DP>];
    __shared__ __attribute__((aligned(1024))) char stats[BWD_WAVES * 2 * STAT_BYTES];
    __shared__ uint32_t masks[BWD_WAVES];
    int linear = (int)blockIdx.x;
    if (owns_keys(kinds, linear)) bwd_dkdv<DP, PART, EXACT>(p, n_tiles, linear, lds, stats, masks);
    else bwd_dq<DP, PART, EXACT>(p, n_tiles, linear, lds, stats, masks);
}

enum Pass { FWD, FWD_EXACT, BWD_EXACT, BWD };
template <int DP, bool PART>
hipError_t run(const StepArgs& a, Pass pass, hipStream_t st) {
    const int n_tiles = (a.c + OWN - 1) / OWN;
    const int n_dkdv = n_tiles * a.n_kv * a.B * a.H_kv, n_dq = n_tiles * a.n_q * a.B * a.H;
    const bool forward = pass == FWD || pass == FWD_EXACT;
    // (short blocks, all key-owning ones first: 2048 heads of 16 rows, d 128, 124 -> 116 us, 512 of 96 98 -> 94, ring of 8 x
    // 96, 32 heads, 97 -> 92)
    const BothKinds kinds = both_kinds(a, n_dkdv, n_dq, pass == BWD_EXACT ? INFINITY : 1.25);
    const dim3 grid((unsigned)(forward ? n_dq : n_dkdv + n_dq)), block(64 * (forward ? FWD_WAVES : BWD_WAVES));
    if (pass == FWD && a.q_pos) {           // (d is 64 or 128: the other forms only exist for these)
        if constexpr ((DP == 64 || DP == 128) && !PART)
            hipLaunchKernelGGL((fwd_split_kernel<DP, PART, false, true>), grid, block, 0, st, a, n_tiles);
    } else if (pass == FWD) hipLaunchKernelGGL((fwd_split_kernel<DP, PART, false>), grid, block, 0, st, a, n_tiles);
    else if (pass == FWD_EXACT) hipLaunchKernelGGL((fwd_split_kernel<DP, PART, true>), grid, block, 0, st, a, n_tiles);
    else if (pass == BWD_EXACT) hipLaunchKernelGGL((bwd_split_kernel<DP, PART, true>), grid, block, 0, st, a, n_tiles, kinds);
    else hipLaunchKernelGGL((bwd_split_kernel<DP, PART, false>), grid, block, 0, st, a, n_tiles, kinds);
    return hipGetLastError();
}
template <int DP>
hipError_t run(const StepArgs& a, Pass pass, hipStream_t st) {
    return a.d % 8 ? run<DP, true>(a, pass, st) : run<DP, false>(a, pass, st);
}
hipError_t run(const StepArgs& a, Pass pass, hipStream_t st) {
    if (a.d <= 32 && a.d % 8 == 0) return run<32, false>(a, pass, st);
    if (a.d <= 64) return run<64>(a, pass, st);
    if (a.d <= 112) return run<112>(a, pass, st);
    return run<128>(a, pass, st);
}

// Both sides' rows come through descriptors with 32-bit byte offsets (fwd_tiles.h reads Q by 64-bit pointers, and
// fwd_mfma_supported looks at the rows of K and V only).  Requests behind a walk's end name up to 32 rows behind the
// block's last sub-tile: their offsets must not wrap into the matrix.
bool rows_in_reach(const StepArgs& a) {
    const int64_t widest = a.stride_s > a.kv_stride_s ? a.stride_s : a.kv_stride_s;
    return ((int64_t)(a.c + 127) / 128 * 128 + OWN) * 2 * widest + 2 * a.d < (int64_t(1) << 31);
}

}  // namespace

// (of shapes that the 128-row matrix-core kernels take.)  128-row kernels / these, us, d 128.
// Forward, by 128-row tiles of all queries: up to 64 always: 2 heads of 256 rows 11 / 8.4, one of 4096 61 / 22
// (full 61 / 24), ring of 4 x 1024, 2 heads 65 / 26.  128: triangular 64 heads of 200 12.1 / 13.0, 32 of 512 16 / 15, 8 of 2048 36 / 23;
// full 32 of 512 15.5 / 17.2, 8 of 2048 35.1 / 32.5, ring of 4 x 128, 32 heads, contiguous 15.1 / 15.4.  256:
// triangular 16 heads of 2048 39 / 42, 4 of 8192 122 / 108, ring of 4 x 1024, 8 heads 66.7 / 68.3, of
// 4 x 2048, 4 heads 121 / 112, full 8 of 4096 78 / 107; d 64: ring of 4 x 1024, 8 heads 49.7 / 45.9.  A single
// block of 128 rows is as well off in one 128-row tile up to 112 columns (d 64 7.9 / 8.3, d 128 10 / 8.5).  An odd number
// of heads has every XCD stream all of them, full blocks of 65 to 128 tiles above 64 columns: d 128, 11 heads of
// 1024 23.0 / 24.3, 13 of 1100 26.0 / 27.4, 15 of 1024 24.2 / 28.0, 9 of 1700 34.3 / 32.0, but 14 of 1152 25.2 / 23.6,
// 15 on 3 of 1024 22.5 / 21.0.  32 columns: 12 heads of 1000 rows, full, 13.8 / 9.8, 32 of 512 8.6 / 8.0; triangular 16
// of 2048 23.7 / 17.5, 32 of 1024 14.4 / 14.3.
bool narrow(const StepArgs& a) { return a.d <= 32 && a.d % 8 == 0; }          // 32 columns computed
bool fwd_split_wanted(const StepArgs& a) {
    const int64_t tiles = (int64_t)((a.c + 127) / 128) * a.B * a.n_q * a.H, walk = (int64_t)a.c * a.n_kv;
    if (a.d > TD || (walk <= 128 && a.d <= 112)) return false;
    if (!rows_in_reach(a)) return false;
    if (tiles <= 64) return true;
    if (tiles <= 128) return walk >= (a.layout == SA_STRIPED || narrow(a) ? 512 : a.d > 64 && a.H == a.H_kv && a.B * a.H % 2 ? 1536 : 1024);
    return tiles <= 256 && uneven(a) && walk >= (narrow(a) ? 2048 : a.d <= 112 ? 4096 : 8192);
}
hipError_t launch_fwd_split(const StepArgs& a, hipStream_t st) { return run(a, FWD, st); }
// Backward step, by 128-row tiles of all keys ("tiles") and key/value heads: four times the workgroups walk a quarter
// of the rows each, which pays while a head has many of them; a last 128-row tile that is nearly empty counts for it,
// so the heads are weighed by the square of what 32-row tiles save there.  Several hundred drawn shapes a line, geometric mean
// (worst) of 128-row time / this one:
//  * up to 64 tiles 1.2 to 2.3; full blocks above 64 columns 1.2 to 1.4 (1.0) up to 40 heads, beyond 1.0 (0.8)
//  * 65 to 128 tiles above 64 columns: triangular, walks of 2048 rows of the group and more, up to 8 heads 1.4 to 2.1
//    (1.2), 16 1.2 (1.05), 20 1.1 (0.9), 30 0.9 (0.8); full with groups of four and more, up to 16 heads 1.5 (1.0), 24 1.3
//    (1.0), 40 1.15 (0.9), beyond 0.9 (0.7); without groups 2 heads of 8192 rows 233 / 257 us
//  * 65 to 128 tiles up to 64 columns, where two workgroups fit a compute unit: 1.2 to 2.5 (1.0), full blocks of short
//    walks excepted (32 heads of 512 rows 19.6 / 18.3 us, but at d 32 16.1 / 17.0, 20 of 512 15.2 / 13.4)
//  * 129 to 512 tiles up to 64 columns, triangular: up to 24 heads 1.15 to 1.5 (1.05), 56 1.1 (0.94), 100 1.0 (0.85),
//    beyond 0.9 (0.7); 32 heads of 2048 rows (512 tiles) 99 / 99, d 32 80 / 82; full, 256: 46.4 / 45.8, 254 / 263
//  * 256 tiles above 64 columns: 8 heads of 4096 137 / 160, 32 on 8 of 4096 500 / 574
//  * 129 to 512 tiles, 32 columns computed, triangular: 32 heads of 1024 28.1 / 21.4 us in 128-row tiles, 16 of 2048 36.8 /
//    34.6, 8 of 4096 57 / 62, 8 of 8192 192 / 205; where the last round of 256 is not three quarters full, 8 of 3000 37 / 50,
//    16 of 3000 69 / 86; one device's queries against all shards' keys leave the 128-row kernel's queries' side short: 8
//    heads 4 x 1024 34 / 55, 4 heads 4 x 4096 136 / 218, 32 on 8 of 8 x 1024 124 / 158; 32 heads 2 x 512 25 / 22.  The rule
//    is 0.3 % (worst 1.2) behind the better kernel of each of 312 shapes
bool bwd_split_wanted(const StepArgs& a) {
    const int64_t t128 = (a.c + 127) / 128, t32 = (a.c + 31) / 32, heads = (int64_t)a.B * a.H_kv, group = a.H / a.H_kv;
    const int64_t keys = t128 * a.n_kv * heads, walk = (int64_t)a.c * a.n_q * group;
    auto up_to = [&](int64_t most) { return heads * t32 * t32 <= most * 16 * t128 * t128; };
    if (a.d > TD || !rows_in_reach(a)) return false;
    if (keys <= 64) return a.d <= 64 || uneven(a) || up_to(40);
    if (a.d > 64) return keys <= 128 && (uneven(a) ? walk >= 2048 && up_to(16) : group >= 4 && up_to(24));
    if (!uneven(a)) return keys <= 128 && walk >= (a.d <= 32 ? 6 : 4) * keys;
    if (keys > 128 && narrow(a)) {
        const int64_t queries = t128 * a.n_q * heads * group;
        if (keys > 512) return false;
        return 2 * queries <= keys ? walk >= 5 * queries : walk >= 12 * keys || (keys <= (keys <= 256 ? 192 : 384) && walk >= 6 * keys);
    }
    return up_to(56) && (keys <= 256 ? walk >= 4 * keys : keys <= 512 && walk > 4 * keys);
}
hipError_t launch_bwd_split(const StepArgs& a, hipStream_t st) { return run(a, BWD, st); }

// bf16 blocks shorter than a 128-row tile, probabilities and dS in fp32 precision.  Against the fp32 instruction on widened
// operands (f32_step.hip), us: forward step, d 128, 4 heads of 64 tokens 15.7 / 7.7, 64 of 96 17.1 / 8.3, 256 of
// 120 38.9 / 25.5, d 64 10.3 / 7.8, 11.1 / 8.0, 20.7 / 14.0, d 32 7.9 / 7.8, 8.0 / 7.8, 13.0 / 13.2 (7.7 is
// what a launch takes).  Error against 64 bits (2-norm, 16 x 127 tokens, d 128): O 2.2e-7 -> 1.6e-7, dQ
// 3.7e-7 -> 3.2e-7, dK 6.1e-7 -> 4.3e-7, dV 6.0e-7 -> 4.1e-7.  A single forward block of many heads stays with the fp32
// instruction up to 32 columns (half of the columns computed here are padding): d 16, 600 heads of 30 rows 10.0 / 11.0,
// 512 8.7 / 8.4, 400 heads of 60 11.4 / 13.1, of 96 15.1 / 16.1, of 127 18.5 / 21.2, 360 11.4 / 11.1, 15.1 / 16.1, 18.6 /
// 18.5; 1024 of 96 23.9 / 33.8, d 32 26.2 / 34.1, d 36 54 / 41.
bool short_exact_wanted(const StepArgs& a, int dtype, bool backward) {
    if (dtype != SA_BF16 || a.d % 4 || a.d > TD || a.c >= 128 || !rows_in_reach(a)) return false;
    return backward || a.n_kv > 1 || a.d > 32 || (int64_t)a.B * a.n_q * a.H <= (a.c <= 32 ? 512 : 384);
}
hipError_t launch_short_exact(const StepArgs& a, bool backward, hipStream_t st) {
    return run(a, backward ? BWD_EXACT : FWD_EXACT, st);
}

}  // namespace sa
