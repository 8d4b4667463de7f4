// Backward ring step on the matrix cores: its kernels (the workgroups' work: bwd_tiles.h, which says what bounds
// them), and which launches take which, in what order.
#include "bwd_tiles.h"
#include "packed.h"

namespace sa {

namespace {

// Head dimensions above 128, both column halves of dK and dV in one workgroup.  bwd_dkdv forms
// S and dP once per half: 12 products of d columns a pair where 8 do.  Here dK^T and dV^T of 32
// keys and 256 columns are the 256 accumulation registers of a wavefront (one per SIMD), the K rows
// 64 of its vector registers and the V rows WIDE_V_REGS k-steps there, the others in LDS, written and
// read by their own wavefront alone.  Q and dO come in stages of 32 rows, three in LDS: stage u + 2 is
// requested when everyone is done with u - 1 and has the whole step u to land, one barrier a step.
// The walk over blocks is the requests' own, two stages ahead; a step knows only its stage's limit
// of the element mask, which is far below zero where nothing is masked (64 matrix products a step
// hide the 16 selects).
// Bound by the matrix cores at the clock the power limit leaves: 8 instead of 12 products of d a pair,
// one wavefront per SIMD.  Backward step (with its dQ kernel), 8 heads of 8192 rows, d 256, full block
// 2210 -> 1761 us, triangular 1282 -> 1014; 12500 rows 6276 -> 5363, 2905 -> 2212; 16 heads of 4096 1166 ->
// 944, 708 -> 562.  One or two k-steps of V in registers measured the same.
constexpr int WIDE_ROWS = 32, WIDE_PART = WIDE_ROWS * 256;         // one 128-column half of a stage's Q or dO
constexpr int WIDE_STAGE = 4 * WIDE_PART;                          // Q, Q, dO, dO
constexpr int WIDE_V_REGS = 1;                                     // of 16 k-steps: what LDS has no room for
constexpr int WIDE_V_LDS = (16 - WIDE_V_REGS) * 1024;              // per wavefront
constexpr int WIDE_NO_MASK = -(1 << 20);

// products of one step, as dkdv_step.  arow: row reads in the next stage, tr0 / tr1: transposing reads
// in the present one.
template <bool NEXT>
__device__ __forceinline__ void wide_step(f32x16& s_cur, f32x16& dp_cur, f32x16& s_next, f32x16& dp_next,
                                 const bf16x8 (&kf)[16],
                                 const bf16x8 (&vf)[WIDE_V_REGS], const char* v_own, float kappa, const char* lds,
                                 const uint32_t (&arow)[8], const uint32_t (&tr0)[4], const uint32_t (&tr1)[4],
                                 const float* stat_cur, const float* stat_next, int h, int mask_lim) {
    bf16x8 qa[16], ga[16], va[16], qt[16], gt[16], pb[2], dsb[2];
    if (NEXT) load_neg_delta(dp_next, stat_next + WIDE_ROWS, h);
    auto fetch = [&](int ks) {
        if (!NEXT) return;
        const char* rows = lds + (ks / 8) * WIDE_PART;
        qa[ks] = dt_read_row(rows, arow[ks % 8]);
        ga[ks] = dt_read_row(rows + 2 * WIDE_PART, arow[ks % 8]);
        va[ks] = ks < WIDE_V_REGS ? vf[ks % WIDE_V_REGS] : dt_read_row(v_own, (ks - WIDE_V_REGS) * 1024);
    };
    // i = 8 (group of 16 rows) + column block
    auto fetch_t = [&](int i) {
        const char* rows = lds + (i % 8 / 4) * WIDE_PART + (i / 8) * 16 * 256;
        gt[i] = dt_read_tr(rows + 2 * WIDE_PART, tr0[i % 4], tr1[i % 4]);
        qt[i] = dt_read_tr(rows, tr0[i % 4], tr1[i % 4]);
    };
    float2 lv[8];
    auto fetch_stat = [&](int i) {
        lv[i] = *reinterpret_cast<const float2*>(stat_cur + 8 * (i / 2) + 4 * h + 2 * (i % 2));
    };
    constexpr int AHEAD = 2, TAHEAD = 3;
    fetch_stat(0);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fetch(i);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        __builtin_amdgcn_sched_barrier(0);          // slices stay in program order
        if (i + AHEAD < 16) fetch(i + AHEAD);
        if (i % 2 == 0 && i < 14) fetch_stat(i / 2 + 1);
        if (i >= 16 - TAHEAD) fetch_t(i - (16 - TAHEAD));
        if (NEXT) {
            if (i == 0) mfma_vgpr_first(s_next, qa[i], kf[i], false);
            else mfma_vgpr_acc(s_next, qa[i], kf[i], false);
            __builtin_amdgcn_sched_barrier(0);
        }
        const float lr = i % 2 ? lv[i / 2].y : lv[i / 2].x;
        float pr = __builtin_amdgcn_exp2f(fmaf(s_cur[i], kappa, -lr));
        if (8 * (i / 4) + (i % 4) < mask_lim) pr = 0.f;
        pb[i / 8][i % 8] = (__bf16)pr;
        dsb[i / 8][i % 8] = (__bf16)(pr * dp_cur[i]);
        if (NEXT) {
            __builtin_amdgcn_sched_barrier(0);
            mfma_vgpr_acc(dp_next, ga[i], va[i], false);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        if (i + TAHEAD < 16) fetch_t(i + TAHEAD);
        acc_mfma(i % 8, gt[i], pb[i / 8]);
        acc_mfma(8 + i % 8, qt[i], dsb[i / 8]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Args: StepArgs, or PackedArgs for packed sequences (packed.h), whose rows are written in bf16
template <bool BY_RANK, typename Args = StepArgs>
__global__ void __launch_bounds__(256, 1)
bwd_dkdv_wide_kernel(Args p, int n_tiles) {
    constexpr bool PACKED = !std::is_same<Args, StepArgs>::value;
    __shared__ __attribute__((aligned(1024))) char lds[3 * WIDE_STAGE];
    __shared__ __attribute__((aligned(1024))) char v_lds[4 * WIDE_V_LDS];
    __shared__ __attribute__((aligned(16))) float stat[3 * 2 * WIDE_ROWS];         // [stage][lse2 | -delta][32]
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int ktile, bh, dev_rank;
    if constexpr (PACKED) {
        if (!enter_sequence<false, BM>(p, (int)blockIdx.x, p.H_kv, n_tiles, ktile, bh)) return;
    } else {
        decode_block<false, BY_RANK>((int)blockIdx.x, n_tiles * p.n_kv, p.B * p.H_kv, ktile, bh);
    }
    decode_rank(ktile, n_tiles, p.n_kv, p.layout, ktile, dev_rank);
    const int dev = p.kv_dev + dev_rank;
    const int b = bh / p.H_kv, kvh = bh - b * p.H_kv;
    const int64_t kv_base = b * p.kv_stride_b + kvh * p.kv_stride_h + (dev - p.kv_dev) * p.kv_shard;
    const int d = p.d;
    const int64_t ss = p.kv_stride_s;
    const int pitch = 2 * (int)p.stride_s, stage_pitch = WIDE_ROWS * pitch;
    const int k0 = ktile * BM, key_own = k0 + 32 * wave + n, key = min(key_own, p.c - 1);

    // The requests: query head, query shard and 32-row stage of the next one, as in the kernel above.
    const int group = p.H / p.H_kv;
    const int dev0 = p.layout != SA_STRIPED ? max(p.q_dev, dev) : p.q_dev, n_st = (p.c + DT_ROWS - 1) / DT_ROWS * 2;
    int q_head = 0, q_dev = dev0, t, lim;           // lim: mask limit of stage 0 but for the lane's part
    dt_rsrc Qr, Gr;
    const float* stat_src;
    auto enter_block = [&]() {
        const int hd = kvh * group + q_head;
        const bool tri = block_kind(q_dev, dev, p.layout) == MASK_TRI;
        const int off = block_off(q_dev, dev, p.layout);
        t = tri ? k0 / WIDE_ROWS : 0;
        if (tri && p.skip_bq > 0)
            t = ((k0 / p.skip_bk * p.skip_bk + off) / p.skip_bq) * p.skip_bq / WIDE_ROWS;
        lim = tri ? k0 + 32 * wave + off : WIDE_NO_MASK;
        const int64_t base = b * p.stride_b + hd * p.stride_h + (q_dev - p.q_dev) * p.q_shard;
        const int64_t sbase = b * p.stat_stride_b + hd * p.stat_stride_h + (int64_t)(q_dev - p.q_dev) * p.c;
        Qr = dt_make_rsrc((const __bf16*)p.q + base, p.c, pitch, d);
        Gr = dt_make_rsrc((const __bf16*)p.dout + base, p.c, pitch, d);
        stat_src = ((tid & WIDE_ROWS) ? p.delta : p.lse) + sbase;
    };
    enter_block();
    uint32_t gl[2][2];
#pragma unroll
    for (int hh = 0; hh < 2; ++hh)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = 8 * wave + 4 * j + (lane >> 4), chunk = (lane & 15) ^ dt_swz(r);
            gl[hh][j] = 128 * hh + 8 * chunk < d ? r * pitch + 256 * hh + (chunk << 4) : DT_OUT_OF_RANGE;
        }
    float rstat;                                    // statistics of the stage requested last
    int lim_req;                                    // and its limit
    bool more = true;                               // stages are left to request
    auto request = [&](int stage) {
        const int at = t * stage_pitch;
        char* dst = lds + stage * WIDE_STAGE + 2 * wave * 1024;
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                dt_load_piece(Qr, at, gl[hh][j], dst + hh * WIDE_PART + j * 1024);
                dt_load_piece(Gr, at, gl[hh][j], dst + (2 + hh) * WIDE_PART + j * 1024);
            }
        const int row = t * WIDE_ROWS + (tid & (WIDE_ROWS - 1));
        rstat = stat_src[min(row, p.c - 1)];
        if (row >= p.c) rstat = (tid & WIDE_ROWS) ? 0.f : INFINITY;       // no query: P and dS are exact zeros
        lim_req = lim == WIDE_NO_MASK ? lim : lim - t * WIDE_ROWS;
        if (++t == n_st) {
            if (++q_dev == p.q_dev + p.n_q) {
                q_dev = dev0;
                more = ++q_head < group;
            }
            if (more) enter_block();
        }
    };
    auto stat_store = [&](int stage) {
        if (tid < 2 * WIDE_ROWS) stat[stage * 2 * WIDE_ROWS + tid] = rstat * ((tid & WIDE_ROWS) ? -1.f : LOG2E);
    };

    bf16x8 kf[16], vf[WIDE_V_REGS];
    char* const v_own = v_lds + wave * WIDE_V_LDS + lane * 16;
    {
        bf16x8 v_all[16];
        if constexpr (PACKED) load_b_frags<16>(v_all, (const __bf16*)p.v + kv_base, p.c, 2 * (int)ss, key, h, d);
        else load_b_frags<16>(v_all, (const __bf16*)p.v + kv_base + (int64_t)key * ss, h, d);
#pragma unroll
        for (int ks = 0; ks < 16; ++ks) {
            if (ks < WIDE_V_REGS) vf[ks % WIDE_V_REGS] = v_all[ks];
            else *reinterpret_cast<bf16x8*>(v_own + (ks - WIDE_V_REGS) * 1024) = v_all[ks];
        }
    }
    if constexpr (PACKED) load_b_frags<16>(kf, (const __bf16*)p.k + kv_base, p.c, 2 * (int)ss, key, h, d);
    else load_b_frags<16>(kf, (const __bf16*)p.k + kv_base + (int64_t)key * ss, h, d);
    request(0);
    const int lim_first = lim_req;
    stat_store(0);
    request(1);
    uint32_t arow[8], tr0[4], tr1[4];
    dt_row_addrs<256>(arow, n, h);
    dt_tr_addrs<256>(tr0, tr1, lane);
    const float kappa = p.scale * LOG2E;
#pragma unroll
    for (int r = 0; r < 256; ++r) acc_zero(r);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();

    f32x16 s_a, s_b, dp_a, dp_b;
    load_neg_delta(dp_a, stat + WIDE_ROWS, h);
#pragma unroll
    for (int ks = 0; ks < 16; ++ks) {
        const char* rows = lds + (ks / 8) * WIDE_PART;
        const bf16x8 qx = dt_read_row(rows, arow[ks % 8]), gx = dt_read_row(rows + 2 * WIDE_PART, arow[ks % 8]);
        const bf16x8 vx = ks < WIDE_V_REGS ? vf[ks % WIDE_V_REGS] : dt_read_row(v_own, (ks - WIDE_V_REGS) * 1024);
        if (ks == 0) mfma_vgpr_first(s_a, qx, kf[ks], false);
        else mfma_vgpr_acc(s_a, qx, kf[ks], false);
        mfma_vgpr_acc(dp_a, gx, vx, false);
    }
    mfma_results_to_valu(s_a, dp_a);

    // stage: of the present step.  The row reads are one stage further on.
    int stage = 0, ahead = 2, lim_cur = lim_first, lim_next = lim_req;         // ahead: stages requested and not done
    auto after = [](int x) { return x == 2 ? 0 : x + 1; };
    auto move = [&](uint32_t (&a)[8], int from) {
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] += from == 2 ? -2 * WIDE_STAGE : WIDE_STAGE;
    };
    move(arow, 0);
    auto step = [&](f32x16& s_cur, f32x16& dp_cur, f32x16& s_next, f32x16& dp_next) {
        const int next = after(stage), free = after(next);
        stat_store(next);
        __builtin_amdgcn_s_waitcnt(0);              // the next stage has landed
        __syncthreads();                            // for everyone; everyone is done with the one before this
        if (more) {
            request(free);
            ++ahead;
        }
        wide_step<true>(s_cur, dp_cur, s_next, dp_next, kf, vf, v_own, kappa, lds, arow, tr0, tr1,
                        stat + stage * 2 * WIDE_ROWS, stat + next * 2 * WIDE_ROWS, h, lim_cur + n - 4 * h);
        lim_cur = lim_next;
        lim_next = lim_req;
        move(arow, next);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            tr0[i] += stage == 2 ? -2 * WIDE_STAGE : WIDE_STAGE;
            tr1[i] += stage == 2 ? -2 * WIDE_STAGE : WIDE_STAGE;
        }
        stage = next;
        --ahead;
    };
    for (;;) {          // every block has an even number of stages
        step(s_a, dp_a, s_b, dp_b);
        if (ahead == 1) break;
        step(s_b, dp_b, s_a, dp_a);
    }
    wide_step<false>(s_b, dp_b, s_a, dp_a, kf, vf, v_own, kappa, lds, arow, tr0, tr1,
                     stat + stage * 2 * WIDE_ROWS, stat, h, lim_cur + n - 4 * h);

    acc_settle();
    if constexpr (PACKED) {
        const int64_t row = kv_base + (int64_t)key * ss;
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            bf16x4 x[2], y[2];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e / 4][e % 4] = (__bf16)acc_read(4 * i + e);
                y[e / 4][e % 4] = (__bf16)(p.scale * acc_read(128 + 4 * i + e));
            }
            store_two_chunks((__bf16*)p.dv + row, 8 * i, x[0], x[1], key_own < p.c, h, d);
            store_two_chunks((__bf16*)p.dk + row, 8 * i, y[0], y[1], key_own < p.c, h, d);
        }
        return;
    }
    if (key_own >= p.c) return;
    float* DK = p.dk + kv_base + (int64_t)key * ss;
    float* DV = p.dv + kv_base + (int64_t)key * ss;
#pragma unroll
    for (int mb = 0; mb < 8; ++mb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int col = 32 * mb + 8 * g + 4 * h;
            if (col >= d) continue;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
            if (!p.fresh) {
                x = *reinterpret_cast<float4*>(DV + col);
                y = *reinterpret_cast<float4*>(DK + col);
            }
            x.x += acc_read(16 * mb + 4 * g + 0); x.y += acc_read(16 * mb + 4 * g + 1);
            x.z += acc_read(16 * mb + 4 * g + 2); x.w += acc_read(16 * mb + 4 * g + 3);
            *reinterpret_cast<float4*>(DV + col) = x;
            y.x = fmaf(p.scale, acc_read(128 + 16 * mb + 4 * g + 0), y.x); y.y = fmaf(p.scale, acc_read(128 + 16 * mb + 4 * g + 1), y.y);
            y.z = fmaf(p.scale, acc_read(128 + 16 * mb + 4 * g + 2), y.z); y.w = fmaf(p.scale, acc_read(128 + 16 * mb + 4 * g + 3), y.w);
            *reinterpret_cast<float4*>(DK + col) = y;
        }
}

template <bool RAGGED, int WALK, int DP, bool PART, bool BY_RANK>
__global__ void __launch_bounds__(256, DP > 128 ? 1 : 2)
bwd_dq_mfma_kernel(StepArgs p, int n_tiles) {
    __shared__ __attribute__((aligned(1024))) char lds0[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds1[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds2[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds3[tile_bytes(DP) * halves_of(DP)];
    bwd_dq<RAGGED, WALK, DP, PART, BY_RANK>(p, n_tiles, (int)blockIdx.x, lds0, lds1, lds2, lds3);
}
// WAVES: wavefronts per SIMD the register budget is cut for.  Up to 64 columns two fit (half the
// operands and accumulators; the loops do not spill), and with half of the products per score it is
// the vector work that needs hiding: 16 heads, d 64, backward step, 12500 tokens triangular
// 1.46 -> 1.37 ms, full 2.87 -> 2.46; 32 heads of 32768, triangular, 17.3 -> 14.7 ms.
template <int WALK, bool RAGGED, int DP, bool PART, int WAVES, bool BY_RANK>
__global__ void __launch_bounds__(256, WAVES)
bwd_dkdv_mfma_kernel(StepArgs p, int n_tiles) {
    __shared__ __attribute__((aligned(1024))) char lds0[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds1[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds2[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds3[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(16))) float stat[KV_STAT_FLOATS];
    bwd_dkdv<WALK, RAGGED, DP, PART, BY_RANK>(p, n_tiles, (int)blockIdx.x, lds0, lds1, lds2, lds3, stat);
}
// Both kinds of workgroups in one launch (each sequence heaviest first; above 512 of a kind by groups of
// heads, see decode_block): where the key-owning ones do not fill the chip, or fill it once and last
// as long as the heaviest, the query-owning ones run beside and behind them instead of after.
// One workgroup per compute unit (the key-owning side's registers).  Up to 64 columns and above 128.
template <bool RAGGED, int DP, bool PART>
__global__ void __launch_bounds__(256, 1)
bwd_both_mfma_kernel(StepArgs p, int n_tiles, PlacedKinds kinds) {
    __shared__ __attribute__((aligned(1024))) char lds0[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds1[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds2[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds3[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(16))) float stat[KV_STAT_FLOATS];
    int linear = (int)blockIdx.x;
    const int keys = __builtin_amdgcn_readfirstlane(owns_keys(kinds, linear));
    linear = __builtin_amdgcn_readfirstlane(linear);        // (both kept scalar)
    if (keys) bwd_dkdv<WALK_RING, RAGGED, DP, PART, false>(p, n_tiles, linear, lds0, lds1, lds2, lds3, stat);
    // (by heads or groups of them, both)
    else bwd_dq<RAGGED, WALK_RING, DP, PART, false>(p, n_tiles, linear, lds0, lds1, lds2, lds3);
}

}  // namespace

bool bwd_mfma_supported(const StepArgs& a, int dtype) {
    // the tile loads address a shard through a buffer descriptor with 32-bit byte offsets:
    // the last row of its last (possibly partial) tile pair must end below 2^31 bytes from
    // its first
    const int64_t widest = a.stride_s > a.kv_stride_s ? a.stride_s : a.kv_stride_s;
    const int64_t rows = (int64_t)(a.c + BM - 1) / BM * BM;
    // one workgroup per (128-row tile, device, batch, head) in a 1-D grid
    if (rows / BM * a.B * a.H * (a.n_q > a.n_kv ? a.n_q : a.n_kv) >= (int64_t(1) << 31)) return false;
    // head dimensions above 128 (two 128-column halves) in whole 16-byte chunks only
    if (a.d > 2 * D || (a.d > D && a.d % 8)) return false;
    return dtype == SA_BF16 && a.d % 4 == 0 && a.c >= BM &&
           rows * 2 * widest + 2 * a.d < (int64_t(1) << 31);
}

// Key-owning workgroups by ranks (decode_block).  Above 128 columns up to 1408 tiles; d 192 and 256, triangular step, us,
// groups : ranks: 24 heads of 4096 529 : 465, 540 : 472, 44 of 4096 856 : 815, 897 : 878, 48 of 4096 849 : 891, 1030 : 1073,
// 64 of 4096 1134 : 1217, 1186 : 1357; heads of few tiles a round or two more, whole backward, 384 of 512 624 : 592, 512 of 512
// 872 : 851, 192 of 1024 .98.
// A device's own queries against more shards of keys: every walk is that device's rows, and short ones leave little to
// balance while an XCD's heads, all at a time, fall out of its L2.  Striped shares, whole backward, groups : ranks: d 128,
// 32 heads 4 x 1024 195 : 211, 64 of 4 x 1024 346 : 390, d 100, 64 of 4 x 1000 319 : 342, d 256, 32 of 8 x 512 340 : 434, of
// 2 x 2048 1 : 1.05; but 64 columns, 32 of 2 x 4096 1 : .94, 64 of 2 x 1024 124 : 118, up to three rounds 24 of 4 x 1000 1 :
// .96, 24 of 2 x 2048 1 : .94, and with 32 columns computed, whose rows are few bytes, all: 64 of 2 x 1024 78 : 70, 32 of 8 x
// 1024 155 : 150.
bool dkdv_by_rank(const StepArgs& a) {
    const int64_t ranks = (int64_t)((a.c + BM - 1) / BM) * a.n_kv, tiles = ranks * a.B * a.H_kv, walk = (int64_t)a.c * a.n_q * (a.H / a.H_kv);
    if (!by_rank(uneven(a), tiles, a.d > 128 ? (ranks <= 4 ? 8 * N_CU : ranks <= 8 ? 6 * N_CU : 6 * N_CU - 1) : a.d > 112 ? MOST_BY_RANK<128, false> : MOST_BY_RANK<64, false>)) return false;
    if (a.n_kv <= a.n_q || a.d <= 32) return true;
    return walk > (a.d > 128 ? 2048 : 2047) || (walk > 512 && tiles <= (a.d <= 112 && a.n_kv <= 2 * a.n_q ? 4 : 3) * N_CU);
}

// Both kinds of workgroups in one launch.  Measured per backward step, one launch / two, us.  Up to 64 columns and above 128 (this
// file's kernels; measured at d 128, when they ran there too): uneven work up to one key-owning workgroup per compute unit: 2048 x
// 2048 triangular, 2 heads 60 / 102, 8 heads 66 / 106, 16 heads (256 workgroups) 92 / 115, 24 heads 137 / 131.  Even work (a full
// block) has no tail to fill, only idle compute units: 128 + 128 workgroups 75 / 108, 256 + 256 144 / 133.  d 256 (two
// key-owning workgroups per tile): 256 of them 109 / 189, 512 207 / 225.
// 65 to 128 columns (bwd_ring.hip, whose query-owning workgroups lose less where one is alone on its compute unit), d 128 and d 100:
//  * uneven work, key tiles: 192 (16 heads of 1536) 51 / 83, 44 / 78, 256 (16 of 2048) 75 / 104, 67 / 98, (32 on 8 of 4096) 452 / 546,
//    419 / 525, 294 (3 of 12500) 392 / 525, 364 / 510, 320 (10 of 4096) 170 / 199, 147 / 186, (20 of 2048) 101 / 111, 88 / 104, (5 of 8192) 292 /
//    361, 270 / 348, 384 (12 of 4096) 191 / 203, 174 / 193, (24 of 2048) 113 / 119, 101 / 109; behind the line 512 (16 of 4096) 263 / 248;
//    four query heads to a key/value head 320 (10 of 4096) 582 / 622, 539 / 591, behind the line 384 699 / 692;
//  * of these, walks of many blocks of two or three tiles: two launches again from 257 key tiles on.  The kinds go out evenly (see
//    launch_both) and the last key walks start late: 987 heads on 141 of 256 rows, d 96, 164 / 144, 1540 on 140 of 235, d 80, 224 /
//    190, 240 on 80, 2 x 253 rows, d 128, 139 / 123; but one tile, 2264 on 283 of 128 rows, d 100, 167 / 196, four, 455 on 65 of 512 205 /
//    210, twelve, 152 on 19 of 1445 351 / 410;
//  * a full block, workgroups of both kinds: 256 (8 heads of 2048) 65 / 99, 59 / 96, 320 (10 of 2048) 93 / 102, 87 / 99, (40 of 512) 38 / 45, 34 / 41,
//    352 (44 of 512) 43 / 45, 38 / 43; behind the line 384 (12 of 2048) 110 / 107;
//  * one device's queries against more shards of keys: its query-owning workgroups, one round at most, walk all of them, and the
//    others fill the chip meanwhile.  Striped, device 7 of 8: 4 heads of 2048 295 / 367, 293 / 361, 16 of 1024 173 / 258, 166 / 248, 32 of
//    1024 (256 and 2048 tiles) 332 / 393, 297 / 353, 32 on 8 of 1024 285 / 323, 263 / 305; 2 of 8192, N 4, 609 / 805, 592 / 789;
//    contiguous 8 of 2048, N 4, 208 / 276, 196 / 266, 4 of 4096, N 8, 797 / 1027, 743 / 991; behind the line, with the key walks in front,
//    64 of 1024, N 4 (512 query tiles) 393 / 342, 32 of 896, N 16 (3584 key tiles) 860 / 658.
bool bwd_one_launch(const StepArgs& a) {
    const int n_tiles = (a.c + BM - 1) / BM, halves = a.d > D ? 2 : 1, group = a.H / a.H_kv;
    const int64_t keys = (int64_t)n_tiles * a.n_kv * a.B * a.H_kv * halves, queries = (int64_t)n_tiles * a.n_q * a.B * a.H;
    if (a.d <= 64 || a.d > D) return uneven(a) ? keys <= N_CU * halves : keys + queries <= N_CU;
    if (a.n_kv > a.n_q && queries <= N_CU && keys <= 8 * N_CU) return true;
    if (!uneven(a)) return keys + queries <= 11 * N_CU / 8;
    if (keys > N_CU && (n_tiles == 2 || n_tiles == 3) && (int64_t)group * a.n_q > 5) return false;
    return keys <= (group < 4 ? 6 : 5) * N_CU / 4;
}

namespace {
template <int WALK, int DP, bool PART, bool BY_RANK = false>
void launch_dq(const StepArgs& a, hipStream_t st, int n_tiles) {
    const dim3 grid((unsigned)n_tiles * a.n_q * a.B * a.H), block(256);
    if constexpr (WALK != WALK_FULL && !BY_RANK)
        // (between 64 and 128 columns computed many heads or few tiles lose, us, groups : ranks: d 100, whole backward, 336 heads of
        // 384 153 : 162, 256 of 2 x 512 409 : 422, 512 of 768 627 : 648)
        if (by_rank(uneven(a), grid.x, MOST_BY_RANK<DP, false>) && (DP != 112 || (a.B * a.H <= 192 && n_tiles * a.n_q >= 4))) return launch_dq<WALK, DP, PART, true>(a, st, n_tiles);
    if (a.c % BM) hipLaunchKernelGGL((bwd_dq_mfma_kernel<true, WALK, DP, PART, BY_RANK>), grid, block, 0, st, a, n_tiles);
    else hipLaunchKernelGGL((bwd_dq_mfma_kernel<false, WALK, DP, PART, BY_RANK>), grid, block, 0, st, a, n_tiles);
}
template <int WALK, int DP, bool PART, int WAVES, bool BY_RANK = false>
void launch_dkdv_waves(const StepArgs& a, hipStream_t st, int n_tiles) {
    const dim3 grid((unsigned)n_tiles * a.n_kv * a.B * a.H_kv * halves_of(DP)), block(256);
    if constexpr (WALK != WALK_FULL && DP <= 128 && !BY_RANK)          // (above: bwd_dkdv_wide_kernel)
        if (dkdv_by_rank(a)) return launch_dkdv_waves<WALK, DP, PART, WAVES, true>(a, st, n_tiles);
    if (a.c % BM) hipLaunchKernelGGL((bwd_dkdv_mfma_kernel<WALK, true, DP, PART, WAVES, BY_RANK>), grid, block, 0, st, a, n_tiles);
    else hipLaunchKernelGGL((bwd_dkdv_mfma_kernel<WALK, false, DP, PART, WAVES, BY_RANK>), grid, block, 0, st, a, n_tiles);
}
template <int WALK, int DP, bool PART>
void launch_dkdv(const StepArgs& a, hipStream_t st, int n_tiles) {
    if constexpr (DP <= 64) {
        // Uneven work that two workgroups per compute unit would hold all at once, or whose longest walk is
        // short, is better taken up one after the other, heaviest first (triangular, whole step: 512
        // workgroups of 4096 rows 0.168 against 0.177 ms; 768 of 1024, 2048 and 4096 rows 116 / 124, 157 /
        // 173, 266 / 257 us; 1536 of 2048 and 4096 291 / 304, 460 / 458).
        const int64_t wgs = (int64_t)n_tiles * a.n_kv * a.B * a.H_kv;
        if (!uneven(a) || (wgs > 2 * N_CU && n_tiles >= 32))
            return launch_dkdv_waves<WALK, DP, PART, 2>(a, st, n_tiles);
    }
    launch_dkdv_waves<WALK, DP, PART, 1>(a, st, n_tiles);
}
template <int DP, bool PART>
hipError_t launch_both(const StepArgs& a, hipStream_t st, int n_tiles) {
    const int n_dkdv = n_tiles * a.n_kv * a.B * a.H_kv * halves_of(DP), n_dq = n_tiles * a.n_q * a.B * a.H;
    // (The ratio, and none for groups: a group's long key walks in front are no gain.  25 calls of 65 to 384 key tiles with
    // bwd_ring.hip's kernels, at d 128 and d 100, time against these: ratio 1.25 0.98 to 1.02, 1.7 0.97 to 1.03; for groups 0.35
    // 0.99 to 1.05, 0.5 0.98 to 1.04: 455 heads on 65 of 512 rows 205 / 211 and 214 us, 32 on 8 of 4096 463 / 461 and 456.)
    // (numbers that are no multiple of 8 one by one: 11 heads of 1600 rows, d 136, 92 us, in units of 8 97; those that are:
    // see both_kinds)
    const double ratio = a.H == a.H_kv ? 1.45 : 0.;
    const PlacedKinds kinds = placed_kinds(a, n_dkdv, n_dq, ratio);
    if constexpr (DP == 112 || DP == 128) {
        return launch_bwd_ring(a, &kinds, n_dkdv + n_dq, st);
    } else {
        const dim3 grid((unsigned)(n_dkdv + n_dq)), block(256);
        if (a.c % BM) hipLaunchKernelGGL((bwd_both_mfma_kernel<true, DP, PART>), grid, block, 0, st, a, n_tiles, kinds);
        else hipLaunchKernelGGL((bwd_both_mfma_kernel<false, DP, PART>), grid, block, 0, st, a, n_tiles, kinds);
        return hipGetLastError();
    }
}
template <int DP, bool PART>
hipError_t launch_bwd_variant(const StepArgs& a, hipStream_t st) {
    const int n_tiles = (a.c + BM - 1) / BM;
    if (bwd_one_launch(a)) return launch_both<DP, PART>(a, st, n_tiles);
    const bool one_block = a.n_q == 1 && a.n_kv == 1 && !a.fresh;
    const bool full = block_kind(a.q_dev, a.kv_dev, a.layout) == MASK_FULL;
    if (!one_block) launch_dq<WALK_RING, DP, PART>(a, st, n_tiles);
    else if (full) launch_dq<WALK_FULL, DP, PART>(a, st, n_tiles);
    else launch_dq<WALK_TRI, DP, PART>(a, st, n_tiles);
    if (hipError_t e = hipGetLastError()) return e;
    if constexpr (DP > 128) {
        // Up to half a key tile per compute unit the two column halves side by side are faster: a wide workgroup
        // lasts 4 / 3 as long.  Full block, d 256, us, halves : wide: 128 tiles (8 heads of 2048) 197 : 224, (32
        // heads on 4 of 4096) 2251 : 2718, 144 278 : 228, 192 280 : 227, 256 315 : 256, 320 475 : 463.  Triangular
        // blocks of up to 256 tiles went to launch_both (16 heads of 2048 204 : 218, 8 of 4096 342 : 385; above it
        // 320 tiles 285 : 239).
        const int64_t tiles = (int64_t)n_tiles * a.n_kv * a.B * a.H_kv;
        if (tiles > N_CU / 2) {
            if (dkdv_by_rank(a)) hipLaunchKernelGGL(bwd_dkdv_wide_kernel<true>, dim3((unsigned)tiles), dim3(256), 0, st, a, n_tiles);
            else hipLaunchKernelGGL(bwd_dkdv_wide_kernel<false>, dim3((unsigned)tiles), dim3(256), 0, st, a, n_tiles);
            return hipGetLastError();
        }
    }
    if constexpr (DP == 112 || DP == 128) return launch_bwd_ring(a, nullptr, n_tiles * a.n_kv * a.B * a.H_kv, st);
    // query heads that share a key/value head are blocks of one walk
    else if (!one_block || a.H != a.H_kv) launch_dkdv<WALK_RING, DP, PART>(a, st, n_tiles);
    else if (full) launch_dkdv<WALK_FULL, DP, PART>(a, st, n_tiles);
    else if constexpr (DP <= 128) launch_dkdv<WALK_TRI, DP, PART>(a, st, n_tiles);      // above: launch_both or wide
    return hipGetLastError();
}
}  // namespace

hipError_t launch_bwd_mfma(const StepArgs& a, hipStream_t st) {
    const bool part = a.d % 8 != 0;
    if (a.d > 128) return launch_bwd_variant<256, false>(a, st);
    if (a.d <= 32 && !part) return launch_bwd_variant<32, false>(a, st);
    if (a.d <= 64) return part ? launch_bwd_variant<64, true>(a, st) : launch_bwd_variant<64, false>(a, st);
    if (a.d <= 112) return part ? launch_bwd_variant<112, true>(a, st) : launch_bwd_variant<112, false>(a, st);
    return part ? launch_bwd_variant<128, true>(a, st) : launch_bwd_variant<128, false>(a, st);
}

hipError_t launch_packed_dkdv_wide(const PackedArgs& p, unsigned workgroups, hipStream_t st) {
    hipLaunchKernelGGL((bwd_dkdv_wide_kernel<false, PackedArgs>), dim3(workgroups), dim3(256), 0, st, p, 0);
    return hipGetLastError();
}

}  // namespace sa
