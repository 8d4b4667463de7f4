// dK and dV above 128 columns, all columns in one workgroup.
#pragma once
#include "acc_file.h"
#include "bwd_tiles.h"
#include "packed.h"

namespace sa {

namespace {

// Head dimensions above 128, both column halves of dK and dV in one workgroup.  The kernel above forms
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
        load_b_frags<16>(v_all, (const __bf16*)p.v + kv_base + (int64_t)key * ss, h, d);
#pragma unroll
        for (int ks = 0; ks < 16; ++ks) {
            if (ks < WIDE_V_REGS) vf[ks % WIDE_V_REGS] = v_all[ks];
            else *reinterpret_cast<bf16x8*>(v_own + (ks - WIDE_V_REGS) * 1024) = v_all[ks];
        }
    }
    load_b_frags<16>(kf, (const __bf16*)p.k + kv_base + (int64_t)key * ss, h, d);
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
    if (key_own >= p.c) return;
    if constexpr (PACKED) {
        const int64_t row = kv_base + (int64_t)key * ss;
#pragma unroll
        for (int mb = 0; mb < 8; ++mb)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int col = 32 * mb + 8 * g + 4 * h;
                if (col >= d) continue;
                bf16x4 x, y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = (__bf16)acc_read(16 * mb + 4 * g + e);
                    y[e] = (__bf16)(p.scale * acc_read(128 + 16 * mb + 4 * g + e));
                }
                *reinterpret_cast<bf16x4*>((__bf16*)p.dv + row + col) = x;
                *reinterpret_cast<bf16x4*>((__bf16*)p.dk + row + col) = y;
            }
        return;
    }
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

}  // namespace

}  // namespace sa
