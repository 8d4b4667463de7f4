// Attention with a window (window.h), backward: what rows beyond the windows add to dK and dV of a sequence's first keys.
//
// A workgroup takes 16 keys, a part of the sequence's rows and, one after the other, the query heads of its group, as decode.hip takes heads and cached
// tokens: rows of Q and dO go from memory to the registers that the products want, once as they lie (S = Q K^T and dP = dO V^T, a lane holding
// rows 4 j + r of key n) and once turned round in registers (dV^T += dO^T P, dK^T += Q^T dS).  P comes from the rows' LSE.  Four wavefronts take tiles of rows in
// turn, their sums meet in LDS.  In bf16 P and dS meet dO and Q as bf16, as in the other kernels.  (At 256 columns 40 registers are spilled, in fp32 74.)
//
// Bound by the latency of its reads: Q and dO are read once more, in both orders (the second from the caches).  2 sequences of up to 16384 rows, 16 heads
// on 8, bf16, 128 columns: 52 us, 2.9 TB/s; joining the parts' sums 17.
#include <hip/hip_bf16.h>

#include "mfma_tiles.h"
#include "window.h"

namespace sa {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t Whole __attribute__((ext_vector_type(4), aligned(8)));       // 16 bytes of a row

constexpr int WAVES = 4, KEYS = 16, BATCH = 8;

template <typename T, int DP> struct Of;        // as in decode.hip
template <int DP> struct Of<__hip_bfloat16, DP> {
    static constexpr int TILE = 32, STEP = 32, CW = DP >= 128 ? 8 : DP / 16, ES = 2;
};
template <int DP> struct Of<float, DP> {
    static constexpr int TILE = 16, STEP = 16, CW = DP >= 64 ? 4 : DP / 16, ES = 4;
};

__device__ inline f32x4 product(u32x4 a, u32x4 b, f32x4 c, __hip_bfloat16*) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ inline f32x4 product(u32x4 a, u32x4 b, f32x4 c, float*) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
    return c;
}

// The 16 bytes of a row from column col on, zeros from column d on; nothing beyond the row is read.
template <typename T>
__device__ inline u32x4 load_chunk(const T* row, int col, int d) {
    constexpr int E = 16 / (int)sizeof(T);
    if (E == 8 && d < 8) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(row);
        return col == 0 ? u32x4{x[0], x[1], 0, 0} : u32x4{0, 0, 0, 0};
    }
    const Whole x = *reinterpret_cast<const Whole*>(row + min(col, d - E));
    if (col + E <= d) return x;
    return E == 8 && col < d ? u32x4{x[2], x[3], 0, 0} : u32x4{0, 0, 0, 0};
}
// CW columns from col on, as dwords; of columns beyond the row anything
template <typename T, int CW>
__device__ inline void load_columns(uint32_t (&to)[CW * sizeof(T) / 4], const T* row, int col, int d) {
    constexpr int BYTES = CW * (int)sizeof(T);
    if constexpr (BYTES == 16) {
        const u32x4 x = load_chunk<T>(row, col, d);
        to[0] = x[0]; to[1] = x[1]; to[2] = x[2]; to[3] = x[3];
    } else if constexpr (BYTES == 8) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(row + min(col, d - CW));
        to[0] = x[0]; to[1] = x[1];
    } else {
        to[0] = *reinterpret_cast<const uint32_t*>(row + min(col, d - CW));
    }
}

// A workgroup's slot, key/value head and block of keys, slots first
struct Place { int slot, kvh, block; };
__device__ inline Place place_of(const WindowArgs& p, int block0) {
    const int rest = (int)blockIdx.x / p.n_slots;
    return {(int)blockIdx.x % p.n_slots, rest % p.H_kv, block0 + rest / p.H_kv};
}
// The sequence of a slot and the slot's place among its own (0: the windows' own).  False: none.
__device__ inline bool find_sequence(const WindowArgs& p, int slot, int& seq, int& place) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int s0 = 0; s0 < p.n_seq; s0 += 64) {
        const int own = s0 + lane < p.n_seq ? slots_of(p, span_of(p, s0 + lane).len) : 0, upto = wave_scan(own);
        const uint64_t past = __builtin_amdgcn_ballot_w64(before + upto > slot);
        if (past) {
            const int l = (int)__builtin_ctzll(past);
            seq = s0 + l;
            place = slot - before - __builtin_amdgcn_readlane(upto - own, l);
            return true;
        }
        before += wave_total(upto);
        if (before >= MOST_COUNTED) return false;
    }
    return false;
}

template <typename T, int DP>
__global__ void __launch_bounds__(64 * WAVES, 1)
window_far_kernel(WindowArgs p, int block0) {
    using O = Of<T, DP>;
    constexpr int TILE = O::TILE, CW = O::CW, ES = O::ES, KS = DP / O::STEP, NM = DP / (16 * CW), NB = DP / 16, E = 16 / ES;
    constexpr int BLOCKS = TILE / 16, TOKENS = 4 * BLOCKS, PITCH = DP + 4;
    constexpr bool BF16 = ES == 2;
    __shared__ __attribute__((aligned(16))) float sums[WAVES][KEYS][PITCH];

    int seq, place;
    const Place at_slot = place_of(p, block0);
    if (!find_sequence(p, at_slot.slot, seq, place) || place == 0) return;
    const Span span = span_of(p, seq);
    const int first = __builtin_amdgcn_readfirstlane(span.first), c = __builtin_amdgcn_readfirstlane(span.len), d = p.d;
    const int a0 = p.window + (place - 1) * p.part, a1 = min(c, a0 + p.part);
    const int kvh = at_slot.kvh, key0 = at_slot.block * KEYS, group = p.H / p.H_kv;
    if (key0 + p.window >= c) return;           // no key of these is seen from further on
    const int lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int key = key0 + n;
    const int64_t key_row = kvh * p.kv_stride_h + (int64_t)(first + min(key, c - 1)) * p.kv_stride_s;
    u32x4 k[KS], v[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        k[ks] = load_chunk<T>((const T*)p.k + key_row, O::STEP * ks + E * j, d);
        v[ks] = load_chunk<T>((const T*)p.v + key_row, O::STEP * ks + E * j, d);
    }
    f32x4 accv[NB], acck[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) accv[i] = acck[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float kappa = p.scale * LOG2E;
    for (int head = kvh * group; head < (kvh + 1) * group; ++head) {
        const T* const Q = (const T*)p.q + head * p.stride_h + first * p.stride_s;
        const T* const G = (const T*)p.dout + head * p.stride_h + first * p.stride_s;
        const float* const lse = p.lse + head * p.stat_stride_h + first;
        const float* const delta = p.delta + head * p.stat_stride_h + first;
        for (int t = a0 + wave * TILE; t < a1; t += WAVES * TILE) {
            // (rows behind the part are its last one, without weight)
            u32x4 qa[BLOCKS][KS], ga[BLOCKS][KS];
            uint32_t qc[TOKENS][NM][CW * ES / 4], gc[TOKENS][NM][CW * ES / 4];
            float own_lse[TOKENS], own_delta[TOKENS];
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                const int64_t at = (int64_t)min(t + 16 * i + n, a1 - 1) * p.stride_s;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    qa[i][ks] = load_chunk<T>(Q + at, O::STEP * ks + E * j, d);
                    ga[i][ks] = load_chunk<T>(G + at, O::STEP * ks + E * j, d);
                }
            }
#pragma unroll
            for (int x = 0; x < TOKENS; ++x) {
                const int a = min(t + 16 * (x / 4) + 4 * j + x % 4, a1 - 1);
                own_lse[x] = lse[a];
                own_delta[x] = delta[a];
            }
#pragma unroll
            for (int x = 0; x < TOKENS; ++x) {
                const int64_t at = (int64_t)min(t + 16 * (x / 4) + 4 * j + x % 4, a1 - 1) * p.stride_s;
#pragma unroll
                for (int m = 0; m < NM; ++m) {
                    load_columns<T, CW>(qc[x][m], Q + at, 16 * CW * m + CW * n, d);
                    load_columns<T, CW>(gc[x][m], G + at, 16 * CW * m + CW * n, d);
                }
            }
            f32x4 s[BLOCKS], dp[BLOCKS];
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                s[i] = dp[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    s[i] = product(qa[i][ks], k[ks], s[i], (T*)nullptr);
                    dp[i] = product(ga[i][ks], v[ks], dp[i], (T*)nullptr);
                }
            }
            float pr[TOKENS], ds[TOKENS];
#pragma unroll
            for (int x = 0; x < TOKENS; ++x) {
                const int a = t + 16 * (x / 4) + 4 * j + x % 4;
                const bool seen = a < a1 && key < p.sinks && a - key >= p.window;
                const float score = s[x / 4][x % 4];
                const float weight = BF16 ? __builtin_amdgcn_exp2f(fmaf(score, kappa, -own_lse[x] * LOG2E)) : expf(score * p.scale - own_lse[x]);
                pr[x] = seen ? weight : 0.f;
                ds[x] = seen ? weight * (dp[x / 4][x % 4] - own_delta[x]) : 0.f;
            }
            if constexpr (BF16) {
                bf16x8 pb, db;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    pb[x] = (__bf16)pr[x];
                    db[x] = (__bf16)ds[x];
                }
#pragma unroll
                for (int m = 0; m < NM; ++m)
#pragma unroll
                    for (int e = 0; e < CW; ++e) {
                        u32x4 g, q;             // column e of the lane's, its eight rows
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t which = e % 2 ? 0x07060302u : 0x05040100u;
                            g[i] = __builtin_amdgcn_perm(gc[2 * i + 1][m][e / 2], gc[2 * i][m][e / 2], which);
                            q[i] = __builtin_amdgcn_perm(qc[2 * i + 1][m][e / 2], qc[2 * i][m][e / 2], which);
                        }
                        accv[m * CW + e] = product(g, __builtin_bit_cast(u32x4, pb), accv[m * CW + e], (T*)nullptr);
                        acck[m * CW + e] = product(q, __builtin_bit_cast(u32x4, db), acck[m * CW + e], (T*)nullptr);
                    }
            } else {
#pragma unroll
                for (int x = 0; x < TOKENS; ++x)
#pragma unroll
                    for (int m = 0; m < NM; ++m)
#pragma unroll
                        for (int e = 0; e < CW; ++e) {
                            accv[m * CW + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(gc[x][m][e]), pr[x], accv[m * CW + e], 0, 0, 0);
                            acck[m * CW + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(qc[x][m][e]), ds[x], acck[m * CW + e], 0, 0, 0);
                        }
            }
        }
    }
    // the four wavefronts' sums
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const f32x4(&acc)[NB] = which ? acck : accv;
        const float mul = which ? p.scale : 1.f;
        if (which) __syncthreads();
#pragma unroll
        for (int m = 0; m < NM; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < CW; ++e) sums[wave][n][16 * CW * m + CW * (4 * j + r) + e] = acc[m * CW + e][r];
        __syncthreads();
        for (int i = threadIdx.x; i < KEYS * (DP / 4); i += 64 * WAVES) {
            const int row = i / (DP / 4), col = 4 * (i - row * (DP / 4));
            if (col >= d) continue;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float4 z = *reinterpret_cast<const float4*>(&sums[w][row][col]);
                y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
            }
            *reinterpret_cast<float4*>(slot_row(p, at_slot.slot, kvh, key0 + row) + which * d + col) = make_float4(mul * y.x, mul * y.y, mul * y.z, mul * y.w);
        }
    }
}

// fp32 up to 128 columns: the windows' own sums come of three bf16 terms, and those of 32 keys that are all faint are too small for these (f32_rows.h).
// which: dV or dK, as of a launch on the sequence alone.  The tile's keys that have no slot are where they end.
__device__ inline bool faint_tile(const WindowArgs& p, int slot, int kvh, int key, int which, int lane) {
    const float least = which ? FAINT * p.scale : FAINT;
    const int end = min(p.c, key / 32 * 32 + 32);
    for (int other = key / 32 * 32; other < end; ++other) {
        const float* from = is_far(p, other) ? slot_row(p, slot, kvh, other) + which * p.d
                                             : (which ? p.dk : p.dv) + kvh * p.kv_stride_h + (int64_t)other * p.kv_stride_s;
        bool loud = false;
        for (int col = lane; col < p.d; col += 64) loud = loud || fabsf(from[col]) >= least;
        if (__builtin_amdgcn_ballot_w64(loud)) return false;
    }
    return true;
}

// dK and dV of a sequence's first keys put together, a wavefront a key: the windows' own sums and each part's, in order.  Where that is no number
// (or, in fp32, faint, of a tile that is: a faint key alone is what peaked scores leave; all of them done over, 700 rows, 8 heads of 64 columns, 130 first
// keys, 287 us, not 51) the row is done over.
template <typename T>
__global__ void __launch_bounds__(64 * WAVES)
window_join_kernel(WindowArgs p, int block0) {
    int seq, place;
    const Place at_slot = place_of(p, block0);
    if (!find_sequence(p, at_slot.slot, seq, place) || place != 0) return;
    const Span span = span_of(p, seq);
    const int first = __builtin_amdgcn_readfirstlane(span.first);
    p.c = __builtin_amdgcn_readfirstlane(span.len);
    const int slots = min(slots_of(p, p.c), p.n_slots - at_slot.slot);
    const int lane = threadIdx.x & 63, kvh = at_slot.kvh, key = __builtin_amdgcn_readfirstlane(at_slot.block * WAVES + ((int)threadIdx.x >> 6));
    if (!is_far(p, key)) return;
    float sum[2][ROW_COLS] = {};
    for (int s0 = 0; s0 < slots; s0 += BATCH) {         // (BATCH of them requested at a time)
        float x[BATCH][2][ROW_COLS];
#pragma unroll
        for (int s = 0; s < BATCH; ++s) {
            const float* from = slot_row(p, at_slot.slot + min(s0 + s, slots - 1), kvh, key);
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
                for (int i = 0; i < ROW_COLS; ++i) x[s][w][i] = lane + 64 * i < p.d ? from[w * p.d + lane + 64 * i] : 0.f;
        }
#pragma unroll
        for (int s = 0; s < BATCH; ++s)
            if (s0 + s < slots)
#pragma unroll
                for (int w = 0; w < 2; ++w)
#pragma unroll
                    for (int i = 0; i < ROW_COLS; ++i) sum[w][i] += x[s][w][i];
    }
    float z[2] = {0.f, 0.f}, loud[2] = {0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int i = 0; i < ROW_COLS; ++i) {
            z[w] = fmaf(sum[w][i], 0.f, z[w]);
            loud[w] = fmaxf(loud[w], fabsf(sum[w][i]));
        }
    bool odd[2];            // dV, dK
#pragma unroll
    for (int w = 0; w < 2; ++w) odd[w] = __builtin_amdgcn_ballot_w64(z[w] != 0.f) != 0;
    // the arguments of a launch on that sequence alone
    const int64_t q = first * p.stride_s, kv = first * p.kv_stride_s;
    p.q = (const T*)p.q + q;
    p.dout = (const T*)p.dout + q;
    p.k = (const T*)p.k + kv;
    p.v = (const T*)p.v + kv;
    p.dk = (float*)((T*)p.dk + kv);
    p.dv = (float*)((T*)p.dv + kv);
    p.lse += first;
    p.delta += first;
    if constexpr (sizeof(T) == 4)
        if (p.d <= 128)
            for (int w = 0; w < 2; ++w)
                odd[w] = odd[w] || (__builtin_amdgcn_ballot_w64(loud[w] >= FAINT) == 0 && __builtin_amdgcn_ballot_w64(loud[w] > 0.f) != 0 &&
                                    faint_tile(p, at_slot.slot, kvh, key, w, lane));
    const int64_t row = kvh * p.kv_stride_h + (int64_t)key * p.kv_stride_s;
#pragma unroll
    for (int i = 0; i < ROW_COLS; ++i)
        if (lane + 64 * i < p.d) {
            if (!odd[0]) store1((T*)p.dv + row + lane + 64 * i, sum[0][i]);
            if (!odd[0] && !odd[1]) store1((T*)p.dk + row + lane + 64 * i, sum[1][i]);
        }
    if (odd[0] || odd[1]) window_dkdv_row<T>(p, kvh, key, 0, p.d, odd[0]);
}

template <typename T>
hipError_t launch(const WindowArgs& p, hipStream_t st) {
    // (slots and heads are fewer than 2^24, as the tiles of the other launches are; of keys as many blocks a launch as make no more than that)
    const int64_t wide = (int64_t)p.n_slots * p.H_kv, fit = ((1 << 24) - 1) / wide, most = fit < 1 ? 1 : fit;
    auto each = [&](int blocks, auto launch) {
        for (int64_t b = 0; b < blocks; b += most) {
            launch(dim3((unsigned)(wide * (blocks - b < most ? blocks - b : most))), (int)b);
            if (hipError_t e = hipGetLastError()) return e;
        }
        return hipSuccess;
    };
    const dim3 block(64 * WAVES);
    if (hipError_t e = each(p.key_rows / KEYS, [&](dim3 grid, int b) {
            if (p.d <= 32) hipLaunchKernelGGL((window_far_kernel<T, 32>), grid, block, 0, st, p, b);
            else if (p.d <= 64) hipLaunchKernelGGL((window_far_kernel<T, 64>), grid, block, 0, st, p, b);
            else if (p.d <= 128) hipLaunchKernelGGL((window_far_kernel<T, 128>), grid, block, 0, st, p, b);
            else hipLaunchKernelGGL((window_far_kernel<T, 256>), grid, block, 0, st, p, b);
        }))
        return e;
    return each((p.sinks + WAVES - 1) / WAVES, [&](dim3 grid, int b) { hipLaunchKernelGGL((window_join_kernel<T>), grid, block, 0, st, p, b); });
}

}  // namespace

hipError_t launch_window_far(const WindowArgs& p, int dtype, hipStream_t st) {
    if (p.n_slots == 0) return hipSuccess;
    return dtype == SA_F32 ? launch<float>(p, st) : launch<__hip_bfloat16>(p, st);
}

}  // namespace sa
