// Attention of one new token a sequence over its paged cache: O = softmax(scale q K^T) V over the sequence's cached rows.
//
// Bound by memory: the cache is read once, 2 d elements a token and key/value head, for 4 d operations of each of the G query
// heads that share it.  bf16, d 128: 2 sequences of 262144 tokens, 16 heads, 4.3 GB in 701 us, 6.1 TB/s; 64 of 1 to 8192, 32 heads on 8, 1.1 GB
// in 207, 5.4; fp32, d 100, 160 MB in 41, 3.8.  (A copy reaches 4.9, a sum of a tensor 3.7.)
//
// Work.  A unit is (sequence, key/value head, 16 query heads of its group); its tokens come in chunks of CHUNK, and all chunks of all
// units, in order, are cut into equal shares, one a workgroup, however the lengths differ.  What a workgroup holds of a unit it
// holds alone is written as result; of a unit that goes over into another workgroup's share it writes an unnormalised sum, its
// reference and its row sum, and a second kernel joins them.  A share has at most two such pieces (its first and its last unit's),
// so the workspace depends on neither the batch nor the lengths.
//
// Inside, a wavefront takes every fourth tile of TILE tokens and keeps its own reference, row sum and accumulators; the four meet in LDS
// at the end of a unit.  Nothing is staged: K and V rows go from memory to the registers that the products want.
//  * S^T = K Q^T by 16 x 16 tiles, tokens as rows: a lane holds 16 bytes of one token's row a product.  The tile's lane (16 j + n)
//    register r is token 4 j + r of query head n.
//  * O^T += V^T P^T: that register, as it stands, is the right operand where the contraction goes through the tokens in that
//    order.  The left one wants, of one column, the lane's tokens: a lane loads a few columns of each of them (16 lanes a whole row, so
//    memory sees whole rows) and turns the little block round in registers (bf16: two tokens a v_perm; fp32: nothing to do).
// The next tile's K rows are requested as soon as this one's scores are formed, its V rows when they are used up.
//
// Probabilities: bf16 storage takes them as two bf16 terms (2^-17 relative; one term would put a second rounding of 2^-9 beside the
// result's own), fp32 as they are; row sums in fp32.  The reference moves only when a lane's sum of a tile passes 2^24 or there is none yet.
//
// What must not be read is not: a 16-token block's descriptor ends with the last cached token, and one whose page number is none
// has a range of zero; both deliver zeros, and the scores are masked.
#include <hip/hip_bf16.h>

#include "mfma_tiles.h"
#include "paged.h"
#include "wave.h"

namespace sa {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int WAVES = 4, HEADS = 16;            // wavefronts a workgroup, query heads a unit
constexpr float MOST = 16777216.f;              // 2^24: a lane's sum of a tile against a reference that stays

// Of a storage type and DP columns computed: tokens a tile, columns of a product over them, columns of a V row a lane loads at once
template <typename T, int DP> struct Of;
template <int DP> struct Of<__hip_bfloat16, DP> {
    static constexpr int TILE = 32, STEP = 32, CW = DP >= 128 ? 8 : DP / 16, ES = 2;
};
template <int DP> struct Of<float, DP> {
    static constexpr int TILE = 16, STEP = 16, CW = DP >= 64 ? 4 : DP / 16, ES = 4;
};
template <typename T> constexpr int CHUNK = WAVES * Of<T, 64>::TILE;

__device__ inline f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ inline f32x4 mfma_f32(uint32_t a, uint32_t b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a), __uint_as_float(b), c, 0, 0, 0);
}
// over the four lanes that hold a query head
__device__ inline float quad_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float quad_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}
// Parts are joined against the largest reference, of parts without a token (or any weight) 0.  A row sum of -1 says that there were
// tokens, all without weight (scores of -inf): nothing beside other parts, no number if there are none.
__device__ inline float reference(float top) { return top == -INFINITY ? 0.f : top; }
__device__ inline void add_sum(float& sum, bool& weightless, float l, float factor) {
    weightless = weightless || l < 0.f;
    sum += (l < 0.f ? 0.f : l) * factor;
}
__device__ inline int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
template <typename T>
__device__ inline int chunks_of(const DecodeArgs& p, int b) {
    const int len = min(max(p.lens[b], 0), p.max_pages * p.page_size);
    return (len + CHUNK<T> - 1) / CHUNK<T>;
}
// units of a sequence
__device__ inline int units_of(const DecodeArgs& p) { return p.H_kv * ((p.H / p.H_kv + HEADS - 1) / HEADS); }

// Where chunk number `at` of all units' chunks lies: the sequence, the chunks of the sequences before it (of one unit); and the share of a
// workgroup.  A wavefront's lanes take the sequences in turn.  (All counts are below 2^31: check_decode.)
struct Shares { int all, each; };
template <typename T>
__device__ inline Shares shares_of(const DecodeArgs& p, int units, int lane) {
    int n = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) n += b0 + lane < p.B ? chunks_of<T>(p, b0 + lane) : 0;
    const int all = wave_total(wave_scan(n)) * units;
    return {all, max(1, (int)(((uint32_t)all + (uint32_t)p.n_wgs - 1) / (uint32_t)p.n_wgs))};
}
template <typename T>
__device__ inline void find_chunk(const DecodeArgs& p, int at, int units, int lane, int& seq, int& before) {
    before = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int own = b0 + lane < p.B ? chunks_of<T>(p, b0 + lane) : 0, upto = wave_scan(own);
        const uint64_t past = __builtin_amdgcn_ballot_w64((before + upto) * units > at);
        if (past) {
            const int l = (int)__builtin_ctzll(past);
            before += __builtin_amdgcn_readlane(upto - own, l);
            seq = b0 + l;
            return;
        }
        before += wave_total(upto);
    }
    seq = p.B;              // (not reached: `at` is one of them)
}

// A unit's piece in the workspace: HEADS rows (as many as the group has) of DP columns, then references and row sums.
__host__ __device__ inline int part_rows(int group) { return group < HEADS ? group : HEADS; }
__host__ __device__ inline int64_t part_floats(int group, int DP) { return (int64_t)part_rows(group) * (DP + 2); }

// WHOLE: a workgroup has one unit, all of it, and there is nothing to join.
template <typename T, int DP, bool WHOLE>
__global__ void __launch_bounds__(64 * WAVES, DP > 128 ? 1 : 2)
decode_kernel(DecodeArgs p) {
    using O = Of<T, DP>;
    constexpr int TILE = O::TILE, CW = O::CW, ES = O::ES, KS = DP / O::STEP, NM = DP / (16 * CW), NB = DP / 16;
    constexpr bool BF16 = ES == 2;
    constexpr int BLOCKS = TILE / 16, TOKENS = 4 * BLOCKS;      // 16-token blocks of a tile, tokens a lane holds of it
    constexpr int PITCH = DP + 4;
    __shared__ __attribute__((aligned(16))) float o_lds[WAVES][HEADS][PITCH];
    __shared__ float m_lds[WAVES][HEADS], l_lds[WAVES][HEADS];

    const int lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4;
    const int wave = scalar((int)threadIdx.x >> 6);
    const int group = p.H / p.H_kv, blocks = (group + HEADS - 1) / HEADS, units = p.H_kv * blocks, d = p.d;
    int mine, at, end;                          // the share and its chunks
    int b, unit, chunk, n_chunks, len;          // where it begins: sequence, unit of it, chunk of that
    const int room = p.max_pages * p.page_size;
    auto enter = [&]() {
        len = scalar(min(max(p.lens[b], 0), room));
        n_chunks = (len + CHUNK<T> - 1) / CHUNK<T>;
    };
    if constexpr (WHOLE) {
        mine = (int)blockIdx.x;
        b = mine / units;
        unit = mine - b * units;
        enter();
        chunk = at = 0;
        end = n_chunks;
    } else {
        // neighbouring shares, which often read the same rows' other heads, on one XCD: consecutive workgroups go round-robin to the 8
        const Shares shares = shares_of<T>(p, units, lane);
        const int n_shares = (int)(((uint32_t)shares.all + (uint32_t)shares.each - 1) / (uint32_t)shares.each), per_xcd = (n_shares + 7) / 8;
        if ((int)blockIdx.x / 8 >= per_xcd) return;
        mine = (int)blockIdx.x % 8 * per_xcd + (int)blockIdx.x / 8;
        if (mine >= n_shares) return;
        at = mine * shares.each;
        end = at + min(shares.each, shares.all - at);
        // (a sequence's chunks, unit by unit, follow those of all sequences before it)
        int before;
        find_chunk<T>(p, at, units, lane, b, before);
        enter();
        const int in = at - before * units;
        unit = (int)((uint32_t)in / (uint32_t)n_chunks);
        chunk = in - unit * n_chunks;
    }
    const float kappa = p.scale * LOG2E;
    const int pitch = (int)p.stride_slot * ES;              // bytes between tokens of a page
    // this lane's bytes of a K block (token n, its columns of each product) and of a V block (token 4 j + r, its columns)
    uint32_t k_at[KS], v_at[4][NM];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int col = O::STEP * ks + (BF16 ? 8 : 4) * j;
        k_at[ks] = col < d ? n * pitch + col * ES : DT_OUT_OF_RANGE;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int m = 0; m < NM; ++m) {
            const int col = 16 * CW * m + CW * n;
            v_at[r][m] = col < d ? (4 * j + r) * pitch + col * ES : DT_OUT_OF_RANGE;
        }
    // bf16, d % 8 == 4: the chunk that holds column d has four elements of whatever follows the row
    const int part_ks = BF16 && d % 8 && ((d >> 3) & 3) == j ? d >> 5 : -1;

    // A piece: the chunks of a unit in this share.  Its first tile's rows and its queries are requested before the piece in front of it is
    // joined and written (`ahead` they are those of the next piece).
    struct Piece { int b, h0, n_heads, first, last, n_chunks, len; };
    Piece now;
    u32x4 q[KS], q_ahead[KS];
    int t0;                                     // this wavefront's next tile: tokens t0 .. t0 + TILE - 1, CHUNK<T> further on the one after it
    // page and place in it of each of its 16-token blocks
    const int step_page = CHUNK<T> / p.page_size, step_in = CHUNK<T> - step_page * p.page_size;
    int page[BLOCKS], in_page[BLOCKS];
    const int32_t* table;
    int64_t head_at;
    u32x4 k[BLOCKS][KS];
    uint32_t v[TOKENS][NM][CW * ES / 4];
    int64_t at_k[BLOCKS], at_v[BLOCKS];         // bytes of the blocks in the caches, of the tile requested last / before it
    int rows_k[BLOCKS], rows_v[BLOCKS];         // tokens that may be read (0: none)
    auto place = [&](int t) {
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            const int token = t + 16 * i;
            rows_k[i] = 0;
            at_k[i] = 0;
            if (token < len) {
                const int id = scalar(table[page[i]]);
                if (id >= 0 && id < p.n_pages) {
                    rows_k[i] = min(16, len - token);
                    at_k[i] = (id * p.stride_page + in_page[i] * p.stride_slot + head_at) * ES;
                }
            }
            page[i] += step_page;
            in_page[i] += step_in;
            if (in_page[i] >= p.page_size) {
                in_page[i] -= p.page_size;
                ++page[i];
            }
        }
    };
    auto rsrc = [&](const void* cache, int64_t bytes, int rows) {
        return __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)cache + bytes), 0, rows ? (rows - 1) * pitch + ES * d : 0, 0x00020000);
    };
    auto load_k = [&]() {
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            const auto s = rsrc(p.k_cache, at_k[i], rows_k[i]);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) k[i][ks] = __builtin_amdgcn_raw_buffer_load_b128(s, k_at[ks], 0, 0);
        }
    };
    auto load_v = [&]() {
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            const auto s = rsrc(p.v_cache, at_v[i], rows_v[i]);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int x = 0; x < NM; ++x) {
                    uint32_t(&to)[CW * ES / 4] = v[4 * i + r][x];
                    if constexpr (CW * ES == 16) {
                        const u32x4 y = __builtin_amdgcn_raw_buffer_load_b128(s, v_at[r][x], 0, 0);
                        to[0] = y[0]; to[1] = y[1]; to[2] = y[2]; to[3] = y[3];
                    } else if constexpr (CW * ES == 8) {
                        const u32x2 y = __builtin_amdgcn_raw_buffer_load_b64(s, v_at[r][x], 0, 0);
                        to[0] = y[0]; to[1] = y[1];
                    } else {
                        to[0] = __builtin_amdgcn_raw_buffer_load_b32(s, v_at[r][x], 0, 0);
                    }
                }
        }
    };
    auto keep_place = [&]() {
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            at_v[i] = at_k[i];
            rows_v[i] = rows_k[i];
        }
    };
    // the piece that begins with chunk `chunk` of (b, unit), `len` tokens long
    auto request = [&]() {
        const int kvh = unit / blocks, h0 = kvh * group + (unit - kvh * blocks) * HEADS;
        const int n_heads = min(HEADS, (kvh + 1) * group - h0);
        const Piece next = {b, h0, n_heads, chunk, min(n_chunks, chunk + (end - at)), n_chunks, len};
        const bool has_head = n < n_heads;
        const T* q_row = (const T*)p.q + b * p.stride_b + (h0 + (has_head ? n : 0)) * p.stride_h;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            constexpr int E = BF16 ? 8 : 4;
            const int col = O::STEP * ks + E * j;
            q_ahead[ks] = u32x4{0, 0, 0, 0};
            if (has_head && col < d) {
                if (!BF16 || col + 8 <= d) q_ahead[ks] = *reinterpret_cast<const u32x4*>(q_row + col);
                else {
                    const u32x2 x = *reinterpret_cast<const u32x2*>(q_row + col);
                    q_ahead[ks][0] = x[0];
                    q_ahead[ks][1] = x[1];
                }
            }
        }
        t0 = next.first * CHUNK<T> + wave * TILE;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            page[i] = (t0 + 16 * i) / p.page_size;
            in_page[i] = t0 + 16 * i - page[i] * p.page_size;
        }
        table = p.table + b * p.table_stride;
        head_at = (int64_t)kvh * p.stride_head;
        if (t0 < min(len, next.last * CHUNK<T>)) {
            place(t0);
            load_k();
            keep_place();
            load_v();
        }
        return next;
    };
    now = request();
    for (;;) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q[ks] = q_ahead[ks];
        const int t_end = min(now.len, now.last * CHUNK<T>);
        f32x4 acc[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        bool seen = false;                      // some token of a page that is one
        for (; t0 < t_end; t0 += CHUNK<T>) {
            f32x4 s[BLOCKS];
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    if constexpr (BF16) {
                        u32x4 x = k[i][ks];
                        if (d % 8) {
                            x[2] = ks == part_ks ? 0 : x[2];
                            x[3] = ks == part_ks ? 0 : x[3];
                        }
                        s[i] = mfma_bf16(x, q[ks], s[i]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[i] = mfma_f32(k[i][ks][e], q[ks][e], s[i]);
                    }
                }
            }
            int rows[BLOCKS];
            bool whole = true;
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                rows[i] = rows_k[i];
                whole = whole && rows[i] == 16;
                seen = seen || rows[i] > 0;
            }
            // the next tile's K rows (behind the last one: nothing, t0 is beyond the unit's tokens here)
            const bool more = t0 + CHUNK<T> < t_end;
            if (more) {
                place(t0 + CHUNK<T>);
                load_k();
            }
            if (!whole) {
#pragma unroll
                for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (4 * j + r >= rows[i]) s[i][r] = -INFINITY;
            }
            float pr[TOKENS], sum = 0.f;
#pragma unroll
            for (int x = 0; x < TOKENS; ++x) {
                pr[x] = __builtin_amdgcn_exp2f(fmaf(s[x / 4][x % 4], kappa, -m));
                sum += pr[x];
            }
            if (__builtin_amdgcn_ballot_w64(!(sum < MOST)) != 0) {          // wave-uniform and rare but for the first tile
                float top = s[0][0];
#pragma unroll
                for (int x = 1; x < TOKENS; ++x) top = fmaxf(top, s[x / 4][x % 4]);
                const float m_new = fmaxf(m, quad_max(top) * kappa), ref = m_new == -INFINITY ? 0.f : m_new;
                const float alpha = __builtin_amdgcn_exp2f(m - ref);
                m = m_new;
                l *= alpha;
#pragma unroll
                for (int i = 0; i < NB; ++i) acc[i] *= alpha;
                sum = 0.f;
#pragma unroll
                for (int x = 0; x < TOKENS; ++x) {
                    pr[x] = __builtin_amdgcn_exp2f(fmaf(s[x / 4][x % 4], kappa, -ref));
                    sum += pr[x];
                }
            }
            l += sum;
            if constexpr (BF16) {
                bf16x8 hi, lo;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    hi[x] = (__bf16)pr[x];
                    lo[x] = (__bf16)(pr[x] - (float)hi[x]);
                }
                const u32x4 ph = __builtin_bit_cast(u32x4, hi), pl = __builtin_bit_cast(u32x4, lo);
#pragma unroll
                for (int x = 0; x < NM; ++x)
#pragma unroll
                    for (int c = 0; c < CW; ++c) {
                        u32x4 a;        // column c of the lane's, its eight tokens
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            a[e] = __builtin_amdgcn_perm(v[2 * e + 1][x][c / 2], v[2 * e][x][c / 2], c % 2 ? 0x07060302u : 0x05040100u);
                        acc[x * CW + c] = mfma_bf16(a, ph, acc[x * CW + c]);
                        acc[x * CW + c] = mfma_bf16(a, pl, acc[x * CW + c]);
                    }
            } else {
#pragma unroll
                for (int r = 0; r < TOKENS; ++r)
#pragma unroll
                    for (int x = 0; x < NM; ++x)
#pragma unroll
                        for (int c = 0; c < CW; ++c)
                            acc[x * CW + c] = mfma_f32(v[r][x][c], __float_as_uint(pr[r]), acc[x * CW + c]);
            }
            if (more) {
                keep_place();
                load_v();
            }
        }

        // on to the next piece: its first requests are on their way while this one is joined
        const Piece done = now;
        at += now.last - now.first;
        const bool last_piece = WHOLE || at >= end;
        if (!last_piece) {
            chunk = 0;
            if (++unit == units) {
                unit = 0;
                do {
                    ++b;
                    enter();
                } while (n_chunks == 0);        // (there is one: `at` is before the end)
            }
            now = request();
        }

        // the four wavefronts' parts
        l = quad_sum(l);
        if (l == 0.f && seen) l = -1.f;
        if (j == 0) {
            m_lds[wave][n] = m;
            l_lds[wave][n] = l;
        }
        __syncthreads();
        float top = m_lds[0][n];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, m_lds[w][n]);
        const float own = __builtin_amdgcn_exp2f(m - reference(top));
#pragma unroll
        for (int x = 0; x < NM; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int c = 0; c < CW; c += 2)
                    *reinterpret_cast<float2*>(&o_lds[wave][n][16 * CW * x + CW * (4 * j + r) + c]) =
                        make_float2(acc[x * CW + c][r] * own, acc[x * CW + c + 1][r] * own);
        __syncthreads();
        const bool complete = done.first == 0 && done.last == done.n_chunks;
        // (a share's piece of a unit that began in another one is its first, of one that ends in another its last)
        float* part = p.parts + ((int64_t)mine * 2 + (done.first > 0 ? 0 : 1)) * part_floats(group, DP);
        for (int i = threadIdx.x; i < done.n_heads * (DP / 4); i += 64 * WAVES) {
            const int row = i / (DP / 4), col = 4 * (i - row * (DP / 4));
            if (col >= d) continue;
            float4 y = *reinterpret_cast<const float4*>(&o_lds[0][row][col]);
            float mx = m_lds[0][row];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) {
                const float4 z = *reinterpret_cast<const float4*>(&o_lds[w][row][col]);
                y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
                mx = fmaxf(mx, m_lds[w][row]);
            }
            float sum = 0.f;
            bool weightless = false;
#pragma unroll
            for (int w = 0; w < WAVES; ++w)
                add_sum(sum, weightless, l_lds[w][row], __builtin_amdgcn_exp2f(m_lds[w][row] - reference(mx)));
            if (sum == 0.f && weightless) sum = -1.f;
            if (complete) {
                // no token: zeros; tokens without any weight: no number
                const float inv = sum < 0.f ? NAN : sum == 0.f ? 0.f : 1.f / sum;
                T* to = (T*)p.out + done.b * p.stride_b + (done.h0 + row) * p.stride_h + col;
                if constexpr (BF16) {
                    bf16x4 z = {(__bf16)(y.x * inv), (__bf16)(y.y * inv), (__bf16)(y.z * inv), (__bf16)(y.w * inv)};
                    *reinterpret_cast<bf16x4*>(to) = z;
                } else {
                    *reinterpret_cast<float4*>(to) = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
                }
                if (p.lse && col == 0) p.lse[done.b * p.stat_stride_b + done.h0 + row] = sum < 0.f ? NAN : (mx + __builtin_amdgcn_logf(sum)) * LN2;
            } else {
                *reinterpret_cast<float4*>(part + row * DP + col) = y;
                if (col == 0) {
                    part[part_rows(group) * DP + row] = mx;
                    part[part_rows(group) * (DP + 1) + row] = sum;
                }
            }
        }
        if (last_piece) break;
        __syncthreads();
    }
}

// Units whose pieces lie in several shares, and sequences without a token.  JOIN_WAVES wavefronts take the pieces of a (sequence, query head) in
// turn; a workgroup has eight wavefronts or, where one is enough for a head, four, of which each has a head of its own.
constexpr int BATCH = 4;
template <typename T, int DP, int JOIN_WAVES>
__global__ void __launch_bounds__(JOIN_WAVES == 1 ? 256 : 64 * JOIN_WAVES)
decode_join_kernel(DecodeArgs p) {
    constexpr int COLS = (DP + 63) / 64, EACH = JOIN_WAVES == 1 ? 4 : 1;
    __shared__ float o_lds[JOIN_WAVES][DP], m_lds[JOIN_WAVES], l_lds[JOIN_WAVES];
    const int lane = threadIdx.x & 63, own_wave = scalar((int)threadIdx.x >> 6), wave = EACH == 1 ? own_wave : 0;
    const int group = p.H / p.H_kv, blocks = (group + HEADS - 1) / HEADS, units = p.H_kv * blocks;
    const int at_head = (int)blockIdx.x * EACH + (EACH == 1 ? 0 : own_wave), b = at_head / p.H, head = at_head - b * p.H;
    if (b >= p.B) return;
    const int kvh = head / group, in_group = head - kvh * group, unit = kvh * blocks + in_group / HEADS, row = in_group % HEADS;
    // (in one pass: the chunks of the sequences before b, and all)
    int before = 0, all = 0;
#pragma unroll 4
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int own = b0 + lane < p.B ? chunks_of<T>(p, b0 + lane) : 0;
        all += own;
        before += b0 + lane < b ? own : 0;
    }
    all = wave_total(wave_scan(all)) * units;
    before = wave_total(wave_scan(before));
    const int n = scalar(chunks_of<T>(p, b));
    const uint32_t share = (uint32_t)max(1, (int)(((uint32_t)all + (uint32_t)p.n_wgs - 1) / (uint32_t)p.n_wgs));
    const uint32_t from = (uint32_t)(before * units + unit * n);
    const int g0 = (int)(from / share), g1 = n ? (int)((from + n - 1) / share) : g0;
    if (n && g0 == g1) return;
    // a wavefront's pieces, BATCH of them requested at a time (they come from other XCDs' workgroups: a round trip to memory each)
    const int pieces = n ? g1 - g0 + 1 : 0, rows = part_rows(group);
    float m = -INFINITY, l = 0.f, acc[COLS] = {};
    bool weightless = false;
    for (int i0 = wave * BATCH; i0 < pieces; i0 += JOIN_WAVES * BATCH) {
        float mg[BATCH], lg[BATCH], x[BATCH][COLS];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int at = min(i0 + i, pieces - 1);
            const float* part = p.parts + ((int64_t)(g0 + at) * 2 + (at == 0 ? 1 : 0)) * part_floats(group, DP);
            mg[i] = part[rows * DP + row];
            lg[i] = part[rows * (DP + 1) + row];
#pragma unroll
            for (int c = 0; c < COLS; ++c) x[i][c] = lane + 64 * c < p.d ? part[row * DP + lane + 64 * c] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            if (i0 + i >= pieces) break;
            const float top = fmaxf(m, mg[i]), a = __builtin_amdgcn_exp2f(m - reference(top)), f = __builtin_amdgcn_exp2f(mg[i] - reference(top));
            l *= a;
            add_sum(l, weightless, lg[i], f);
#pragma unroll
            for (int c = 0; c < COLS; ++c) acc[c] = acc[c] * a + x[i][c] * f;
            m = top;
        }
    }
    T* const to = (T*)p.out + b * p.stride_b + head * p.stride_h;
    if constexpr (JOIN_WAVES == 1) {
        if (weightless && l == 0.f) l = NAN;
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int c = 0; c < COLS; ++c)
            if (lane + 64 * c < p.d) {
                if constexpr (sizeof(T) == 2) reinterpret_cast<__bf16*>(to)[lane + 64 * c] = (__bf16)(acc[c] * inv);
                else to[lane + 64 * c] = acc[c] * inv;
            }
        if (p.lse && lane == 0) p.lse[b * p.stat_stride_b + head] = (m + __builtin_amdgcn_logf(l)) * LN2;
        return;
    }
#pragma unroll
    for (int c = 0; c < COLS; ++c)
        if (lane + 64 * c < DP) o_lds[wave][lane + 64 * c] = acc[c];
    if (lane == 0) {
        m_lds[wave] = m;
        l_lds[wave] = weightless && l == 0.f ? -1.f : l;
    }
    __syncthreads();
    float top = m_lds[0];
#pragma unroll
    for (int w = 1; w < JOIN_WAVES; ++w) top = fmaxf(top, m_lds[w]);
    float f[JOIN_WAVES], sum = 0.f;
    weightless = false;
#pragma unroll
    for (int w = 0; w < JOIN_WAVES; ++w) {
        f[w] = __builtin_amdgcn_exp2f(m_lds[w] - reference(top));
        add_sum(sum, weightless, l_lds[w], f[w]);
    }
    if (sum == 0.f && weightless) sum = NAN;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    for (int col = threadIdx.x; col < p.d; col += 64 * JOIN_WAVES) {
        float y = 0.f;
#pragma unroll
        for (int w = 0; w < JOIN_WAVES; ++w) y += o_lds[w][col] * f[w];
        if constexpr (sizeof(T) == 2) reinterpret_cast<__bf16*>(to)[col] = (__bf16)(y * inv);
        else to[col] = y * inv;
    }
    if (p.lse && threadIdx.x == 0) p.lse[b * p.stat_stride_b + head] = (top + __builtin_amdgcn_logf(sum)) * LN2;
}

constexpr int columns(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 128 ? 128 : 256; }
// Shares: as many workgroups as the chip holds at once or nearly.  64 sequences of up to 8192 tokens, 8 key/value heads, us, 1, 2, 3, 4 a compute
// unit: d 128 204, 208, 226, 208, 128 of up to 1000 72, 65, 73, 67, d 64 132, 117, 114, 122, d 32 (32 of up to 16384, 16 heads) 218, 192, 177, 179.
constexpr int workgroups(int DP) { return N_CU * (DP <= 32 ? 3 : 2); }

template <typename T, int DP>
hipError_t launch(DecodeArgs a, hipStream_t st) {
    // Where no sequence can have more than eight rounds (above 128 columns four), a unit to a workgroup and nothing to join, whatever the lengths
    // are.  us, shares : units, 32 heads on 8, d 128, tables of up to 250 tokens, 16 sequences 13.6 : 11.0, 128 24.4 : 15.6, 500 38 : 30, 1000
    // 61 : 58, 16 of 1000 16.5 : 13.9, but one of 1500 13.8 : 17.0, 64 of 2000 58 : 63; d 256, 8 heads on 2, 16 of 250 13.9 : 11.0, but 1000 13.9 : 23;
    // fp32, 16 of 500 18.8 : 17.1, but 1000 22.6 : 29.  (11 us of these are the calls'.)
    if ((int64_t)a.max_pages * a.page_size <= (DP > 128 ? 4 : 8) * CHUNK<T>) {
        const int group = a.H / a.H_kv;
        hipLaunchKernelGGL((decode_kernel<T, DP, true>), dim3((unsigned)(a.B * a.H_kv * ((group + HEADS - 1) / HEADS))), dim3(64 * WAVES), 0, st, a);
        return hipGetLastError();
    }
    a.n_wgs = workgroups(DP);
    hipLaunchKernelGGL((decode_kernel<T, DP, false>), dim3((unsigned)a.n_wgs), dim3(64 * WAVES), 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
    // Eight wavefronts a head where there are few heads, whose units then have many pieces, us, one : eight, 32 heads on 8: a sequence of
    // 8000 tokens 25.0 : 14.9, of 65536 69 : 57, 4 of up to 100000 174 : 169, 16 of up to 4000 37.1 : 37.4; 32 of up to 2000 30.7 : 32.3, 128 of up to
    // 1100 73 : 83.
    if ((int64_t)a.B * a.H <= 512) hipLaunchKernelGGL((decode_join_kernel<T, DP, 8>), dim3((unsigned)a.B * a.H), dim3(64 * 8), 0, st, a);
    else hipLaunchKernelGGL((decode_join_kernel<T, DP, 1>), dim3(((unsigned)(a.B * a.H) + 3) / 4), dim3(64 * 4), 0, st, a);
    return hipGetLastError();
}
template <typename T>
hipError_t launch(const DecodeArgs& a, hipStream_t st) {
    switch (columns(a.d)) {
        case 32: return launch<T, 32>(a, st);
        case 64: return launch<T, 64>(a, st);
        case 128: return launch<T, 128>(a, st);
        default: return launch<T, 256>(a, st);
    }
}

}  // namespace

int64_t decode_workspace(int H, int H_kv, int d) {
    const int DP = columns(d);
    return (int64_t)workgroups(DP) * 2 * part_floats(H / H_kv, DP) * 4;
}

hipError_t launch_decode(const DecodeArgs& a, int dtype, hipStream_t st) {
    return dtype == SA_F32 ? launch<float>(a, st) : launch<__hip_bfloat16>(a, st);
}

}  // namespace sa
