// Attention of drafted tokens over the paged cache: each of a sequence's drafted tokens over all tokens in front of the draft and those of the draft that
// its mask names.
//
// As decode.hip has it for one token, with rows in the place of query heads: a unit is (sequence, key/value head, 16, 64 or 128 of the sequence's rows), row
// i G + g being drafted token i and query head g of the group of G.  Shares of chunks, references and sums of their own for wavefronts and pieces,
// and the joining of pieces in a second launch are as there; a sequence has as many units as its own draft needs.  Two kernels: tree_kernel takes 16 rows
// with everything in registers, as a new token's heads; tree_tiles_kernel more, through LDS.  Bound by memory where there is much of it: 32 sequences of 1 to
// 8192 tokens, drafts of up to 32, 32 heads on 8 of 128 columns, 174 us, 3.5 TB/s, 12 of it the joining; else by a launch's latency: one of 1500, 8 drafted,
// 13.5 us, both launches.
//
// What a row does not see has a score of -inf.  Its weight of zero would still make a NaN of an infinite or NaN value, so such tokens are taken out of the
// products and added to the rows that see them by vector instructions; only tiles with drafted tokens are looked at for them.
#include <hip/hip_bf16.h>

#include "mfma_tiles.h"
#include "paged.h"
#include "wave.h"

namespace sa {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int WAVES = 4;                        // wavefronts a workgroup
constexpr float MOST = 16777216.f;              // 2^24: a lane's sum of a tile against a reference that stays

// Of a storage type and DP columns computed: tokens a tile, columns of a product over them, columns of a V row a lane loads at once
template <typename T, int DP> struct Of;
template <int DP> struct Of<__hip_bfloat16, DP> {
    static constexpr int TILE = 32, STEP = 32, CW = DP >= 128 ? 8 : DP / 16, ES = 2;
};
template <int DP> struct Of<float, DP> {
    static constexpr int TILE = 16, STEP = 16, CW = DP >= 64 ? 4 : DP / 16, ES = 4;
};
template <typename T> constexpr int CHUNK = WAVES * Of<T, 64>::TILE;      // tree_kernel
constexpr int TILE_CHUNK = DT_ROWS;                                        // tree_tiles_kernel

__device__ inline f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ inline f32x4 mfma_f32(uint32_t a, uint32_t b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a), __uint_as_float(b), c, 0, 0, 0);
}
// over the four lanes that hold a row
__device__ inline float quad_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float quad_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}
// Parts are joined against the largest reference, of parts without a token (or any weight) 0.  A row sum of -1 says that the row saw tokens, all
// without weight (scores of -inf): nothing beside other parts, no number if there are none.
__device__ inline float reference(float top) { return top == -INFINITY ? 0.f : top; }
__device__ inline void add_sum(float& sum, bool& weightless, float l, float factor) {
    weightless = weightless || l < 0.f;
    sum += (l < 0.f ? 0.f : l) * factor;
}
__device__ inline int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }

// a sequence: tokens in front of its draft, all, rows
struct Sequence { int before, len, rows; };
__device__ inline Sequence sequence(const TreeArgs& p, int b) {
    const int room = p.max_pages * p.page_size, drafted = p.drafts ? min(max(p.drafts[b], 0), p.T) : p.T;
    const int before = min(max(p.lens[b], 0), room);
    return {before, min(before + drafted, room), drafted * (p.H / p.H_kv)};
}
// its chunks, and its units
template <int CH> __device__ inline int chunks_of(const Sequence& x) { return (x.len + CH - 1) / CH; }
template <int ROWS> __device__ inline int units_of(const TreeArgs& p, const Sequence& x) { return p.H_kv * ((x.rows + ROWS - 1) / ROWS); }
// the chunks of all its units
template <int CH, int ROWS>
__device__ inline int work_of(const TreeArgs& p, int b) {
    const Sequence x = sequence(p, b);
    return chunks_of<CH>(x) * units_of<ROWS>(p, x);
}

// Where chunk number `at` of all units' chunks lies: the sequence, the chunks before it; and the share of a workgroup.  A wavefront's lanes take the
// sequences in turn.  (All counts are below 2^31: check_tree.)
__device__ inline int share_of(int all, int n_wgs) { return max(1, (int)(((uint32_t)all + (uint32_t)n_wgs - 1) / (uint32_t)n_wgs)); }
template <int CH, int ROWS>
__device__ inline int all_work(const TreeArgs& p, int lane) {
    int n = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) n += b0 + lane < p.B ? work_of<CH, ROWS>(p, b0 + lane) : 0;
    return wave_total(wave_scan(n));
}
template <int CH, int ROWS>
__device__ inline void find_chunk(const TreeArgs& p, int at, int lane, int& seq, int& before) {
    before = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int own = b0 + lane < p.B ? work_of<CH, ROWS>(p, b0 + lane) : 0, upto = wave_scan(own);
        const uint64_t past = __builtin_amdgcn_ballot_w64(before + upto > at);
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

// A unit's piece in the workspace: its rows of DP columns, then references and row sums.
__host__ __device__ inline int64_t part_floats(int rows, int DP) { return (int64_t)rows * (DP + 2); }

// an infinite or NaN element of a dword
template <int ES> __device__ inline bool odd_word(uint32_t w) {
    return (w & 0x7f800000u) == 0x7f800000u || (ES == 2 && (w & 0x7f80u) == 0x7f80u);
}
template <int ES> __device__ inline float element(const uint32_t* words, int i) {
    return __uint_as_float(ES == 4 ? words[i] : i % 2 ? words[i / 2] & 0xffff0000u : words[i / 2] << 16);
}

// WHOLE: a workgroup has one unit, all of it, and there is nothing to join.
template <typename T, int DP, bool WHOLE>
__global__ void __launch_bounds__(64 * WAVES, DP > 128 ? 1 : 2)
tree_kernel(TreeArgs p) {
    using O = Of<T, DP>;
    constexpr int TILE = O::TILE, CW = O::CW, ES = O::ES, KS = DP / O::STEP, NM = DP / (16 * CW), NB = DP / 16;
    constexpr bool BF16 = ES == 2;
    constexpr int BLOCKS = TILE / 16, TOKENS = 4 * BLOCKS;      // 16-token blocks of a tile, tokens a lane holds of it
    constexpr int PITCH = DP + 4, ROWS = 16, CH = CHUNK<T>;
    __shared__ __attribute__((aligned(16))) float o_lds[WAVES][ROWS][PITCH];
    __shared__ float m_lds[WAVES][ROWS], l_lds[WAVES][ROWS];

    const int lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4;
    const int wave = scalar((int)threadIdx.x >> 6);
    const int group = p.H / p.H_kv, d = p.d;
    int mine, at, end;                          // the share and its chunks
    int b, unit, chunk, n_chunks, units;        // where it begins: sequence, unit of it, chunk of that; the sequence's
    Sequence seq;
    auto enter = [&]() {
        seq = sequence(p, b);
        seq = {scalar(seq.before), scalar(seq.len), scalar(seq.rows)};
        n_chunks = chunks_of<CH>(seq);
        units = units_of<ROWS>(p, seq);
    };
    if constexpr (WHOLE) {
        mine = (int)blockIdx.x;
        const int most = p.H_kv * ((p.T * group + ROWS - 1) / ROWS);
        b = mine / most;
        unit = mine - b * most;
        enter();
        if (unit >= units) return;
        chunk = at = 0;
        end = n_chunks;
    } else {
        // neighbouring shares, which often read the same rows for other ones, on one XCD: consecutive workgroups go round-robin to the 8
        const int all = all_work<CH, ROWS>(p, lane), each = share_of(all, p.n_wgs);
        const int n_shares = (int)(((uint32_t)all + (uint32_t)each - 1) / (uint32_t)each), per_xcd = (n_shares + 7) / 8;
        if ((int)blockIdx.x / 8 >= per_xcd) return;
        mine = (int)blockIdx.x % 8 * per_xcd + (int)blockIdx.x / 8;
        if (mine >= n_shares) return;
        at = mine * each;
        end = at + min(each, all - at);
        // (a sequence's chunks, unit by unit, follow those of all sequences before it)
        int before;
        find_chunk<CH, ROWS>(p, at, lane, b, before);
        enter();
        const int in = at - before;
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
    // joined and written.
    struct Piece { int b, kvh, row0, rows, first, last, n_chunks, before, len; };
    Piece now;
    u32x4 q[KS];
    uint64_t sees;                              // the row's mask
    int t0;                                     // this wavefront's next tile: tokens t0 .. t0 + TILE - 1, CH further on the one after it
    // page and place in it of each of its 16-token blocks
    const int step_page = CH / p.page_size, step_in = CH - step_page * p.page_size;
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
            if (token < seq.len) {
                const int id = scalar(table[page[i]]);
                if (id >= 0 && id < p.n_pages) {
                    rows_k[i] = min(16, seq.len - token);
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
    // the piece that begins with chunk `chunk` of (b, unit)
    auto request = [&]() {
        const int blocks = units / p.H_kv, kvh = unit / blocks, row0 = (unit - kvh * blocks) * ROWS;
        const Piece next = {b, kvh, row0, min(ROWS, seq.rows - row0), chunk, min(n_chunks, chunk + (end - at)), n_chunks, seq.before, seq.len};
        const bool has_row = n < next.rows;
        const int row = row0 + (has_row ? n : 0), i = row / group, head = kvh * group + row - i * group;
        const T* q_row = (const T*)p.q + b * p.stride_b + i * p.stride_t + head * p.stride_h;
        sees = has_row ? (uint64_t)p.seen[b * p.seen_stride + i] : 0;
        // (all requested at once, without branches: from the row's last 16 bytes where a chunk goes beyond them; a row of eight bytes twice)
        typedef uint32_t Chunk __attribute__((ext_vector_type(4), aligned(8)));
        typedef uint32_t Half __attribute__((ext_vector_type(2)));
        constexpr int E = BF16 ? 8 : 4;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if (BF16 && d < 8) {
                const Half x = *reinterpret_cast<const Half*>(q_row);
                q[ks] = u32x4{x[0], x[1], 0, 0};
            } else {
                q[ks] = *reinterpret_cast<const Chunk*>(q_row + min(O::STEP * ks + E * j, d - E));
            }
        }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int col = O::STEP * ks + (BF16 ? 8 : 4) * j;
                const u32x4 x = q[ks];
                if (col >= d) q[ks] = u32x4{0, 0, 0, 0};
                else if (BF16 && col + 8 > d && d >= 8) q[ks] = u32x4{x[2], x[3], 0, 0};
            }
        t0 = next.first * CH + wave * TILE;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            page[i] = (t0 + 16 * i) / p.page_size;
            in_page[i] = t0 + 16 * i - page[i] * p.page_size;
        }
        table = p.table + b * p.table_stride;
        head_at = (int64_t)kvh * p.stride_head;
        if (t0 < min(seq.len, next.last * CH)) {
            place(t0);
            load_k();
            keep_place();
            load_v();
        }
        return next;
    };
    now = request();
    for (;;) {
        const int t_end = min(now.len, now.last * CH);
        f32x4 acc[NB];
        float top = -INFINITY, l = 0.f;
        bool saw = false;                       // some token that the row sees, in a page that is one
#pragma unroll
        for (int i = 0; i < NB; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (; t0 < t_end; t0 += CH) {
            f32x4 s[BLOCKS];
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    u32x4 x = k[i][ks];
                    if (BF16 && d % 8) {
                        x[2] = ks == part_ks ? 0 : x[2];
                        x[3] = ks == part_ks ? 0 : x[3];
                    }
                    if constexpr (BF16) s[i] = mfma_bf16(x, q[ks], s[i]);
                    else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[i] = mfma_f32(x[e], q[ks][e], s[i]);
                    }
                }
            }
            int rows[BLOCKS];
            bool whole = t0 + TILE <= now.before;
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                rows[i] = rows_k[i];
                whole = whole && rows[i] == 16;
            }
            const bool drafted = t0 + TILE > now.before;
            const int tile_at = t0;
            // the next tile's K rows (behind the last one: nothing, t0 is beyond the unit's tokens here)
            const bool more = t0 + CH < t_end;
            if (more) {
                place(t0 + CH);
                load_k();
            }
            // a lane's token x of the tile is seen by its row
            auto seen = [&](int x) {
                const int row = 4 * j + x % 4, nth = tile_at + 16 * (x / 4) + row - now.before;        // of the draft; negative: before it
                return row < rows[x / 4] && (nth < 0 || ((sees >> (nth & 63)) & 1));
            };
            if (!whole) {
#pragma unroll
                    for (int x = 0; x < TOKENS; ++x) {
                        const bool sees_it = seen(x);
                        saw = saw || sees_it;
                        if (!sees_it) s[x / 4][x % 4] = -INFINITY;
                    }
            } else {
                saw = true;
            }
            float pr[TOKENS];
            float sum = 0.f;
#pragma unroll
            for (int x = 0; x < TOKENS; ++x) {
                pr[x] = __builtin_amdgcn_exp2f(fmaf(s[x / 4][x % 4], kappa, -top));
                sum += pr[x];
            }
            if (__builtin_amdgcn_ballot_w64(!(sum < MOST)) != 0) {          // wave-uniform and rare but for the first tile
                float mx = s[0][0];
#pragma unroll
                for (int x = 1; x < TOKENS; ++x) mx = fmaxf(mx, s[x / 4][x % 4]);
                const float m_new = fmaxf(top, quad_max(mx) * kappa), ref = m_new == -INFINITY ? 0.f : m_new;
                const float alpha = __builtin_amdgcn_exp2f(top - ref);
                top = m_new;
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
            if (drafted) {
                // values that are no numbers, of tokens that some rows do not see
                bool odd_values = false;
#pragma unroll
                for (int x = 0; x < TOKENS; ++x)
#pragma unroll
                    for (int y = 0; y < NM; ++y)
#pragma unroll
                        for (int c = 0; c < CW * ES / 4; ++c) odd_values = odd_values || odd_word<ES>(v[x][y][c]);
                if (__builtin_amdgcn_ballot_w64(odd_values) != 0) {
#pragma unroll
                    for (int x = 0; x < TOKENS; ++x) {
                        bool odd = false;
#pragma unroll
                        for (int y = 0; y < NM; ++y)
#pragma unroll
                            for (int c = 0; c < CW * ES / 4; ++c) odd = odd || odd_word<ES>(v[x][y][c]);
                        const uint64_t who = __builtin_amdgcn_ballot_w64(odd);
#pragma unroll 1
                        for (int jj = 0; jj < 4; ++jj) {
                            if (!((who >> (16 * jj)) & 0xffff)) continue;
                            const float w = __shfl(pr[x], 16 * jj + n);
                            const bool sees_it = __shfl((int)seen(x), 16 * jj + n) != 0;
#pragma unroll
                            for (int y = 0; y < NM; ++y)
#pragma unroll
                                for (int c = 0; c < CW; ++c)
#pragma unroll
                                    for (int r = 0; r < 4; ++r) {
                                        const float value = __shfl(element<ES>(v[x][y], c), 16 * jj + 4 * j + r);
                                        if (sees_it) acc[y * CW + c][r] += w * value;
                                    }
                        }
                        if ((who >> (16 * j)) & 0xffff) {
#pragma unroll
                            for (int y = 0; y < NM; ++y)
#pragma unroll
                                for (int c = 0; c < CW * ES / 4; ++c) v[x][y][c] = 0;
                        }
                    }
                }
            }
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
                } while (n_chunks == 0 || units == 0);        // (there is one: `at` is before the end)
            }
            now = request();
        }

        // the four wavefronts' parts
        l = quad_sum(l);
        const uint64_t some = __builtin_amdgcn_ballot_w64(saw);
        if (l == 0.f && (((some >> n) | (some >> (16 + n)) | (some >> (32 + n)) | (some >> (48 + n))) & 1)) l = -1.f;
        if (j == 0) {
            m_lds[wave][n] = top;
            l_lds[wave][n] = l;
        }
        __syncthreads();
        float all = m_lds[0][n];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) all = fmaxf(all, m_lds[w][n]);
        const float own = __builtin_amdgcn_exp2f(top - reference(all));
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
        float* part = p.parts + ((int64_t)mine * 2 + (done.first > 0 ? 0 : 1)) * part_floats(ROWS, DP);
        for (int i = threadIdx.x; i < done.rows * (DP / 4); i += 64 * WAVES) {
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
                const int at_row = done.row0 + row, t = at_row / group, head = done.kvh * group + at_row - t * group;
                T* to = (T*)p.out + done.b * p.stride_b + t * p.stride_t + head * p.stride_h + col;
                if constexpr (BF16) {
                    bf16x4 z = {(__bf16)(y.x * inv), (__bf16)(y.y * inv), (__bf16)(y.z * inv), (__bf16)(y.w * inv)};
                    *reinterpret_cast<bf16x4*>(to) = z;
                } else {
                    *reinterpret_cast<float4*>(to) = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
                }
                if (p.lse && col == 0)
                    p.lse[done.b * p.stat_stride_b + t * p.stat_stride_t + head] = sum < 0.f ? NAN : (mx + __builtin_amdgcn_logf(sum)) * LN2;
            } else {
                *reinterpret_cast<float4*>(part + row * DP + col) = y;
                if (col == 0) {
                    part[ROWS * DP + row] = mx;
                    part[ROWS * (DP + 1) + row] = sum;
                }
            }
        }
        if (last_piece) break;
        __syncthreads();
    }
}

// bf16, up to 128 columns, more than 16 rows a key/value head: as attention of whole blocks has it, tiles of 64 tokens go straight into LDS (mfma_tiles.h),
// two buffers, and R groups of 32 rows read them; S^T = K Q^T and O^T += V^T P^T by 32 x 32 products, a lane holding 16 tokens of one row.  R = 4: a
// wavefront each; R = 2: two wavefronts each, of which either takes 32 tokens of a tile, joined at the end of a piece.  A tile is requested while the one
// before it is computed, each wavefront one 16-token block of it: its page, its descriptor.  (Four half tiles, three on their way, a barrier for each: 208 us
// where this takes 174, 32 sequences' drafts of up to 32.)
//
// Bound by memory: a token costs a compute unit 512 bytes (d 128), 65 clocks at 4.9 TB/s, and 24 products of 32 clocks for each 32 tokens and rows, on
// four SIMDs 24 clocks a token and 128 rows.  It takes 1.4 times that (174 us): R goes by the longest draft that there can be, so a shorter one's unit leaves
// wavefronts idle; every tile passes the tests for drafted tokens' values; shares spill 48 to 56 registers at 128 columns, between pieces.
template <int DP> constexpr int KV_BYTES = 2 * tile_bytes(DP);
template <int DP, int R, bool PART, bool WHOLE>
__global__ void __launch_bounds__(64 * WAVES, 2)
tree_tiles_kernel(TreeArgs p) {
    constexpr int ROWS = 32 * R, SHARING = WAVES / R, SUBS = 2 / SHARING, CH = TILE_CHUNK, KS = ksteps_of(DP), MB = blocks_of(DP);
    static_assert(R == 2 || R == 4, "one or two wavefronts a row group");
    __shared__ __attribute__((aligned(1024))) char lds[2][KV_BYTES<DP>];        // [buffer][K | V]
    __shared__ int rows_lds[2][4];                                              // tokens of each 16-token block
    __shared__ float stat_lds[R][2][32];

    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = scalar((int)threadIdx.x >> 6), rg = wave / SHARING, part_of = wave % SHARING;      // row group; its tokens of a tile: SUBS sub-tiles
    const int group = p.H / p.H_kv, d = p.d;
    int mine, at, end, b, unit, chunk, n_chunks, units;       // as in tree_kernel
    Sequence seq;
    auto enter = [&]() {
        seq = sequence(p, b);
        seq = {scalar(seq.before), scalar(seq.len), scalar(seq.rows)};
        n_chunks = chunks_of<CH>(seq);
        units = units_of<ROWS>(p, seq);
    };
    if constexpr (WHOLE) {
        mine = (int)blockIdx.x;
        const int most = p.H_kv * ((p.T * group + ROWS - 1) / ROWS);
        b = mine / most;
        unit = mine - b * most;
        enter();
        if (unit >= units) return;
        chunk = at = 0;
        end = n_chunks;
    } else {
        const int all = all_work<CH, ROWS>(p, lane), each = share_of(all, p.n_wgs);
        const int n_shares = (int)(((uint32_t)all + (uint32_t)each - 1) / (uint32_t)each), per_xcd = (n_shares + 7) / 8;
        if ((int)blockIdx.x / 8 >= per_xcd) return;
        mine = (int)blockIdx.x % 8 * per_xcd + (int)blockIdx.x / 8;
        if (mine >= n_shares) return;
        at = mine * each;
        end = at + min(each, all - at);
        int before;
        find_chunk<CH, ROWS>(p, at, lane, b, before);
        b = scalar(b);
        enter();
        const int in = at - before;
        unit = scalar((int)((uint32_t)in / (uint32_t)n_chunks));
        chunk = scalar(in - unit * n_chunks);
    }
    const float kappa = p.scale * LOG2E;
    const int pitch = (int)p.stride_slot * 2;               // bytes between tokens of a page
    uint32_t arow[8], tr0[4], tr1[4], g[4];                 // g: of a 16-token block, as of a tile's first one
    dt_row_addrs<DP>(arow, n, h);
    dt_tr_addrs<DP>(tr0, tr1, lane);
    dt_load_offsets<DP>(g, lane, 0, pitch, d);
    // PART, d % 8 == 4: the chunk that holds column d has four elements of whatever follows the row
    const int part_ks = PART && ((d >> 3) & 1) == h ? d >> 4 : -1;

    struct Piece { int b, kvh, row0, rows, first, last, n_chunks, before; };
    Piece now;
    bf16x8 q[8];
    uint64_t sees;                              // the row's mask
    const int step_page = CH / p.page_size, step_in = CH - step_page * p.page_size;
    int page, in_page, token, id;               // of this wavefront's block of the tile to request next; its page's number in the cache
    const int32_t* table;
    int64_t head_at;
    auto look_up = [&]() { id = token < seq.len ? table[page] : -1; };
    auto request = [&](int buffer) {
        const int page_id = scalar(id);
        int rows = 0;
        int64_t from = 0;
        if (page_id >= 0 && page_id < p.n_pages) {
            rows = min(16, seq.len - token);
            from = (page_id * p.stride_page + in_page * p.stride_slot + head_at) * 2;
        }
        dt_rsrc k = dt_make_rsrc((const char*)p.k_cache + from, rows, pitch, d), v = dt_make_rsrc((const char*)p.v_cache + from, rows, pitch, d);
        if (rows == 0) k[2] = v[2] = 0;         // nothing is in range: zeros
#pragma unroll
        for (int i = 0; i < 4; ++i) {           // (kept scalar)
            k[i] = scalar(k[i]);
            v[i] = scalar(v[i]);
        }
        dt_load<DP>(k, 0, lds[buffer], g, wave);
        dt_load<DP>(v, 0, lds[buffer] + tile_bytes(DP), g, wave);
        if (lane == 0) rows_lds[buffer][wave] = rows;
        token += CH;
        page += step_page;
        in_page += step_in;
        if (in_page >= p.page_size) {
            in_page -= p.page_size;
            ++page;
        }
        look_up();
    };
    // the piece that begins with chunk `chunk` of (b, unit): its first tile and its queries
    auto begin = [&]() {
        const int blocks = units / p.H_kv, kvh = unit / blocks, row0 = (unit - kvh * blocks) * ROWS;
        const Piece next = {b, kvh, row0, min(ROWS, seq.rows - row0), chunk, min(n_chunks, chunk + (end - at)), n_chunks, seq.before};
        token = next.first * CH + 16 * wave;
        page = token / p.page_size;
        in_page = token - page * p.page_size;
        table = p.table + b * p.table_stride;
        head_at = (int64_t)kvh * p.stride_head;
        look_up();
        if (next.first < next.last) request(0);
        const bool has_row = 32 * rg + n < next.rows;
        const int row = row0 + (has_row ? 32 * rg + n : 0), i = row / group, head = kvh * group + row - i * group;
        sees = has_row ? (uint64_t)p.seen[b * p.seen_stride + i] : 0;
        const __bf16* const q_row = (const __bf16*)p.q + b * p.stride_b + i * p.stride_t + head * p.stride_h;
        if (d < 8) load_b_frags<8>(q, q_row, h, d);
        else {
            // (all requested at once, without branches: from the row's last eight columns where a chunk goes beyond them)
            typedef __bf16 Chunk __attribute__((ext_vector_type(8), aligned(8)));
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) q[ks] = *reinterpret_cast<const Chunk*>(q_row + min(16 * ks + 8 * h, d - 8));
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int beyond = 16 * ks + 8 * h + 8 - d;         // columns
                const bf16x8 x = q[ks], z = {0, 0, 0, 0, 0, 0, 0, 0};
                q[ks] = beyond <= 0 ? x : beyond == 4 ? __builtin_shufflevector(x, z, 4, 5, 6, 7, 8, 9, 10, 11) : z;
            }
        }
        return next;
    };
    now = begin();
    for (;;) {
        f32x16 acc[MB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[mb][r] = 0.f;
        float top = -INFINITY, l = 0.f;
        bool saw = false;                       // some token that the row sees, in a page that is one
        for (int t = now.first; t < now.last; ++t) {
            const int buffer = scalar((t - now.first) & 1);
            __builtin_amdgcn_s_waitcnt(0);      // this wavefront's loads have landed ...
            __syncthreads();                    // ... and everyone's; the other buffer has been read
            if (t + 1 < now.last) request(buffer ^ 1);
            if (32 * rg >= now.rows) continue;  // no row here
#pragma unroll 1
            for (int sub = part_of * SUBS; sub < part_of * SUBS + SUBS; ++sub) {
                const char* const k = lds[buffer] + sub * (tile_bytes(DP) / 2);
                const char* const v = k + tile_bytes(DP);
                const int t0 = t * CH + 32 * sub, rows0 = scalar(rows_lds[buffer][2 * sub]), rows1 = scalar(rows_lds[buffer][2 * sub + 1]);
                if (rows0 + rows1 == 0) continue;
                // operands are read from LDS this many products ahead of their use
                constexpr int AHEAD_K = 3, AHEAD_V = 2;
                bf16x8 ka[KS], va[2 * MB];
                auto read_v = [&](int i) { va[i] = dt_read_tr(v + i / MB * 16 * row_bytes(DP), tr0[i % MB], tr1[i % MB]); };
                f32x16 s;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
                for (int ks = 0; ks < AHEAD_K; ++ks) ka[ks] = dt_read_row(k, arow[ks]);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    __builtin_amdgcn_sched_barrier(0);
                    if (ks + AHEAD_K < KS) ka[ks + AHEAD_K] = dt_read_row(k, arow[ks + AHEAD_K]);
                    s = mfma(PART ? zero_beyond_d(ka[ks], ks == part_ks) : ka[ks], q[ks], s);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < AHEAD_V; ++i) read_v(i);
                const bool drafted = t0 + 32 > now.before;
                // register r is seen: a token that there is, in front of the draft or named by the mask
                auto seen = [&](int r, uint64_t mask, int n0, int n1) {
                    const int in = 8 * (r / 4) + 4 * h + r % 4, nth = t0 + in - now.before;
                    return in % 16 < (r < 8 ? n0 : n1) && (nth < 0 || ((mask >> (nth & 63)) & 1));
                };
                if (drafted || rows0 + rows1 < 32) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const bool sees_it = seen(r, sees, rows0, rows1);
                        saw = saw || sees_it;
                        if (!sees_it) s[r] = -INFINITY;
                    }
                } else {
                    saw = true;
                }
                float pr[16], sum = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    pr[r] = __builtin_amdgcn_exp2f(fmaf(s[r], kappa, -top));
                    sum += pr[r];
                }
                if (__builtin_amdgcn_ballot_w64(!(sum < MOST)) != 0) {          // wave-uniform and rare but for the first one
                    float mx = s[0];
#pragma unroll
                    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
                    const float m_new = fmaxf(top, half_wave_max(mx) * kappa), ref = reference(m_new);
                    const float alpha = __builtin_amdgcn_exp2f(top - ref);
                    top = m_new;
                    l *= alpha;
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[mb][r] *= alpha;
                    sum = 0.f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        pr[r] = __builtin_amdgcn_exp2f(fmaf(s[r], kappa, -ref));
                        sum += pr[r];
                    }
                }
                l += sum;
                // values that are no numbers, of tokens that some rows do not see
                uint32_t odd = 0;               // tokens of the sub-tile
                if (drafted) {
#pragma unroll 1
                    for (int y = 0; y < 32; y += 8) {       // eight tokens at a time, eight lanes each
                        const int in = y + lane / 8;
                        bool bad = false;
#pragma unroll
                        for (int c = 0; c < DP / 64; ++c) {
                            typedef uint32_t u32x4a __attribute__((ext_vector_type(4)));
                            const u32x4a w = *reinterpret_cast<const u32x4a*>(v + dt_chunk_at<DP>(in, lane % 8 + 8 * c));
                            bad = bad || odd_word<2>(w[0]) || odd_word<2>(w[1]) || odd_word<2>(w[2]) || odd_word<2>(w[3]);
                        }
                        const uint64_t who = __builtin_amdgcn_ballot_w64(bad);
#pragma unroll
                        for (int e = 0; e < 8; ++e) odd |= ((who >> (8 * e)) & 0xff ? 1u : 0u) << (y + e);
                    }
                    odd = scalar(odd);
                    if (odd) {
                        // (what the masks need is formed anew here, not kept from above for this)
                        uint32_t mask_lo = (uint32_t)sees, mask_hi = (uint32_t)(sees >> 32);
                        int n0 = rows0, n1 = rows1;
                        asm volatile("" : "+v"(mask_lo), "+v"(mask_hi), "+s"(n0), "+s"(n1));
                        const uint64_t mask = (uint64_t)mask_hi << 32 | mask_lo;
#pragma unroll 1
                        for (uint32_t left = odd; left != 0; left &= left - 1) {
                            const int in = __builtin_ctz(left);
                            float w = 0.f;
                            int sees_it = 0;
#pragma unroll
                            for (int r = 0; r < 16; ++r)
                                if (8 * (r / 4) + 4 * h + r % 4 == in) {
                                    w = pr[r];
                                    sees_it = seen(r, mask, n0, n1);
                                }
                            const int owner = n + 32 * ((in >> 2) & 1);         // of the two lanes of a row the one that holds the token
                            w = __shfl(w, owner);
                            sees_it = __shfl(sees_it, owner);
#pragma unroll
                            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                                for (int r = 0; r < 16; ++r) {
                                    const int column = 32 * mb + 8 * (r / 4) + 4 * h + r % 4;
                                    const __bf16 value = *reinterpret_cast<const __bf16*>(v + dt_chunk_at<DP>(in, column / 8) + 2 * (column % 8));
                                    if (sees_it) acc[mb][r] += w * (float)value;
                                }
                        }
                    }
                }
                bf16x8 hi[2], lo[2];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    hi[r / 8][r % 8] = (__bf16)pr[r];
                    lo[r / 8][r % 8] = (__bf16)(pr[r] - (float)hi[r / 8][r % 8]);
                }
#pragma unroll
                for (int i = 0; i < 2 * MB; ++i) {
                    __builtin_amdgcn_sched_barrier(0);
                    if (i + AHEAD_V < 2 * MB) read_v(i + AHEAD_V);
                    if (odd) {                  // (wave-uniform)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if ((odd >> (16 * (i / MB) + 8 * (e / 4) + 4 * h + e % 4)) & 1) va[i][e] = (__bf16)0.f;
                    }
                    acc[i % MB] = mfma(va[i], hi[i / MB], acc[i % MB]);
                    acc[i % MB] = mfma(va[i], lo[i / MB], acc[i % MB]);
                }
            }
        }

        // on to the next piece: its first tile is on its way while this one is joined and written
        const Piece done = now;
        at += now.last - now.first;
        const bool last_piece = WHOLE || at >= end;
        __syncthreads();                        // everyone has read the last tile
        if (!last_piece) {
            chunk = 0;
            if (++unit == units) {
                unit = 0;
                do {
                    ++b;
                    enter();
                } while (n_chunks == 0 || units == 0);
            }
            now = begin();
        }
        l = half_wave_sum(l);
        const uint64_t some = __builtin_amdgcn_ballot_w64(saw);
        if (l == 0.f && (((some >> n) | (some >> (32 + n))) & 1)) l = -1.f;
        if constexpr (SHARING == 2) {
            // the second wavefront's part, through the buffer that the next tile does not go to
            float* const other = reinterpret_cast<float*>(lds[1]) + rg * MB * 16 * 64;
            if (part_of == 1) {
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int r = 0; r < 16; ++r) other[(mb * 16 + r) * 64 + lane] = acc[mb][r];
                if (h == 0) {
                    stat_lds[rg][0][n] = top;
                    stat_lds[rg][1][n] = l;
                }
            }
            meet();
            if (part_of == 0) {
                const float m1 = stat_lds[rg][0][n], l1 = stat_lds[rg][1][n], all = fmaxf(top, m1);
                const float f0 = __builtin_amdgcn_exp2f(top - reference(all)), f1 = __builtin_amdgcn_exp2f(m1 - reference(all));
                float sum = 0.f;
                bool weightless = false;
                add_sum(sum, weightless, l, f0);
                add_sum(sum, weightless, l1, f1);
                l = sum == 0.f && weightless ? -1.f : sum;
                top = all;
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[mb][r] = acc[mb][r] * f0 + other[(mb * 16 + r) * 64 + lane] * f1;
            }
        }
        const int in_unit = 32 * rg + n;
        if (part_of == 0 && in_unit < done.rows) {
            if (done.first == 0 && done.last == done.n_chunks) {
                // no token: zeros; tokens without any weight: no number
                const float inv = l < 0.f ? NAN : l == 0.f ? 0.f : 1.f / l;
                const int at_row = done.row0 + in_unit, i = at_row / group, head = done.kvh * group + at_row - i * group;
                __bf16* const to = (__bf16*)p.out + done.b * p.stride_b + i * p.stride_t + head * p.stride_h;
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int column = 32 * mb + 8 * c + 4 * h;
                        if (column >= d) continue;
                        bf16x4 z;
#pragma unroll
                        for (int e = 0; e < 4; ++e) z[e] = (__bf16)(acc[mb][4 * c + e] * inv);
                        *reinterpret_cast<bf16x4*>(to + column) = z;
                    }
                if (p.lse && h == 0) p.lse[done.b * p.stat_stride_b + i * p.stat_stride_t + head] = l < 0.f ? NAN : (top + __builtin_amdgcn_logf(l)) * LN2;
            } else {
                float* const part = p.parts + ((int64_t)mine * 2 + (done.first > 0 ? 0 : 1)) * part_floats(ROWS, DP);
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        *reinterpret_cast<float4*>(part + in_unit * DP + 32 * mb + 8 * c + 4 * h) =
                            make_float4(acc[mb][4 * c], acc[mb][4 * c + 1], acc[mb][4 * c + 2], acc[mb][4 * c + 3]);
                if (h == 0) {
                    part[ROWS * DP + in_unit] = top;
                    part[ROWS * (DP + 1) + in_unit] = l;
                }
            }
        }
        if (last_piece) break;
    }
}

// Units whose pieces lie in several shares.  (Each has a chunk: a row is one of a drafted token's, cached itself, and the launches that share chunks have room
// for more than one.)

// Where the pieces of a unit lie: shares g0 .. g1; the chunks before it and all, in one pass over the sequences.
struct Pieces { int g0, g1; };
template <int CH, int ROWS>
__device__ inline Pieces pieces_of(const TreeArgs& p, const Sequence& seq, int b, int kvh, int in_unit, int lane) {
    const int n = chunks_of<CH>(seq), unit = kvh * (units_of<ROWS>(p, seq) / p.H_kv) + in_unit / ROWS;
    int before = 0, all = 0;
#pragma unroll 4
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int own = b0 + lane < p.B ? work_of<CH, ROWS>(p, b0 + lane) : 0;
        all += own;
        before += b0 + lane < b ? own : 0;
    }
    all = wave_total(wave_scan(all));
    before = wave_total(wave_scan(before));
    const uint32_t share = (uint32_t)share_of(all, p.n_wgs), from = (uint32_t)(before + unit * n);
    return {(int)(from / share), (int)((from + n - 1) / share)};
}
template <int DP, int ROWS>
__device__ inline const float* piece(const TreeArgs& p, const Pieces& x, int i) {
    return p.parts + ((int64_t)(x.g0 + i) * 2 + (i == 0 ? 1 : 0)) * part_floats(ROWS, DP);
}

// Few rows, whose units then have many pieces: eight wavefronts take a row's in turn, BATCH of them requested at a time (they come from other XCDs'
// workgroups: a round trip to memory each).
constexpr int BATCH = 4, JOIN_WAVES = 8;
template <typename T, int DP, int CH, int ROWS>
__global__ void __launch_bounds__(64 * JOIN_WAVES)
tree_join_kernel(TreeArgs p) {
    constexpr int COLS = (DP + 63) / 64;
    __shared__ float o_lds[JOIN_WAVES][DP], m_lds[JOIN_WAVES], l_lds[JOIN_WAVES];
    const int lane = threadIdx.x & 63, wave = scalar((int)threadIdx.x >> 6);
    const int group = p.H / p.H_kv, at_row = (int)blockIdx.x;
    const int b = at_row / (p.T * p.H), t = (at_row - b * p.T * p.H) / p.H, head = at_row - (b * p.T + t) * p.H;
    Sequence seq = sequence(p, b);
    seq = {scalar(seq.before), scalar(seq.len), scalar(seq.rows)};
    const int kvh = head / group, in_unit = t * group + head - kvh * group, row = in_unit % ROWS;
    if (in_unit >= seq.rows) return;
    const Pieces x = pieces_of<CH, ROWS>(p, seq, b, kvh, in_unit, lane);
    if (x.g0 == x.g1) return;
    const int pieces = x.g1 - x.g0 + 1;
    float m = -INFINITY, l = 0.f, acc[COLS] = {};
    bool weightless = false;
    for (int i0 = wave * BATCH; i0 < pieces; i0 += JOIN_WAVES * BATCH) {
        float mg[BATCH], lg[BATCH], y[BATCH][COLS];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const float* part = piece<DP, ROWS>(p, x, min(i0 + i, pieces - 1));
            mg[i] = part[ROWS * DP + row];
            lg[i] = part[ROWS * (DP + 1) + row];
#pragma unroll
            for (int c = 0; c < COLS; ++c) y[i][c] = lane + 64 * c < p.d ? part[row * DP + lane + 64 * c] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            if (i0 + i >= pieces) break;
            const float top = fmaxf(m, mg[i]), a = __builtin_amdgcn_exp2f(m - reference(top)), f = __builtin_amdgcn_exp2f(mg[i] - reference(top));
            l *= a;
            add_sum(l, weightless, lg[i], f);
#pragma unroll
            for (int c = 0; c < COLS; ++c) acc[c] = acc[c] * a + y[i][c] * f;
            m = top;
        }
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
    T* const to = (T*)p.out + b * p.stride_b + t * p.stride_t + head * p.stride_h;
    for (int col = threadIdx.x; col < p.d; col += 64 * JOIN_WAVES) {
        float y = 0.f;
#pragma unroll
        for (int w = 0; w < JOIN_WAVES; ++w) y += o_lds[w][col] * f[w];
        if constexpr (sizeof(T) == 2) reinterpret_cast<__bf16*>(to)[col] = (__bf16)(y * inv);
        else to[col] = y * inv;
    }
    if (p.lse && threadIdx.x == 0) p.lse[b * p.stat_stride_b + t * p.stat_stride_t + head] = (top + __builtin_amdgcn_logf(sum)) * LN2;
}

// Many rows: a wavefront has four neighbouring ones of a unit, 16 lanes each, which have their pieces in common.  (A wavefront a row: 21 us for 32 sequences'
// drafts of up to 32, 32 heads, where this takes 12.)
template <typename T, int DP, int CH, int ROWS>
__global__ void __launch_bounds__(256)
tree_join_rows_kernel(TreeArgs p) {
    constexpr int COLS = DP / 16, TWO = 2;      // columns a lane; pieces requested at a time
    typedef float Floats __attribute__((ext_vector_type(COLS < 4 ? COLS : 4)));
    constexpr int W = COLS < 4 ? COLS : 4, N = COLS / W;
    const int lane = threadIdx.x & 63, group = p.H / p.H_kv, fours = (p.T * group + 3) / 4;
    const int at = scalar((int)blockIdx.x * 4 + ((int)threadIdx.x >> 6)), b = at / (p.H_kv * fours), kvh = (at - b * p.H_kv * fours) / fours;
    if (b >= p.B) return;
    const int first = 4 * (at - (b * p.H_kv + kvh) * fours), in_unit = first + lane / 16, row = in_unit % ROWS;
    Sequence seq = sequence(p, b);
    seq = {scalar(seq.before), scalar(seq.len), scalar(seq.rows)};
    if (first >= seq.rows) return;
    const Pieces x = pieces_of<CH, ROWS>(p, seq, b, kvh, first, lane);
    if (x.g0 == x.g1) return;
    const int pieces = x.g1 - x.g0 + 1;
    float m = -INFINITY, l = 0.f;
    Floats acc[N] = {};
    bool weightless = false;
    for (int i0 = 0; i0 < pieces; i0 += TWO) {
        float mg[TWO], lg[TWO];
        Floats y[TWO][N];
#pragma unroll
        for (int i = 0; i < TWO; ++i) {
            const float* part = piece<DP, ROWS>(p, x, min(i0 + i, pieces - 1));
            mg[i] = part[ROWS * DP + row];
            lg[i] = part[ROWS * (DP + 1) + row];
#pragma unroll
            for (int c = 0; c < N; ++c) y[i][c] = *reinterpret_cast<const Floats*>(part + row * DP + W * (lane % 16 + 16 * c));
        }
#pragma unroll
        for (int i = 0; i < TWO; ++i) {
            if (i0 + i >= pieces) break;
            const float top = fmaxf(m, mg[i]), a = __builtin_amdgcn_exp2f(m - reference(top)), f = __builtin_amdgcn_exp2f(mg[i] - reference(top));
            l *= a;
            add_sum(l, weightless, lg[i], f);
#pragma unroll
            for (int c = 0; c < N; ++c) acc[c] = acc[c] * a + y[i][c] * f;
            m = top;
        }
    }
    if (in_unit >= seq.rows) return;
    if (weightless && l == 0.f) l = NAN;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int t = in_unit / group, head = kvh * group + in_unit - t * group;
    T* const to = (T*)p.out + b * p.stride_b + t * p.stride_t + head * p.stride_h;
#pragma unroll
    for (int c = 0; c < N; ++c) {
        const int col = W * (lane % 16 + 16 * c);
        if (col >= p.d) continue;
        if constexpr (sizeof(T) == 2) {
            typedef __bf16 Out __attribute__((ext_vector_type(W)));
            Out z;
#pragma unroll
            for (int e = 0; e < W; ++e) z[e] = (__bf16)(acc[c][e] * inv);
            *reinterpret_cast<Out*>(to + col) = z;
        } else {
            *reinterpret_cast<Floats*>(to + col) = acc[c] * inv;
        }
    }
    if (p.lse && lane % 16 == 0) p.lse[b * p.stat_stride_b + t * p.stat_stride_t + head] = (m + __builtin_amdgcn_logf(l)) * LN2;
}

constexpr int columns(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 128 ? 128 : 256; }
constexpr int tile_columns(int d) { return d <= 64 ? 64 : 128; }
// tree_tiles_kernel's launches
constexpr bool in_tiles(int rows, int d, int dtype) { return dtype == SA_BF16 && d <= 128 && rows > 16; }
// of those, launches of few units and tokens, which 16 rows a unit take less time for although they read the cache once for each: more workgroups share
// them, and code and parts are smaller.  us, tiles : 16 rows, d 128, 32 heads on 8 if not said: 8 drafted tokens (32 rows a unit), one sequence of 1500
// 17.8 : 13.8, 6000 24.2 : 18.7, 16000 32.0 : 30.0, 24000 36.9 : 39.2, 60000 58 : 81; 32 drafted, 1500 x 4 34.6 : 29.3, 6000 48 : 30, 16000 62 : 85; 32 of 1500,
// 8 heads on 1, 29.6 : 22.3; but 16 of 300, 32 drafted (1024 units) 24.6 : 35.1, 64 of 500, 16 drafted 34.6 : 86.9.
bool in_few_rows(const TreeArgs& a) {
    const int64_t units = (int64_t)a.B * a.H_kv * ((a.T * (a.H / a.H_kv) + 15) / 16);
    return units <= 256 && units * a.max_pages * a.page_size <= 400000;
}
constexpr int row_groups(int rows) { return rows <= 64 ? 2 : 4; }
constexpr int workgroups(int DP) { return N_CU * (DP > 128 ? 1 : 2); }

template <int ROWS>
unsigned all_units(const TreeArgs& a) { return (unsigned)(a.B * a.H_kv * ((a.T * (a.H / a.H_kv) + ROWS - 1) / ROWS)); }
// A workgroup a row where rows are few or units have 32 pieces and more (us, this : four rows a wavefront, whole call, 32 heads on 8 if not said: one
// sequence of 16000 tokens, 32 drafted, 44.5 : 62.2; 2 of 16171, 8 on 1, 35, 41 : 66; 5 of 10000, 8 on 1, 15, 27 : 50; 2 of 8000, 32, 43.7 : 47.0; but 16 of
// 4000, 8 on 1, 32, 16 pieces, 58 : 48; 8 of 4000, 32, 8 pieces, 85 : 60).
template <typename T, int DP, int CH, int ROWS>
hipError_t join(const TreeArgs& a, hipStream_t st) {
    const int64_t all = (int64_t)a.B * a.T * a.H, fours = (int64_t)a.B * a.H_kv * ((a.T * (a.H / a.H_kv) + 3) / 4);
    if (all <= 512 || (int64_t)all_units<ROWS>(a) * 32 <= a.n_wgs) hipLaunchKernelGGL((tree_join_kernel<T, DP, CH, ROWS>), dim3((unsigned)all), dim3(64 * JOIN_WAVES), 0, st, a);
    else hipLaunchKernelGGL((tree_join_rows_kernel<T, DP, CH, ROWS>), dim3((unsigned)((fours + 3) / 4)), dim3(64 * 4), 0, st, a);
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch(TreeArgs a, hipStream_t st) {
    // (decode.hip's rule for units of a workgroup each)
    if ((int64_t)a.max_pages * a.page_size <= (DP > 128 ? 4 : 8) * CHUNK<T>) {
        hipLaunchKernelGGL((tree_kernel<T, DP, true>), dim3(all_units<16>(a)), dim3(64 * WAVES), 0, st, a);
        return hipGetLastError();
    }
    a.n_wgs = workgroups(DP);
    hipLaunchKernelGGL((tree_kernel<T, DP, false>), dim3((unsigned)a.n_wgs), dim3(64 * WAVES), 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
    return join<T, DP, CHUNK<T>, 16>(a, st);
}
template <typename T>
hipError_t launch(const TreeArgs& a, hipStream_t st) {
    switch (columns(a.d)) {
        case 32: return launch<T, 32>(a, st);
        case 64: return launch<T, 64>(a, st);
        case 128: return launch<T, 128>(a, st);
        default: return launch<T, 256>(a, st);
    }
}
template <int DP, int R, bool PART>
hipError_t launch_tiles(TreeArgs a, hipStream_t st) {
    if ((int64_t)a.max_pages * a.page_size <= 16 * TILE_CHUNK) {
        hipLaunchKernelGGL((tree_tiles_kernel<DP, R, PART, true>), dim3(all_units<32 * R>(a)), dim3(64 * WAVES), 0, st, a);
        return hipGetLastError();
    }
    a.n_wgs = workgroups(DP);
    hipLaunchKernelGGL((tree_tiles_kernel<DP, R, PART, false>), dim3((unsigned)a.n_wgs), dim3(64 * WAVES), 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
    return join<__hip_bfloat16, DP, TILE_CHUNK, 32 * R>(a, st);
}
template <int DP, bool PART>
hipError_t launch_tiles(const TreeArgs& a, hipStream_t st) {
    return row_groups(a.T * (a.H / a.H_kv)) == 2 ? launch_tiles<DP, 2, PART>(a, st) : launch_tiles<DP, 4, PART>(a, st);
}

}  // namespace

int64_t tree_workspace(int rows, int d, int dtype) {
    if (in_tiles(rows, d, dtype)) return (int64_t)workgroups(tile_columns(d)) * 2 * part_floats(32 * row_groups(rows), tile_columns(d)) * 4;
    return (int64_t)workgroups(columns(d)) * 2 * part_floats(16, columns(d)) * 4;
}

hipError_t launch_tree(const TreeArgs& a, int dtype, hipStream_t st) {
    if (dtype == SA_F32) return launch<float>(a, st);
    if (in_tiles(a.T * (a.H / a.H_kv), a.d, dtype) && !in_few_rows(a)) {
        if (a.d <= 64) return a.d % 8 ? launch_tiles<64, true>(a, st) : launch_tiles<64, false>(a, st);
        return a.d % 8 ? launch_tiles<128, true>(a, st) : launch_tiles<128, false>(a, st);
    }
    return launch<__hip_bfloat16>(a, st);
}

}  // namespace sa
