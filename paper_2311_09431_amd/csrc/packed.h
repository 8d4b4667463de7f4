// Packed sequences: rows of n_seq sequences lie end to end, sequence s in rows offsets[s] .. offsets[s + 1] - 1, and attend
// causally to themselves.  A sequence is one triangular block of the ring step's kernels; what is added here is how a
// workgroup finds its own.
#pragma once
#include "mfma_tiles.h"
#include "sa_internal.h"
#include "wave.h"

namespace sa {

// StepArgs of one block (B = 1, one device, triangular), its pointers those of row 0; c is set by the workgroup
struct PackedArgs : StepArgs {
    const int32_t* offsets;     // device, n_seq + 1
    int n_seq, rows, max_len;   // rows of the tensors; rows of a sequence beyond max_len are not looked at
    int n_ranks;                // tiles of all sequences, at most
    int es;                     // bytes of an element
    bool by_rank;               // workgroup order: by ranks over all heads, or in groups of heads (decode_block)
};

// Tiles of `tile` rows that sequences without a common row can have, whatever their lengths.  (Of sequences that share rows there can be more; a
// launch then leaves out the lightest.)
inline int64_t most_tiles(const PackedArgs& p, int tile) {
    const int64_t each = ((int64_t)p.max_len + tile - 1) / tile, by_rows = (int64_t)p.rows / tile + p.n_seq;
    return each * p.n_seq < by_rows ? each * p.n_seq : by_rows;
}

// Order of a bf16 launch's 128-row tiles: by ranks over all heads, which leaves the lightest tiles to the end, but in groups of heads, whose K and V
// (Q and dO) an XCD's cache then serves, where those of all are too many for the cache behind it.  us, groups : ranks, forward: d 100, 6 sequences of
// up to 4096, 32 heads (227 MB) 514 : 586, 64 (453 MB) .76, 2 of up to 8192, 32 heads (196 MB) 850 : 881; but 16 heads 1, 3 of up to 4096, 64
// heads (168 MB, 54 tiles) 357 : 340, 64 of up to 300, 64 heads (258 MB) 1.08; four query heads share them: 8 of up to 4096, 32 on 8, d 128,
// 564 : 554, 16 of up to 1000 100 : 96.  Over 336 forward launches, d 100 to 256, 0.3 % from the better of the two, ranks always 2.8.  Whole
// training pass, d 128, 6 of up to 4096, 64 heads, 4763 : 5201, 2 of up to 8192 7868 : 8267, 3 of up to 4096 1596 : 1533, 64 of up to 300
// 927 : 908, d 256 11048 : 12182, 18441 : 19421, 3560 : 3495, 1989 : 1863.
inline bool by_rank_wanted(const PackedArgs& p) {
    return 4. * p.rows * p.H_kv * p.d < 180e6 * (p.H / p.H_kv) || p.n_ranks < 64 || p.max_len < 400;
}

// Rows first .. first + len - 1 of sequence s.  Whatever the offsets hold, they lie within the tensors: an offset below zero or
// behind the last row is taken as the nearest one that is none, a sequence that ends before it begins is empty.
struct Span { int first, len; };
__device__ inline Span span_of(const PackedArgs& p, int s) {
    const int first = min(max(p.offsets[s], 0), p.rows), end = min(max(p.offsets[s + 1], first), p.rows);
    return {first, min(end - first, p.max_len)};
}
template <int TILE>
__device__ inline int tiles_of(Span x) { return (x.len + TILE - 1) / TILE; }

hipError_t launch_packed_fwd(PackedArgs p, hipStream_t st);
hipError_t launch_packed_bwd(const PackedArgs& p, hipStream_t st);
hipError_t launch_packed_bwd_ring(const PackedArgs& p, bool both, hipStream_t st);     // dK and dV at 65 to 128 columns; both: dQ too
hipError_t launch_packed_dkdv_wide(const PackedArgs& p, unsigned workgroups, hipStream_t st);         // above 128, all of them in a workgroup
// bf16 launches of few tiles (the backward's forms delta too)
bool packed_split_wanted(const PackedArgs& p, bool backward);
hipError_t launch_packed_split(PackedArgs p, bool backward, hipStream_t st);
// the other rules of the bf16 backward (packed_bwd.hip; n_ranks: 128-row tiles), and of fp32 (packed_f32.hip: up to 128 columns, above)
bool packed_one_launch(const PackedArgs& p);
bool packed_two_wavefronts(const PackedArgs& p);
bool packed_all_columns(const PackedArgs& p);
F32Route packed_f32_route(const PackedArgs& p, bool backward);
bool packed_f32_few(const PackedArgs& p, bool backward);
// (placed_kinds; as a ring step's, from 0.5 to 3 the same to 2 %)
inline double packed_ratio(const PackedArgs& p) { return p.H == p.H_kv ? 1.45 : 0.; }
hipError_t launch_packed_delta(const PackedArgs& p, int dtype, hipStream_t st);
hipError_t launch_packed_f32(PackedArgs p, bool backward, hipStream_t st);
hipError_t launch_packed_f32x3(PackedArgs p, bool backward, hipStream_t st);
hipError_t launch_packed_f32x3_split(PackedArgs p, bool backward, hipStream_t st);

// A lane's sum of tiles that weigh w or more, with those of one sequence more.  It stops above any rank (a launch has fewer workgroups):
// offsets that give the same rows to many sequences could pass 2^31, and a search that goes by a wrapped sum could leave the table.
constexpr int MOST_COUNTED = 1 << 24;
__host__ __device__ inline int add_tiles(int sum, int tiles, int w) {
    const int next = sum + (tiles >= w ? tiles - w + 1 : 0);
    return next < MOST_COUNTED ? next : MOST_COUNTED;
}

// Tile `rank` of all sequences' tiles, the heaviest first: a sequence of t tiles has one of each weight 1 .. t (query tile i
// walks i + 1 key tiles, key tile i is walked by t - i query tiles).  C(w) = sum over sequences of max(0, t - w + 1) tiles weigh w or
// more; the tile's weight is the largest w with C(w) > rank, found by halving, and among the sequences that have one of it the tile is
// that of number rank - C(w + 1).  Every wavefront looks for itself, 64 sequences at a time in its lanes.  False: fewer tiles than that.
// The first 64 sequences stay in registers: about 1 us.  Of more every sum reads the others' offsets again, n_seq / 64 rounds in turn, so a launch's
// lookups grow with n_seq times its tiles.  ns a row, 64, 256, 1000, 4000 sequences of 16 to 256 rows, 16 heads: forward, d 128, 4.9, 5.5, 6.7,
// 12.3, d 64 3.0, 2.7, 4.2, 8.4; backward 16.0, 17.2, 20.5, 38, d 64 10.4, 11.8, 16.3, 34; fp32, d 128, forward 17.9, 15.9, 16.3, 20.9.
template <int TILE>
__device__ inline bool find_tile(const PackedArgs& p, int rank, int& seq, int& weight) {
    const int lane = threadIdx.x & 63;
    const int own = lane < p.n_seq ? tiles_of<TILE>(span_of(p, lane)) : 0;      // of the first 64 sequences
    auto count = [&](int w) {
        int n = add_tiles(0, own, w);
        for (int s = 64 + lane; s < p.n_seq; s += 64) n = add_tiles(n, tiles_of<TILE>(span_of(p, s)), w);
        return wave_total(wave_scan(n));
    };
    int behind = count(1);
    if (rank >= behind) return false;
    int lo = 1, hi = (p.max_len + TILE - 1) / TILE + 1;      // C(lo) > rank >= C(hi)
    behind = 0;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1, c = count(mid);
        if (c > rank) lo = mid;
        else {
            hi = mid;
            behind = c;
        }
    }
    weight = lo;
    int left = rank - behind;           // so many sequences with such a tile come before it
    for (int s0 = 0; s0 < p.n_seq; s0 += 64) {
        const int t = s0 == 0 ? own : s0 + lane < p.n_seq ? tiles_of<TILE>(span_of(p, s0 + lane)) : 0;
        const uint64_t has = __builtin_amdgcn_ballot_w64(t >= lo);
        const int n = __builtin_popcountll(has);
        if (left < n) {
            const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(has >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)has, 0));
            const uint64_t mine = __builtin_amdgcn_ballot_w64(t >= lo && before == left);
            seq = s0 + (int)__builtin_ctzll(mine);
            return true;
        }
        left -= n;
    }
    return false;                       // (not reached: C counted them)
}

// The workgroup's sequence, tile and head: p becomes the arguments of a launch on that sequence alone, n_tiles its tiles,
// rank the tile's place among them (0: the heaviest).  False: none, the launch has more workgroups than there are tiles.  which: gets the sequence.
template <bool SNAKE, int TILE>
__device__ inline bool enter_sequence(PackedArgs& p, int linear, int n_heads, int& n_tiles, int& rank, int& head, int* which = nullptr) {
    if (p.by_rank) decode_block<SNAKE, true>(linear, p.n_ranks, n_heads, rank, head);
    else decode_block<SNAKE, false>(linear, p.n_ranks, n_heads, rank, head);
    int seq, weight;
    if (!find_tile<TILE>(p, rank, seq, weight)) return false;
    if (which) *which = seq;
    const Span x = span_of(p, seq);
    const int first = __builtin_amdgcn_readfirstlane(x.first);
    p.c = __builtin_amdgcn_readfirstlane(x.len);
    n_tiles = (p.c + TILE - 1) / TILE;
    rank = n_tiles - weight;
    const int64_t q = p.es * p.stride_s * first, kv = p.es * p.kv_stride_s * first;         // bytes
    p.q = (const char*)p.q + q;
    p.k = (const char*)p.k + kv;
    p.v = (const char*)p.v + kv;
    p.dout = (const char*)p.dout + q;
    p.o = (float*)((char*)p.o + q);
    p.dq = (float*)((char*)p.dq + q);
    p.dk = (float*)((char*)p.dk + kv);
    p.dv = (float*)((char*)p.dv + kv);
    p.lse += first;
    p.delta += first;
    return true;
}

}  // namespace sa
