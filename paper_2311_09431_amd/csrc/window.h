// Attention with a sliding window and a few first tokens that stay visible, over packed sequences (packed.h): row a of a sequence sees key b where
// b <= a and (a - b < window or b < sinks).  The packed kernels' workgroups, whose walk leaves out the tiles that no row of theirs sees: a
// query-owning one's goes over the tiles with first keys, then on to those of its rows' windows; a key-owning one's ends with the last row
// whose window reaches back to its keys.
//
// What the rows further on add to dK and dV of the first keys is, but for short ways, formed by workgroups of their own (window_far.hip), each for a part of
// a sequence's rows: in the key-owning workgroup it would be a walk over the whole sequence beside others of a window's length.  Such keys'
// sums stay in fp32 in the workspace, of the window's rows and of each part's, until they are put together.
#pragma once
#include "f32_rows.h"
#include "packed.h"

namespace sa {

struct WindowArgs : PackedArgs {
    int window, sinks;          // 1 .. max_len, 0 .. max_len
    // backward, workspace: slots of H_kv x key_rows x (dV, dK) x d, one of a sequence's windows and one of each `part` of its rows behind
    float* work;
    int part, key_rows, n_slots;
    int slot;                   // the sequence's first one, set by the workgroup; -1: none
};
// Whether there are such workgroups: two launches more, against the time of a walk, rows of all heads of a group.  (Gradient in
// us, walking on / with them.  bf16: 1 x 1100 rows, 4 heads, 64 columns, window 64: 55.5 / 43.0; 4 x 1100, 8 heads, 128 columns, window 256: 80.5 /
// 77.0; 1 x 600: 41.4 / 42.4; 8 x 300, 16 heads, 100 columns: 55.2 / 77.5.  fp32, the same four: 114 / 63, 221 / 193, 69.6 / 40.7, 137 / 157.)
// The rows of a part, as many as make about 1024 workgroups of all (key/value heads and blocks of 16 first keys are workgroups too) but two tiles a
// wavefront, one with groups of four heads or more (3449 rows, 16 heads on 2, window 18, 130 first keys, gradient: 183 us, of 256 a block 878; 7921, 4 on 1, 44, 130: 148,
// 447), and the slots that sequences without a common row can have; 0: key-owning workgroups walk on.
//
// Many first keys fill the chip by themselves while all walk on, where blocks of 16 have work in proportion: key/value heads times blocks times all
// rows, against the longest walk's.  (With parts of 256 rows a block, fp32 128: 1 x 16384, 8 heads, 128 columns, window 1024, first keys 64, 256, 512, 2048, walking on / with them: 741 / 394, 750 / 613,
// 762 / 1169, 892 / 2449, fp32 3065 / 1677, 3139 / 2334, 3090 / 3218, 3677 / 11938; 4 of up to 4000, 32 heads on 8, 500, first keys 64, 256: 792 / 615,
// 794 / 1455; 1 x 8000, 8 heads on 2, 64 columns, 500, 1024, 3000: 928 / 530, 1005 / 1271.)
inline bool has_far(const WindowArgs& p) {
    const int64_t behind = p.max_len - p.window;
    return p.sinks > 0 && behind * (p.H / p.H_kv) > (p.es == 2 ? 1024 : 256) &&
           (double)p.H_kv * (p.key_rows / 16) * p.rows <= 192. * (double)behind;
}
inline void set_far(WindowArgs& p) {
    p.key_rows = (int)(((int64_t)p.sinks + 15) / 16 * 16);
    p.n_slots = 0;
    if (!has_far(p)) return;
    const int64_t all = (int64_t)p.n_seq * p.max_len, rows = all < p.rows ? all : p.rows;
    const int least = (p.es == 2 ? 128 : 64) * (p.H / p.H_kv < 4 ? 2 : 1);
    const int64_t each = rows * p.H_kv * (p.key_rows / 16) / 1024;
    p.part = (int)((each / least + 1) * least);
    const int64_t longer = rows / (p.window + 1) < p.n_seq ? rows / (p.window + 1) : p.n_seq;      // sequences that are longer than the window
    const int64_t slots = 2 * longer + rows / p.part;
    p.n_slots = slots < (1 << 24) ? (int)slots : 0;         // (more: more than a launch takes)
}
inline int64_t far_bytes(const WindowArgs& p) { return (int64_t)p.n_slots * p.H_kv * p.key_rows * 2 * p.d * 4; }
hipError_t launch_window_far(const WindowArgs& p, int dtype, hipStream_t st);
hipError_t launch_window_fwd(WindowArgs p, hipStream_t st);
int window_split_waves(const WindowArgs& p);                                           // workgroups of 32 rows (packed_split.hip); 0: not wanted
hipError_t launch_window_split(WindowArgs p, int waves, hipStream_t st);
bool window_bwd_split_wanted(const WindowArgs& p);
hipError_t launch_window_bwd_split(WindowArgs p, hipStream_t st);
hipError_t launch_window_bwd(WindowArgs p, hipStream_t st);
hipError_t launch_window_f32(WindowArgs p, bool backward, hipStream_t st);
hipError_t launch_window_f32x3(WindowArgs p, bool backward, hipStream_t st);           // up to 128 columns
hipError_t launch_window_f32x3_split(WindowArgs p, bool backward, hipStream_t st);     // by workgroups of 32 rows

// the first key of row a's window
__device__ inline int window_start(const WindowArgs& p, int a) { return max(0, a - p.window + 1); }
// one past the last row that a key-owning workgroup walks to for keys first .. last
__device__ inline int walk_end(const WindowArgs& p, int first, int last) { return p.n_slots == 0 && first < p.sinks ? p.c : min(p.c, last + p.window); }
__device__ inline int walk_end(const WindowArgs& p, int key) { return walk_end(p, key, key); }
// the key's sums are put together from those of its window's rows and those further on
__device__ inline bool is_far(const WindowArgs& p, int key) { return p.n_slots > 0 && key < p.sinks && key + p.window < p.c; }
// slots of a sequence of len rows; of those before sequence seq (a wavefront's lanes take the sequences in turn)
__device__ inline int slots_of(const WindowArgs& p, int len) { return p.n_slots > 0 && len > p.window ? 1 + (len - p.window + p.part - 1) / p.part : 0; }
__device__ inline int slots_before(const WindowArgs& p, int seq) {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int s = lane; s < seq; s += 64) {
        const int next = n + slots_of(p, span_of(p, s).len);
        n = next < MOST_COUNTED ? next : MOST_COUNTED;          // (as add_tiles)
    }
    return wave_total(wave_scan(n));
}
// A key-owning workgroup's slot, where its keys have one: sequences without a common row have n_slots, of others the last ones may have none.
__device__ inline int find_slot(const WindowArgs& p, int seq, int k0) {
    if (k0 >= p.sinks || p.c <= p.window) return -1;
    const int slot = slots_before(p, seq);
    return slot < p.n_slots ? slot : -1;
}
// a key's dV and dK, d columns each, in a slot
__device__ inline float* slot_row(const WindowArgs& p, int slot, int kvh, int key) {
    return p.work + (((int64_t)slot * p.H_kv + kvh) * p.key_rows + key) * 2 * p.d;
}

// A walk over key tiles of TK rows without pairs: where it begins, and the tile behind the one at t0; start: the window's first sub-tile of 32
__device__ inline int first_tile(const WindowArgs& p, int start) { return p.sinks == 0 ? start : 0; }
template <int TK>
__device__ inline int next_tile(const WindowArgs& p, int t0, int start) {
    const int t = t0 + TK;
    return t >= p.sinks && t < start ? start : t;
}
// row a sees `key`, of those up to its own
__device__ inline bool in_window(const WindowArgs& p, int key, int a) { return key > a - p.window || key < p.sinks; }

// The walk of a query-owning workgroup of PAIR rows from q0 on, over tiles of PAIR keys, `tiles` of them up to its own.
template <int PAIR>
struct WindowWalk {
    int firsts = 0, start = 0, masked = 0, n = 0;      // tiles with first keys; the window's first one; up to where some row does not see a key; all
    __device__ WindowWalk() {}
    __device__ WindowWalk(const WindowArgs& p, int q0, int tiles) {
        start = window_start(p, q0) / PAIR;
        firsts = min(start, (p.sinks + PAIR - 1) / PAIR);
        n = firsts + tiles - start;
        // (the last row's window begins above this; those with first keys are few, and masked too)
        const int below = q0 + PAIR - 1 - p.window;
        masked = below < 0 ? 0 : min(n - 1, firsts + below / PAIR + 1 - start);
    }
    __device__ int at(int i) const { return i < firsts ? i : i - firsts + start; }
    // where the keys of its tile i end that some row can see (whole: bytes up to the last row's end, as a descriptor has them): in the tiles of first keys with
    // the last of these.  The loads deliver zeros for those behind them, or one of these that is no number would send all later rows to be done over.
    __device__ int reach(const WindowArgs& p, int i, int whole, int pitch) const {
        return __builtin_amdgcn_readfirstlane(i < firsts ? whole - (p.c - min(p.sinks, p.c)) * pitch : whole);
    }
};
// the same for tiles of TK rows, as a number of rows
template <int TK>
__device__ inline int rows_to_read(const WindowArgs& p, int t0, int start) { return t0 + TK <= start ? min(p.sinks, p.c) : p.c; }

// Rows done over, as f32_rows.h has them: nothing but the pairs that the mask allows, one wavefront a row.  The tiles multiply masked pairs with
// a weight of zero, of which an infinite or NaN element makes a NaN.
//
// A wavefront goes over 64 of a row's keys in about 7 us (128 columns, bf16: rows come from the L2, 16 on their way), and has up to 32 rows to do over
// one after the other.  So what is bound to be no number is settled as soon as that is known: a row whose sum is none (bf16), with a NaN or +inf score (fp32),
// without a number for its LSE or delta (gradient), sums whose every column is NaN; and dV stays where dK alone is none.  4096 rows, 16 heads on 8, window
// 512, all NaN: forward 56, gradient 239 us (of numbers 49 and 145; walked to the end 6600 and 36700).  What stays are rows and keys within a
// tile of those that see what is no number: a value of NaN 1.5 and 5.1 ms, in windows of 4096 12 and 44.
__device__ inline void store1(float* to, float x) { *to = x; }
__device__ inline void store1(__hip_bfloat16* to, float x) { *reinterpret_cast<__bf16*>(to) = (__bf16)x; }

// Some register of NB 32-column blocks from column col0 on is infinite or NaN.  PART: columns from d on hold what follows the rows, and are not
// looked at.
template <int NB, bool PART, typename Acc>
__device__ inline bool window_odd(const Acc& acc, int h, int d, int col0 = 0) {
    if constexpr (!PART) return not_finite<NB>(acc);
    float z = 0.f;
#pragma unroll
    for (int mb = 0; mb < NB; ++mb)
#pragma unroll
        for (int r = 0; r < 16; ++r) z = fmaf(col0 + 32 * mb + reg_row(r, h) < d ? acc[mb][r] : 0.f, 0.f, z);
    return z != 0.f;
}
// Sums of products as a row done over has them: bf16's products are whole in fp32, fp32's are summed in fp64 (f32_rows.h).
template <typename T> struct RowSum { typedef double Type; };
template <> struct RowSum<__hip_bfloat16> { typedef float Type; };
// a lane's number and its 15 neighbours'
template <int TURN> __device__ inline float turned(float x) { return __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), 0x120 + TURN, 0xf, 0xf, true)); }
template <int TURN> __device__ inline double turned(double x) {
    return __hiloint2double(__builtin_amdgcn_mov_dpp(__double2hiint(x), 0x120 + TURN, 0xf, 0xf, true), __builtin_amdgcn_mov_dpp(__double2loint(x), 0x120 + TURN, 0xf, 0xf, true));
}
template <typename S> __device__ inline S sum_of_16(S x) {
    x += turned<8>(x);
    x += turned<4>(x);
    x += turned<2>(x);
    return x + turned<1>(x);
}
// This lane's number, formed anew, so that nothing of these rows is kept in a register before them.
__device__ inline int lane_anew() {
    int x = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+v"(x));
    return x;
}
// four elements as they lie in memory
template <typename T> struct Four;
template <> struct Four<float> {
    float4 raw;
    __device__ void load(const float* p) { raw = *reinterpret_cast<const float4*>(p); }
    __device__ float at(int i) const { return i == 0 ? raw.x : i == 1 ? raw.y : i == 2 ? raw.z : raw.w; }
};
template <> struct Four<__hip_bfloat16> {
    uint2 raw;
    __device__ void load(const __hip_bfloat16* p) { raw = *reinterpret_cast<const uint2*>(p); }
    __device__ float at(int i) const {
        const uint32_t w = i < 2 ? raw.x : raw.y;
        return __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
    }
};
// Rows that are asked for before one is looked at: else a row's way from the L2, most of a microsecond, would come 64 times.
template <typename T> constexpr int AHEAD = sizeof(T) == 2 ? 16 : 8;
// Lane i: x times row i of n (of the last ones that of row n - 1).  16 lanes read a row together, each has 16 rows.
template <typename T>
__device__ inline float window_dots(const T* x, const T* rows, int64_t ss, int n, int d, int lane) {
    typedef typename RowSum<T>::Type S;
    S sum[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] = 0;
#pragma unroll 1
    for (int col0 = 0; col0 < d; col0 += 64) {
        const int col = col0 + 4 * (lane & 15), at = min(col, d - 4);
        Four<T> own;
        own.load(x + at);
#pragma unroll
        for (int i0 = 0; i0 < 16; i0 += AHEAD<T>) {
            Four<T> y[AHEAD<T>];
#pragma unroll
            for (int i = 0; i < AHEAD<T>; ++i) y[i].load(rows + min((lane & 48) + i0 + i, n - 1) * ss + at);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < AHEAD<T>; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[i0 + i] = fma(col < d ? (S)own.at(e) : S(0), col < d ? (S)y[i].at(e) : S(0), sum[i0 + i]);
        }
    }
    float mine = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float total = (float)sum_of_16(sum[i]);
        if ((lane & 15) == i) mine = total;
    }
    return mine;
}
// A lane has four columns, from `col` on (of the last lanes those of an earlier one, which are not stored).
__device__ inline int window_col(int col0, int end_col, int lane) { return min(col0 + 4 * lane, end_col - 4); }
// acc += sum over n rows of rows' weights (lane i holds row i's)
template <typename T>
__device__ inline void window_add(float4& acc, float weight, const T* rows, int64_t ss, int n, int col) {
    typedef typename RowSum<T>::Type S;
    S sum[4] = {0, 0, 0, 0};
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += AHEAD<T>) {
        int first = i0;
        asm volatile("" : "+v"(first));         // (rows' places in vector registers, of which there are enough here)
        Four<T> x[AHEAD<T>];
#pragma unroll
        for (int i = 0; i < AHEAD<T>; ++i) x[i].load(rows + min(first + i, n - 1) * ss + col);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < AHEAD<T>; ++i) {
            if (i0 + i >= n) break;
            const S w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), i0 + i));
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = fma(w, (S)x[i].at(e), sum[e]);
        }
    }
    acc.x += (float)sum[0];
    acc.y += (float)sum[1];
    acc.z += (float)sum[2];
    acc.w += (float)sum[3];
}
// No column of a sum can become a number any more.
__device__ inline bool lost(float4 x) {
    return __builtin_amdgcn_ballot_w64(x.x == x.x || x.y == x.y || x.z == x.z || x.w == x.w) == 0;
}
__device__ inline float4 no_numbers() { return make_float4(NAN, NAN, NAN, NAN); }
template <typename T>
__device__ inline void window_store(T* row, float4 x, float mul, int col0, int end_col, int lane) {
    const int col = col0 + 4 * lane;
    if (col >= end_col) return;
    store1(row + col, mul * x.x);
    store1(row + col + 1, mul * x.y);
    store1(row + col + 2, mul * x.z);
    store1(row + col + 3, mul * x.w);
}
// the keys of row a in ranges: body(first, end), as long as it says so
template <typename Body>
__device__ inline void window_ranges(const WindowArgs& p, int a, Body body) {
    const int lo = window_start(p, a);
    bool on = true;
#pragma unroll 1
    for (int i = 0; i < 2 && on; ++i) on = body(i ? lo : 0, i ? a + 1 : min(p.sinks, lo));
}
// Every element of n rows is a number and finite.
template <typename T>
__device__ inline bool all_finite(const T* rows, int64_t ss, int n, int d, int lane) {
    static_assert(AHEAD<T> == 16, "four rows a load, 64 of them");
    float z = 0.f;
#pragma unroll 1
    for (int r0 = 0; r0 < n; r0 += 64)
#pragma unroll 1
        for (int col0 = 0; col0 < d; col0 += 64) {
            const int at = min(col0 + 4 * (lane & 15), d - 4);
            Four<T> y[AHEAD<T>];
#pragma unroll
            for (int i = 0; i < AHEAD<T>; ++i) y[i].load(rows + min(r0 + 4 * i + (lane >> 4), n - 1) * ss + at);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < AHEAD<T>; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) z = fmaf(y[i].at(e), 0.f, z);
        }
    return __builtin_amdgcn_ballot_w64(z != 0.f) == 0;
}
// bf16, a row whose scores are numbers (its row sum is one) and some of whose results are not: what the tiles of PAIR rows and keys have stored of it stands, but
// for columns that a value of a hidden key may have reached, one in the tile that the window begins in or in the row's own.  These are done over, up to where
// all of them are NaN.
template <int PAIR>
__device__ inline void window_fwd_row(const WindowArgs& p, int hd, int a) {
    typedef __hip_bfloat16 T;
    const int lane = lane_anew();
    const int64_t row = hd * p.stride_h + (int64_t)a * p.stride_s, kv_base = (hd / (p.H / p.H_kv)) * p.kv_stride_h;
    const int q0 = a / PAIR * PAIR, lo = max(window_start(p, q0) / PAIR * PAIR, p.sinks), hi = min(p.c, q0 + PAIR);
    const T* const V0 = (const T*)p.v + kv_base;
    if (all_finite<T>(V0 + lo * p.kv_stride_s, p.kv_stride_s, window_start(p, a) - lo, p.d, lane) &&
        all_finite<T>(V0 + (a + 1) * p.kv_stride_s, p.kv_stride_s, hi - a - 1, p.d, lane))
        return;
    const T* const q = (const T*)p.q + row;
    T* const O = (T*)p.o + row;
    const int col = window_col(0, p.d, lane);
    Four<T> tiles;
    tiles.load(O + col);
    float m = -INFINITY, l = 0.f;
    // (a column that stays is NaN here, and none to wait for)
    float4 acc = make_float4(fabsf(tiles.at(0)) < INFINITY ? NAN : 0.f, fabsf(tiles.at(1)) < INFINITY ? NAN : 0.f,
                             fabsf(tiles.at(2)) < INFINITY ? NAN : 0.f, fabsf(tiles.at(3)) < INFINITY ? NAN : 0.f);
    window_ranges(p, a, [&](int first, int end) {
#pragma unroll 1
        for (int k0 = first; k0 < end; k0 += 64) {
            const int n = min(64, end - k0);
            const float dot = window_dots<T>(q, (const T*)p.k + kv_base + (int64_t)k0 * p.kv_stride_s, p.kv_stride_s, n, p.d, lane);
            const float s = lane < n ? p.scale * dot : -INFINITY;
            const float m_new = fmaxf(m, wave_max(s)), ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = m == -INFINITY ? 0.f : expf(m - m_new);
            const float pr = lane < n ? expf(s - ref) : 0.f;
            l = l * alpha + wave_sum(pr);
            acc = make_float4(acc.x * alpha, acc.y * alpha, acc.z * alpha, acc.w * alpha);
            window_add<T>(acc, pr, V0 + (int64_t)k0 * p.kv_stride_s, p.kv_stride_s, n, col);
            if (lost(acc)) return false;
            m = m_new;
        }
        return true;
    });
    if (4 * lane >= p.d) return;
    const float inv = 1.f / l, got[4] = {acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (!(fabsf(tiles.at(e)) < INFINITY)) store1(O + col + e, got[e]);
}
// fp32 (terms of an infinite number are NaN: the tiles' results and row sum say nothing)
template <typename T>
__device__ inline void window_fwd_row(const WindowArgs& p, int hd, int a) {
    const int lane = lane_anew();
    const int64_t row = hd * p.stride_h + (int64_t)a * p.stride_s, kv_base = (hd / (p.H / p.H_kv)) * p.kv_stride_h;
    const T* q = (const T*)p.q + row;
    T* O = (T*)p.o + row;
    const int col = window_col(0, p.d, lane);
    float m = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    bool no_values = false;
    window_ranges(p, a, [&](int first, int end) {
#pragma unroll 1
        for (int k0 = first; k0 < end; k0 += 64) {
            const T* K = (const T*)p.k + kv_base + (int64_t)k0 * p.kv_stride_s;
            const T* V = (const T*)p.v + kv_base + (int64_t)k0 * p.kv_stride_s;
            const int n = min(64, end - k0);
            const bool valid = lane < n;
            const float dot = window_dots<T>(q, K, p.kv_stride_s, n, p.d, lane), s = valid ? p.scale * dot : -INFINITY;
            if (__builtin_amdgcn_ballot_w64(!(s < INFINITY))) {         // a NaN or +inf score: the row is no number
                l = NAN;
                return false;
            }
            const float m_new = fmaxf(m, wave_max(s)), ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = m == -INFINITY ? 0.f : expf(m - m_new);
            const float pr = valid ? expf(s - ref) : 0.f;
            l = l * alpha + wave_sum(pr);
            acc = make_float4(acc.x * alpha, acc.y * alpha, acc.z * alpha, acc.w * alpha);
            if (!no_values) window_add<T>(acc, pr, V, p.kv_stride_s, n, col);
            no_values = no_values || lost(acc);
            m = m_new;
        }
        return true;
    });
    window_store<T>(O, acc, 1.f / l, 0, p.d, lane);          // (every key it sees at -inf: no number)
    if (lane == 0) p.lse[hd * p.stat_stride_h + a] = l == 0.f ? NAN : m + logf(l);
}
template <typename T>
__device__ inline void window_dq_row(const WindowArgs& p, int hd, int a) {
    const int lane = lane_anew();
    const int64_t row = hd * p.stride_h + (int64_t)a * p.stride_s, kv_base = (hd / (p.H / p.H_kv)) * p.kv_stride_h;
    const T* q = (const T*)p.q + row;
    const T* g = (const T*)p.dout + row;
    const float lse = p.lse[hd * p.stat_stride_h + a], delta = p.delta[hd * p.stat_stride_h + a];
    const int col = window_col(0, p.d, lane);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    window_ranges(p, a, [&](int first, int end) {
#pragma unroll 1
        for (int k0 = first; k0 < end; k0 += 64) {
            const T* K = (const T*)p.k + kv_base + (int64_t)k0 * p.kv_stride_s;
            const T* V = (const T*)p.v + kv_base + (int64_t)k0 * p.kv_stride_s;
            const int n = min(64, end - k0);
            float ds = NAN;
            if (lse == lse && delta == delta) {
                const float x = window_dots<T>(q, K, p.kv_stride_s, n, p.d, lane), dp = window_dots<T>(g, V, p.kv_stride_s, n, p.d, lane);
                ds = lane < n ? expf(p.scale * x - lse) * (dp - delta) : 0.f;
            }
            if (__builtin_amdgcn_ballot_w64(ds != ds)) {                // in every column
                acc = no_numbers();
                return false;
            }
            window_add<T>(acc, ds, K, p.kv_stride_s, n, col);
            if (lost(acc)) return false;
        }
        return true;
    });
    window_store<T>((T*)p.dq + row, acc, p.scale, 0, p.d, lane);
}
// columns col0 .. end_col - 1 of dK and dV, of all rows that see the key; both: not dK alone, where dV's sums are numbers
template <typename T>
__device__ inline void window_dkdv_row(const WindowArgs& p, int kvh, int key, int col0, int end_col, bool both = true) {
    const int lane = lane_anew();
    const int group = p.H / p.H_kv, end = key < p.sinks ? p.c : min(p.c, key + p.window);
    const int64_t row = kvh * p.kv_stride_h + (int64_t)key * p.kv_stride_s;
    // A row without a number for its LSE leaves none in dV and dK, one without delta none in dK: looked for first, in less than a hundredth of the time.
    bool no_lse = false, no_delta = false;
#pragma unroll 1
    for (int hd = kvh * group; hd < (kvh + 1) * group; ++hd)
#pragma unroll 4
        for (int a = key + lane; a < end; a += 64) {
            const float l = p.lse[hd * p.stat_stride_h + a], e = p.delta[hd * p.stat_stride_h + a];
            no_lse = no_lse || l != l;
            no_delta = no_delta || e != e;
        }
    bool no_v = __builtin_amdgcn_ballot_w64(no_lse) != 0, no_k = no_v || __builtin_amdgcn_ballot_w64(no_delta) != 0;
    no_v = no_v || !both;
    const int col = window_col(col0, end_col, lane);
    float4 acck = make_float4(0.f, 0.f, 0.f, 0.f), accv = acck;
    if (no_k) acck = no_numbers();
    if (no_v) accv = no_numbers();
#pragma unroll 1
    for (int hd = kvh * group; hd < (kvh + 1) * group; ++hd) {
        const float* lse = p.lse + hd * p.stat_stride_h;
        const float* delta = p.delta + hd * p.stat_stride_h;
#pragma unroll 1
        for (int a0 = key; a0 < end && !(no_v && no_k); a0 += 64) {
            const T* Q = (const T*)p.q + hd * p.stride_h + (int64_t)a0 * p.stride_s;
            const T* G = (const T*)p.dout + hd * p.stride_h + (int64_t)a0 * p.stride_s;
            const int n = min(64, end - a0), a = a0 + min(lane, n - 1);
            const float x = window_dots<T>((const T*)p.k + row, Q, p.stride_s, n, p.d, lane), pr = expf(p.scale * x - lse[a]);
            if (!no_v) window_add<T>(accv, pr, G, p.stride_s, n, col);
            if (!no_k) {
                const float dp = window_dots<T>((const T*)p.v + row, G, p.stride_s, n, p.d, lane);
                window_add<T>(acck, pr * (dp - delta[a]), Q, p.stride_s, n, col);
            }
            no_v = no_v || lost(accv);
            no_k = no_k || lost(acck);
        }
    }
    if (both) window_store<T>((T*)p.dv + row, accv, 1.f, col0, end_col, lane);
    window_store<T>((T*)p.dk + row, acck, p.scale, col0, end_col, lane);
}
// The rows set in a mask, as each_row has them: the launch's arguments are read and its sequence looked up anew, so that nothing of either has to be
// kept until here.  first_row: of the wavefront within its workgroup's tile.  row(arguments, head, row of the sequence, its bit).
template <bool SNAKE, int TILE, typename Row>
__device__ inline void each_window_row(uint32_t rows, int linear, int n_heads, int first_row, Row row) {
    if (rows == 0) return;
    WindowArgs p = static_cast<const WindowArgs&>(launch_args());
    int n_tiles, rank, head;
    if (!enter_sequence<SNAKE, TILE>(p, linear, n_heads, n_tiles, rank, head)) return;
    first_row += TILE * (SNAKE ? n_tiles - 1 - rank : rank);        // (query tiles: the heaviest, the first in order, is the last)
#pragma unroll 1
    for (; rows != 0; rows &= rows - 1) row(p, head, first_row + __builtin_ctz(rows), (int)__builtin_ctz(rows));
}
// of a launch with both kinds of workgroups those that own keys, which come first
__device__ inline int key_workgroups() {
    const WindowArgs& launched = static_cast<const WindowArgs&>(launch_args());
    return launched.n_ranks * launched.H_kv;
}

}  // namespace sa
