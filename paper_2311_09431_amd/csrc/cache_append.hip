// New keys and values into the slots of a paged cache, keys rotated on the way; the queries of the same rows rotated beside.
//
// A row's angles pos base^(-2i/d) are formed in revolutions in double precision (position ids reach 10^6, where fp32 is off by
// 0.05 rad), reduced to [-1/2, 1/2] there, and only the fraction is rounded to fp32: an angle is off by 2^-24 of half a turn at
// most.  A workgroup forms the sines and cosines of its rows once, in LDS, for all heads, then its threads take chunks of
// columns: a rotated one and its partner d/2 further on, 16 bytes each, or a piece of V.
//
// Bound by memory: (H + 2 H_kv) d elements a row are read and written (and H_kv d more written where rotated keys are kept).  16384 rows,
// 32 heads on 8, d 128, bf16, keys kept: 436 MB in 79 us, 5.5 TB/s (a copy reaches 4.9).  d = 100, whose halves are no whole 16-byte chunks and lie
// across lines: 9265 rows of 32 heads on 8, bf16, 178 MB in 44 us, 4.0 TB/s (in pieces of 4 bytes throughout 54, 3.3), 2468 rows of 32 heads, fp32, keys
// kept, 221 MB in 54 to 60, 3.7 to 4.1.  Requesting two to four pairs of chunks at a time changes nothing.
#include <hip/hip_bf16.h>

#include "paged.h"

namespace sa {

namespace {

constexpr int THREADS = 256, MOST_ROWS = 8, MOST_WORKGROUPS = (1 << 24) - 1;

// 16 bytes of a row, or the two-element pieces at the end of a half that is no whole number of them.  (Rows begin at multiples of four elements,
// halves of two.)
template <typename T> struct Element;
template <> struct Element<float> { typedef float Raw; };
template <> struct Element<__hip_bfloat16> { typedef __bf16 Raw; };
template <typename T> constexpr int N = 16 / (int)sizeof(T);
template <typename T, bool PART>
struct Chunk {
    typedef typename Element<T>::Raw Raw;
    typedef Raw Whole __attribute__((ext_vector_type(N<T>), aligned(2 * sizeof(T))));
    typedef Raw Pair __attribute__((ext_vector_type(2)));
    Whole x;
    __device__ void load(const T* p, int n) {
        if (!PART || n >= N<T>) x = *reinterpret_cast<const Whole*>(p);
        else {
#pragma unroll
            for (int i = 0; i < N<T> - 2; i += 2)
                if (i < n) {
                    const Pair y = *reinterpret_cast<const Pair*>(p + i);
                    x[i] = y[0];
                    x[i + 1] = y[1];
                }
        }
    }
    __device__ void store(T* p, int n) const {
        if (!PART || n >= N<T>) *reinterpret_cast<Whole*>(p) = x;
        else {
#pragma unroll
            for (int i = 0; i < N<T> - 2; i += 2)
                if (i < n) *reinterpret_cast<Pair*>(p + i) = Pair{x[i], x[i + 1]};
        }
    }
};

// PART: halves are no whole chunks
template <typename T, bool PART>
__global__ void __launch_bounds__(THREADS)
cache_append_kernel(AppendArgs p) {
    __shared__ float2 turn[MOST_ROWS][128];         // cosine, sine of pair i
    const int half = p.d / 2, row0 = (int)blockIdx.x * p.wg_rows, rows = min(p.wg_rows, p.rows - row0);
    const int pairs = (half + N<T> - 1) / N<T>;     // chunk pairs of a head
    const int nq = p.q ? p.H * pairs : 0, nk = p.H_kv * pairs, per_row = nq + 2 * nk, all = rows * per_row;
    struct Item {
        Chunk<T, PART> lo, hi;
        T *to, *cache;
        const float2* turn;                         // NULL: not rotated
        int n;
    };
    Item a;
    auto request = [&](int x) {
        const int r = x / per_row;
        int y = x - r * per_row;
        const int64_t row = row0 + r;
        const T* from;
        a.to = a.cache = nullptr;
        const bool is_q = y < nq, is_v = y >= nq + nk;
        y -= is_q ? 0 : is_v ? nq + nk : nq;
        const int head = y / pairs, i = (y - head * pairs) * N<T>;
        a.n = half - i;
        a.turn = p.pos && !is_v ? &turn[r][i] : nullptr;
        if (is_q) {
            const int64_t at = row * p.stride_s + head * p.stride_h + i;
            from = (const T*)p.q + at;
            a.to = (T*)p.q_out + at;
        } else {
            const int64_t at = row * p.kv_stride_s + head * p.kv_stride_h + i;
            from = (const T*)(is_v ? p.v : p.k) + at;
            if (!is_v && p.k_out) a.to = (T*)p.k_out + at;
            const int64_t slot = p.slot[row];
            if (slot >= 0 && slot < p.n_slots) {
                const int page = (int)slot / p.page_size, in_page = (int)slot - page * p.page_size;
                a.cache = (T*)(is_v ? p.v_cache : p.k_cache) + page * p.stride_page + in_page * p.stride_slot + head * p.stride_head + i;
            }
        }
        a.lo.load(from, a.n);
        a.hi.load(from + half, a.n);
    };
    auto finish = [&]() {
        if (a.turn) {
#pragma unroll
            for (int e = 0; e < N<T>; ++e) {
                const float2 cs = a.turn[e];        // (behind the half: anything)
                const float lo = (float)a.lo.x[e], hi = (float)a.hi.x[e];
                a.lo.x[e] = (typename Element<T>::Raw)(lo * cs.x - hi * cs.y);
                a.hi.x[e] = (typename Element<T>::Raw)(hi * cs.x + lo * cs.y);
            }
        }
        if (a.to) {
            a.lo.store(a.to, a.n);
            a.hi.store(a.to + half, a.n);
        }
        if (a.cache) {
            a.lo.store(a.cache, a.n);
            a.hi.store(a.cache + half, a.n);
        }
    };
    // (the first ones are on their way while the angles are formed)
    int x = threadIdx.x;
    if (x < all) request(x);
    if (p.pos) {
        for (int y = threadIdx.x; y < rows * half; y += THREADS) {
            const int r = y / half, i = y - r * half;
            const double t = (double)p.pos[row0 + r] * (exp2(-2.0 * i / p.d * p.log2_base) * 0.15915494309189535);
            float s, c;
            sincospif(2.f * (float)(t - rint(t)), &s, &c);
            turn[r][i] = make_float2(c, s);
        }
        __syncthreads();
    }
    while (x < all) {
        finish();
        x += THREADS;
        if (x < all) request(x);
    }
}

// As many rows a workgroup as its threads have chunks for, mostly one: what a workgroup does one after the other is what takes time, us, 1,
// 2, 4, 8 rows: 7 sequences of up to 701, 32 heads, d 100, fp32, 57, 56, 81, 120, 8 of up to 1000, 32 on 8, bf16, 19, 19, 25, 37, d 128
// 4 of up to 4096 38, 39, 42, 43; d 32, 16 heads (96 chunks a row) 13.5, 13.2, 13.1, 13.2.
template <typename T, bool PART>
hipError_t launch(AppendArgs a, hipStream_t st) {
    const int per_row = ((a.q ? a.H : 0) + 2 * a.H_kv) * ((a.d / 2 + N<T> - 1) / N<T>);
    a.wg_rows = THREADS / per_row < 1 ? 1 : THREADS / per_row > MOST_ROWS ? MOST_ROWS : THREADS / per_row;
    // (a launch holds fewer than 2^32 threads: more rows go in several)
    const int64_t all = a.rows, most = (int64_t)MOST_WORKGROUPS * a.wg_rows;
    for (int64_t first = 0; first < all; first += most) {
        AppendArgs p = a;
        p.rows = (int)(all - first < most ? all - first : most);
        p.k = (const T*)a.k + first * a.kv_stride_s;
        p.v = (const T*)a.v + first * a.kv_stride_s;
        if (a.k_out) p.k_out = (T*)a.k_out + first * a.kv_stride_s;
        if (a.q) {
            p.q = (const T*)a.q + first * a.stride_s;
            p.q_out = (T*)a.q_out + first * a.stride_s;
        }
        if (a.pos) p.pos = a.pos + first;
        p.slot = a.slot + first;
        hipLaunchKernelGGL((cache_append_kernel<T, PART>), dim3((unsigned)((p.rows + (int64_t)a.wg_rows - 1) / a.wg_rows)), dim3(THREADS), 0, st, p);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, int dtype, hipStream_t st) {
    if (dtype == SA_F32) return a.d / 2 % N<float> ? launch<float, true>(a, st) : launch<float, false>(a, st);
    return a.d / 2 % N<__hip_bfloat16> ? launch<__hip_bfloat16, true>(a, st) : launch<__hip_bfloat16, false>(a, st);
}

}  // namespace sa
