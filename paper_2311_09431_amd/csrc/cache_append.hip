// New keys and values into the slots of a paged cache, keys rotated on the way; the queries of the same rows rotated beside.
//
// A row's angles pos base^(-2i/d) are formed in revolutions in double precision (position ids reach 10^6, where fp32 is off by
// 0.05 rad), reduced to [-1/2, 1/2] there, and only the fraction is rounded to fp32: an angle is off by 2^-24 of half a turn at
// most.  A workgroup forms the sines and cosines of its rows once, in LDS, for all heads, then its threads take chunks of
// columns: a rotated one and its partner d/2 further on, 16 bytes each, or a piece of V.
//
// Bound by memory: (H + 2 H_kv) d elements a row are read and written (and H_kv d more written where rotated keys are kept).  16384 rows,
// 32 heads on 8, d 128, bf16: 436 MB in 79 us, 5.5 TB/s (a copy reaches 4.9).  d = 100, whose halves are no whole 16-byte chunks, goes by
// 8 bytes (bf16 4): 4.0 TB/s.
#include <hip/hip_bf16.h>

#include "paged.h"

namespace sa {

namespace {

constexpr int THREADS = 256, MOST_ROWS = 8, MOST_WORKGROUPS = (1 << 24) - 1;

// N elements, widened and back (one rounding)
template <typename T, int N> struct Chunk;
template <int N> struct Chunk<float, N> {
    typedef float Raw __attribute__((ext_vector_type(N)));
    Raw x;
    __device__ void load(const float* p) { x = *reinterpret_cast<const Raw*>(p); }
    __device__ void store(float* p) const { *reinterpret_cast<Raw*>(p) = x; }
    __device__ float at(int i) const { return x[i]; }
    __device__ void set(int i, float v) { x[i] = v; }
};
template <int N> struct Chunk<__hip_bfloat16, N> {
    typedef __bf16 Raw __attribute__((ext_vector_type(N)));
    Raw x;
    __device__ void load(const __hip_bfloat16* p) { x = *reinterpret_cast<const Raw*>(p); }
    __device__ void store(__hip_bfloat16* p) const { *reinterpret_cast<Raw*>(p) = x; }
    __device__ float at(int i) const { return (float)x[i]; }
    __device__ void set(int i, float v) { x[i] = (__bf16)v; }
};

// N: elements a chunk
template <typename T, int N>
__global__ void __launch_bounds__(THREADS)
cache_append_kernel(AppendArgs p) {
    __shared__ float2 turn[MOST_ROWS][128];         // cosine, sine of pair i
    const int half = p.d / 2, row0 = (int)blockIdx.x * p.wg_rows, rows = min(p.wg_rows, p.rows - row0);
    if (p.pos) {
        for (int x = threadIdx.x; x < rows * half; x += THREADS) {
            const int r = x / half, i = x - r * half;
            const double t = (double)p.pos[row0 + r] * (exp2(-2.0 * i / p.d * p.log2_base) * 0.15915494309189535);
            float s, c;
            sincospif(2.f * (float)(t - rint(t)), &s, &c);
            turn[r][i] = make_float2(c, s);
        }
        __syncthreads();
    }
    const int pairs = half / N;                     // chunk pairs of a head
    const int nq = p.q ? p.H * pairs : 0, nk = p.H_kv * pairs, per_row = nq + 2 * nk;
    for (int x = threadIdx.x; x < rows * per_row; x += THREADS) {
        const int r = x / per_row;
        int y = x - r * per_row;
        const int64_t row = row0 + r;
        const T* from;
        T *to = nullptr, *cache = nullptr;
        const bool is_q = y < nq, is_v = y >= nq + nk;
        y -= is_q ? 0 : is_v ? nq + nk : nq;
        const int head = y / pairs, i = (y - head * pairs) * N;
        if (is_q) {
            const int64_t at = row * p.stride_s + head * p.stride_h + i;
            from = (const T*)p.q + at;
            to = (T*)p.q_out + at;
        } else {
            const int64_t at = row * p.kv_stride_s + head * p.kv_stride_h + i;
            from = (const T*)(is_v ? p.v : p.k) + at;
            if (!is_v && p.k_out) to = (T*)p.k_out + at;
            const int64_t slot = p.slot[row];
            if (slot >= 0 && slot < p.n_slots) {
                const int page = (int)slot / p.page_size, in_page = (int)slot - page * p.page_size;
                cache = (T*)(is_v ? p.v_cache : p.k_cache) + page * p.stride_page + in_page * p.stride_slot + head * p.stride_head + i;
            }
        }
        Chunk<T, N> lo, hi;
        lo.load(from);
        hi.load(from + half);
        if (p.pos && !is_v) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float2 cs = turn[r][i + e];
                const float a = lo.at(e), b = hi.at(e);
                lo.set(e, a * cs.x - b * cs.y);
                hi.set(e, b * cs.x + a * cs.y);
            }
        }
        if (to) {
            lo.store(to);
            hi.store(to + half);
        }
        if (cache) {
            lo.store(cache);
            hi.store(cache + half);
        }
    }
}

// As many rows a workgroup as its threads have chunks for, mostly one: what a workgroup does one after the other is what takes time, us, 1,
// 2, 4, 8 rows: 7 sequences of up to 701, 32 heads, d 100, fp32, 57, 56, 81, 120, 8 of up to 1000, 32 on 8, bf16, 19, 19, 25, 37, d 128
// 4 of up to 4096 38, 39, 42, 43; d 32, 16 heads (96 chunks a row) 13.5, 13.2, 13.1, 13.2.
template <typename T, int N>
hipError_t launch(AppendArgs a, hipStream_t st) {
    const int per_row = ((a.q ? a.H : 0) + 2 * a.H_kv) * (a.d / 2 / N);
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
        hipLaunchKernelGGL((cache_append_kernel<T, N>), dim3((unsigned)((p.rows + (int64_t)a.wg_rows - 1) / a.wg_rows)), dim3(THREADS), 0, st, p);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

// whole 16-byte chunks everywhere
bool whole_chunks(const AppendArgs& a, int n) {
    return (a.d / 2) % n == 0 && ((a.stride_h | a.stride_s | a.kv_stride_h | a.kv_stride_s | a.stride_page | a.stride_slot | a.stride_head) % n) == 0;
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, int dtype, hipStream_t st) {
    if (dtype == SA_F32) return whole_chunks(a, 4) ? launch<float, 4>(a, st) : launch<float, 2>(a, st);
    return whole_chunks(a, 8) ? launch<__hip_bfloat16, 8>(a, st) : launch<__hip_bfloat16, 2>(a, st);
}

}  // namespace sa
