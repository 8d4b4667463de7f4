// Moving what a paged cache holds: pages, or their first tokens, onto other pages; the accepted tokens of drafts up behind the tokens in front of them.
//
// Bound by memory: each byte is read and written once.  Rows are moved in units of 16 bytes where all rows begin at multiples of that, otherwise of 8
// (a row is a multiple of four elements).  2048 pages of 64 tokens, 8 heads of 128 columns, bf16: 215 us, 5.0 TB/s of reads and writes; a part of 64 pages: 4.4 us,
// the launch.
#include <algorithm>

#include "paged.h"

namespace sa {

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <int BYTES> struct UnitOf { typedef u32x4 Type; };
template <> struct UnitOf<8> { typedef u32x2 Type; };

constexpr int THREADS = 256, EACH = 4;          // copy: units a thread requests at a time

// sizes and strides in units
struct Units { int row; int64_t page, slot, head; };
template <int BYTES, typename Args>
Units units_of(const Args& a, int es) {
    return {a.d * es / BYTES, a.stride_page * es / BYTES, a.stride_slot * es / BYTES, a.stride_head * es / BYTES};
}
template <typename Args>
bool in_16_bytes(const Args& a, int es) {
    return a.d * es % 16 == 0 && a.stride_page * es % 16 == 0 && a.stride_slot * es % 16 == 0 && a.stride_head * es % 16 == 0;
}

// A workgroup: EACH * THREADS units of a page's keys or values.  A unit's number counts along memory: `inner` units one after the other, then slots or
// heads (heads_apart: slots first), then the others.
template <int BYTES>
__global__ void __launch_bounds__(THREADS)
cache_copy_kernel(CopyArgs p, Units s, bool heads_apart) {
    typedef typename UnitOf<BYTES>::Type Unit;
    const int i = (int)blockIdx.x;
    const int from = p.from[i], to = p.to[i], tokens = p.tokens ? min(max(p.tokens[i], 0), p.page_size) : p.page_size;
    if (from < 0 || from >= p.n_pages || to < 0 || to >= p.n_pages || from == to) return;
    Unit* const cache = (Unit*)(blockIdx.z ? p.v_cache : p.k_cache);
    const Unit* const src = cache + from * s.page;
    Unit* const dst = cache + to * s.page;
    // rows that lie one behind the other are one run
    const uint32_t runs_inner = heads_apart ? tokens : p.H_kv, outer = heads_apart ? p.H_kv : tokens;
    const int64_t stride_inner = heads_apart ? s.slot : s.head, stride_outer = heads_apart ? s.head : s.slot;
    uint32_t run = s.row, inner = runs_inner, n_outer = outer;
    if (stride_inner == run) {
        run *= inner;
        inner = 1;
        if (stride_outer == run) {
            run *= n_outer;
            n_outer = 1;
        }
    }
    const uint32_t all = run * inner * n_outer;
    for (uint32_t u0 = blockIdx.y * EACH * THREADS; u0 < all; u0 += gridDim.y * EACH * THREADS) {
        Unit x[EACH];
        int64_t at[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            uint32_t u = u0 + e * THREADS + threadIdx.x;
            at[e] = -1;
            if (u >= all) continue;
            if (inner * n_outer == 1) at[e] = u;
            else {
                const uint32_t r = u / run, o = r / inner;
                at[e] = (int64_t)o * stride_outer + (int64_t)(r - o * inner) * stride_inner + (u - r * run);
            }
            x[e] = src[at[e]];
        }
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            if (at[e] >= 0) dst[at[e]] = x[e];
    }
}

// A workgroup: a sequence.  Its first lanes look up where the accepted tokens lie, a token each (one after the other in every thread: 7.7 us, not
// 4.6, for 64 sequences, drafts of up to 32, 8 heads of 128 columns, bf16; bound by latency: a launch and four loads that depend on each other).  Then
// its threads take units of the tokens' keys and values, and each moves its unit of BATCH tokens at a time: as the tokens chosen ascend, none of a later
// batch has been written yet.
constexpr int BATCH = 8, MOST_DRAFTED = 64;
template <int BYTES>
__global__ void __launch_bounds__(1024)
cache_accept_kernel(AcceptArgs p, Units s) {
    typedef typename UnitOf<BYTES>::Type Unit;
    __shared__ int64_t from[MOST_DRAFTED], to[MOST_DRAFTED];            // units from a cache's first, to: -1 where nothing is moved
    const int b = (int)blockIdx.x, room = p.max_pages * p.page_size, tid = (int)threadIdx.x;
    const int length = p.lens[b], taken = p.accepted[b], which = tid < p.T ? p.chosen[b * p.chosen_stride + tid] : -1;
    const int lens = max(length, 0), n = min(max(taken, 0), p.T);
    if (tid < n) {
        const int32_t* table = p.table + b * p.table_stride;
        int64_t at[2] = {-1, -1};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t token = (int64_t)lens + (i ? tid : which);
            if (which < 0 || which >= p.T || which == tid || token >= room) continue;
            const int page = (int)token / p.page_size, id = table[page];
            if (id >= 0 && id < p.n_pages) at[i] = id * s.page + ((int)token - page * p.page_size) * s.slot;
        }
        from[tid] = at[0];
        to[tid] = at[0] < 0 ? -1 : at[1];
    }
    __syncthreads();            // (and all have read the length before it may be written)
    if (p.lens_after && tid == 0) p.lens_after[b] = lens + n;
    const int per_cache = p.H_kv * s.row;
    for (int u = tid; u < 2 * per_cache; u += blockDim.x) {
        Unit* const cache = (Unit*)(u < per_cache ? p.k_cache : p.v_cache);
        const int in = u < per_cache ? u : u - per_cache, head = in / s.row;
        Unit* const column = cache + head * s.head + (in - head * s.row);
        for (int i0 = 0; i0 < n; i0 += BATCH) {
            Unit x[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (i0 + i < n && to[i0 + i] >= 0) x[i] = column[from[i0 + i]];
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (i0 + i < n && to[i0 + i] >= 0) column[to[i0 + i]] = x[i];
        }
    }
}

template <int BYTES>
hipError_t copy(const CopyArgs& a, int es, hipStream_t st) {
    const Units s = units_of<BYTES>(a, es);
    const bool heads_apart = a.stride_head >= a.page_size * a.stride_slot;
    const int64_t most = (int64_t)a.page_size * a.H_kv * s.row, slices = (most + EACH * THREADS - 1) / (EACH * THREADS);
    // (a launch holds fewer than 2^32 threads, and fewer than 2^16 workgroups along y; n: up to 2^22)
    const int64_t most_slices = std::min((1 << 22) / a.n, 65535);
    const unsigned y = (unsigned)(slices < most_slices ? slices : most_slices);
    hipLaunchKernelGGL(cache_copy_kernel<BYTES>, dim3((unsigned)a.n, y, 2), dim3(THREADS), 0, st, a, s, heads_apart);
    return hipGetLastError();
}
template <int BYTES>
hipError_t accept(const AcceptArgs& a, int es, hipStream_t st) {
    const Units s = units_of<BYTES>(a, es);
    const int64_t all = 2ll * a.H_kv * s.row;
    const unsigned threads = all >= 1024 ? 1024 : (unsigned)((all + 63) / 64 * 64);
    // (a launch holds fewer than 2^32 threads: of 2^22 sequences of 1024 the last one goes in a launch of its own)
    const int most = (int)(((int64_t(1) << 32) - 1) / threads);
    for (int64_t first = 0; first < a.B; first += most) {
        AcceptArgs p = a;
        p.B = (int)std::min<int64_t>(a.B - first, most);
        if (a.table) p.table = a.table + first * a.table_stride;
        p.lens = a.lens + first;
        p.chosen = a.chosen + first * a.chosen_stride;
        p.accepted = a.accepted + first;
        if (a.lens_after) p.lens_after = a.lens_after + first;
        hipLaunchKernelGGL(cache_accept_kernel<BYTES>, dim3((unsigned)p.B), dim3(threads), 0, st, p, s);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_cache_copy(const CopyArgs& a, int dtype, hipStream_t st) {
    const int es = dtype == SA_F32 ? 4 : 2;
    return in_16_bytes(a, es) ? copy<16>(a, es, st) : copy<8>(a, es, st);
}
hipError_t launch_cache_accept(const AcceptArgs& a, int dtype, hipStream_t st) {
    const int es = dtype == SA_F32 ? 4 : 2;
    return in_16_bytes(a, es) ? accept<16>(a, es, st) : accept<8>(a, es, st);
}

}  // namespace sa
