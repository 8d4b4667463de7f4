// Gradient of causal attention over packed sequences, bf16: the ring step's workgroups (bwd_tiles.h; dK and dV at 65 to 128 columns: packed_bwd_ring.hip), each on one
// 128-row tile of one sequence (packed.h), and delta = rowsum(dO * O) before them.
#include "bwd_tiles.h"
#include "f32_rows.h"
#include "packed.h"

namespace sa {

namespace {

// 16 lanes a row and head, eight columns a lane and turn
template <typename T>
__global__ void __launch_bounds__(256)
packed_delta_kernel(const T* __restrict__ o, const T* __restrict__ dout, float* __restrict__ delta, int rows, int H, int d, int64_t sh,
                    int64_t ss, int64_t stat_sh) {
    const int l = threadIdx.x & 15;
    const int64_t n = (int64_t)rows * H;
    for (int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); i < n; i += (int64_t)gridDim.x * 16) {
        const int64_t row = i / H;
        const int h = (int)(i - row * H);
        const int64_t at = row * ss + h * sh;
        float acc = 0.f;
        for (int t = 8 * l; t < d; t += 128) {
            float4 x = ld4<T>(o + at + t), y = ld4<T>(dout + at + t);
            acc += x.x * y.x + x.y * y.y + x.z * y.z + x.w * y.w;
            if (t + 4 >= d) break;
            x = ld4<T>(o + at + t + 4);
            y = ld4<T>(dout + at + t + 4);
            acc += x.x * y.x + x.y * y.y + x.z * y.z + x.w * y.w;
        }
#pragma unroll
        for (int by = 8; by > 0; by >>= 1) acc += __shfl_xor(acc, by, 16);
        if (l == 0) delta[h * stat_sh + row] = acc;
    }
}

template <int DP, bool PART>
__global__ void __launch_bounds__(256, DP > 128 ? 1 : 2)
packed_dq_kernel(PackedArgs p) {
    __shared__ __attribute__((aligned(1024))) char lds0[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds1[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds2[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds3[tile_bytes(DP) * halves_of(DP)];
    int n_tiles, rank, head;
    if (!enter_sequence<true, BM>(p, (int)blockIdx.x, p.H, n_tiles, rank, head)) return;
    bwd_dq<true, WALK_TRI, DP, PART, false, true>(p, n_tiles, rank * p.H + head, lds0, lds1, lds2, lds3);
}

// up to 64 columns and above 128
template <int DP, bool PART>
__global__ void __launch_bounds__(256, DP > 64 ? 1 : 2)
packed_dkdv_kernel(PackedArgs p) {
    __shared__ __attribute__((aligned(1024))) char lds0[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds1[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds2[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(1024))) char lds3[tile_bytes(DP) * halves_of(DP)];
    __shared__ __attribute__((aligned(16))) float stat[KV_STAT_FLOATS];
    const int heads = p.H_kv * halves_of(DP);
    int n_tiles, rank, head;
    if (!enter_sequence<false, BM>(p, (int)blockIdx.x, heads, n_tiles, rank, head)) return;
    bwd_dkdv<WALK_RING, true, DP, PART, false, true>(p, n_tiles, rank * heads + head, lds0, lds1, lds2, lds3, stat);
}

template <int DP, bool PART>
hipError_t launch(PackedArgs p, hipStream_t st) {
    p.n_ranks = (int)most_tiles(p, BM);
    const int64_t n_dq = (int64_t)p.n_ranks * p.H, n_dkdv = (int64_t)p.n_ranks * p.H_kv * halves_of(DP);
    p.by_rank = by_rank(true, n_dq, MOST_BY_RANK<DP, false>);
    hipLaunchKernelGGL((packed_dq_kernel<DP, PART>), dim3((unsigned)n_dq), dim3(256), 0, st, p);
    if (hipError_t e = hipGetLastError()) return e;
    p.by_rank = by_rank(true, n_dkdv, MOST_BY_RANK<DP, false>);
    if constexpr (DP == 112 || DP == 128) return launch_packed_bwd_ring(p, st);
    else hipLaunchKernelGGL((packed_dkdv_kernel<DP, PART>), dim3((unsigned)n_dkdv), dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_delta(const PackedArgs& p, const void* out, int dtype, hipStream_t st) {
    int64_t g = ((int64_t)p.rows * p.H + 15) / 16;
    if (g > 16384) g = 16384;
    auto go = [&](auto* o) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(o)>>;
        hipLaunchKernelGGL(packed_delta_kernel<T>, dim3((unsigned)g), dim3(256), 0, st, o, (const T*)p.dout, const_cast<float*>(p.delta),
                           p.rows, p.H, p.d, p.stride_h, p.stride_s, p.stat_stride_h);
    };
    if (dtype == SA_F32) go((const float*)out);
    else go((const __hip_bfloat16*)out);
    return hipGetLastError();
}

hipError_t launch_packed_bwd(const PackedArgs& p, hipStream_t st) {
    const bool part = p.d % 8 != 0;
    if (p.d > 128) return part ? launch<256, true>(p, st) : launch<256, false>(p, st);
    if (p.d <= 32 && !part) return launch<32, false>(p, st);
    if (p.d <= 64) return part ? launch<64, true>(p, st) : launch<64, false>(p, st);
    if (p.d <= 112) return part ? launch<112, true>(p, st) : launch<112, false>(p, st);
    return part ? launch<128, true>(p, st) : launch<128, false>(p, st);
}

}  // namespace sa
