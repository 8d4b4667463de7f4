// delta = rowsum(dO * O) of packed rows, where no query-owning workgroups form it first.  Bound by memory, at these launches' sizes by the launch:
// 1602 rows of 16 heads, d 64, fp32, 13 MB in 5 us.
#include "f32_rows.h"
#include "packed.h"

namespace sa {

namespace {

// delta = rowsum(dO * O): 16 lanes a row and head, eight columns a lane and turn
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

template <typename T>
hipError_t launch(const PackedArgs& p, hipStream_t st) {
    const int64_t g = ((int64_t)p.rows * p.H + 15) / 16;
    hipLaunchKernelGGL(packed_delta_kernel<T>, dim3((unsigned)(g < 16384 ? g : 16384)), dim3(256), 0, st, (const T*)p.o, (const T*)p.dout,
                       const_cast<float*>(p.delta), p.rows, p.H, p.d, p.stride_h, p.stride_s, p.stat_stride_h);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_delta(const PackedArgs& p, int dtype, hipStream_t st) {
    return dtype == SA_F32 ? launch<float>(p, st) : launch<__hip_bfloat16>(p, st);
}

}  // namespace sa
