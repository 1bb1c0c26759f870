// Rows of fp32, fp16 or bf16 to signed 8-bit codes with one scale each:
//     top = max |x|,  scale = top / 127 (rounded to fp32),  code = nearest integer to x * 127 / top, ties to even
//
// The code is that of the exact quotient, so that it does not depend on the order of roundings.  In fp64: x * (127 / top) is off by less
// than 2^-45.  A quotient of two 24-bit numbers that is not itself halfway between two integers is at least 2^-25 * 2^-7 away from
// there, so rounding to a grid of 2^-36 first (adding and taking away 1.5 * 2^16) moves values that are halfway exactly back
// onto it and no other across it.
//
// Bound: memory, M * K * (element + 1) bytes.
#include <algorithm>

#include "products.h"

namespace rtoss {

namespace {

template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ x, int8_t* __restrict__ q, float* __restrict__ scale, int64_t M,
                                                            int K, int64_t ldx, int64_t ldq)
{
    __shared__ float tops[4];
    const int tid = threadIdx.x;
    for (int64_t m = blockIdx.x; m < M; m += gridDim.x) {
        const T* row = x + m * ldx;
        float top = 0.f;
        bool odd = false;  // a value that is not finite
        for (int k = tid; k < K; k += 256) {
            const float v = __builtin_fabsf(to_f32(row[k]));
            odd |= !(v < __builtin_inff());
            top = __builtin_fmaxf(top, v);
        }
        if (odd) top = __builtin_inff();
        for (int d = 32; d; d >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, d));
        __syncthreads();
        if ((tid & 63) == 0) tops[tid >> 6] = top;
        __syncthreads();
        top = __builtin_fmaxf(__builtin_fmaxf(tops[0], tops[1]), __builtin_fmaxf(tops[2], tops[3]));
        const bool finite = top < __builtin_inff();
        const double f = finite && top > 0.f ? 127.0 / (double)top : 0.0;
        if (tid == 0) scale[m] = finite ? top / 127.f : __builtin_nanf("");
        for (int k = tid; k < K; k += 256) {
            const double c = 98304.0, v = f == 0.0 ? 0.0 : (double)to_f32(row[k]) * f;
            q[m * ldq + k] = (int8_t)(int)__builtin_rint((v + c) - c);
        }
    }
}

}  // namespace

rtoss_status launch_quantize_rows(const void* x, rtoss_dtype dt, int64_t M, int K, int64_t ldx, int8_t* q, int64_t ldq, float* scale, hipStream_t s)
{
    const unsigned grid = (unsigned)std::min<int64_t>(M, 65536);
    switch (dt) {
    case RTOSS_F32: quantize_rows_kernel<float><<<grid, 256, 0, s>>>((const float*)x, q, scale, M, K, ldx, ldq); break;
    case RTOSS_F16: quantize_rows_kernel<f16_t><<<grid, 256, 0, s>>>((const f16_t*)x, q, scale, M, K, ldx, ldq); break;
    case RTOSS_BF16: quantize_rows_kernel<bf16_t><<<grid, 256, 0, s>>>((const bf16_t*)x, q, scale, M, K, ldx, ldq); break;
    }
    return check_hip(hipGetLastError(), "quantize_rows launch");
}

}  // namespace rtoss
