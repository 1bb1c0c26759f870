// Rows of fp32, fp16 or bf16 to signed 8-bit codes with one scale each:
//     top = max |x|,  scale = top / 127 (rounded to fp32),  code = nearest integer to x * 127 / top, ties to even
//
// The code is that of the exact quotient, so that it does not depend on the order of roundings.  In fp64: x * (127 / top) is off by less
// than 2^-45.  A quotient of two 24-bit numbers that is not itself halfway between two integers is at least 2^-25 * 2^-7 away from
// there, so rounding to a grid of 2^-36 first (adding and taking away 1.5 * 2^16) moves values that are halfway exactly back
// onto it and no other across it.
//
// Adding 1.5 * 2^52 then rounds to an integer, ties to even, whose low bits are the number's.
//
// A row is held in registers between the search for its largest value and the codes: LANES lanes, 16 bytes at a time, VPT times, at
// whatever address it starts.  Magnitudes are compared as bit patterns (infinities and NaN are the largest), two 16-bit ones at once.
// Bound: memory, M * K * (element + 1) bytes; one row: a chain of latencies.  Measured: bf16 1 x 4096 3.0 us, 8192 x 10944 54 us (4.9 TB/s), fp16 51200 x 256 7.8 us
#include <algorithm>

#include "products.h"

namespace rtoss {

namespace {

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

template <typename T> __device__ __forceinline__ uint32_t largest(uint32_t top, u32x4 v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) top = max(top, v[i] & 0x7fffffffu);
        else top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu)));
    }
    return top;
}
// the largest magnitude as a value, from the largest pattern of each half
template <typename T> __device__ __forceinline__ float top_value(uint32_t top)
{
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, top);
    else return to_f32(T{(uint16_t)max(top & 0xffffu, top >> 16)});
}

// 16 bytes of a row from element k on, zeros past its end
template <typename T> __device__ __forceinline__ u32x4 load_vector(const T* row, int k, int K)
{
    constexpr int E = 16 / (int)sizeof(T);
    u32x4 v = {0u, 0u, 0u, 0u};
    if (k + E <= K) {
        __builtin_memcpy(&v, row + k, 16);
    } else if (k < K) {
        T t[E] = {};
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (k + e < K) t[e] = row[k + e];
        __builtin_memcpy(&v, t, 16);
    }
    return v;
}

// f: 127 / top, or 0 for a row without codes
template <typename T> __device__ __forceinline__ void store_codes(int8_t* q, int k, int K, u32x4 v, double f)
{
    constexpr int E = 16 / (int)sizeof(T);
    uint32_t word[E / 4];
#pragma unroll
    for (int w = 0; w < E / 4; ++w) {
        uint32_t code[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int at = 4 * w + e;
            float x;
            if constexpr (sizeof(T) == 4) x = __builtin_bit_cast(float, (uint32_t)v[at]);
            else x = to_f32(T{(uint16_t)(v[at / 2] >> 16 * (at & 1))});
            const double c = 98304.0, magic = 6755399441055744.0;
            code[e] = (uint32_t)__builtin_bit_cast(uint64_t, (((double)x * f + c) - c) + magic);
        }
        const uint32_t lo = __builtin_amdgcn_perm(code[1], code[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(code[3], code[2], 0x04000c0cu);
        word[w] = f == 0.0 ? 0u : lo | hi;
    }
    if (k + E <= K) {
        __builtin_memcpy(q + k, word, E);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (k + e < K) q[k + e] = (int8_t)(word[e / 4] >> 8 * (e & 3));
    }
}

// VPT = 0: a row that is too long for the registers is read twice.
template <typename T, int LANES, int VPT>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void quantize_rows_kernel(const T* __restrict__ x, int8_t* __restrict__ q, float* __restrict__ scale,
                                                                                   int64_t M, int K, int64_t ldx, int64_t ldq)
{
    constexpr int E = 16 / (int)sizeof(T), BLOCK = LANES < 256 ? 256 : LANES, ROWS = BLOCK / LANES;
    __shared__ uint32_t tops[BLOCK / 64];
    const int at = threadIdx.x % LANES;
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < M; first += (int64_t)gridDim.x * ROWS) {
        const int64_t m = first + threadIdx.x / LANES;
        const int64_t row = m < M ? m : M - 1;         // (past the last: the last again, not stored)
        const T* from = x + row * ldx;
        u32x4 v[VPT ? VPT : 1];
        uint32_t top = 0;
        if constexpr (VPT > 0) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) v[i] = load_vector(from, (i * LANES + at) * E, K);
#pragma unroll
            for (int i = 0; i < VPT; ++i) top = largest<T>(top, v[i]);
        } else {
            for (int k = at * E; k < K; k += LANES * E) top = largest<T>(top, load_vector(from, k, K));
        }
        // the row's lanes: patterns of the two halves are kept apart until the end
#pragma unroll
        for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) {
            const uint32_t other = (uint32_t)__shfl_xor((int)top, d);
            if constexpr (sizeof(T) == 4) top = max(top, other);
            else top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, other)));
        }
        float t = top_value<T>(top);
        if constexpr (LANES > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) tops[threadIdx.x / 64] = __builtin_bit_cast(uint32_t, t);
            __syncthreads();
            uint32_t all = tops[0];
#pragma unroll
            for (int w = 1; w < BLOCK / 64; ++w) all = max(all, tops[w]);
            t = __builtin_bit_cast(float, all);
        }
        const bool finite = t < __builtin_inff();  // (false for NaN)
        const double f = finite && t > 0.f ? 127.0 / (double)t : 0.0;
        if (m >= M) continue;
        if (at == 0) scale[m] = finite ? t / 127.f : __builtin_nanf("");
        int8_t* to = q + m * ldq;
        if constexpr (VPT > 0) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if ((i * LANES + at) * E < K) store_codes<T>(to, (i * LANES + at) * E, K, v[i], f);
        } else {
            for (int k = at * E; k < K; k += LANES * E) store_codes<T>(to, k, K, load_vector(from, k, K), f);
        }
    }
}

template <typename T, int LANES, int VPT>
rtoss_status launch(const T* x, int64_t M, int K, int64_t ldx, int8_t* q, int64_t ldq, float* scale, hipStream_t s)
{
    constexpr int BLOCK = LANES < 256 ? 256 : LANES, ROWS = BLOCK / LANES;
    const unsigned grid = (unsigned)std::min<int64_t>((M + ROWS - 1) / ROWS, kMaxGridGroups / 4);
    quantize_rows_kernel<T, LANES, VPT><<<grid, BLOCK, 0, s>>>(x, q, scale, M, K, ldx, ldq);
    return check_hip(hipGetLastError(), "quantize_rows launch");
}

// The fewest lanes that hold a row in four vectors each.
template <typename T> rtoss_status launch_lanes(const void* x_, int64_t M, int K, int64_t ldx, int8_t* q, int64_t ldq, float* scale, hipStream_t s)
{
    const T* x = (const T*)x_;
    const int vectors = (int)(((int64_t)K * (int)sizeof(T) + 15) / 16);
    if (vectors <= 16) return launch<T, 16, 1>(x, M, K, ldx, q, ldq, scale, s);
#define RTOSS_LANES(LANES)                                                                     \
    if (vectors <= 2 * LANES) return launch<T, LANES, 2>(x, M, K, ldx, q, ldq, scale, s);      \
    if (vectors <= 4 * LANES) return launch<T, LANES, 4>(x, M, K, ldx, q, ldq, scale, s)
    RTOSS_LANES(16);
    RTOSS_LANES(64);
    RTOSS_LANES(256);
    RTOSS_LANES(1024);
#undef RTOSS_LANES
    return launch<T, 1024, 0>(x, M, K, ldx, q, ldq, scale, s);
}

}  // namespace

rtoss_status launch_quantize_rows(const void* x, rtoss_dtype dt, int64_t M, int K, int64_t ldx, int8_t* q, int64_t ldq, float* scale, hipStream_t s)
{
    switch (dt) {
    case RTOSS_F32: return launch_lanes<float>(x, M, K, ldx, q, ldq, scale, s);
    case RTOSS_F16: return launch_lanes<f16_t>(x, M, K, ldx, q, ldq, scale, s);
    case RTOSS_BF16: return launch_lanes<bf16_t>(x, M, K, ldx, q, ldq, scale, s);
    }
    return fail(RTOSS_EDTYPE, "bad dtype %d", (int)dt);
}

}  // namespace rtoss
