// Gradients of the gated block's two projections from that of its result h = act(g) * u:
//     dg = dh * u * act'(g),   du = dh * act(g)
// with s = 1 / (1 + exp(-g)) for SiLU: act = g s, act' = s (1 + g (1 - s)).  fp32; dg and du are rounded once to the operands' type, in
// which the products behind read them.  (A reciprocal is off by 1 ulp at most, far below that rounding; in fp32 it is one of three
// roundings of the product.)
//
// Bound: memory, five tensors of M * F elements.
#include <algorithm>

#include "products.h"

namespace rtoss {

namespace {

template <typename T, int ACT> __device__ __forceinline__ void slopes(float g, float u, float dh, float& dg, float& du)
{
    if constexpr (ACT == 0) {
        dg = dh * u;
        du = dh * g;
    } else if constexpr (ACT == 1) {
        dg = g > 0.f ? dh * u : 0.f;
        du = g > 0.f ? dh * g : 0.f;
    } else {
        const float s = __builtin_amdgcn_rcpf(1.f + __expf(-g));
        dg = dh * u * (s * (1.f + g * (1.f - s)));
        du = dh * (g * s);
    }
}

// VEC: 16 bytes a lane and step; `n` elements in one run (dh as wide as a row), all starts aligned to 16 bytes.
template <typename T, int ACT, bool VEC>
__global__ __launch_bounds__(256) void gated_slopes_kernel(const T* __restrict__ dh, const T* __restrict__ gate, const T* __restrict__ up,
                                                           T* __restrict__ dg, T* __restrict__ du, int64_t n, int F, int64_t ldh)
{
    constexpr int E = VEC ? 16 / (int)sizeof(T) : 1;
    const int64_t step = (int64_t)gridDim.x * 256 * E;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * E; i < n; i += step) {
        if (VEC && i + E <= n) {
            T g[E], u[E], h[E], og[E], ou[E];
            *(u32x4*)g = *(const u32x4*)(gate + i);
            *(u32x4*)u = *(const u32x4*)(up + i);
            *(u32x4*)h = *(const u32x4*)(dh + i);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float a, b;
                slopes<T, ACT>(to_f32(g[e]), to_f32(u[e]), to_f32(h[e]), a, b);
                store_from_f32(og + e, a);
                store_from_f32(ou + e, b);
            }
            *(u32x4*)(dg + i) = *(u32x4*)og;
            *(u32x4*)(du + i) = *(u32x4*)ou;
        } else {
            for (int64_t j = i; j < n && j < i + E; ++j) {
                float a, b;
                const int64_t at = VEC ? j : j / F * ldh + j % F;
                slopes<T, ACT>(to_f32(gate[j]), to_f32(up[j]), to_f32(dh[at]), a, b);
                store_from_f32(dg + j, a);
                store_from_f32(du + j, b);
            }
        }
    }
}

template <typename T>
rtoss_status launch(rtoss_act act, int64_t n, int F, const void* dh, int64_t ldh, const void* gate, const void* up, void* dg, void* du, hipStream_t s)
{
    const bool vec = ldh == F && ((uintptr_t)dh | (uintptr_t)gate | (uintptr_t)up | (uintptr_t)dg | (uintptr_t)du) % 16 == 0;
    const int64_t per = 256 * (vec ? 16 / (int)sizeof(T) : 1);
    const unsigned grid = (unsigned)std::min<int64_t>((n + per - 1) / per, 16384);
    auto go = [&](auto kernel) {
        kernel<<<grid, 256, 0, s>>>((const T*)dh, (const T*)gate, (const T*)up, (T*)dg, (T*)du, n, F, ldh);
        return check_hip(hipGetLastError(), "gated_slopes launch");
    };
    switch (act) {
    case RTOSS_ACT_NONE: return vec ? go(gated_slopes_kernel<T, 0, true>) : go(gated_slopes_kernel<T, 0, false>);
    case RTOSS_ACT_RELU: return vec ? go(gated_slopes_kernel<T, 1, true>) : go(gated_slopes_kernel<T, 1, false>);
    default: return vec ? go(gated_slopes_kernel<T, 2, true>) : go(gated_slopes_kernel<T, 2, false>);
    }
}

}  // namespace

rtoss_status launch_gated_slopes(rtoss_dtype dt, rtoss_act act, int64_t M, int F, const void* dh, int64_t ldh, const void* gate, const void* up,
                                 void* dg, void* du, hipStream_t s)
{
    const int64_t n = M * F;
    switch (dt) {
    case RTOSS_F32: return launch<float>(act, n, F, dh, ldh, gate, up, dg, du, s);
    case RTOSS_F16: return launch<f16_t>(act, n, F, dh, ldh, gate, up, dg, du, s);
    default: return launch<bf16_t>(act, n, F, dh, ldh, gate, up, dg, du, s);
    }
}

}  // namespace rtoss
