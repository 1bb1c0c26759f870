// Gradients of the gated block's two projections from that of its result h = act(g) * u:
//     dg = dh * u * act'(g),   du = dh * act(g)
// with s = 1 / (1 + exp(-g)) for SiLU: act = g s, act' = s (1 + g (1 - s)).  In fp32 the quotients are those of the forward pass, to the bit; in 16 bits a
// reciprocal off by 1 ulp, far below the rounding.
//
// dg and du are rounded once to the operands' type, in which the products behind read them: the 2-norm of the gradients' error is sqrt 2 times that of
// unrounded ones (bf16 2.34e-3 and 1.66e-3, fp16 2.9e-4 and 2.1e-4, of which the gradients' own rounding is the smaller figure).  Held in two parts of 16 bits each
// they would double the matrix products, 94 % of the time (8192 x 4096, 10944).  So in fp16 they have its range: below 2^-14 they have fewer bits, above
// 65504 they are infinite.
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
        // (products by 0 and a NaN kept, as the formula has it: what is not finite in dh, u or g stays visible)
        dg = dh * u * (g > 0.f ? 1.f : g <= 0.f ? 0.f : g);
        du = dh * (g < 0.f ? 0.f : g);
    } else if constexpr (sizeof(T) == 4) {
        const float s = 1.f / (1.f + __expf(-g));
        dg = dh * u * (s * (1.f + g * (1.f - s)));
        du = dh * silu_divided(g);
    } else {
        const float s = __builtin_amdgcn_rcpf(1.f + __expf(-g));
        dg = dh * u * (s * (1.f + g * (1.f - s)));
        du = dh * (g * s);
    }
}

// A lane takes 16 bytes of dg and du at a time; their rows are whole numbers of such pieces, with zeros past the row's end.  VEC: so are the
// rows of the inputs, without gaps.
template <typename T, int ACT, bool VEC>
__global__ __launch_bounds__(256) void gated_slopes_kernel(const T* __restrict__ dh, const T* __restrict__ gate, const T* __restrict__ up,
                                                           T* __restrict__ dg, T* __restrict__ du, int64_t pieces, int per_row, int F, int64_t ldh,
                                                           uint32_t* __restrict__ counters, int counts)
{
    constexpr int E = 16 / (int)sizeof(T);
    // VEC: one run of pieces; otherwise a row of workgroups for each row (or every gridDim.y-th), so that there is none to find
    const int64_t step = VEC ? (int64_t)gridDim.x * 256 : per_row * (int64_t)gridDim.y;
    const int at = (int)blockIdx.x * 256 + (int)threadIdx.x;
    if (blockIdx.y == 0)
        for (int i = at; i < counts; i += (int)gridDim.x * 256) counters[i] = 0;
    if (!VEC && at >= per_row) return;
    int64_t m = blockIdx.y;
    for (int64_t i = VEC ? at : m * per_row + at; i < pieces; i += step, m += gridDim.y) {
        T g[E], u[E], h[E], og[E], ou[E];
        if (VEC) {
            *(u32x4*)g = *(const u32x4*)(gate + i * E);
            *(u32x4*)u = *(const u32x4*)(up + i * E);
            *(u32x4*)h = *(const u32x4*)(dh + i * E);
        } else {
            const int f = at * E;
            const T *pg = gate + m * F + f, *pu = up + m * F + f, *ph = dh + m * ldh + f;
            if (f + E <= F) {  // (at whatever address)
                __builtin_memcpy(g, pg, 16);
                __builtin_memcpy(u, pu, 16);
                __builtin_memcpy(h, ph, 16);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) g[e] = u[e] = h[e] = T{};
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (f + e < F) g[e] = pg[e], u[e] = pu[e], h[e] = ph[e];
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            float a, b;
            slopes<T, ACT>(to_f32(g[e]), to_f32(u[e]), to_f32(h[e]), a, b);
            store_from_f32(og + e, a);
            store_from_f32(ou + e, b);
        }
        *(u32x4*)(dg + i * E) = *(u32x4*)og;
        *(u32x4*)(du + i * E) = *(u32x4*)ou;
    }
}

template <typename T>
rtoss_status launch(rtoss_act act, int64_t M, int F, const void* dh, int64_t ldh, const void* gate, const void* up, void* dg, void* du,
                    uint32_t* counters, int counts, hipStream_t s)
{
    constexpr int E = 16 / (int)sizeof(T);
    const bool vec = F % E == 0 && ldh == F && ((uintptr_t)dh | (uintptr_t)gate | (uintptr_t)up) % 16 == 0;
    const int per_row = (F + E - 1) / E;
    const int64_t pieces = M * per_row;
    const dim3 grid = vec ? dim3((unsigned)std::min<int64_t>((pieces + 255) / 256, 16384)) : dim3((per_row + 255) / 256, (unsigned)std::min<int64_t>(M, 16384));
    auto go = [&](auto kernel) {
        kernel<<<grid, 256, 0, s>>>((const T*)dh, (const T*)gate, (const T*)up, (T*)dg, (T*)du, pieces, per_row, F, ldh, counters, counts);
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
                                 void* dg, void* du, uint32_t* counters, int counts, hipStream_t s)
{
    switch (dt) {
    case RTOSS_F32: return launch<float>(act, M, F, dh, ldh, gate, up, dg, du, counters, counts, s);
    case RTOSS_F16: return launch<f16_t>(act, M, F, dh, ldh, gate, up, dg, du, counters, counts, s);
    default: return launch<bf16_t>(act, M, F, dh, ldh, gate, up, dg, du, counters, counts, s);
    }
}

}  // namespace rtoss
