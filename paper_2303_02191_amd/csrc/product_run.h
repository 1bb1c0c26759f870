// Output stage of the tiled products: runs of neighbouring channels that a lane holds of a row.
#pragma once
#include "products.h"

namespace rtoss {

// N neighbouring values of a row, `left` of which exist; vec: the row's runs are aligned to 16 bytes.
template <typename TO, int N> __device__ __forceinline__ void store_run(TO* p, const float (&v)[N], int left, bool vec)
{
    static_assert(N % 8 == 0 || N == 4, "whole pieces of 16 bytes, or half of one");
    if (vec && left >= N) {
        constexpr int E = 16 / (int)sizeof(TO);
        if constexpr (N < E) *(uint2*)p = uint2{pack2_from_f32<TO>(v[0], v[1]), pack2_from_f32<TO>(v[2], v[3])};
#pragma unroll
        for (int i = 0; i < N / E; ++i) {
            if constexpr (sizeof(TO) == 4) *(f32x4*)(p + i * E) = f32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
            else *(u32x4*)(p + i * E) = pack8_from_f32<TO>(v + i * E);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < left) store_from_f32(p + i, v[i]);
}
template <typename TO, int N> __device__ __forceinline__ void add_run(const TO* p, float (&v)[N], int left, bool vec)
{
    static_assert(N % 8 == 0, "whole pieces of 16 bytes");
    if (vec && left >= N) {
        constexpr int E = 16 / (int)sizeof(TO);
#pragma unroll
        for (int i = 0; i < N / E; ++i) {
            TO t[E];
            *(u32x4*)t = *(const u32x4*)(p + i * E);
#pragma unroll
            for (int e = 0; e < E; ++e) v[i * E + e] += to_f32(t[e]);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < left) v[i] += to_f32(p[i]);
}

// The stage for channels n .. n+RUN-1 of any rows.
template <int FORM, typename T, typename TO, int RUN> struct RunOutput {
    static constexpr bool kScales = sizeof(T) == 1;
    typedef typename AccOf<T>::type Acc;
    float s0[kScales ? RUN : 1], s1[kScales && FORM == kGated ? RUN : 1], bias[FORM == kScaled ? RUN : 1];
    int n, left;
    bool vec, vec_kept, vec_residual;

    static __device__ __forceinline__ bool aligned(const void* p, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld * (int)sizeof(TO) % 16 == 0; }

    __device__ __forceinline__ RunOutput(const Product& p, int n_) : n(n_), left(p.N - n_)
    {
        vec = aligned(p.y, p.ldy);
        vec_kept = aligned(p.y0, p.N) && aligned(p.y1, p.N);
        vec_residual = aligned(p.residual, p.ldr);
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            const int at = n + (i < left ? i : 0);
            if constexpr (kScales) s0[i] = p.s0 ? p.s0[at] : 1.f;
            if constexpr (kScales && FORM == kGated) s1[i] = p.s1 ? p.s1[at] : 1.f;
            if constexpr (FORM == kScaled) bias[i] = p.bias ? p.bias[at] : 0.f;
        }
    }
    __device__ __forceinline__ void values(float (&v)[RUN], const Acc (&acc)[RUN / 4], const float* s, float sa) const
    {
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            v[i] = (float)acc[i / 4][i % 4];  // (whole numbers above 2^24 round here, to 24 bits as every fp32 value)
            if constexpr (kScales) v[i] = v[i] * sa * s[i];
        }
    }
    __device__ __forceinline__ void store(const Product& p, int64_t m, const Acc (&first)[RUN / 4], const Acc (&second)[RUN / 4]) const
    {
        store(p, m, kScales && p.sa ? p.sa[m] : 1.f, first, second);
    }
    __device__ __forceinline__ void store(const Product& p, int64_t m, float sa, const Acc (&first)[RUN / 4], const Acc (&second)[RUN / 4]) const
    {
        float v[RUN];
        values(v, first, s0, sa);
        if constexpr (FORM == kScaled) {
            if (p.bias)
#pragma unroll
                for (int i = 0; i < RUN; ++i) v[i] += bias[i];
            gate_act<RUN>(v, p.act);
            if (p.residual) add_run<TO, RUN>((const TO*)p.residual + m * p.ldr + n, v, left, vec_residual);
        } else if constexpr (FORM == kGated) {
            float u[RUN];
            values(u, second, s1, sa);
            if (p.y0) {
                store_run<TO, RUN>((TO*)p.y0 + m * p.N + n, v, left, vec_kept);
                store_run<TO, RUN>((TO*)p.y1 + m * p.N + n, u, left, vec_kept);
            }
            gate_act<RUN>(v, p.act);
#pragma unroll
            for (int i = 0; i < RUN; ++i) v[i] *= u[i];
        }
        store_run<TO, RUN>((TO*)p.y + m * p.ldy + n, v, left, vec);
    }
};

}  // namespace rtoss
