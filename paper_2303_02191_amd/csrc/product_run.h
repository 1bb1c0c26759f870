// Output stage of the tiled products: runs of neighbouring channels that a lane holds of a row.
#pragma once
#include "products.h"

namespace rtoss {

// How runs of a row can be stored and loaded: in pieces of 16 bytes (of 8, a run of 8), in words, or (16-bit types) with an element alone in
// front and behind where the row starts between two words.
enum Runs { kRunPieces = 0, kRunWords, kRunElements };
template <typename TO> __device__ __forceinline__ Runs runs_of(const void* p, int64_t ld)
{
    const uintptr_t at = (uintptr_t)p | (uintptr_t)(ld * (int)sizeof(TO));
    return at % 16 == 0 ? kRunPieces : at % 4 == 0 ? kRunWords : kRunElements;
}

// `words` words at p, a multiple of 4
template <int WORDS> __device__ __forceinline__ void store_words(void* p, const uint32_t* w)
{
#pragma unroll
    for (int i = 0; i + 4 <= WORDS; i += 4) __builtin_memcpy(__builtin_assume_aligned((char*)p + 4 * i, 4), w + i, 16);
    if constexpr (WORDS & 2) __builtin_memcpy(__builtin_assume_aligned((char*)p + 4 * (WORDS & ~3), 4), w + (WORDS & ~3), 8);
    if constexpr (WORDS & 1) __builtin_memcpy(__builtin_assume_aligned((char*)p + 4 * (WORDS & ~1), 4), w + (WORDS & ~1), 4);
}

// N neighbouring values of a row, `left` of which exist.
template <typename TO, int N> __device__ __forceinline__ void store_run(TO* p, const float (&v)[N], int left, Runs runs)
{
    static_assert(N % 4 == 0, "whole words");
    if (left < N) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) store_from_f32(p + i, v[i]);
        return;
    }
    if constexpr (sizeof(TO) == 4) {
        uint32_t w[N];
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = __builtin_bit_cast(uint32_t, v[i]);
        store_words<N>(p, w);
    } else {
        if (runs != kRunElements || (uintptr_t)p % 4 == 0) {
            uint32_t w[N / 2];
#pragma unroll
            for (int i = 0; i < N / 2; ++i) w[i] = pack2_from_f32<TO>(v[2 * i], v[2 * i + 1]);
            if (N == 4 && runs == kRunPieces) *(uint2*)p = uint2{w[0], w[1]};
            else store_words<N / 2>(p, w);
        } else {
            uint32_t w[N / 2 - 1];
#pragma unroll
            for (int i = 0; i < N / 2 - 1; ++i) w[i] = pack2_from_f32<TO>(v[2 * i + 1], v[2 * i + 2]);
            store_from_f32(p, v[0]);
            store_words<N / 2 - 1>(p + 1, w);
            store_from_f32(p + N - 1, v[N - 1]);
        }
    }
}
template <typename TO, int N> __device__ __forceinline__ void add_run(const TO* p, float (&v)[N], int left, Runs runs)
{
    if (left >= N && (sizeof(TO) == 4 || runs != kRunElements)) {
        TO t[N];
        __builtin_memcpy(t, __builtin_assume_aligned(p, 4), sizeof t);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += to_f32(t[i]);
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
    Runs runs, kept, residual;

    __device__ __forceinline__ RunOutput(const Product& p, int n_) : n(n_), left(p.N - n_)
    {
        runs = runs_of<TO>(p.y, p.ldy);
        kept = runs_of<TO>((const void*)((uintptr_t)p.y0 | (uintptr_t)p.y1), p.ldk);
        residual = runs_of<TO>(p.residual, p.ldr);
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
    // A row's scale, read before other rows are stored: a wait for a load is one for all stores before it.
    static __device__ __forceinline__ float scale(const Product& p, int64_t m) { return kScales && p.sa ? p.sa[min(m, (int64_t)p.M - 1)] : 1.f; }
    __device__ __forceinline__ void store(const Product& p, int64_t m, float sa, const Acc (&first)[RUN / 4], const Acc (&second)[RUN / 4]) const
    {
        float v[RUN];
        values(v, first, s0, sa);
        if constexpr (FORM == kScaled) {
            if (p.bias)
#pragma unroll
                for (int i = 0; i < RUN; ++i) v[i] += bias[i];
            gate_act<RUN>(v, p.act);
            if (p.residual) add_run<TO, RUN>((const TO*)p.residual + m * p.ldr + n, v, left, residual);
        } else if constexpr (FORM == kGated) {
            float u[RUN];
            values(u, second, s1, sa);
            if (p.y0) {
                store_run<TO, RUN>((TO*)p.y0 + m * p.ldk + n, v, left, kept);
                store_run<TO, RUN>((TO*)p.y1 + m * p.ldk + n, u, left, kept);
            }
            gate_act<RUN>(v, p.act);
#pragma unroll
            for (int i = 0; i < RUN; ++i) v[i] *= u[i];
        }
        store_run<TO, RUN>((TO*)p.y + m * p.ldy + n, v, left, runs);
    }
};

}  // namespace rtoss
