// Internal declarations of the 8-bit products and the gated feed-forward block: what their kernels share.
#pragma once
#include "common.h"
#include "dtypes.h"
#include "epilogue.h"
#include "mma.h"

namespace rtoss {

// What a launch computes.  A product has rows m (tokens, positions) of a left operand and rows n (output channels) of a right one, and
// sums over r:
//   kScaled       y[m][n] = act(sa[m] * s0[n] * sum_r a0[m][r] b0[n][r] + bias[n]) + residual[m][n]      8-bit operands, whole-number sums
//   kGated        y[m][n] = act(g) * u,  g = sum_r a0[m][r] b0[n][r],  u = sum_r a0[m][r] b1[n][r]       (8 bits: each scaled as above)
//   kBackRows     y[m][n] = sum_r a0[m][r] b0[r][n] + sum_r a1[m][r] b1[r][n]                            gradient of the rows
//   kBackWeights  y0[m][n] = sum_r a0[r][m] b0[r][n],  y1 likewise from a1                               gradients of both weights
enum ProductForm { kScaled = 0, kGated, kBackRows, kBackWeights };

struct Product {
    const void *a0, *a1, *b0, *b1;
    int64_t lda, ldb;  // elements from one row in memory to the next
    int M, N, R;
    int act;
    const float *sa, *s0, *s1, *bias;  // nullptr: 1, 1, 1, 0
    const void* residual;
    void *y, *y0, *y1;  // kGated: y0, y1 keep g and u, or nullptr
    int64_t ldr, ldy;   // of residual and y (y0 and y1 are plain)
};

// ReLU keeps a NaN, as the plain comparison does (a row that could not be quantized stays visible); SiLU: epilogue.h.
template <int N> __device__ __forceinline__ void gate_act(float (&v)[N], int act)
{
    if (act == 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];
    } else if (act == 2) {
        epi_silu<N>(v);
    }
}

// Four neighbouring values of a row, `left` of which exist.  VEC: the row's runs of four are aligned to their size.
template <typename TO> __device__ __forceinline__ void store4(TO* p, const float (&v)[4], int left, bool vec)
{
    if (vec && left >= 4) {
        if constexpr (sizeof(TO) == 4) *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
        else *(uint2*)p = uint2{pack2_from_f32<TO>(v[0], v[1]), pack2_from_f32<TO>(v[2], v[3])};
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) store_from_f32(p + i, v[i]);
}
template <typename TO> __device__ __forceinline__ void load4(const TO* p, float (&v)[4], int left, bool vec)
{
    if (vec && left >= 4) {
        if constexpr (sizeof(TO) == 4) {
            const f32x4 t = *(const f32x4*)p;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = t[i];
        } else {
            TO t[4];
            *(uint2*)t = *(const uint2*)p;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = to_f32(t[i]);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < left ? to_f32(p[i]) : 0.f;
}
// Whether runs of four elements of TO that start at multiples of four in rows `ld` apart are aligned to their size.
template <typename TO> __host__ __device__ __forceinline__ bool runs_of_4(const void* p, int64_t ld)
{
    return ((uintptr_t)p % (4 * sizeof(TO))) == 0 && ld % 4 == 0;
}

// Accumulators of the 16-bit types and fp32 are fp32, of 8-bit operands 32-bit integers (exact for R < 2^17).
typedef int i32x4 __attribute__((ext_vector_type(4)));
template <typename T> struct AccOf { typedef f32x4 type; };
template <> struct AccOf<int8_t> { typedef i32x4 type; };
template <typename T> struct Mma16 : Dense16<T> {};
template <> struct Mma16<int8_t> {
    static __device__ __forceinline__ i32x4 mma(u32x4 a, u32x4 b, i32x4 c)
    {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
    }
};

// Output stage for four neighbouring channels n .. n+3 of row m; `left` of them exist.  acc1: kGated's second sum.
struct ProductVec {
    bool y, kept, residual;  // runs of four are aligned
};
template <typename TO> __device__ __forceinline__ ProductVec product_vec(const Product& p)
{
    return ProductVec{runs_of_4<TO>(p.y, p.ldy), runs_of_4<TO>(p.y0, p.N) && runs_of_4<TO>(p.y1, p.N), runs_of_4<TO>(p.residual, p.ldr)};
}
template <typename T, typename ACC> __device__ __forceinline__ void scaled4(float (&v)[4], ACC acc, float sa, const float* s, int left)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = (float)acc[i];  // (whole numbers above 2^24 round here, to 24 bits as every fp32 value)
        if constexpr (sizeof(T) == 1) {
            v[i] *= sa;
            if (s && i < left) v[i] *= s[i];
        }
    }
}
template <int FORM, typename T, typename TO, typename ACC>
__device__ __forceinline__ void product_output(const Product& p, const ProductVec& vec, int64_t m, int n, float sa, ACC acc0, ACC acc1)
{
    const int left = p.N - n;
    if (left <= 0) return;
    float v[4];
    scaled4<T>(v, acc0, sa, p.s0 ? p.s0 + n : nullptr, left);
    if constexpr (FORM == kScaled) {
        if (p.bias)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += i < left ? p.bias[n + i] : 0.f;
        gate_act<4>(v, p.act);
        if (p.residual) {
            float r[4];
            load4((const TO*)p.residual + m * p.ldr + n, r, left, vec.residual);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += r[i];
        }
    } else if constexpr (FORM == kGated) {
        float u[4];
        scaled4<T>(u, acc1, sa, p.s1 ? p.s1 + n : nullptr, left);
        if (p.y0) {
            store4((TO*)p.y0 + m * p.N + n, v, left, vec.kept);
            store4((TO*)p.y1 + m * p.N + n, u, left, vec.kept);
        }
        gate_act<4>(v, p.act);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= u[i];
    }
    store4((TO*)p.y + m * p.ldy + n, v, left, vec.y);
}

// ----- launchers -----
rtoss_status launch_quantize_rows(const void* x, rtoss_dtype dt, int64_t M, int K, int64_t ldx, int8_t* q, int64_t ldq, float* scale,
                                  hipStream_t s);
// kScaled and kGated on 8-bit operands, kGated and the gradients on operands of the result's type (product_any.hip)
rtoss_status launch_product_any(ProductForm form, bool bits8, rtoss_dtype out, const Product& p, hipStream_t s);
// kScaled and kGated of few rows, of any alignment (product_few.hip)
bool product_few_ok(ProductForm form, const Product& p);
rtoss_status launch_product_few(ProductForm form, bool bits8, rtoss_dtype out, const Product& p, hipStream_t s);
// every form on whole 16-byte pieces of rows, in tiles of 256 x 256 results (product_tiles.hip)
bool product_pieces_ok(ProductForm form, const Product& p, int eb);
bool product_tiles_ok(ProductForm form, bool bits8, rtoss_dtype out, const Product& p);
rtoss_status launch_product_tiles(ProductForm form, bool bits8, rtoss_dtype out, const Product& p, hipStream_t s);
// the same in small tiles, 0: 64 x 64, 1: 128 x 64, 2: 128 x 128 (product_mid.hip)
rtoss_status launch_product_mid(ProductForm form, bool bits8, rtoss_dtype out, int tile, const Product& p, hipStream_t s);
// ... of few tiles: the sum split over the waves of a workgroup (product_slices.hip)
rtoss_status launch_product_slices(ProductForm form, bool bits8, rtoss_dtype out, const Product& p, hipStream_t s);
// dg = dh * u * act'(g), du = dh * act(g), both [M][ldd] with zeros from column F on (gated_slopes.hip); ldd: slopes_pitch
inline int64_t slopes_pitch(int F, rtoss_dtype dt) { return (int64_t)align_up((size_t)F, 16 / elem_bytes(dt)); }
rtoss_status launch_gated_slopes(rtoss_dtype dt, rtoss_act act, int64_t M, int F, const void* dh, int64_t ldh, const void* gate, const void* up,
                                 void* dg, void* du, hipStream_t s);

}  // namespace rtoss
