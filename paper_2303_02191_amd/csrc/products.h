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
    int64_t ldr, ldy, ldk;  // of residual, y and what is kept (kBackWeights: ldy of both)
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

// ----- launchers -----
rtoss_status launch_quantize_rows(const void* x, rtoss_dtype dt, int64_t M, int K, int64_t ldx, int8_t* q, int64_t ldq, float* scale,
                                  hipStream_t s);
// Every form: kScaled and kGated on 8-bit operands, kGated and the gradients on operands of the result's type.
bool product_pieces_ok(ProductForm form, const Product& p, int eb);  // rows are whole 16-byte pieces (product_tiles.hip)
// ... in tiles of 128 or 256 rows and 128 or 256 channels (kTiles), of 8- and 16-bit operands (product_tiles.hip); the last for whole pieces only
bool product_tiles_ok(bool bits8, rtoss_dtype out, const Product& p);
constexpr struct { int rows, channels; } kTiles[3] = {{128, 128}, {256, 128}, {256, 256}};
rtoss_status launch_product_tiles(ProductForm form, bool bits8, rtoss_dtype out, int tile, const Product& p, hipStream_t s);
// ... of few tiles, and fp32: the sum split over the waves of a workgroup (product_slices.hip).  The tile, rows x channels of a matrix: kSlices;
// gradients take the last.  kSliceTiles: the last, one for every wave (fp32, kGated).
constexpr int kSliceTiles = 5;
constexpr int kMaxSliceTiles = 0xffffffff / 512 / 16 * 8;  // (half of what a grid of 512 lanes each may have)
constexpr struct { int rows, channels, gated; } kSlices[kSliceTiles] = {{16, 16, 16}, {32, 16, 16}, {32, 32, 32}, {64, 32, 16}, {64, 64, 32}};
rtoss_status launch_product_slices(ProductForm form, bool bits8, rtoss_dtype out, int tile, const Product& p, hipStream_t s);
// both gradients in one launch, that of the rows in tiles of 64 (high) or 16 rows, each sum in parts; one without a result (y) is left out
struct SumParts {
    int parts;          // workgroups of a tile
    bool each;          // every wave of a workgroup has a tile of its own (one part; rows: high)
    float* sums;        // of more parts than one: [tile][part][elements of a tile]
    uint32_t* arrived;  // [tile], zero
};
rtoss_status launch_product_slices_back(rtoss_dtype dt, bool high, const Product& rows, const Product& weights, SumParts row_parts, SumParts weight_parts,
                                        hipStream_t s);
// dg = dh * u * act'(g), du = dh * act(g), both [M][ldd] with zeros from column F on (gated_slopes.hip); ldd: slopes_pitch.  Clears `counts` words.
inline int64_t slopes_pitch(int F, rtoss_dtype dt) { return (int64_t)align_up((size_t)F, 16 / elem_bytes(dt)); }
rtoss_status launch_gated_slopes(rtoss_dtype dt, rtoss_act act, int64_t M, int F, const void* dh, int64_t ldh, const void* gate, const void* up,
                                 void* dg, void* du, uint32_t* counters, int counts, hipStream_t s);

}  // namespace rtoss
