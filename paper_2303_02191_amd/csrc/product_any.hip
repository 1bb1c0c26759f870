// Products of any sizes, pitches and alignments: the 8-bit product, the gated block and its gradients where rows are not whole
// 16-byte pieces.
//
// A workgroup owns a tile of 64 x 64 results; the sum runs over stages of 64 bytes a row, through registers into LDS (a piece of a row
// that is whole is loaded as 16 bytes at whatever address it starts, others element by element with zeros past the end).  Four
// waves of 32 x 32 results each.  The right operand's rows are the matrix instruction's first operand, so that a lane holds four
// neighbouring channels of one row.
#include <algorithm>

#include "products.h"

namespace rtoss {

namespace {

constexpr int kTile = 64;
constexpr int kPitch = 80;  // bytes of a staged row: 64, and 16 that spread neighbouring rows over the banks

// 16 bytes of a staged row: elements r .. of operand row i, zeros outside.  ROWS: r is the direction in which memory is contiguous.
template <typename T, bool ROWS>
__device__ __forceinline__ u32x4 load_piece(const T* __restrict__ p, int64_t ld, int64_t i, int rows, int r, int R)
{
    constexpr int E = 16 / (int)sizeof(T);
    u32x4 out = {0u, 0u, 0u, 0u};
    if (i >= rows || r >= R) return out;
    if constexpr (ROWS) {
        const T* at = p + i * ld + r;
        if (r + E <= R) {
            __builtin_memcpy(&out, at, 16);
            return out;
        }
        T v[E] = {};
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (r + e < R) v[e] = at[e];
        __builtin_memcpy(&out, v, 16);
    } else {
        T v[E] = {};
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (r + e < R) v[e] = p[(int64_t)(r + e) * ld + i];
        __builtin_memcpy(&out, v, 16);
    }
    return out;
}

template <typename T, typename TO, int FORM> __global__ __launch_bounds__(256, 2) void product_any_kernel(Product p, int tiles_n, int64_t tiles)
{
    typedef typename AccOf<T>::type Acc;
    constexpr int E = 16 / (int)sizeof(T), STAGE = 4 * E;
    constexpr bool A_ROWS = FORM != kBackWeights, B_ROWS = FORM == kScaled || FORM == kGated;
    constexpr int SUMS = FORM == kGated ? 2 : 1;  // (products that share the left operand)
    __shared__ __attribute__((aligned(16))) char lds[(1 + SUMS) * kTile * kPitch];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int c = lane & 15, q = lane >> 4;
    const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
    const T *a0 = (const T*)p.a0, *b0 = (const T*)p.b0;
    if (FORM == kBackWeights && blockIdx.y) {
        a0 = (const T*)p.a1;
        p.y = p.y1;
    }
    const ProductVec vec = product_vec<TO>(p);
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int64_t m0 = t / tiles_n * kTile;
        const int n0 = (int)(t % tiles_n) * kTile;
        Acc acc[SUMS][2][2];
#pragma unroll
        for (int s = 0; s < SUMS; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[s][i >> 1][i & 1] = Acc{0, 0, 0, 0};
        const int passes = FORM == kBackRows ? 2 : 1;  // (the second pair of operands adds to the same sums)
        for (int pass = 0; pass < passes; ++pass) {
            const T* a = pass ? (const T*)p.a1 : a0;
            const T* b = pass ? (const T*)p.b1 : b0;
            for (int r0 = 0; r0 < p.R; r0 += STAGE) {
                // (memory's contiguous direction across neighbouring lanes)
                const int ai = A_ROWS ? tid >> 2 : tid & 63, aq = A_ROWS ? tid & 3 : tid >> 6;
                const int bi = B_ROWS ? tid >> 2 : tid & 63, bq = B_ROWS ? tid & 3 : tid >> 6;
                const u32x4 av = load_piece<T, A_ROWS>(a, p.lda, m0 + ai, p.M, r0 + aq * E, p.R);
                u32x4 bv[SUMS];
                bv[0] = load_piece<T, B_ROWS>(b, p.ldb, n0 + bi, p.N, r0 + bq * E, p.R);
                if constexpr (SUMS == 2) bv[1] = load_piece<T, B_ROWS>((const T*)p.b1, p.ldb, n0 + bi, p.N, r0 + bq * E, p.R);
                __syncthreads();  // everybody is done with the stage before
                *(u32x4*)(lds + ai * kPitch + aq * 16) = av;
#pragma unroll
                for (int s = 0; s < SUMS; ++s) *(u32x4*)(lds + (1 + s) * kTile * kPitch + bi * kPitch + bq * 16) = bv[s];
                __syncthreads();
                u32x4 af[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) af[i] = *(const u32x4*)(lds + (wm + 16 * i + c) * kPitch + q * 16);
#pragma unroll
                for (int s = 0; s < SUMS; ++s)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const u32x4 bf = *(const u32x4*)(lds + ((1 + s) * kTile + wn + 16 * j + c) * kPitch + q * 16);
#pragma unroll
                        for (int i = 0; i < 2; ++i) acc[s][i][j] = Mma16<T>::mma(bf, af[i], acc[s][i][j]);
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t m = m0 + wm + 16 * i + c;
            if (m >= p.M) continue;
            const float sa = sizeof(T) == 1 && p.sa ? p.sa[m] : 1.f;
#pragma unroll
            for (int j = 0; j < 2; ++j)
                product_output<FORM, T, TO>(p, vec, m, n0 + wn + 16 * j + 4 * q, sa, acc[0][i][j], acc[SUMS - 1][i][j]);
        }
    }
}

template <typename T, typename TO, int FORM> rtoss_status launch(const Product& p, hipStream_t s)
{
    const int tiles_n = (p.N + kTile - 1) / kTile;
    const int64_t tiles = ((int64_t)p.M + kTile - 1) / kTile * tiles_n;
    const dim3 grid((unsigned)std::min<int64_t>(tiles, kMaxGridGroups), FORM == kBackWeights ? 2 : 1);
    product_any_kernel<T, TO, FORM><<<grid, 256, 0, s>>>(p, tiles_n, tiles);
    return check_hip(hipGetLastError(), "product launch");
}

template <typename T, typename TO> rtoss_status launch_form(ProductForm form, const Product& p, hipStream_t s)
{
    if constexpr (sizeof(T) == 1) {
        return form == kScaled ? launch<T, TO, kScaled>(p, s) : launch<T, TO, kGated>(p, s);
    } else {
        return form == kGated      ? launch<T, TO, kGated>(p, s)
               : form == kBackRows ? launch<T, TO, kBackRows>(p, s)
                                   : launch<T, TO, kBackWeights>(p, s);
    }
}

}  // namespace

rtoss_status launch_product_any(ProductForm form, bool bits8, rtoss_dtype out, const Product& p, hipStream_t s)
{
    switch (out) {
    case RTOSS_F32: return bits8 ? launch_form<int8_t, float>(form, p, s) : launch_form<float, float>(form, p, s);
    case RTOSS_F16: return bits8 ? launch_form<int8_t, f16_t>(form, p, s) : launch_form<f16_t, f16_t>(form, p, s);
    case RTOSS_BF16: return bits8 ? launch_form<int8_t, bf16_t>(form, p, s) : launch_form<bf16_t, bf16_t>(form, p, s);
    }
    return fail(RTOSS_EDTYPE, "bad dtype %d", (int)out);
}

}  // namespace rtoss
