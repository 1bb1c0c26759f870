// Products of few rows (single tokens, small batches): the 8-bit product and the gated block where reading the weights is all the work.
//
// A workgroup owns 16 channels (of both weights, for the gated block) and all rows; its waves take the sum's pieces of 128 bytes of a
// row in turn, straight from memory into registers (every weight is used once: there is nothing to stage), and their sums are joined
// in LDS.  Lane (c, q) of a fragment has row c and 32 neighbouring bytes at 32 q of the piece, for two matrix instructions, so that a
// row's piece is one run of 128 bytes; both operands have the sum in this order.  Rows start and end anywhere: whole pieces are loaded
// at whatever address, what is behind the last whole one element by element.
// Bound: memory.  A wave has U pieces of each weight under way.
#include <algorithm>

#include "products.h"

namespace rtoss {

namespace {

constexpr int kPiece = 128;  // bytes of a row

template <typename T> __device__ __forceinline__ u32x4 load_past(const T* row, int r, int R)
{
    constexpr int E = 16 / (int)sizeof(T);
    u32x4 out = {0u, 0u, 0u, 0u};
    if (r + E <= R) {
        __builtin_memcpy(&out, row + r, 16);
        return out;
    }
    T v[E] = {};
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (r + e < R) v[e] = row[r + e];
    __builtin_memcpy(&out, v, 16);
    return out;
}

template <typename T, typename TO, int FORM, int MT, int WAVES, int U>
__global__ __launch_bounds__(64 * WAVES, 2) void product_few_kernel(Product p)
{
    typedef typename AccOf<T>::type Acc;
    constexpr int SUMS = FORM == kGated ? 2 : 1;
    constexpr int E = 16 / (int)sizeof(T), PIECE = kPiece / (int)sizeof(T);
    __shared__ __attribute__((aligned(16))) Acc joined[WAVES][SUMS * MT][64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, q = lane >> 4;
    const int n0 = (int)blockIdx.x * 16;
    // (rows past the last: the last again, not stored)
    const T* w[SUMS];
    w[0] = (const T*)p.b0 + (int64_t)min(n0 + c, p.N - 1) * p.ldb;
    if constexpr (SUMS == 2) w[1] = (const T*)p.b1 + (int64_t)min(n0 + c, p.N - 1) * p.ldb;
    const T* x[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) x[t] = (const T*)p.a0 + (int64_t)min(16 * t + c, p.M - 1) * p.lda;

    Acc acc[SUMS][MT];
#pragma unroll
    for (int i = 0; i < SUMS * MT; ++i) acc[i / MT][i % MT] = Acc{0, 0, 0, 0};
    const int pieces = p.R / PIECE;  // whole ones
    int k = wave;
    for (; k + (U - 1) * WAVES < pieces; k += U * WAVES) {
        u32x4 wf[U][SUMS][2], xf[U][MT][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = (k + u * WAVES) * PIECE + q * 2 * E;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int s = 0; s < SUMS; ++s) __builtin_memcpy(&wf[u][s][h], w[s] + r + h * E, 16);
#pragma unroll
                for (int t = 0; t < MT; ++t) __builtin_memcpy(&xf[u][t][h], x[t] + r + h * E, 16);
            }
        }
        __builtin_amdgcn_sched_barrier(0);  // (all loads under way before the first product)
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int s = 0; s < SUMS; ++s)
#pragma unroll
                    for (int t = 0; t < MT; ++t) acc[s][t] = Mma16<T>::mma(wf[u][s][h], xf[u][t][h], acc[s][t]);
    }
    for (; k * PIECE < p.R; k += WAVES) {  // what is left, the row's end among it
        const int r = k * PIECE + q * 2 * E;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 wf[SUMS], xf[MT];
#pragma unroll
            for (int s = 0; s < SUMS; ++s) wf[s] = load_past(w[s], r + h * E, p.R);
#pragma unroll
            for (int t = 0; t < MT; ++t) xf[t] = load_past(x[t], r + h * E, p.R);
#pragma unroll
            for (int s = 0; s < SUMS; ++s)
#pragma unroll
                for (int t = 0; t < MT; ++t) acc[s][t] = Mma16<T>::mma(wf[s], xf[t], acc[s][t]);
        }
    }
#pragma unroll
    for (int s = 0; s < SUMS; ++s)
#pragma unroll
        for (int t = 0; t < MT; ++t) joined[wave][s * MT + t][lane] = acc[s][t];
    __syncthreads();
    const int t = wave;  // wave t has rows 16 t ..
    const int64_t m = 16 * t + c;
    if (t >= MT || m >= p.M) return;
    Acc sum[SUMS];
#pragma unroll
    for (int s = 0; s < SUMS; ++s) {
        sum[s] = joined[0][s * MT + t][lane];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum[s] += joined[v][s * MT + t][lane];
    }
    const float sa = sizeof(T) == 1 && p.sa ? p.sa[m] : 1.f;
    product_output<FORM, T, TO>(p, product_vec<TO>(p), m, n0 + 4 * q, sa, sum[0], sum[SUMS - 1]);
}

template <typename T, typename TO, int FORM, int MT> rtoss_status launch(const Product& p, hipStream_t s)
{
    constexpr int WAVES = 8, U = FORM == kGated ? (MT > 2 ? 2 : 4) : 4;
    product_few_kernel<T, TO, FORM, MT, WAVES, U><<<(unsigned)((p.N + 15) / 16), 64 * WAVES, 0, s>>>(p);
    return check_hip(hipGetLastError(), "product launch");
}

template <typename T, typename TO, int FORM> rtoss_status launch_rows(const Product& p, hipStream_t s)
{
    return p.M <= 16 ? launch<T, TO, FORM, 1>(p, s) : p.M <= 32 ? launch<T, TO, FORM, 2>(p, s) : launch<T, TO, FORM, 4>(p, s);
}

template <typename TO> rtoss_status launch_bits8(ProductForm form, const Product& p, hipStream_t s)
{
    return form == kScaled ? launch_rows<int8_t, TO, kScaled>(p, s) : launch_rows<int8_t, TO, kGated>(p, s);
}

}  // namespace

bool product_few_ok(ProductForm form, const Product& p) { return (form == kScaled || form == kGated) && p.M <= 64; }

rtoss_status launch_product_few(ProductForm form, bool bits8, rtoss_dtype out, const Product& p, hipStream_t s)
{
    switch (out) {
    case RTOSS_F32: return bits8 ? launch_bits8<float>(form, p, s) : launch_rows<float, float, kGated>(p, s);
    case RTOSS_F16: return bits8 ? launch_bits8<f16_t>(form, p, s) : launch_rows<f16_t, f16_t, kGated>(p, s);
    default: return bits8 ? launch_bits8<bf16_t>(form, p, s) : launch_rows<bf16_t, bf16_t, kGated>(p, s);
    }
}

}  // namespace rtoss
