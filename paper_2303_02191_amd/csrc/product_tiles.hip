// Products of whole 16-byte pieces in tiles of 256 x 256 results: the 8-bit product and the gated block where there are rows enough.
#include <algorithm>

#include "product_run.h"
#include "work_order.h"

namespace rtoss {

namespace {

constexpr int kTileM = 256, kTileN = 256;
constexpr int kStage = 128;                 // bytes of a row in a stage
constexpr int kRegion = 128 * kStage;       // half of an operand's rows
constexpr int kBuffer = 4 * kRegion;        // A half 0, A half 1, B half 0, B half 1
constexpr int kGroupM = 4;                  // row tiles that neighbouring workgroups share

__device__ __forceinline__ void fence() { asm volatile("" ::: "memory"); }

// An operand's rows from some row on, as a bounded buffer: loads past the matrix give nothing.
struct Source {
    const char* p;
    int64_t left;  // bytes from p to the matrix's end
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t at(int64_t offset) const
    {
        const int64_t n = left - offset;
        return __builtin_amdgcn_make_buffer_rsrc((void*)(p + offset), 0, (int)(uint32_t)(n < 0 ? 0 : n > 0xfffffff0ll ? 0xfffffff0ll : n), 0x00027000);
    }
};

template <typename T, typename TO, int FORM>
__global__ __launch_bounds__(512, 2) void product_tiles_kernel(Product p, int tiles_m, int tiles_n, int tiles, int per_xcd)
{
    typedef typename AccOf<T>::type Acc;
    constexpr bool GATED = FORM == kGated;
    constexpr int EB = (int)sizeof(T);
    constexpr int COLS = GATED ? kTileN / 2 : kTileN;  // channels of a tile
    extern __shared__ __attribute__((aligned(16))) char smem[];  // two buffers
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 2, wn = wave & 3;
    const int c = lane & 15, q = lane >> 4;

    const int work = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);
    if (work >= tiles) return;
    const int group = work / (kGroupM * tiles_n), at = work - group * (kGroupM * tiles_n);
    const int high = min(kGroupM, tiles_m - group * kGroupM);
    const int64_t m0 = (int64_t)(group * kGroupM + at % high) * kTileM;
    const int n0 = at / high * COLS;

    const int64_t lda = p.lda * EB, ldb = p.ldb * EB, row = (int64_t)p.R * EB;
    const int S = (int)((row + kStage - 1) / kStage);
    const int tail = (int)((row - (int64_t)(S - 1) * kStage) / 16);  // pieces of a row in the last stage
    const Source a{(const char*)p.a0 + m0 * lda, (p.M - 1 - m0) * lda + row};
    const Source b0{(const char*)p.b0 + n0 * ldb, (p.N - 1 - n0) * ldb + row};
    const Source b1{(const char*)(GATED ? p.b1 : p.b0) + n0 * ldb, (p.N - 1 - n0) * ldb + row};

    // ---- copies: a region of 128 rows is 16 instructions of 8 rows x 128 bytes, two per wave; piece k of row r lies at place k ^ (r % 8) ----
    const int sub = lane >> 3, piece = (lane & 7) ^ sub;
    uint32_t va[2], vb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int rho = wave * 16 + i * 8 + sub;
        va[i] = (uint32_t)((rho >> 6) * 128 + (rho & 63)) * (uint32_t)lda + piece * 16;
        const int slot = rho >> 5, j = rho >> 4 & 1, r = rho & 15;
        const int ch = GATED ? slot * 32 + 8 * (r >> 2) + 4 * j + (r & 3) : slot * 64 + 16 * (r >> 2) + 4 * j + (r & 3);
        vb[i] = (uint32_t)ch * (uint32_t)ldb + piece * 16;
    }
    // kind: 0, 1 halves of A; 2, 3 halves of B
    auto issue = [&](int stage, int kind) {
        char* to = smem + (stage & 1) * kBuffer + kind * kRegion + wave * 2048;
        const int64_t k = (int64_t)min(stage, S - 1) * kStage;
        const __amdgpu_buffer_rsrc_t from = kind == 0   ? a.at(k)
                                            : kind == 1 ? a.at(k + 64 * lda)
                                            : kind == 2 ? b0.at(k)
                                                        : b1.at(k + (GATED ? 0 : 8 * ldb));
#pragma unroll
        for (int i = 0; i < 2; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(to + i * 1024), 16, kind < 2 ? va[i] : vb[i], 0, 0, 0);
    };

    Acc acc[8][4];
#pragma unroll
    for (int i = 0; i < 32; ++i) acc[i >> 2][i & 3] = Acc{0, 0, 0, 0};
    u32x4 af[4][2], bf[2][2][2];  // [tile][step], [half][tile][step]
    const int at0 = c * kStage + ((q ^ (c & 7)) * 16);  // place of piece q of row c; of piece 4 + q: the same with bit 6 flipped
    auto read_a = [&](int buf, int half) {
        const char* base = smem + buf * kBuffer + half * kRegion + wm * 64 * kStage;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s) af[t][s] = *(const u32x4*)(base + t * 16 * kStage + (at0 ^ (s * 64)));
    };
    auto read_b = [&](int buf, int half) {
        const char* base = smem + buf * kBuffer + (2 + half) * kRegion + wn * 32 * kStage;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s) bf[half][t][s] = *(const u32x4*)(base + t * 16 * kStage + (at0 ^ (s * 64)));
    };
    auto clear_past = [&](u32x4& f, int s) {
        if (4 * s + q >= tail) f = u32x4{0u, 0u, 0u, 0u};
    };
    auto multiply = [&](int ma, int nb) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) acc[ma * 4 + t][nb * 2 + u] = Mma16<T>::mma(bf[nb][u][s], af[t][s], acc[ma * 4 + t][nb * 2 + u]);
        __builtin_amdgcn_s_setprio(0);
    };
    auto meet = [&] {
        fence();
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        fence();
    };
    constexpr int kWait = 0x0f70 | 10;  // vmcnt(10): the copies of all but the five newest regions have landed
    auto landed = [&] {
        fence();
        __builtin_amdgcn_s_waitcnt(kWait);
    };
    // one stage: four quadrants of the wave's tile
    auto stage_of = [&](int s, auto first) {
        constexpr int X = decltype(first)::value;  // the half of B whose operands are there already
        const bool part = s == S - 1 && tail < 8;  // uniform: the rows end in this stage
        const int buf = X;  // (stage parity)
        read_a(buf, 0);
        issue(s + 1, 1);
        landed();
        __builtin_amdgcn_s_waitcnt(0xc87f);  // lgkmcnt(8): and the reads in front of this stage's
        meet();
        if (part) {
#pragma unroll
            for (int i = 0; i < 8; ++i) clear_past(af[i >> 1][i & 1], i & 1);
#pragma unroll
            for (int i = 0; i < 4; ++i) clear_past(bf[X][i >> 1][i & 1], i & 1);
        }
        multiply(0, X);
        meet();

        read_b(buf, 1 - X);
        issue(s + 2, 2 + X);
        landed();
        meet();
        if (part) {
#pragma unroll
            for (int i = 0; i < 4; ++i) clear_past(bf[1 - X][i >> 1][i & 1], i & 1);
        }
        multiply(0, 1 - X);
        meet();

        read_a(buf, 1);
        issue(s + 2, 0);
        landed();
        meet();
        if (part) {
#pragma unroll
            for (int i = 0; i < 8; ++i) clear_past(af[i >> 1][i & 1], i & 1);
        }
        multiply(1, 1 - X);
        meet();

        read_b(1 - buf, 1 - X);  // (of the next stage; behind the last one of something that nobody uses)
        issue(s + 2, 3 - X);
        landed();
        meet();
        multiply(1, X);
        meet();
    };

    issue(0, 2), issue(0, 0), issue(0, 3), issue(0, 1), issue(1, 3), issue(1, 0), issue(1, 2);
    landed();
    meet();
    read_b(0, 0);
    if (wm) meet();  // the waves of one half are half a quadrant behind the others'
    for (int s = 0;;) {
        stage_of(s, std::integral_constant<int, 0>{});
        if (++s == S) break;
        stage_of(s, std::integral_constant<int, 1>{});
        if (++s == S) break;
    }
    if (!wm) meet();
    __builtin_amdgcn_s_waitcnt(0x0f70);  // the surplus copies have landed: LDS may be given away

    // ---- results: a lane holds 16 neighbouring channels (gated: 8 of each projection) of eight rows ----
    constexpr int RUN = GATED ? 8 : 16;
    const int n = n0 + wn * (GATED ? 32 : 64) + RUN * q;
    if (n >= p.N) return;
    const RunOutput<FORM, T, TO, RUN> out(p, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t m = m0 + wm * 128 + i * 16 + c;
        if (m >= p.M) continue;
        Acc first[RUN / 4], second[RUN / 4];
#pragma unroll
        for (int t = 0; t < RUN / 4; ++t) {
            first[t] = acc[i][t];
            second[t] = acc[i][GATED ? 2 + t : t];
        }
        out.store(p, m, first, second);
    }
}

template <typename T, typename TO, int FORM> rtoss_status launch(const Product& p, hipStream_t s)
{
    constexpr int COLS = FORM == kGated ? kTileN / 2 : kTileN;
    static LaunchOnce once;
    DeviceInfo dev;
    if (rtoss_status st = current_device(&dev)) return st;
    const auto kernel = product_tiles_kernel<T, TO, FORM>;
    if (rtoss_status st = ensure_dynamic_lds((const void*)kernel, 2 * kBuffer, once, dev.device, "LDS of a product")) return st;
    const int tiles_m = (int)(((int64_t)p.M + kTileM - 1) / kTileM), tiles_n = (p.N + COLS - 1) / COLS;
    const int64_t tiles = (int64_t)tiles_m * tiles_n;
    const int64_t per_xcd = (tiles + 7) / 8;
    kernel<<<(unsigned)(per_xcd * 8), 512, 2 * kBuffer, s>>>(p, tiles_m, tiles_n, (int)tiles, (int)per_xcd);
    return check_hip(hipGetLastError(), "product launch");
}

}  // namespace

bool product_pieces_ok(const Product& p, int eb, bool two)
{
    const uintptr_t all = (uintptr_t)p.a0 | (uintptr_t)p.b0 | (two ? (uintptr_t)p.b1 : 0);
    // (a tile's rows are 32-bit offsets from its first)
    return all % 16 == 0 && p.lda * eb % 16 == 0 && p.ldb * eb % 16 == 0 && (int64_t)p.R * eb % 16 == 0 && p.R > 0 && p.lda * eb <= 1 << 23 &&
           p.ldb * eb <= 1 << 23;
}

bool product_tiles_ok(ProductForm form, bool bits8, rtoss_dtype out, const Product& p)
{
    if (form != kScaled && form != kGated) return false;
    if (!product_pieces_ok(p, bits8 ? 1 : elem_bytes(out), form == kGated)) return false;
    const int cols = form == kGated ? kTileN / 2 : kTileN;
    return (((int64_t)p.M + kTileM - 1) / kTileM) * ((p.N + cols - 1) / cols) <= kMaxGridGroups / 2;
}

rtoss_status launch_product_tiles(ProductForm form, bool bits8, rtoss_dtype out, const Product& p, hipStream_t s)
{
    switch (out) {
    case RTOSS_F32:
        return !bits8 ? launch<float, float, kGated>(p, s) : form == kScaled ? launch<int8_t, float, kScaled>(p, s) : launch<int8_t, float, kGated>(p, s);
    case RTOSS_F16:
        return !bits8 ? launch<f16_t, f16_t, kGated>(p, s) : form == kScaled ? launch<int8_t, f16_t, kScaled>(p, s) : launch<int8_t, f16_t, kGated>(p, s);
    default:
        return !bits8 ? launch<bf16_t, bf16_t, kGated>(p, s) : form == kScaled ? launch<int8_t, bf16_t, kScaled>(p, s) : launch<int8_t, bf16_t, kGated>(p, s);
    }
}

}  // namespace rtoss
