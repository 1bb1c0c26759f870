// Products of whole 16-byte pieces in small tiles: launches that 256 x 256 tiles would leave most of the chip without work.
//
// A workgroup of four waves (2 x 2) owns BM x BN results; the sum runs over stages of 128 bytes of a row through a ring of BUFS buffers in
// LDS, one barrier a stage.  Operands lie in LDS as in product_tiles.hip.
// Bound: the copies, some 64 bytes a cycle and CU; the waves of two or more workgroups of a CU fill each other's waits.
#include <algorithm>

#include "product_run.h"
#include "product_tile.h"

namespace rtoss {

namespace {

template <typename T, typename TO, int FORM, int BM, int BN, int BUFS>
__global__ __launch_bounds__(256, 2) void product_mid_kernel(Product p, int tiles_m, int tiles_n, int tiles, int per_xcd)
{
    typedef typename AccOf<T>::type Acc;
    constexpr bool GATED = FORM == kGated;
    constexpr bool A_ACROSS = FORM == kBackWeights, B_ACROSS = FORM == kBackRows || FORM == kBackWeights;
    constexpr int EB = (int)sizeof(T), STAGE = kStage / EB;  // rows of the sum in a stage
    constexpr int COLS = GATED ? BN / 2 : BN;                // channels of a tile
    constexpr int MT = BM / 32, NT = BN / 32;                // 16 x 16 tiles of a wave
    constexpr int A_BYTES = BM * kStage, B_BYTES = BN * kStage, BUFFER = A_BYTES + B_BYTES;
    constexpr int A_COPIES = BM / 32, B_COPIES = BN / 32;    // instructions of a wave and stage
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const int c = lane & 15, q = lane >> 4;

    // (XCD-contiguous, rows fastest: the weights are read once, the rows stay in the XCD's L2)
    const int work = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);
    if (work >= tiles) return;
    int tile_m = work % tiles_m;
    const int n0 = work / tiles_m * COLS;
    if constexpr (FORM == kBackWeights) {  // the second weight's tiles are behind the first's
        const int one = tiles_m / 2;
        if (tile_m >= one) {
            tile_m -= one;
            p.a0 = p.a1;
            p.y = p.y1;
        }
    }
    const int64_t m0 = (int64_t)tile_m * BM;

    const int64_t lda = p.lda * EB, ldb = p.ldb * EB, row = (int64_t)p.R * EB;
    const int S1 = (p.R + STAGE - 1) / STAGE, S = FORM == kBackRows ? 2 * S1 : S1;
    const int rest = p.R - (S1 - 1) * STAGE;  // rows of the sum in the last stage
    auto whole = [](int64_t bytes) { return (bytes + 15) & ~(int64_t)15; };  // (dg and du, whose rows are padded)
    auto rows_from = [&](const void* base, int64_t ld, int64_t first, int64_t rows) {
        return Source{(const char*)base + first * ld, (rows - 1 - first) * ld + whole(row)};
    };
    auto columns_from = [&](const void* base, int64_t ld, int64_t first, int64_t columns) {
        return Source{(const char*)base + first * EB, (int64_t)(p.R - 1) * ld + whole((columns - first) * EB)};
    };
    const Source a0 = A_ACROSS ? columns_from(p.a0, lda, m0, p.M) : rows_from(p.a0, lda, m0, p.M);
    const Source a1 = FORM == kBackRows ? rows_from(p.a1, lda, m0, p.M) : a0;
    const Source b0 = B_ACROSS ? columns_from(p.b0, ldb, n0, p.N) : rows_from(p.b0, ldb, n0, p.N);
    const Source b1 = GATED ? rows_from(p.b1, ldb, n0, p.N) : FORM == kBackRows ? columns_from(p.b1, ldb, n0, p.N) : b0;

    // ---- copies; a lane's channel is such that its results are neighbouring channels.  Gated: the second half of B's rows are w_up's ----
    typedef Across<T, BM < 64 ? 64 : BM> AcrossA;
    typedef Across<T, BN> AcrossB;
    const int sub = lane >> 3, piece = (lane & 7) ^ sub;
    uint32_t va[A_COPIES], vb[B_COPIES];
#pragma unroll
    for (int i = 0; i < A_COPIES; ++i) {
        const int k = i * 4 + wave;  // copy instruction of the operand
        if constexpr (A_ACROSS) {
            const int r = k * AcrossA::kCopyRows + lane / AcrossA::kPieces;
            va[i] = (uint32_t)r * (uint32_t)lda + (lane % AcrossA::kPieces ^ AcrossA::spread(r)) * 16;
        } else {
            va[i] = (uint32_t)(k * 8 + sub) * (uint32_t)lda + piece * 16;
        }
    }
#pragma unroll
    for (int i = 0; i < B_COPIES; ++i) {
        const int k = i * 4 + wave;
        if constexpr (B_ACROSS) {
            const int r = k * AcrossB::kCopyRows + lane / AcrossB::kPieces;
            vb[i] = (uint32_t)r * (uint32_t)ldb + (lane % AcrossB::kPieces ^ AcrossB::spread(r)) * 16;
        } else {
            constexpr int TILES = GATED ? NT / 2 : NT;  // of a wave and matrix
            const int rho = (k * 8 + sub) % COLS, slot = rho / (16 * TILES), t = rho / 16 % TILES, r = rho & 15;
            vb[i] = (uint32_t)(slot * 16 * TILES + 4 * TILES * (r >> 2) + 4 * t + (r & 3)) * (uint32_t)ldb + piece * 16;
        }
    }
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_offset(smem)) + wave * 1024;
    auto issue = [&](int stage, int buf) {
        const uint32_t to = lds0 + buf * BUFFER;
        int st = min(stage, S - 1);
        const bool second = FORM == kBackRows && st >= S1;  // uniform: the second pair of operands
        if (second) st -= S1;
        const __amdgpu_buffer_rsrc_t from_a = (second ? a1 : a0).at(A_ACROSS ? (int64_t)st * STAGE * lda : (int64_t)st * kStage);
        const int64_t kb = B_ACROSS ? (int64_t)st * STAGE * ldb : (int64_t)st * kStage;
        const __amdgpu_buffer_rsrc_t from_b = (second ? b1 : b0).at(kb);
        const __amdgpu_buffer_rsrc_t from_up = GATED ? b1.at(kb) : from_b;
#pragma unroll
        for (int i = 0; i < A_COPIES; ++i) copy16_bounded(from_a, va[i], to + i * 4096);
#pragma unroll
        for (int i = 0; i < B_COPIES; ++i) copy16_bounded(GATED && i >= B_COPIES / 2 ? from_up : from_b, vb[i], to + A_BYTES + i * 4096);
    };

    Acc acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT * NT; ++i) acc[i / NT][i % NT] = Acc{0, 0, 0, 0};
    // places of the wave's fragments in a buffer
    const int at0 = c * kStage + ((q ^ (c & 7)) * 16);
    int at_a[MT], at_b[NT];
#pragma unroll
    for (int t = 0; t < MT; ++t) at_a[t] = A_ACROSS ? AcrossA::address(wm * MT + t, c, q) : (wm * MT + t) * 16 * kStage + at0;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int rows16 = GATED ? t / (NT / 2) * (COLS / 16) + wn * (NT / 2) + t % (NT / 2) : wn * NT + t;
        at_b[t] = A_BYTES + (B_ACROSS ? AcrossB::address(wn * NT + t, c, q) : rows16 * 16 * kStage + at0);
    }
    struct Operands {
        u32x4 a[2][MT], b[2][NT];
    } even, odd;  // of two stages
    auto read = [&](int buf, Operands& o) {
        const char* base = smem + buf * BUFFER;
#pragma unroll
        for (int step = 0; step < 2; ++step) {
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                if constexpr (A_ACROSS) o.a[step][t] = AcrossA::read(base + at_a[t] + step * (A_BYTES / 2));
                else o.a[step][t] = *(const u32x4*)(base + (at_a[t] ^ (step * 64)));
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if constexpr (B_ACROSS) o.b[step][t] = AcrossB::read(base + at_b[t] + step * (B_BYTES / 2));
                else o.b[step][t] = *(const u32x4*)(base + (at_b[t] ^ (step * 64)));
            }
        }
    };
    constexpr int PER_STAGE = A_COPIES + B_COPIES;
    static_assert((BUFS - 1) * PER_STAGE < 64, "the counter's range");
    auto landed = [&](auto stages) {  // all copies but those of so many stages; this wave's reads are done
        constexpr int COPIES = decltype(stages)::value * PER_STAGE;
        fence();
        __builtin_amdgcn_s_waitcnt(0x0070 | (COPIES & 15) | (COPIES >> 4) << 14);
        __builtin_amdgcn_s_barrier();
        fence();
    };
    // Stage s is in registers: its buffer is copied over, the next stage is read, and s is multiplied meanwhile.
    auto stage_of = [&](int s, Operands& now, Operands& next) {
        landed(std::integral_constant<int, BUFS - 2>{});
        const int buf = s % BUFS;
        read(buf + 1 == BUFS ? 0 : buf + 1, next);
        issue(s + BUFS, buf);
        __builtin_amdgcn_sched_barrier(0);
        if (__builtin_expect(rest < STAGE && (s == S - 1 || (FORM == kBackRows && s == S1 - 1)), 0)) {  // uniform: the sum ends in this stage
#pragma unroll
            for (int step = 0; step < 2; ++step) {
                const int valid = rest - (4 * step + q) * (16 / EB);
#pragma unroll
                for (int t = 0; t < MT; ++t) keep_first<T>(now.a[step][t], valid);
#pragma unroll
                for (int t = 0; t < NT; ++t) keep_first<T>(now.b[step][t], valid);
            }
        }
#pragma unroll
        for (int step = 0; step < 2; ++step)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = Mma16<T>::mma(now.b[step][j], now.a[step][i], acc[i][j]);
    };
#pragma unroll
    for (int s = 0; s < BUFS; ++s) issue(s, s);
    landed(std::integral_constant<int, BUFS - 1>{});
    read(0, even);
    for (int s = 0;;) {
        stage_of(s, even, odd);
        if (++s == S) break;
        stage_of(s, odd, even);
        if (++s == S) break;
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);  // the surplus copies have landed: LDS may be given away

    constexpr int RUN = GATED ? 2 * NT : B_ACROSS ? 4 : 4 * NT, RUNS = B_ACROSS ? NT : 1;
#pragma unroll
    for (int u = 0; u < RUNS; ++u) {
        const int n = n0 + (B_ACROSS ? (wn * NT + u) * 16 : wn * (COLS / 2)) + RUN * q;
        if (n >= p.N) continue;
        const RunOutput<FORM, T, TO, RUN> out(p, n);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int64_t m = m0 + (wm * MT + i) * 16 + c;
            if (m >= p.M) continue;
            Acc first[RUN / 4], second[RUN / 4];
#pragma unroll
            for (int t = 0; t < RUN / 4; ++t) {
                first[t] = acc[i][u + t];
                second[t] = acc[i][GATED ? NT / 2 + t : u + t];
            }
            out.store(p, m, first, second);
        }
    }
}

template <typename T, typename TO, int FORM, int BM, int BN, int BUFS> rtoss_status launch(const Product& p, hipStream_t s)
{
    constexpr int COLS = FORM == kGated ? BN / 2 : BN, LDS = BUFS * (BM + BN) * kStage;
    static LaunchOnce once;
    DeviceInfo dev;
    if (rtoss_status st = current_device(&dev)) return st;
    const auto kernel = product_mid_kernel<T, TO, FORM, BM, BN, BUFS>;
    if (rtoss_status st = ensure_dynamic_lds((const void*)kernel, LDS, once, dev.device, "LDS of a product")) return st;
    const int tiles_m = (int)(((int64_t)p.M + BM - 1) / BM) * (FORM == kBackWeights ? 2 : 1), tiles_n = (p.N + COLS - 1) / COLS;
    const int64_t tiles = (int64_t)tiles_m * tiles_n, per_xcd = (tiles + 7) / 8;
    kernel<<<(unsigned)(per_xcd * 8), 256, LDS, s>>>(p, tiles_m, tiles_n, (int)tiles, (int)per_xcd);
    return check_hip(hipGetLastError(), "product launch");
}

template <typename T, typename TO, int FORM> rtoss_status launch_tile(int tile, const Product& p, hipStream_t s)
{
    switch (tile) {
    case 0: return launch<T, TO, FORM, 64, 64, 4>(p, s);
    case 4: return launch<T, TO, FORM, 64, 64, 8>(p, s);
    case 5: return launch<T, TO, FORM, 128, 64, 6>(p, s);
    case 6: return launch<T, TO, FORM, 128, 128, 4>(p, s);
    case 1: return launch<T, TO, FORM, 128, 64, 3>(p, s);
    default: return launch<T, TO, FORM, 128, 128, 2>(p, s);
    }
}

template <typename T> rtoss_status launch_form(ProductForm form, int tile, const Product& p, hipStream_t s)
{
    return form == kGated ? launch_tile<T, T, kGated>(tile, p, s) : form == kBackRows ? launch_tile<T, T, kBackRows>(tile, p, s)
                                                                                      : launch_tile<T, T, kBackWeights>(tile, p, s);
}
template <typename TO> rtoss_status launch_bits8(ProductForm form, int tile, const Product& p, hipStream_t s)
{
    return form == kScaled ? launch_tile<int8_t, TO, kScaled>(tile, p, s) : launch_tile<int8_t, TO, kGated>(tile, p, s);
}

}  // namespace

rtoss_status launch_product_mid(ProductForm form, bool bits8, rtoss_dtype out, int tile, const Product& p, hipStream_t s)
{
    switch (out) {
    case RTOSS_F32: return bits8 ? launch_bits8<float>(form, tile, p, s) : launch_form<float>(form, tile, p, s);
    case RTOSS_F16: return bits8 ? launch_bits8<f16_t>(form, tile, p, s) : launch_form<f16_t>(form, tile, p, s);
    default: return bits8 ? launch_bits8<bf16_t>(form, tile, p, s) : launch_form<bf16_t>(form, tile, p, s);
    }
}

}  // namespace rtoss
