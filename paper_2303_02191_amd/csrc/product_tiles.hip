// Products in tiles of 256 x 256, 256 x 128 and 128 x 128 results: the 8-bit product, the gated block and its gradients where there are rows
// enough.  Bound: the matrix instructions.
//
// A workgroup is eight waves, two per SIMD; of 256 x 256 results wave (wm, wn) of 2 x 4 owns 128 x 64 (128 accumulator registers), of
// 256 x 128 or 128 x 128 one of 4 x 2 owns 64 x 64 or 32 x 64.  The sum runs over stages of 128 bytes of a row, in buffers in LDS of regions of
// 16 KB: the halves of the left operand's rows, and one or two of the right one.  A stage is two parts (128 rows: one), in each of which a
// wave reads operands, of half of its rows, and multiplies them, with a barrier behind either.  The waves of the second four run half a
// part behind the first, so that on every SIMD one wave multiplies while the other reads.
//   - A wave holds the right operand of a stage for both parts, so that the first reads 8 + 8 vectors of 1 KB (256 x 128: 8 + 4) and the
//     second 8 (4), beside 64 (32) matrix instructions each.
//   - Two buffers: a stage's first part starts the copies of the second half of the rows for the next stage, the second those of all else for the
//     stage after that.  Every place has been read by both halves of the waves a barrier before; a region has a stage and a half to
//     arrive, and the wait in front of a part's barrier covers what the next part reads, whoever copied it.
//   - 128 rows: four buffers, copies three stages ahead.
// Behind the last stage the last one is copied again into free regions, so that every wait can count copies.
//
// Operands that memory holds by rows of the sum's direction (weights and rows of the forward pass) lie in LDS as rows of 128 bytes, those
// that it holds across (weights in the gradient of the rows; both in that of the weights) as 128 columns of each of the stage's
// rows, and are transposed by the read (ds_read_b64_tr_b16: lane 4k + j of 16 gives the address of four columns, lane i gets
// column i of the four rows that lanes 4k .. 4k+3 name, k = 0 .. 3).  Pieces of 16 bytes are exchanged within a row so that the reads spread
// over the banks.  Rows that are no whole pieces come through registers (product_words.h), in tiles of 128 channels.
//
// Measured: 8-bit 8192 x 8192 x 8192 403 us (2.73 POP/s; a library product 2.06; matrix instructions with reads of LDS and nothing else
// 3.3), gated block bf16 8192 rows x 4096 -> 10944 1040 us (1.41 PFLOP/s; a library product of 8192^3 1.5, instructions with reads 1.7), its
// gradients with dg and du 2420 us (1.21 PFLOP/s; library products of operands that lie across 1.17 and 1.03).  A tile costs 6 to 9 us besides
// its stages (its first copies, the output stage).  Workgroups that take several tiles and copy the next one's stages during the output
// stage: 3 % faster at 8192 rows, 10 to 19 % slower where every workgroup has one, for what it takes to find the copies' place.
#include <algorithm>

#include "product_run.h"
#include "product_tile.h"
#include "product_words.h"

namespace rtoss {

namespace {

constexpr int kRegion = 128 * kStage;       // 128 rows of an operand
constexpr int kGroupM = 4;                  // row tiles that neighbouring workgroups share

template <typename T, typename TO, int FORM, int TILE_M, int TILE_N, int ROWS>
__global__ __launch_bounds__(512, 2) void product_tiles_kernel(Product p, int tiles_m, int tiles_n, int tiles, int per_xcd)
{
    typedef typename AccOf<T>::type Acc;
    constexpr bool GATED = FORM == kGated;
    constexpr bool A_ACROSS = FORM == kBackWeights, B_ACROSS = FORM == kBackRows || FORM == kBackWeights;
    constexpr int EB = (int)sizeof(T), STAGE = kStage / EB;  // rows of the sum in a stage
    constexpr int COLS = GATED ? TILE_N / 2 : TILE_N;        // channels of a tile
    constexpr int WN = TILE_N / 64, WM = 8 / WN, MT = 8 / WM;  // waves across channels and rows; row tiles of a wave in half of the rows
    constexpr int HALVES = TILE_M / 128, B_REGIONS = TILE_N / 128, kBuffer = (HALVES + B_REGIONS) * kRegion;  // halves of A, then B
    constexpr int BUFFERS = HALVES == 2 ? 2 : 4;
    extern __shared__ __attribute__((aligned(16))) char smem[];  // stage s in buffer s % BUFFERS
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const bool late = wave >= 4;  // the second wave of a SIMD
    const int c = lane & 15, q = lane >> 4;

    const int work = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);
    if (work >= tiles) return;
    const int group = work / (kGroupM * tiles_n), at = work - group * (kGroupM * tiles_n);
    const int high = min(kGroupM, tiles_m - group * kGroupM);
    int tile_m = group * kGroupM + at % high;
    if constexpr (FORM == kBackWeights) {  // the second weight's tiles are behind the first's
        const int one = tiles_m / 2;
        if (tile_m >= one) {
            tile_m -= one;
            p.a0 = p.a1;
            p.y = p.y1;
        }
    }
    const int64_t m0 = (int64_t)tile_m * TILE_M;
    const int n0 = at / high * COLS;

    const int64_t lda = p.lda * EB, ldb = p.ldb * EB, row = (int64_t)p.R * EB;
    const int S1 = (int)(((int64_t)p.R + STAGE - 1) / STAGE), S = FORM == kBackRows ? 2 * S1 : S1;
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

    // ---- copies: a region is 16 instructions of 1 KB, two per wave.  By rows: 8 rows of 128 bytes, piece k of row r at place k ^ (r % 8).
    // A lane's channel is such that its results are neighbouring channels ----
    const int sub = lane >> 3, piece = (lane & 7) ^ sub;
    constexpr int PIECES = Across<T, 128>::kPieces, COPY_ROWS = Across<T, 128>::kCopyRows;
    struct Place {  // of a lane's pieces: two of each half of A, then two of B
        char* smem;
        int wave, lane;
        bool late;
        // a region's row of B -> channel of the tile (gated: runs of 8 channels a lane in 32 of a wave; otherwise of 16 in 64, of which a region
        // has half where there are two, the second 8 channels on)
        static __device__ __forceinline__ int channel(int rho)
        {
            const int r = rho & 15, tile = rho >> 4;
            if constexpr (GATED) return (tile * 16 & COLS - 1) / 32 * 32 + 8 * (r >> 2) + 4 * (tile & 1) + (r & 3);
            else if constexpr (B_REGIONS == 2) return (tile >> 1) * 64 + 16 * (r >> 2) + 4 * (tile & 1) + (r & 3);
            else return (tile >> 2) * 64 + 16 * (r >> 2) + 4 * (tile & 3) + (r & 3);
        }
        static __device__ __forceinline__ bool of_a(int i) { return i < 2 * HALVES; }
        __device__ __forceinline__ int row(int i, int lane) const
        {
            if (of_a(i) ? A_ACROSS : B_ACROSS) return (wave * 2 + i % 2) * COPY_ROWS + lane / PIECES;
            const int rho = wave * 16 + i % 2 * 8 + lane / 8;
            return of_a(i) ? i / 2 * 128 + rho : channel(rho);
        }
        static __device__ __forceinline__ int column(int i) { return of_a(i) ? i / 2 * 128 : 0; }
        __device__ __forceinline__ bool up(int i) const { return GATED && !of_a(i) && late; }
        __device__ __forceinline__ char* to(int i, int stage) const
        {
            const int spread = (of_a(i) ? A_ACROSS : B_ACROSS) ? Across<T, 128>::spread((wave * 2 + i % 2) * COPY_ROWS + lane / PIECES) : lane >> 3;
            return smem + stage % BUFFERS * kBuffer + i / 2 * kRegion + wave * 2048 + i % 2 * 1024 + (lane ^ spread) * 16;
        }
    };
    uint32_t va[2], vb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int rho = wave * 16 + i * 8 + sub;
        const int r_across = (wave * 2 + i) * COPY_ROWS + lane / PIECES, at_across = (lane % PIECES ^ Across<T, 128>::spread(r_across)) * 16;
        if constexpr (A_ACROSS) va[i] = (uint32_t)r_across * (uint32_t)lda + at_across;
        else va[i] = (uint32_t)rho * (uint32_t)lda + piece * 16;
        if constexpr (B_ACROSS) {
            vb[i] = (uint32_t)r_across * (uint32_t)ldb + at_across;
        } else {
            vb[i] = (uint32_t)Place::channel(rho) * (uint32_t)ldb + piece * 16;
        }
    }
    // kind: the halves of A, then the regions of B.  Gated with one region: w_gate's rows, then w_up's, which are the upper waves' to copy
    auto issue = [&](int stage, int kind) {
        char* to = smem + stage % BUFFERS * kBuffer + kind * kRegion + wave * 2048;
        int st = min(stage, S - 1);
        const bool second = FORM == kBackRows && st >= S1;  // uniform: the second pair of operands
        if (second) st -= S1;
        __amdgpu_buffer_rsrc_t from;
        if (kind < HALVES) {
            const int64_t k = A_ACROSS ? (int64_t)st * STAGE * lda : (int64_t)st * kStage;
            from = (second ? a1 : a0).at(k + kind * (A_ACROSS ? 128 * EB : 128 * lda));
        } else {
            const int64_t k = B_ACROSS ? (int64_t)st * STAGE * ldb : (int64_t)st * kStage;
            const bool other = GATED ? (B_REGIONS == 2 ? kind == HALVES + 1 : late) : second;
            from = (other ? b1 : b0).at(k + (kind - HALVES) * (GATED ? 0 : B_ACROSS ? 128 * EB : 8 * ldb));
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
        {
            const uint32_t offset = kind < HALVES ? va[i] : vb[i];
            if constexpr (B_ACROSS) copy16_bounded(from, offset, __builtin_amdgcn_readfirstlane(lds_offset(to + i * 1024)));
            else __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(to + i * 1024), 16, offset, 0, 0, 0);
        }
    };

    // ---- rows that are no whole pieces: through registers, a stage's pieces of a lane at once ----
    static_assert(ROWS == kWhole || B_REGIONS == 1, "the second region's channels");
    constexpr int PA = A_ACROSS ? PIECES : 8, PB = B_ACROSS ? PIECES : 8;
    const Place place{smem, wave, lane, late};
    StageInRegisters<T, FORM, ROWS == kWhole ? kWords : ROWS, 2 * HALVES + 2, 2 * HALVES, PA, PB, Place> in_registers(p, place, m0, n0, S1, lane);
    Acc acc[HALVES * MT][4];
#pragma unroll
    for (int i = 0; i < HALVES * MT * 4; ++i) acc[i >> 2][i & 3] = Acc{0, 0, 0, 0};
    u32x4 af[MT][2], bf[4][2];  // [tile][step]
    const int at0 = c * kStage + ((q ^ (c & 7)) * 16);  // by rows: place of piece q of row c; of piece 4 + q: the same with bit 6 flipped
    int at_a[MT], at_b[4 / B_REGIONS];
#pragma unroll
    for (int t = 0; t < MT; ++t) at_a[t] = A_ACROSS ? Across<T, 128>::address(wm * MT + t, c, q) : (wm * MT + t) * 16 * kStage + at0;
    // (two regions: two of the wave's tiles in each, at the same place)
    constexpr int PLACES = 4 / B_REGIONS;
#pragma unroll
    for (int t = 0; t < PLACES; ++t) {
        const int tile = GATED && B_REGIONS == 1 ? (t >> 1) * (COLS / 16) + wn * 2 + (t & 1) : wn * PLACES + t;
        at_b[t] = B_ACROSS ? Across<T, 128>::address(tile, c, q) : tile * 16 * kStage + at0;
    }
    auto read_a = [&](int buf, int half) {
        const char* base = smem + buf * kBuffer + half * kRegion;
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if constexpr (A_ACROSS) af[t][s] = Across<T, 128>::read(base + at_a[t] + s * (kRegion / 2));
                else af[t][s] = *(const u32x4*)(base + (at_a[t] ^ (s * 64)));
            }
    };
    auto read_b = [&](int buf) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const char* base = smem + buf * kBuffer + (HALVES + t / PLACES) * kRegion;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if constexpr (B_ACROSS) bf[t][s] = Across<T, 128>::read(base + at_b[t % PLACES] + s * (kRegion / 2));
                else bf[t][s] = *(const u32x4*)(base + (at_b[t % PLACES] ^ (s * 64)));
            }
        }
    };
    auto clear_past = [&](u32x4& f, int s) { keep_first<T>(f, rest - (4 * s + q) * (16 / EB)); };
    auto multiply = [&](int ma) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int u = 0; u < 4; ++u) acc[ma * MT + t][u] = Mma16<T>::mma(bf[u][s], af[t][s], acc[ma * MT + t][u]);
        __builtin_amdgcn_s_setprio(0);
    };
    auto meet = [&] {
        fence();
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        fence();
    };
    constexpr int BEHIND = HALVES == 2 ? 4 + 2 * B_REGIONS : 8;
    auto landed = [&] {  // vmcnt: the copies of all but the newest regions, two of A and those of B (one half: two stages'); lgkmcnt(0): operands
        fence();
        __builtin_amdgcn_s_waitcnt(ROWS == kWhole ? 0x0070 | BEHIND : 0xc07f);
    };
    auto issue_first = [&](int stage) {
#pragma unroll
        for (int r = 0; r < B_REGIONS; ++r) issue(stage, HALVES + r);
        issue(stage, 0);
    };
    if constexpr (ROWS == kWhole) {
        if constexpr (HALVES == 2) issue_first(0), issue(0, 1), issue_first(1);
        else issue_first(0), issue_first(1), issue_first(2);
    } else {
        if (S > 0) {  // (a sum of nothing has no memory behind its operands)
            in_registers.load(0);
            in_registers.store(0);
        }
        if (S > 1) in_registers.load(1);
    }
    landed();
    meet();
    if (late) meet();  // half of the waves are a part behind the others
    for (int s = 0; s < S; ++s) {
        const bool part = rest < STAGE && (s == S - 1 || (FORM == kBackRows && s == S1 - 1));  // uniform: the sum ends in this stage
        const int buf = s % BUFFERS;
        // (the buffer that is filled has been read: both groups of waves are past a barrier behind its last part)
        auto fill = [&] {
            if constexpr (ROWS == kWhole) {
                issue_first(s + (HALVES == 2 ? 2 : 3));
            } else if (s + 1 < S) {
                in_registers.store(s + 1);
                if (s + 2 < S) in_registers.load(s + 2);
            }
        };
        read_b(buf);
        read_a(buf, 0);
        if constexpr (HALVES == 1) fill();
        else if constexpr (ROWS == kWhole) issue(s + 1, 1);
        landed();
        meet();
        if (ROWS == kWhole && part) {
#pragma unroll
            for (int i = 0; i < 2 * MT; ++i) clear_past(af[i >> 1][i & 1], i & 1);
#pragma unroll
            for (int i = 0; i < 8; ++i) clear_past(bf[i >> 1][i & 1], i & 1);
        }
        multiply(0);
        meet();
        if constexpr (HALVES == 1) continue;

        read_a(buf, 1);
        fill();
        landed();
        meet();
        if (ROWS == kWhole && part) {
#pragma unroll
            for (int i = 0; i < 2 * MT; ++i) clear_past(af[i >> 1][i & 1], i & 1);
        }
        multiply(HALVES - 1);
        meet();
    }
    if (!late) meet();
    __builtin_amdgcn_s_waitcnt(0x0f70);  // the surplus copies have landed: LDS may be given away

    // ---- results: a lane holds 16 neighbouring channels (gated: 8 of each projection; across: four times 4) of eight rows ----
    constexpr int RUN = GATED ? 8 : B_ACROSS ? 4 : 16, RUNS = B_ACROSS ? 4 : 1;
#pragma unroll
    for (int u = 0; u < RUNS; ++u) {
        // (across: 16 columns a tile, of 128 in a region)
        const int column = B_REGIONS == 2 ? (u >> 1) * 128 + wn * 32 + (u & 1) * 16 : wn * 64 + u * 16;
        const int n = n0 + (GATED ? wn * 32 : B_ACROSS ? column : wn * 64) + RUN * q;
        if (n >= p.N) continue;
        typedef RunOutput<FORM, T, TO, RUN> Output;
        const Output out(p, n);
        auto row_of = [&](int i) { return m0 + i / MT * 128 + (wm * MT + i % MT) * 16 + c; };
        float next = Output::scale(p, row_of(0));
#pragma unroll
        for (int i = 0; i < HALVES * MT; ++i) {
            const float sa = next;
            if (i + 1 < HALVES * MT) next = Output::scale(p, row_of(i + 1));
            if (row_of(i) < p.M) {
                Acc first[RUN / 4], second[RUN / 4];
#pragma unroll
                for (int t = 0; t < RUN / 4; ++t) {
                    first[t] = acc[i][u + t];
                    second[t] = acc[i][GATED ? 2 + t : u + t];
                }
                out.store(p, row_of(i), sa, first, second);
            }
        }
    }
}

template <typename T, typename TO, int FORM, int TILE_M, int TILE_N, int ROWS> rtoss_status launch(const Product& p, hipStream_t s)
{
    constexpr int COLS = FORM == kGated ? TILE_N / 2 : TILE_N, LDS = TILE_M == 256 ? 2 * (2 + TILE_N / 128) * kRegion : 4 * 2 * kRegion;
    static LaunchOnce once;
    DeviceInfo dev;
    if (rtoss_status st = current_device(&dev)) return st;
    const auto kernel = product_tiles_kernel<T, TO, FORM, TILE_M, TILE_N, ROWS>;
    if (rtoss_status st = ensure_dynamic_lds((const void*)kernel, LDS, once, dev.device, "LDS of a product")) return st;
    const int tiles_m = (int)(((int64_t)p.M + TILE_M - 1) / TILE_M) * (FORM == kBackWeights ? 2 : 1), tiles_n = (p.N + COLS - 1) / COLS;
    const int64_t tiles = (int64_t)tiles_m * tiles_n;
    const int64_t per_xcd = (tiles + 7) / 8;
    kernel<<<(unsigned)(per_xcd * 8), 512, LDS, s>>>(p, tiles_m, tiles_n, (int)tiles, (int)per_xcd);
    return check_hip(hipGetLastError(), "product launch");
}

}  // namespace

bool product_pieces_ok(ProductForm form, const Product& p, int eb)
{
    const bool a_across = form == kBackWeights, b_across = a_across || form == kBackRows;
    // (a tile's rows and a stage's are 32-bit offsets from its first)
    const auto whole = [&](const void* q, int64_t ld) { return (uintptr_t)q % 16 == 0 && ld * eb % 16 == 0 && ld * eb <= 1 << 23; };
    if (!whole(p.a0, p.lda) || !whole(p.b0, p.ldb)) return false;
    if (form >= kBackRows && !whole(p.a1, p.lda)) return false;
    if ((form == kGated || form == kBackRows) && !whole(p.b1, p.ldb)) return false;
    // rows end with a whole piece; those of dg and du are padded to one
    return p.R > 0 && (b_across ? (int64_t)p.N * eb % 16 == 0 : (int64_t)p.R * eb % 16 == 0);
}

bool product_tiles_ok(bool bits8, rtoss_dtype out, const Product& p)
{
    return (bits8 || out != RTOSS_F32) && p.R > 0 && (((int64_t)p.M + 127) / 128) * (((int64_t)p.N + 63) / 64) <= kMaxGridGroups / 4;
}

namespace {
template <typename T, typename TO, int FORM, int ROWS> rtoss_status launch_rows(int tile, const Product& p, hipStream_t s)
{
    if constexpr (ROWS == kWhole)
        if (tile == 2) return launch<T, TO, FORM, 256, 256, ROWS>(p, s);
    return tile == 0 ? launch<T, TO, FORM, 128, 128, ROWS>(p, s) : launch<T, TO, FORM, 256, 128, ROWS>(p, s);
}
template <typename T, typename TO, int FORM> rtoss_status launch_tile(int tile, const Product& p, hipStream_t s)
{
    switch (product_rows((ProductForm)FORM, p, (int)sizeof(T))) {
    case kWhole: return launch_rows<T, TO, FORM, kWhole>(tile, p, s);
    case kWords: return launch_rows<T, TO, FORM, kWords>(tile, p, s);
    default: return launch_rows<T, TO, FORM, sizeof(T) == 4 ? kWords : kBytes>(tile, p, s);  // (elements of four bytes are words)
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

rtoss_status launch_product_tiles(ProductForm form, bool bits8, rtoss_dtype out, int tile, const Product& p, hipStream_t s)
{
    switch (out) {
    case RTOSS_F32: return launch_bits8<float>(form, tile, p, s);  // (8-bit operands: product_tiles_ok)
    case RTOSS_F16: return bits8 ? launch_bits8<f16_t>(form, tile, p, s) : launch_form<f16_t>(form, tile, p, s);
    default: return bits8 ? launch_bits8<bf16_t>(form, tile, p, s) : launch_form<bf16_t>(form, tile, p, s);
    }
}

}  // namespace rtoss
