// Products whose results are few tiles, and those in fp32: the sum split over the waves of a workgroup.
//
// A workgroup owns a tile of 16 x 16 to 64 x 64 results, and each of its eight waves all of them for every eighth stage of 128 bytes of the
// sum, through 4 to 16 KB of its own in LDS: no barrier before the sums are joined, and an operand is read from LDS once, where
// waves that share a stage would read it twice (waves of 32 x 32: 48 KB of LDS a stage, here 32).  Of the two waves of a SIMD one
// multiplies while the other waits for its copies.  Operands lie in LDS as in product_tiles.hip; rows that are no whole pieces come through
// registers (product_words.h).
//   - Both gradients in one launch, of workgroups of four waves, two on a CU.  Long sums of few tiles are shared by workgroups: fp32 31 rows
//     384 -> 3310 50 us without, 20 with.
//   - Of many tiles with short sums, and of fp32 in general, every wave has one of its own, and nothing is joined.
// Bound: weights' bytes where there are few rows (bf16 1 x 4096 -> 10944 twice 34 us, 5.2 TB/s; 8-bit 1 x 4096 x 4096 5.2 us, of which a launch
// is 3), otherwise the copies, 64 bytes a cycle and CU (8-bit 256 x 4096 x 4096 10 us); fp32: the splitting and six bf16 products (1024 ->
// 2752 of 512, 2048, 8192 rows, nothing kept, 45 to 53, 171, 543 us, 110 to 170 TFLOP/s; a library product of 8192^3 153).
#include <algorithm>

#include "fp32_split.h"
#include "product_run.h"
#include "product_tile.h"
#include "product_words.h"

namespace rtoss {

namespace {

// A long sum of few tiles is shared by `parts` workgroups: each leaves what it summed in memory, and the last of a tile's to arrive adds them, in their
// order.  What crosses XCDs is written and read by atomic operations of the device's scope, past the L2s, with a wait in front of the count; a fence
// of that scope would write back all of an L2.
__device__ __forceinline__ void put_part(f32x4* at, f32x4 v)
{
    typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
    const u64x2 halves = __builtin_bit_cast(u64x2, v);
    __hip_atomic_store((uint64_t*)at, halves[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store((uint64_t*)at + 1, halves[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x4 get_part(const f32x4* at)
{
    typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
    const u64x2 halves = {__hip_atomic_load((const uint64_t*)at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT),
                          __hip_atomic_load((const uint64_t*)at + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)};
    return __builtin_bit_cast(f32x4, halves);
}

// How the waves of a workgroup share the work: a tile, a part of a tile's sum, or a tile each.
enum Shared { kTile, kPart, kTileEach };

// `work` of tiles_m x tiles_n (x sum_parts.parts); kTileEach: the wave's
template <typename T, typename TO, int FORM, int ROWS, int BM, int BN, int WAVES, int SHARED>
__device__ __forceinline__ void product_slices(Product p, int work, int tiles_m, int tiles_n, SumParts sum_parts = {})
{
    constexpr bool PARTS = SHARED == kPart, EACH = SHARED == kTileEach;
    typedef typename AccOf<T>::type Acc;
    constexpr bool GATED = FORM == kGated;
    constexpr bool A_ACROSS = FORM == kBackWeights, B_ACROSS = FORM == kBackRows || FORM == kBackWeights;
    constexpr int EB = (int)sizeof(T), STAGE = kStage / EB;  // rows of the sum in a stage
    constexpr int COLS = GATED ? BN / 2 : BN;                // channels of a tile
    constexpr int MT = BM / 16, NT = BN / 16;                // 16 x 16 tiles
    constexpr int A_BYTES = BM * kStage, B_BYTES = BN * kStage, BUFFER = A_BYTES + B_BYTES;
    constexpr int A_COPIES = BM / 8, B_COPIES = BN / 8;      // instructions of a stage
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, q = lane >> 4;

    // in groups of eight row tiles, rows fastest: the workgroups that run on an XCD at a time share rows and channels in its L2
    const int part = PARTS ? work / (tiles_m * tiles_n) : 0;
    if constexpr (PARTS) work -= part * (tiles_m * tiles_n);
    constexpr int GROUP = 8;
    const int group = work / (GROUP * tiles_n), in_group = work - group * (GROUP * tiles_n);
    const int high = min(GROUP, tiles_m - group * GROUP);
    int tile_m = group * GROUP + in_group % high;
    const int n0 = in_group / high * COLS;
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
    const int S1 = (int)(((int64_t)p.R + STAGE - 1) / STAGE), S = FORM == kBackRows ? 2 * S1 : S1;
    const int rest = p.R - (S1 - 1) * STAGE;  // rows of the sum in the last stage
    const int begin = (PARTS ? (int)((int64_t)S * part / sum_parts.parts) : 0) + (EACH ? 0 : wave);
    const int end = PARTS ? (int)((int64_t)S * (part + 1) / sum_parts.parts) : S;
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

    // ---- copies; a lane's channel is such that its results are neighbouring channels (gated: those of four
    // neighbouring lanes are).  Gated: the second half of B's rows are w_up's ----
    typedef Across<T, 64> AcrossA, AcrossB;
    static_assert((!A_ACROSS || BM == 64) && (!B_ACROSS || BN == 64), "operands that lie across");
    const int sub = lane >> 3, piece = (lane & 7) ^ sub;
    uint32_t va[A_COPIES], vb[B_COPIES];
#pragma unroll
    for (int i = 0; i < A_COPIES; ++i) {
        const int k = i;  // copy instruction of the operand
        if constexpr (A_ACROSS) {
            const int r = k * AcrossA::kCopyRows + lane / AcrossA::kPieces;
            va[i] = (uint32_t)r * (uint32_t)lda + (lane % AcrossA::kPieces ^ AcrossA::spread(r)) * 16;
        } else {
            va[i] = (uint32_t)(k * 8 + sub) * (uint32_t)lda + piece * 16;
        }
    }
#pragma unroll
    for (int i = 0; i < B_COPIES; ++i) {
        const int k = i;
        if constexpr (B_ACROSS) {
            const int r = k * AcrossB::kCopyRows + lane / AcrossB::kPieces;
            vb[i] = (uint32_t)r * (uint32_t)ldb + (lane % AcrossB::kPieces ^ AcrossB::spread(r)) * 16;
        } else {
            const int rho = (k * 8 + sub) % COLS, t = rho / 16, r = rho & 15;
            vb[i] = (uint32_t)(GATED ? rho : 4 * NT * (r >> 2) + 4 * t + (r & 3)) * (uint32_t)ldb + piece * 16;
        }
    }
    char* const own = smem + wave * BUFFER;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_offset(smem)) + wave * BUFFER;
    struct From {
        __amdgpu_buffer_rsrc_t a, b, up;
    };
    auto source = [&](int stage) {
        int st = stage;
        const bool second = FORM == kBackRows && st >= S1;  // uniform: the second pair of operands
        if (second) st -= S1;
        const int64_t kb = B_ACROSS ? (int64_t)st * STAGE * ldb : (int64_t)st * kStage;
        From f;
        f.a = (second ? a1 : a0).at(A_ACROSS ? (int64_t)st * STAGE * lda : (int64_t)st * kStage);
        f.b = (second ? b1 : b0).at(kb);
        f.up = GATED ? b1.at(kb) : f.b;
        return f;
    };
    constexpr int PIECES = A_COPIES + B_COPIES, STEP = EACH ? 1 : WAVES;
    auto copy = [&](const From& f, uint32_t to, auto which) {
        constexpr int I = decltype(which)::value;
        if constexpr (I < A_COPIES) copy16_bounded(f.a, va[I], to + I * 1024);
        else copy16_bounded(GATED && I - A_COPIES >= B_COPIES / 2 ? f.up : f.b, vb[I - A_COPIES], to + A_BYTES + (I - A_COPIES) * 1024);
    };

    Acc acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT * NT; ++i) acc[i / NT][i % NT] = Acc{0, 0, 0, 0};
    // places of the wave's fragments in a buffer
    const int at0 = c * kStage + ((q ^ (c & 7)) * 16);
    int at_a[MT], at_b[NT];
#pragma unroll
    for (int t = 0; t < MT; ++t) at_a[t] = A_ACROSS ? AcrossA::address(t, c, q) : t * 16 * kStage + at0;
#pragma unroll
    for (int t = 0; t < NT; ++t) at_b[t] = A_BYTES + (B_ACROSS ? AcrossB::address(t, c, q) : t * 16 * kStage + at0);
    // ---- what the output stage reads, before the sum.  Wave w stores the units w, w + WAVES, ..: of a row tile, PART channel tiles (gated: one of
    // each projection); it reads ahead for the first
    constexpr int PART = NT == 1 ? 1 : 2, SHARE = NT / PART, UNITS = MT * SHARE;
    static_assert(!GATED || NT >= 2, "a wave's share of the results");
    // a lane's channels: 4 PART neighbouring ones; gated: 4 of each projection; across: 4 of each tile
    constexpr int RUN = GATED || B_ACROSS ? 4 : 4 * PART, RUNS = B_ACROSS ? PART : 1;
    auto row_of = [&](int unit) { return m0 + unit / SHARE * 16 + c; };
    auto channel_of = [&](int unit, int u) {
        const int share = unit % SHARE;
        return n0 + (B_ACROSS ? (PART * share + u) * 16 + 4 * q : GATED ? 16 * share + 4 * q : 4 * NT * q + 4 * PART * share);
    };
    typedef RunOutput<FORM, T, TO, RUN> Output;
    auto scale_of = [&](int unit) { return Output::scale(p, row_of(unit)); };
    const int first_unit = EACH ? 0 : wave;
    const Output first_out(p, min(channel_of(first_unit, 0), p.N - 1));  // (across: it holds nothing but the place)
    const float first_scale = scale_of(first_unit);

    // to `sum`; `plain`: fp32 by the fp32 instruction
    auto read_and_multiply = [&](const char* base, int s, Acc (&sum)[MT][NT], auto plain, auto&& then) {
        u32x4 af[2][MT], bf[2][NT];
        auto read_step = [&](int step) {
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                if constexpr (A_ACROSS) af[step][t] = AcrossA::read(base + at_a[t] + step * (A_BYTES / 2));
                else af[step][t] = *(const u32x4*)(base + (at_a[t] ^ (step * 64)));
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if constexpr (B_ACROSS) bf[step][t] = AcrossB::read(base + at_b[t] + step * (B_BYTES / 2));
                else bf[step][t] = *(const u32x4*)(base + (at_b[t] ^ (step * 64)));
            }
        };
        auto multiply_step = [&](int step) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < MT; ++i) sum[i][n] = Mma16<T>::mma(bf[step][n], af[step][i], sum[i][n]);
        };
        if constexpr (ROWS != kWhole && EB < 4) {  // (the next stage is in registers too: one step at a time)
#pragma unroll
            for (int step = 0; step < 2; ++step) {
                read_step(step);
                multiply_step(step);
                __builtin_amdgcn_sched_barrier(0);
            }
            return;
        }
        read_step(0);
        read_step(1);
        then();
        if (ROWS == kWhole && __builtin_expect(rest < STAGE && (s == S - 1 || (FORM == kBackRows && s == S1 - 1)), 0)) {  // uniform: the sum ends here
#pragma unroll
            for (int step = 0; step < 2; ++step) {
                const int valid = rest - (4 * step + q) * (16 / EB);
#pragma unroll
                for (int t = 0; t < MT; ++t) keep_first<T>(af[step][t], valid);
#pragma unroll
                for (int t = 0; t < NT; ++t) keep_first<T>(bf[step][t], valid);
            }
        }
        if constexpr (decltype(plain)::value) {
#pragma unroll
            for (int step = 0; step < 2; ++step) {  // of 16 products, four instructions of one of each q
                if (step && rest <= 16 && S1 == 1) break;  // uniform
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            sum[i][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, (uint32_t)bf[step][n][e]),
                                                                             __builtin_bit_cast(float, (uint32_t)af[step][i][e]), sum[i][n], 0, 0, 0);
            }
        } else if constexpr (sizeof(T) == 4) {
            // six products of bf16 parts (fp32_split.h), smallest first, all into one accumulator (more would not fit the registers beside another
            // stage).  2-norm of the gated block's error, K = 16, 512, 2048 and a wave for each tile: 0.7, 4.8, 9.9e-7, of library products in
            // fp32 1.1, 5.7, 11.5e-7; of sums split over eight waves, K = 1024, 2.3e-7 and 8.1e-7.
            Split8 bs[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) bs[n] = split8(bf[0][n], bf[1][n]);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const Split8 as = split8(af[0][i], af[1][i]);
                split_steps<kSplitSix>([&](auto k) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) split_step<decltype(k)::value>(bs[n], as, sum[i][n], sum[i][n]);
                });
            }
        } else {
            multiply_step(0);
            multiply_step(1);
        }
    };
    // fp32 sums of fewer than eight products take the fp32 instruction: what the six parts leave out is more than its roundings there.  2-norm of the
    // error and the largest in 2^-24 of the sum of magnitudes, K = 1, 2, 4, 8, 32:
    //     fp32 instruction  2.5e-8 (1.0)  3.1e-8 (1.9)  4.0e-8 (2.9)  5.4e-8 (3.8)  10.2e-8 (4.6)
    //     six parts         4.0e-8 (4.3)  4.0e-8 (4.4)  3.8e-8 (3.8)  4.0e-8 (3.0)   4.4e-8 (2.1)
    // Time: the same, but 43 us for 40 where every tile is one such sum (gradients of 2 rows, 990 -> 7682).
    // And a wave's sums are formed once more so if there is a NaN among them: an infinite operand's parts make a NaN of what may be infinite.  The NaN alone
    // are replaced, so that a result does not depend on other rows and channels.  Looking for them takes 0 to 4 % (all 0.4 us of 11 where a sum is one
    // stage); with a NaN in every tile 8192, 512 rows x 1024 -> 2752 take 1380, 97 us for 655, 45.
    const bool few = sizeof(T) == 4 && p.R * (FORM == kBackRows ? 2 : 1) < 8;  // uniform
    const int from = few ? end : begin;
    constexpr std::integral_constant<bool, sizeof(T) == 4> plain;
    auto by_fp32 = [&](auto&& run) {
        if constexpr (decltype(plain)::value) {
            Acc all = {0, 0, 0, 0};  // NaN where one of its terms is (infinities of both signs: looked for in vain)
#pragma unroll
            for (int i = 0; i < MT * NT; ++i) all += acc[i / NT][i % NT];
            if (__builtin_expect(!few && __ballot(__builtin_isnan(all[0] + all[1] + all[2] + all[3])) == 0, 1)) return;
            Acc sum[MT][NT];
#pragma unroll
            for (int i = 0; i < MT * NT; ++i) sum[i / NT][i % NT] = Acc{0, 0, 0, 0};
            run(sum);
#pragma unroll
            for (int i = 0; i < MT * NT * 4; ++i) {
                const float v = acc[i / 4 / NT][i / 4 % NT][i % 4];
                acc[i / 4 / NT][i / 4 % NT][i % 4] = few || __builtin_isnan(v) ? sum[i / 4 / NT][i / 4 % NT][i % 4] : v;
            }
        }
    };
    if constexpr (ROWS == kWhole) {
        auto issue = [&](int s) {
            const From f = source(s);
            static_for<PIECES>([&](auto k) { copy(f, lds0, k); });
        };
        auto landed = [] {
            fence();
            __builtin_amdgcn_s_waitcnt(0x0f70);  // the stage has landed
            fence();
        };
        auto read = [] {
            fence();
            __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): its place is free
            fence();
        };
        if (from < end) issue(from);
        for (int s = from; s < end; s += STEP) {
            landed();
            read_and_multiply(own, s, acc, std::false_type{}, [&] {
                read();
                if (s + STEP < end) issue(s + STEP);
                __builtin_amdgcn_sched_barrier(0);
            });
        }
        by_fp32([&](auto& sum) {
            for (int s = begin; s < end; s += STEP) {
                issue(s);
                landed();
                read_and_multiply(own, s, sum, plain, read);
            }
        });
    } else {
        // ---- through registers: a stage is loaded while the one before is multiplied.  (One wave's LDS instructions run in their order.) ----
        constexpr int PA = A_ACROSS ? AcrossA::kPieces : 8, PB = B_ACROSS ? AcrossB::kPieces : 8;
        struct Place {
            char* own;
            int lane;
            static __device__ __forceinline__ int row(int i, int lane)
            {
                const bool of_a = i < A_COPIES;
                const int k = of_a ? i : i - A_COPIES, r = of_a ? k * (64 / PA) + lane / PA : k * (64 / PB) + lane / PB;
                if (of_a || B_ACROSS) return r;
                const int in = r % COLS;
                return GATED ? in : 4 * NT * ((in & 15) >> 2) + 4 * (in / 16) + (in & 3);
            }
            static __device__ __forceinline__ int column(int) { return 0; }
            static __device__ __forceinline__ bool up(int i) { return GATED && i - A_COPIES >= B_COPIES / 2; }
            __device__ __forceinline__ char* to(int i, int) const
            {
                const int k = i < A_COPIES ? i : i - A_COPIES;
                const int spread = (i < A_COPIES ? A_ACROSS : B_ACROSS) ? AcrossA::spread(k * AcrossA::kCopyRows + lane / AcrossA::kPieces) : lane >> 3;
                return own + (i < A_COPIES ? 0 : A_BYTES) + k * 1024 + (lane ^ spread) * 16;
            }
        };
        const Place place{own, lane};
        typedef StageInRegisters<T, FORM, ROWS, PIECES, A_COPIES, PA, PB, Place> Stage;
        Stage in_registers(p, place, m0, n0, S1, lane);
        if (from < end) in_registers.load(from);
        for (int s = from; s < end; s += STEP) {
            in_registers.store(s);
            if (s + STEP < end) in_registers.load(s + STEP);
            fence();
            read_and_multiply(own, s, acc, std::false_type{}, [&] {});
            fence();
        }
        by_fp32([&](auto& sum) {
            // (nothing of it is kept through the loop above.  Without offsets of whole stages the gated block spills less there, 2048 x 333 -> 2801 122 us
            // with and 108 without; the gradients more, 512 x 1023 -> 2751 127 and 136)
            Stage stage(p, place, m0, n0, S1, Stage::unknown(lane), !GATED);
            for (int s = begin; s < end; s += STEP) {
                stage.load(s);
                stage.store(s);
                fence();
                read_and_multiply(own, s, sum, plain, [&] {});
                fence();
            }
        });
    }

    struct Sum {
        Acc of[PART];
    };
    auto finish = [&](int unit, const Output& out, float sa, const Sum& of) {
        const auto& sum = of.of;
        const int64_t m = row_of(unit);
        if (m >= p.M) return;
#pragma unroll
        for (int u = 0; u < RUNS; ++u) {
            const int n = channel_of(unit, u);
            if (n >= p.N) continue;
            if constexpr (B_ACROSS) {
                const Acc one[1] = {sum[u]};
                Output(p, n).store(p, m, sa, one, one);
            } else if constexpr (GATED) {
                const Acc first[1] = {sum[0]}, second[1] = {sum[PART - 1]};
                out.store(p, m, sa, first, second);
            } else {
                out.store(p, m, sa, sum, sum);
            }
        }
    };
    auto finish_next = [&](int unit, const Sum& sum) {
        finish(unit, Output(p, min(channel_of(unit, 0), p.N - 1)), scale_of(unit), sum);
    };
    if constexpr (EACH) {
        static_for<UNITS>([&](auto which) {
            constexpr int unit = which, share = unit % SHARE;
            Sum sum;
#pragma unroll
            for (int t = 0; t < PART; ++t) sum.of[t] = acc[unit / SHARE][GATED ? NT / 2 * t + share : PART * share + t];
            if constexpr (unit == 0) finish(unit, first_out, first_scale, sum);
            else finish_next(unit, sum);
        });
        return;
    }

    // ---- join ----
    __syncthreads();
    Acc* const joined = (Acc*)smem;  // [wave][row tile][channel tile][lane]
    static_assert(MT * NT * 1024 <= BUFFER, "the sums fit the waves' places");
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n) joined[((wave * MT + i) * NT + n) * 64 + lane] = acc[i][n];
    __syncthreads();
    auto sum_of = [&](int unit) {
        const int share = unit % SHARE;
        Sum sum;
#pragma unroll
        for (int t = 0; t < PART; ++t) {
            const Acc* from = joined + (unit / SHARE * NT + (GATED ? NT / 2 * t + share : PART * share + t)) * 64 + lane;
            sum.of[t] = from[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) sum.of[t] += from[w * MT * NT * 64];
        }
        return sum;
    };
    if constexpr (PARTS) {
        const int parts = sum_parts.parts;
        if (parts > 1) {
            Acc* const tile = (Acc*)sum_parts.sums + (int64_t)work * parts * (BM * BN / 4);  // [part][unit][its share][lane]
            auto at = [&](int of, int unit, int t) { return tile + of * (BM * BN / 4) + (unit * PART + t) * 64 + lane; };
            for (int unit = wave; unit < UNITS; unit += WAVES) {
                const Sum sum = sum_of(unit);
#pragma unroll
                for (int t = 0; t < PART; ++t) put_part(at(part, unit, t), sum.of[t]);
            }
            fence();
            __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): the wave's part is there
            fence();
            __syncthreads();
            uint32_t* const before = (uint32_t*)smem;
            if (tid == 0) *before = __hip_atomic_fetch_add(sum_parts.arrived + work, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __syncthreads();
            if (*before != (uint32_t)parts - 1) return;
            for (int unit = wave; unit < UNITS; unit += WAVES) {
                Sum sum{};
#pragma unroll 4
                for (int of = 0; of < parts; ++of)
#pragma unroll
                    for (int t = 0; t < PART; ++t) sum.of[t] += get_part(at(of, unit, t));
                finish_next(unit, sum);
            }
            return;
        }
    }
    if (wave < UNITS) finish(wave, first_out, first_scale, sum_of(wave));
    if constexpr (UNITS > WAVES)
        for (int unit = wave + WAVES; unit < UNITS; unit += WAVES) finish_next(unit, sum_of(unit));
}

template <typename T, typename TO, int FORM, int ROWS, int BM, int BN, int WAVES, bool EACH>
__global__ __launch_bounds__(64 * WAVES, 2) void product_slices_kernel(Product p, int tiles_m, int tiles_n, int tiles, int per_xcd)
{
    int work = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);  // (XCD-contiguous)
    if constexpr (EACH) work = work * WAVES + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (work < tiles) product_slices<T, TO, FORM, ROWS, BM, BN, WAVES, EACH ? kTileEach : kTile>(p, work, tiles_m, tiles_n);
}

// Both gradients in one launch (or one, by the same code): they share nothing but dg and du, and each alone leaves most of the chip without work.
// Every XCD has its share of the rows' tiles, whose sums are long, and behind them its share of the weights'.  ROWS_EACH, WEIGHTS_EACH: of these
// every wave has one.
template <typename T, int ROWS, int BM, int WAVES, bool ROWS_EACH, bool WEIGHTS_EACH>
__global__ __launch_bounds__(64 * WAVES, 2) void product_slices_back_kernel(Product rows, Product weights, int rows_m, int rows_n, int rows_per_xcd,
                                                                            int weights_m, int weights_n, int weights_per_xcd, SumParts row_parts,
                                                                            SumParts weight_parts)
{
    const int xcd = (int)(blockIdx.x % 8), at = (int)(blockIdx.x / 8), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (at < rows_per_xcd) {
        int work = xcd * rows_per_xcd + at;
        if constexpr (ROWS_EACH) work = work * WAVES + wave;
        if (work < rows_m * rows_n * row_parts.parts)
            product_slices<T, T, kBackRows, ROWS, BM, 64, WAVES, ROWS_EACH ? kTileEach : kPart>(rows, work, rows_m, rows_n, row_parts);
    } else {
        int work = xcd * weights_per_xcd + at - rows_per_xcd;
        if constexpr (WEIGHTS_EACH) work = work * WAVES + wave;
        if (work < weights_m * weights_n * weight_parts.parts)
            product_slices<T, T, kBackWeights, ROWS, 64, 64, WAVES, WEIGHTS_EACH ? kTileEach : kPart>(weights, work, weights_m, weights_n, weight_parts);
    }
}

template <typename T, typename TO, int FORM, int ROWS, int BM, int BN, bool EACH = false> rtoss_status launch(const Product& p, hipStream_t s)
{
    constexpr int WAVES = 8, COLS = FORM == kGated ? BN / 2 : BN, LDS = WAVES * (BM + BN) * kStage;
    static LaunchOnce once;
    DeviceInfo dev;
    if (rtoss_status st = current_device(&dev)) return st;
    const auto kernel = product_slices_kernel<T, TO, FORM, ROWS, BM, BN, WAVES, EACH>;
    if (rtoss_status st = ensure_dynamic_lds((const void*)kernel, LDS, once, dev.device, "LDS of a product")) return st;
    const int tiles_m = (int)(((int64_t)p.M + BM - 1) / BM) * (FORM == kBackWeights ? 2 : 1), tiles_n = (p.N + COLS - 1) / COLS;
    const int64_t tiles = (int64_t)tiles_m * tiles_n, per_xcd = ((EACH ? (tiles + WAVES - 1) / WAVES : tiles) + 7) / 8;
    kernel<<<(unsigned)(per_xcd * 8), 64 * WAVES, LDS, s>>>(p, tiles_m, tiles_n, (int)tiles, (int)per_xcd);
    return check_hip(hipGetLastError(), "product launch");
}

template <typename T, int ROWS, int BM, bool ROWS_EACH, bool WEIGHTS_EACH>
rtoss_status launch_back(const Product& rows, const Product& weights, SumParts row_parts, SumParts weight_parts, hipStream_t s)
{
    constexpr int WAVES = 4, LDS = WAVES * (64 + 64) * kStage;
    static LaunchOnce once;
    DeviceInfo dev;
    if (rtoss_status st = current_device(&dev)) return st;
    const auto kernel = product_slices_back_kernel<T, ROWS, BM, WAVES, ROWS_EACH, WEIGHTS_EACH>;
    if (rtoss_status st = ensure_dynamic_lds((const void*)kernel, LDS, once, dev.device, "LDS of a product")) return st;
    const auto up = [](int64_t n, int by) { return (int)((n + by - 1) / by); };  // (of no result: none)
    const int rows_m = rows.y ? up(rows.M, BM) : 0, rows_n = up(rows.N, 64), weights_m = weights.y ? 2 * up(weights.M, 64) : 0, weights_n = up(weights.N, 64);
    const auto per_xcd = [](int64_t tiles, bool each) { return ((each ? (tiles + WAVES - 1) / WAVES : tiles) + 7) / 8; };
    const int64_t rows_per_xcd = per_xcd((int64_t)rows_m * rows_n * row_parts.parts, ROWS_EACH);
    const int64_t weights_per_xcd = per_xcd((int64_t)weights_m * weights_n * weight_parts.parts, WEIGHTS_EACH);
    kernel<<<(unsigned)((rows_per_xcd + weights_per_xcd) * 8), 64 * WAVES, LDS, s>>>(rows, weights, rows_m, rows_n, (int)rows_per_xcd, weights_m, weights_n,
                                                                                       (int)weights_per_xcd, row_parts, weight_parts);
    return check_hip(hipGetLastError(), "product launch");
}

template <typename T, typename TO, int FORM, int ROWS> rtoss_status launch_tile(int tile, const Product& p, hipStream_t s)
{
    constexpr int G = FORM == kGated ? 2 : 1;  // (rows of both weights)
    if constexpr (FORM == kScaled || FORM == kGated) {
        switch (tile) {
        case 0: return launch<T, TO, FORM, ROWS, 16, 16 * G>(p, s);
        case 1: return launch<T, TO, FORM, ROWS, 32, 16 * G>(p, s);
        case 2: return launch<T, TO, FORM, ROWS, 32, 32 * G>(p, s);
        case 3: return launch<T, TO, FORM, ROWS, 64, 32>(p, s);
        }
    }
    if constexpr (sizeof(T) == 4 && FORM == kGated)
        if (tile == kSliceTiles) return launch<T, TO, FORM, ROWS, 64, 64, true>(p, s);
    return launch<T, TO, FORM, ROWS, 64, 64>(p, s);
}

template <typename T, typename TO, int FORM> rtoss_status launch_rows(int tile, const Product& p, hipStream_t s)
{
    switch (product_rows((ProductForm)FORM, p, (int)sizeof(T))) {
    case kWhole: return launch_tile<T, TO, FORM, kWhole>(tile, p, s);
    case kWords: return launch_tile<T, TO, FORM, kWords>(tile, p, s);
    default: return launch_tile<T, TO, FORM, sizeof(T) == 4 ? kWords : kBytes>(tile, p, s);  // (elements of four bytes are words)
    }
}

template <typename T> rtoss_status launch_form(ProductForm form, int tile, const Product& p, hipStream_t s)
{
    return form == kGated ? launch_rows<T, T, kGated>(tile, p, s) : form == kBackRows ? launch_rows<T, T, kBackRows>(tile, p, s)
                                                                                       : launch_rows<T, T, kBackWeights>(tile, p, s);
}
template <typename TO> rtoss_status launch_bits8(ProductForm form, int tile, const Product& p, hipStream_t s)
{
    return form == kScaled ? launch_rows<int8_t, TO, kScaled>(tile, p, s) : launch_rows<int8_t, TO, kGated>(tile, p, s);
}

}  // namespace

rtoss_status launch_product_slices(ProductForm form, bool bits8, rtoss_dtype out, int tile, const Product& p, hipStream_t s)
{
    switch (out) {
    case RTOSS_F32: return bits8 ? launch_bits8<float>(form, tile, p, s) : launch_form<float>(form, tile, p, s);
    case RTOSS_F16: return bits8 ? launch_bits8<f16_t>(form, tile, p, s) : launch_form<f16_t>(form, tile, p, s);
    default: return bits8 ? launch_bits8<bf16_t>(form, tile, p, s) : launch_form<bf16_t>(form, tile, p, s);
    }
}

namespace {
template <typename T>
rtoss_status launch_back_rows(bool high, const Product& rows, const Product& weights, SumParts row_parts, SumParts weight_parts, hipStream_t s)
{
    const auto tile = [&](auto mode) {
        constexpr int ROWS = decltype(mode)::value;
        const bool each = weight_parts.each;
        const auto go = high ? row_parts.each ? each ? launch_back<T, ROWS, 64, true, true> : launch_back<T, ROWS, 64, true, false>
                                              : each ? launch_back<T, ROWS, 64, false, true> : launch_back<T, ROWS, 64, false, false>
                             : each ? launch_back<T, ROWS, 16, false, true> : launch_back<T, ROWS, 16, false, false>;
        return go(rows, weights, row_parts, weight_parts, s);
    };
    switch (std::max(product_rows(kBackRows, rows, (int)sizeof(T)), product_rows(kBackWeights, weights, (int)sizeof(T)))) {
    case kWhole: return tile(std::integral_constant<int, kWhole>{});
    case kWords: return tile(std::integral_constant<int, kWords>{});
    default: return tile(std::integral_constant<int, sizeof(T) == 4 ? kWords : kBytes>{});
    }
}
}  // namespace

rtoss_status launch_product_slices_back(rtoss_dtype dt, bool high, const Product& rows, const Product& weights, SumParts row_parts, SumParts weight_parts,
                                        hipStream_t s)
{
    switch (dt) {
    case RTOSS_F32: return launch_back_rows<float>(high, rows, weights, row_parts, weight_parts, s);
    case RTOSS_F16: return launch_back_rows<f16_t>(high, rows, weights, row_parts, weight_parts, s);
    default: return launch_back_rows<bf16_t>(high, rows, weights, row_parts, weight_parts, s);
    }
}

}  // namespace rtoss
