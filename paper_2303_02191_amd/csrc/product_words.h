// Stages of operands whose rows are no whole 16-byte pieces: through registers, loaded a stage before they are stored to LDS.
//
// Rows that do not begin on words (kBytes) are loaded in pieces of whole words and shifted on the way to LDS: a lane's last bytes are the first word
// of the lane beside it, and those of the last piece of a row come from a load of their own, one for eight instructions.  A fifth word loaded for
// every piece took as many registers as pieces (slices of 64 x 64 spilled) and twice the loads: 8-bit 512 x 4091 x 4096 57 us, 36 now.
#pragma once

#include "mma.h"
#include "product_tile.h"

namespace rtoss {

// A lane's COUNT pieces of a stage, the first A_COUNT of A.  Of an instruction's 64 lanes PA (A) or PB (B) have a row's pieces, the rows of one
// follow each other.  Place, of piece i of a lane:
//   row(i, lane)   its row of the tile; channel of the tile; row of the stage where the operand lies across
//   column(i)      there, the column of the tile that the instruction begins with
//   up(i)          it is w_up's
//   to(i, stage)   its place in LDS
template <typename T, int FORM, int ROWS, int COUNT, int A_COUNT, int PA, int PB, typename Place> struct StageInRegisters {
    static constexpr bool A_ACROSS = FORM == kBackWeights, B_ACROSS = FORM == kBackRows || FORM == kBackWeights;
    static constexpr int EB = (int)sizeof(T), E = 16 / EB, STAGE = kStage / EB;
    static constexpr int ENDS = ROWS == kBytes ? (COUNT + 7) / 8 : 0, KEPT = ENDS ? ENDS : 1;
    static_assert(ROWS == kWords || (ROWS == kBytes && EB < 4), "fp32 rows begin on words");

    const Product& p;
    const Place& place;
    const int64_t m0;
    const int n0, S1, lane;
    const int64_t lda = p.lda * EB, ldb = p.ldb * EB;
    // Where all pieces of a stage can be loaded whole, offsets from the tile that do not change, on a uniform base.  (Of rows further apart every
    // piece is found by itself.)
    const bool near;
    uint32_t at_piece[COUNT], at_end[KEPT];
    u32x4 piece_in[COUNT];
    uint32_t end_in[KEPT];

    static __device__ __forceinline__ bool is_a(int i) { return i < A_COUNT; }
    static __device__ __forceinline__ bool across(int i) { return is_a(i) ? A_ACROSS : B_ACROSS; }
    static __device__ __forceinline__ int pieces(int i) { return is_a(i) ? PA : PB; }
    __device__ __forceinline__ int64_t pitch(int i) const { return is_a(i) ? lda : ldb; }
    __device__ __forceinline__ int64_t columns(int i) const { return is_a(i) ? p.M - m0 : (int64_t)p.N - n0; }  // or rows, or channels
    __device__ __forceinline__ int in_pair(int stage) const { return FORM == kBackRows && stage >= S1 ? stage - S1 : stage; }
    __device__ __forceinline__ const char* base(int i, int stage) const  // of the tile
    {
        const bool second = FORM == kBackRows && stage >= S1;
        if (is_a(i)) return (const char*)(second ? p.a1 : p.a0) + m0 * (A_ACROSS ? EB : lda);
        return (const char*)(second || place.up(i) ? p.b1 : p.b0) + n0 * (B_ACROSS ? EB : ldb);
    }
    __device__ __forceinline__ const char* stage_base(int i, int stage) const
    {
        return base(i, stage) + in_pair(stage) * (across(i) ? STAGE * pitch(i) : (int64_t)kStage);
    }
    // Offset of a row of piece i and of a 16-byte piece in it.  Rows past the last are the last again.  Across, columns past the last are what
    // lies behind, in the row after, and those further off that again.
    __device__ __forceinline__ uint32_t near_row(int i, int lane) const
    {
        const int row = place.row(i, lane);
        return (uint32_t)(across(i) ? row : (int)min((int64_t)row, columns(i) - 1)) * (uint32_t)pitch(i);
    }
    __device__ __forceinline__ uint32_t near_piece(int i, int piece) const
    {
        if (!across(i)) return piece * 16;
        const int last = (int)min(columns(i), (int64_t)256) - 1;
        return min(place.column(i) / E + piece, last / E + (ROWS == kBytes)) * 16;
    }
    __device__ __forceinline__ bool inside(int stage) const  // uniform
    {
        constexpr int BEHIND = ROWS == kBytes ? 36 : 16;  // bytes that are loaded from a row's last piece on
        const int64_t end = (in_pair(stage) + 1) * (int64_t)STAGE;
        return near && (A_ACROSS || B_ACROSS ? end < p.R && (!A_ACROSS || lda >= BEHIND) && ldb >= BEHIND : end <= p.R);
    }
    static __device__ __forceinline__ int end_of(int j, int lane) { return min(8 * j + (lane & 7), COUNT - 1); }  // whose row's end a lane loads

    __device__ __forceinline__ StageInRegisters(const Product& p, const Place& place, int64_t m0, int n0, int S1, int lane, bool whole_stages = true)
        : p(p), place(place), m0(m0), n0(n0), S1(S1), lane(lane), near(whole_stages && lda <= 1 << 24 && ldb <= 1 << 24)
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) at_piece[i] = near_row(i, lane) + near_piece(i, lane % pieces(i));
#pragma unroll
        for (int j = 0; j < ENDS; ++j) {
            const int i = end_of(j, lane);
            at_end[j] = near_row(i, lane) + near_piece(i, pieces(i)) - 1;
        }
    }

    // Otherwise: words of a row that exists, from a piece on, those past its last being that one again; `have` elements of the piece exist
    struct Words {
        const uint32_t* at;
        int more;
        __device__ __forceinline__ uint32_t operator[](int w) const { return at[min(w, more)]; }
    };
    __device__ __forceinline__ Words words(int i, int lane, int piece, int stage, int& have) const
    {
        const int st = in_pair(stage);
        const int64_t row = across(i) ? (int64_t)st * STAGE + place.row(i, lane) : min((int64_t)place.row(i, lane), columns(i) - 1);
        const int64_t end = across(i) ? columns(i) : p.R, from = (across(i) ? place.column(i) : (int64_t)st * STAGE) + piece * E;
        have = across(i) && row >= p.R ? 0 : (int)min((int64_t)E, end - from);
        const uintptr_t at = (uintptr_t)base(i, stage) + (across(i) ? min(row, (int64_t)p.R - 1) : row) * pitch(i);
        const int64_t last = (end * EB + (int64_t)(at & 3) - 1) >> 2, first = min((from * EB) >> 2, last);
        return Words{(const uint32_t*)(at & ~(uintptr_t)3) + first, (int)min(last - first, (int64_t)4)};
    }
    // (nothing of it is worth a register in the loop)
    static __device__ __forceinline__ int unknown(int lane)
    {
        asm volatile("" : "+v"(lane));
        return lane;
    }

    __device__ __forceinline__ void load(int stage)
    {
        if (inside(stage)) {
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const char* at = stage_base(i, stage) + at_piece[i];
                if constexpr (ROWS == kBytes) at -= (uintptr_t)at & 3;
                piece_in[i] = *(const u32x4_words*)at;
            }
#pragma unroll
            for (int j = 0; j < ENDS; ++j) {
                const char* at = stage_base(end_of(j, lane), stage) + at_end[j];
                end_in[j] = *(const uint32_t*)(at - ((uintptr_t)at & 3));
            }
        } else {
            const int here = unknown(lane);
            int have;
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const Words from = words(i, here, here % pieces(i), stage, have);
#pragma unroll
                for (int w = 0; w < 4; ++w) piece_in[i][w] = from[w];
            }
#pragma unroll
            for (int j = 0; j < ENDS; ++j) {
                const int i = end_of(j, here);
                end_in[j] = words(i, here, pieces(i) - 1, stage, have)[4];
            }
        }
    }
    __device__ __forceinline__ void store(int stage)
    {
        const bool whole = inside(stage);
        static_for<COUNT>([&](auto which) {
            constexpr int i = which, P = i < A_COUNT ? PA : PB;
            u32x4 v = piece_in[i];
            if constexpr (ROWS == kBytes) {
                // (the rows of a lane are whole fours of rows apart, also the channels: it shifts all by as much)
                const uint32_t shift = (uint32_t)(uintptr_t)base(i, stage) + (uint32_t)(lane / P & 3) * (uint32_t)pitch(i);
                const uint32_t next = __builtin_amdgcn_update_dpp(0, v[0], 0x101, 0xf, 0xf, true);  // the next lane's
                uint32_t end = end_in[i / 8];  // of lane i % 8 of those with the row
                if constexpr (P - 1 != i % 8) end = __builtin_amdgcn_update_dpp(0, end, 0x110 + P - 1 - i % 8, 0xf, 0xf, true);
                const uint32_t behind = (lane & (P - 1)) == P - 1 ? end : next;
                v = u32x4{__builtin_amdgcn_alignbyte(v[1], v[0], shift), __builtin_amdgcn_alignbyte(v[2], v[1], shift),
                          __builtin_amdgcn_alignbyte(v[3], v[2], shift), __builtin_amdgcn_alignbyte(behind, v[3], shift)};
            }
            if (!whole) {  // words that do not exist: other ones, cut off here
                const int here = unknown(lane);
                int have;
                (void)words(i, here, here % P, stage, have);
                keep_first<T>(v, have);
            }
            *(u32x4*)place.to(i, stage) = v;
        });
    }
};

}  // namespace rtoss
