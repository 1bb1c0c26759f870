// What the tiled products share: bounded copies into LDS and operands that lie across.
#pragma once
#include "products.h"

namespace rtoss {

constexpr int kStage = 128;  // bytes of a row in a stage

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

// The elements r .. r+E-1 of the sum that a lane holds of a fragment, of which `valid` exist: zeros for the others.
template <typename T> __device__ __forceinline__ void keep_first(u32x4& f, int valid)
{
    constexpr int E = 4 / (int)sizeof(T);  // of a word
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const int have = valid - d * E;
        const uint32_t mask = have >= E ? ~0u : have <= 0 ? 0u : (1u << (have * 8 * (int)sizeof(T) & 31)) - 1;
        f[d] &= mask;
    }
}

// Reads of an operand that lies across: [rows of the sum][COLUMNS].
template <typename T, int COLUMNS> struct Across {
    static_assert(COLUMNS == 64 || COLUMNS == 128, "rows of a stage");
    static constexpr int kRowBytes = COLUMNS * (int)sizeof(T);
    static constexpr int kPieces = kRowBytes / 16, kCopyRows = 64 / kPieces;  // pieces of a row, rows of a copy instruction
    static constexpr int kReads = sizeof(T) == 4 ? 4 : 2;   // per fragment
    // Piece k of row r lies at place k ^ spread(r): the rows 4 q (+ e) of an fp32 read, 8 q .. 8 q + 3 (+ 4) of a transposing one, spread over
    // the 64 banks (256 bytes).
    static __device__ __forceinline__ int spread(int r)
    {
        return sizeof(T) == 4 ? (r >> 2 & 3) << 2 : COLUMNS == 128 ? ((r & 3) | (r >> 1 & 4)) << 1 : ((r >> 1 & 1) | (r >> 2 & 2)) << 1;
    }
    // a lane's address of the fragment of columns 16 t .. 16 t + 15 in step 0
    static __device__ __forceinline__ int address(int t, int c, int q)
    {
        if constexpr (sizeof(T) == 4) return 4 * q * kRowBytes + ((4 * t ^ spread(4 * q)) * 16) + 4 * c;
        const int r = 8 * q + (c >> 2);
        return r * kRowBytes + ((2 * t ^ spread(r)) * 16) + (c & 3) * 8;
    }
    static __device__ __forceinline__ u32x4 read(const char* at)  // + step * (half a region)
    {
        u32x4 f;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = *(const uint32_t*)(at + e * kRowBytes);
        } else {
            typedef short s4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s4* Lds;
            const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at));
            const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + 4 * kRowBytes)));
            f = u32x4{lo.x, lo.y, hi.x, hi.y};
        }
        return f;
    }
};

// 16 bytes a lane from a bounded buffer to LDS, lane i to `to` + 16 i.  (Written out: in front of the transposing reads the compiler waits for
// all copies that it knows of.  Nothing is loaded into registers; every wait for these copies is written out too.)
__device__ __forceinline__ uint32_t lds_offset(const char* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }
__device__ __forceinline__ void copy16_bounded(__amdgpu_buffer_rsrc_t from, uint32_t offset, uint32_t to)  // (to: uniform)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(from) : "memory", "m0");
}

// How rows lie in memory, and a stage comes into LDS:
//   kWhole  pieces of 16 bytes start at multiples of 16 bytes: copies
//   kWords  ... at multiples of 4: through registers
//   kBytes  ... anywhere: through registers, with the word behind (a load of 16 bytes that is not aligned to a word takes 64 cycles instead of 16)
enum Rows { kWhole = 0, kWords, kBytes };

typedef uint32_t u32x4_words __attribute__((ext_vector_type(4), aligned(4)));  // on words

// kWhole, kWords or kBytes for operands of `eb`-byte elements.
inline Rows product_rows(ProductForm form, const Product& p, int eb)
{
    if (product_pieces_ok(form, p, eb)) return kWhole;
    const bool a1 = form == kBackRows || form == kBackWeights, b1 = form == kGated || form == kBackRows;
    const uintptr_t starts = (uintptr_t)p.a0 | (uintptr_t)p.b0 | (a1 ? (uintptr_t)p.a1 : 0) | (b1 ? (uintptr_t)p.b1 : 0);
    return (starts | (uintptr_t)(p.lda * eb) | (uintptr_t)(p.ldb * eb)) % 4 == 0 ? kWords : kBytes;
}

}  // namespace rtoss
