// Device helpers shared by the kernels of the paged cache (gfx950): where a
// token's rows are, 8-bit rows, the sequence of a token.
#pragma once

#include <hip/hip_runtime.h>

#include "attention_tile.h"
#include "quan_sequence.h"

namespace quan {
namespace {

// Elements of a 16-byte chunk of a row.
constexpr int chunk_elems(CacheForm f) { return 16 / cache_elem_size(f); }

// Slot of a position on its page, and the page's first row of head 0; -1: the
// sequence has no such page.
struct Slot {
    int row, slot;
};
__device__ __forceinline__ Slot slot_of(const Cache &c, int seq, int position)
{
    const int page_at = fast_div(position, c.by_page);
    const int page = c.table[int64_t(seq) * c.table_pages + page_at];
    const int slot = position - page_at * c.page_tokens;
    return {page >= 0 && page < c.pages ? page * c.heads * c.page_tokens : -1, slot};
}

// A row's factor 2^e: the byte is e + 127 (255: infinity, which keeps a NaN one).
__device__ __forceinline__ float factor_of(unsigned byte)
{
    return __uint_as_float(byte << 23);
}
// The byte of a row whose largest magnitude has the bits `top`: the least e >=
// -117 with top <= 448 * 2^e = 1.75 * 2^(e + 8), so that nothing is beyond the
// largest 8-bit value and 2^-9, the least, times 2^e is no less than fp32's normal
// numbers; 255 for infinities and NaN.
__device__ __forceinline__ unsigned factor_byte(unsigned top)
{
    return top >= 0x7f800000u ? 255u : unsigned(max(int((top + 0x1fffffu) >> 23) - 8, 10));
}
// The byte of the largest finite rows: 256 times their factor is beyond fp32, so
// that their reals end at 240, the next lower value.
constexpr unsigned kLastByte = 247;
// 2^-e.
__device__ __forceinline__ float inverse_of(unsigned byte)
{
    return __uint_as_float((254u - byte) << 23);
}
typedef float f32x2 __attribute__((ext_vector_type(2)));
// 4 reals in 8 bits each, to nearest even (none is beyond 448).
__device__ __forceinline__ int to_e4m3(float a, float b, float c, float d)
{
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
__device__ __forceinline__ f32x4 from_e4m3(int v)
{
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(v, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(v, true);
    return f32x4{a[0], a[1], b[0], b[1]};
}

// 8 probabilities as bf16 numbers, and in their place what those leave, for a second
// such operand.  They are cut, not rounded, so that neither part is negative, and what
// is left has 2^-23 of the number added, so that it is not 0 either: an infinity of v
// times both is that infinity twice.  (Rounded, it was NaN where the rest was 0 or
// below.  The rest is under 2^-7 of the number's binade and rounded to 8 bits: off by
// 2^-16 of the number at most, twice what two rounded parts are off by.)
__device__ __forceinline__ bf16x8 cut(f32x8 &v)
{
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    u32x4 high;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const unsigned a = __float_as_uint(v[2 * e]), b = __float_as_uint(v[2 * e + 1]);
        high[e] = __builtin_amdgcn_perm(b, a, 0x07060302);
        v[2 * e] = fmaf(v[2 * e], 1.0f + 0x1p-23f, -__uint_as_float(a & 0xffff0000u));
        v[2 * e + 1] = fmaf(v[2 * e + 1], 1.0f + 0x1p-23f, -__uint_as_float(b & 0xffff0000u));
    }
    return __builtin_bit_cast(bf16x8, high);
}

// Tokens of a sequence: of image `img`, from `at` on.
struct Tokens {
    int img, at, len;
};
__device__ __forceinline__ Tokens tokens_of(const Sequences &s, const int32_t *first, int seq)
{
    if (first == nullptr)
        return {seq, 0, s.tokens};
    const int a = min(max(first[seq], 0), s.tokens), b = min(max(first[seq + 1], a), s.tokens);
    return {0, a, b - a};
}

}  // namespace
}  // namespace quan
