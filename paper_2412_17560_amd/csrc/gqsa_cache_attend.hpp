// What the attentions over the cache share (gqsa_cache_attend, gqsa_cache_attend_tree): codes as numbers, what a tree's row sees, and the weight of a part.  Included by
// .hip files only, after the HIP runtime.
#pragma once

#include "gqsa_cache.hpp"

namespace gqsa {
namespace {

// Eight codes as four pairs of fp16 numbers.  A byte 0000cccc is the fp8 (E4M3) number c 2^-9 -- subnormal up to 7, of the lowest exponent from 8 on -- so
// that the conversion from fp8 with a scale of 2^9 gives c, exactly, two at a time: seven instructions (with the code spliced into the low bits of
// 1024, which is then taken off, nine, three of them dearer).
__device__ __forceinline__ void decode(uint32_t x, half2_t (&q)[4])
{
    const uint32_t even = x & 0x0F0F0F0Fu, odd = x >> 4 & 0x0F0F0F0Fu;
    q[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(even, 512.0f, false);
    q[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(even, 512.0f, true);
    q[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(odd, 512.0f, false);
    q[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(odd, 512.0f, true);
}

__device__ __forceinline__ half8_t join(half2_t a, half2_t b, half2_t c, half2_t d)
{
    const half4_t ab = __builtin_shufflevector(a, b, 0, 1, 2, 3), cd = __builtin_shufflevector(c, d, 0, 1, 2, 3);
    return __builtin_shufflevector(ab, cd, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ half2_t as_half2(uint32_t v) { return __builtin_bit_cast(half2_t, v); }

// The same number, of which the compiler does not know that: what is computed from it stays where it is written, in a branch that is seldom taken,
// rather than ahead of the loop in registers that are not there.
__device__ __forceinline__ int opaque(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// Of a tree's row, which of the tile's 32 tokens it sees: those before all rows, and those of the rows that its mask names.  `from`: the row whose token is the
// tile's first (below 0: that many tokens before the rows); `left`: tokens from there to the sequence's end.
__device__ __forceinline__ uint32_t seen_of(const uint32_t* mask, int words, int from, int left)
{
    const int w = from >> 5, shift = from & 31;
    const uint32_t held[2] = {mask[min(max(w, 0), words - 1)], mask[min(max(w + 1, 0), words - 1)]};       // (no branches: the loads are under way together)
    const auto word = [&](int i) { return w + i < 0 ? ~0u : w + i < words ? held[i] : 0u; };
    const uint64_t both = uint64_t{word(1)} << 32 | word(0);
    return static_cast<uint32_t>(both >> shift) & (left >= 32 ? ~0u : (1u << max(left, 0)) - 1u);
}

__device__ __forceinline__ float weight_of(float top, float most) { return top == kMinusInf ? 0.0f : __builtin_amdgcn_exp2f(top - most); }

}  // namespace
}  // namespace gqsa
