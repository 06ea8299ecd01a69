// What the attentions over the cache share (gqsa_cache_attend, gqsa_cache_attend_tree): codes as numbers, what a tree's row sees, and partial results that
// workgroups leave for each other.  Included by .hip files only, after the HIP runtime.
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

// One tile for one wavefront.  S^T = K Q^T and O^T = V^T P^T: a lane's scores are then the elements of the operand P^T that the second product wants
// from it, whatever the tokens' order, as the value codes lie in the same.
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

// Partial results, which workgroups on other XCDs read: stores and loads at the agent's scope (sc1), past the caches that are not coherent, by offsets
// in floats.  Nobody has read such a place before in the same launch, and a launch begins with empty caches.
struct Partials {
    __amdgpu_buffer_rsrc_t buffer;
    static constexpr int kAgent = 16;       // sc1

    __device__ __forceinline__ Partials(float* base, int floats) : buffer(__builtin_amdgcn_make_buffer_rsrc(base, 0, floats * 4, 0x00020000)) {}
    __device__ __forceinline__ void store4(int at, float4_t v) const
    {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), buffer, at * 4, 0, kAgent);
    }
    __device__ __forceinline__ void store2(int at, float a, float b) const
    {
        typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
        __builtin_amdgcn_raw_buffer_store_b64(u32x2_t{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)}, buffer, at * 4, 0, kAgent);
    }
    __device__ __forceinline__ float4_t load4(int at) const
    {
        return __builtin_bit_cast(float4_t, __builtin_amdgcn_raw_buffer_load_b128(buffer, at * 4, 0, kAgent));
    }
    __device__ __forceinline__ float2 load2(int at) const
    {
        typedef float float2_t __attribute__((ext_vector_type(2)));
        const float2_t v = __builtin_bit_cast(float2_t, __builtin_amdgcn_raw_buffer_load_b64(buffer, at * 4, 0, kAgent));
        return {v[0], v[1]};
    }
};

// (32 / 16 / 8, us: 131072 tokens, 8 heads for 64 45.3 / 42.7 / 42.0; 32768 tokens, 1 for 16 17.8 / 14.5 / 14.5; 4 x 20000 tokens, 4 rows, 8 for 64 40.8 / 41.3 / 44.5)
constexpr int kFan = 16;        // parts that one workgroup joins alone, unless they are themselves joined ones
constexpr int kMostParts = (kAttendWorkgroups + kFan - 1) / kFan;       // of which there are up to so many
static_assert(kMostParts >= kFan, "");

// Joins `parts` (up to kMostParts) partial results of `rows` rows in their order -- place(p): where part p lies -- and hands each four elements of a row to
// `sink`.  All loads are under way together (or kAhead parts' at a time), or each round of them would cost the latency of memory anew.
// Called by a whole workgroup; `scratch` is LDS for (2 kMostParts + 1) ROWS floats.
template <int D, int ROWS, int THREADS, typename Place, typename Sink>
__device__ __forceinline__ void join(const Partials& partials, int rows, int parts, float* scratch, Place place, Sink sink)
{
    constexpr int kSets = (ROWS * (D / 4) + THREADS - 1) / THREADS;      // fours of elements per thread
    constexpr int kAhead = 32 / kSets < kFan ? 32 / kSets : kFan;
    float4_t x[kAhead][kSets];
    const auto load = [&](int p0) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (p0 + j >= parts) break;
            const int from = place(p0 + j);
#pragma unroll
            for (int k = 0; k < kSets; ++k) x[j][k] = partials.load4(from + min(static_cast<int>(threadIdx.x) + k * THREADS, rows * (D / 4) - 1) * 4);
        }
    };
    load(0);
    float* weights = scratch;               // [part][row]: maximum, then weight
    float* sums = scratch + kMostParts * ROWS;
    float* tops = sums + kMostParts * ROWS;      // of all parts
    for (int i = threadIdx.x; i < parts * rows; i += THREADS) {
        const int part = i / rows, r = i - part * rows;
        const float2 top_sum = partials.load2(place(part) + ROWS * D + 2 * r);
        weights[part * ROWS + r] = top_sum.x, sums[part * ROWS + r] = top_sum.y;
    }
    __syncthreads();
    constexpr int kWeights = (kMostParts * ROWS + THREADS - 1) / THREADS;       // per thread
    float mine[kWeights];
#pragma unroll
    for (int k = 0; k < kWeights; ++k) {
        const int i = threadIdx.x + k * THREADS;
        if (i >= parts * rows) break;
        const int part = i / rows, r = i - part * rows;
        float top = kMinusInf;
        for (int q = 0; q < parts; ++q) top = fmaxf(top, weights[q * ROWS + r]);
        mine[k] = weight_of(weights[part * ROWS + r], top);
        if (part == 0) tops[r] = top;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kWeights; ++k) {
        const int i = threadIdx.x + k * THREADS;
        if (i >= parts * rows) break;
        const int part = i / rows, r = i - part * rows;
        weights[part * ROWS + r] = mine[k];
    }
    __syncthreads();
    float4_t v[kSets];
    float s[kSets];
#pragma unroll
    for (int k = 0; k < kSets; ++k) v[k] = float4_t{0.0f, 0.0f, 0.0f, 0.0f}, s[k] = 0.0f;
    for (int p0 = 0; p0 < parts; p0 += kAhead) {
        if (p0 > 0) load(p0);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (p0 + j >= parts) break;
#pragma unroll
            for (int k = 0; k < kSets; ++k) {
                const int r = min(static_cast<int>(threadIdx.x + k * THREADS) / (D / 4), rows - 1);
                const float w = weights[(p0 + j) * ROWS + r];
                s[k] += w * sums[(p0 + j) * ROWS + r];
                v[k] += w * x[j][k];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kSets; ++k) {
        const int of = threadIdx.x + k * THREADS;
        if (of < rows * (D / 4)) sink(of / (D / 4), 4 * (of % (D / 4)), v[k], tops[of / (D / 4)], s[k]);
    }
    __syncthreads();       // (`scratch` is free again)
}

}  // namespace
}  // namespace gqsa
