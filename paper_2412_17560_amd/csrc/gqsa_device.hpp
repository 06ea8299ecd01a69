// Device code that the kernels of gqsa_cache.hip and gqsa_prompt.hip share.  Included by .hip files only, after the HIP runtime.
#pragma once

#include "gqsa_attention.hpp"

namespace gqsa {
namespace {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef float float16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr float kMinusInf = -__builtin_inff();

// Sum over the lanes up to and including this one.
__device__ __forceinline__ int64_t running_sum(int64_t v, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t other = __shfl_up(v, d);
        if (lane >= d) v += other;
    }
    return v;
}

// Of units dealt to the sequences in order, count(b) to sequence b: the sequence that unit `unit` belongs to and the unit's number there;
// false if there are fewer units.  Called by whole wavefronts.
template <typename Count>
__device__ __forceinline__ bool locate(int n_seqs, int64_t unit, int lane, Count&& count, int* b, int64_t* within)
{
    int64_t before = 0;
    for (int b0 = 0; b0 < n_seqs; b0 += 64) {
        const int64_t mine = b0 + lane < n_seqs ? count(b0 + lane) : 0;
        const int64_t upto = running_sum(mine, lane);
        const unsigned long long past = __ballot(before + upto > unit);
        if (past) {
            const int who = __ffsll(past) - 1;
            *b = b0 + who;
            *within = unit - before - __shfl(upto - mine, who);
            return true;
        }
        before += __shfl(upto, 63);
    }
    return false;
}

template <typename Count>
__device__ __forceinline__ int64_t total_of(int n_seqs, int lane, Count&& count)
{
    int64_t sum = 0;
    for (int b = lane; b < n_seqs; b += 64) sum += count(b);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    return sum;
}

// Values that are not finite, where a mask hides some of them from some rows: a product with a weight of 0 would make them NaN for every row.  The
// product then takes `finite_part` and a second one counts, for each row and element, the +infinities, -infinities and NaN that the row sees.
__device__ __forceinline__ half8_t finite_part(half8_t v)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_fabsf16(v[i]) <= static_cast<_Float16>(65504.0f) ? v[i] : static_cast<_Float16>(0.0f);
    return v;
}

__device__ __forceinline__ half8_t not_finite(half8_t v)
{
    half8_t m;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        m[i] = static_cast<_Float16>(__builtin_fabsf16(v[i]) <= static_cast<_Float16>(65504.0f) ? 0.0f
                                     : v[i] != v[i] ? 16384.0f : v[i] > static_cast<_Float16>(0.0f) ? 1.0f : 128.0f);
    return m;
}

// What those counts (of at most 64 values) add to the row's sum.
__device__ __forceinline__ float from_counts(float count)
{
    const int n = static_cast<int>(count), up = n & 127, down = n >> 7 & 127;
    if (n >= 16384 || (up && down)) return __builtin_nanf("");
    return up ? __builtin_inff() : down ? -__builtin_inff() : 0.0f;
}

}  // namespace
}  // namespace gqsa
