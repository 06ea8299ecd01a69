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

// Softmax weights are rounded to fp16, as the second product takes them.  The reference that a row's scores are taken off is held kRoom powers of two below the largest
// score that it has followed, so that this one has the weight 2^kRoom, and it follows when a score would pass 2^(kRoom + kSlack), which is inside fp16.  What is left below
// is then fp16's range to 2^-14 and, with fewer bits, 2^-24: a weight vanishes at 2^-32 of the row's largest or below.  (With the largest at 1, at 2^-25: 131072 tokens
// of e^-17.8 times the first one's weight lost four fifths of their sum.)
constexpr float kSlack = 8.0f, kRoom = 7.0f;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// (sums that would pass 2^32 stay at its end: what the arrays on the device say is not trusted to be sound)
template <int CONTROL, int ROWS>
__device__ __forceinline__ unsigned add_from(unsigned v)
{
    return __builtin_elementwise_add_sat(v, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CONTROL, ROWS, 0xF, false)));
}

// Sum over the lanes up to and including this one: within the rows of 16 lanes by shifts, then the rows' sums handed on.
__device__ __forceinline__ unsigned running_sum(unsigned v)
{
    v = add_from<0x111, 0xF>(v);        // from the lane 1 before
    v = add_from<0x112, 0xF>(v);        // 2
    v = add_from<0x114, 0xF>(v);        // 4
    v = add_from<0x118, 0xF>(v);        // 8
    v = add_from<0x142, 0xA>(v);        // lane 15 of the row before, into the second and the fourth row
    return add_from<0x143, 0xC>(v);     // lane 31, into the third and the fourth
}

template <int CONTROL, int ROWS>
__device__ __forceinline__ unsigned most_from(unsigned v)
{
    return max(v, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CONTROL, ROWS, 0xF, false)));
}

// The largest of all lanes' numbers.
__device__ __forceinline__ unsigned largest(unsigned v)
{
    v = most_from<0x118, 0xF>(most_from<0x114, 0xF>(most_from<0x112, 0xF>(most_from<0x111, 0xF>(v))));
    return __builtin_amdgcn_readlane(static_cast<int>(most_from<0x143, 0xC>(most_from<0x142, 0xA>(v))), 63);
}

// Units dealt to the sequences in order, count(seq) to a sequence that load(b) has fetched (a struct of three ints): how many there are (0 if it is 2^31 or
// more, which no sound call has), and to which sequence a unit belongs and as the how manieth.  Lane l holds the l-th sequence, so that
// no load waits for another.  Called by whole wavefronts; sequences beyond the first 64 are fetched again by locate().
template <typename Seq, typename Load, typename Count>
struct Deal {
    int n_seqs, lane;
    Load load;
    Count count;
    Seq seq;
    unsigned own, upto, of_first, total;

    __device__ __forceinline__ Deal(int n_seqs_, int lane_, Load load_, Count count_) : n_seqs(n_seqs_), lane(lane_), load(load_), count(count_)
    {
        seq = load(min(lane, n_seqs - 1));
        recount();
    }

    // (again, where count() has changed)
    __device__ __forceinline__ void recount()
    {
        own = lane < n_seqs ? count(seq) : 0u;
        upto = running_sum(own);
        total = of_first = last(upto);
        for (int b0 = 64; b0 < n_seqs; b0 += 64)
            total = __builtin_elementwise_add_sat(total, last(running_sum(b0 + lane < n_seqs ? count(load(b0 + lane)) : 0u)));
        if (total > 0x7FFFFFFFu) total = 0;
    }

    __device__ static __forceinline__ unsigned last(unsigned v) { return __builtin_amdgcn_readlane(static_cast<int>(v), 63); }

    // unit < total
    __device__ __forceinline__ Seq locate(unsigned unit, int* b, int* within) const
    {
        unsigned before = 0, sum = upto, mine = own, all = of_first;
        Seq held = seq;
        int b0 = 0;
        while (unit >= before + all && b0 + 64 < n_seqs) {
            before += all;
            b0 += 64;
            held = load(min(b0 + lane, n_seqs - 1));
            mine = b0 + lane < n_seqs ? count(held) : 0u;
            sum = running_sum(mine);
            all = last(sum);
        }
        const int who = __builtin_ctzll(__builtin_amdgcn_ballot_w64(before + sum > unit));
        *b = b0 + who;
        *within = unit - before - __builtin_amdgcn_readlane(static_cast<int>(sum - mine), who);
        return {__builtin_amdgcn_readlane(held.start, who), __builtin_amdgcn_readlane(held.rows, who), __builtin_amdgcn_readlane(held.length, who)};
    }
};

template <typename Seq, typename Load, typename Count>
__device__ __forceinline__ Deal<Seq, Load, Count> deal_out(int n_seqs, int lane, Load load, Count count)
{
    return {n_seqs, lane, load, count};
}

}  // namespace
}  // namespace gqsa
