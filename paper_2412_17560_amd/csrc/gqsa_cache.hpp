// The paged cache of keys and values in 4 bits as its kernels see it: the order of a tile, where the tiles of a sequence lie, which rows of a call
// are which tokens, and the quantisation of a group.  Included by .hip files only, after the HIP runtime.
//
// 32 tokens of one head are a tile, laid out as the matrix cores take it, so that a wavefront's loads are whole runs of memory and
// a lane finds the 8 elements of its operand in one word (D = head_dim, l = lane, quad = l / 16):
//   keys     D / 16 words a lane; word j D / 32 + g: elements 32 g + 8 quad .. + 7 of token 16 j + l % 16;
//   values   D / 16 words a lane; word c: element 16 c + l % 16 of the tokens 4 quad .. + 3 and 16 + 4 quad .. + 3;
//            (words w of all lanes: byte (w / 4) 1024 + l 16 + (w % 4) 4 of the region)
//   key parameters    token by token, group by group: low, step;
//   value parameters  group by group, quad by quad: step of those 8 tokens, low of those 8 tokens.
// Code e of a word is at bits 8 (e % 4) + 4 (e / 4), so that one AND leaves four neighbouring ones in the bytes of a register.
#pragma once

#include <climits>

#include "gqsa_device.hpp"

namespace gqsa {
namespace {

constexpr int kThreads = 256;

__host__ __device__ constexpr int word_offset(int w, int lane) { return (w >> 2) * 1024 + lane * 16 + (w & 3) * 4; }
__host__ __device__ constexpr int nibble(int e) { return 8 * (e & 3) + 4 * (e >> 2); }
// The token of slot i of a word of value codes, and back.
__host__ __device__ constexpr int slot_token(int quad, int i) { return 4 * quad + (i & 3) + (i & 4) * 4; }

struct Pool {
    uint8_t* base;
    int64_t n_pages;
    int page_shift, kv_heads;      // log2 of a page's tokens

    template <int D>
    __device__ uint8_t* tile(int64_t page, int head, int tile_of_sequence) const
    {
        const int tiles = 1 << (page_shift - 5);
        return base + ((page * kv_heads + head) * tiles + (tile_of_sequence & (tiles - 1))) * int64_t{tile_bytes(D)};
    }
};

struct Sequence {
    int start, rows, length;       // its rows are start .. start + rows - 1, its tokens 0 .. length - 1, the last of them those of the rows
};

// (a length counts as at least 0 and at most `most`)
__device__ __forceinline__ Sequence sequence(const Sequences& s, int most, int b)
{
    const Rows rows = rows_between(s.row_starts ? s.row_starts[b] : b, s.row_starts ? s.row_starts[b + 1] : b + 1, s.n_rows);
    Sequence q;
    q.start = rows.start;
    q.rows = rows.count;
    q.length = min(max(s.lengths[b], 0), most);
    return q;
}

// What a sequence's pages hold, if they are all there.
__device__ __forceinline__ int most_tokens(const Sequences& s, int page_shift)
{
    return static_cast<int>(min(int64_t{s.max_pages} << page_shift, int64_t{INT_MAX - 4096}));
}

// --------------------------------------------------------------------------- into the cache and out of it
struct CopyArgs {
    Pool pool;
    Heads k, v;
    Sequences seqs;
};

// The tiles that the rows of a sequence lie in, from the first one's (which may be below 0) to the last one's (which may lie beyond the pages).
__device__ __forceinline__ int tiles_of_rows(const Sequence& q)
{
    return q.rows == 0 ? 0 : ((q.length - 1) >> 5) - ((q.length - q.rows) >> 5) + 1;
}

struct Unit {
    Sequence seq;
    int tile, head;
    int64_t page;       // -1: none
};

__device__ __forceinline__ bool unit_of(const CopyArgs& a, Unit* u)
{
    const auto deal = deal_out<Sequence>(a.seqs.n_seqs, threadIdx.x & 63, [&](int s) { return sequence(a.seqs, INT_MAX, s); },
                                         [](const Sequence& q) { return static_cast<unsigned>(tiles_of_rows(q)); });
    if (blockIdx.x >= deal.total) return false;
    int b, within;
    u->seq = deal.locate(blockIdx.x, &b, &within);
    u->tile = ((u->seq.length - u->seq.rows) >> 5) + within;
    u->head = blockIdx.y;
    u->page = -1;
    const int of = u->tile >> (a.pool.page_shift - 5);
    if (of >= 0 && of < a.seqs.max_pages) {        // (a row beyond the pages is left out, not written over the last token)
        const int page = a.seqs.pages[int64_t{b} * a.seqs.max_pages + of];
        if (page >= 0 && page < a.pool.n_pages) u->page = page;
    }
    return true;
}

template <int N>
struct Quantised {
    _Float16 low, step;
    uint32_t code[N];
};

// N elements of a group whose other elements are with the neighbouring 32 / N - 1 lanes.
template <int N>
__device__ __forceinline__ Quantised<N> quantise(const half8_t (&x)[N / 8])
{
    float low = __builtin_inff(), high = -__builtin_inff();
    int bad = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float v = static_cast<float>(x[i / 8][i % 8]);
        bad |= !(__builtin_fabsf(v) <= 65504.0f);
        low = fminf(low, v), high = fmaxf(high, v);
    }
#pragma unroll
    for (int d = 1; d < 32 / N; d *= 2) {
        low = fminf(low, __shfl_xor(low, d)), high = fmaxf(high, __shfl_xor(high, d));
        bad |= __shfl_xor(bad, d);
    }
    Quantised<N> q;
    q.low = bad ? static_cast<_Float16>(__builtin_nanf("")) : static_cast<_Float16>(low);
    uint16_t step_bits = __builtin_bit_cast(uint16_t, static_cast<_Float16>(bad ? 0.0f : (high - low) / 15.0f));
    // (what the largest code would stand for, rounded once as it is when it is read: a sum rounded to fp32 first reaches 65520, from where on fp16 is infinity, too soon)
    if (__builtin_fmaf16(static_cast<_Float16>(15.0f), __builtin_bit_cast(_Float16, step_bits), q.low) > static_cast<_Float16>(65504.0f)) --step_bits;
    q.step = __builtin_bit_cast(_Float16, step_bits);
    // (x - low) / step as one rounded division: with the rounded reciprocal, a product, its exact remainder and one correction.  The corrected
    // quotient is off by 2^-23 of its last place before it is rounded, and no quotient by a number of 11 bits lies that near to the middle
    // between two fp32 numbers, so the rounding is the division's.
    const float step = static_cast<float>(q.step), divisor = step > 0.0f ? step : 1.0f, inverse = 1.0f / divisor;
    const float highest = step > 0.0f ? 15.0f : 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float over = static_cast<float>(x[i / 8][i % 8]) - low, first = over * inverse;
        const float quotient = __builtin_fmaf(__builtin_fmaf(-first, divisor, over), inverse, first);
        q.code[i] = static_cast<uint32_t>(fmaxf(fminf(__builtin_rintf(quotient), highest), 0.0f));
    }
    return q;
}

inline gqsa_status_t on_device(const gqsa_cache* c)
{
    int dev = -1;
    GQSA_HIP(hipGetDevice(&dev));
    if (dev != c->device) return GQSA_ERR_HIP;
    return GQSA_OK;
}

inline Pool pool_of(const gqsa_cache* c)
{
    return {c->d_pages, c->n_pages, __builtin_ctz(static_cast<unsigned>(c->page_tokens)), c->kv_heads};
}

// Units of a copy: no more than a tile for every 32 rows and two more for every sequence.
inline dim3 copy_grid(const gqsa_cache* c, const Sequences& s)
{
    return dim3(static_cast<unsigned>(s.n_rows / kTileTokens + 2 * int64_t{s.n_seqs}), static_cast<unsigned>(c->kv_heads));
}

}  // namespace
}  // namespace gqsa
