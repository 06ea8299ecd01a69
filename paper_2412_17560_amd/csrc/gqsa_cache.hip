// A paged cache of keys and values in 4 bits (gqsa_cache_append, gqsa_cache_read) and the attention of the newest tokens over it
// (gqsa_cache_attend).
//
// 32 tokens of one head are a tile, laid out as the matrix cores take it, so that a wavefront's loads are whole runs of memory and
// a lane finds the 8 elements of its operand in one word (D = head_dim, l = lane, quad = l / 16):
//   keys     D / 16 words a lane; word j D / 32 + g: elements 32 g + 8 quad .. + 7 of token 16 j + l % 16;
//   values   D / 16 words a lane; word c: element 16 c + l % 16 of the tokens 4 quad .. + 3 and 16 + 4 quad .. + 3;
//            (words w of all lanes: byte (w / 4) 1024 + l 16 + (w % 4) 4 of the region)
//   key parameters    token by token, group by group: low, step;
//   value parameters  group by group, quad by quad: step of those 8 tokens, low of those 8 tokens.
// Code e of a word is at bits 8 (e % 4) + 4 (e / 4), so that one AND leaves four neighbouring ones in the bytes of a register.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>

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

// One workgroup per tile that gets rows, and head: 8 threads to a token.  The tile is put together in LDS -- a word of key codes is of one token, but one of
// value codes of 8 -- and written in runs of 16 bytes; of a tile that keeps earlier tokens, only the new ones' words and halves are
// written, and words of value codes that they share are read first (nobody else writes the tile).
// Few tokens are a chain of waits: lengths and starts, the page's number, the rows (asked for only when the page is known to be there, though they do not depend on it), then
// LDS, the bytes of a word of value codes one after the other, each waited for.  1 token of 16 sequences and 8 heads takes 5.1 us, where an empty launch takes 1.6.  Many
// are bound by that chain and by the arithmetic of 32 codes a thread: 8192 tokens of 8 heads of 128 take 15 to 16 us, 44 MB at 2.8 TB/s; their bytes alone would take 8.5.
template <int D>
__global__ __launch_bounds__(kThreads) void append_kernel(CopyArgs a)
{
    constexpr int kOwn = D / 8;                    // elements of a token per thread
    constexpr int kParameters = 32 * D;            // where the parameters start in a tile
    __shared__ alignas(16) uint8_t image[tile_bytes(D)];
    __shared__ alignas(16) uint8_t v_codes[kTileTokens][D + 4];
    Unit u;
    if (!unit_of(a, &u) || u.page < 0) return;
    uint8_t* tile = a.pool.tile<D>(u.page, u.head, u.tile);
    // of the tile's tokens, from .. to - 1 are new
    const int first = u.seq.length - u.seq.rows - u.tile * kTileTokens;       // the rows' first token
    const int from = max(first, 0), to = min(u.seq.length - u.tile * kTileTokens, kTileTokens);

    const int t = threadIdx.x >> 3, part = threadIdx.x & 7, group = part * kOwn / kGroupChannels;
    const bool leads = part % (kGroupChannels / kOwn) == 0, fresh = t >= from && t < to;
    const bool all = from == 0 && to == kTileTokens;
    constexpr int kWords = D / 16 * 64 / kThreads;      // words of value codes per thread
    uint32_t old[kWords] = {};
    if (!all) {
#pragma unroll
        // (Whether wanted or not, ahead of everything else, and with one store under one condition below.  Loaded only where a word is shared, in branches of three
        // ways with a store in two of them, the heads of 64 were compiled to a store whose 64-bit address had its upper half set on two of the ways only, and faulted.)
        for (int i = 0; i < kWords; ++i) {
            const int at = i * kThreads + threadIdx.x;
            old[i] = *reinterpret_cast<const uint32_t*>(tile + 16 * D + word_offset(at >> 6, at & 63));
        }
    }
    if (fresh) {
        const int64_t row = u.seq.start + (t - first);
        const uint16_t* k_at = a.k.data + row * a.k.row + u.head * a.k.head + part * kOwn;
        const uint16_t* v_at = a.v.data + row * a.v.row + u.head * a.v.head + part * kOwn;
        half8_t x[kOwn / 8], y[kOwn / 8];
#pragma unroll
        for (int i = 0; i < kOwn / 8; ++i) {
            x[i] = reinterpret_cast<const half8_t*>(k_at)[i];
            y[i] = reinterpret_cast<const half8_t*>(v_at)[i];
        }
        const Quantised<kOwn> k = quantise<kOwn>(x);
#pragma unroll
        for (int i = 0; i < kOwn / 8; ++i) {
            uint32_t word = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) word |= k.code[8 * i + e] << nibble(e);
            const int quad = (part * kOwn + 8 * i) % kGroupChannels / 8;
            *reinterpret_cast<uint32_t*>(image + word_offset((t >> 4) * (D / 32) + group, quad * 16 + (t & 15))) = word;
        }
        if (leads) *reinterpret_cast<half2_t*>(image + kParameters + (t * (D / 32) + group) * 4) = half2_t{k.low, k.step};
        const Quantised<kOwn> v = quantise<kOwn>(y);
#pragma unroll
        for (int i = 0; i < kOwn; i += 4)
            *reinterpret_cast<uint32_t*>(&v_codes[t][part * kOwn + i]) =
                v.code[i] | v.code[i + 1] << 8 | v.code[i + 2] << 16 | v.code[i + 3] << 24;
        if (leads) {
            const int quad = (t >> 2) & 3, slot = (t & 3) + (t >> 4) * 4;
            _Float16* at = reinterpret_cast<_Float16*>(image + kParameters + 4 * D + (group * 4 + quad) * 32) + slot;
            at[0] = v.step;
            at[8] = v.low;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        const int c = (i * kThreads + threadIdx.x) >> 6, l = threadIdx.x & 63, quad = l >> 4;
        uint32_t word = 0, kept = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int token = slot_token(quad, e);
            const bool is_new = token >= from && token < to;
            word |= (is_new ? uint32_t{v_codes[token][16 * c + (l & 15)]} : 0u) << nibble(e);
            kept |= (is_new ? 0u : 15u) << nibble(e);
        }
        const int at = 16 * D + word_offset(c, l);
        if (all) *reinterpret_cast<uint32_t*>(image + at) = word;
        else if (kept != ~0u) *reinterpret_cast<uint32_t*>(tile + at) = word | (old[i] & kept);
    }
    if (all) {
        __syncthreads();
        for (int i = threadIdx.x; i < tile_bytes(D) / 16; i += kThreads)
            reinterpret_cast<u32x4_t*>(tile)[i] = reinterpret_cast<const u32x4_t*>(image)[i];
    } else if (fresh) {
#pragma unroll
        for (int i = 0; i < kOwn / 8; ++i) {
            const int at = word_offset((t >> 4) * (D / 32) + group, (part * kOwn + 8 * i) % kGroupChannels / 8 * 16 + (t & 15));
            *reinterpret_cast<uint32_t*>(tile + at) = *reinterpret_cast<const uint32_t*>(image + at);
        }
        if (leads) {
            const int k_at = kParameters + (t * (D / 32) + group) * 4;
            const int v_at = kParameters + 4 * D + (group * 4 + ((t >> 2) & 3)) * 32 + 2 * ((t & 3) + (t >> 4) * 4);
            *reinterpret_cast<uint32_t*>(tile + k_at) = *reinterpret_cast<const uint32_t*>(image + k_at);
            *reinterpret_cast<uint16_t*>(tile + v_at) = *reinterpret_cast<const uint16_t*>(image + v_at);
            *reinterpret_cast<uint16_t*>(tile + v_at + 16) = *reinterpret_cast<const uint16_t*>(image + v_at + 16);
        }
    }
}

// The same deal.  A tile comes into LDS in runs of 16 bytes, as the codes of a token are spread over words of other tokens; bound by the same chain: 8192 tokens of
// 8 heads of 128 take 11 to 12 us (3.8 TB/s), 1 of 16 sequences and 8 heads 3.3.
template <int D>
__global__ __launch_bounds__(kThreads) void read_kernel(CopyArgs a)
{
    constexpr int kOwn = D / 8;
    constexpr int kParameters = 32 * D;
    __shared__ alignas(16) uint8_t image[tile_bytes(D)];
    Unit u;
    if (!unit_of(a, &u)) return;
    if (u.page >= 0) {
        const uint8_t* tile = a.pool.tile<D>(u.page, u.head, u.tile);
        for (int i = threadIdx.x; i < tile_bytes(D) / 16; i += kThreads)
            reinterpret_cast<u32x4_t*>(image)[i] = reinterpret_cast<const u32x4_t*>(tile)[i];
    }
    __syncthreads();
    const int first = u.seq.length - u.seq.rows;
    const int t = threadIdx.x >> 3, part = threadIdx.x & 7;
    const int token = u.tile * kTileTokens + t;
    if (token < first || token >= u.seq.length) return;
    half8_t x[kOwn / 8] = {}, y[kOwn / 8] = {};
    if (u.page >= 0) {
        const int group = part * kOwn / kGroupChannels, quad = (t >> 2) & 3, slot = (t & 3) + (t >> 4) * 4;
        const half2_t k = *reinterpret_cast<const half2_t*>(image + kParameters + (t * (D / 32) + group) * 4);
        const _Float16* v = reinterpret_cast<const _Float16*>(image + kParameters + 4 * D + (group * 4 + quad) * 32) + slot;
        const _Float16 v_step = v[0], v_low = v[8];
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int element = part * kOwn + i;
            const uint32_t kw = *reinterpret_cast<const uint32_t*>(
                image + word_offset((t >> 4) * (D / 32) + group, element % kGroupChannels / 8 * 16 + (t & 15)));
            const uint32_t vw = *reinterpret_cast<const uint32_t*>(image + 16 * D + word_offset(element / 16, quad * 16 + element % 16));
            x[i / 8][i % 8] = __builtin_fmaf16(static_cast<_Float16>(static_cast<float>(kw >> nibble(i % 8) & 15u)), k[1], k[0]);
            y[i / 8][i % 8] = __builtin_fmaf16(static_cast<_Float16>(static_cast<float>(vw >> (8 * (slot & 3) + 4 * (slot >> 2)) & 15u)), v_step, v_low);
        }
    }
    const int64_t row = u.seq.start + (token - first);
    uint16_t* k_at = a.k.data + row * a.k.row + u.head * a.k.head + part * kOwn;
    uint16_t* v_at = a.v.data + row * a.v.row + u.head * a.v.head + part * kOwn;
#pragma unroll
    for (int i = 0; i < kOwn / 8; ++i) {
        reinterpret_cast<half8_t*>(k_at)[i] = x[i];
        reinterpret_cast<half8_t*>(v_at)[i] = y[i];
    }
}

// --------------------------------------------------------------------------- attention over the cache
struct AttendArgs {
    Pool pool;
    Heads q, out;
    Sequences seqs;
    float* partials;
    int32_t* arrivals;
    int heads_per_group;
    float scale_log2;       // |scale| times log2(e): the softmax is taken to base 2
    bool negate;            // the queries, as scale is negative: the largest score is then the one of the largest product
};

// A tile as it is loaded: codes of keys and of values, parameters (16 bytes a lane with D = 128, 8 with D = 64).
template <int D>
struct Raw {
    typedef uint32_t words_t __attribute__((ext_vector_type(D / 32)));
    u32x4_t k[D / 64], v[D / 64];
    words_t parameters;
    int first_token;        // -1: no tile
};

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

// Between a wavefront's writes to its own part of LDS and its reads of other lanes' words: LDS takes a wavefront's operations in order, so
// only the compiler has to keep it.
__device__ __forceinline__ void wave_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// What one wavefront knows of its 16 query rows: lane l holds row l % 16; of the sums over the tokens, the tokens of its quad.
template <int D>
struct RowState {
    float top;                  // the scores' reference (times scale_log2)
    float sum;                  // of the quad's tokens
    float4_t out[D / 16];       // elements 16 c + 4 quad + r of row l % 16
};

// Of a lane's words of a tile's parameters, clears those of the tokens from `left` on, so that they stand for zero.
template <int D>
__device__ __forceinline__ void hide(typename Raw<D>::words_t& parameters, int lane, int left)
{
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        const int at = (lane * (D / 32) + i) * 4;
        if (at < 4 * D) {
            if (at / (D / 8) >= left) parameters[i] = 0;
        } else {
            const int o = at - 4 * D, t = slot_token((o >> 5) & 3, (o & 15) >> 1);
            if (t >= left) parameters[i] = 0;
            else if (t + 1 >= left) parameters[i] &= 0xFFFFu;
        }
    }
}

// The same number, of which the compiler does not know that: what is computed from it stays where it is written, in a branch that is seldom taken,
// rather than ahead of the loop in registers that are not there.
__device__ __forceinline__ int opaque(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// One tile for one wavefront.  S^T = K Q^T and O^T = V^T P^T: a lane's scores are then the elements of the operand P^T that the second product wants
// from it, whatever the tokens' order, as the value codes lie in the same.
template <int D, bool EDGE>
__device__ __forceinline__ void attend_tile(const Raw<D>& raw, uint32_t* stage, const half8_t (&q)[D / 32], RowState<D>& state, int lane,
                                            int length, int limit, float scale_log2)
{
    const int first_token = raw.first_token;
    typedef typename Raw<D>::words_t words_t;
    const int quad = lane >> 4;
    words_t parameters = raw.parameters;
    if constexpr (EDGE) hide<D>(parameters, opaque(lane), length - first_token);      // (older codes, NaN)
    wave_lds_order();
    reinterpret_cast<words_t*>(stage)[lane] = parameters;
    wave_lds_order();
    // Where rows differ in what they see of the tile, a value that is NaN (others are finite) would reach the rows that do not see it.  Such
    // groups of values stand for zero in the products; which tokens they are of, nan_of says.
    uint32_t nan_of[D / 32];
    bool wild = false;
    if constexpr (EDGE) {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) odd |= ((parameters[i] & 0x7C007C00u) + 0x04000400u & 0x80008000u) != 0;
        wild = __any(odd);
        if (wild) {
            const int t = opaque(lane) & 31, slot = (t & 3) + (t >> 4) * 4;
#pragma unroll
            for (int g = 0; g < D / 32; ++g) {
                const half2_t low = as_half2(stage[D + (g * 4 + (t >> 2 & 3)) * 8 + 4 + (slot >> 1)]);
                const _Float16 v = low[slot & 1];
                nan_of[g] = static_cast<uint32_t>(__builtin_amdgcn_ballot_w64(v != v));
            }
            if (opaque(lane) >= 32) {
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const half2_t h = as_half2(parameters[i]);
                    parameters[i] &= (h[0] == h[0] ? 0xFFFFu : 0u) | (h[1] == h[1] ? 0xFFFF0000u : 0u);
                }
            }
            wave_lds_order();
            reinterpret_cast<words_t*>(stage)[lane] = parameters;
            wave_lds_order();
        }
    }

    float4_t s[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        s[j] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
        const words_t p = *reinterpret_cast<const words_t*>(stage + (16 * j + (lane & 15)) * (D / 32));
#pragma unroll
        for (int g = 0; g < D / 32; ++g) {
            const int w = j * (D / 32) + g;
            const half2_t both = as_half2(p[g]);
            const half2_t low = {both[0], both[0]}, step = {both[1], both[1]};
            half2_t c[4];
            decode(raw.k[w >> 2][w & 3], c);
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = __builtin_elementwise_fma(c[i], step, low);
            s[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(join(c[0], c[1], c[2], c[3]), q[g], s[j], 0, 0, 0);
        }
    }
    half8_t value[D / 16];         // (ahead of the softmax, whose chain of waits this fills)
#pragma unroll
    for (int g = 0; g < D / 32; ++g) {
        const u32x4_t* at = reinterpret_cast<const u32x4_t*>(stage + D + (g * 4 + quad) * 8);
        const u32x4_t step = at[0], low = at[1];               // of the quad's tokens
#pragma unroll
        for (int c = 2 * g; c < 2 * g + 2; ++c) {
            half2_t v[4];
            decode(raw.v[c >> 2][c & 3], v);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __builtin_elementwise_fma(v[i], as_half2(step[i]), as_half2(low[i]));
            value[c] = join(v[0], v[1], v[2], v[3]);
        }
    }
    if constexpr (EDGE) {
        const int left = limit - first_token - 4 * opaque(quad);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (slot_token(0, i) >= left) s[i >> 2][i & 3] = kMinusInf;
    }
    float most = kMinusInf;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, s[i >> 2][i & 3]);
    most *= scale_log2;
    // (the reference follows only where a score lies far above it)
    if (__any(most > state.top + (kRoom + kSlack) || (state.top == kMinusInf && most > kMinusInf))) {
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        const float top = fmaxf(state.top, most - kRoom);
        const float shrink = top == kMinusInf ? 1.0f : __builtin_amdgcn_exp2f(state.top - top);
        state.top = top;
        state.sum *= shrink;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) state.out[c] *= shrink;
    }
    const float reference = state.top == kMinusInf ? 0.0f : state.top;
    half8_t p;
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = static_cast<_Float16>(__builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 2][i & 3], scale_log2, -reference)));
    // (the sum of the weights as the product has them, rounded: half the additions)
    const half2_t ones = {static_cast<_Float16>(1.0f), static_cast<_Float16>(1.0f)};
#pragma unroll
    for (int i = 0; i < 4; ++i) state.sum = __builtin_amdgcn_fdot2(half2_t{p[2 * i], p[2 * i + 1]}, ones, state.sum, false);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) state.out[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(value[c], p, state.out[c], 0, 0, 0);
    if (EDGE && wild) {
        const int left = limit - first_token;
        const uint32_t sees = left >= 32 ? ~0u : (1u << max(left, 0)) - 1u;
#pragma unroll
        for (int g = 0; g < D / 32; ++g)
            if (nan_of[g] & sees) state.out[2 * g] = state.out[2 * g + 1] = __builtin_nanf("") + float4_t{};
    }
}

__device__ __forceinline__ float weight_of(float top, float most) { return top == kMinusInf ? 0.0f : __builtin_amdgcn_exp2f(top - most); }

template <int D, int WAVES>
struct alignas(16) AttendShared {
    uint32_t stage[WAVES][2 * D];
    float out[WAVES][kRowBlock][D + 4];       // (+ 4: rows start in different banks)
    float top[WAVES][kRowBlock], sum[WAVES][kRowBlock];
    int last;
};

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

constexpr int kHeld = 2;             // tiles that a wavefront holds: the one at work, and those under way
constexpr int kAttendWaves = 4;      // wavefronts of a workgroup; a step: one tile for each

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

__device__ __forceinline__ int steps_of(const Sequence& q, int step_tiles)
{
    return max(static_cast<int>(static_cast<unsigned>(q.length + step_tiles * kTileTokens - 1) / static_cast<unsigned>(step_tiles * kTileTokens)), 1);
}

// Of 0 / 1 / 2 / 4 / 8 steps a workgroup, us: 143 tokens of 32 heads 7.4 / 6.45 / 6.45 / 6.4 / 6.4; 8 x 3000 tokens, 4 rows, 2 for 14 of 64 11.7 / 11.8 / 9.9 / 10.0 / 10.0;
// 32768 tokens, 1 for 16 16.0 / 14.3 / 14.5 / 14.4 / 14.4; 131072, 8 for 64 44.2 / 43.6 / 42.7 / 43.8 / 43.8; 64 sequences of up to 40 tokens, 8 for 32 6.9 / 7.1 / 7.1 / 7.2 / 7.2.
constexpr unsigned kFewSteps = 2;

// The work is dealt by steps of 128 or 256 tokens, not by sequences or heads: of all steps, in the order sequence, head, block of 16 rows, token, every
// workgroup takes a run, all of one length or one more.  Where a segment (one block of rows of one head) lies in several workgroups, each
// leaves its maximum, sum and weighted sum in the workspace, and the last to arrive joins them in the order of the tokens.
//
// One row for a head of the cache is bound by memory: 16 x 4096 tokens of 32 heads of 128, 336 MB, take 62 to 66 us, 5.1 to 5.4 TB/s; the same with all tiles in the L2 caches
// 49 us, as the vector instructions (88 of them turn a tile's 1024 words of keys into numbers, 88 the values; a softmax of 16 x 32 scores 60; 16 products) are issued in
// half of the cycles.  Several rows for a head hide nothing more: up to 16 cost what one costs, and every further 16 the reading and the instructions anew: 8 ragged sequences of up to
// 16003 tokens, 5 rows of 32 heads for 8, take 35.5 us.  Their 80 MB are read twice, 31 us at the rate of a copy, and decoded twice, 43 % of the cycles.  (Two blocks of rows under one decoding,
// with queries in LDS: 38 us here, 29.5 instead of 35.9 for 32 sequences of 2000 tokens and 3 rows, but 23.7 instead of 14.8 for 1 head for 32 over 32768 tokens, where the
// joins' work doubles.  Workgroups of both blocks beside each other on one XCD: 36.7.)
// A single short sequence is a chain of waits: 143 tokens of 32 heads 6.4 us (a workgroup has a head's five tiles, a wavefront one or two of them; nothing is joined).  512 workgroups are what fits at once: with 1024, half of them ran after the others
// (121 us instead of 75); with 3 or 4 wavefronts a SIMD, the state goes to memory.
template <int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attend_kernel(AttendArgs a)
{
    constexpr int kThreads = 64 * WAVES;
    constexpr int kPartial = kRowBlock * (D + 2);
    __shared__ AttendShared<D, WAVES> shared;
    static_assert(sizeof(shared.out) >= (2 * kMostParts + 1) * kRowBlock * sizeof(float), "");
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), quad = lane >> 4;
    const unsigned per = a.heads_per_group;
    const Partials partials(a.partials, 3 * kAttendWorkgroups * kPartial);
    const auto blocks_of = [&](const Sequence& q) { return static_cast<int>((static_cast<unsigned>(q.rows) * per + kRowBlock - 1) / kRowBlock); };
    // A step is one tile for every wavefront; or two, where there are so few that a workgroup has one or two of them: half the parts to join.
    int step_tiles = WAVES;
    const int most_length = most_tokens(a.seqs, a.pool.page_shift);
    auto deal = deal_out<Sequence>(a.seqs.n_seqs, lane, [&](int b) { return sequence(a.seqs, most_length, b); }, [&](const Sequence& q) {
        return static_cast<unsigned>(min(static_cast<int64_t>(blocks_of(q)) * steps_of(q, step_tiles) * a.pool.kv_heads, int64_t{INT_MAX}));
    });
    if (deal.total <= kFewSteps * gridDim.x) {
        step_tiles = 2 * WAVES;
        deal.recount();
    }
    const unsigned total = deal.total, workers = min(gridDim.x, total), me = blockIdx.x;
    if (me >= workers) return;
    const unsigned share = total / workers, more = total - share * workers;      // the first `more` workgroups take one step more
    const auto start_of = [&](unsigned w) { return w * share + min(w, more); };
    const auto owner_of = [&](unsigned step) {
        const unsigned longer = more * (share + 1);
        return step < longer ? step / (share + 1) : more + (step - longer) / share;
    };
    int at = start_of(me);
    const int end = start_of(me + 1);
    int b, within;
    Sequence seq = deal.locate(at, &b, &within);
    while (at < end) {
        const int blocks = blocks_of(seq), steps = steps_of(seq, step_tiles);
        if (within >= blocks * steps * a.pool.kv_heads) {       // (on to the next sequence that has rows)
            within = 0;
            seq = sequence(a.seqs, most_length, ++b);
            continue;
        }
        const int segment = static_cast<unsigned>(within) / static_cast<unsigned>(steps), from = within - segment * steps;
        const int to = min(steps, from + (end - at));
        const int head = blocks == 1 ? segment : static_cast<unsigned>(segment) / static_cast<unsigned>(blocks);
        const unsigned row0 = (segment - head * blocks) * kRowBlock;        // of the sequence's rows times the heads of a group
        const int rows = min(static_cast<unsigned>(kRowBlock), seq.rows * per - row0);
        const unsigned token0 = row0 / per, head0 = row0 - token0 * per;    // row r of the block: head (head0 + r) % per of the group, token further on
        const int before = seq.length - seq.rows;

        // this lane's row
        const bool is_row = (lane & 15) < rows;
        const unsigned ahead = (head0 + (lane & 15)) / per;
        const int row = token0 + ahead, q_head = head * per + (head0 + (lane & 15) - ahead * per);
        const int limit = is_row ? before + row + 1 : 0;     // tokens it sees
        // (an infinity as NaN: it makes a row NaN, which scores of -infinity only would not)
        half8_t q[D / 32];
        const uint16_t* q_at = a.q.data + int64_t{seq.start + row} * a.q.row + q_head * a.q.head + 8 * quad;
#pragma unroll
        for (int g = 0; g < D / 32; ++g) {
            q[g] = half8_t{};
            if (is_row) q[g] = *reinterpret_cast<const half8_t*>(q_at + 32 * g);
            if (a.negate) q[g] = -q[g];
            q[g] += q[g] - q[g];
        }
        const int least = before + token0 + 1, most = before + token0 + (head0 + rows - 1) / per + 1;    // tokens that the block's first and last row see
        const int tiles = uniform(min((max(most, 0) + kTileTokens - 1) / kTileTokens, to * step_tiles));

        RowState<D> state;
        state.top = kMinusInf;
        state.sum = 0.0f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) state.out[c] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};

        // The wavefront's tiles are every WAVES-th one; lane i knows the page of the i-th of the next 64, so that no load waits for another.
        const int32_t* table = a.seqs.pages + int64_t{b} * a.seqs.max_pages;
        const int first_tile = uniform(from * step_tiles + wave), count = max(tiles - first_tile + WAVES - 1, 0) / WAVES;
        int page_of_lane = 0;
        // (always the same number of loads, past the end and for absent pages of some tile that is there: where loads are sometimes left out, the
        // compiler cannot tell those of the tile at work from those under way, and waits for all)
        const auto load = [&](int i, Raw<D>& raw) {
            const int of = min(i, count - 1);
            if ((i & 63) == 0 && i < count) page_of_lane = opaque(table[min(first_tile + (i + lane) * WAVES, tiles - 1) >> (a.pool.page_shift - 5)]);
            const int page = __builtin_amdgcn_readlane(page_of_lane, of & 63);
            const bool there = page >= 0 && page < a.pool.n_pages;
            const int t = first_tile + of * WAVES;
            raw.first_token = there && i < count ? t * kTileTokens : -1;
            const uint8_t* tile = a.pool.tile<D>(there ? page : 0, head, t);
#pragma unroll
            for (int w = 0; w < D / 64; ++w) {
                raw.k[w] = *reinterpret_cast<const u32x4_t*>(tile + w * 1024 + lane * 16);
                raw.v[w] = *reinterpret_cast<const u32x4_t*>(tile + 16 * D + w * 1024 + lane * 16);
            }
            raw.parameters = *reinterpret_cast<const typename Raw<D>::words_t*>(tile + 32 * D + lane * (D / 8));
        };
        const auto attend = [&](const Raw<D>& raw) {
            if (raw.first_token < 0) return;
            if (raw.first_token + kTileTokens > least) attend_tile<D, true>(raw, shared.stage[wave], q, state, lane, seq.length, limit, a.scale_log2);
            else attend_tile<D, false>(raw, shared.stage[wave], q, state, lane, seq.length, limit, a.scale_log2);
        };
        // kHeld - 1 tiles ahead, in registers that are not copied
        if (count > 0) {
            Raw<D> held[kHeld];
#pragma unroll
            for (int i = 0; i < kHeld - 1; ++i) load(i, held[i]);
            for (int i = 0; i < count; i += kHeld) {
#pragma unroll
                for (int j = 0; j < kHeld; ++j) {
                    load(i + j + kHeld - 1, held[(j + kHeld - 1) % kHeld]);
                    attend(held[j]);
                }
            }
        }

        // the wavefronts' results together
        float sum = state.sum + __shfl_xor(state.sum, 16);
        sum += __shfl_xor(sum, 32);
        if (is_row) {
            if (quad == 0) shared.top[wave][lane] = state.top, shared.sum[wave][lane] = sum;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) *reinterpret_cast<float4_t*>(&shared.out[wave][lane & 15][16 * c + 4 * quad]) = state.out[c];
        }
        __syncthreads();
        const bool whole = from == 0 && to == steps;
        const auto write = [&](int r, int column, float4_t v, float s) {
            const unsigned on = (head0 + r) / per;
            const int to_head = head * per + (head0 + r - on * per);
            const float inverse = s == 0.0f ? 0.0f : 1.0f / s;       // (a row that sees nothing: all sums are 0)
            half4_t y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = static_cast<_Float16>(v[i] * inverse);
            *reinterpret_cast<half4_t*>(a.out.data + int64_t{seq.start + static_cast<int>(token0 + on)} * a.out.row + to_head * a.out.head + column) = y;
        };
        const auto put = [&](int part, int r, int column, float4_t v, float top, float s) {
            partials.store4(part + r * D + column, v);
            if (column == 0) partials.store2(part + kRowBlock * D + 2 * r, top, s);
        };
        const int partial = (2 * me + (from == 0 ? 1 : 0)) * kPartial;
        for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
            const int r = i / (D / 4), column = 4 * (i % (D / 4));
            float top = shared.top[0][r];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) top = fmaxf(top, shared.top[w][r]);
            float4_t v = {0.0f, 0.0f, 0.0f, 0.0f};
            float s = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = weight_of(shared.top[w][r], top);
                s += f * shared.sum[w][r];
                v += f * *reinterpret_cast<const float4_t*>(&shared.out[w][r][column]);
            }
            if (whole) write(r, column, v, s);
            else put(partial, r, column, v, top, s);
        }
        if (!whole) {
            // The first workgroup of the segment, and how many there are.  Up to kFan parts the last workgroup to arrive joins
            // them; of more, every kFan neighbours are joined by the last of them to arrive, and the last of those joins the results: else one
            // workgroup would read all parts alone (of 64 parts of 8 rows 262 KB).
            const unsigned segment_start = at - from, w0 = owner_of(segment_start);
            const int parts = owner_of(segment_start + steps - 1) - w0 + 1, mine = me - w0;
            // The counters count a part only when all its stores have arrived.  (A release and an acquire around the counters would write back and empty whole L2 caches: 3 times the kernel's time.)
            const auto arrived_last = [&](int* counter, int all) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
                if (threadIdx.x == 0) {
                    shared.last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == all - 1;
                    if (shared.last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // (for the next call)
                }
                __syncthreads();
                return shared.last != 0;
            };
            const auto part_of = [&](int p) { return static_cast<int>(2 * (w0 + p) + (p == 0 ? 1 : 0)) * kPartial; };
            // A counter and a place of a group's result go by a workgroup of the group that is not the segment's first: that one may be the last of the segment
            // before, but no workgroup is behind the first of two segments.
            const auto slot_of = [&](int g) { return w0 + max(g * kFan, 1); };
            const auto joint_of = [&](int g) { return static_cast<int>(2 * kAttendWorkgroups + slot_of(g)) * kPartial; };
            const auto finish = [&](int r, int column, float4_t v, float, float s) { write(r, column, v, s); };
            if (parts <= kFan) {
                if (arrived_last(a.arrivals + slot_of(0), parts)) join<D, kRowBlock, kThreads>(partials, rows, parts, &shared.out[0][0][0], part_of, finish);
            } else {
                const int g = mine / kFan, groups = (parts + kFan - 1) / kFan;
                if (arrived_last(a.arrivals + slot_of(g), min(kFan, parts - g * kFan))) {
                    join<D, kRowBlock, kThreads>(partials, rows, min(kFan, parts - g * kFan), &shared.out[0][0][0], [&](int p) { return part_of(g * kFan + p); },
                                      [&](int r, int column, float4_t v, float top, float s) { put(joint_of(g), r, column, v, top, s); });
                    if (arrived_last(a.arrivals + kAttendWorkgroups + slot_of(0), groups)) join<D, kRowBlock, kThreads>(partials, rows, groups, &shared.out[0][0][0], joint_of, finish);
                }
            }
        }
        __syncthreads();       // (LDS is free again)
        at += to - from;
        within += to - from;
    }
}

gqsa_status_t on_device(const gqsa_cache* c)
{
    int dev = -1;
    GQSA_HIP(hipGetDevice(&dev));
    if (dev != c->device) return GQSA_ERR_HIP;
    return GQSA_OK;
}

Pool pool_of(const gqsa_cache* c)
{
    return {c->d_pages, c->n_pages, __builtin_ctz(static_cast<unsigned>(c->page_tokens)), c->kv_heads};
}

}  // namespace

gqsa_status_t cache_allocate(gqsa_cache* c)
{
    GQSA_HIP(hipGetDevice(&c->device));
    void* p = nullptr;
    GQSA_HIP(hipMalloc(&p, static_cast<size_t>(c->device_bytes())));
    c->d_pages = static_cast<uint8_t*>(p);
    GQSA_HIP(hipMalloc(&p, static_cast<size_t>(c->partial_floats()) * 4));
    c->d_partials = static_cast<float*>(p);
    GQSA_HIP(hipMalloc(&p, kAttendWorkgroups * 2 * 4));
    c->d_arrivals = static_cast<int32_t*>(p);
    GQSA_HIP(hipMemset(c->d_pages, 0, static_cast<size_t>(c->device_bytes())));
    GQSA_HIP(hipMemset(c->d_arrivals, 0, kAttendWorkgroups * 2 * 4));
    GQSA_HIP(hipDeviceSynchronize());
    return GQSA_OK;
}

void cache_release(gqsa_cache* c)
{
    if (c->d_pages) (void)hipFree(c->d_pages);
    if (c->d_partials) (void)hipFree(c->d_partials);
    if (c->d_arrivals) (void)hipFree(c->d_arrivals);
    c->d_pages = nullptr;
    c->d_partials = nullptr;
    c->d_arrivals = nullptr;
}

// Units of a copy: no more than a tile for every 32 rows and two more for every sequence.
static dim3 copy_grid(const gqsa_cache* c, const Sequences& s)
{
    return dim3(static_cast<unsigned>(s.n_rows / kTileTokens + 2 * int64_t{s.n_seqs}), static_cast<unsigned>(c->kv_heads));
}

gqsa_status_t cache_append(gqsa_cache* c, const Heads& k, const Heads& v, const Sequences& seqs, void* stream)
{
    if (gqsa_status_t st = on_device(c)) return st;
    const CopyArgs a{pool_of(c), k, v, seqs};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (c->head_dim == 128) hipLaunchKernelGGL(append_kernel<128>, copy_grid(c, seqs), dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL(append_kernel<64>, copy_grid(c, seqs), dim3(kThreads), 0, s, a);
    GQSA_HIP(hipGetLastError());
    return GQSA_OK;
}

gqsa_status_t cache_read(gqsa_cache* c, const Heads& k, const Heads& v, const Sequences& seqs, void* stream)
{
    if (gqsa_status_t st = on_device(c)) return st;
    const CopyArgs a{pool_of(c), k, v, seqs};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (c->head_dim == 128) hipLaunchKernelGGL(read_kernel<128>, copy_grid(c, seqs), dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL(read_kernel<64>, copy_grid(c, seqs), dim3(kThreads), 0, s, a);
    GQSA_HIP(hipGetLastError());
    return GQSA_OK;
}

gqsa_status_t cache_attend(gqsa_cache* c, const Heads& q, int q_heads, const Sequences& seqs, float scale, const Heads& out, void* stream)
{
    if (gqsa_status_t st = on_device(c)) return st;
    const int per = q_heads / c->kv_heads;
    const AttendArgs a{pool_of(c), q, out, seqs, c->d_partials, c->d_arrivals, per,
                       // (not 0, so that a masked score stays -infinity: 1e-30 leaves every weight at 1)
                       std::max(std::fabs(scale) * 1.44269504088896341f, 1e-30f), scale < 0.0f};
    // No more workgroups than there can be steps.  (The kernel counts them, and rows of a group, in 32 bits.)
    if (seqs.n_rows * per > (1 << 30)) return GQSA_ERR_SHAPE;
    const double blocks = (static_cast<double>(seqs.n_rows) * per / kRowBlock + seqs.n_seqs) * c->kv_heads;
    const double steps = blocks * (static_cast<double>(seqs.max_pages) * c->page_tokens / (kAttendWaves * kTileTokens) + 1.0);
    if (steps > INT_MAX) return GQSA_ERR_SHAPE;
    const unsigned grid = static_cast<unsigned>(std::max(1.0, std::min<double>(kAttendWorkgroups, steps)));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 threads(64 * kAttendWaves);
    if (c->head_dim == 128) hipLaunchKernelGGL((attend_kernel<128, kAttendWaves>), dim3(grid), threads, 0, s, a);
    else hipLaunchKernelGGL((attend_kernel<64, kAttendWaves>), dim3(grid), threads, 0, s, a);
    GQSA_HIP(hipGetLastError());
    return GQSA_OK;
}

}  // namespace gqsa
