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
// Code e of a word is at bits 4 (e / 2) + 16 (e % 2), so that one AND leaves two neighbouring ones in the halves of a register.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "gqsa_device.hpp"

namespace gqsa {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__host__ __device__ constexpr int word_offset(int w, int lane) { return (w >> 2) * 1024 + lane * 16 + (w & 3) * 4; }
__host__ __device__ constexpr int nibble(int e) { return 4 * (e >> 1) + 16 * (e & 1); }
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

__device__ __forceinline__ Sequence sequence(const Sequences& s, int page_shift, int b)
{
    const int n = static_cast<int>(s.n_rows);
    const int first = s.row_starts ? s.row_starts[b] : b, end = s.row_starts ? s.row_starts[b + 1] : b + 1;
    Sequence q;
    q.start = min(max(first, 0), n);
    q.rows = max(min(end, n) - q.start, 0);
    const int64_t most = int64_t{s.max_pages} << page_shift;
    q.length = static_cast<int>(min(static_cast<int64_t>(max(s.lengths[b], 0)), min(most, int64_t{INT_MAX - 4096})));
    return q;
}

// --------------------------------------------------------------------------- into the cache and out of it
struct CopyArgs {
    Pool pool;
    Heads k, v;
    Sequences seqs;
};

// The tiles that the rows of a sequence lie in, from the first one's (which may be below 0) on.
__device__ __forceinline__ int64_t tiles_of_rows(const Sequence& q)
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
    int b;
    int64_t within;
    const auto count = [&](int s) { return tiles_of_rows(sequence(a.seqs, a.pool.page_shift, s)); };
    if (!locate(a.seqs.n_seqs, blockIdx.x, threadIdx.x & 63, count, &b, &within)) return false;
    u->seq = sequence(a.seqs, a.pool.page_shift, b);
    u->tile = ((u->seq.length - u->seq.rows) >> 5) + static_cast<int>(within);
    u->head = blockIdx.y;
    u->page = -1;
    if (u->tile >= 0) {
        const int page = a.seqs.pages[int64_t{b} * a.seqs.max_pages + (u->tile >> (a.pool.page_shift - 5))];
        if (page >= 0 && page < a.pool.n_pages) u->page = page;
    }
    return true;
}

template <int N>
struct Quantised {
    _Float16 low, step;
    uint8_t code[N];
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
    q.step = bad ? static_cast<_Float16>(0.0f) : static_cast<_Float16>((high - low) / 15.0f);
    const float step = static_cast<float>(q.step);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float v = static_cast<float>(x[i / 8][i % 8]);
        q.code[i] = step > 0.0f ? static_cast<uint8_t>(fminf(__builtin_rintf((v - low) / step), 15.0f)) : 0;
    }
    return q;
}

// One workgroup per tile that gets rows, and head: 8 threads to a token.  A word of key codes belongs to one token; one of value codes to 8
// tokens, so those are put together in LDS, and a word that keeps earlier tokens is read first (nobody else writes the tile).
template <int D>
__global__ __launch_bounds__(kThreads) void append_kernel(CopyArgs a)
{
    constexpr int kOwn = D / 8;                    // elements of a token per thread
    constexpr int kParameters = 32 * D;            // where the parameters start in a tile
    __shared__ uint8_t v_codes[kTileTokens][D];
    Unit u;
    if (!unit_of(a, &u) || u.page < 0) return;
    uint8_t* tile = a.pool.tile<D>(u.page, u.head, u.tile);
    const int first = u.seq.length - u.seq.rows;   // the rows' first token
    const auto is_new = [&](int t) { const int token = u.tile * kTileTokens + t; return token >= first && token < u.seq.length; };

    const int t = threadIdx.x >> 3, part = threadIdx.x & 7;
    if (is_new(t)) {
        const int64_t row = u.seq.start + (u.tile * kTileTokens + t - first);
        const uint16_t* k_at = a.k.data + row * a.k.row + u.head * a.k.head + part * kOwn;
        const uint16_t* v_at = a.v.data + row * a.v.row + u.head * a.v.head + part * kOwn;
        half8_t x[kOwn / 8], y[kOwn / 8];
#pragma unroll
        for (int i = 0; i < kOwn / 8; ++i) {
            x[i] = reinterpret_cast<const half8_t*>(k_at)[i];
            y[i] = reinterpret_cast<const half8_t*>(v_at)[i];
        }
        const int group = part * kOwn / kGroupChannels;
        const bool leads = part % (kGroupChannels / kOwn) == 0;
        const Quantised<kOwn> k = quantise<kOwn>(x);
#pragma unroll
        for (int i = 0; i < kOwn / 8; ++i) {
            uint32_t word = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) word |= uint32_t{k.code[8 * i + e]} << nibble(e);
            const int quad = (part * kOwn + 8 * i) % kGroupChannels / 8;
            const int w = (t >> 4) * (D / 32) + group;
            *reinterpret_cast<uint32_t*>(tile + word_offset(w, quad * 16 + (t & 15))) = word;
        }
        if (leads) {
            const half2_t both = {k.low, k.step};
            *reinterpret_cast<half2_t*>(tile + kParameters + (t * (D / 32) + group) * 4) = both;
        }
        const Quantised<kOwn> v = quantise<kOwn>(y);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) v_codes[t][part * kOwn + i] = v.code[i];
        if (leads) {
            const int quad = (t >> 2) & 3, slot = (t & 3) + (t >> 4) * 4;
            _Float16* at = reinterpret_cast<_Float16*>(tile + kParameters + 4 * D + (group * 4 + quad) * 32) + slot;
            at[0] = v.step;
            at[8] = v.low;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < D / 16 * 64; i += kThreads) {
        const int c = i >> 6, l = i & 63, quad = l >> 4;
        uint32_t word = 0, kept = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int token = slot_token(quad, e);
            if (is_new(token)) word |= uint32_t{v_codes[token][16 * c + (l & 15)]} << nibble(e);
            else kept |= 15u << nibble(e);
        }
        if (kept == ~0u) continue;
        uint32_t* at = reinterpret_cast<uint32_t*>(tile + 16 * D + word_offset(c, l));
        if (kept) word |= *at & kept;
        *at = word;
    }
}

template <int D>
__global__ __launch_bounds__(kThreads) void read_kernel(CopyArgs a)
{
    constexpr int kOwn = D / 8;
    constexpr int kParameters = 32 * D;
    Unit u;
    if (!unit_of(a, &u)) return;
    const int first = u.seq.length - u.seq.rows;
    const int t = threadIdx.x >> 3, part = threadIdx.x & 7;
    const int token = u.tile * kTileTokens + t;
    if (token < first || token >= u.seq.length) return;
    half8_t x[kOwn / 8] = {}, y[kOwn / 8] = {};
    if (u.page >= 0) {
        const uint8_t* tile = a.pool.tile<D>(u.page, u.head, u.tile);
        const int group = part * kOwn / kGroupChannels, quad = (t >> 2) & 3, slot = (t & 3) + (t >> 4) * 4;
        const half2_t k = *reinterpret_cast<const half2_t*>(tile + kParameters + (t * (D / 32) + group) * 4);
        const _Float16* v = reinterpret_cast<const _Float16*>(tile + kParameters + 4 * D + (group * 4 + quad) * 32) + slot;
        const _Float16 v_step = v[0], v_low = v[8];
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int element = part * kOwn + i;
            const uint32_t kw = *reinterpret_cast<const uint32_t*>(
                tile + word_offset((t >> 4) * (D / 32) + group, element % kGroupChannels / 8 * 16 + (t & 15)));
            const uint32_t vw = *reinterpret_cast<const uint32_t*>(tile + 16 * D + word_offset(element / 16, quad * 16 + element % 16));
            x[i / 8][i % 8] = __builtin_fmaf16(static_cast<_Float16>(static_cast<float>(kw >> nibble(i % 8) & 15u)), k[1], k[0]);
            y[i / 8][i % 8] = __builtin_fmaf16(static_cast<_Float16>(static_cast<float>(vw >> nibble(slot) & 15u)), v_step, v_low);
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
    float scale_log2;       // scale times log2(e): the softmax is taken to base 2
};

// A tile as it is loaded: codes of keys and of values, parameters (16 bytes a lane with D = 128, 8 with D = 64).
template <int D>
struct Raw {
    u32x4_t k[D / 64], v[D / 64];
    uint32_t parameters[D / 32];
};

// Two fp16 numbers of eight codes each time: (x & mask) in the low bits of 1024 (0x6400), taken off again, is exact, and so is
// the multiply-add by 1/16 for codes four bits higher up.
__device__ __forceinline__ void decode(uint32_t x, half2_t (&q)[4])
{
    const half2_t off = {static_cast<_Float16>(-1024.0f), static_cast<_Float16>(-1024.0f)};
    const half2_t sixteenth = {static_cast<_Float16>(0.0625f), static_cast<_Float16>(0.0625f)};
    const half2_t off16 = {static_cast<_Float16>(-64.0f), static_cast<_Float16>(-64.0f)};
    const uint32_t y = x >> 8;
    q[0] = __builtin_bit_cast(half2_t, (x & 0x000F000Fu) | 0x64006400u) + off;
    q[1] = __builtin_elementwise_fma(__builtin_bit_cast(half2_t, (x & 0x00F000F0u) | 0x64006400u), sixteenth, off16);
    q[2] = __builtin_bit_cast(half2_t, (y & 0x000F000Fu) | 0x64006400u) + off;
    q[3] = __builtin_elementwise_fma(__builtin_bit_cast(half2_t, (y & 0x00F000F0u) | 0x64006400u), sixteenth, off16);
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

constexpr float kSlack = 8.0f;      // powers of two that a score may lie above the reference before the reference follows

// One tile for one wavefront.  S^T = K Q^T and O^T = V^T P^T: a lane's scores are then the elements of the operand P^T that the second product wants
// from it, whatever the tokens' order, as the value codes lie in the same.
template <int D>
__device__ __forceinline__ void attend_tile(const Raw<D>& raw, uint32_t* stage, const half8_t (&q)[D / 32], RowState<D>& state, int lane,
                                            int first_token, int length, int limit, bool edge, float scale_log2)
{
    constexpr int kWords = D / 32;            // words of parameters a lane stages
    const int quad = lane >> 4;
    uint32_t parameters[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i) parameters[i] = raw.parameters[i];
    if (edge) {
        // whatever lies behind the last token (older codes, NaN) stands for zero
        const int left = length - first_token;
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const int at = (lane * kWords + i) * 4;
            if (at < 4 * D) {
                if (at / (D / 8) >= left) parameters[i] = 0;
            } else {
                const int o = at - 4 * D, t = slot_token((o >> 5) & 3, (o & 15) >> 1);
                if (t >= left) parameters[i] = 0;
                else if (t + 1 >= left) parameters[i] &= 0xFFFFu;
            }
        }
    }
    wave_lds_order();
#pragma unroll
    for (int i = 0; i < kWords; ++i) stage[lane * kWords + i] = parameters[i];
    wave_lds_order();

    float4_t s[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        s[j] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
        const uint32_t* p = stage + (16 * j + (lane & 15)) * (D / 32);
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
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = s[i >> 2][i & 3] * scale_log2;
    if (edge) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (first_token + slot_token(quad, i) >= limit) x[i] = kMinusInf;
    }
    float most = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    // The reference follows only where a score lies far above it: p then reaches 2^8 at most, well inside fp16.
    if (__any(most > state.top + kSlack || (state.top == kMinusInf && most > kMinusInf))) {
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        const float top = fmaxf(state.top, most);
        const float shrink = top == kMinusInf ? 1.0f : __builtin_amdgcn_exp2f(state.top - top);
        state.top = top;
        state.sum *= shrink;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) state.out[c] *= shrink;
    }
    const float reference = state.top == kMinusInf ? 0.0f : state.top;
    half8_t p;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float e = __builtin_amdgcn_exp2f(x[i] - reference);
        state.sum += e;
        p[i] = static_cast<_Float16>(e);
    }
    const auto values = [&](int c) {
        const uint32_t* at = stage + D + (c / 2 * 4 + quad) * 8;
        half2_t v[4];
        decode(raw.v[c >> 2][c & 3], v);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_elementwise_fma(v[i], as_half2(at[i]), as_half2(at[4 + i]));
        return join(v[0], v[1], v[2], v[3]);
    };
    // Only where rows differ in what they see of the tile can a value that is not finite reach a row that does not see it.
    bool wild = false;
    if (edge) {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const half2_t h = as_half2(parameters[i]);
            odd |= !(__builtin_fabsf16(h[0]) <= static_cast<_Float16>(65504.0f)) || !(__builtin_fabsf16(h[1]) <= static_cast<_Float16>(65504.0f));
        }
        wild = __any(odd);
    }
    if (!wild) {
#pragma unroll
        for (int c = 0; c < D / 16; ++c) state.out[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(values(c), p, state.out[c], 0, 0, 0);
    } else {
        half8_t sees;
#pragma unroll
        for (int i = 0; i < 8; ++i) sees[i] = static_cast<_Float16>(first_token + slot_token(quad, i) < limit ? 1.0f : 0.0f);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            const half8_t v = values(c);
            state.out[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(finite_part(v), p, state.out[c], 0, 0, 0);
            const float4_t count = __builtin_amdgcn_mfma_f32_16x16x32_f16(not_finite(v), sees, float4_t{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) state.out[c][r] += from_counts(count[r]);
            __builtin_amdgcn_sched_barrier(0);      // (one after the other: few registers, not speed)
        }
    }
}

__device__ __forceinline__ float weight_of(float top, float most) { return top == kMinusInf ? 0.0f : __builtin_amdgcn_exp2f(top - most); }

template <int D>
struct alignas(16) AttendShared {
    uint32_t stage[kWaves][2 * D];
    float out[kWaves][kRowBlock][D + 4];       // (+ 4: rows start in different banks)
    float top[kWaves][kRowBlock], sum[kWaves][kRowBlock];
    int last;
};

__device__ __forceinline__ void store_partial(float* at, float a, float b)
{
    const uint64_t both = uint64_t{__builtin_bit_cast(uint32_t, b)} << 32 | __builtin_bit_cast(uint32_t, a);
    __hip_atomic_store(reinterpret_cast<uint64_t*>(at), both, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ float2 load_partial(const float* at)
{
    const uint64_t both = __hip_atomic_load(reinterpret_cast<const uint64_t*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return {__builtin_bit_cast(float, static_cast<uint32_t>(both)), __builtin_bit_cast(float, static_cast<uint32_t>(both >> 32))};
}

constexpr int kStepTiles = kWaves;      // a step: one tile for every wavefront of a workgroup

// The work is dealt by steps of 128 tokens, not by sequences or heads: workgroup w takes the steps w T / W .. (w + 1) T / W - 1 of all T, in the order
// sequence, head, block of 16 rows, token.  Where a segment (one block of rows of one head) lies in several workgroups, each leaves its maximum,
// sum and weighted sum in the workspace, and the last to arrive joins them in the order of the tokens.
template <int D>
__global__ __launch_bounds__(kThreads, 4) void attend_kernel(AttendArgs a)
{
    constexpr int kPartial = kRowBlock * (D + 2);
    __shared__ AttendShared<D> shared;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quad = lane >> 4;
    const int per = a.heads_per_group;
    const auto blocks_of = [&](const Sequence& q) { return (int64_t{q.rows} * per + kRowBlock - 1) / kRowBlock; };
    const auto steps_of = [&](const Sequence& q) { return max((q.length + kStepTiles * kTileTokens - 1) / (kStepTiles * kTileTokens), 1); };
    const auto count = [&](int b) {
        const Sequence q = sequence(a.seqs, a.pool.page_shift, b);
        return blocks_of(q) * steps_of(q) * a.pool.kv_heads;
    };
    const int64_t total = total_of(a.seqs.n_seqs, lane, count);
    const int64_t workers = min(static_cast<int64_t>(gridDim.x), total);
    const int64_t me = blockIdx.x;
    if (me >= workers) return;
    int64_t at = me * total / workers;
    const int64_t end = (me + 1) * total / workers;
    int b;
    int64_t within;
    if (!locate(a.seqs.n_seqs, at, lane, count, &b, &within)) return;
    b = __builtin_amdgcn_readfirstlane(b);

    Sequence seq = sequence(a.seqs, a.pool.page_shift, b);
    while (at < end) {
        const int64_t blocks = blocks_of(seq);
        const int steps = steps_of(seq);
        if (within >= blocks * steps * a.pool.kv_heads) {       // (on to the next sequence that has rows)
            within = 0;
            seq = sequence(a.seqs, a.pool.page_shift, ++b);
            continue;
        }
        const int64_t segment = within / steps;
        const int from = static_cast<int>(within - segment * steps);
        const int to = static_cast<int>(min(static_cast<int64_t>(steps), from + (end - at)));
        const int head = static_cast<int>(segment / blocks);
        const int64_t row0 = (segment - head * blocks) * kRowBlock;        // of the sequence's rows times the heads of a group
        const int rows = static_cast<int>(min(int64_t{kRowBlock}, int64_t{seq.rows} * per - row0));

        // this lane's row
        const int64_t mine = row0 + (lane & 15);
        const bool is_row = (lane & 15) < rows;
        const int row = is_row ? static_cast<int>(mine / per) : 0;
        const int q_head = head * per + static_cast<int>(mine - int64_t{row} * per);
        const int limit = is_row ? seq.length - seq.rows + row + 1 : 0;     // tokens it sees
        half8_t q[D / 32];
#pragma unroll
        for (int g = 0; g < D / 32; ++g) {
            q[g] = half8_t{};
            if (is_row) q[g] = *reinterpret_cast<const half8_t*>(a.q.data + (int64_t{seq.start} + row) * a.q.row + q_head * a.q.head + 32 * g + 8 * quad);
        }
        const int least = seq.length - seq.rows + static_cast<int>(row0 / per) + 1;                 // tokens that the block's first and last row see
        const int most = seq.length - seq.rows + static_cast<int>((row0 + rows - 1) / per) + 1;
        const int tiles = min((max(most, 0) + kTileTokens - 1) / kTileTokens, to * kStepTiles);

        RowState<D> state;
        state.top = kMinusInf;
        state.sum = 0.0f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) state.out[c] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};

        const int32_t* table = a.seqs.pages + int64_t{b} * a.seqs.max_pages;
        const auto load = [&](int t, Raw<D>& raw) {
            const int page = __builtin_amdgcn_readfirstlane(table[t >> (a.pool.page_shift - 5)]);
            if (page < 0 || page >= a.pool.n_pages) return false;
            const uint8_t* tile = a.pool.tile<D>(page, head, t);
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                raw.k[i] = *reinterpret_cast<const u32x4_t*>(tile + i * 1024 + lane * 16);
                raw.v[i] = *reinterpret_cast<const u32x4_t*>(tile + 16 * D + i * 1024 + lane * 16);
            }
            const uint32_t* p = reinterpret_cast<const uint32_t*>(tile + 32 * D) + lane * (D / 32);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) raw.parameters[i] = p[i];
            return true;
        };
        Raw<D> next;
        bool there = false;
        int t = from * kStepTiles + wave;
        if (t < tiles) there = load(t, next);
        while (t < tiles) {
            const Raw<D> raw = next;
            const bool here = there;
            const int now = t;
            t += kStepTiles;
            if (t < tiles) there = load(t, next);
            const int first_token = now * kTileTokens;
            if (here) attend_tile<D>(raw, shared.stage[wave], q, state, lane, first_token, seq.length, limit, first_token + kTileTokens > least, a.scale_log2);
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
            const int64_t of = row0 + r;
            const int token = static_cast<int>(of / per);
            const int to_head = head * per + static_cast<int>(of - int64_t{token} * per);
            half4_t y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = s == 0.0f ? static_cast<_Float16>(0.0f) : static_cast<_Float16>(v[i] / s);
            *reinterpret_cast<half4_t*>(a.out.data + (int64_t{seq.start} + token) * a.out.row + to_head * a.out.head + column) = y;
        };
        float* partial = a.partials + (2 * me + (from == 0 ? 1 : 0)) * kPartial;
        for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
            const int r = i / (D / 4), column = 4 * (i % (D / 4));
            float top = shared.top[0][r];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) top = fmaxf(top, shared.top[w][r]);
            float4_t v = {0.0f, 0.0f, 0.0f, 0.0f};
            float s = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float f = weight_of(shared.top[w][r], top);
                s += f * shared.sum[w][r];
                v += f * *reinterpret_cast<const float4_t*>(&shared.out[w][r][column]);
            }
            if (whole) {
                write(r, column, v, s);
            } else {
                store_partial(partial + r * D + column, v[0], v[1]);
                store_partial(partial + r * D + column + 2, v[2], v[3]);
                if (column == 0) store_partial(partial + kRowBlock * D + 2 * r, top, s);
            }
        }
        if (!whole) {
            // the first workgroup of the segment (its number names the counter) and the last
            const int64_t segment_start = at - from, segment_end = segment_start + steps;
            const int64_t w0 = ((segment_start + 1) * workers - 1) / total, w1 = (segment_end * workers - 1) / total;
            const int parts = static_cast<int>(w1 - w0) + 1;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // every thread's part is where the others can see it
            __syncthreads();
            if (threadIdx.x == 0)
                shared.last = __hip_atomic_fetch_add(a.arrivals + w0, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
            __syncthreads();
            if (shared.last) {
                const int columns = rows * (D / 4), teams = max(1, kThreads / columns);
                for (int i = threadIdx.x; i < columns * teams; i += kThreads) {
                    const int team = i / columns, of = i - team * columns, r = of / (D / 4), column = 4 * (of % (D / 4));
                    float top = kMinusInf, s = 0.0f;
                    float4_t v = {0.0f, 0.0f, 0.0f, 0.0f};
                    const auto part_at = [&](int p) { return a.partials + (2 * (w0 + p) + (p == 0 ? 1 : 0)) * kPartial; };
                    constexpr int kAhead = 4;
                    for (int p0 = team; p0 < parts; p0 += teams * kAhead) {
                        float2 x[kAhead], y[kAhead], z[kAhead];
#pragma unroll
                        for (int j = 0; j < kAhead; ++j) {
                            const float* from_part = part_at(min(p0 + j * teams, parts - 1));
                            x[j] = load_partial(from_part + r * D + column);
                            y[j] = load_partial(from_part + r * D + column + 2);
                            z[j] = load_partial(from_part + kRowBlock * D + 2 * r);
                        }
#pragma unroll
                        for (int j = 0; j < kAhead; ++j) {
                            if (p0 + j * teams >= parts) break;
                            const float both = fmaxf(top, z[j].x);
                            const float f = weight_of(top, both), g = weight_of(z[j].x, both);
                            s = f * s + g * z[j].y;
                            v = f * v + g * float4_t{x[j].x, x[j].y, y[j].x, y[j].y};
                            top = both;
                        }
                    }
                    if (teams == 1) {
                        write(r, column, v, s);
                    } else {
                        float* out = &shared.out[0][0][0] + i * 6;
                        out[0] = top, out[1] = s, out[2] = v[0], out[3] = v[1], out[4] = v[2], out[5] = v[3];
                    }
                }
                if (teams > 1) {
                    __syncthreads();
                    for (int of = threadIdx.x; of < columns; of += kThreads) {
                        const float* in = &shared.out[0][0][0];
                        float top = kMinusInf;
                        for (int k = 0; k < teams; ++k) top = fmaxf(top, in[(k * columns + of) * 6]);
                        float s = 0.0f;
                        float4_t v = {0.0f, 0.0f, 0.0f, 0.0f};
                        for (int k = 0; k < teams; ++k) {
                            const float* p = in + (k * columns + of) * 6;
                            const float f = weight_of(p[0], top);
                            s += f * p[1];
                            v += f * float4_t{p[2], p[3], p[4], p[5]};
                        }
                        write(of / (D / 4), 4 * (of % (D / 4)), v, s);
                    }
                }
                if (threadIdx.x == 0) __hip_atomic_store(a.arrivals + w0, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
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
    GQSA_HIP(hipMalloc(&p, kAttendWorkgroups * 4));
    c->d_arrivals = static_cast<int32_t*>(p);
    GQSA_HIP(hipMemset(c->d_pages, 0, static_cast<size_t>(c->device_bytes())));
    GQSA_HIP(hipMemset(c->d_arrivals, 0, kAttendWorkgroups * 4));
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
    const AttendArgs a{pool_of(c), q, out, seqs, c->d_partials, c->d_arrivals, per, scale * 1.44269504088896341f};
    // no more workgroups than there can be steps
    const double blocks = (static_cast<double>(seqs.n_rows) * per / kRowBlock + seqs.n_seqs) * c->kv_heads;
    const double steps = static_cast<double>(seqs.max_pages) * c->page_tokens / (kStepTiles * kTileTokens) + 1.0;
    const unsigned grid = static_cast<unsigned>(std::max(1.0, std::min<double>(kAttendWorkgroups, blocks * steps)));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (c->head_dim == 128) hipLaunchKernelGGL(attend_kernel<128>, dim3(grid), dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL(attend_kernel<64>, dim3(grid), dim3(kThreads), 0, s, a);
    GQSA_HIP(hipGetLastError());
    return GQSA_OK;
}

}  // namespace gqsa
