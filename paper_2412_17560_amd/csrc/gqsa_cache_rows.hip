// Rows on their way into the cache and within it: new queries and keys normed and rotated, keys and values quantised into their pages in the same launch
// (gqsa_cache_append_rotated), and tokens of the newest rows moved to the front of them (gqsa_cache_keep).
//   r = 1 / sqrt(mean(x^2) + eps),   u = x (r w),   (a, b) -> (a c - b s, a s + b c),   fp16,   then low, step and codes of groups of 32
#include <hip/hip_runtime.h>

#include "gqsa_cache.hpp"

namespace gqsa {
namespace {

// Which of a tile's 32 tokens are written, and what of a tile is put together in LDS.
template <int D>
struct alignas(16) TileImage {
    uint8_t image[tile_bytes(D)];
    uint8_t v_codes[kTileTokens][D + 4];
};

// A thread's part of a token: D / 8 elements of it, with 8 threads to a token.
template <int D>
struct Codes {
    static constexpr int kOwn = D / 8;
    uint32_t k_words[kOwn / 8];     // codes of keys, as they are held
    uint32_t v_bytes[kOwn / 4];     // codes of values, a byte each
    uint32_t k_parameters;          // low, step of the group
    uint16_t v_step, v_low;
};

template <int D>
__device__ __forceinline__ int key_word(int t, int element) { return word_offset((t >> 4) * (D / 32) + element / kGroupChannels, element % kGroupChannels / 8 * 16 + (t & 15)); }
template <int D>
__device__ __forceinline__ int key_parameters(int t, int group) { return 32 * D + (t * (D / 32) + group) * 4; }
// (step; low is 16 bytes further on)
template <int D>
__device__ __forceinline__ int value_parameters(int t, int group) { return 36 * D + (group * 4 + (t >> 2 & 3)) * 32 + 2 * ((t & 3) + (t >> 4) * 4); }

// Four bits as the bytes 0x0F or 0 of a word.
__device__ __forceinline__ uint32_t spread(uint32_t four) { return ((four * 0x00204081u) & 0x01010101u) * 15u; }

// Of a tile, the tokens of `fresh` (bit t: token t) written from what their threads hold; the others are left.  A word of value codes holds 8 tokens: thread i
// puts the two words of two neighbouring elements together, from 8 reads of two bytes each, and takes the codes that stay from the tile.
// Called by whole workgroups; `shared` is free again after a barrier.
template <int D>
__device__ __forceinline__ void put_tile(uint8_t* tile, uint32_t fresh, const Codes<D>& own, TileImage<D>& shared)
{
    constexpr int kOwn = D / 8, kPairs = 2 * D;
    const int t = threadIdx.x >> 3, part = threadIdx.x & 7, group = part * kOwn / kGroupChannels;
    const bool leads = part % (kGroupChannels / kOwn) == 0, mine = fresh >> t & 1, all = fresh == ~0u;
    const int quad = (threadIdx.x / (D / 2)) & 3, element = 2 * (threadIdx.x % (D / 2));
    const int at = 16 * D + word_offset(element / 16, quad * 16 + element % 16);
    const uint32_t written = spread(fresh >> 4 * quad & 15u) | spread(fresh >> (16 + 4 * quad) & 15u) << 4;
    // (asked for by every thread, and stored below under one condition)
    const uint32_t old0 = *reinterpret_cast<const uint32_t*>(tile + at), old1 = *reinterpret_cast<const uint32_t*>(tile + at + 16);
    if (mine) {
#pragma unroll
        for (int i = 0; i < kOwn / 8; ++i) *reinterpret_cast<uint32_t*>(shared.image + key_word<D>(t, part * kOwn + 8 * i)) = own.k_words[i];
#pragma unroll
        for (int i = 0; i < kOwn / 4; ++i) *reinterpret_cast<uint32_t*>(&shared.v_codes[t][part * kOwn + 4 * i]) = own.v_bytes[i];
        if (leads) {
            *reinterpret_cast<uint32_t*>(shared.image + key_parameters<D>(t, group)) = own.k_parameters;
            *reinterpret_cast<uint16_t*>(shared.image + value_parameters<D>(t, group)) = own.v_step;
            *reinterpret_cast<uint16_t*>(shared.image + value_parameters<D>(t, group) + 16) = own.v_low;
        }
    }
    __syncthreads();
    if (kPairs == kThreads || threadIdx.x < kPairs) {
        uint32_t two[8];        // codes of both elements of the word's tokens, in its order
#pragma unroll
        for (int i = 0; i < 8; ++i) two[i] = *reinterpret_cast<const uint16_t*>(&shared.v_codes[slot_token(quad, i)][element]);
        uint32_t word[2] = {0, 0};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t a = two[4 * h] | two[4 * h + 1] << 16, b = two[4 * h + 2] | two[4 * h + 3] << 16;
            // (of tokens that are not written anything may lie there)
            word[0] |= (__builtin_amdgcn_perm(b, a, 0x06040200u) & 0x0F0F0F0Fu) << 4 * h;
            word[1] |= (__builtin_amdgcn_perm(b, a, 0x07050301u) & 0x0F0F0F0Fu) << 4 * h;
        }
        word[0] = (word[0] & written) | (old0 & ~written);
        word[1] = (word[1] & written) | (old1 & ~written);
        uint8_t* to = all ? shared.image : tile;
        if (written != 0) {
            *reinterpret_cast<uint32_t*>(to + at) = word[0];
            *reinterpret_cast<uint32_t*>(to + at + 16) = word[1];
        }
    }
    if (all) {
        __syncthreads();
        for (int i = threadIdx.x; i < tile_bytes(D) / 16; i += kThreads)
            reinterpret_cast<u32x4_t*>(tile)[i] = reinterpret_cast<const u32x4_t*>(shared.image)[i];
    } else if (mine) {
#pragma unroll
        for (int i = 0; i < kOwn / 8; ++i) *reinterpret_cast<uint32_t*>(tile + key_word<D>(t, part * kOwn + 8 * i)) = own.k_words[i];
        if (leads) {
            *reinterpret_cast<uint32_t*>(tile + key_parameters<D>(t, group)) = own.k_parameters;
            *reinterpret_cast<uint16_t*>(tile + value_parameters<D>(t, group)) = own.v_step;
            *reinterpret_cast<uint16_t*>(tile + value_parameters<D>(t, group) + 16) = own.v_low;
        }
    }
}

// --------------------------------------------------------------------------- norm, rotation and append
struct RotatedArgs {
    CopyArgs copy;                  // k, v and the sequences
    Heads q, q_out, k_out;          // (k_out: no pointer, not wanted)
    const uint16_t *q_weight, *k_weight;
    const float* table;
    const int32_t* positions;       // none: a token's place in its sequence
    int64_t n_positions;
    int q_heads, turned;            // turned: rotary_dim / 16
    float eps;
};

// The append with its rotation: 8192 tokens of 32 query heads and 8 of the cache take 49 us (178 MB, 34 at the rate of a copy); norm and rotation, and append, in launches of
// their own some 50 (34 and 16), and a launch more.  One token of 32 heads takes 5.5.  Bound: for prompts by the vector units, busy for 60 % of the cycles,
// and memory (3.7 TB/s) in turn: the workgroups of the cache alone take 22 us, those of the queries alone 37, both without norms 45; for single tokens by the chain of waits
// (lengths -> page -> rows and positions -> table -> LDS -> tile).  They come first in the grid: taken in turn
// with those of the queries 64 us instead of 61 with the read.
//
// Query heads of one workgroup: kQuerySets times what a wavefront takes of a row at once, 16 elements a lane; a wavefront takes one row.
// (1, 2, 4 sets: 8192 tokens 72, 61, 61 us with the read, 501 rows of 28 heads of 64 11.5, 10.7, 11.1.)
constexpr int kQuerySets = 2, kQueryRows = kThreads / 64;
constexpr int query_heads_of(int head_dim) { return kQuerySets * 1024 / head_dim; }

// 1 / sqrt(x) in 64 bits, from the hardware's estimate by one step (a start that is off by 2^-14 or less leaves 2^-27, two 2^-52; the estimate is far better),
// and rounded to 32: a factor that does not depend on the order in which the squares were added.
__device__ __forceinline__ float root_of(double x)
{
    const double y = __builtin_amdgcn_rsq(x);
    double z = y * __builtin_fma(-0.5 * x * y, y, 1.5);
    z = z * __builtin_fma(-0.5 * x * z, z, 1.5);
    return static_cast<float>(x > 0.0 && x < __builtin_inf() ? z : y);
}

// The rotation of one token as D / 16 lanes need it: lane p has two runs of 8 elements of a head that are each other's partners, so that nothing is exchanged but the norm's sum.
template <int D, bool INTERLEAVED>
struct Turn {
    static constexpr int kLanes = D / 16;
    int run_a, run_b;
    bool turns;
    float4_t by[4];             // cosine and sine of the lane's 8 pairs

    __device__ __forceinline__ Turn(const RotatedArgs& a, int p, int64_t row, int token)
    {
        turns = p < a.turned;
        run_a = INTERLEAVED || !turns ? 2 * p : p, run_b = INTERLEAVED || !turns ? 2 * p + 1 : p + a.turned;
        if (!turns) return;
        const int position = a.positions ? a.positions[row] : token;
#pragma unroll
        for (int i = 0; i < 4; ++i) by[i] = __builtin_nanf("") + float4_t{};
        if (position < 0 || position >= a.n_positions) return;      // (nothing is read for it: a table may have no rows at all)
        const float4_t* table = reinterpret_cast<const float4_t*>(a.table + (static_cast<int64_t>(position) * a.turned + p) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) by[i] = table[i];
    }

    struct Runs {
        half8_t a, b;
    };
    __device__ __forceinline__ Runs load(const uint16_t* head) const { return {*reinterpret_cast<const half8_t*>(head + 8 * run_a), *reinterpret_cast<const half8_t*>(head + 8 * run_b)}; }
    __device__ __forceinline__ void store(uint16_t* head, const Runs& x) const
    {
        *reinterpret_cast<half8_t*>(head + 8 * run_a) = x.a;
        *reinterpret_cast<half8_t*>(head + 8 * run_b) = x.b;
    }

    // (called by all lanes of the head)
    __device__ __forceinline__ Runs apply(const Runs& from, const uint16_t* weight, float eps) const
    {
        float x[2][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[0][i] = static_cast<float>(from.a[i]), x[1][i] = static_cast<float>(from.b[i]);
        if (weight) {
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const double v = static_cast<double>(x[i / 8][i % 8]);
                sum = __builtin_fma(v, v, sum);
            }
#pragma unroll
            for (int d = 1; d < kLanes; d *= 2) sum += __shfl_xor(sum, d);
            const float factor = root_of(sum * (1.0 / D) + static_cast<double>(eps));
            const Runs w = load(weight);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[0][i] *= factor * static_cast<float>(w.a[i]), x[1][i] *= factor * static_cast<float>(w.b[i]);
        }
        if (turns) {
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float c = by[2 * r + i / 2][2 * (i % 2)], s = by[2 * r + i / 2][2 * (i % 2) + 1], u = x[r][2 * i], v = x[r][2 * i + 1];
                        x[r][2 * i] = u * c - v * s, x[r][2 * i + 1] = u * s + v * c;
                    }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float c = by[i / 2][2 * (i % 2)], s = by[i / 2][2 * (i % 2) + 1], u = x[0][i], v = x[1][i];
                    x[0][i] = u * c - v * s, x[1][i] = u * s + v * c;
                }
            }
        }
        Runs to;
#pragma unroll
        for (int i = 0; i < 8; ++i) to.a[i] = static_cast<_Float16>(x[0][i]), to.b[i] = static_cast<_Float16>(x[1][i]);
        return to;
    }
};

// One workgroup per tile that gets rows, and head of the cache: 8 threads to a token, which norm and rotate its key as Turn has it, hand it over by way of LDS to have a run of its
// elements each, and quantise these; or per kQueryRows rows of a tile and several query heads.
template <int D, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void append_rotated_kernel(RotatedArgs a)
{
    constexpr int kOwn = D / 8, kRuns = kOwn / 8, kLanes = D / 16;
    __shared__ TileImage<D> shared;
    __shared__ alignas(16) uint16_t keys[kTileTokens][D + 8];
    Unit u;
    if (!unit_of(a.copy, &u)) return;
    const int tile_token = u.tile * kTileTokens, first = u.seq.length - u.seq.rows - tile_token;       // the rows' first token, from the tile's on
    const int from = max(first, 0), to = min(u.seq.length - tile_token, kTileTokens);

    if (static_cast<int>(blockIdx.y) >= a.copy.pool.kv_heads) {
        const int of = blockIdx.y - a.copy.pool.kv_heads, lane = threadIdx.x & 63;
        const int t = of % (kTileTokens / kQueryRows) * kQueryRows + (threadIdx.x >> 6), head0 = of / (kTileTokens / kQueryRows) * query_heads_of(D) + lane / kLanes;
        if (t < from || t >= to) return;
        const int64_t row = u.seq.start + (t - first);
        const Turn<D, INTERLEAVED> turn(a, lane % kLanes, row, tile_token + t);
        const uint16_t* q = a.q.data + row * a.q.row;
        typename Turn<D, INTERLEAVED>::Runs x[kQuerySets] = {};
#pragma unroll
        for (int i = 0; i < kQuerySets; ++i)
            if (head0 + i * (64 / kLanes) < a.q_heads) x[i] = turn.load(q + (head0 + i * (64 / kLanes)) * a.q.head);
#pragma unroll
        for (int i = 0; i < kQuerySets; ++i) {
            const int head = head0 + i * (64 / kLanes);
            const auto y = turn.apply(x[i], a.q_weight, a.eps);
            if (head < a.q_heads) turn.store(a.q_out.data + row * a.q_out.row + head * a.q_out.head, y);
        }
        return;
    }

    const int t = threadIdx.x >> 3, part = threadIdx.x & 7;
    const bool fresh = t >= from && t < to;
    Codes<D> codes{};
    if (fresh) {
        const int64_t row = u.seq.start + (t - first);
        const uint16_t* v_at = a.copy.v.data + row * a.copy.v.row + u.head * a.copy.v.head + part * kOwn;
        half8_t x[kRuns], y[kRuns];
#pragma unroll
        for (int r = 0; r < kRuns; ++r) y[r] = reinterpret_cast<const half8_t*>(v_at)[r];
        if (part < kLanes) {        // (with heads of 64 half of the threads)
            const Turn<D, INTERLEAVED> turn(a, part, row, tile_token + t);
            const auto key = turn.apply(turn.load(a.copy.k.data + row * a.copy.k.row + u.head * a.copy.k.head), a.k_weight, a.eps);
            if (a.k_out.data) turn.store(a.k_out.data + row * a.k_out.row + u.head * a.k_out.head, key);
            turn.store(keys[t], key);
        }
        // (a token's threads are of one wavefront, whose operations LDS takes in order)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int r = 0; r < kRuns; ++r) x[r] = *reinterpret_cast<const half8_t*>(&keys[t][part * kOwn + 8 * r]);
        const Quantised<kOwn> k = quantise<kOwn>(x);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) codes.k_words[i / 8] |= k.code[i] << nibble(i % 8);
        codes.k_parameters = __builtin_bit_cast(uint32_t, half2_t{k.low, k.step});
        const Quantised<kOwn> v = quantise<kOwn>(y);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) codes.v_bytes[i / 4] |= v.code[i] << 8 * (i % 4);
        codes.v_step = __builtin_bit_cast(uint16_t, v.step), codes.v_low = __builtin_bit_cast(uint16_t, v.low);
    }
    if (u.page < 0 || to <= from) return;
    const uint32_t below = to == kTileTokens ? ~0u : (1u << to) - 1u;
    put_tile<D>(a.copy.pool.tile<D>(u.page, u.head, u.tile), below & ~((1u << from) - 1u), codes, shared);
}

// --------------------------------------------------------------------------- tokens moved within the cache
struct KeepArgs {
    Pool pool;
    Sequences seqs;
    const int32_t *path, *accepted;
};

// Codes and parameters are moved as they are: quantised anew, a token's values would move too.  8 rows of 32 heads take 4 us, 16 sequences of up to 64 rows of 8 heads 5:
// launch and the chain lengths -> path -> page -> words -> LDS -> tile; bytes do not count.
// One workgroup per sequence and head.  Tile by tile of the tokens that are written, from the first on: what goes into a tile is read before it is written,
// and a token is never taken from a place before its own, so nothing is read that an earlier tile has written.
template <int D>
__global__ __launch_bounds__(kThreads) void keep_kernel(KeepArgs a)
{
    constexpr int kOwn = D / 8;
    __shared__ TileImage<D> shared;
    const int b = blockIdx.x, head = blockIdx.y;
    const Sequence seq = sequence(a.seqs, INT_MAX, b);
    const int kept = min(a.accepted[b], seq.rows - 1) + 1, before = seq.length - seq.rows;
    if (kept <= 0) return;
    const int t = threadIdx.x >> 3, part = threadIdx.x & 7, group = part * kOwn / kGroupChannels;
    const int32_t* pages = a.seqs.pages + int64_t{b} * a.seqs.max_pages;
    const auto tile_of = [&](int tile) -> uint8_t* {
        const int of = tile >> (a.pool.page_shift - 5);
        if (tile < 0 || of >= a.seqs.max_pages) return nullptr;
        const int page = pages[of];
        return page >= 0 && page < a.pool.n_pages ? a.pool.tile<D>(page, head, tile) : nullptr;
    };
    for (int tile = max(before, 0) >> 5; tile <= (before + kept - 1) >> 5; ++tile) {
        const int i = tile * kTileTokens + t - before;
        const int of = i >= 0 && i < kept ? a.path[seq.start + i] : -1;
        uint8_t* to = tile_of(tile);
        const int token = before + of;
        const uint8_t* source = of > i && of < seq.rows && i >= 0 ? tile_of(token >> 5) : nullptr;
        const bool moves = to && source;
        Codes<D> codes{};
        if (moves) {
            const int s = token & 31, quad = s >> 2 & 3, shift = 8 * (s & 3) + 4 * (s >> 4);
#pragma unroll
            for (int r = 0; r < kOwn / 8; ++r) codes.k_words[r] = *reinterpret_cast<const uint32_t*>(source + key_word<D>(s, part * kOwn + 8 * r));
#pragma unroll
            for (int e = 0; e < kOwn; ++e) {
                const int element = part * kOwn + e;
                const uint32_t word = *reinterpret_cast<const uint32_t*>(source + 16 * D + word_offset(element / 16, quad * 16 + element % 16));
                codes.v_bytes[e / 4] |= (word >> shift & 15u) << 8 * (e % 4);
            }
            codes.k_parameters = *reinterpret_cast<const uint32_t*>(source + key_parameters<D>(s, group));
            codes.v_step = *reinterpret_cast<const uint16_t*>(source + value_parameters<D>(s, group));
            codes.v_low = *reinterpret_cast<const uint16_t*>(source + value_parameters<D>(s, group) + 16);
        }
        // a wavefront has 8 tokens
        __shared__ uint32_t fresh_of[kThreads / 64];
        const uint64_t lanes = __builtin_amdgcn_ballot_w64(moves && part == 0);
        if ((threadIdx.x & 63) == 0) {
            uint32_t eight = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) eight |= static_cast<uint32_t>(lanes >> 8 * j & 1) << j;
            fresh_of[threadIdx.x >> 6] = eight;
        }
        __syncthreads();        // (and every source has been read)
        const uint32_t fresh = fresh_of[0] | fresh_of[1] << 8 | fresh_of[2] << 16 | fresh_of[3] << 24;
        if (fresh != 0) put_tile<D>(to, fresh, codes, shared);
        __syncthreads();
    }
}

template <int D>
void launch_append(const RotatedArgs& a, bool interleaved, dim3 grid, hipStream_t s)
{
    if (interleaved) hipLaunchKernelGGL((append_rotated_kernel<D, true>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((append_rotated_kernel<D, false>), grid, dim3(kThreads), 0, s, a);
}

}  // namespace

gqsa_status_t cache_append_rotated(gqsa_cache* c, const RotateCall& call, const Heads& v, const Sequences& seqs, void* stream)
{
    if (gqsa_status_t st = on_device(c)) return st;
    const RotatedArgs a{{pool_of(c), call.k, v, seqs}, call.q, call.q_out, call.k_out, call.q_weight, call.k_weight, call.table, call.positions,
                        call.n_positions, call.q_heads, call.rotary_dim / 16, call.eps};
    dim3 grid = copy_grid(c, seqs);
    grid.y += kTileTokens / kQueryRows * ((call.q_heads + query_heads_of(c->head_dim) - 1) / query_heads_of(c->head_dim));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (c->head_dim == 128) launch_append<128>(a, call.interleaved != 0, grid, s);
    else launch_append<64>(a, call.interleaved != 0, grid, s);
    GQSA_HIP(hipGetLastError());
    return GQSA_OK;
}

gqsa_status_t cache_keep(gqsa_cache* c, const Sequences& seqs, const int32_t* path, const int32_t* accepted, void* stream)
{
    if (gqsa_status_t st = on_device(c)) return st;
    const KeepArgs a{pool_of(c), seqs, path, accepted};
    const dim3 grid(static_cast<unsigned>(seqs.n_seqs), static_cast<unsigned>(c->kv_heads));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (c->head_dim == 128) hipLaunchKernelGGL(keep_kernel<128>, grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL(keep_kernel<64>, grid, dim3(kThreads), 0, s, a);
    GQSA_HIP(hipGetLastError());
    return GQSA_OK;
}

}  // namespace gqsa
