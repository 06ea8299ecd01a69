// Causal attention over packed prompts with grouped heads (gqsa_prompt_attend): o = softmax(scale q K^T) V, a row over the keys up to
// its own.  One pass over the keys with the running maximum and sum of each row; scores never leave the registers.
//
// A workgroup of 4 wavefronts takes 128 query rows of one head, a wavefront 32 of them; keys and values come in tiles of 64, copied from
// memory straight into LDS, one tile ahead of the one at work.  Both products are 32x32x16 ones, taken the other way round --
// S^T = K Q^T, O^T = V^T P^T -- because then a lane holds scores of one query row only (its maximum and sum need one exchange, between the two
// halves of the wavefront) and holds them as the second product wants its operand; V^T comes out of LDS by transposing reads.
//
// Long prompts are bound by what the matrix cores and the vector units do in turn: 8192 tokens of 32 heads of 128 for 8 (550 GFLOP) take 541 to 566 us, by the card's
// clock, 1016 to 971 TFLOP/s, where a large library product of fp16 reaches 1113; the matrix cores are busy for 53 % of the cycles and the vector units for 46 %.  Without
// its copies into LDS the kernel takes 502 of 546 us, copies alone 196.  Each exponential costs as much as two other instructions, and a tile has 64 of them for
// every 64 lanes' row; with the weights' sum by dot products of what the second product takes, and the reference that follows only now and then, little else is
// left beside it.  Ragged batches pay for blocks that are not full -- the last of a sequence goes through all its keys, with one wavefront of four at work where it
// has a few rows -- and for the end, when few blocks are left: 7 sequences of up to 2500 tokens, 40 heads for 8, take 290 to 299 us, 781 to 757 TFLOP/s of the scores that the mask
// leaves.  Counted in tiles a workgroup's share is 16 % more than those scores, the longest row of blocks on one of 512 places 19 %; both units together are busy for 78 % of the cycles.
// One short prompt is a chain of waits: 15 tokens of 32 heads 5.3 us.  In between, one block's keys in turn set the time: 1000 tokens of 40 heads 27 us, 385 TFLOP/s of 1113.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "gqsa_device.hpp"

namespace gqsa {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kWaveRows = 32;       // query rows of a wavefront
constexpr int kTileKeys = 64;

typedef short short4_t __attribute__((ext_vector_type(4)));

// Where a row of a tile keeps its run `chunk` of 8 elements.  Keys: 16 neighbouring rows read the same run, so the runs are spread by the
// row over all banks; values: 4 neighbouring rows read 4 neighbouring runs.
template <int D>
__device__ __forceinline__ int key_place(int row, int chunk) { return chunk ^ (D == 128 ? row & 15 : (row >> 1) & 7); }
template <int D>
__device__ __forceinline__ int value_place(int row, int chunk) { return chunk ^ (D == 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1)); }

template <int D>
struct alignas(256) PromptShared {
    uint16_t k[2][kTileKeys * D], v[2][kTileKeys * D];
};

__device__ __forceinline__ uint32_t lds_address(const void* p)
{
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) uint8_t*)p));
}

// N KiB from memory into LDS at `to`, a KiB at a time: 16 bytes a lane from `from` + at[i].  (The first wait states are for scalar registers
// that a vector instruction may have written just before, which the compiler does not see to inside a statement; one is for m0.)
template <int N>
__device__ __forceinline__ void copy_in(uint32_t to, uint64_t from, const uint32_t (&at)[N])
{
    static_assert(N == 2 || N == 4, "");
    if constexpr (N == 4)
        asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %2, %1\n\t"
                     "s_add_u32 m0, m0, 1024\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %1\n\t"
                     "s_add_u32 m0, m0, 1024\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %1\n\t"
                     "s_add_u32 m0, m0, 1024\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %5, %1"
                     : "+{m0}"(to) : "s"(from), "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]) : "memory", "scc");
    else
        asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %2, %1\n\t"
                     "s_add_u32 m0, m0, 1024\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %1"
                     : "+{m0}"(to) : "s"(from), "v"(at[0]), "v"(at[1]) : "memory", "scc");
}

// Whether one of eight numbers is an infinity or a NaN: where the exponent's bits are all set, adding its lowest one carries into the sign's place.
__device__ __forceinline__ bool some_not_finite(u32x4_t x)
{
    uint32_t over = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) over |= (x[e] & 0x7C007C00u) + 0x04000400u;
    return (over & 0x80008000u) != 0;
}

// The same of this thread's part of a tile of values.
template <int D>
__device__ __forceinline__ bool some_not_finite(const uint16_t* tile)
{
    bool some = false;
#pragma unroll
    for (int i = 0; i < kTileKeys * D / 8 / kThreads; ++i) some |= some_not_finite(*reinterpret_cast<const u32x4_t*>(tile + (i * kThreads + threadIdx.x) * 8));
    return some;
}

// Numbers that are not finite as 0.
__device__ __forceinline__ half8_t finite_part(half8_t v)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_fabsf16(v[i]) <= static_cast<_Float16>(65504.0f) ? v[i] : static_cast<_Float16>(0.0f);
    return v;
}

// Infinite values.  A row's element is infinite if the row sees one there, and NaN if it sees a NaN or both infinities, whatever the weights; but the product makes NaN of an infinity
// whose weight is rounded to 0, and so does a rescaling by 0 later on.  So elements that see values which are not finite are written anew, as the sum of those
// values; `to` is where the lane's first element went, null if its row is to stay as it is.  (Called by whole wavefronts, seldom: the wavefront goes once more through
// its rows' values, 64 keys at a time, and looks closer at keys that hold such a value.)
template <int D>
__device__ __forceinline__ void write_not_finite(const uint16_t* v, int64_t v_row, int keys, int sees, int lane, uint16_t* to)
{
    constexpr int kLanes = D / 8, kAtOnce = 64 / kLanes;        // lanes to a key, keys to a load of 16 bytes a lane
    float16_t sum[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d) sum[d] = float16_t{};
    for (int first = 0; first < keys; first += 64) {
        uint32_t odd = 0;           // bit i: this lane's part of key first + i kAtOnce + lane / kLanes
        u32x4_t x[64 / kAtOnce];
#pragma unroll
        for (int i = 0; i < 64 / kAtOnce; ++i)
            x[i] = *reinterpret_cast<const u32x4_t*>(v + min(first + i * kAtOnce + lane / kLanes, keys - 1) * v_row + 8 * (lane % kLanes));
#pragma unroll
        for (int i = 0; i < 64 / kAtOnce; ++i) odd |= (some_not_finite(x[i]) ? 1u : 0u) << i;
        if (!__any(odd)) continue;
        for (int i = 0; i < 64; ++i) {
            const int key = first + i;
            const bool mine = lane / kLanes == i % kAtOnce && (odd >> (i / kAtOnce) & 1);
            if (key >= keys || !__any(mine)) continue;
            const uint16_t* at = v + key * v_row + 4 * (lane >> 5);
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const half4_t y = *reinterpret_cast<const half4_t*>(at + 32 * d + 8 * r);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float value = static_cast<float>(y[e]);
                        if (key < sees && !(__builtin_fabsf(value) < __builtin_inff())) sum[d][4 * r + e] += value;
                    }
                }
        }
    }
    if (!to) return;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (!(sum[d][r] == 0.0f)) to[32 * d + 8 * (r >> 2) + (r & 3)] = __builtin_bit_cast(uint16_t, static_cast<_Float16>(sum[d][r]));
}

// The slot-th of the blocks of up to 64 sequences in the order of the keys they see, the most first: `level` is how many times ROWS those are, the last block of
// lane l's sequence is at level ends of lane l, the one before it a level lower, and so on.
template <int ROWS, typename Deal>
__device__ __forceinline__ auto longest_first(const Deal& deal, unsigned slot, int* b, int* block)
{
    const unsigned ends = max(static_cast<unsigned>(deal.seq.length + ROWS - 1) / ROWS, deal.own);
    const auto above = [&](unsigned level) { return Deal::last(running_sum(min(ends > level ? ends - level : 0u, deal.own))); };
    unsigned low = 0, level = largest(deal.own ? ends : 0u), before = 0;       // above(low) > slot, above(level) = before <= slot
    while (level - low > 1) {
        const unsigned middle = (low + level) / 2, n = above(middle);
        if (n > slot) low = middle;
        else level = middle, before = n;
    }
    const uint64_t there = __builtin_amdgcn_ballot_w64(ends >= level && level + deal.own > ends);
    const unsigned rank = __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(there >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(there), 0));
    const int who = __builtin_ctzll(there & __builtin_amdgcn_ballot_w64(rank == slot - before));
    *b = who;
    *block = __builtin_amdgcn_readlane(static_cast<int>(deal.own + level - ends), who) - 1;
    auto seq = deal.seq;
    seq.start = __builtin_amdgcn_readlane(seq.start, who), seq.rows = __builtin_amdgcn_readlane(seq.rows, who);
    seq.length = __builtin_amdgcn_readlane(seq.length, who);
    return seq;
}

// SPLIT: how many wavefronts share their rows, each with every SPLIT-th part of a tile's keys.  With 2 a workgroup has 64 rows instead of 128.
template <int D, int SPLIT>
__global__ __launch_bounds__(kThreads, 2) void prompt_kernel(PromptCall c, bool negate, bool mixed)
{
    constexpr int kGroups = kWaves / SPLIT, kBlockRows = kGroups * kWaveRows;
    constexpr int kPieces = 2 / SPLIT;               // runs of 32 keys of a tile that a wavefront takes
    constexpr int kCopies = D / 32;                  // KiB of a tile of keys that a wavefront copies
    constexpr int kCopyRows = 512 / D;               // rows in one of them
    constexpr int kLanesPerRow = D / 8;
    __shared__ PromptShared<D> shared;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5;
    const int group = wave % kGroups, part = wave / kGroups;

    struct Prompt {
        int start, rows, length;       // query rows, and where they start; keys
    };
    const auto rows_of = [](const int32_t* starts, int64_t n, int b) { return rows_between(starts[b], starts[b + 1], n); };
    // Heads vary fastest, those of a group on one XCD (workgroup i runs on XCD i % 8); blocks with more keys come first, of each
    // sequence or (mixed) of all, so that what runs last is short.
    const unsigned slot = blockIdx.x / static_cast<unsigned>(c.q_heads), of = blockIdx.x % static_cast<unsigned>(c.q_heads);
    const int head = c.q_heads % 8 == 0 ? of % 8 * (c.q_heads / 8) + of / 8 : of;
    const auto deal = deal_out<Prompt>(c.n_seqs, lane, [&](int b) {
        const Rows q_rows = rows_of(c.q_starts, c.n_q_rows, b);
        return Prompt{q_rows.start, q_rows.count, rows_of(c.k_starts, c.n_k_rows, b).count};
    }, [](const Prompt& p) { return static_cast<unsigned>(p.rows + kBlockRows - 1) / kBlockRows; });
    if (slot >= deal.total) return;
    int b, block;
    Prompt prompt;
    if (mixed) prompt = longest_first<kBlockRows>(deal, slot, &b, &block);
    else prompt = deal.locate(deal.total - 1 - slot, &b, &block);
    const int q_start = prompt.start, n_q = prompt.rows, n_k = prompt.length, k_start = rows_of(c.k_starts, c.n_k_rows, b).start;
    const int behind = n_k - n_q;                    // row r sees keys 0 .. r + behind
    const int row0 = block * kBlockRows, wave_row0 = row0 + group * kWaveRows;
    const int row = wave_row0 + (lane & 31);
    const int sees = row + behind + 1;
    const int keys = max(min(n_q, row0 + kBlockRows) + behind, 0);                               // that some row of the block sees
    const int wave_keys = wave_row0 < n_q ? max(min(n_q, wave_row0 + kWaveRows) + behind, 0) : 0;
    const int tiles = (keys + kTileKeys - 1) / kTileKeys;

    // the query rows, and what this lane copies of a tile
    half8_t q[D / 16];
    const uint16_t* q_at = c.q.data + (int64_t{q_start} + min(row, n_q - 1)) * c.q.row + head * c.q.head + 8 * half;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) q[i] = *reinterpret_cast<const half8_t*>(q_at + 16 * i);
    if (negate) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) q[i] = -q[i];
    }
    const int kv_head = head / (c.q_heads / c.kv_heads);
    const uint64_t k_from = reinterpret_cast<uint64_t>(c.k.data + int64_t{k_start} * c.k.row + kv_head * c.k.head);
    const uint64_t v_from = reinterpret_cast<uint64_t>(c.v.data + int64_t{k_start} * c.v.row + kv_head * c.v.head);
    const auto copy = [&](int tile, int buffer) {
        uint32_t k_lane[kCopies], v_lane[kCopies];
        const int last = n_k - 1 - tile * kTileKeys;      // keys that do not exist are the last one again: no row sees them
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int r = kCopies * kCopyRows * wave + kCopyRows * i + lane / kLanesPerRow, at = lane % kLanesPerRow;
            k_lane[i] = 2u * (static_cast<uint32_t>(min(r, last)) * static_cast<uint32_t>(c.k.row) + 8u * key_place<D>(r, at));
            v_lane[i] = 2u * (static_cast<uint32_t>(min(r, last)) * static_cast<uint32_t>(c.v.row) + 8u * value_place<D>(r, at));
        }
        const uint32_t to = wave * kCopies * 1024u;
        copy_in<kCopies>(lds_address(shared.k[buffer]) + to, k_from + uint64_t{2} * (uint64_t{static_cast<uint32_t>(tile * kTileKeys)} * static_cast<uint64_t>(c.k.row)), k_lane);
        copy_in<kCopies>(lds_address(shared.v[buffer]) + to, v_from + uint64_t{2} * (uint64_t{static_cast<uint32_t>(tile * kTileKeys)} * static_cast<uint64_t>(c.v.row)), v_lane);
    };

    float16_t out[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i) out[i] = float16_t{};
    float top = kMinusInf, sum = 0.0f;          // the scores' reference, the weights' sum
    bool wild = false;

    if (tiles > 0) copy(0, 0);
    for (int tile = 0; tile < tiles; ++tile) {
        const int buffer = tile & 1, first = tile * kTileKeys;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // this wavefront's part of the tile has arrived,
        __syncthreads();                                       // everybody's has, and nobody reads the other buffer any more
        if (tile + 1 < tiles) copy(tile + 1, buffer ^ 1);
        const int mine = first + 32 * kPieces * part;          // this wavefront's first key
        const bool active = mine < wave_keys;                 // (the same for a whole wavefront)
        const uint16_t *k_tile = shared.k[buffer], *v_tile = shared.v[buffer];
        // The two (with keys of an earlier part three) tiles that some rows see in part: a weight of 0 would not keep the other rows from values that are not
        // finite.  The product takes 0 in their place; what they make of the rows that see them is seen to at the end.
        if (first + kTileKeys > row0 + behind + 1 && __builtin_expect(__syncthreads_or(some_not_finite<D>(v_tile)), 0)) {
            wild = true;
#pragma unroll
            for (int i = 0; i < kTileKeys * D / 8 / kThreads; ++i) {
                half8_t* at = reinterpret_cast<half8_t*>(&shared.v[buffer][(i * kThreads + threadIdx.x) * 8]);
                *at = finite_part(*at);
            }
            __syncthreads();
        }
        if (!active) continue;

        float16_t s[kPieces];
#pragma unroll
        for (int j = 0; j < kPieces; ++j) s[j] = float16_t{};
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                const int r = 32 * (kPieces * part + j) + (lane & 31);
                const half8_t k = *reinterpret_cast<const half8_t*>(k_tile + r * D + 8 * key_place<D>(r, 2 * i + half));
                s[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q[i], s[j], 0, 0, 0);
            }
        }
        // element r of s[j] is key 32 j + r % 4 + 8 (r / 4) + 4 half of the wavefront's
        if (mine + 32 * kPieces > wave_row0 + behind + 1) {
#pragma unroll
            for (int j = 0; j < kPieces; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (mine + 32 * j + (r & 3) + 8 * (r >> 2) + 4 * half >= sees) s[j][r] = kMinusInf;
        }
        float most = kMinusInf;
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, s[j][r]);
        most *= c.scale;
        if (__any(most > top + (kRoom + kSlack) || (top == kMinusInf && most > kMinusInf))) {
            most = fmaxf(most, __shfl_xor(most, 32));
            const float higher = fmaxf(top, most - kRoom);
            const float shrink = higher == kMinusInf ? 1.0f : __builtin_amdgcn_exp2f(top - higher);
            top = higher;
            sum *= shrink;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) out[i] *= shrink;
        }
        const float reference = top == kMinusInf ? 0.0f : top;
        half8_t p[2 * kPieces];
#pragma unroll
        for (int i = 0; i < 2 * kPieces; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[i][e] = static_cast<_Float16>(__builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 1][8 * (i & 1) + e], c.scale, -reference)));
            }
        // (the sum of the weights as the product has them, rounded: half the additions)
        const half2_t ones = {static_cast<_Float16>(1.0f), static_cast<_Float16>(1.0f)};
#pragma unroll
        for (int i = 0; i < 2 * kPieces; ++i)
#pragma unroll
            for (int e = 0; e < 8; e += 2) sum = __builtin_amdgcn_fdot2(half2_t{p[i][e], p[i][e + 1]}, ones, sum, false);
        __builtin_amdgcn_s_setprio(1);      // (products ahead of the other wavefronts' softmax: 1.5 % at 8192 tokens, -3 to 1 % at fewer)
        // The operand V^T: 16 lanes read 4 keys x 16 elements, each 4 elements of a key, and get 4 keys of an element each.
        const auto turned = [&](const uint16_t* tile, int i, int d) {
            short4_t part[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = 16 * i + 8 * h + 4 * half + ((lane & 15) >> 2), e = 32 * d + (lane & 16) + 4 * (lane & 3);
                const uint16_t* at = tile + r * D + 8 * value_place<D>(r, e >> 3) + (e & 7);
                part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t*)at);
            }
            return __builtin_shufflevector(__builtin_bit_cast(half4_t, part[0]), __builtin_bit_cast(half4_t, part[1]), 0, 1, 2, 3, 4, 5, 6, 7);
        };
#pragma unroll
        for (int i = 0; i < 2 * kPieces; ++i)
#pragma unroll
            for (int d = 0; d < D / 32; ++d) out[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(turned(v_tile, 2 * kPieces * part + i, d), p[i], out[d], 0, 0, 0);
        __builtin_amdgcn_s_setprio(0);
    }

    sum += __shfl_xor(sum, 32);
    if constexpr (SPLIT > 1) {
        // the other part of the keys, by way of LDS
        float* meet = reinterpret_cast<float*>(&shared) + group * (16 * (D / 32) + 2) * 64 + lane;
        __syncthreads();
        if (part == 1) {
            meet[0] = top, meet[64] = sum;
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) meet[(2 + 16 * d + r) * 64] = out[d][r];
        }
        __syncthreads();
        if (part == 1) return;
        const float other = meet[0], both = fmaxf(top, other);
        const float f = top == kMinusInf ? 0.0f : __builtin_amdgcn_exp2f(top - both), g = other == kMinusInf ? 0.0f : __builtin_amdgcn_exp2f(other - both);
        sum = f * sum + g * meet[64];
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) out[d][r] = f * out[d][r] + g * meet[(2 + 16 * d + r) * 64];
    }
    // (from the lane's number anew: kept from the loop's start, it would take registers from the loop, up to 5 %)
    int own_lane = lane;
    asm volatile("" : "+v"(own_lane));
    const int own_row = wave_row0 + (own_lane & 31);
    float largest_out = 0.0f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) largest_out = __builtin_elementwise_maximum(largest_out, __builtin_fabsf(out[d][r]));
    // (a row without keys: all sums are 0; one with scores of -infinity only is NaN)
    const float inverse = own_row + behind < 0 ? 0.0f : sum == 0.0f ? __builtin_nanf("") : 1.0f / sum;
    uint16_t* to = c.out.data + (int64_t{q_start} + own_row) * c.out.row + head * c.out.head + 4 * (own_lane >> 5);
    if (own_row < n_q) {
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                half4_t y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = static_cast<_Float16>(out[d][4 * r + e] * inverse);
                *reinterpret_cast<half4_t*>(to + 32 * d + 8 * r) = y;
            }
    }
    // The second look stands behind the stores: ahead of them, its instructions would have to be jumped over (128 tokens of 32 heads 8.0 us instead of 7.7).  A row whose sum is
    // not finite, or that has scores of -infinity only, is NaN throughout and stays so.
    const bool sound = sum > 0.0f && sum < __builtin_inff();
    if (__builtin_expect(wild || __any(!(largest_out < __builtin_inff()) && sound), 0))
        write_not_finite<D>(reinterpret_cast<const uint16_t*>(v_from), c.v.row, wave_keys, own_row + behind + 1, own_lane, own_row < n_q && sound ? to : nullptr);
}

}  // namespace

gqsa_status_t prompt_attend(const PromptCall& call, void* stream)
{
    PromptCall c = call;
    const bool negate = c.scale < 0.0f;     // of the queries instead: the largest score is then the one of the largest product
    // (the softmax is taken to base 2; not 0, so that a masked score stays -infinity: 1e-30 leaves every weight at 1)
    c.scale = std::max(std::fabs(c.scale) * 1.44269504088896341f, 1e-30f);
    // Few workgroups: rows shared by two wavefronts, so that there are twice as many.  us of own / shared rows, heads of 128, by the workgroups of 128 rows
    // (bound below):
    //   keys of 1000 and more: 32: 1 row, 2000 keys, 32 heads 44.1 / 32.2; 224: 2000 x 14 heads 52.9 / 40.0; 256: 2000 rows, 4000 keys, 16 heads 97.7 / 82.0; 320: 1000 x 40
    //     29.7 / 26.7; 352: 1300 x 32 34.5 / 29.0; 384: 1500 x 32 42.0 / 36.4; 448: 4000 x 14 96.9 / 85.3; 576: 1024 x 64 32.4 / 34.5; 2080: 8192 x 32 for 8 543 / 652;
    //   fewer: 64: 128 x 32 8.0 / 7.6; 96: 256 x 32 10.5 / 9.3; 192: 700 x 32 19.3 / 17.5; 256: 900 x 32 23.6 / 20.5; 320: 4 x 194 x 32 10.3 / 11.6; 384: 700 x 64 23.0 / 23.0;
    //     392: 2 x 800 x 28 28.1 / 27.0; 448: 8 x 100 x 32 8.4 / 9.6; one tile of keys (15 x 32) 5.2 / 5.8, 16 x 64 x 14 6.5 / 7.5.
    // (Four tiles in LDS instead of two, where every workgroup has a compute unit for itself, took 1.1 to 1.25 times as long.)
    const auto blocks_of = [&](int rows) { return (c.n_q_rows / rows + c.n_seqs) * c.q_heads; };      // no fewer than there are
    const int64_t whole = blocks_of(kWaves * kWaveRows), half = blocks_of(kWaves * kWaveRows / 2);
    const bool split = c.n_k_rows > kTileKeys * int64_t{c.n_seqs} && whole <= (c.n_k_rows >= int64_t{1000} * c.n_seqs ? 512 : 256);
    const int64_t blocks = split ? half : whole;
    if (blocks > (int64_t{1} << 23)) return GQSA_ERR_SHAPE;
    // Blocks of all sequences in the order of their keys, not one sequence after the other, where more of them than run at once would otherwise end with a
    // long one -- us of either order, ragged lengths up to: 6 x 900, 32 heads for 8 63.4 / 61.2; 12 x 800 68.3 / 68.4; 30 x 500 72.8 / 72.0; 3 x 1500 52.2 / 50.2; 20 x 1000, 14 heads
    // of 64 36.7 / 31.0 -- but not where the keys and values that an XCD's workgroups are at would then pass its L2 (4 MiB): 7 x 2500, 40 heads 294 / 300 or, of other lengths,
    // 235 / 231; 12 x 3000 397 / 394; nor where a sequence is a block or so, as 64 x 40: 21.6 / 21.2.
    const int64_t heads_at_once = (c.kv_heads + 7) / 8;
    const bool mixed = !split && c.n_seqs > 1 && c.n_seqs <= 64 && blocks > 512 && c.n_k_rows >= int64_t{kWaves} * kWaveRows * c.n_seqs &&
                       c.n_k_rows * c.head_dim * 4 * heads_at_once <= (int64_t{4} << 20);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 grid(static_cast<unsigned>(blocks));
    if (c.head_dim == 128) {
        if (split) hipLaunchKernelGGL((prompt_kernel<128, 2>), grid, dim3(kThreads), 0, s, c, negate, mixed);
        else hipLaunchKernelGGL((prompt_kernel<128, 1>), grid, dim3(kThreads), 0, s, c, negate, mixed);
    } else {
        if (split) hipLaunchKernelGGL((prompt_kernel<64, 2>), grid, dim3(kThreads), 0, s, c, negate, mixed);
        else hipLaunchKernelGGL((prompt_kernel<64, 1>), grid, dim3(kThreads), 0, s, c, negate, mixed);
    }
    GQSA_HIP(hipGetLastError());
    return GQSA_OK;
}

}  // namespace gqsa
