// Attention of a tree's rows over the 4-bit cache where a head of the cache has many rows (gqsa_cache_attend_tree; with few of them, the kernel of gqsa_cache_attend has it).
//   s_j = scale q k_j for the tokens j before the rows and those of the rows that the mask names;   m = max s_j,   out = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m)
// in one pass over the tokens: maximum (as a reference that follows it from 2^7 below, see kRoom in gqsa_device.hpp), sum and weighted sum go along in fp32, weights are rounded to
// fp16 as the second product takes them, and their sum is of the rounded ones, so that the rounding of the largest weight cancels.
//
// What the kernel for few rows spends its time on is turning codes into numbers, anew for every 16 rows.  Here a workgroup of 8 wavefronts takes 128 rows of a
// head of the cache (or 64), and 128 tokens at a time: every wavefront turns half a tile of 32 tokens into fp16 numbers in LDS, one step ahead of the products, and
// then takes 32 rows with every second (fourth) part of the step's tokens.  Both products are 32x32x16 ones, S^T = K Q^T and O^T = V^T P^T: a lane holds scores
// of one row only, and holds them as the second product wants its operand, if keys go into the first one in the order in which a word of value codes has its tokens.
//
// Bound: 16 sequences of 4160 tokens, 64 rows of 32 heads over 8 (69 GFLOP, 52 us at the rate of a large fp16 product): 94 us, of which the join is 7 and start and end some 12;
// within the steps of some 4800 cycles the vector units are busy for 43 % of the cycles (softmax, numbers of codes), the matrix cores for 31 %, LDS for 32 %.  Without the products
// it would be 80, without making numbers 77, with them but without their stores to LDS 79, without exponentials 88, without reading operands 96: the stores, 64 KB a step, stand most in the way.  One sequence of
// 131072 tokens, 16 rows of 64 heads over 8 (69 GFLOP): 100 us.  The kernel for few rows takes 202 and 166 for these.
// Weights made between the products that do not need them yet gain 1 %.
// Not kept: halves of the workgroup out of phase, one at products and one at numbers, with two barriers a step (no faster, and registers in memory); 32 rows a workgroup without sharing
// through LDS (16 x 1000 tokens with 128 rows of 8 heads 29 us instead of 37, 16 x 4160 with 256 131 instead of 94); 256 rows a workgroup, so that numbers are made half as often
// (16 x 4160 with 256 rows 128 us instead of 94, heads of 64 too: half as many blocks are dealt, more of them lie in several workgroups); priorities around the second product (no change); joining within
// the launch by the workgroup that ends last (31 to 50 us on top, for the 4 to 7 of the second launch).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "gqsa_cache_attend.hpp"

namespace gqsa {
namespace {

typedef float float2_t __attribute__((ext_vector_type(2)));

constexpr int kTreeThreads = 512, kTreeWaves = kTreeThreads / 64;
constexpr int kStepTiles = 4;           // of 32 tokens

// A block of rows whose steps begin in a workgroup and go on in the next ones.
struct Split {
    int parts;              // workgroups that have a share; 0: there is no such block
    int rows, token, head, head0;       // row r of it: head `head` + (head0 + r) % heads_per_group of query row `token` + (head0 + r) / heads_per_group
};

struct TreeArgs {
    Pool pool;
    Heads q, out;
    Sequences seqs;
    float* partials;
    Split* splits;          // of every workgroup
    const uint32_t* masks;
    int mask_words;
    int heads_per_group;
    float scale_log2;       // |scale| times log2(e): the softmax is taken to base 2
    bool negate;            // the queries, as scale is negative
};

template <int D>
struct alignas(1024) TreeShared {
    uint16_t k[2][kStepTiles][kTileTokens * D], v[2][kStepTiles][kTileTokens * D];
    uint8_t raw[kTreeWaves][2][1024 + 256];     // half a tile as it is held: key codes and parameters, value codes and parameters
    uint32_t nan_of[2][kStepTiles][D / 32];     // of a tile's group of values: the tokens that are NaN, where some rows do not see them
    int first[2][kStepTiles];                   // a tile's first token; -1: absent
};

// Where the run `run` of 8 elements of a token's key lies in a tile, and the 8 tokens of `quad` of an element of values: spread over the banks by token and element.
template <int D>
__device__ __forceinline__ int key_at(int token, int run) { return token * D + 8 * (run ^ (D == 128 ? token & 15 : (token >> 1) & 7)); }
__device__ __forceinline__ int value_at(int element, int quad) { return element * 32 + 8 * (quad ^ (element >> 2 & 3)); }

__device__ __forceinline__ uint32_t lds_address(const void* p)
{
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) uint8_t*)p));
}

// The token of a tile that row m of the first product's operand is: scores then lie as a word of value codes has its tokens.
__device__ __forceinline__ int token_of_row(int m) { return (m & 7) | (m & 8) << 1 | (m & 16) >> 1; }

// Half a tile's codes (16 bytes a lane) and parameters (4 bytes a lane) of keys, or of values, straight into LDS.  Not before the wavefront's reads of what lies there have
// returned, as they have where what they gave has been used.  (The wait states are for scalar registers that a vector instruction may have written just before, which the
// compiler does not see to inside a statement; one is for m0.)
__device__ __forceinline__ void copy_half(uint32_t to, const uint8_t* tile, uint32_t codes, uint32_t parameters)
{
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %2, %1\n\t"
                 "s_add_u32 m0, m0, 1024\n\ts_nop 0\n\tglobal_load_lds_dword %3, %1"
                 : "+{m0}"(to) : "s"(tile), "v"(codes), "v"(parameters) : "memory", "scc");
}

template <typename T>
__device__ __forceinline__ T lds_read(uint32_t at) { return *(const __attribute__((address_space(3))) T*)static_cast<uintptr_t>(at); }
template <typename T>
__device__ __forceinline__ void lds_write(uint32_t at, T v) { *(__attribute__((address_space(3))) T*)static_cast<uintptr_t>(at) = v; }

// Where a lane finds what it reads and writes: numbers of the loop's start, as they would otherwise be made again in every step (a fifth of its vector instructions).
template <int D>
struct Places {
    static constexpr uint32_t kTile = kTileTokens * D * 2, kBuffer = kStepTiles * kTile;
    uint32_t k_read, v_read;                        // operands: the first run of 8 elements, 8 tokens of the first quad; the others by their place's bits
    uint32_t k_write, v_write;                      // as numbers
    uint32_t raw_codes, raw_keys, raw_values;       // as they were copied
    uint32_t codes, parameters;                     // in a tile of the cache, of its keys

    // first: the first of the wavefront's tiles to read; tile, part: what it turns into numbers
    __device__ __forceinline__ Places(const TreeShared<D>& shared, int lane, int wave, int first, int tile, int part)
    {
        const int l = lane & 31, half = lane >> 5, quad = lane >> 4, of = lane & 15;
        const uint32_t k = lds_address(shared.k), v = lds_address(shared.v), raw = lds_address(shared.raw[wave]);
        k_read = k + first * kTile + 2 * key_at<D>(token_of_row(l), half);
        v_read = v + first * kTile + 2 * value_at(l, half);
        k_write = k + tile * kTile + 2 * key_at<D>(16 * part + of, quad);
        v_write = v + tile * kTile + 2 * value_at(16 * part * (D / 32) + of, quad);
        raw_codes = raw + lane * 16 + (D == 128 ? 0 : part * 8);
        raw_keys = raw + 1024 + ((D == 128 ? 0 : 16 * part) + of) * (D / 8);
        raw_values = raw + 1280 + 1024 + ((D == 128 ? 0 : part) * 4 + quad) * 32;
        codes = lane * 16 + (D == 128 ? part * 1024 : 0);
        parameters = 32 * D + lane * 4 + (D == 128 ? part * 256 : 0);
        asm volatile("" : "+v"(k_read), "+v"(v_read), "+v"(k_write), "+v"(v_write), "+v"(raw_codes), "+v"(raw_keys), "+v"(raw_values), "+v"(codes), "+v"(parameters));
    }
};

template <int D>
struct RawHalf {
    typedef uint32_t words_t __attribute__((ext_vector_type(D / 32)));
    words_t k, v, k_parameters;
    u32x4_t step[D / 64], low[D / 64];      // of the quad's tokens, of each group

    // (from LDS, once the copies have arrived)
    __device__ __forceinline__ void fetch_keys(const Places<D>& at)
    {
        k = lds_read<words_t>(at.raw_codes);
        k_parameters = lds_read<words_t>(at.raw_keys);
    }
    __device__ __forceinline__ void fetch_values(const Places<D>& at)
    {
        v = lds_read<words_t>(at.raw_codes + 1280);
#pragma unroll
        for (int g = 0; g < D / 64; ++g) step[g] = lds_read<u32x4_t>(at.raw_values + 128 * g), low[g] = lds_read<u32x4_t>(at.raw_values + 128 * g + 16);
    }
};

// What an edge asks for, where some rows do not see some of the tile's tokens, or it has `left` tokens only (an absent one none): those behind stand for zero, and values
// that are NaN stand for zero too, but are noted.
template <int D>
__device__ __forceinline__ void trim_keys(RawHalf<D>& raw, int half, int lane, int left)
{
    if (16 * half + (lane & 15) >= left) raw.k_parameters = raw.k_parameters & 0u;
}

template <int D>
__device__ __forceinline__ void trim_values(RawHalf<D>& raw, int half, int lane, int left, uint32_t* nan_of)
{
    const int quad = lane >> 4;
#pragma unroll
    for (int g = 0; g < D / 64; ++g) {
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int t = slot_token(quad, i), shift = 16 * (i & 1);
            const uint32_t bits = raw.low[g][i >> 1] >> shift & 0x7FFFu;
            const bool is_nan = bits > 0x7C00u;
            if (is_nan && t < left) bad |= 1u << t;
            if (is_nan || t >= left) raw.low[g][i >> 1] &= ~(0xFFFFu << shift), raw.step[g][i >> 1] &= ~(0xFFFFu << shift);
        }
        bad |= __shfl_xor(bad, 16);
        bad |= __shfl_xor(bad, 32);
        if (lane == 0) nan_of[half * (D / 64) + g] = bad;
    }
}

// Word `i` of a half into LDS as numbers, in two stages (2 i, 2 i + 1) that share `c`, so that they fit between products.
template <int D>
__device__ __forceinline__ void put_keys(const RawHalf<D>& raw, const Places<D>& at, uint32_t buffer, int stage, half2_t (&c)[4])
{
    const int g = stage / 2;
    if (stage % 2 == 0) {
        decode(raw.k[g], c);
        return;
    }
    const half2_t both = as_half2(raw.k_parameters[g]);
    const half2_t low = {both[0], both[0]}, step = {both[1], both[1]};
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = __builtin_elementwise_fma(c[i], step, low);
    lds_write((at.k_write + buffer) ^ (64 * g), join(c[0], c[1], c[2], c[3]));         // (run 4 g + quad)
}

template <int D>
__device__ __forceinline__ void put_values(const RawHalf<D>& raw, const Places<D>& at, uint32_t buffer, int stage, half2_t (&c)[4])
{
    const int u = stage / 2;
    if (stage % 2 == 0) {
        decode(raw.v[u], c);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = __builtin_elementwise_fma(c[i], as_half2(raw.step[u / 2][i]), as_half2(raw.low[u / 2][i]));
    lds_write(at.v_write + buffer + 1024 * u, join(c[0], c[1], c[2], c[3]));           // (16 elements further on)
}

// N operands from LDS and the N products that they go into, with the next ones always under way (left alone, the compiler waits for every read where it has issued it).  The
// first ones have been asked for before.  STAGES pieces of other work are done between the products, which leave the vector units free for most of their time.
constexpr int kAhead = 2;

template <int N, int STAGES, typename Read, typename Product, typename Aside>
__device__ __forceinline__ void stream_operands(half8_t (&x)[2][kAhead], Read read, Product product, Aside aside)
{
    static_assert(N % kAhead == 0, "");
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n % kAhead == 0 && n + kAhead < N) {
#pragma unroll
            for (int e = 0; e < kAhead; ++e) x[(n / kAhead + 1) & 1][e] = read(n + kAhead + e);
        }
        __builtin_amdgcn_sched_barrier(0);
        product(n, x[n / kAhead & 1][n % kAhead]);
#pragma unroll
        for (int i = n * STAGES / N; i < (n + 1) * STAGES / N; ++i) aside(i);
        __builtin_amdgcn_sched_barrier(0);
    }
}

__device__ __forceinline__ int tree_steps(int tokens)
{
    return max(static_cast<int>(static_cast<unsigned>(tokens + kStepTiles * kTileTokens - 1) / static_cast<unsigned>(kStepTiles * kTileTokens)), 1);
}

// As in the attention of few rows, all steps of all sequences, heads and blocks of rows are dealt evenly to the workgroups, one to a CU (LDS holds no more).  Where a block lies in several of them each leaves its
// maximum, sum and weighted sum of every row in the workspace, and a second launch joins them.  GROUPS: wavefronts with rows of their own.
template <int D, int GROUPS>
__global__ __launch_bounds__(kTreeThreads, 2) void tree_kernel(TreeArgs a)
{
    constexpr int kRows = 32 * GROUPS, kParts = kTreeWaves / GROUPS, kPieces = kStepTiles / kParts;
    constexpr int kPartial = kRows * (D + 2);
    __shared__ TreeShared<D> shared;
    static_assert(sizeof(shared.k) + sizeof(shared.v) >= kTreeWaves * ((kParts - 1) * (4 * (D / 32) / kParts) * 1024 + 512), "");
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5;
    const int group = wave % GROUPS, part = wave / GROUPS;
    const unsigned per = a.heads_per_group;
    const auto blocks_of = [&](const Sequence& q) { return static_cast<int>((static_cast<unsigned>(q.rows) * per + kRows - 1) / kRows); };
    // (rows are counted from a sequence's true end, also where that lies beyond its pages)
    const int room = most_tokens(a.seqs, a.pool.page_shift);
    const auto steps_of = [&](const Sequence& q) { return tree_steps(min(q.length, room)); };
    const auto deal = deal_out<Sequence>(a.seqs.n_seqs, lane, [&](int b) { return sequence(a.seqs, INT_MAX, b); }, [&](const Sequence& q) {
        return static_cast<unsigned>(min(static_cast<int64_t>(blocks_of(q)) * steps_of(q) * a.pool.kv_heads, int64_t{INT_MAX}));
    });
    const unsigned total = deal.total, workers = min(gridDim.x, total), me = blockIdx.x;
    if (threadIdx.x == 0) a.splits[me].parts = 0;
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
        const int blocks = blocks_of(seq), steps = steps_of(seq);
        if (within >= blocks * steps * a.pool.kv_heads) {       // (on to the next sequence that has rows)
            within = 0;
            seq = sequence(a.seqs, INT_MAX, ++b);
            continue;
        }
        const int segment = static_cast<unsigned>(within) / static_cast<unsigned>(steps), from = within - segment * steps;
        const int to = min(steps, from + (end - at));
        const int head = blocks == 1 ? segment : static_cast<unsigned>(segment) / static_cast<unsigned>(blocks);
        const unsigned row0 = (segment - head * blocks) * kRows;        // of the sequence's rows times the heads of a group
        const int rows = min(static_cast<unsigned>(kRows), seq.rows * per - row0);
        const unsigned token0 = row0 / per, head0 = row0 - token0 * per;    // row r of the block: head (head0 + r) % per of the group, token further on
        const int before = seq.length - seq.rows, tokens = min(seq.length, room);

        // this lane's row
        const int own = 32 * group + (lane & 31);
        const bool is_row = own < rows, active = 32 * group < rows;     // (active: the same for a whole wavefront)
        const unsigned ahead = (head0 + own) / per;
        const int row = token0 + ahead, q_head = head * per + (head0 + own - ahead * per);
        half8_t q[D / 16];
        const uint16_t* q_at = a.q.data + int64_t{seq.start + row} * a.q.row + q_head * a.q.head + 8 * half;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            q[i] = half8_t{};
            if (is_row) q[i] = *reinterpret_cast<const half8_t*>(q_at + 16 * i);
            if (a.negate) q[i] = -q[i];
            q[i] += q[i] - q[i];        // (an infinity as NaN: it makes a row NaN, which scores of -infinity only would not)
        }
        const uint32_t* mask = a.masks + int64_t{seq.start + static_cast<int>(token0 + (head0 + min(own, rows - 1)) / per)} * a.mask_words;

        float16_t out[D / 32];
#pragma unroll
        for (int d = 0; d < D / 32; ++d) out[d] = float16_t{};
        float top = kMinusInf, sum = 0.0f;

        // The wavefront turns half of every fourth tile into numbers; lane i knows where the i-th of the next 64 lies, so that no load waits for another.
        const int32_t* table = a.seqs.pages + int64_t{b} * a.seqs.max_pages;
        const int tiles = uniform(min((tokens + kTileTokens - 1) / kTileTokens, to * kStepTiles));
        const int my_tile = wave >> 1, my_half = wave & 1, count = to - from;
        const Places<D> places(shared, opaque(lane), wave, kPieces * part, my_tile, my_half);
        // (always the same number of loads: past the end and for absent pages of some tile that is there)
        int next_first = -1, after_first = -1;         // of the tile that is turned into numbers in this step, and of the one after it; -1: absent
        const uint8_t* after_tile = nullptr;
        uint32_t tile_of_lane[2] = {};
        int first_of_lane = -1;
        const auto load_keys = [&](int i) {
            if ((i & 63) == 0) {
                const int tile = (from + i + opaque(lane)) * kStepTiles + my_tile;
                const int page = table[max(min(tile, tiles - 1), 0) >> (a.pool.page_shift - 5)];
                const bool there = tile < tiles && page >= 0 && page < a.pool.n_pages;
                const uint64_t at = reinterpret_cast<uint64_t>(a.pool.tile<D>(there ? page : 0, head, tile));
                tile_of_lane[0] = static_cast<uint32_t>(at), tile_of_lane[1] = static_cast<uint32_t>(at >> 32);
                first_of_lane = there ? tile * kTileTokens : -1;
                asm volatile("" : "+v"(tile_of_lane[0]), "+v"(tile_of_lane[1]), "+v"(first_of_lane));
            }
            const uint32_t low = __builtin_amdgcn_readlane(tile_of_lane[0], i & 63), high = __builtin_amdgcn_readlane(tile_of_lane[1], i & 63);
            after_first = __builtin_amdgcn_readlane(first_of_lane, i & 63);
            after_tile = reinterpret_cast<const uint8_t*>(uint64_t{high} << 32 | low);
            copy_half(lds_address(shared.raw[wave][0]), after_tile, places.codes, places.parameters);
        };
        const auto load_values = [&] { copy_half(lds_address(shared.raw[wave][1]), after_tile, places.codes + 16 * D, places.parameters + 4 * D); };
        RawHalf<D> raw;
        const auto left_of = [&](int first_token) { return first_token < 0 ? 0 : tokens - first_token; };
        // (what has been asked for since may still be under way: two loads)
        const auto fetch_keys = [&] {
            asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
            raw.fetch_keys(places);
            if (next_first < 0 || next_first + kTileTokens > before) trim_keys<D>(raw, my_half, opaque(lane), left_of(next_first));
        };
        const auto fetch_values = [&](int buffer) {
            asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
            raw.fetch_values(places);
            if (next_first < 0 || next_first + kTileTokens > before) trim_values<D>(raw, my_half, opaque(lane), left_of(next_first), shared.nan_of[buffer][my_tile]);
            if (my_half == 0 && opaque(lane) == 0) shared.first[buffer][my_tile] = next_first;
        };
        constexpr int kStages = 2 * (D / 32);
        half2_t c[4];
        const auto put_keys_of = [&](int buffer) { return [&, at = buffer * Places<D>::kBuffer](int stage) { put_keys<D>(raw, places, at, stage, c); }; };
        const auto put_values_of = [&](int buffer) { return [&, at = buffer * Places<D>::kBuffer](int stage) { put_values<D>(raw, places, at, stage, c); }; };
        const auto every = [&](auto aside) {
#pragma unroll
            for (int i = 0; i < kStages; ++i) aside(i);
        };
        int first[kPieces];
        uint32_t seen[kPieces];
        bool all_seen;
        half8_t p[2 * kPieces];
        float16_t s[kPieces] = {};
        half8_t x[2][kAhead];
        const auto key_operand = [&](int buffer, int n) {       // (run 2 i + half)
            return lds_read<half8_t>(((places.k_read + buffer * Places<D>::kBuffer) ^ (32 * (n / kPieces))) + n % kPieces * Places<D>::kTile);
        };
        const auto value_operand = [&](int buffer, int n) {     // (32 elements further on)
            const int i = n / (D / 32), d = n % (D / 32);
            return lds_read<half8_t>(((places.v_read + buffer * Places<D>::kBuffer) ^ (32 * (i & 1))) + (i >> 1) * Places<D>::kTile + d * 2048);
        };
        const auto score = [&](int buffer) {
#pragma unroll
            for (int e = 0; e < kAhead; ++e) x[0][e] = key_operand(buffer, e);
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                first[j] = shared.first[buffer][kPieces * part + j];       // (made uniform when it is needed)
                s[j] = float16_t{};
            }
            stream_operands<D / 16 * kPieces, kStages>(x, [&](int n) { return key_operand(buffer, n); },
                                                       [&](int n, half8_t k) { s[n % kPieces] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q[n / kPieces], s[n % kPieces], 0, 0, 0); },
                                                       put_keys_of(buffer ^ 1));
        };
        const auto ask_for_values = [&](int buffer) {
#pragma unroll
            for (int e = 0; e < kAhead; ++e) x[0][e] = value_operand(buffer, e);
        };
        // The weights of 8 / (D / 32) scores; D / 32 times these are an operand, the next of which is made between the products with the one before.
        float reference;
        const auto weigh_more = [&](int n) {
            constexpr int kOnce = 8 / (D / 32);
            const int i = n / (D / 32), e0 = n % (D / 32) * kOnce;
            const half2_t ones = {static_cast<_Float16>(1.0f), static_cast<_Float16>(1.0f)};
#pragma unroll
            for (int e = e0; e < e0 + kOnce; ++e)
                p[i][e] = static_cast<_Float16>(__builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 1][8 * (i & 1) + e], a.scale_log2, -reference)));
            // (the sum of the weights as the product has them, rounded: half the additions)
#pragma unroll
            for (int e = e0; e < e0 + kOnce; e += 2) sum = __builtin_amdgcn_fdot2(half2_t{p[i][e], p[i][e + 1]}, ones, sum, false);
        };
        const auto weigh = [&] {
            all_seen = true;
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                first[j] = uniform(first[j]);
                all_seen &= first[j] >= 0 && first[j] + kTileTokens <= before;
            }
            // element r of s[j] is row r % 4 + 8 (r / 4) + 4 half of the operand
            if (!all_seen) {
#pragma unroll
                for (int j = 0; j < kPieces; ++j) seen[j] = seen_of(mask, a.mask_words, first[j] - before, tokens - first[j]);
#pragma unroll
                for (int j = 0; j < kPieces; ++j) {
                    if (!is_row || first[j] < 0) seen[j] = 0;
                    const uint32_t sees = seen[j] >> 4 * half;
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (!(sees >> token_of_row((r & 3) + 8 * (r >> 2)) & 1)) s[j][r] = kMinusInf;
                }
            }
            float most = kMinusInf;
#pragma unroll
            for (int j = 0; j < kPieces; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) most = fmaxf(most, s[j][r]);
            most *= a.scale_log2;
            if (__any(most > top + (kRoom + kSlack) || (top == kMinusInf && most > kMinusInf))) {
                most = fmaxf(most, __shfl_xor(most, 32));
                const float higher = fmaxf(top, most - kRoom);
                const float shrink = higher == kMinusInf ? 1.0f : __builtin_amdgcn_exp2f(top - higher);
                top = higher;
                sum *= shrink;
#pragma unroll
                for (int d = 0; d < D / 32; ++d) out[d] *= shrink;
            }
            reference = top == kMinusInf ? 0.0f : top;
#pragma unroll
            for (int n = 0; n < D / 32; ++n) weigh_more(n);
        };
        const auto add_values = [&](int buffer) {
            const auto put = put_values_of(buffer ^ 1);
            constexpr int kProducts = 2 * kPieces * (D / 32);
            stream_operands<kProducts, kProducts>(x, [&](int n) { return value_operand(buffer, n); },
                                                  [&](int n, half8_t v) { out[n % (D / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p[n / (D / 32)], out[n % (D / 32)], 0, 0, 0); },
                                                  [&](int n) {
                                                      if (n + D / 32 < kProducts) weigh_more(n + D / 32);
#pragma unroll
                                                      for (int i = n * kStages / kProducts; i < (n + 1) * kStages / kProducts; ++i) put(i);
                                                  });
            if (!all_seen) {
#pragma unroll
                for (int j = 0; j < kPieces; ++j) {
                    if (first[j] < 0 || first[j] + kTileTokens <= before) continue;       // (nothing was noted)
#pragma unroll
                    for (int d = 0; d < D / 32; ++d)
                        if (shared.nan_of[buffer][kPieces * part + j][d] & seen[j]) out[d] = __builtin_nanf("") + float16_t{};
                }
            }
        };
        // While a step is at its products, the next one's tiles are turned into numbers -- keys between the first products, values between the second -- and the
        // one's after it are on their way.  (Past the last step numbers are made of what lies there, for nobody.)
        load_keys(0);
        load_values();
        next_first = after_first;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        fetch_keys();
        fetch_values(0);
        every(put_keys_of(0));
        every(put_values_of(0));
        load_keys(1);
        load_values();
        next_first = after_first;
        fetch_keys();
        for (int i = 0; i < count; ++i) {
            __syncthreads();            // the step's tiles are there, and nobody reads the ones before any more
            if (active) score(i & 1);
            else every(put_keys_of(~i & 1));
            load_keys(i + 2);
            fetch_values(~i & 1);
            if (active) {
                ask_for_values(i & 1);
                weigh();
                add_values(i & 1);
            } else {
                every(put_values_of(~i & 1));
            }
            load_values();
            next_first = after_first;
            fetch_keys();
        }

        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // (copies past the end may be under way)

        // The parts' results together, by way of LDS: of the fours of elements that a lane holds every part takes its share from the others.
        constexpr int kFours = 4 * (D / 32), kShare = kFours / kParts;
        sum += __shfl_xor(sum, 32);
        __syncthreads();
        const int l = opaque(lane);
        const uint32_t fours = lds_address(&shared) + l * 16, states = lds_address(&shared) + kTreeWaves * (kParts - 1) * kShare * 1024 + l * 8;
        const auto four = [&](int f) { return float4_t{out[f / 4][4 * (f % 4)], out[f / 4][4 * (f % 4) + 1], out[f / 4][4 * (f % 4) + 2], out[f / 4][4 * (f % 4) + 3]}; };
        // (where part `giver` of a group leaves the f-th four for part `taker`)
        const auto place = [&](int giver, int taker, int f) {
            return fours + static_cast<uint32_t>((((group * kParts + taker) * (kParts - 1) + (giver < taker ? giver : giver - 1)) * kShare + f) * 1024);
        };
        float4_t mine[kShare];
#pragma unroll
        for (int taker = 0; taker < kParts; ++taker) {
            if (taker == part) {
#pragma unroll
                for (int f = 0; f < kShare; ++f) mine[f] = four(taker * kShare + f);
            } else {
#pragma unroll
                for (int f = 0; f < kShare; ++f) lds_write(place(part, taker, f), four(taker * kShare + f));
            }
        }
        lds_write(states + (group * kParts + part) * 512, float2_t{top, sum});
        __syncthreads();
        float highest = top;
        float2_t other[kParts];
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            other[p] = lds_read<float2_t>(states + (group * kParts + p) * 512);
            highest = fmaxf(highest, other[p][0]);
        }
        const float own_weight = weight_of(top, highest);
        sum = 0.0f;
#pragma unroll
        for (int f = 0; f < kShare; ++f) mine[f] *= own_weight;
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            const float weight = weight_of(other[p][0], highest);
            sum += weight * other[p][1];
            if (p == part) continue;
#pragma unroll
            for (int f = 0; f < kShare; ++f) mine[f] += weight * lds_read<float4_t>(place(p, part, f));
        }
        const bool whole = from == 0 && to == steps;
        if (is_row) {
            const float inverse = sum == 0.0f ? 0.0f : 1.0f / sum;       // (a row that sees nothing: all sums are 0)
            uint16_t* y = a.out.data + int64_t{seq.start + row} * a.out.row + q_head * a.out.head;
            float* kept = a.partials + static_cast<int64_t>(2 * me + (from == 0 ? 1 : 0)) * kPartial;
            const int r = 32 * group + (l & 31);
#pragma unroll
            for (int f = 0; f < kShare; ++f) {
                const int at_four = part * kShare + f, column = 32 * (at_four / 4) + 8 * (at_four % 4) + 4 * half;
                if (whole) *reinterpret_cast<half4_t*>(y + column) = __builtin_convertvector(mine[f] * inverse, half4_t);
                else *reinterpret_cast<float4_t*>(kept + r * D + column) = mine[f];
            }
            if (!whole && part == 0 && half == 0) *reinterpret_cast<float2_t*>(kept + kRows * D + 2 * r) = float2_t{highest, sum};
        }
        if (from == 0 && to < steps && threadIdx.x == 0) {      // (the last segment that the workgroup has, if any)
            const unsigned last = owner_of(at + steps - 1);
            a.splits[me] = {static_cast<int>(last - me) + 1, rows, seq.start + static_cast<int>(token0), static_cast<int>(head * per), static_cast<int>(head0)};
        }
        at += to - from;
        within += to - from;
        if (at < end) __syncthreads();       // (LDS is free again)
    }
}

// The parts' results of the blocks that lie in several workgroups, in an order that hangs on the lengths alone.  A workgroup takes 4 rows of a block at a time: D / 4 threads to a row, each
// with four elements, and the rest of the threads for other parts.  (4 x 8128 tokens, 512 rows of 8 heads, with 256, 512, 1024, 2048, 4096 workgroups 110, 102, 99.5, 99.6, 101 us in all.)
constexpr int kJoinRows = 4, kJoinThreads = 256, kJoinWorkgroups = 1024;

template <int D, int ROWS>
__global__ __launch_bounds__(kJoinThreads) __attribute__((amdgpu_waves_per_eu(2, 4))) void tree_join_kernel(TreeArgs a, int workgroups)
{
    constexpr int kPartial = ROWS * (D + 2), kLanes = D / 4, kSlices = kJoinThreads / kJoinRows / kLanes, kAhead = 8;
    static_assert(kTreeWorkgroups <= kJoinThreads && kSlices > 1, "");
    __shared__ int list[kTreeWorkgroups], counts[kJoinThreads / 64];
    __shared__ float4_t shares[kSlices][kJoinRows][kLanes];
    __shared__ float2_t states[kSlices][kJoinRows];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool has = static_cast<int>(threadIdx.x) < workgroups && a.splits[threadIdx.x].parts > 0;
    const uint64_t all = __builtin_amdgcn_ballot_w64(has);
    if (lane == 0) counts[wave] = __builtin_popcountll(all);
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kJoinThreads / 64; ++w) before += w < wave ? counts[w] : 0, total += counts[w];
    if (has) list[before + __builtin_popcountll(all & ((uint64_t{1} << lane) - 1))] = threadIdx.x;
    __syncthreads();
    const int of = threadIdx.x % kLanes, row = threadIdx.x / kLanes % kJoinRows, slice = threadIdx.x / (kLanes * kJoinRows);
    for (int unit = blockIdx.x; unit < total * (ROWS / kJoinRows); unit += gridDim.x) {
        const int begun_in = list[unit / (ROWS / kJoinRows)], row0 = unit % (ROWS / kJoinRows) * kJoinRows;
        const Split split = a.splits[begun_in];
        if (row0 >= split.rows) continue;
        const int r = min(row0 + row, split.rows - 1);
        const auto part = [&](int p) { return a.partials + static_cast<int64_t>(2 * (begun_in + p) + (p == 0 ? 1 : 0)) * kPartial; };
        float top = kMinusInf, sum = 0.0f;
        float4_t v = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int p0 = slice; p0 < split.parts; p0 += kSlices * kAhead) {
            float2_t state[kAhead];
            float4_t x[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const float* from = part(min(p0 + kSlices * j, split.parts - 1));
                state[j] = *reinterpret_cast<const float2_t*>(from + ROWS * D + 2 * r);
                x[j] = *reinterpret_cast<const float4_t*>(from + r * D + 4 * of);
            }
            __builtin_amdgcn_sched_barrier(0);      // (all of them under way together)
            float highest = top;
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (p0 + kSlices * j >= split.parts) state[j] = float2_t{kMinusInf, 0.0f};
                highest = fmaxf(highest, state[j][0]);
            }
            const float weight = weight_of(top, highest);
            sum *= weight, v *= weight, top = highest;
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (p0 + kSlices * j >= split.parts) break;
                const float w = weight_of(state[j][0], highest);
                sum += w * state[j][1], v += w * x[j];
            }
        }
        shares[slice][row][of] = v;
        if (of == 0) states[slice][row] = float2_t{top, sum};
        __syncthreads();
        if (slice == 0 && row0 + row < split.rows) {
            float highest = kMinusInf;
#pragma unroll
            for (int i = 0; i < kSlices; ++i) highest = fmaxf(highest, states[i][row][0]);
            v = float4_t{0.0f, 0.0f, 0.0f, 0.0f}, sum = 0.0f;
#pragma unroll
            for (int i = 0; i < kSlices; ++i) {
                const float w = weight_of(states[i][row][0], highest);
                sum += w * states[i][row][1], v += w * shares[i][row][of];
            }
            const unsigned on = static_cast<unsigned>(split.head0 + r) / static_cast<unsigned>(a.heads_per_group);
            const int head = split.head + (split.head0 + r - static_cast<int>(on) * a.heads_per_group);
            const float inverse = sum == 0.0f ? 0.0f : 1.0f / sum;       // (a row that sees nothing: all sums are 0)
            *reinterpret_cast<half4_t*>(a.out.data + int64_t{split.token + static_cast<int>(on)} * a.out.row + head * a.out.head + 4 * of) = __builtin_convertvector(v * inverse, half4_t);
        }
        __syncthreads();
    }
}

template <int D, int GROUPS>
void launch_tree(const TreeArgs& a, unsigned workgroups, hipStream_t s)
{
    constexpr int kRows = 32 * GROUPS;
    hipLaunchKernelGGL((tree_kernel<D, GROUPS>), dim3(workgroups), dim3(kTreeThreads), 0, s, a);
    hipLaunchKernelGGL((tree_join_kernel<D, kRows>), dim3(kJoinWorkgroups), dim3(kJoinThreads), 0, s, a, static_cast<int>(workgroups));
}

}  // namespace

gqsa_status_t tree_attend(gqsa_cache* c, const Heads& q, int q_heads, const Sequences& seqs, const uint32_t* masks, int mask_words, float scale,
                          const Heads& out, void* stream)
{
    const int per = q_heads / c->kv_heads;
    const TreeArgs a{pool_of(c), q, out, seqs, c->d_partials, reinterpret_cast<Split*>(c->d_partials + int64_t{2} * kTreeWorkgroups * kTreeRows * (c->head_dim + 2)), masks, mask_words, per,
                     // (not 0, so that a masked score stays -infinity: 1e-30 leaves every weight at 1)
                     std::max(std::fabs(scale) * 1.44269504088896341f, 1e-30f), scale < 0.0f};
    const int groups = seqs.n_rows * per > 64 * int64_t{seqs.n_seqs} ? 4 : 2;
    const double blocks = (static_cast<double>(seqs.n_rows) * per / (32 * groups) + seqs.n_seqs) * c->kv_heads;
    const double steps = blocks * (static_cast<double>(seqs.max_pages) * c->page_tokens / (kStepTiles * kTileTokens) + 1.0);
    const unsigned workgroups = static_cast<unsigned>(std::max(1.0, std::min<double>(kTreeWorkgroups, steps)));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (c->head_dim == 128) {
        if (groups == 4) launch_tree<128, 4>(a, workgroups, s);
        else launch_tree<128, 2>(a, workgroups, s);
    } else {
        if (groups == 4) launch_tree<64, 4>(a, workgroups, s);
        else launch_tree<64, 2>(a, workgroups, s);
    }
    GQSA_HIP(hipGetLastError());
    return GQSA_OK;
}

}  // namespace gqsa
