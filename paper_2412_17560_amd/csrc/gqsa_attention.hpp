// Internal definitions of the operators between the q/k/v and the o product (include/gqsa_attention.h): what the C boundary
// (gqsa_attention_api.cpp) hands to the kernels (gqsa_rotate.hip, gqsa_cache.hip, gqsa_cache_rows.hip, gqsa_tree.hip, gqsa_prompt.hip).
#pragma once

#include <cstdint>
#include <cstdio>

#include "gqsa_attention.h"

// (used where the HIP runtime is included; an error that has been reported is taken off the runtime's record, where the next launch would find it)
#define GQSA_HIP(call)                                                                   \
    do {                                                                                 \
        const hipError_t e_ = (call);                                                    \
        if (e_ != hipSuccess) {                                                          \
            std::fprintf(stderr, "libgqsa: %s: %s\n", #call, hipGetErrorString(e_));    \
            (void)hipGetLastError();                                                     \
            return GQSA_ERR_HIP;                                                         \
        }                                                                                \
    } while (0)

namespace gqsa {

// A [rows, heads, head_dim] array of fp16: elements of a head side by side, distances in elements.
struct Heads {
    uint16_t* data;
    int64_t row, head;
};

struct RotateCall {
    Heads q, k, q_out, k_out;
    const uint16_t *q_weight, *k_weight;
    const float* table;
    const int32_t* positions;
    int64_t n_rows, n_positions;
    int q_heads, k_heads, head_dim, rotary_dim, interleaved;
    float eps, one_over_dim;
};

// The tokens of a 4-bit cache are held in tiles of 32 of one head: what 16x16x32 products take (gqsa_cache.hpp says in which order).
constexpr int kTileTokens = 32;
constexpr int kGroupChannels = 32;      // elements that share low and step
constexpr int tile_bytes(int head_dim) { return kTileTokens * head_dim + 2 * kTileTokens * (head_dim / kGroupChannels) * 4; }

constexpr int kAttendWorkgroups = 512;      // the most workgroups of one attention over the cache: two to a compute unit
constexpr int kRowBlock = 16;               // query rows (rows of a sequence times the heads of a group) per product

constexpr int kTreeWorkgroups = 256;        // the most workgroups of one attention of trees: one to a compute unit
constexpr int kTreeRows = 128;              // rows of a block there

// The rows that a sequence has, from the two ends that an array on the device gives, which may be anything: none outside 0 .. n - 1 (n at most 2^25).  Both
// ends are brought into 0 .. n before one is taken off the other, as their difference may not fit 32 bits.
struct Rows {
    int start, count;
};
constexpr Rows rows_between(int first, int end, int64_t n)
{
    const int most = static_cast<int>(n);
    const int start = first < 0 ? 0 : first < most ? first : most;
    const int stop = end < start ? start : end < most ? end : most;
    return {start, stop - start};
}

// Where the rows, pages and lengths of a call's sequences are.
struct Sequences {
    const int32_t *pages, *lengths, *row_starts;
    int64_t n_rows;
    int max_pages, n_seqs;
};

}  // namespace gqsa

struct gqsa_cache {
    int64_t n_pages = 0;
    int page_tokens = 0, kv_heads = 0, head_dim = 0;
    int device = -1;
    uint8_t* d_pages = nullptr;
    float* d_partials = nullptr;    // partial results of up to kRowBlock rows: two of every workgroup, one of several together; or those of trees
    int32_t* d_arrivals = nullptr;  // two counters for every workgroup, zero between calls

    int64_t device_bytes() const { return n_pages * kv_heads * (page_tokens / gqsa::kTileTokens) * int64_t{gqsa::tile_bytes(head_dim)}; }
    int64_t partial_floats() const
    {
        // (of trees two blocks of rows for every workgroup, and five numbers)
        const int64_t few = int64_t{gqsa::kAttendWorkgroups} * 3 * gqsa::kRowBlock * (head_dim + 2);
        const int64_t trees = int64_t{2} * gqsa::kTreeWorkgroups * gqsa::kTreeRows * (head_dim + 2) + gqsa::kTreeWorkgroups * 5;
        return few > trees ? few : trees;
    }
    int64_t workspace_bytes() const { return partial_floats() * 4 + int64_t{gqsa::kAttendWorkgroups} * 2 * 4; }
};

namespace gqsa {

gqsa_status_t rotate(const RotateCall& call, void* stream);

gqsa_status_t cache_allocate(gqsa_cache* c);
void cache_release(gqsa_cache* c);
gqsa_status_t cache_append(gqsa_cache* c, const Heads& k, const Heads& v, const Sequences& seqs, void* stream);
gqsa_status_t cache_read(gqsa_cache* c, const Heads& k, const Heads& v, const Sequences& seqs, void* stream);
gqsa_status_t cache_attend(gqsa_cache* c, const Heads& q, int q_heads, const Sequences& seqs, float scale, const Heads& out, void* stream);
gqsa_status_t cache_append_rotated(gqsa_cache* c, const RotateCall& call, const Heads& v, const Sequences& seqs, void* stream);
gqsa_status_t cache_attend_tree(gqsa_cache* c, const Heads& q, int q_heads, const Sequences& seqs, const uint32_t* masks, int mask_words, float scale,
                                const Heads& out, void* stream);
gqsa_status_t tree_attend(gqsa_cache* c, const Heads& q, int q_heads, const Sequences& seqs, const uint32_t* masks, int mask_words, float scale,
                          const Heads& out, void* stream);
gqsa_status_t cache_keep(gqsa_cache* c, const Sequences& seqs, const int32_t* path, const int32_t* accepted, void* stream);

struct PromptCall {
    Heads q, k, v, out;
    const int32_t *q_starts, *k_starts;
    int64_t n_q_rows, n_k_rows;
    int q_heads, kv_heads, head_dim, n_seqs;
    float scale;
};
gqsa_status_t prompt_attend(const PromptCall& call, void* stream);

}  // namespace gqsa
