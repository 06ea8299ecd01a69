// extern "C" surface of include/gqsa_attention.h: argument checking and the life of a cache handle.  The arithmetic is in
// gqsa_rotate.hip, gqsa_cache.hip, gqsa_cache_rows.hip, gqsa_tree.hip and gqsa_prompt.hip.
#include <cmath>
#include <cstdint>
#include <new>

#include "gqsa_attention.hpp"

namespace {

constexpr int kMaxHeads = 1024;
constexpr int64_t kMaxKeyDistance = int64_t{1} << 23;     // between rows of a prompt's keys: the rows of a tile are addressed with 32 bits
constexpr int64_t kMaxRows = int64_t{1} << 25;     // (a launch has fewer than 2^32 threads)

bool aligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// A [rows, heads, head_dim] array as the kernels want it.  Distances are bounded so that the largest offset fits 63 bits.
gqsa_status_t take(const void* p, int64_t row, int64_t head, gqsa::Heads* out)
{
    if (!p) return GQSA_ERR_NULL;
    if (row < 0 || head < 0 || row > (int64_t{1} << 31) || head > (int64_t{1} << 40)) return GQSA_ERR_SHAPE;
    if (!aligned(p, 16) || row % 8 != 0 || head % 8 != 0) return GQSA_ERR_ALIGN;
    *out = {static_cast<uint16_t*>(const_cast<void*>(p)), row, head};
    return GQSA_OK;
}

gqsa_status_t check_heads(int q_heads, int kv_heads)
{
    if (q_heads < 1 || kv_heads < 1) return GQSA_ERR_SHAPE;
    if (q_heads % kv_heads != 0) return GQSA_ERR_SHAPE;
    return q_heads <= kMaxHeads ? GQSA_OK : GQSA_ERR_UNSUPPORTED;
}

gqsa_status_t take_sequences(const int32_t* pages, int max_pages, const int32_t* lengths, const int32_t* row_starts, int n_seqs,
                             int64_t n_rows, gqsa::Sequences* out)
{
    if (!pages || !lengths) return GQSA_ERR_NULL;
    if (n_rows < 0 || n_rows > kMaxRows || n_seqs < 1 || max_pages < 1) return GQSA_ERR_SHAPE;
    if (n_seqs > 65536 || max_pages > (1 << 20)) return GQSA_ERR_UNSUPPORTED;
    if (!row_starts && n_rows != n_seqs) return GQSA_ERR_SHAPE;
    if (!aligned(pages, 4) || !aligned(lengths, 4) || !aligned(row_starts, 4)) return GQSA_ERR_ALIGN;
    *out = {pages, lengths, row_starts, n_rows, max_pages, n_seqs};
    return GQSA_OK;
}

// Norms and rotation of a call; `any_positions`: a NULL is a token's place.
gqsa_status_t take_rotation(const void* q_weight, const void* k_weight, float eps, const float* table, int64_t n_positions, int rotary_dim, int interleaved,
                            const int32_t* positions, bool any_positions, int head_dim, gqsa::RotateCall* c)
{
    if (n_positions < 0) return GQSA_ERR_SHAPE;
    if (head_dim < 16 || head_dim > 256 || head_dim % 16 != 0) return GQSA_ERR_UNSUPPORTED;
    if (rotary_dim < 0 || rotary_dim > head_dim || rotary_dim % 16 != 0) return GQSA_ERR_UNSUPPORTED;
    if (rotary_dim > 0 && (!table || (!positions && !any_positions))) return GQSA_ERR_NULL;
    if (!aligned(q_weight, 16) || !aligned(k_weight, 16) || !aligned(table, 16) || !aligned(positions, 4)) return GQSA_ERR_ALIGN;
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return GQSA_ERR_RANGE;
    c->q_weight = static_cast<const uint16_t*>(q_weight);
    c->k_weight = static_cast<const uint16_t*>(k_weight);
    c->table = table;
    c->positions = positions;
    c->n_positions = n_positions;
    c->head_dim = head_dim;
    c->rotary_dim = rotary_dim;
    c->interleaved = interleaved != 0;
    c->eps = eps;
    return GQSA_OK;
}

}  // namespace

extern "C" {

gqsa_status_t gqsa_qk_norm_rotate(const void* q, int64_t q_row_stride, int64_t q_head_stride, int q_heads,
                                  const void* k, int64_t k_row_stride, int64_t k_head_stride, int k_heads,
                                  int64_t n_rows, int head_dim, const void* q_weight, const void* k_weight, float eps,
                                  const float* table, int64_t n_positions, int rotary_dim, int interleaved, const int32_t* positions,
                                  void* q_out, int64_t q_out_row_stride, int64_t q_out_head_stride,
                                  void* k_out, int64_t k_out_row_stride, int64_t k_out_head_stride, void* hip_stream)
{
    gqsa::RotateCall c{};
    if (n_rows == 0) return GQSA_OK;
    if (gqsa_status_t st = take(q, q_row_stride, q_head_stride, &c.q)) return st;
    if (gqsa_status_t st = take(q_out, q_out_row_stride, q_out_head_stride, &c.q_out)) return st;
    if (q_heads < 1 || k_heads < 0 || n_rows < 0 || n_rows > kMaxRows || n_positions < 0) return GQSA_ERR_SHAPE;
    if (q_heads > kMaxHeads || k_heads > kMaxHeads) return GQSA_ERR_UNSUPPORTED;
    if (k_heads > 0) {
        if (gqsa_status_t st = take(k, k_row_stride, k_head_stride, &c.k)) return st;
        if (gqsa_status_t st = take(k_out, k_out_row_stride, k_out_head_stride, &c.k_out)) return st;
    }
    if (gqsa_status_t st = take_rotation(q_weight, k_weight, eps, table, n_positions, rotary_dim, interleaved, positions, false, head_dim, &c)) return st;
    c.n_rows = n_rows;
    c.q_heads = q_heads;
    c.k_heads = k_heads;
    c.one_over_dim = 1.0f / static_cast<float>(head_dim);
    return gqsa::rotate(c, hip_stream);
}

gqsa_status_t gqsa_cache_create(int64_t n_pages, int page_tokens, int kv_heads, int head_dim, gqsa_cache_t* out)
{
    if (out) *out = nullptr;
    if (!out) return GQSA_ERR_NULL;
    if (n_pages < 1 || page_tokens < 1 || kv_heads < 1) return GQSA_ERR_SHAPE;
    if (n_pages > (int64_t{1} << 30) || kv_heads > kMaxHeads || page_tokens < gqsa::kTileTokens || page_tokens > 4096 ||
        (page_tokens & (page_tokens - 1)) != 0 || (head_dim != 64 && head_dim != 128))
        return GQSA_ERR_UNSUPPORTED;
    gqsa_cache* c = new (std::nothrow) gqsa_cache;
    if (!c) return GQSA_ERR_ALLOC;
    c->n_pages = n_pages;
    c->page_tokens = page_tokens;
    c->kv_heads = kv_heads;
    c->head_dim = head_dim;
    if (gqsa_status_t st = gqsa::cache_allocate(c)) {
        gqsa::cache_release(c);
        delete c;
        return st;
    }
    *out = c;
    return GQSA_OK;
}

gqsa_status_t gqsa_cache_info(gqsa_cache_t c, gqsa_cache_info_t* out)
{
    if (!c || !out) return GQSA_ERR_NULL;
    out->n_pages = c->n_pages;
    out->page_tokens = c->page_tokens;
    out->kv_heads = c->kv_heads;
    out->head_dim = c->head_dim;
    out->token_bytes = gqsa::tile_bytes(c->head_dim) / gqsa::kTileTokens;
    out->device_bytes = c->device_bytes();
    out->workspace_bytes = c->workspace_bytes();
    return GQSA_OK;
}

void gqsa_cache_free(gqsa_cache_t c)
{
    if (!c) return;
    gqsa::cache_release(c);
    delete c;
}

gqsa_status_t gqsa_cache_append(gqsa_cache_t c, const void* k, int64_t k_row_stride, int64_t k_head_stride,
                                const void* v, int64_t v_row_stride, int64_t v_head_stride, int64_t n_rows,
                                const int32_t* pages, int max_pages, const int32_t* lengths, const int32_t* row_starts,
                                int n_seqs, void* hip_stream)
{
    if (!c) return GQSA_ERR_NULL;
    if (n_rows == 0) return GQSA_OK;
    gqsa::Heads kh, vh;
    gqsa::Sequences seqs;
    if (gqsa_status_t st = take(k, k_row_stride, k_head_stride, &kh)) return st;
    if (gqsa_status_t st = take(v, v_row_stride, v_head_stride, &vh)) return st;
    if (gqsa_status_t st = take_sequences(pages, max_pages, lengths, row_starts, n_seqs, n_rows, &seqs)) return st;
    return gqsa::cache_append(c, kh, vh, seqs, hip_stream);
}

gqsa_status_t gqsa_cache_append_rotated(gqsa_cache_t c, const void* q, int64_t q_row_stride, int64_t q_head_stride, int q_heads,
                                        const void* k, int64_t k_row_stride, int64_t k_head_stride,
                                        const void* v, int64_t v_row_stride, int64_t v_head_stride, int64_t n_rows,
                                        const void* q_weight, const void* k_weight, float eps,
                                        const float* table, int64_t n_positions, int rotary_dim, int interleaved, const int32_t* positions,
                                        void* q_out, int64_t q_out_row_stride, int64_t q_out_head_stride,
                                        void* k_out, int64_t k_out_row_stride, int64_t k_out_head_stride,
                                        const int32_t* pages, int max_pages, const int32_t* lengths, const int32_t* row_starts,
                                        int n_seqs, void* hip_stream)
{
    if (!c) return GQSA_ERR_NULL;
    if (n_rows == 0) return GQSA_OK;
    gqsa::RotateCall call{};
    gqsa::Heads vh;
    gqsa::Sequences seqs;
    if (q_heads < 0) return GQSA_ERR_SHAPE;
    if (q_heads > kMaxHeads) return GQSA_ERR_UNSUPPORTED;
    if (q_heads > 0) {
        if (gqsa_status_t st = take(q, q_row_stride, q_head_stride, &call.q)) return st;
        if (gqsa_status_t st = take(q_out, q_out_row_stride, q_out_head_stride, &call.q_out)) return st;
    }
    if (gqsa_status_t st = take(k, k_row_stride, k_head_stride, &call.k)) return st;
    if (gqsa_status_t st = take(v, v_row_stride, v_head_stride, &vh)) return st;
    if (k_out) {
        if (gqsa_status_t st = take(k_out, k_out_row_stride, k_out_head_stride, &call.k_out)) return st;
    }
    if (gqsa_status_t st = take_rotation(q_weight, k_weight, eps, table, n_positions, rotary_dim, interleaved, positions, true, c->head_dim, &call)) return st;
    if (gqsa_status_t st = take_sequences(pages, max_pages, lengths, row_starts, n_seqs, n_rows, &seqs)) return st;
    call.q_heads = q_heads;
    return gqsa::cache_append_rotated(c, call, vh, seqs, hip_stream);
}

gqsa_status_t gqsa_cache_keep(gqsa_cache_t c, int64_t n_rows, const int32_t* pages, int max_pages, const int32_t* lengths, const int32_t* row_starts,
                              int n_seqs, const int32_t* path, const int32_t* accepted, void* hip_stream)
{
    if (!c) return GQSA_ERR_NULL;
    if (n_rows == 0) return GQSA_OK;
    gqsa::Sequences seqs;
    if (gqsa_status_t st = take_sequences(pages, max_pages, lengths, row_starts, n_seqs, n_rows, &seqs)) return st;
    if (!path || !accepted) return GQSA_ERR_NULL;
    if (!aligned(path, 4) || !aligned(accepted, 4)) return GQSA_ERR_ALIGN;
    return gqsa::cache_keep(c, seqs, path, accepted, hip_stream);
}

gqsa_status_t gqsa_cache_read(gqsa_cache_t c, void* k_out, int64_t k_row_stride, int64_t k_head_stride,
                              void* v_out, int64_t v_row_stride, int64_t v_head_stride, int64_t n_rows,
                              const int32_t* pages, int max_pages, const int32_t* lengths, const int32_t* row_starts,
                              int n_seqs, void* hip_stream)
{
    if (!c) return GQSA_ERR_NULL;
    if (n_rows == 0) return GQSA_OK;
    gqsa::Heads kh, vh;
    gqsa::Sequences seqs;
    if (gqsa_status_t st = take(k_out, k_row_stride, k_head_stride, &kh)) return st;
    if (gqsa_status_t st = take(v_out, v_row_stride, v_head_stride, &vh)) return st;
    if (gqsa_status_t st = take_sequences(pages, max_pages, lengths, row_starts, n_seqs, n_rows, &seqs)) return st;
    return gqsa::cache_read(c, kh, vh, seqs, hip_stream);
}

static gqsa_status_t take_attention(gqsa_cache_t c, const void* q, int64_t q_row_stride, int64_t q_head_stride, int q_heads, int64_t n_rows,
                                    const int32_t* pages, int max_pages, const int32_t* lengths, const int32_t* row_starts, int n_seqs, float scale,
                                    void* out, int64_t out_row_stride, int64_t out_head_stride, gqsa::Heads* qh, gqsa::Heads* oh, gqsa::Sequences* seqs)
{
    if (gqsa_status_t st = take(q, q_row_stride, q_head_stride, qh)) return st;
    if (gqsa_status_t st = take(out, out_row_stride, out_head_stride, oh)) return st;
    if (gqsa_status_t st = check_heads(q_heads, c->kv_heads)) return st;
    if (gqsa_status_t st = take_sequences(pages, max_pages, lengths, row_starts, n_seqs, n_rows, seqs)) return st;
    return std::isfinite(scale) ? GQSA_OK : GQSA_ERR_RANGE;
}

gqsa_status_t gqsa_cache_attend(gqsa_cache_t c, const void* q, int64_t q_row_stride, int64_t q_head_stride, int q_heads,
                                int64_t n_rows, const int32_t* pages, int max_pages, const int32_t* lengths,
                                const int32_t* row_starts, int n_seqs, float scale, void* out, int64_t out_row_stride,
                                int64_t out_head_stride, void* hip_stream)
{
    if (!c) return GQSA_ERR_NULL;
    if (n_rows == 0) return GQSA_OK;
    gqsa::Heads qh, oh;
    gqsa::Sequences seqs;
    if (gqsa_status_t st = take_attention(c, q, q_row_stride, q_head_stride, q_heads, n_rows, pages, max_pages, lengths, row_starts, n_seqs, scale,
                                          out, out_row_stride, out_head_stride, &qh, &oh, &seqs))
        return st;
    return gqsa::cache_attend(c, qh, q_heads, seqs, scale, oh, hip_stream);
}

gqsa_status_t gqsa_cache_attend_tree(gqsa_cache_t c, const void* q, int64_t q_row_stride, int64_t q_head_stride, int q_heads,
                                     int64_t n_rows, const int32_t* pages, int max_pages, const int32_t* lengths,
                                     const int32_t* row_starts, int n_seqs, const int32_t* masks, int mask_words, float scale,
                                     void* out, int64_t out_row_stride, int64_t out_head_stride, void* hip_stream)
{
    if (!c) return GQSA_ERR_NULL;
    if (n_rows == 0) return GQSA_OK;
    gqsa::Heads qh, oh;
    gqsa::Sequences seqs;
    if (gqsa_status_t st = take_attention(c, q, q_row_stride, q_head_stride, q_heads, n_rows, pages, max_pages, lengths, row_starts, n_seqs, scale,
                                          out, out_row_stride, out_head_stride, &qh, &oh, &seqs))
        return st;
    if (!masks) return GQSA_ERR_NULL;
    if (mask_words < 1) return GQSA_ERR_SHAPE;
    if (mask_words > (1 << 15)) return GQSA_ERR_UNSUPPORTED;
    if (!aligned(masks, 4)) return GQSA_ERR_ALIGN;
    return gqsa::cache_attend_tree(c, qh, q_heads, seqs, reinterpret_cast<const uint32_t*>(masks), mask_words, scale, oh, hip_stream);
}

gqsa_status_t gqsa_prompt_attend(const void* q, int64_t q_row_stride, int64_t q_head_stride, int q_heads, int64_t n_q_rows,
                                 const void* k, int64_t k_row_stride, int64_t k_head_stride,
                                 const void* v, int64_t v_row_stride, int64_t v_head_stride, int kv_heads, int64_t n_k_rows,
                                 int head_dim, const int32_t* q_starts, const int32_t* k_starts, int n_seqs, float scale,
                                 void* out, int64_t out_row_stride, int64_t out_head_stride, void* hip_stream)
{
    gqsa::PromptCall c{};
    if (n_q_rows == 0) return GQSA_OK;
    if (gqsa_status_t st = take(q, q_row_stride, q_head_stride, &c.q)) return st;
    if (n_k_rows > 0) {
        if (gqsa_status_t st = take(k, k_row_stride, k_head_stride, &c.k)) return st;
        if (gqsa_status_t st = take(v, v_row_stride, v_head_stride, &c.v)) return st;
        if (k_row_stride > kMaxKeyDistance || v_row_stride > kMaxKeyDistance) return GQSA_ERR_UNSUPPORTED;
    }
    if (gqsa_status_t st = take(out, out_row_stride, out_head_stride, &c.out)) return st;
    if (!q_starts || !k_starts) return GQSA_ERR_NULL;
    if (gqsa_status_t st = check_heads(q_heads, kv_heads)) return st;
    if (n_q_rows < 0 || n_q_rows > kMaxRows || n_k_rows < 0 || n_k_rows > kMaxRows || n_seqs < 1) return GQSA_ERR_SHAPE;
    if (n_seqs > 65536 || (head_dim != 64 && head_dim != 128)) return GQSA_ERR_UNSUPPORTED;
    if (!aligned(q_starts, 4) || !aligned(k_starts, 4)) return GQSA_ERR_ALIGN;
    if (!std::isfinite(scale)) return GQSA_ERR_RANGE;
    c.q_starts = q_starts;
    c.k_starts = k_starts;
    c.n_q_rows = n_q_rows;
    c.n_k_rows = n_k_rows;
    c.q_heads = q_heads;
    c.kv_heads = kv_heads;
    c.head_dim = head_dim;
    c.n_seqs = n_seqs;
    c.scale = scale;
    return gqsa::prompt_attend(c, hip_stream);
}

}  // extern "C"
