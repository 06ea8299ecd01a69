// extern "C" surface of include/gqsa_verify.h: argument checking and the life of the handle.  The arithmetic is in gqsa_verify.hip.
#include <cstdint>
#include <new>

#include "gqsa_verify.hpp"

namespace {

constexpr int64_t kMostRows = int64_t{1} << 25;
constexpr int kMostSeqs = 65536, kMostVocab = 1 << 22;

bool words(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

}  // namespace

extern "C" {

gqsa_status_t gqsa_verify_create(int max_seqs, int max_vocab, gqsa_verifier_t* out)
{
    if (out) *out = nullptr;
    if (!out) return GQSA_ERR_NULL;
    if (max_seqs < 1 || max_vocab < 1) return GQSA_ERR_SHAPE;
    if (max_seqs > kMostSeqs || max_vocab > kMostVocab) return GQSA_ERR_UNSUPPORTED;
    if (int64_t{max_seqs} * max_vocab > (int64_t{1} << 34)) return GQSA_ERR_SHAPE;      // (a launch has fewer than 2^32 threads)
    gqsa_verifier* v = new (std::nothrow) gqsa_verifier;
    if (!v) return GQSA_ERR_ALLOC;
    v->max_seqs = max_seqs;
    v->max_vocab = max_vocab;
    if (gqsa_status_t st = gqsa::verifier_allocate(v)) {
        gqsa::verifier_release(v);
        delete v;
        return st;
    }
    *out = v;
    return GQSA_OK;
}

void gqsa_verify_free(gqsa_verifier_t v)
{
    if (!v) return;
    gqsa::verifier_release(v);
    delete v;
}

gqsa_status_t gqsa_verify(gqsa_verifier_t v, const float* target, int64_t target_row, const float* draft, int64_t draft_row, int vocab, int64_t n_rows,
                          const int32_t* tokens, const int32_t* parents, const float* uniforms, const float* finals, const int32_t* row_starts, int n_seqs,
                          int32_t* path, int32_t* out, int32_t* accepted, void* hip_stream)
{
    if (!v) return GQSA_ERR_NULL;
    if (n_rows == 0) {      // (nothing but `accepted`, whatever the rest is)
        if (n_seqs < 0) return GQSA_ERR_SHAPE;
        if (n_seqs == 0) return GQSA_OK;
        if (!accepted) return GQSA_ERR_NULL;
        if (!words(accepted)) return GQSA_ERR_ALIGN;
        if (n_seqs > v->max_seqs) return GQSA_ERR_BUFSIZE;
        gqsa::VerifyCall c{};
        c.accepted = accepted, c.vocab = 1, c.n_seqs = n_seqs;
        return gqsa::verify(v, c, hip_stream);
    }
    if (n_rows < 0 || n_rows > kMostRows || n_seqs < 1 || vocab < 1) return GQSA_ERR_SHAPE;
    if (!finals || !accepted || !target || !tokens || !uniforms || !path || !out) return GQSA_ERR_NULL;
    if (target_row < 0 || draft_row < 0 || target_row > (int64_t{1} << 31) || draft_row > (int64_t{1} << 31)) return GQSA_ERR_SHAPE;
    if (!row_starts && n_rows != n_seqs) return GQSA_ERR_SHAPE;
    if (draft && parents) return GQSA_ERR_UNSUPPORTED;
    if (!words(target) || !words(draft) || !words(tokens) || !words(parents) || !words(uniforms) || !words(finals) || !words(row_starts) || !words(path) ||
        !words(out) || !words(accepted))
        return GQSA_ERR_ALIGN;
    if (n_seqs > v->max_seqs || vocab > v->max_vocab) return GQSA_ERR_BUFSIZE;
    const gqsa::VerifyCall c{target, draft, target_row, draft_row, n_rows, tokens, parents, row_starts, uniforms, finals, path, out, accepted, vocab, n_seqs};
    return gqsa::verify(v, c, hip_stream);
}

}  // extern "C"
