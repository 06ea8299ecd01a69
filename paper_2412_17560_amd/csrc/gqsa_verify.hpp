// Internal definitions of the verification of drafted tokens (include/gqsa_verify.h): what the C boundary (gqsa_verify_api.cpp) hands to the kernel (gqsa_verify.hip).
#pragma once

#include <cstdint>

#include "gqsa_attention.hpp"
#include "gqsa_verify.h"

namespace gqsa {

constexpr int kVerifyChunk = 16384, kVerifyRun = 2048;      // of the vocabulary: a workgroup's share of a sequence, a wavefront's

struct VerifyCall {
    const float *target, *draft;
    int64_t target_row, draft_row, n_rows;
    const int32_t *tokens, *parents, *row_starts;
    const float *uniforms, *finals;
    int32_t *path, *out, *accepted;
    int vocab, n_seqs;

    int chunks() const { return (vocab + kVerifyChunk - 1) / kVerifyChunk; }
};

}  // namespace gqsa

struct gqsa_verifier {
    int max_seqs = 0, max_vocab = 0;
    int device = -1;
    double* d_sums = nullptr;       // of every run of every sequence
    int32_t* d_arrivals = nullptr;  // a counter for every sequence, zero between calls

    int64_t max_runs() const { return int64_t{max_seqs} * ((int64_t{max_vocab} + gqsa::kVerifyRun - 1) / gqsa::kVerifyRun); }
};

namespace gqsa {

gqsa_status_t verifier_allocate(gqsa_verifier* v);
void verifier_release(gqsa_verifier* v);
gqsa_status_t verify(gqsa_verifier* v, const VerifyCall& call, void* stream);

}  // namespace gqsa
