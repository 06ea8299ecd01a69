// Verification of drafted tokens against the target's probabilities (gqsa_verify): which rows stand, the way through them, and one more token drawn from what is
// left of the probabilities behind the way's last row.
//
// Whether a row stands hangs on one probability of the target and one of the draft; of a whole row of the vocabulary only the way's last one is read, once.
// Its weights are summed in 64 bits: where the drawn token's running sum passes v times the whole is then the same whatever the order of additions
// (a vocabulary of 128256 has as many borders, and sums in 32 bits would move each of them by 10^-7).
//
// A workgroup takes 4096 tokens of a sequence's vocabulary and finds the way by itself, as this is quicker than to be told.  The sums of its tokens' weights go to the
// workspace, and the last workgroup of a sequence to arrive looks for the token: among the sums first, then among the 4096 of one workgroup.
#include <hip/hip_runtime.h>

#include "gqsa_device.hpp"
#include "gqsa_verify.hpp"

namespace gqsa {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMostRows = 1024;                         // of a sequence that are looked at
constexpr int kSteps = kVerifyChunk / (4 * kThreads);   // of four weights a thread
constexpr int kMostChunks = (1 << 22) / kVerifyChunk;

// (a row of probabilities may begin at any word)
typedef float loose4_t __attribute__((ext_vector_type(4), aligned(4)));

struct VerifyShared {
    int parent[kMostRows], token[kMostRows], path[kMostRows];
    float probability[kMostRows], drawn_from[kMostRows], uniform[kMostRows];
    bool stands[kMostRows], again[kMostRows];
    uint32_t taken[kVerifyChunk / 32];      // of the chunk's tokens, those of children
    double upto[kMostChunks];               // running sums of the chunks
    double part[kSteps][kWaves];
    int row, depth, last, chunk, found, last_positive;
};

__device__ __forceinline__ float probability_of(float p) { return p > 0.0f && p < __builtin_inff() ? p : 0.0f; }

__device__ __forceinline__ double wave_sum_upto(double v, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double before = __shfl_up(v, d);
        if (lane >= d) v += before;
    }
    return v;
}

// Four weights from token `at` on: of `target`, less those of `draft` where there is one, 0 for the tokens of `taken` (their chunk's from `at` on).
__device__ __forceinline__ void load4(const float* target, const float* draft, int at, int vocab, uint32_t taken, double (&w)[4])
{
    float p[4] = {}, d[4] = {};
    if (at + 3 < vocab) {
        const loose4_t v = *reinterpret_cast<const loose4_t*>(target + at);
        p[0] = v[0], p[1] = v[1], p[2] = v[2], p[3] = v[3];
        if (draft) {
            const loose4_t u = *reinterpret_cast<const loose4_t*>(draft + at);
            d[0] = u[0], d[1] = u[1], d[2] = u[2], d[3] = u[3];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (at + e >= vocab) continue;
            p[e] = target[at + e];
            if (draft) d[e] = draft[at + e];
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const double less = static_cast<double>(probability_of(p[e])) - static_cast<double>(probability_of(d[e]));
        w[e] = less > 0.0 && !(taken >> e & 1) ? less : 0.0;
    }
}

struct Weights {
    const float *target, *draft;
    int vocab;
    const uint32_t* taken;      // (none: no token is)

    __device__ __forceinline__ void load(int chunk, double (&w)[kSteps][4]) const
    {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int within = (s * kThreads + threadIdx.x) * 4;
            load4(target, draft, chunk * kVerifyChunk + within, vocab, taken ? taken[within / 32] >> within % 32 : 0u, w[s]);
        }
    }
};

// The sum of a chunk's weights, for every thread.
__device__ __forceinline__ double chunk_sum(const double (&w)[kSteps][4], VerifyShared& shared)
{
    double sum = 0.0;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) sum += (w[s][0] + w[s][1]) + (w[s][2] + w[s][3]);
#pragma unroll
    for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared.part[0][threadIdx.x >> 6] = sum;
    __syncthreads();
    return (shared.part[0][0] + shared.part[0][1]) + (shared.part[0][2] + shared.part[0][3]);
}

// Of the chunk's tokens, the first at which the running sum (from `before` on) passes `border`, or the last of a positive weight.
__device__ __forceinline__ int find_token(const double (&w)[kSteps][4], int chunk, double before, double border, VerifyShared& shared)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double upto[kSteps];
    if (threadIdx.x == 0) shared.found = 1 << 30, shared.last_positive = -1;
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        upto[s] = wave_sum_upto((w[s][0] + w[s][1]) + (w[s][2] + w[s][3]), lane);
        if (lane == 63) shared.part[s][wave] = upto[s];
    }
    __syncthreads();
    int found = 1 << 30, last = -1;
    double sum = before;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
            if (v == wave) {
                const double own = (w[s][0] + w[s][1]) + (w[s][2] + w[s][3]);
                double running = sum + (upto[s] - own);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at = chunk * kVerifyChunk + (s * kThreads + threadIdx.x) * 4 + e;
                    running += w[s][e];
                    if (w[s][e] > 0.0) {
                        last = at;
                        if (running > border && found == 1 << 30) found = at;
                    }
                }
            }
            sum += shared.part[s][v];
        }
    if (found != 1 << 30) atomicMin(&shared.found, found);
    if (last >= 0) atomicMax(&shared.last_positive, last);
    __syncthreads();
    return shared.found != 1 << 30 ? shared.found : shared.last_positive;
}

__global__ __launch_bounds__(kThreads) void verify_kernel(VerifyCall c, int chunks, double* sums, int32_t* arrivals)
{
    __shared__ VerifyShared shared;
    const int b = blockIdx.x / static_cast<unsigned>(chunks), chunk = blockIdx.x % static_cast<unsigned>(chunks), lane = threadIdx.x & 63;
    const Rows rows = rows_between(c.row_starts ? c.row_starts[b] : b, c.row_starts ? c.row_starts[b + 1] : b + 1, c.n_rows);
    if (rows.count == 0) {
        if (chunk == 0 && threadIdx.x == 0) c.accepted[b] = -1;
        return;
    }
    const int n = min(rows.count, kMostRows);
    const int64_t start = rows.start;

    // what each row hangs on
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int token = c.tokens[start + i];
        int parent = i == 0 ? -1 : c.parents ? c.parents[start + i] : i - 1;
        if (parent >= i) parent = -1;
        float p = 0.0f, d = 1.0f;
        if (parent >= 0 && token >= 0 && token < c.vocab) {
            p = probability_of(c.target[(start + parent) * c.target_row + token]);
            if (c.draft) d = probability_of(c.draft[(start + i) * c.draft_row + token]);
        }
        shared.parent[i] = parent < 0 ? -1 : parent, shared.token[i] = token;
        shared.probability[i] = p, shared.drawn_from[i] = d, shared.uniform[i] = c.uniforms[start + i];
    }
    for (int i = threadIdx.x; i < kVerifyChunk / 32; i += kThreads) shared.taken[i] = 0;
    __syncthreads();
    if (c.parents) {
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const int parent = shared.parent[i], token = shared.token[i];
            bool again = false;
            if (parent >= 0)
                for (int j = parent + 1; j < i; ++j) again |= shared.parent[j] == parent && shared.token[j] == token;
            shared.again[i] = again;
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int parent = shared.parent[i];
        double m = shared.drawn_from[i], p = shared.probability[i];
        if (c.parents && parent >= 0) {
            for (int j = parent + 1; j < i; ++j)
                if (shared.parent[j] == parent && !shared.again[j]) m -= static_cast<double>(shared.probability[j]);
            if (shared.again[i]) p = 0.0;
        }
        shared.stands[i] = parent >= 0 && p > 0.0 && static_cast<double>(shared.uniform[i]) * m < p;
    }
    __syncthreads();

    // the way
    if (threadIdx.x < 64) {
        int row = 0, depth = 0;
        if (lane == 0) shared.path[0] = 0;
        for (;;) {
            int next = -1;
            for (int i0 = (row + 1) & ~63; i0 < n && next < 0; i0 += 64) {
                const int i = i0 + lane;
                const uint64_t children = __builtin_amdgcn_ballot_w64(i > row && i < n && shared.parent[min(i, n - 1)] == row && shared.stands[min(i, n - 1)]);
                if (children) next = i0 + __builtin_ctzll(children);
            }
            if (next < 0) break;
            row = next;
            if (lane == 0) shared.path[++depth] = row;
        }
        if (lane == 0) shared.row = row, shared.depth = depth;
    }
    __syncthreads();
    const int row = shared.row, depth = shared.depth;

    // this chunk's weights
    Weights weights{c.target + (start + row) * c.target_row, nullptr, c.vocab, nullptr};
    if (c.draft) {
        if (row + 1 < n) weights.draft = c.draft + (start + row + 1) * c.draft_row;
    }
    const auto mark = [&](int of) {      // the tokens of the last row's children, of that chunk's
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const int within = shared.token[i] - of * kVerifyChunk;
            if (shared.parent[i] == row && within >= 0 && within < kVerifyChunk) atomicOr(&shared.taken[within / 32], 1u << within % 32);
        }
        __syncthreads();
    };
    if (!c.draft) {
        weights.taken = shared.taken;
        mark(chunk);
    }
    double w[kSteps][4];
    weights.load(chunk, w);
    const double sum = chunk_sum(w, shared);
    double* all = sums + int64_t{b} * chunks;
    if (threadIdx.x == 0) {
        __hip_atomic_store(all + chunk, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        shared.last = __hip_atomic_fetch_add(arrivals + b, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == chunks - 1;
        if (shared.last) __hip_atomic_store(arrivals + b, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // (for the next call)
    }
    __syncthreads();
    if (!shared.last) return;

    // the last workgroup of the sequence: the running sums of the chunks, then of one chunk's tokens
    for (int i = threadIdx.x; i < chunks; i += kThreads) shared.upto[i] = __hip_atomic_load(all + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const auto run_up = [&] {
        if (threadIdx.x < 64) {
            double before = 0.0;
            for (int i0 = 0; i0 < chunks; i0 += 64) {
                const int i = min(i0 + lane, chunks - 1);
                const double upto = before + wave_sum_upto(i0 + lane < chunks ? shared.upto[i] : 0.0, lane);
                if (i0 + lane < chunks) shared.upto[i] = upto;
                before = __shfl(upto, 63);
            }
        }
        __syncthreads();
    };
    run_up();
    if (!(shared.upto[chunks - 1] > 0.0)) {         // (seldom: nothing is left, so all of the target's)
        weights.draft = nullptr, weights.taken = nullptr;
        for (int i = 0; i < chunks; ++i) {
            weights.load(i, w);
            const double own = chunk_sum(w, shared);
            if (threadIdx.x == 0) shared.upto[i] = own;
        }
        __syncthreads();
        run_up();
    }
    const double whole = shared.upto[chunks - 1], border = static_cast<double>(c.finals[b]) * whole;
    if (threadIdx.x < 64) {
        int at = -1, last = 0;
        for (int i0 = 0; i0 < chunks && at < 0; i0 += 64) {
            const int i = min(i0 + lane, chunks - 1);
            const double upto = shared.upto[i];
            const uint64_t beyond = __builtin_amdgcn_ballot_w64(i0 + lane < chunks && upto > border);
            const uint64_t grows = __builtin_amdgcn_ballot_w64(i0 + lane < chunks && upto > (i > 0 ? shared.upto[i - 1] : 0.0));
            if (beyond) at = i0 + __builtin_ctzll(beyond);
            if (grows) last = i0 + 63 - __builtin_clzll(grows);
        }
        if (lane == 0) shared.chunk = at < 0 ? last : at;
    }
    __syncthreads();
    const int of = shared.chunk;
    if (weights.taken && of != chunk) {
        for (int i = threadIdx.x; i < kVerifyChunk / 32; i += kThreads) shared.taken[i] = 0;
        __syncthreads();
        mark(of);
    }
    weights.load(of, w);
    const int drawn = find_token(w, of, of > 0 ? shared.upto[of - 1] : 0.0, border, shared);
    for (int i = threadIdx.x; i < rows.count; i += kThreads) {
        c.path[start + i] = i <= depth ? shared.path[i] : -1;
        c.out[start + i] = i < depth ? shared.token[shared.path[i + 1]] : i == depth ? drawn : -1;
    }
    if (threadIdx.x == 0) c.accepted[b] = depth;
}

}  // namespace

gqsa_status_t verifier_allocate(gqsa_verifier* v)
{
    GQSA_HIP(hipGetDevice(&v->device));
    void* p = nullptr;
    GQSA_HIP(hipMalloc(&p, static_cast<size_t>(v->max_chunks()) * sizeof(double)));
    v->d_sums = static_cast<double*>(p);
    GQSA_HIP(hipMalloc(&p, static_cast<size_t>(v->max_seqs) * sizeof(int32_t)));
    v->d_arrivals = static_cast<int32_t*>(p);
    GQSA_HIP(hipMemset(v->d_arrivals, 0, static_cast<size_t>(v->max_seqs) * sizeof(int32_t)));
    GQSA_HIP(hipDeviceSynchronize());
    return GQSA_OK;
}

void verifier_release(gqsa_verifier* v)
{
    if (v->d_sums) (void)hipFree(v->d_sums);
    if (v->d_arrivals) (void)hipFree(v->d_arrivals);
    v->d_sums = nullptr;
    v->d_arrivals = nullptr;
}

gqsa_status_t verify(gqsa_verifier* v, const VerifyCall& call, void* stream)
{
    int dev = -1;
    GQSA_HIP(hipGetDevice(&dev));
    if (dev != v->device) return GQSA_ERR_HIP;
    const int chunks = call.chunks();
    const unsigned grid = static_cast<unsigned>(call.n_seqs) * static_cast<unsigned>(chunks);
    hipLaunchKernelGGL(verify_kernel, dim3(grid), dim3(kThreads), 0, static_cast<hipStream_t>(stream), call, chunks, v->d_sums, v->d_arrivals);
    GQSA_HIP(hipGetLastError());
    return GQSA_OK;
}

}  // namespace gqsa
