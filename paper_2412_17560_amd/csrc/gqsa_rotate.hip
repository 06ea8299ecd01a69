// Norms of queries and keys per head with the rotation by position in the same pass (gqsa_qk_norm_rotate):
//   u = x rsqrt(mean(x^2) + eps) w,   (a, b) -> (a c - b s, a s + b c)
// Every element is read and written once and nothing else of note is: the kernel is bound by memory for many rows and by the launch for
// few.  A lane holds two runs of 8 elements of a head whose elements are each other's partners in the rotation (runs p and
// p + rotary_dim / 16, or two neighbouring runs), so that the rotation needs no exchange between lanes and the norm's sum
// one over the head_dim / 16 lanes of a head; (c, s) of its 8 pairs stay in registers over all heads of a row.
// 8192 rows of 72 heads of 128 take 62 us, 4.9 TB/s of the 5.2 that a large copy reaches; one row 3.0 us, where an empty launch takes 1.6.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gqsa_attention.hpp"

namespace gqsa {
namespace {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

struct Pair {
    half8_t a, b;
};

// LANES (a power of two) lanes to a head; each wavefront takes one row and every `stride`-th set of 64 / LANES heads of it.
template <int LANES, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateCall c, int waves_per_row)
{
    constexpr int kHeadsAtOnce = 64 / LANES;
    const int lane = threadIdx.x & 63;
    const int64_t wave = blockIdx.x * int64_t{kThreads / 64} + (threadIdx.x >> 6);
    const int64_t row = wave / waves_per_row;
    if (row >= c.n_rows) return;
    const int part = static_cast<int>(wave - row * waves_per_row);
    const int p = lane % LANES, turned = c.rotary_dim / 16;
    const bool held = p < c.head_dim / 16, turns = p < turned;
    int run_a, run_b;                      // the lane's two runs of 8 elements
    if (INTERLEAVED) run_a = 2 * p, run_b = 2 * p + 1;
    else if (turns) run_a = p, run_b = p + turned;
    else run_a = 2 * p, run_b = 2 * p + 1;

    float cos_[8], sin_[8];
    if (held && turns) {
        const int64_t position = c.positions[row];
        const bool there = position >= 0 && position < c.n_positions;
        const float4_t* t = reinterpret_cast<const float4_t*>(c.table + ((there ? position : 0) * turned + p) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float4_t v = {__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
            if (there) v = t[i];
            cos_[2 * i] = v[0], sin_[2 * i] = v[1], cos_[2 * i + 1] = v[2], sin_[2 * i + 1] = v[3];
        }
    }

    const int heads = c.q_heads + c.k_heads;
    const auto place = [&](int head, bool out) -> uint16_t* {
        const bool is_q = head < c.q_heads;
        const Heads& a = is_q ? (out ? c.q_out : c.q) : (out ? c.k_out : c.k);
        return a.data + row * a.row + (is_q ? head : head - c.q_heads) * a.head;
    };
    const auto load = [&](int head) {
        Pair x{};
        if (held && head < heads) {
            const uint16_t* at = place(head, false);
            x.a = *reinterpret_cast<const half8_t*>(at + 8 * run_a);
            x.b = *reinterpret_cast<const half8_t*>(at + 8 * run_b);
        }
        return x;
    };
    const int first = part * kHeadsAtOnce + lane / LANES, stride = waves_per_row * kHeadsAtOnce;
    Pair next = load(first);
    for (int head0 = part * kHeadsAtOnce; head0 < heads; head0 += stride) {
        const int head = head0 + lane / LANES;
        const Pair x = next;
        next = load(head + stride);        // (the next heads' loads are under way while these are computed)
        float a[8], b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = static_cast<float>(x.a[i]), b[i] = static_cast<float>(x.b[i]);
        const uint16_t* weight = head < c.q_heads ? c.q_weight : c.k_weight;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(a[i], a[i], __builtin_fmaf(b[i], b[i], sum));
#pragma unroll
        for (int m = 1; m < LANES; m *= 2) sum += __shfl_xor(sum, m);
        if (!held || head >= heads) continue;
        if (weight) {
            const float r = rsqrtf(__builtin_fmaf(sum, c.one_over_dim, c.eps));
            const half8_t wa = *reinterpret_cast<const half8_t*>(weight + 8 * run_a);
            const half8_t wb = *reinterpret_cast<const half8_t*>(weight + 8 * run_b);
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] *= r * static_cast<float>(wa[i]), b[i] *= r * static_cast<float>(wb[i]);
        }
        if (turns) {
            if (INTERLEAVED) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a0 = a[2 * i], a1 = a[2 * i + 1], b0 = b[2 * i], b1 = b[2 * i + 1];
                    a[2 * i] = a0 * cos_[i] - a1 * sin_[i], a[2 * i + 1] = a0 * sin_[i] + a1 * cos_[i];
                    b[2 * i] = b0 * cos_[4 + i] - b1 * sin_[4 + i], b[2 * i + 1] = b0 * sin_[4 + i] + b1 * cos_[4 + i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float a0 = a[i], b0 = b[i];
                    a[i] = a0 * cos_[i] - b0 * sin_[i], b[i] = a0 * sin_[i] + b0 * cos_[i];
                }
            }
        }
        half8_t ya, yb;
#pragma unroll
        for (int i = 0; i < 8; ++i) ya[i] = static_cast<_Float16>(a[i]), yb[i] = static_cast<_Float16>(b[i]);
        uint16_t* at = place(head, true);
        *reinterpret_cast<half8_t*>(at + 8 * run_a) = ya;
        *reinterpret_cast<half8_t*>(at + 8 * run_b) = yb;
    }
}

template <int LANES>
void launch(const RotateCall& c, hipStream_t s)
{
    constexpr int kHeadsAtOnce = 64 / LANES;
    const int sets = (c.q_heads + c.k_heads + kHeadsAtOnce - 1) / kHeadsAtOnce;
    // A wavefront keeps its row's part of the table in registers over all the heads it takes, so few to a row read it less often; but there should be some
    // four times as many as the chip holds at once (7 a SIMD), or the last of them run alone: 8192 rows of 72 heads of 128 took 73.6 us with
    // 8192 wavefronts, 66.0, 63.1 and 62.6 with 16384, 32768 and all of one set of heads each; 16384 rows of 40 heads of 64 41.9, 41.6, 39.5, 41.0.
    const int waves_per_row = static_cast<int>(std::min<int64_t>(sets, std::max<int64_t>(1, 32768 / c.n_rows)));
    const int64_t waves = c.n_rows * waves_per_row;
    const dim3 grid(static_cast<unsigned>((waves + kThreads / 64 - 1) / (kThreads / 64)));
    if (c.interleaved) hipLaunchKernelGGL((rotate_kernel<LANES, true>), grid, dim3(kThreads), 0, s, c, waves_per_row);
    else hipLaunchKernelGGL((rotate_kernel<LANES, false>), grid, dim3(kThreads), 0, s, c, waves_per_row);
}

}  // namespace

gqsa_status_t rotate(const RotateCall& call, void* stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int runs = call.head_dim / 16;
    if (runs > 8) launch<16>(call, s);
    else if (runs > 4) launch<8>(call, s);
    else if (runs > 2) launch<4>(call, s);
    else if (runs > 1) launch<2>(call, s);
    else launch<1>(call, s);
    GQSA_HIP(hipGetLastError());
    return GQSA_OK;
}

}  // namespace gqsa
