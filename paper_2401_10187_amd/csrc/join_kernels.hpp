// What joins the parts that workgroups of the operators leave: sums of gradients, and the maxima and sums of softmaxes.
#pragma once
#include "factored_core.hpp"

namespace km {

// Sums over parts that lie `step` elements apart, in their order; columns past `cols` of a row of the result get zeros (a
// vocabulary may end before a factor's columns do).  Many parts of few elements (gradients of factors and norms, a part from each workgroup): a
// workgroup takes 64 elements and its 16 groups of 16 threads every 16th part.  Few parts of many elements (dX): a thread takes 4 elements.
// Bound by memory, most of it the last-level cache's: 2 x 16 MiB in 256 parts 7.5 us (4.5 TB/s).
struct SumJob {
    const float* in;
    void* out;
    int64_t n, step;                       // elements of the result
    int parts;
    int64_t row, cols;                     // a row's elements, of which `cols` were written
    int64_t blocks;                        // workgroups before the next job's (set by sum_up)
};
constexpr int SUM_FEW = 16, SUM_JOBS = 5;
struct SumArgs {
    SumJob job[SUM_JOBS];
    int64_t first;                         // of all workgroups, where this launch's start (set by sum_up)
};

inline int sum_span(const SumJob& j) { return j.parts <= SUM_FEW ? 1024 : 64; }

template <typename T>
__global__ __launch_bounds__(256) void sum_parts(SumArgs a)
{
    int64_t block = a.first + blockIdx.x;
    int which = 0;
    while (which + 1 < SUM_JOBS && block >= a.job[which].blocks) block -= a.job[which++].blocks;
    const SumJob job = a.job[which];
    const bool few = job.parts <= SUM_FEW;
    const int e = few ? threadIdx.x : threadIdx.x & 15, y = few ? 0 : threadIdx.x >> 4, by = few ? 1 : 16;
    const int64_t at = block * (few ? 1024 : 64) + 4 * e;
    const bool vec = (job.n & 3) == 0 && (job.step & 3) == 0;
    f32x4 sum = {0, 0, 0, 0};
    if (vec) {
        if (at < job.n) {
            const float* p = job.in + at;
#pragma unroll 8
            for (int i = y; i < job.parts; i += by) sum += *reinterpret_cast<const f32x4*>(p + i * job.step);
        }
    } else {
#pragma unroll 4
        for (int i = y; i < job.parts; i += by)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[k] += at + k < job.n ? job.in[i * job.step + at + k] : 0.0f;
    }
    if (!few) {
        __shared__ f32x4 s[16][16];
        s[y][e] = sum;
        __syncthreads();
        if (y) return;
#pragma unroll
        for (int i = 1; i < 16; ++i) sum += s[i][e];
    }
    if (job.cols < job.row)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if ((at + k) % job.row >= job.cols) sum[k] = 0.0f;
    T* const out = (T*)job.out;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (at + k < job.n) out[at + k] = from_f32<T>(sum[k]);
}

// The parts of every token's softmax joined, 16 lanes to a token, four loads of a lane at once.  Bound by latency: 8192 tokens of 4 parts 5 us, one token
// of 256 parts 3 us (6 with one load at a time).
static __global__ __launch_bounds__(256) void loss_join(const float2* __restrict__ partial, const float* __restrict__ picked, const int64_t* __restrict__ targets,
                                                        int64_t vocab, int tokens, int parts, float* __restrict__ loss, float* __restrict__ lse)
{
    const int t = blockIdx.x * 16 + (threadIdx.x >> 4), e = threadIdx.x & 15;
    if (t >= tokens) return;
    const int64_t target = targets[t];
    const bool counts = target >= 0 && target < vocab;
    const float logit = e == 0 && counts ? picked[t] : 0.0f;
    float top = -INFINITY, sum = 0;
    for (int i = e; i < parts; i += 64) {
        float2 p[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = i + 16 * j < parts ? partial[(int64_t)t * parts + i + 16 * j] : make_float2(-INFINITY, 0.0f);
        const float high = fmaxf(fmaxf(fmaxf(p[0].x, p[1].x), fmaxf(p[2].x, p[3].x)), top), from = high == -INFINITY ? 0.0f : high;
        sum *= __builtin_amdgcn_exp2f(top - from);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += p[j].y * __builtin_amdgcn_exp2f(p[j].x - from);
        top = high;
    }
#pragma unroll
    for (int d = 8; d; d >>= 1) {
        const float other_top = __shfl_xor(top, d), other_sum = __shfl_xor(sum, d), high = fmaxf(top, other_top);
        const float from = high == -INFINITY ? 0.0f : high;
        sum = sum * __builtin_amdgcn_exp2f(top - from) + other_sum * __builtin_amdgcn_exp2f(other_top - from);
        top = high;
    }
    if (e) return;
    const float l = (top + __builtin_amdgcn_logf(sum)) * LN2;
    lse[t] = l;
    loss[t] = counts ? l - logit : 0.0f;
}

}  // namespace km
