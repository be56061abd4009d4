// Layer norm over rows of H elements: y = (x - mean) rstd w + b, and its backward pass with the gradients of w and b.
//
// Both are one pass over memory.  A team of 64, 256 or 1024 threads takes a row, CH pieces of VEC elements (16 bytes) a
// thread, and keeps it in registers between the row's mean, the sum of squares about that mean (which so cannot cancel) and the
// results.  The backward pass needs two sums of a row, sum dxhat and sum dxhat xhat; each thread also adds up dw and db of the columns that are
// its own in every row, in fp32.  A workgroup's teams join theirs in LDS, in their order, and the workgroups' sums are added
// by sum_parts, so the result does not depend on timing.  Bound by memory; few rows: by latency.  8192 rows of 4096 bf16: forward 25.8 us
// (5.2 TB/s, part of it from the last-level cache), backward 44.3 us (4.5 TB/s) and 4.7 us of sum_parts; one row: 3.2 us.
// Rows longer than a team holds are read again for each step (CH = 0).
#pragma once
#include "factored_core.hpp"

namespace km {

struct NormArgs {
    const void* x;
    const void* dy;
    const void* w;
    const void* b;                         // may be null
    void* y;                               // or dx
    float* mean;
    float* rstd;
    float* dw;                             // backward: parts x 2 x H, dw before db
    int64_t ldx, lddy;
    float eps;
    int rows, H;
};

template <typename T, int VEC> struct NormPiece { typedef T type __attribute__((ext_vector_type(VEC))); };
template <typename T> struct NormPiece<T, 1> { struct type { T v; __device__ T& operator[](int) { return v; } __device__ const T& operator[](int) const { return v; } }; };

// The sums of K values over a team, in every one of its threads.  All threads of the workgroup call it.
template <int NT, int K> __device__ __forceinline__ void team_sum(float (&v)[K], float (*s)[K])
{
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int d = 32; d; d >>= 1) v[k] += __shfl_xor(v[k], d);
    if constexpr (NT > 64) {
        const int wave = threadIdx.x >> 6, first = wave / (NT / 64) * (NT / 64);
        __syncthreads();                   // s may still be read for the sum before
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) s[wave][k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = 0;
#pragma unroll
            for (int i = 0; i < NT / 64; ++i) v[k] += s[first + i][k];
        }
    }
}

// Rows of any length: a thread adds up 256 pieces at a time and then these sums (2^30 elements in one go, 4 million squares a thread: rstd off by 2e-3).
template <int CH, int K> __device__ __forceinline__ void add_some(float (&sum)[K], float (&some)[K], int i)
{
    if (CH > 0 || i % 256 != 255) return;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        sum[k] += some[k];
        some[k] = 0;
    }
}
template <int K> __device__ __forceinline__ void add_rest(float (&sum)[K], const float (&some)[K])
{
#pragma unroll
    for (int k = 0; k < K; ++k) sum[k] += some[k];
}

// CH pieces of VEC elements in a thread's registers, or (CH = 0) as many as it takes.
#define NORM_PIECES(i) _Pragma("unroll UNROLL") for (int i = 0; i < (CH ? CH : pieces); ++i)

template <typename T, int VEC, int NT, int CH>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void norm_forward(NormArgs a)
{
    typedef typename NormPiece<T, VEC>::type Piece;
    constexpr int THREADS = NT < 256 ? 256 : NT, TEAMS = THREADS / NT, UNROLL = CH ? CH : 1;
    __shared__ float s[THREADS / 64][1];
    const int tid = threadIdx.x % NT, pieces = (a.H + NT * VEC - 1) / (NT * VEC);
    const int row = blockIdx.x * TEAMS + threadIdx.x / NT;
    const bool there = row < a.rows;
    const T* const x = (const T*)a.x + (int64_t)(there ? row : 0) * a.ldx;
    Piece v[CH ? CH : 1];
    float sum[1] = {0}, some[1] = {0};
    NORM_PIECES(i) {
        const int at = (i * NT + tid) * VEC;
        if (at >= a.H) continue;
        const Piece p = *reinterpret_cast<const Piece*>(x + at);
        if constexpr (CH > 0) v[i] = p;
#pragma unroll
        for (int e = 0; e < VEC; ++e) some[0] += to_f32<T>(p[e]);
        add_some<CH>(sum, some, i);
    }
    add_rest(sum, some);
    team_sum<NT, 1>(sum, s);
    const float mean = sum[0] / a.H;
    float square[1] = {0};
    some[0] = 0;
    NORM_PIECES(i) {
        const int at = (i * NT + tid) * VEC;
        if (at >= a.H) continue;
        Piece p;
        if constexpr (CH > 0) p = v[i];
        else p = *reinterpret_cast<const Piece*>(x + at);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float d = to_f32<T>(p[e]) - mean;
            some[0] += d * d;
        }
        add_some<CH>(square, some, i);
    }
    add_rest(square, some);
    team_sum<NT, 1>(square, s);
    const float rstd = 1.0f / sqrtf(square[0] / a.H + a.eps);
    if (!there) return;
    if (tid == 0) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
    T* const y = (T*)a.y + (int64_t)row * a.H;
    NORM_PIECES(i) {
        const int at = (i * NT + tid) * VEC;
        if (at >= a.H) continue;
        Piece p, o, b = {};
        if constexpr (CH > 0) p = v[i];
        else p = *reinterpret_cast<const Piece*>(x + at);
        const Piece w = *reinterpret_cast<const Piece*>((const T*)a.w + at);
        if (a.b) b = *reinterpret_cast<const Piece*>((const T*)a.b + at);
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] = from_f32<T>((to_f32<T>(p[e]) - mean) * rstd * to_f32<T>(w[e]) + (a.b ? to_f32<T>(b[e]) : 0.0f));
        *reinterpret_cast<Piece*>(y + at) = o;
    }
}

// dx, and in registers dw and db of a workgroup's rows.  With CH = 0 it leaves dw and db to norm_columns.
template <typename T, int VEC, int NT, int CH>
__global__ __launch_bounds__(1024) void norm_backward(NormArgs a)
{
    typedef typename NormPiece<T, VEC>::type Piece;
    constexpr int TEAMS = 1024 / NT, UNROLL = CH ? CH : 1;
    __shared__ float s[16][2];
    extern __shared__ float joined[];      // 2 x H, where there are several teams
    const int tid = threadIdx.x % NT, team = threadIdx.x / NT, pieces = (a.H + NT * VEC - 1) / (NT * VEC);
    float dw[CH ? CH : 1][VEC], db[CH ? CH : 1][VEC];
    Piece w[CH ? CH : 1];
    if constexpr (CH > 0) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int at = (i * NT + tid) * VEC;
            if (at < a.H) w[i] = *reinterpret_cast<const Piece*>((const T*)a.w + at);
#pragma unroll
            for (int e = 0; e < VEC; ++e) dw[i][e] = db[i][e] = 0;
        }
    }
    // the next row of a team is loaded while one is worked on
    Piece ax[CH ? CH : 1], ad[CH ? CH : 1];
    float amean = 0, arstd = 0;
    auto load = [&](int row) __attribute__((always_inline)) {
        if constexpr (CH > 0) {
            if (row >= a.rows) return;
            const T* const x = (const T*)a.x + (int64_t)row * a.ldx;
            const T* const dy = (const T*)a.dy + (int64_t)row * a.lddy;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int at = (i * NT + tid) * VEC;
                if (at >= a.H) continue;
                ax[i] = *reinterpret_cast<const Piece*>(x + at);
                ad[i] = *reinterpret_cast<const Piece*>(dy + at);
            }
            amean = a.mean[row];
            arstd = a.rstd[row];
        }
    };
    load(blockIdx.x * TEAMS + team);
    for (int first = blockIdx.x * TEAMS; first < a.rows; first += gridDim.x * TEAMS) {
        const int row = first + team;
        const bool there = row < a.rows;
        const int64_t r = there ? row : 0;
        const T* const x = (const T*)a.x + r * a.ldx;
        const T* const dy = (const T*)a.dy + r * a.lddy;
        const float mean = CH > 0 ? amean : a.mean[r], rstd = CH > 0 ? arstd : a.rstd[r];
        Piece px[CH ? CH : 1], pd[CH ? CH : 1];
        if constexpr (CH > 0) {
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                px[i] = ax[i];
                pd[i] = ad[i];
            }
            load(row + gridDim.x * TEAMS);
        }
        float sums[2] = {0, 0}, some[2] = {0, 0};
        NORM_PIECES(i) {
            const int at = (i * NT + tid) * VEC;
            if (at >= a.H || !there) continue;
            Piece p, d, ww;
            if constexpr (CH > 0) {
                p = px[i];
                d = pd[i];
                ww = w[i];
            } else {
                p = *reinterpret_cast<const Piece*>(x + at);
                d = *reinterpret_cast<const Piece*>(dy + at);
                ww = *reinterpret_cast<const Piece*>((const T*)a.w + at);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float xhat = (to_f32<T>(p[e]) - mean) * rstd, g = to_f32<T>(d[e]), dxhat = g * to_f32<T>(ww[e]);
                some[0] += dxhat;
                some[1] += dxhat * xhat;
                if constexpr (CH > 0) {
                    dw[i][e] += g * xhat;
                    db[i][e] += g;
                }
            }
            add_some<CH>(sums, some, i);
        }
        add_rest(sums, some);
        team_sum<NT, 2>(sums, s);
        const float m1 = sums[0] / a.H, m2 = sums[1] / a.H;
        if (!there) continue;
        T* const dx = (T*)a.y + r * a.H;
        NORM_PIECES(i) {
            const int at = (i * NT + tid) * VEC;
            if (at >= a.H) continue;
            Piece p, d, ww, o;
            if constexpr (CH > 0) {
                p = px[i];
                d = pd[i];
                ww = w[i];
            } else {
                p = *reinterpret_cast<const Piece*>(x + at);
                d = *reinterpret_cast<const Piece*>(dy + at);
                ww = *reinterpret_cast<const Piece*>((const T*)a.w + at);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float xhat = (to_f32<T>(p[e]) - mean) * rstd;
                o[e] = from_f32<T>(rstd * (to_f32<T>(d[e]) * to_f32<T>(ww[e]) - m1 - xhat * m2));
            }
            *reinterpret_cast<Piece*>(dx + at) = o;
        }
    }
    if constexpr (CH > 0) {
        float* const part = a.dw + (int64_t)blockIdx.x * 2 * a.H;
        for (int k = 0; k < TEAMS; ++k) {
            if (team == k) {
#pragma unroll
                for (int i = 0; i < CH; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const int at = (i * NT + tid) * VEC + e;
                        if (at >= a.H) continue;
                        float* const out = k == TEAMS - 1 ? part : joined;
                        out[at] = k ? joined[at] + dw[i][e] : dw[i][e];
                        out[a.H + at] = k ? joined[a.H + at] + db[i][e] : db[i][e];
                    }
            }
            if (TEAMS > 1) __syncthreads();
        }
    }
}

// dw and db of rows too long for norm_backward's registers: a thread has a column, a workgroup a slice of the rows.
template <typename T>
__global__ __launch_bounds__(256) void norm_columns(NormArgs a)
{
    const int at = blockIdx.x * 256 + threadIdx.x;
    if (at >= a.H) return;
    float dw = 0, db = 0;
    for (int row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float g = to_f32<T>(((const T*)a.dy)[(int64_t)row * a.lddy + at]);
        dw += g * ((to_f32<T>(((const T*)a.x)[(int64_t)row * a.ldx + at]) - a.mean[row]) * a.rstd[row]);
        db += g;
    }
    float* const part = a.dw + (int64_t)blockIdx.y * 2 * a.H;
    part[at] = dw;
    part[a.H + at] = db;
}

}  // namespace km
