// The forward pass of the gated block and of the loss: Z_t block by block on the matrix cores, and what becomes of it, act(Zg) Zu or the
// running maximum and sum of a softmax, in the registers in which it is.
//
// A workgroup holds the parts of F1 and F2 that its blocks of columns need in LDS, laid out as fragments, and goes over its tokens.  A unit is one
// token times 16*N columns q2 of U and Z: one wavefront computes them from the token's row (read straight into operand registers) without
// exchanging anything with another one, so there is no barrier after the factors are in place.  A unit's U stays in registers, where it is
// the right operand of Z = F1^T U (chained order); lanes own N neighbouring columns, so that N blocks side by side are stored in pieces of N
// elements.  Few tokens: the columns q1 and q2 are cut over more workgroups (grid y and z).
//
// Bounds and figures, bf16, 8192 tokens:
//   gated 64x128,64x128  112 us: 86 GFLOP (both parts of U counted; 770 TFLOP/s), 336 MB (3.0 TB/s).  A result costs 11 vector instructions, two
//       of them at a quarter of the rate, so that the vector units are busy for 62% of the time and the matrix cores for 39%, and the two wavefronts of a
//       SIMD hide only part of one behind the other.  Units of 32 columns, four wavefronts a SIMD, the next block's products among a block's
//       activations, X a unit ahead: 121, 148, 134, 117 us.
//   loss 64x256,64x256  147 us with loss_join: 155 GFLOP (1050 TFLOP/s) and 537 million exponentials and additions: vector units 69%, matrix cores 46%.
#pragma once
#include "factored_core.hpp"

namespace km {

struct ForwardArgs {
    const void* x;
    const void* f1[2];                     // gate and up; the loss has one product
    const void* f2[2];
    void* y;                               // gated: T x Q1*Q2
    const int64_t* targets;                // loss: T
    float2* partial;                       // loss: T x parts, maximum (times log2 e) and sum of a unit's columns
    float* picked;                         // loss: T, the target's logit; written where there is one
    int64_t ldx, vocab;
    int tokens, P1, Q1, P2, Q2;            // Q1: of the loss only the columns that reach into the vocabulary
    int ld1, n2;                           // columns of F1 in memory; columns of F2 that are used (fewer than Q2 only if the vocabulary is)
    int q1_step, q2_step;                  // columns of a workgroup: multiples of 16 and 16*N
    int parts;
    int y_vec, f_vec;                      // rows can be written N elements at a time, the factors' read four
    int y_stream;                          // y is larger than the caches: written past them
};

template <typename T, int OP, int KC1, int KC2, int N, int THREADS>
__global__ __launch_bounds__(THREADS) void factored_forward(ForwardArgs a)
{
    typedef typename Op<T>::Frag Frag;
    typedef T Piece __attribute__((ext_vector_type(N)));
    constexpr int BR = OP == OP_LOSS ? 1 : 2, B1 = 2 * KC1;
    constexpr bool SPLIT = Op<T>::split, AHEAD = OP == OP_LOSS && KC1 * KC2 * (int)sizeof(T) <= 8;      // the next unit's X is loaded while one is worked on (the gated block's two products leave no registers)
    extern __shared__ __align__(32) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const Lane<T> at(lane);
    const int c = at.c, g = at.g;
    const int q1_first = blockIdx.y * a.q1_step, q2_first = blockIdx.z * a.q2_step;
    const int q1_count = min(a.q1_step, a.Q1 - q1_first), q2_count = min(a.q2_step, a.n2 - q2_first);
    const int q1_blocks = (q1_count + 15) >> 4, units = (q2_count + 16 * N - 1) / (16 * N);

    // F1: rows q1, contraction p1 (mixed, as X's rows are read).  F2: rows q2, contraction p2 (straight); row v of a unit's 16*N is column (v%16)*N + v/16
    T* const s1 = reinterpret_cast<T*>(smem);
    const int s1_branch = q1_blocks * KC1 * FRAG;
    T* const s2 = s1 + BR * s1_branch;
    const int s2_branch = units * N * KC2 * FRAG;
#pragma unroll
    for (int b = 0; b < BR; ++b) {
        lay_out<MIXED, true>(s1 + b * s1_branch, (const T*)a.f1[b] + q1_first, q1_count, a.P1, a.ld1, q1_blocks, KC1, a.f_vec, threadIdx.x, blockDim.x, InPlace());
        lay_out<STRAIGHT, true>(s2 + b * s2_branch, (const T*)a.f2[b] + q2_first, q2_count, a.P2, a.Q2, units * N, KC2, a.f_vec, threadIdx.x, blockDim.x, [](int col) {
            const int in = col % (16 * N);
            return col - in + (in % N) * 16 + in / N;
        });
    }
    __syncthreads();

    // This wavefront's units, `step` apart
    const unsigned step = gridDim.x * waves, start = blockIdx.x * waves + wave;
    const int t_step = step / units, block_step = step % units;
    int t = start / units, block = start % units;
    const int total = a.P1 * a.P2;
    const bool ragged = a.P2 % 8 != 0;
    Frag xf[AHEAD ? KC2 : 1][B1];
    auto load_x = [&](int t, int k, Frag (&f)[B1]) __attribute__((always_inline)) {
        const T* const x = (const T*)a.x + t * a.ldx;
#pragma unroll
        for (int i = 0; i < B1; ++i) {
            const int p1 = mixed_row(16 * i + c), p2 = 32 * k + 8 * g;
            // Short rows are in two fragments: p1 = 4 to 6 are in the second one.  (Classes without them ask for them all the same, and then read nothing: the
            // loads are scheduled better so.  1500 tokens 128x128,128x256: 62.5 us, 65.2 with WHOLE; one token 64x128,64x128 5.4, 5.8.)
            f[i] = eight_of_row<false>(x, p1 * a.P2 + p2, p1 < a.P1 && p2 < a.P2, total, ragged && (16 * (i | 1) + 15) * a.P2 + 32 * k + 32 > total, KC1 * KC2 == 1);
        }
    };
    if constexpr (AHEAD)
        if (t < a.tokens)
#pragma unroll
            for (int k = 0; k < KC2; ++k) load_x(t, k, xf[k]);

    while (t < a.tokens) {
        Frag u[BR][KC1][N], rest[BR][SPLIT ? KC1 : 1][SPLIT ? N : 1];
#pragma unroll
        for (int b = 0; b < BR; ++b) {
            f32x4 acc[B1][N];
#pragma unroll
            for (int i = 0; i < B1; ++i)
#pragma unroll
                for (int n = 0; n < N; ++n) acc[i][n] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < KC2; ++k) {
                if constexpr (!AHEAD) load_x(t, k, xf[0]);
                Frag f[N];
#pragma unroll
                for (int n = 0; n < N; ++n) f[n] = at.get_rows(s2 + b * s2_branch, (block * N + n) * KC2 + k);
#pragma unroll
                for (int i = 0; i < B1; ++i)
#pragma unroll
                    for (int n = 0; n < N; ++n) Op<T>::mma(acc[i][n], xf[AHEAD ? k : 0][i], f[n]);
            }
            // the loss's logits are in units of log 2, for its exponentials; so is SiLU's gate
            if (OP == OP_LOSS || (OP == OP_SILU && b == 0))
#pragma unroll
                for (int i = 0; i < B1; ++i)
#pragma unroll
                    for (int n = 0; n < N; ++n) acc[i][n] *= LOG2E;
#pragma unroll
            for (int k = 0; k < KC1; ++k)
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    u[b][k][n] = chain<T>(acc[2 * k][n], acc[2 * k + 1][n]);
                    if constexpr (SPLIT) rest[b][k][n] = chain_rest(acc[2 * k][n], acc[2 * k + 1][n], u[b][k][n]);
                }
        }
        int t_next = t + t_step, block_next = block + block_step;
        if (block_next >= units) {
            block_next -= units;
            ++t_next;
        }
        if constexpr (AHEAD)
            if (t_next < a.tokens)
#pragma unroll
                for (int k = 0; k < KC2; ++k) load_x(t_next, k, xf[k]);

        const int col = q2_first + block * 16 * N + c * N;                  // this lane's first column
        const bool columns_inside = q2_first + (block + 1) * 16 * N <= a.n2;
        Frag f1[BR][KC1];                   // of the block that comes next
        auto load_f1 = [&](int qb) __attribute__((always_inline)) {
#pragma unroll
            for (int b = 0; b < BR; ++b)
#pragma unroll
                for (int k = 0; k < KC1; ++k) f1[b][k] = at.get_rows(s1 + b * s1_branch, qb * KC1 + k);
        };
        // Z of the block whose F1 is there, plus `start`; then the next block's F1 is on its way
        auto product = [&](f32x4 (&z)[BR][N], int qb, const f32x4 (&start)[N]) __attribute__((always_inline)) {
#pragma unroll
            for (int b = 0; b < BR; ++b)
#pragma unroll
                for (int k = 0; k < KC1; ++k) {
#pragma unroll
                    for (int n = 0; n < N; ++n) z[b][n] = Op<T>::product(f1[b][k], u[b][k][n], k ? z[b][n] : start[n]);
                    if constexpr (SPLIT)
#pragma unroll
                        for (int n = 0; n < N; ++n) Op<T>::mma(z[b][n], f1[b][k], rest[b][k][n]);
                }
            load_f1(qb + 1 < q1_blocks ? qb + 1 : 0);
        };
        load_f1(0);

        if constexpr (OP != OP_LOSS) {
            T* const y = (T*)a.y + ((int64_t)t * a.Q1 + q1_first + 4 * g) * a.Q2 + col;
            auto finish = [&](const f32x4 (&z)[BR][N], int qb, auto whole, auto past) __attribute__((always_inline)) {
                Piece h[4];
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int n = 0; n < N; ++n) h[r][n] = from_f32<T>(gate<OP == OP_GELU>(z[0][n][r], z[1][n][r]));
                T* const row = y + (int64_t)qb * 16 * a.Q2;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if constexpr (whole.value) {
                        Piece* const to = reinterpret_cast<Piece*>(row + (int64_t)r * a.Q2);
                        if constexpr (past.value) __builtin_nontemporal_store(h[r], to);
                        else *to = h[r];
                    } else {
#pragma unroll
                        for (int n = 0; n < N; ++n)
                            if (qb * 16 + 4 * g + r < q1_count && col + n < a.n2) row[(int64_t)r * a.Q2 + n] = h[r][n];
                    }
                }
            };
            f32x4 z[BR][N], zero[N];
#pragma unroll
            for (int n = 0; n < N; ++n) zero[n] = f32x4{0, 0, 0, 0};
            int qb = 0;
            if (a.y_vec && columns_inside) {
                if (a.y_stream)
                    for (; qb < q1_count >> 4; ++qb) {
                        product(z, qb, zero);
                        finish(z, qb, Yes(), Yes());
                    }
                else
                    for (; qb < q1_count >> 4; ++qb) {
                        product(z, qb, zero);
                        finish(z, qb, Yes(), No());
                    }
            }
            for (; qb < q1_blocks; ++qb) {
                product(z, qb, zero);
                finish(z, qb, No(), No());
            }
        } else {
            const int64_t target = a.targets[t];
            const int target_q1 = target >= 0 && target < a.vocab ? (int)((unsigned)target / (unsigned)a.Q2) : -1, target_q2 = (int)target - target_q1 * a.Q2;
            // What of block qb lies outside the vocabulary is -inf.
            auto cut = [&](f32x4 (&z)[N], int qb) __attribute__((always_inline)) {
                const int64_t first = (int64_t)(q1_first + qb * 16 + 4 * g) * a.Q2 + col;
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (col + n >= a.n2 || first + (int64_t)r * a.Q2 + n >= a.vocab) z[n][r] = -INFINITY;
            };
            auto highest = [&](const f32x4 (&z)[N]) __attribute__((always_inline)) {
                float high = z[0][0];
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) high = fmaxf(high, z[n][r]);
                return high;
            };
            auto add_up = [&](const f32x4 (&z)[N], float from) __attribute__((always_inline)) {
                float s[4] = {0, 0, 0, 0};
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[r] += __builtin_amdgcn_exp2f(z[n][r] - from);
                return (s[0] + s[1]) + (s[2] + s[3]);
            };
            // A lane's exponentials are relative to its highest logit in the first block.  It need not be the highest of all: a sum in fp32 holds
            // terms of up to 2^127.  So the products' sums start from minus that reference, and a logit costs an exponential and an addition.
            // Columns past the end start from -inf instead.  Blocks up to `inside` have no row that is outside the vocabulary or reaches out of it.
            const int inside = q1_blocks - (q1_count & 15 || (int64_t)(q1_first + q1_count) * a.Q2 > a.vocab);
            f32x4 z[2][BR][N], start[N];
            auto start_from = [&](float v) __attribute__((always_inline)) {
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const float f = col + n < a.n2 ? v : -INFINITY;
                    start[n] = f32x4{f, f, f, f};
                }
            };
            start_from(0.0f);
            product(z[0], 0, start);
            if (inside < 1) cut(z[0][0], 0);
            float top = highest(z[0][0]);
            if (!(fabsf(top) < INFINITY)) top = 0.0f;       // nothing of the vocabulary, or beyond numbers: see below
            float sum = add_up(z[0][0], top);
            start_from(-top);
            int qb = 1;
            // (two blocks in turn: one's products while the other's exponentials are taken)
            if (qb < inside) {
                product(z[0], qb, start);
                for (; qb + 2 < inside; qb += 2) {
                    product(z[1], qb + 1, start);
                    sum += add_up(z[0][0], 0.0f);
                    product(z[0], qb + 2, start);
                    sum += add_up(z[1][0], 0.0f);
                }
                sum += add_up(z[0][0], 0.0f);
                ++qb;
            }
            for (; qb < q1_blocks; ++qb) {
                product(z[0], qb, start);
                if (qb >= inside) cut(z[0][0], qb);
                sum += add_up(z[0][0], 0.0f);
            }
            if (__any(sum > 0x1p100f)) {                    // logits more than 2^100 times the reference's: once more, with the highest so far
                load_f1(0);
                start_from(0.0f);
                top = -INFINITY;
                sum = 0;
                for (int qb = 0; qb < q1_blocks; ++qb) {
                    product(z[0], qb, start);
                    cut(z[0][0], qb);
                    const float high = fmaxf(highest(z[0][0]), top), from = high == -INFINITY ? 0.0f : high;
                    sum = sum * __builtin_amdgcn_exp2f(top - from) + add_up(z[0][0], from);
                    top = high;
                }
            }
            if (sum == 0) top = -INFINITY;                  // nothing of the vocabulary in this lane
#pragma unroll
            for (int d = 32; d; d >>= 1) {
                const float other_top = __shfl_xor(top, d), other_sum = __shfl_xor(sum, d), high = fmaxf(top, other_top);
                const float from = high == -INFINITY ? 0.0f : high;
                sum = sum * __builtin_amdgcn_exp2f(top - from) + other_sum * __builtin_amdgcn_exp2f(other_top - from);
                top = high;
            }
            const int part = blockIdx.y * ((a.n2 + 16 * N - 1) / (16 * N)) + q2_first / (16 * N) + block;
            if (lane == 0) a.partial[(int64_t)t * a.parts + part] = make_float2(top, sum);

            // the target's logit, where it is in this unit: its column of U times its column of F1, over the four lanes that share the column
            const int in = target_q2 - (q2_first + block * 16 * N);
            if (target_q1 >= q1_first && target_q1 < q1_first + q1_count && in >= 0 && in < 16 * N) {
                float logit = 0;
#pragma unroll
                for (int k = 0; k < KC1; ++k) {
                    const Frag f = at.get_row(s1, ((target_q1 - q1_first) >> 4) * KC1 + k, (target_q1 - q1_first) & 15);
#pragma unroll
                    for (int n = 0; n < N; ++n)
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            float v = to_f32<T>(u[0][k][n][j]);
                            if constexpr (SPLIT) v += to_f32<T>(rest[0][k][n][j]);
                            if (in % N == n) logit = __builtin_fmaf(v, to_f32<T>(f[j]), logit);
                        }
                }
                logit += __shfl_xor(logit, 16);
                logit += __shfl_xor(logit, 32);
                if (lane == in / N) a.picked[t] = logit * LN2;
            }
        }
        t = t_next;
        block = block_next;
    }
}

}  // namespace km
