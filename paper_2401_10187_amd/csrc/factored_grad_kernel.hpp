// The backward pass of the gated block and of the loss.  Z_t is computed again block by block (it is never
// written), becomes dZ_t in the registers in which it is, and all four products that follow from it are taken at once:
//     dU_t = F1 dZ_t,   dX_t = dU_t F2^T,   dF1 = sum_t U_t dZ_t^T,   dF2 = sum_t X_t^T dU_t.
//
// A workgroup owns a block of R1 columns q1 and R2 = 16*N*W columns q2, holds those parts of F1 and F2 in LDS, and goes over every S-th token.  Each of
// its W wavefronts owns 16*N columns q2: it computes their U, Z, dZ and dU and adds to their dF2 without exchanging anything.  dF1 and dX
// add over q2, so U, dZ (a chunk of C1 rows q1 at a time) and dU go through LDS, and the wavefronts share the results' blocks instead.  Everything is
// written to LDS as the fragments that lie in registers; where a product needs an operand the other way round (F1 for dU, X for dF2, all
// of those of dF1 and dX) it is read crossed, so each lies there once.  dF1 and dF2 stay in registers until the tokens are done; the S
// workgroups' sums are added up in a fixed order by sum_parts.  Where the columns need more than one block, dX is a sum too, of an fp32 part
// from each block.
//
// bf16: Z from U in two parts, as in the forward pass (the probabilities have to fit the forward pass's sum); dZ, dU and the U of dF1 are rounded to one
// bf16 each, as they are where layers keep their activations and gradients in bf16.  A gradient so has two such roundings before its own, errors of
// 2.9e-3 of its norm where one rounding leaves 1.7e-3 (2.3e-3 for the loss: where p is small the target's dZ is near -1, which bf16 holds).  The target's dZ is
// p - 1 before it is rounded, so that likely targets have no larger errors.  With dU in two parts dX and dF2 would have 2.4e-3, and the gated kernel
// take 357 us instead of 308 (8192 tokens 64x128,64x128); with dZ in two parts for dU 387, for dF1 too 662.
//
// Bounds and figures, bf16, 8192 tokens: gated 64x128,64x128 308 us, 189 GFLOP with both parts of U (610 TFLOP/s); loss 64x256,64x256 390 us, 326 GFLOP (835
// TFLOP/s).  Matrix cores, vector units and LDS are each busy for 30 to 50% of the time; the rest are waits that the two wavefronts of a SIMD, held
// together by a barrier for each chunk, do not hide from each other.  About 30 us of it are the factors on their way into LDS and the sums on
// their way out.  More wavefronts have no registers; four of 32 columns, two tokens in turn, waves half a chunk apart: no quicker.
#pragma once
#include "factored_core.hpp"

namespace km {

struct GradArgs {
    const void* x;
    const void* f1[2];
    const void* f2[2];
    const void* dh;                        // gated: T x Q1*Q2
    const int64_t* targets;                // loss: T
    const float* dloss;
    const float* lse;
    void* dx;                              // T x P1*P2, or (dx_parts) fp32, one after the other for each block of columns
    float* df1[2];                         // parts x P1 x ld1
    float* df2[2];                         // parts x P2 x Q2
    int64_t ldx, lddh, vocab;
    int tokens, P1, Q1, P2, Q2, ld1, n2;   // as in ForwardArgs
    int q1_step;                           // columns q1 of a block: a multiple of C1, at most R1
    int f_vec, dx_parts;                   // the factors can be read four elements at a time
};

// Sizes of a variant: P1 <= 32*KC1, P2 <= 32*KC2; W wavefronts of 16*N columns; R1 and C1 as above; DEEP buffers of a chunk's dZ (with two, a
// wavefront goes on to the next chunk while others still read this one); XLDS: X goes through LDS.
template <typename T_, int OP_, int KC1_, int KC2_, int W_, int N_, int R1_, bool XLDS_ = true>
struct GradShape {
    typedef T_ T;
    static constexpr int OP = OP_, KC1 = KC1_, KC2 = KC2_, W = W_, N = N_, R1 = R1_, C1 = 32;
    static constexpr bool XLDS = XLDS_;
    static constexpr int BR = OP == OP_LOSS ? 1 : 2, R2 = 16 * N * W, KCQ = R2 / 32, B1 = 2 * KC1, B2 = 2 * KC2, BC = C1 / 16;
    static_assert(R2 % 32 == 0 && R1 % C1 == 0 && C1 % 32 == 0, "whole fragments");
    // elements of LDS, the first four per branch: F1 [q1 block][p1 chunk]; F2 [q2 block][p2 chunk]; U, later dU, [q2 block][p1 chunk]; a chunk's
    // dZ [q1 block][q2 chunk]; X [p1 block][p2 chunk].  Contractions are mixed in F1 and U, chained in dU, straight in F2, dZ and X; rows are
    // mixed in F1 and X.
    static constexpr int F1 = R1 / 16 * KC1 * FRAG_LDS<T>, F2 = R2 / 16 * KC2 * FRAG_LDS<T>, UL = R2 / 16 * KC1 * FRAG_LDS<T>, DZ = BC * KCQ * FRAG, XA = XLDS ? B1 * KC2 * FRAG_LDS<T> : 0;
    static constexpr int lds(int deep) { return (BR * (F1 + F2 + UL + deep * DZ) + XA) * (int)sizeof(T); }
    static constexpr int DEEP = lds(2) <= 160 * 1024 ? 2 : 1, LDS_BYTES = lds(DEEP);
    // the blocks of a chunk of dF1 are dealt out to WP x WQ wavefronts, EP x EQ to each; those of dX to wavefronts by their p2, EX sets of
    // them where there are more than wavefronts, to PX wavefronts each where there are fewer
    static constexpr int WQ = 2, WP = W / WQ, EP = (B1 + WP - 1) / WP, EQ = BC / WQ;
    static constexpr int PX = W / B2 ? W / B2 : 1, EX = W / B2 ? 1 : (B2 + W - 1) / W, DX = (B1 + PX - 1) / PX;
    static constexpr int XPIECES = XLDS ? (32 * KC1 * 4 * KC2 + W * 64 - 1) / (W * 64) : 0;      // of 8 elements, in a thread
    // of these, loaded a token ahead: 32 registers at most (gated, 512 tokens 96x64,128x64 fp32: 313 us, 448 with all of them)
    static constexpr int XAHEAD = XPIECES < 4 ? XPIECES : 4;
    // registers that are taken over a whole token: dU, dF1, dF2, U; and the U that a wavefront needs for dF1, where that leaves enough for the rest (52x200,
    // 65x251, 999 tokens: 117 us read from LDS for each chunk, 146 in registers, because others then go to memory)
    static constexpr int WITHOUT_UREG = 4 * BR * (N * (B1 + B2) + R1 / C1 * EP * EQ) + 8 * BR * KC1 * N, UREGS = BR * EP * KCQ * (int)sizeof(T) * 2;
    static constexpr bool UREG = UREGS <= 32 && WITHOUT_UREG + UREGS <= (W == 8 ? 160 : 320);
    static constexpr int HELD = WITHOUT_UREG + (UREG ? UREGS : 0);
    // (the limits leave room for the rest; gated, 512 tokens 128x64,64x64 fp32: 237 us, 320 where 360 are allowed)
    static constexpr bool FITS = LDS_BYTES <= 160 * 1024 && HELD <= (W == 8 ? 180 : 260);
};

// The variant for a class of P1 and P2: the first of these that fits LDS and registers.  Most columns q2 first (each reads F1 for 16*N columns
// at once; sums over q2 stay inside a workgroup), then most columns q1.  Eight wavefronts for bf16: two on a SIMD hide some of each other's waits; gated,
// 8192 tokens 64x128,64x128: 308 us against 676 with four of 32 columns, whose registers do not suffice.
template <bool FITS, class S, class... More> struct FitOr { typedef S type; };
template <class S, class Next, class... More> struct FitOr<false, S, Next, More...> { typedef typename FitOr<Next::FITS, Next, More...>::type type; };
template <class S, class... More> using FirstFit = typename FitOr<S::FITS, S, More...>::type;

template <typename T, int OP, int K1, int K2> struct GradChoice;
template <int K1, int K2> struct GradChoice<bf16, OP_LOSS, K1, K2> {
    typedef FirstFit<GradShape<bf16, OP_LOSS, K1, K2, 8, 2, 256>, GradShape<bf16, OP_LOSS, K1, K2, 8, 1, 256>, GradShape<bf16, OP_LOSS, K1, K2, 8, 1, 128>,
                     GradShape<bf16, OP_LOSS, K1, K2, 8, 1, 64>> type;
};
template <int OP, int K1, int K2> struct GradChoice<bf16, OP, K1, K2> {
    typedef FirstFit<GradShape<bf16, OP, K1, K2, 8, 1, 128>, GradShape<bf16, OP, K1, K2, 8, 1, 64>, GradShape<bf16, OP, K1, K2, 4, 1, 64>, GradShape<bf16, OP, K1, K2, 4, 1, 32>> type;
};
template <int K1, int K2> struct GradChoice<float, OP_LOSS, K1, K2> {
    typedef FirstFit<GradShape<float, OP_LOSS, K1, K2, 4, 2, 128>, GradShape<float, OP_LOSS, K1, K2, 4, 1, 128>, GradShape<float, OP_LOSS, K1, K2, 4, 1, 64>,
                     GradShape<float, OP_LOSS, K1, K2, 4, 1, 32>> type;
};
template <int OP, int K1, int K2> struct GradChoice<float, OP, K1, K2> {
    typedef FirstFit<GradShape<float, OP, K1, K2, 4, 1, 64>, GradShape<float, OP, K1, K2, 4, 1, 32>, GradShape<float, OP, K1, K2, 2, 1, 64>, GradShape<float, OP, K1, K2, 2, 1, 32>,
                     GradShape<float, OP, K1, K2, 2, 1, 32, false>> type;
};

template <class Sh>
__global__ __launch_bounds__(Sh::W * 64) void factored_grad(GradArgs a)
{
    typedef typename Sh::T T;
    typedef typename Op<T>::Frag Frag;
    typedef T Piece __attribute__((ext_vector_type(Sh::N)));
    constexpr int OP = Sh::OP, BR = Sh::BR, KC1 = Sh::KC1, KC2 = Sh::KC2, N = Sh::N, W = Sh::W, KCQ = Sh::KCQ, B1 = Sh::B1, B2 = Sh::B2, BC = Sh::BC;
    constexpr int CHUNKS = Sh::R1 / Sh::C1, THREADS = W * 64;
    constexpr bool SPLIT = Op<T>::split;
    // Sums over q2 leave out what is past its end.  (Forward and backward, with and without: the gated block in fp32, 1000 tokens 52x50,65x20 111 and 127 us, 64x64,64x64
    // 120 and 118, 32x64,32x100 106 and 104.  bf16's products are short, and the branch keeps them apart: 2000 tokens 64x128,64x128 131 and 126 us, though 52x50,65x20
    // 115 and 142.  The loss's columns are many: 1000 tokens 64x256,64x256 bf16 101 and 96, 32x128,64x256 fp32 156 and 152, though 32x128,64x33 77 and 82.)
    constexpr bool FEW_COLUMNS = !SPLIT && OP != OP_LOSS;
    // (The gated kernels ask whether a row is short in classes without short ones too: 2000 tokens 52x50,65x20 bf16 143 us, 172 without the question,
    // 64x128,64x128 130 and 126; the loss, 8192 tokens 64x256,64x256: 574 us with it, 534 without.)
    constexpr bool WHOLE = OP == OP_LOSS && KC1 * KC2 > 1;
    extern __shared__ __align__(32) unsigned char smem[];
    T* const s1 = reinterpret_cast<T*>(smem);
    T* const sz = s1 + BR * Sh::F1;                        // (what chunks read is within the 64 KB that one address register reaches)
    T* const su = sz + BR * Sh::DEEP * Sh::DZ;
    T* const sx = su + BR * Sh::UL;
    T* const s2 = sx + Sh::XA;

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Lane<T> at(tid & 63);
    const int c = at.c, g = at.g;
    const int q1_first = blockIdx.y * a.q1_step, q2_first = blockIdx.z * Sh::R2;
    const int q1_count = min(a.q1_step, a.Q1 - q1_first), q2_count = min(Sh::R2, a.n2 - q2_first);
    const int nchunks = (q1_count + Sh::C1 - 1) / Sh::C1;
    const int col = wave * 16 * N + c * N;                 // this lane's first column of the block
    const int total = a.P1 * a.P2;                         // elements of a token's row

#pragma unroll
    for (int b = 0; b < BR; ++b) {
        lay_out<MIXED, false>(s1 + b * Sh::F1, (const T*)a.f1[b] + q1_first, q1_count, a.P1, a.ld1, nchunks * BC, KC1, a.f_vec, tid, THREADS, MixedRows());
        lay_out<STRAIGHT, false>(s2 + b * Sh::F2, (const T*)a.f2[b] + q2_first, q2_count, a.P2, a.Q2, N * W, KC2, a.f_vec, tid, THREADS, [](int col) {
            const int in = col % (16 * N);
            return col - in + (in % N) * 16 + in / N;
        });
    }
    // what of U, dU, dZ and X lies outside the columns and rows is multiplied by zeros, so it must not be NaN
    for (int i = tid; i < (BR * (Sh::UL + Sh::DEEP * Sh::DZ) + Sh::XA) / 4; i += THREADS) reinterpret_cast<typename Op<T>::Quad*>(sz)[i] = typename Op<T>::Quad{};

    f32x4 df1[CHUNKS][BR][Sh::EP][Sh::EQ], df2[BR][B2][N];
#pragma unroll
    for (int b = 0; b < BR; ++b) {
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
            for (int d = 0; d < Sh::EP; ++d)
#pragma unroll
                for (int e = 0; e < Sh::EQ; ++e) df1[i][b][d][e] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < B2; ++i)
#pragma unroll
            for (int n = 0; n < N; ++n) df2[b][i][n] = f32x4{0, 0, 0, 0};
    }
    const int wp = wave / Sh::WQ, wq = wave % Sh::WQ, px = wave % B2, ix = wave / B2;

    // A token's X on its way to LDS: pieces of 8 elements of a row, the next token's are loaded while one is worked on
    const int row_pieces = (a.P2 + 7) >> 3, pieces = a.P1 * row_pieces, magic = (65536 + row_pieces - 1) / row_pieces;      // (at most 2048 pieces: exact)
    Frag xp[Sh::XAHEAD ? Sh::XAHEAD : 1];
    auto load_x = [&](int t) __attribute__((always_inline)) {
        const T* const x = (const T*)a.x + t * a.ldx;
#pragma unroll
        for (int i = 0; i < Sh::XAHEAD; ++i) {
            const int piece = tid + i * THREADS, p1 = piece * magic >> 16, k = 8 * (piece - p1 * row_pieces);
            xp[i] = eight_of_row<WHOLE>(x, p1 * a.P2 + k, piece < pieces, total, a.P2 % 8 != 0, i == 0);
        }
    };
    auto store_x = [&](const T* x) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < Sh::XPIECES; ++i) {
            const int piece = tid + i * THREADS, p1 = piece * magic >> 16, k = 8 * (piece - p1 * row_pieces);
            if (piece < pieces) at.put_straight(sx, mixed_row(p1), k, KC2, i < Sh::XAHEAD ? xp[i] : eight_of_row<WHOLE>(x, p1 * a.P2 + k, true, total, a.P2 % 8 != 0, false));
        }
    };

    // dH of the next chunk, likewise
    Piece dhp[OP == OP_LOSS ? 1 : BC][4];
    auto load_dh = [&](int t, int ch) __attribute__((always_inline)) {
        const int rows = t < a.tokens ? q1_count - ch * Sh::C1 : 0;
        const Span<T> dh((const T*)a.dh + (rows > 0 ? t : 0) * a.lddh + (int64_t)(q1_first + ch * Sh::C1) * a.Q2 + q2_first, min(Sh::C1, max(0, rows)) * a.Q2 - q2_first);
#pragma unroll
        for (int h = 0; h < BC; ++h)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int n = 0; n < N; ++n) dhp[h][r][n] = dh.get(col + n < q2_count ? mixed_row(16 * h + 4 * g + r) * a.Q2 + col + n : NOWHERE);
    };
    // Logits that are no word's: in columns past n2, in rows past Q1, and in the last column q1 of a vocabulary in some columns q2.  Wavefronts and
    // chunks that hold some mask them, in the form that also takes the 1 off the target.  (F1's zeros there do not: Z is -lse, whose exponential may be infinite.)
    const bool edge = OP == OP_LOSS && (wave + 1) * 16 * N > q2_count, idle = OP == OP_LOSS && wave * 16 * N >= q2_count;
    int words[N];                          // columns q1 of the block, from the first, that are words in each of this lane's columns q2
#pragma unroll
    for (int n = 0; n < N; ++n) words[n] = col + n < q2_count ? a.Q1 - q1_first - (OP == OP_LOSS && (int64_t)(a.Q1 - 1) * a.Q2 + q2_first + col + n >= a.vocab) : 0;
    const int cut_chunk = OP == OP_LOSS && ((int64_t)a.Q1 * a.Q2 > a.vocab || a.Q1 % Sh::C1) && a.Q1 - q1_first <= q1_count ? nchunks - 1 : -1;

    int t = blockIdx.x;
    // A token's target, weight and logarithm of the sum; the next token's are loaded while one is worked on
    int64_t target = 0, target_ahead = 0;
    float dloss = 0, dloss_ahead = 0, lse = 0, lse_ahead = 0;
    auto load_facts = [&](int t) __attribute__((always_inline)) {
        if constexpr (OP == OP_LOSS) {
            t = min(t, a.tokens - 1);
            target_ahead = a.targets[t];
            dloss_ahead = a.dloss[t];
            lse_ahead = a.lse[t];
        }
    };
    // Goes on to a token with a target; those without one get no gradient, whatever X holds.
    auto settle = [&]() __attribute__((always_inline)) {
        if constexpr (OP == OP_LOSS) {
            target = target_ahead;
            dloss = dloss_ahead;
            lse = lse_ahead;
            if (t >= a.tokens || (target >= 0 && target < a.vocab)) return;
            do {
                if (a.dx_parts) {
                    float* const dx = (float*)a.dx + ((int64_t)(blockIdx.y * gridDim.z + blockIdx.z) * a.tokens + t) * (int64_t)total;
                    for (int i = tid; i < total; i += THREADS) dx[i] = 0.0f;
                } else {
                    T* const dx = (T*)a.dx + t * (int64_t)total;
                    for (int i = tid; i < total; i += THREADS) dx[i] = (T)0.0f;
                }
                t += gridDim.x;
                if (t >= a.tokens) return;
                target = a.targets[t];
            } while (target < 0 || target >= a.vocab);
            dloss = a.dloss[t];
            lse = a.lse[t];
            load_x(t);
        }
    };
    if (t < a.tokens) load_x(t);
    load_facts(t);
    if constexpr (OP != OP_LOSS) load_dh(t, 0);
    settle();
    __syncthreads();
    while (t < a.tokens) {
        const T* const x = (const T*)a.x + t * a.ldx;
        // The loss: logits are in units of log 2, and their products' sums start from -lse, so exponentials of Z are the probabilities.
        // The token's weight comes in with U for dF1 and with dU.  The target's dZ, p - 1, is taken before it is rounded, by the
        // wavefront that has its column, in its chunk.
        float weight = 1.0f, from = 0.0f;
        int target_q1 = -1, target_q2 = -1;                // its place in the block; -1: not this wavefront's
        if constexpr (OP == OP_LOSS) {
            const int q1 = (int)((unsigned)target / (unsigned)a.Q2), q2 = (int)target - q1 * a.Q2 - q2_first;
            const bool here = q1 >= q1_first && q1 < q1_first + q1_count && q2 >= 0 && q2 < q2_count && q2 / (16 * N) == wave;
            target_q1 = __builtin_amdgcn_readfirstlane(here ? q1 - q1_first : -1);
            target_q2 = __builtin_amdgcn_readfirstlane(here ? q2 : -1);
            weight = dloss;
            from = -lse * LOG2E;
        }
        const int target_chunk = target_q1 >> 5;
        static_assert(Sh::C1 == 32, "rows of a chunk");
        const f32x4 start = {from, from, from, from};
        store_x(x);
        __syncthreads();
        if (t + (int)gridDim.x < a.tokens) load_x(t + gridDim.x);
        load_facts(t + gridDim.x);

        // U of this wavefront's columns: in registers for Z, in LDS for dF1
        Frag u[BR][KC1][N], rest[BR][SPLIT ? KC1 : 1][SPLIT ? N : 1];
        f32x4 du[BR][B1][N];
#pragma unroll
        for (int b = 0; b < BR; ++b) {
#pragma unroll
            for (int i = 0; i < B1; ++i)
#pragma unroll
                for (int n = 0; n < N; ++n) du[b][i][n] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < KC2; ++k) {
                Frag f[N];
#pragma unroll
                for (int n = 0; n < N; ++n) f[n] = at.get(s2 + b * Sh::F2, (wave * N + n) * KC2 + k);
#pragma unroll
                for (int i = 0; i < B1; ++i) {
                    const Frag xf = Sh::XLDS ? at.get(sx, i * KC2 + k)
                                             : eight_of_row<WHOLE>(x, mixed_row(16 * i + c) * a.P2 + 32 * k + 8 * g, mixed_row(16 * i + c) < a.P1 && 32 * k + 8 * g < a.P2, total, a.P2 % 8 != 0, true);
#pragma unroll
                    for (int n = 0; n < N; ++n) Op<T>::mma(du[b][i][n], xf, f[n]);
                }
            }
#pragma unroll
            for (int k = 0; k < KC1; ++k)
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    f32x4 &lo = du[b][2 * k][n], &hi = du[b][2 * k + 1][n];
                    if constexpr (OP == OP_LOSS) {
                        at.put(su + b * Sh::UL, (wave * N + n) * KC1 + k, chain<T>(lo * weight, hi * weight));
                        lo *= LOG2E;
                        hi *= LOG2E;
                    }
                    u[b][k][n] = chain<T>(lo, hi);
                    if constexpr (SPLIT) rest[b][k][n] = chain_rest(lo, hi, u[b][k][n]);
                    if constexpr (OP != OP_LOSS) at.put(su + b * Sh::UL, (wave * N + n) * KC1 + k, u[b][k][n]);
                }
#pragma unroll
            for (int i = 0; i < B1; ++i)
#pragma unroll
                for (int n = 0; n < N; ++n) du[b][i][n] = f32x4{0, 0, 0, 0};
        }

        // A chunk's Z, dZ, what it adds to dU, and dZ into LDS.  No branches: what a wavefront has next to do beside it fills its waits.
        auto z_part = [&](int ch, auto marked) __attribute__((always_inline)) {
            T* const szb = sz + (ch % Sh::DEEP) * BR * Sh::DZ;
            Piece d[OP == OP_LOSS ? 1 : BC][4];
            if constexpr (OP != OP_LOSS) {
#pragma unroll
                for (int h = 0; h < BC; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) d[h][r] = dhp[h][r];
                const bool more = ch + 1 < nchunks;
                load_dh(more ? t : t + (int)gridDim.x, more ? ch + 1 : 0);
            }
#pragma unroll
            for (int pair = 0; pair < BC / 2; ++pair) {
                f32x4 dz[2][BR][N];
                // (both blocks' products in turn: four sums that do not wait for each other)
#pragma unroll
                for (int b = 0; b < BR; ++b)
#pragma unroll
                    for (int k = 0; k < KC1; ++k) {
                        Frag f[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h) f[h] = at.get(s1 + b * Sh::F1, (ch * BC + pair * 2 + h) * KC1 + k);
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int n = 0; n < N; ++n) dz[h][b][n] = Op<T>::product(f[h], u[b][k][n], k ? dz[h][b][n] : start);
                        if constexpr (SPLIT)
#pragma unroll
                            for (int h = 0; h < 2; ++h)
#pragma unroll
                                for (int n = 0; n < N; ++n) Op<T>::mma(dz[h][b][n], f[h], rest[b][k][n]);
                    }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    f32x4 (&z)[BR][N] = dz[h];
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int n = 0; n < N; ++n) {
                            if constexpr (OP == OP_LOSS) z[0][n][r] = __builtin_amdgcn_exp2f(z[0][n][r]);
                            else {
                                float slope;
                                const float act = activate<OP == OP_GELU>(z[0][n][r], slope), dv = to_f32<T>(d[pair * 2 + h][r][n]);
                                z[0][n][r] = slope * z[1][n][r] * dv;      // (a slope of 0 first: the others' product may be infinite)
                                z[1][n][r] = dv * act;
                            }
                        }
                    if constexpr (marked.value) {
                        const int row = (ch * BC + pair * 2) * 16 + mixed_row(16 * h + 4 * g);
#pragma unroll
                        for (int n = 0; n < N; ++n) {
                            int end = words[n], hit = target_q2 == col + n ? target_q1 : -1;
                            asm volatile("" : "+v"(end), "+v"(hit));      // (or comparisons for all chunks would be kept in registers)
#pragma unroll
                            for (int r = 0; r < 4; ++r) z[0][n][r] = row + r < end ? z[0][n][r] - (row + r == hit ? 1.0f : 0.0f) : 0.0f;
                        }
                    }
                }
#pragma unroll
                for (int b = 0; b < BR; ++b) {
                    Frag f[N];
#pragma unroll
                    for (int n = 0; n < N; ++n) f[n] = chain<T>(dz[0][b][n], dz[1][b][n]);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            Piece p;
#pragma unroll
                            for (int n = 0; n < N; ++n) p[n] = f[n][4 * h + r];
                            *reinterpret_cast<Piece*>(rows_slot_at(szb + b * Sh::DZ, (pair * 2 + (h ^ (g & 1))) * KCQ + (col >> 5), 4 * g + r, col & 31)) = p;
                        }
#pragma unroll
                    for (int i = 0; i < B1; ++i) {
                        const Frag p = at.template crossed<MIXED>(s1 + b * Sh::F1, ch * BC + pair * 2, KC1, i);
#pragma unroll
                        for (int n = 0; n < N; ++n) Op<T>::mma(du[b][i][n], p, f[n]);
                    }
                }
            }
        };
        Frag ur[Sh::UREG ? BR : 1][Sh::UREG ? Sh::EP : 1][Sh::UREG ? KCQ : 1];
        // What a chunk adds to dF1.
        auto f_part = [&](int ch) __attribute__((always_inline)) {
            const T* const szb = sz + (ch % Sh::DEEP) * BR * Sh::DZ;
#pragma unroll
            for (int b = 0; b < BR; ++b) {
                f32x4 odd[Sh::EP][Sh::EQ];  // odd steps add up apart from even ones, so that two sums are under way
#pragma unroll
                for (int d = 0; d < Sh::EP; ++d)
#pragma unroll
                    for (int e = 0; e < Sh::EQ; ++e) odd[d][e] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < KCQ; ++k) {
                    if (FEW_COLUMNS && k && 32 * k >= q2_count) continue;
                    Frag z[Sh::EQ];
#pragma unroll
                    for (int e = 0; e < Sh::EQ; ++e) z[e] = at.get_rows(szb + b * Sh::DZ, (wq + e * Sh::WQ) * KCQ + k);
#pragma unroll
                    for (int d = 0; d < Sh::EP; ++d) {
                        Frag f;
                        if constexpr (Sh::UREG) f = ur[b][d][k];
                        else f = at.template crossed_columns<N>(su + b * Sh::UL, 2 * k, KC1, min(wp + d * Sh::WP, B1 - 1));
#pragma unroll
                        for (int e = 0; e < Sh::EQ; ++e) {
                            if (k % 2) Op<T>::mma(odd[d][e], f, z[e]);
                            else Op<T>::mma(df1[ch][b][d][e], f, z[e]);
                        }
                    }
                }
                if constexpr (KCQ > 1)
#pragma unroll
                    for (int d = 0; d < Sh::EP; ++d)
#pragma unroll
                        for (int e = 0; e < Sh::EQ; ++e) df1[ch][b][d][e] += odd[d][e];
            }
        };
        auto z_of = [&](int ch) __attribute__((always_inline)) {
            if constexpr (OP == OP_LOSS) {
                if (idle) return;          // (its part of dZ stays zeros)
                if (edge || ch == cut_chunk || ch == target_chunk) z_part(ch, Yes());
                else z_part(ch, No());
            } else z_part(ch, No());
        };
        z_of(0);
#pragma unroll
        for (int ch = 0; ch < CHUNKS; ++ch) {
            if (ch >= nchunks) continue;
            __syncthreads();
            if (Sh::UREG && ch == 0)
#pragma unroll
                for (int b = 0; b < BR; ++b)
#pragma unroll
                    for (int d = 0; d < Sh::EP; ++d)
#pragma unroll
                        for (int k = 0; k < KCQ; ++k) ur[b][d][k] = at.template crossed_columns<N>(su + b * Sh::UL, 2 * k, KC1, min(wp + d * Sh::WP, B1 - 1));
            f_part(ch);
            if (ch + 1 < CHUNKS && ch + 1 < nchunks) {
                if constexpr (Sh::DEEP == 1) __syncthreads();             // dZ's buffer is free again
                z_of(ch + 1);
            }
        }
        __syncthreads();                   // so is U

        // dF2 from dU in registers; dU through LDS, in U's place, for dX
        Frag df[BR][KC1][N];
#pragma unroll
        for (int b = 0; b < BR; ++b)
#pragma unroll
            for (int k = 0; k < KC1; ++k)
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    df[b][k][n] = chain<T>(du[b][2 * k][n] * weight, du[b][2 * k + 1][n] * weight);
                    at.put(su + b * Sh::UL, (wave * N + n) * KC1 + k, df[b][k][n]);
                }
#pragma unroll
        for (int i = 0; i < B2; ++i)
#pragma unroll
            for (int k = 0; k < KC1; ++k) {
                Frag p;
                if constexpr (Sh::XLDS) p = at.template crossed<STRAIGHT, true>(sx, 2 * k, KC2, i);
                else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int p1 = 32 * k + 16 * (j / 4) + 4 * g + j % 4;
                        p[j] = x[p1 < a.P1 && 16 * i + c < a.P2 ? p1 * a.P2 + 16 * i + c : 0];      // (elsewhere dU is 0 or dF2 not written)
                    }
                }
#pragma unroll
                for (int b = 0; b < BR; ++b)
#pragma unroll
                    for (int n = 0; n < N; ++n) Op<T>::mma(df2[b][i][n], p, df[b][k][n]);
            }
        __syncthreads();
        const Span<T> dx((T*)a.dx + t * (int64_t)total, total);
        const Span<float> dx_part((float*)a.dx + ((int64_t)(blockIdx.y * gridDim.z + blockIdx.z) * a.tokens + t) * (int64_t)total, total);
        if (ix < Sh::PX)
#pragma unroll
            for (int e = 0; e < Sh::EX; ++e) {
                const int p = px + e * W;
                if (p >= B2) continue;
                f32x4 acc[Sh::DX];
#pragma unroll
                for (int d = 0; d < Sh::DX; ++d) acc[d] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int b = 0; b < BR; ++b)
#pragma unroll
                    for (int k = 0; k < KCQ; ++k) {
                        if (FEW_COLUMNS && k && 32 * k >= q2_count) continue;
                        const Frag f = at.template crossed<STRAIGHT>(s2 + b * Sh::F2, 2 * k, KC2, p);
#pragma unroll
                        for (int d = 0; d < Sh::DX; ++d) Op<T>::mma(acc[d], at.template crossed<CHAINED>(su + b * Sh::UL, 2 * k, KC1, min(ix + d * Sh::PX, B1 - 1)), f);
                    }
#pragma unroll
                for (int d = 0; d < Sh::DX; ++d)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int i = ix + d * Sh::PX, p1 = 16 * i + 4 * g + r, p2 = 16 * p + c;
                        const unsigned to = i < B1 && p1 < a.P1 && p2 < a.P2 ? p1 * a.P2 + p2 : NOWHERE;
                        if (a.dx_parts) dx_part.set(to, acc[d][r]);
                        else dx.set(to, from_f32<T>(acc[d][r]));
                    }
            }
        t += gridDim.x;
        settle();
    }

    // this workgroup's sums: dF1 is one of its columns q1 and a part for each (slice of tokens, block of q2); dF2 likewise
#pragma unroll
    for (int b = 0; b < BR; ++b) {
        float* const o1 = a.df1[b] + (int64_t)(blockIdx.x * gridDim.z + blockIdx.z) * a.P1 * a.ld1;
#pragma unroll
        for (int ch = 0; ch < CHUNKS; ++ch)
#pragma unroll
            for (int d = 0; d < Sh::EP; ++d)
#pragma unroll
                for (int e = 0; e < Sh::EQ; ++e) {
                    const int i = wp + d * Sh::WP, q1 = (ch * BC + wq + e * Sh::WQ) * 16 + c;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int p1 = 16 * i + 4 * g + r;
                        if (i < B1 && p1 < a.P1 && q1 < q1_count) o1[(int64_t)p1 * a.ld1 + q1_first + q1] = df1[ch][b][d][e][r];
                    }
                }
        float* const o2 = a.df2[b] + (int64_t)(blockIdx.x * gridDim.y + blockIdx.y) * a.P2 * a.Q2;
#pragma unroll
        for (int i = 0; i < B2; ++i)
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int p2 = 16 * i + 4 * g + r;
                    if (p2 < a.P2 && col + n < q2_count) o2[(int64_t)p2 * a.Q2 + q2_first + col + n] = df2[b][i][n][r];
                }
    }
}

}  // namespace km
