// The C-ABI of the operators around the Kron-Matmul: argument checks, the choice of kernels and their launches.
// Nothing here allocates or throws.
#include "../../include/kronmatmul.h"
#include "operators.hpp"
#include "join_kernels.hpp"
#include "layer_norm_kernel.hpp"

namespace km {

// (defined in the units that compile them)
#define KM_DECLARE(T, OP) template <> const ForwardVariant* forward_variants<T, OP>(); template <> const GradVariant* grad_variants<T, OP>();
KM_DECLARE(bf16, OP_SILU)
KM_DECLARE(bf16, OP_GELU)
KM_DECLARE(bf16, OP_LOSS)
KM_DECLARE(float, OP_SILU)
KM_DECLARE(float, OP_GELU)
KM_DECLARE(float, OP_LOSS)

namespace {

constexpr int MOST_ROWS = 1 << 30;         // kernels step past the last row in 32 bits
constexpr int MOST_COLUMNS = 1 << 22;      // and reach 64 rows of Q2 elements in 31 bits of bytes

// Blocks of columns are a launch's y and z.
bool launchable(dim3 grid) { return grid.y <= 65535 && grid.z <= 65535; }

// HIP takes fewer than 2^32 work-items along a launch (workgroups have up to 1024): what has more workgroups than these is several launches.
constexpr int MOST_GROUPS = 1 << 21;

// Workgroups that are worth having: one on each compute unit.
constexpr int UNITS = 256;

size_t element_size(km_dtype d) { return d == KM_F32 ? 4 : 2; }
bool known(km_dtype d) { return d == KM_F32 || d == KM_BF16; }
bool fits(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
int64_t up(int64_t n, int64_t unit) { return (n + unit - 1) / unit * unit; }
size_t piece(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
km_status done(hipError_t e)
{
    if (e == hipSuccess) return KM_OK;
    (void)hipGetLastError();
    return KM_ELAUNCH;
}

struct Region { const void* at; size_t bytes; };
// Do outputs overlap inputs or each other?
bool collide(const Region* out, int outs, const Region* in, int ins)
{
    auto meet = [](const Region& a, const Region& b) {
        const uintptr_t p = (uintptr_t)a.at, q = (uintptr_t)b.at;
        return a.at && b.at && a.bytes && b.bytes && p < q + b.bytes && q < p + a.bytes;
    };
    for (int i = 0; i < outs; ++i) {
        for (int j = 0; j < ins; ++j)
            if (meet(out[i], in[j])) return true;
        for (int j = 0; j < i; ++j)
            if (meet(out[i], out[j])) return true;
    }
    return false;
}
// Bytes from the first element of M rows `ld` apart to the last one.
size_t reach(int64_t m, int64_t ld, int64_t row, size_t size) { return m ? (size_t)((m - 1) * ld + row) * size : 0; }

km_status check_workspace(size_t need, const void* workspace, size_t bytes)
{
    if (need == 0) return KM_OK;
    if (!workspace || bytes < need) return KM_ENOMEM;
    return fits(workspace, 16) ? KM_OK : KM_EINVAL;
}

hipError_t sum_up(SumArgs& a, int jobs, km_dtype dtype, hipStream_t stream)
{
    int64_t blocks = 0;
    for (int i = 0; i < jobs; ++i) {
        a.job[i].blocks = (a.job[i].n + sum_span(a.job[i]) - 1) / sum_span(a.job[i]);
        blocks += a.job[i].blocks;
    }
    for (a.first = 0; a.first < blocks; a.first += MOST_GROUPS) {
        const unsigned groups = (unsigned)(blocks - a.first < MOST_GROUPS ? blocks - a.first : MOST_GROUPS);
        if (dtype == KM_F32) hipLaunchKernelGGL(sum_parts<float>, dim3(groups), dim3(256), 0, stream, a);
        else hipLaunchKernelGGL(sum_parts<bf16>, dim3(groups), dim3(256), 0, stream, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---- layer norm

// The team that holds a row in registers: by the row's pieces of `vec` elements.  Small teams leave more rows in flight (1000 x 3380 fp32 forward: 10.1 us
// with 1024 threads of 2 pieces, 7.9 with 256 of 4); the backward pass, whose workgroups have 1024 threads, has no registers for more than 2 pieces and
// their sums there (14.5 and 23.3).
struct Team { int threads, pieces; };
Team team_for(int H, int vec, bool backward)
{
    const int64_t n = ((int64_t)H + vec - 1) / vec;
    if (n <= 64 * 2) return {64, 2};
    if (n <= 256 * 2) return {256, 2};
    if (n <= 256 * 4 && !backward) return {256, 4};
    if (n <= 1024 * 2) return {1024, 2};
    if (n <= 1024 * 8) return {1024, 8};
    return {256, 0};
}

template <typename T, int VEC> hipError_t norm_forward_of(const NormArgs& a, Team team, hipStream_t stream)
{
    const int teams = team.threads < 256 ? 256 / team.threads : 1, most = teams * MOST_GROUPS, rows = a.rows;
    if (rows > most) {
        for (int first = 0; first < rows; first += most) {
            NormArgs some = a;
            some.x = (const T*)a.x + first * a.ldx;
            some.y = (T*)a.y + (int64_t)first * a.H;
            some.mean += first;
            some.rstd += first;
            some.rows = rows - first < most ? rows - first : most;
            const hipError_t e = norm_forward_of<T, VEC>(some, team, stream);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    const dim3 grid((a.rows + teams - 1) / teams);
    if (team.pieces == 0) hipLaunchKernelGGL((norm_forward<T, VEC, 256, 0>), grid, dim3(256), 0, stream, a);
    else if (team.threads == 64) hipLaunchKernelGGL((norm_forward<T, VEC, 64, 2>), grid, dim3(256), 0, stream, a);
    else if (team.threads == 256 && team.pieces == 4) hipLaunchKernelGGL((norm_forward<T, VEC, 256, 4>), grid, dim3(256), 0, stream, a);
    else if (team.threads == 256) hipLaunchKernelGGL((norm_forward<T, VEC, 256, 2>), grid, dim3(256), 0, stream, a);
    else if (team.pieces == 2) hipLaunchKernelGGL((norm_forward<T, VEC, 1024, 2>), grid, dim3(1024), 0, stream, a);
    else hipLaunchKernelGGL((norm_forward<T, VEC, 1024, 8>), grid, dim3(1024), 0, stream, a);
    return hipGetLastError();
}

// Workgroups of the backward pass, each with sums of its own.
int norm_parts(int M, Team team)
{
    const int teams = 1024 / team.threads, groups = (M + teams - 1) / teams;
    return groups < UNITS ? groups : UNITS;
}

template <typename T, int VEC> hipError_t norm_backward_of(const NormArgs& a, Team team, int parts, hipStream_t stream)
{
    const dim3 grid(parts), block(1024);
    const int lds = team.threads < 1024 && team.pieces ? 2 * a.H * 4 : 0;      // 32 KB at most
    if (team.pieces == 0) {
        hipLaunchKernelGGL((norm_backward<T, VEC, 256, 0>), grid, block, 0, stream, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(norm_columns<T>, dim3((a.H + 255) / 256, parts), dim3(256), 0, stream, a);
    }
    else if (team.threads == 64) hipLaunchKernelGGL((norm_backward<T, VEC, 64, 2>), grid, block, lds, stream, a);
    else if (team.threads == 256) hipLaunchKernelGGL((norm_backward<T, VEC, 256, 2>), grid, block, lds, stream, a);
    else if (team.pieces == 2) hipLaunchKernelGGL((norm_backward<T, VEC, 1024, 2>), grid, block, lds, stream, a);
    else hipLaunchKernelGGL((norm_backward<T, VEC, 1024, 8>), grid, block, lds, stream, a);
    return hipGetLastError();
}

// ---- products of two factors

struct Shape { int P1, Q1, P2, Q2; };

km_status check_shape(int M, const int* P, const int* Q, km_dtype dtype, Shape& s)
{
    if (M < 0 || M > MOST_ROWS || !P || !Q || !known(dtype)) return KM_EINVAL;
    if (P[0] < 1 || P[1] < 1 || Q[0] < 1 || Q[1] < 1) return KM_EINVAL;
    if (Q[1] > MOST_COLUMNS || (int64_t)Q[0] * Q[1] > INT32_MAX || (int64_t)P[0] * P[1] > INT32_MAX) return KM_EINVAL;
    if (P[0] > 128 || P[1] > 128) return KM_EUNSUPPORTED;
    s = {P[0], Q[0], P[1], Q[1]};
    return KM_OK;
}

// The part of the product that a vocabulary reaches into.
struct Columns { int q1, q2; };
// Columns q1 beyond these need more than a launch's 65535 blocks in every variant (the widest block is 160 KB of LDS, 64 bytes a column), and less than a
// block more of them is within 32 bits, so that plans can be made of any number up to here.
constexpr int MOST_Q1 = 1 << 28;
km_status check_columns(km_status shape, Columns cols) { return shape == KM_OK && cols.q1 > MOST_Q1 ? KM_EUNSUPPORTED : shape; }
Columns columns_of(const Shape& s, int64_t vocab)
{
    return {(int)((vocab + s.Q2 - 1) / s.Q2), (int)(vocab < s.Q2 ? vocab : s.Q2)};
}

// Can four neighbours of a factor's row be read at once?
bool factors_vec(const void* const* f1, const void* const* f2, const Shape& s, int branches, int size)
{
    bool ok = s.Q1 % 4 == 0 && s.Q2 % 4 == 0;
    for (int b = 0; b < branches; ++b) ok = ok && fits(f1[b], 4 * size) && fits(f2[b], 4 * size);
    return ok;
}

struct ForwardPlan {
    const ForwardVariant* v;
    int q1_step, q2_step, parts, threads, lds;
    dim3 grid;
};

const ForwardVariant* forward_table(int op, km_dtype dtype)
{
    if (dtype == KM_F32) return op == OP_LOSS ? forward_variants<float, OP_LOSS>() : op == OP_GELU ? forward_variants<float, OP_GELU>() : forward_variants<float, OP_SILU>();
    return op == OP_LOSS ? forward_variants<bf16, OP_LOSS>() : op == OP_GELU ? forward_variants<bf16, OP_GELU>() : forward_variants<bf16, OP_SILU>();
}
const GradVariant* grad_table(int op, km_dtype dtype)
{
    if (dtype == KM_F32) return op == OP_LOSS ? grad_variants<float, OP_LOSS>() : op == OP_GELU ? grad_variants<float, OP_GELU>() : grad_variants<float, OP_SILU>();
    return op == OP_LOSS ? grad_variants<bf16, OP_LOSS>() : op == OP_GELU ? grad_variants<bf16, OP_GELU>() : grad_variants<bf16, OP_SILU>();
}
int class_of(int p) { return (p + 31) / 32; }
int class_index(const Shape& s) { return (class_of(s.P1) - 1) * CLASSES + class_of(s.P2) - 1; }

ForwardPlan plan_forward(int op, km_dtype dtype, int M, const Shape& s, Columns cols)
{
    const ForwardVariant *const wide = forward_table(op, dtype) + class_index(s), *const narrow = wide + CLASSES * CLASSES;
    const int branches = op == OP_LOSS ? 1 : 2;
    ForwardPlan p;
    // Wide units read F1 from LDS less often and store longer pieces; they need enough units to fill the wavefronts (loss 64x256,64x256 bf16: 128 tokens
    // 13.6 us wide, 11.1 narrow; 512 tokens 17.6 wide, 22.8 narrow)
    p.v = (int64_t)M * ((cols.q2 + 16 * wide->n - 1) / (16 * wide->n)) >= 4 * UNITS ? wide : narrow;
    const int unit = 16 * p.v->n;
    const int64_t column = branches * (int)element_size(dtype) * FRAG / 16;    // bytes of a column in LDS, for 32 indices
    const int64_t column1 = column * class_of(s.P1), column2 = column * class_of(s.P2);
    p.q1_step = (int)up(cols.q1, 16);
    p.q2_step = (int)up(cols.q2, unit);
    auto halve = [](int n, int u) { return (int)up((n + 1) / 2, u); };
    while (column1 * p.q1_step + column2 * p.q2_step > LDS_MOST) {
        if ((column1 * p.q1_step > column2 * p.q2_step && p.q1_step > 16) || p.q2_step <= unit) p.q1_step = halve(p.q1_step, 16);
        else p.q2_step = halve(p.q2_step, unit);
    }
    // few tokens: the columns q1 over more workgroups, until there are four wavefronts with work on each compute unit, or eight if U, which each workgroup
    // computes again, is no more work than Z (512 tokens 64x128,64x128: fp32 51 us, 71 with four, bf16 15, 18 with four; 64 tokens of the loss 64x256,64x256 fp32
    // 16, 21 with four; but 200 tokens 128x128,128x256 fp32 81, 59 with four); four for the loss in bf16, which writes nothing (200 tokens 128x128,128x256 20 us, 26 with
    // eight; 1294 tokens 105x93,74x4 22 and 25, 32x512,32x64 17 and 19; but 512 tokens 128x512,32x32 18 and 13)
    const int64_t units = (int64_t)M * ((cols.q2 + unit - 1) / unit);
    auto wanted = [&] { return ((op != OP_LOSS || dtype == KM_F32) && 2 * class_of(s.P2) <= p.q1_step / 16 ? 8 : 4) * UNITS; };
    while (p.q1_step > 16 && units * ((cols.q1 + p.q1_step - 1) / p.q1_step) < wanted()) p.q1_step = halve(p.q1_step, 16);
    auto ny = [&] { return (cols.q1 + p.q1_step - 1) / p.q1_step; };
    auto nz = [&] { return (cols.q2 + p.q2_step - 1) / p.q2_step; };
    while ((int64_t)M * ny() * nz() < UNITS && p.q2_step > unit) p.q2_step = halve(p.q2_step, unit);
    const int64_t own = (int64_t)M * (p.q2_step / unit);                       // units of a block of columns
    p.threads = own * 64 >= p.v->threads ? p.v->threads : 256;
    const int64_t groups = (own + p.threads / 64 - 1) / (p.threads / 64), some = up(UNITS, (int64_t)ny() * nz()) / ((int64_t)ny() * nz());
    p.grid = dim3((unsigned)(groups < some ? groups : some), ny(), nz());
    p.lds = (int)(column1 * p.q1_step + column2 * p.q2_step);
    p.parts = ny() * ((cols.q2 + unit - 1) / unit);
    return p;
}

struct GradPlan {
    const GradVariant* v;
    int q1_step;
    dim3 grid;
    bool dx_parts;
    int tokens;                            // of a launch
    int parts1, parts2;                    // of dF1 and dF2
    size_t df1, df2, dx, bytes;            // bytes of a branch's parts, with several launches of their sum in front of them; of dX's; of everything
};

// Blocks of columns each leave a part of dX.  Tokens are taken some at a time, so that a launch's parts are no more bytes than these (or one token's for each
// workgroup): they are summed up right after it, and the next launch has the same place.  So are the factors' parts, together with the sums so far.
// Each launch brings the factors into LDS again and has workgroups that wait for the last one.  4096 tokens, bf16 gated 128x128,128x256: 2.1 GB in one launch
// 4.08 ms, in two 4.12, in nine of 256 MiB 4.33; fp32 loss 128x128,128x256: 4.3 GB in one 7.62, in five 7.82, in 17 7.90.
constexpr size_t DX_PARTS = (size_t)1 << 30;

GradPlan plan_grad(int op, km_dtype dtype, int M, const Shape& s, Columns cols)
{
    const GradVariant* const v = grad_table(op, dtype) + class_index(s);
    GradPlan p;
    p.v = v;
    const int nz = (cols.q2 + v->r2 - 1) / v->r2;
    int ny = (cols.q1 + v->r1 - 1) / v->r1;
    p.q1_step = (int)up((cols.q1 + ny - 1) / ny, v->c1);
    // few tokens: more, smaller blocks of columns until half of the compute units have one (loss and gated block of 64x256,64x256 and 64x128,64x128 bf16: one
    // token 20 and 16 us, 27 and 20 without; 64 tokens 30 and 24, with two for each unit 38 and 29)
    while ((int64_t)M * ny * nz < UNITS / 2 && p.q1_step > v->c1) {
        p.q1_step = (int)up(p.q1_step / 2, v->c1);
        ny = (cols.q1 + p.q1_step - 1) / p.q1_step;
    }
    ny = (cols.q1 + p.q1_step - 1) / p.q1_step;
    int slices = UNITS / (ny * nz);
    slices = slices < 1 ? 1 : slices > M ? M : slices;
    p.grid = dim3(slices, ny, nz);
    p.dx_parts = ny * nz > 1;
    p.parts1 = slices * nz;
    p.parts2 = slices * ny;
    const int branches = op == OP_LOSS ? 1 : 2;
    p.tokens = M;
    p.dx = 0;
    if (p.dx_parts && M) {
        const size_t token = (size_t)ny * nz * s.P1 * s.P2 * 4, most = DX_PARTS / token / slices;
        const int64_t launch = (most ? most : 1) * slices, launches = (M + launch - 1) / launch, even = up((M + launches - 1) / launches, slices);
        p.tokens = (int)(even < M ? even : M);
        p.dx = piece(token * p.tokens);
    }
    const int sums = p.tokens < M;
    p.df1 = piece((size_t)(p.parts1 + sums) * s.P1 * s.Q1 * 4);
    p.df2 = piece((size_t)(p.parts2 + sums) * s.P2 * s.Q2 * 4);
    p.bytes = M ? branches * (p.df1 + p.df2) + p.dx : 0;
    return p;
}

// The backward pass of either operation; `a` comes with the inputs and the sizes.
km_status run_grad(int op, km_dtype dtype, int M, const Shape& s, Columns cols, GradArgs& a, void* dX, void* const* d1, void* const* d2,
                   void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    const GradPlan p = plan_grad(op, dtype, M, s, cols);
    if (M && !launchable(p.grid)) return KM_EUNSUPPORTED;
    const km_status ws = check_workspace(p.bytes, workspace, workspace_bytes);
    if (ws != KM_OK) return ws;
    const int branches = op == OP_LOSS ? 1 : 2;
    const int64_t n1 = (int64_t)s.P1 * s.Q1, n2 = (int64_t)s.P2 * s.Q2, row = (int64_t)s.P1 * s.P2, size = (int64_t)element_size(dtype);
    const bool several = p.tokens < M;     // launches: sums of those before are one part more, in front of the others
    SumArgs sum = {}, far = {};            // the last launch's sums; those before
    int jobs = 0;
    char* at = (char*)workspace;
    for (int b = 0; b < branches; ++b) {
        void* const* out = b ? d2 : d1;
        float *const s1 = (float*)at, *const s2 = (float*)(at + p.df1);
        a.df1[b] = several ? s1 + n1 : s1;
        a.df2[b] = several ? s2 + n2 : s2;
        at += p.df1 + p.df2;
        far.job[jobs] = {a.df1[b], s1, n1, n1, p.parts1, s.Q1, cols.q1};
        far.job[jobs + 1] = {a.df2[b], s2, n2, n2, p.parts2, s.Q2, cols.q2};
        sum.job[jobs++] = {s1, out[0], n1, n1, M ? p.parts1 + several : 0, s.Q1, cols.q1};
        sum.job[jobs++] = {s2, out[1], n2, n2, M ? p.parts2 + several : 0, s.Q2, cols.q2};
    }
    a.P1 = s.P1; a.P2 = s.P2; a.Q2 = s.Q2; a.ld1 = s.Q1;
    a.Q1 = cols.q1; a.n2 = cols.q2;
    a.q1_step = p.q1_step;
    a.f_vec = factors_vec(a.f1, a.f2, s, branches, (int)size);
    a.dx_parts = p.dx_parts;
    for (int64_t first = 0; first < M; first += p.tokens) {
        GradArgs some = a;
        some.tokens = (int)(M - first < p.tokens ? M - first : p.tokens);
        some.x = (const char*)a.x + first * a.ldx * size;
        if (a.dh) some.dh = (const char*)a.dh + first * a.lddh * size;
        if (op == OP_LOSS) {
            some.targets += first;
            some.dloss += first;
            some.lse += first;
        }
        void* const dx = (char*)dX + first * row * size;
        some.dx = p.dx_parts ? at : dx;
        hipError_t e = p.v->launch(some, p.grid, stream);
        if (e != hipSuccess) return done(e);
        if (!p.dx_parts) continue;
        const int64_t n = some.tokens * row;
        const SumJob job = {(const float*)at, dx, n, n, (int)(p.grid.y * p.grid.z), n, n};
        if (first + p.tokens >= M) {
            sum.job[jobs++] = job;
            break;
        }
        SumArgs parts = {};
        parts.job[0] = job;
        e = sum_up(parts, 1, dtype, stream);
        if (e == hipSuccess) e = sum_up(far, jobs, KM_F32, stream);
        if (e != hipSuccess) return done(e);
        for (int i = 0; first == 0 && i < jobs; ++i) {
            far.job[i].in = sum.job[i].in;
            far.job[i].parts = sum.job[i].parts;
        }
    }
    return done(sum_up(sum, jobs, dtype, stream));
}

km_status run_forward(int op, km_dtype dtype, const ForwardPlan& p, ForwardArgs& a, int M, const Shape& s, Columns cols, hipStream_t stream)
{
    if (!launchable(p.grid)) return KM_EUNSUPPORTED;
    a.tokens = M;
    a.P1 = s.P1; a.P2 = s.P2; a.Q2 = s.Q2; a.ld1 = s.Q1;
    a.Q1 = cols.q1; a.n2 = cols.q2;
    a.q1_step = p.q1_step; a.q2_step = p.q2_step;
    a.parts = p.parts;
    const int size = (int)element_size(dtype);
    a.f_vec = factors_vec(a.f1, a.f2, s, op == OP_LOSS ? 1 : 2, size);
    // (8192 x 16384 bf16 133 -> 119 us; what fits the 256 MB cache is left there for its reader)
    a.y_stream = (int64_t)M * s.Q1 * s.Q2 * size > ((int64_t)192 << 20);
    a.y_vec = op != OP_LOSS && s.Q2 % p.v->n == 0 && fits(a.y, p.v->n * size);
    return done(p.v->launch(a, p.grid, p.threads, p.lds, stream));
}

}  // namespace
}  // namespace km

using namespace km;

extern "C" {

km_status kronmatmul_layer_norm(int M, int H, const void* X, long long ldx, const void* weight, const void* bias, float eps, void* Y, float* mean,
                                float* rstd, km_dtype dtype, void* stream)
{
    if (M < 0 || M > MOST_ROWS || H < 1 || H > MOST_ROWS || ldx < H || !known(dtype) || !(eps >= 0)) return KM_EINVAL;
    if (!X || !weight || !Y || !mean || !rstd) return KM_EINVAL;
    const size_t size = element_size(dtype);
    if (!fits(X, size) || !fits(weight, size) || !fits(bias, size) || !fits(Y, size) || !fits(mean, 4) || !fits(rstd, 4)) return KM_EINVAL;
    const Region out[] = {{Y, reach(M, H, H, size)}, {mean, (size_t)M * 4}, {rstd, (size_t)M * 4}};
    const Region in[] = {{X, reach(M, ldx, H, size)}, {weight, H * size}, {bias, H * size}};
    if (collide(out, 3, in, 3)) return KM_EINVAL;
    if (M == 0) return KM_OK;
    NormArgs a = {};
    a.x = X; a.w = weight; a.b = bias; a.y = Y; a.mean = mean; a.rstd = rstd;
    a.ldx = ldx; a.eps = eps; a.rows = M; a.H = H;
    const int whole = 16 / (int)size;
    const bool vec = H % whole == 0 && ldx % whole == 0 && fits(X, 16) && fits(Y, 16) && fits(weight, 16) && fits(bias, 16);
    const Team team = team_for(H, vec ? whole : 1, false);
    if (dtype == KM_F32) return done(vec ? norm_forward_of<float, 4>(a, team, (hipStream_t)stream) : norm_forward_of<float, 1>(a, team, (hipStream_t)stream));
    return done(vec ? norm_forward_of<bf16, 8>(a, team, (hipStream_t)stream) : norm_forward_of<bf16, 1>(a, team, (hipStream_t)stream));
}

km_status kronmatmul_layer_norm_grad_workspace_size(int M, int H, km_dtype dtype, size_t* bytes)
{
    if (!bytes || M < 0 || M > MOST_ROWS || H < 1 || H > MOST_ROWS || !known(dtype)) return KM_EINVAL;
    // (whichever team it will be: unaligned rows have larger ones, and so fewer parts)
    *bytes = M ? (size_t)norm_parts(M, {1024, 2}) * 2 * H * 4 : 0;
    return KM_OK;
}

km_status kronmatmul_layer_norm_grad(int M, int H, const void* dY, long long lddy, const void* X, long long ldx, const void* weight, const float* mean,
                                     const float* rstd, void* dX, void* dweight, void* dbias, km_dtype dtype, void* workspace, size_t workspace_bytes,
                                     void* stream)
{
    size_t need = 0;
    const km_status s = kronmatmul_layer_norm_grad_workspace_size(M, H, dtype, &need);
    if (s != KM_OK) return s;
    if (lddy < H || ldx < H || !dY || !X || !weight || !mean || !rstd || !dX || !dweight) return KM_EINVAL;
    const size_t size = element_size(dtype);
    if (!fits(X, size) || !fits(dY, size) || !fits(weight, size) || !fits(dX, size) || !fits(dweight, size) || !fits(dbias, size) || !fits(mean, 4) ||
        !fits(rstd, 4))
        return KM_EINVAL;
    const Region out[] = {{dX, reach(M, H, H, size)}, {dweight, H * size}, {dbias, H * size}, {workspace, need}};
    const Region in[] = {{X, reach(M, ldx, H, size)}, {dY, reach(M, lddy, H, size)}, {weight, H * size}, {mean, (size_t)M * 4}, {rstd, (size_t)M * 4}};
    if (collide(out, 4, in, 5)) return KM_EINVAL;
    const km_status ws = check_workspace(need, workspace, workspace_bytes);
    if (ws != KM_OK) return ws;
    int parts = 0;
    if (M) {
        NormArgs a = {};
        a.x = X; a.dy = dY; a.w = weight; a.y = dX; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
        a.dw = (float*)workspace;
        a.ldx = ldx; a.lddy = lddy; a.rows = M; a.H = H;
        const int whole = 16 / (int)size;
        const bool vec = H % whole == 0 && ldx % whole == 0 && lddy % whole == 0 && fits(X, 16) && fits(dY, 16) && fits(dX, 16) && fits(weight, 16);
        const Team team = team_for(H, vec ? whole : 1, true);
        parts = norm_parts(M, team);
        const hipStream_t st = (hipStream_t)stream;
        const hipError_t e = dtype == KM_F32 ? (vec ? norm_backward_of<float, 4>(a, team, parts, st) : norm_backward_of<float, 1>(a, team, parts, st))
                                             : (vec ? norm_backward_of<bf16, 8>(a, team, parts, st) : norm_backward_of<bf16, 1>(a, team, parts, st));
        if (e != hipSuccess) return done(e);
    }
    SumArgs sum = {};
    const int64_t apart = 2 * (int64_t)H;
    sum.job[0] = {(const float*)workspace, dweight, H, apart, parts, H, H};
    sum.job[1] = {(const float*)workspace + H, dbias, H, apart, parts, H, H};
    return done(sum_up(sum, dbias ? 2 : 1, dtype, (hipStream_t)stream));
}

km_status kronmatmul_gated(int M, const int* P, const int* Q, const void* X, long long ldx, const void* const* gate, const void* const* up_, km_activation act,
                           void* H, km_dtype dtype, void* stream)
{
    Shape s;
    km_status ok = check_shape(M, P, Q, dtype, s);
    if (ok != KM_OK && ok != KM_EUNSUPPORTED) return ok;
    if (act != KM_ACT_SILU && act != KM_ACT_GELU_TANH) return KM_EINVAL;
    const Columns cols = {Q[0], Q[1]};
    ok = check_columns(ok, cols);
    if (!X || !H || !gate || !up_ || ldx < (int64_t)P[0] * P[1]) return KM_EINVAL;
    const size_t size = element_size(dtype);
    Region in[5] = {{X, reach(M, ldx, (int64_t)P[0] * P[1], size)}};
    for (int i = 0; i < 2; ++i) {
        if (!gate[i] || !up_[i] || !fits(gate[i], size) || !fits(up_[i], size)) return KM_EINVAL;
        in[1 + 2 * i] = {gate[i], (size_t)P[i] * Q[i] * size};
        in[2 + 2 * i] = {up_[i], (size_t)P[i] * Q[i] * size};
    }
    const Region out[] = {{H, (size_t)M * Q[0] * Q[1] * size}};
    if (!fits(X, size) || !fits(H, size) || collide(out, 1, in, 5)) return KM_EINVAL;
    if (ok != KM_OK || M == 0) return ok;
    const int op = act == KM_ACT_SILU ? OP_SILU : OP_GELU;
    ForwardArgs a = {};
    a.x = X; a.y = H; a.ldx = ldx;
    a.f1[0] = gate[0]; a.f2[0] = gate[1]; a.f1[1] = up_[0]; a.f2[1] = up_[1];
    return run_forward(op, dtype, plan_forward(op, dtype, M, s, cols), a, M, s, cols, (hipStream_t)stream);
}

km_status kronmatmul_gated_grad_workspace_size(int M, const int* P, const int* Q, km_dtype dtype, size_t* bytes)
{
    Shape s;
    if (!bytes) return KM_EINVAL;
    km_status ok = check_shape(M, P, Q, dtype, s);
    if (ok != KM_OK) return ok;
    const Columns cols = {s.Q1, s.Q2};
    ok = check_columns(ok, cols);
    if (ok != KM_OK) return ok;
    *bytes = plan_grad(OP_SILU, dtype, M, s, cols).bytes;      // (both activations have the same variants)
    return KM_OK;
}

km_status kronmatmul_gated_grad(int M, const int* P, const int* Q, const void* dH, long long lddh, const void* X, long long ldx, const void* const* gate,
                                const void* const* up_, km_activation act, void* dX, void* const* dgate, void* const* dup, km_dtype dtype, void* workspace,
                                size_t workspace_bytes, void* stream)
{
    Shape s;
    km_status ok = check_shape(M, P, Q, dtype, s);
    if (ok != KM_OK && ok != KM_EUNSUPPORTED) return ok;
    if (act != KM_ACT_SILU && act != KM_ACT_GELU_TANH) return KM_EINVAL;
    const Columns cols = {Q[0], Q[1]};
    ok = check_columns(ok, cols);
    if (!X || !dH || !dX || !gate || !up_ || !dgate || !dup || ldx < (int64_t)P[0] * P[1] || lddh < (int64_t)Q[0] * Q[1]) return KM_EINVAL;
    const size_t size = element_size(dtype);
    Region in[6] = {{X, reach(M, ldx, (int64_t)P[0] * P[1], size)}, {dH, reach(M, lddh, (int64_t)Q[0] * Q[1], size)}};
    Region out[6] = {{dX, (size_t)M * P[0] * P[1] * size}};
    for (int i = 0; i < 2; ++i) {
        const size_t bytes = (size_t)P[i] * Q[i] * size;
        const void* all[] = {gate[i], up_[i], dgate[i], dup[i]};
        for (const void* p : all)
            if (!p || !fits(p, size)) return KM_EINVAL;
        in[2 + 2 * i] = {gate[i], bytes};
        in[3 + 2 * i] = {up_[i], bytes};
        out[1 + 2 * i] = {dgate[i], bytes};
        out[2 + 2 * i] = {dup[i], bytes};
    }
    if (!fits(X, size) || !fits(dH, size) || !fits(dX, size)) return KM_EINVAL;
    const int op = act == KM_ACT_SILU ? OP_SILU : OP_GELU;
    out[5] = {workspace, ok == KM_OK ? plan_grad(op, dtype, M, s, cols).bytes : 0};
    if (collide(out, 6, in, 6)) return KM_EINVAL;
    if (ok != KM_OK) return ok;
    GradArgs a = {};
    a.x = X; a.dh = dH; a.ldx = ldx; a.lddh = lddh;
    a.f1[0] = gate[0]; a.f2[0] = gate[1]; a.f1[1] = up_[0]; a.f2[1] = up_[1];
    return run_grad(op, dtype, M, s, cols, a, dX, dgate, dup, workspace, workspace_bytes, (hipStream_t)stream);
}

km_status kronmatmul_cross_entropy_workspace_size(int M, const int* P, const int* Q, long long vocab, km_dtype dtype, size_t* bytes)
{
    Shape s;
    if (!bytes) return KM_EINVAL;
    km_status ok = check_shape(M, P, Q, dtype, s);
    if (ok != KM_OK) return ok;
    if (vocab < 1 || vocab > (int64_t)s.Q1 * s.Q2) return KM_EINVAL;
    const Columns cols = columns_of(s, vocab);
    ok = check_columns(ok, cols);
    if (ok != KM_OK) return ok;
    *bytes = M ? piece((size_t)M * plan_forward(OP_LOSS, dtype, M, s, cols).parts * 8) + (size_t)M * 4 : 0;
    return KM_OK;
}

km_status kronmatmul_cross_entropy(int M, const int* P, const int* Q, long long vocab, const void* X, long long ldx, const void* const* F,
                                   const long long* targets, float* loss, float* lse, km_dtype dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    Shape s;
    km_status ok = check_shape(M, P, Q, dtype, s);
    if (ok != KM_OK && ok != KM_EUNSUPPORTED) return ok;
    if (!X || !F || !F[0] || !F[1] || !targets || !loss || !lse || ldx < (int64_t)P[0] * P[1]) return KM_EINVAL;
    if (vocab < 1 || vocab > (int64_t)Q[0] * Q[1]) return KM_EINVAL;
    const size_t size = element_size(dtype);
    if (!fits(X, size) || !fits(F[0], size) || !fits(F[1], size) || !fits(targets, 8) || !fits(loss, 4) || !fits(lse, 4)) return KM_EINVAL;
    const Columns cols = columns_of({P[0], Q[0], P[1], Q[1]}, vocab);
    ok = check_columns(ok, cols);
    ForwardPlan p = {};
    size_t first = 0, need = 0;
    if (ok == KM_OK && M) {
        p = plan_forward(OP_LOSS, dtype, M, s, cols);
        first = piece((size_t)M * p.parts * 8);
        need = first + (size_t)M * 4;
    }
    const Region in[] = {{X, reach(M, ldx, (int64_t)P[0] * P[1], size)}, {F[0], (size_t)P[0] * Q[0] * size}, {F[1], (size_t)P[1] * Q[1] * size}, {targets, (size_t)M * 8}};
    const Region out[] = {{loss, (size_t)M * 4}, {lse, (size_t)M * 4}, {workspace, need}};
    if (collide(out, 3, in, 4)) return KM_EINVAL;
    if (ok != KM_OK || M == 0) return ok;
    const km_status ws = check_workspace(need, workspace, workspace_bytes);
    if (ws != KM_OK) return ws;
    ForwardArgs a = {};
    a.x = X; a.ldx = ldx; a.vocab = vocab;
    a.f1[0] = F[0]; a.f2[0] = F[1];
    a.targets = (const int64_t*)targets;
    a.partial = (float2*)workspace;
    a.picked = (float*)((char*)workspace + first);
    const km_status ran = run_forward(OP_LOSS, dtype, p, a, M, s, cols, (hipStream_t)stream);
    if (ran != KM_OK) return ran;
    for (int first = 0; first < M; first += 16 * MOST_GROUPS) {
        const int tokens = M - first < 16 * MOST_GROUPS ? M - first : 16 * MOST_GROUPS;
        hipLaunchKernelGGL(loss_join, dim3((tokens + 15) / 16), dim3(256), 0, (hipStream_t)stream, a.partial + (int64_t)first * p.parts, a.picked + first, a.targets + first,
                           (int64_t)vocab, tokens, p.parts, loss + first, lse + first);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return done(e);
    }
    return KM_OK;
}

km_status kronmatmul_cross_entropy_grad_workspace_size(int M, const int* P, const int* Q, long long vocab, km_dtype dtype, size_t* bytes)
{
    Shape s;
    if (!bytes) return KM_EINVAL;
    km_status ok = check_shape(M, P, Q, dtype, s);
    if (ok != KM_OK) return ok;
    if (vocab < 1 || vocab > (int64_t)s.Q1 * s.Q2) return KM_EINVAL;
    const Columns cols = columns_of(s, vocab);
    ok = check_columns(ok, cols);
    if (ok != KM_OK) return ok;
    *bytes = plan_grad(OP_LOSS, dtype, M, s, cols).bytes;
    return KM_OK;
}

km_status kronmatmul_cross_entropy_grad(int M, const int* P, const int* Q, long long vocab, const float* dloss, const void* X, long long ldx,
                                        const void* const* F, const long long* targets, const float* lse, void* dX, void* const* dF, km_dtype dtype,
                                        void* workspace, size_t workspace_bytes, void* stream)
{
    Shape s;
    km_status ok = check_shape(M, P, Q, dtype, s);
    if (ok != KM_OK && ok != KM_EUNSUPPORTED) return ok;
    if (!X || !F || !F[0] || !F[1] || !targets || !dloss || !lse || !dX || !dF || !dF[0] || !dF[1] || ldx < (int64_t)P[0] * P[1]) return KM_EINVAL;
    if (vocab < 1 || vocab > (int64_t)Q[0] * Q[1]) return KM_EINVAL;
    const size_t size = element_size(dtype);
    if (!fits(X, size) || !fits(F[0], size) || !fits(F[1], size) || !fits(dX, size) || !fits(dF[0], size) || !fits(dF[1], size) || !fits(targets, 8) ||
        !fits(dloss, 4) || !fits(lse, 4))
        return KM_EINVAL;
    const Columns cols = columns_of({P[0], Q[0], P[1], Q[1]}, vocab);
    ok = check_columns(ok, cols);
    const size_t b1 = (size_t)P[0] * Q[0] * size, b2 = (size_t)P[1] * Q[1] * size;
    const Region in[] = {{X, reach(M, ldx, (int64_t)P[0] * P[1], size)}, {F[0], b1}, {F[1], b2}, {targets, (size_t)M * 8}, {dloss, (size_t)M * 4}, {lse, (size_t)M * 4}};
    const Region out[] = {{dX, (size_t)M * P[0] * P[1] * size}, {dF[0], b1}, {dF[1], b2}, {workspace, ok == KM_OK ? plan_grad(OP_LOSS, dtype, M, s, cols).bytes : 0}};
    if (collide(out, 4, in, 6)) return KM_EINVAL;
    if (ok != KM_OK) return ok;
    GradArgs a = {};
    a.x = X; a.ldx = ldx; a.vocab = vocab;
    a.f1[0] = F[0]; a.f2[0] = F[1];
    a.targets = (const int64_t*)targets;
    a.dloss = dloss;
    a.lse = lse;
    return run_grad(OP_LOSS, dtype, M, s, cols, a, dX, dF, nullptr, workspace, workspace_bytes, (hipStream_t)stream);
}

}  // extern "C"
