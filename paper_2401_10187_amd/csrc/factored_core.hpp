// What the kernels of Kronecker-factored layers share: tokens whose row of P1*P2 elements is a matrix X_t (P1 x P2), multiplied by
// F1 (x) F2 on the matrix cores, F1 being P1 x Q1 and F2 P2 x Q2:
//     U_t = X_t F2   (P1 x Q2),      Z_t = F1^T U_t   (Q1 x Q2, element q1*Q2+q2 of the token's row of the product).
//
// The products run on 16x16 blocks.  A fragment is what one such product reads of an operand: 16 rows times 32 contraction
// indices, eight of them in each lane (row = lane % 16; which eight depends on lane / 16 = g).  The order of the
// contraction indices is free as long as both operands have the same one, and two orders are used:
//     straight  g, j -> 8g + j                      a row's eight elements follow each other in memory
//     chained   g, j -> 16(j/4) + 4g + j%4          the eight elements are those that lane holds of two result blocks, one above the other
// A block of results has its rows 4g..4g+3 and column lane % 16 in a lane.  With the chained order, results (U, dZ, dU) become the
// right operand of the next product in the registers in which they are, without a pass through LDS.
// MIXED, a third order, is the chained one with j/4 turned over for g = 1, 3.  It is what results chain to whose left operand's rows were mixed:
// rows 4 to 7 and 12 to 15 of two row blocks exchanged (mixed_row).  Crossed reads (below) of fragments in this order meet all banks of LDS.
//
// bf16: one product of 16x16x32, sums in fp32.  U is rounded once more before Z is computed from it: to the sum of two
// bf16 (16 bits of mantissa), at the price of a second product, because logits reach 20 and more, where one bf16 would be wrong in the
// second decimal place and a loss or probability with it.  fp32: eight products of 16x16x4.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace km {

typedef __bf16 bf16;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int FRAG = 512;                  // elements of a fragment: 64 lanes x 8
template <typename T> constexpr int FRAG_LDS = sizeof(T) == 2 ? FRAG : 67 * 8;      // and what it takes of LDS (see piece_of)

template <typename T> struct Op;
template <> struct Op<bf16> {
    typedef bf16x8 Frag;
    typedef bf16x4 Quad;
    static constexpr bool split = true;    // U as a sum of two fragments
    static __device__ __forceinline__ f32x4 product(const Frag& a, const Frag& b, const f32x4& plus) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, plus, 0, 0, 0); }
    static __device__ __forceinline__ void mma(f32x4& d, const Frag& a, const Frag& b) { d = product(a, b, d); }
};
template <> struct Op<float> {
    typedef f32x8 Frag;
    typedef f32x4 Quad;
    static constexpr bool split = false;
    static __device__ __forceinline__ f32x4 product(const Frag& a, const Frag& b, f32x4 plus)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) plus = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], plus, 0, 0, 0);
        return plus;
    }
    static __device__ __forceinline__ void mma(f32x4& d, const Frag& a, const Frag& b) { d = product(a, b, d); }
};

template <typename T> __device__ __forceinline__ float to_f32(T v) { return (float)v; }
template <typename T> __device__ __forceinline__ T from_f32(float v) { return (T)v; }     // bf16: to the nearest, ties to even

// Two result blocks, rows 0-15 and 16-31 of a contraction, as the fragment of their chained order.
template <typename T> __device__ __forceinline__ typename Op<T>::Frag chain(const f32x4& lo, const f32x4& hi)
{
    f32x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    if constexpr (sizeof(T) == 4) return v;
    else return __builtin_convertvector(v, bf16x8);
}
// What rounding to `hi` left over.
__device__ __forceinline__ bf16x8 chain_rest(const f32x4& lo, const f32x4& hi, const bf16x8& rounded)
{
    f32x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_convertvector(v - __builtin_convertvector(rounded, f32x8), bf16x8);
}

enum Order { STRAIGHT, CHAINED, MIXED };
// Position of contraction index k (of one chunk of 32) in a fragment's row: the row's lane is row%16 + 16*group.
template <Order O> __device__ __forceinline__ int frag_group(int k) { return O == STRAIGHT ? k >> 3 : (k & 15) >> 2; }
template <Order O> __device__ __forceinline__ int frag_slot(int k) { return O == STRAIGHT ? k & 7 : (((k >> 4) ^ (O == MIXED ? (k >> 2) & 1 : 0)) << 2) | (k & 3); }
__device__ __forceinline__ int mixed_row(int row) { return row ^ ((row & 4) << 2); }

// Fragments lie one after the other in LDS, [row block][chunk], 64 pieces of eight elements each.  Where a piece lies, and which half of it comes
// first, is chosen for the 64 banks.  A wavefront reads a fragment by 16 lanes at a time, of which rows 0-3 and 12-15 are those of one group and rows 4-11
// of the next; and crossed (below).
//   bf16  A piece is 4 banks.  Row r of group g is piece 16 g + (r + 8 (g/2)) % 16.  A crossed read takes a half of each piece of 8 rows by 4
//         groups; in the mixed order these are different halves in neighbouring groups.
//   fp32  A piece is 8 banks and is read by halves.  A crossed read takes one element of each lane's own: 4 of a piece, of 4 rows 4 apart by 4 groups, or
//         all 8, of 4 such rows by 2 groups.  Row 4h+j of group g is piece place + 17 j, the place 0 to 15 by the bits of h and g as below, and its
//         halves are exchanged where g is 1 or 2: all of these reads meet 64 different banks, and the rows of one h are a constant apart, so that
//         addresses are few.  (Three pieces of 67 are not used.)  1024 tokens 32x128,64x256, the gradient: 130 us with bf16's places, 123 with these.
template <typename T> __device__ __forceinline__ int piece_of(int lane)
{
    if constexpr (sizeof(T) == 2) return (lane & 48) | ((lane + (lane >> 5) * 8) & 15);
    else {
        const int h0 = lane >> 2 & 1, h1 = lane >> 3 & 1, g0 = lane >> 4 & 1, g1 = lane >> 5;
        return (h0 ^ h1 ^ g0) + 2 * g0 + 4 * h1 + 8 * g1 + 17 * (lane & 3);
    }
}
template <typename T> __device__ __forceinline__ int half_of(int group) { return sizeof(T) == 2 ? 0 : ((group ^ (group >> 1)) & 1) * 4; }

// Fragments that are not read crossed lie without gaps: row r of group g is piece 16 g + r with the last two bits of r turned over by g, fp32: its halves
// exchanged where g is odd.  That is for these reads too, and for dZ's writes (rows_slot_at).
__device__ __forceinline__ int turned_rows(int lane) { return (lane & 60) | ((lane ^ (lane >> 4)) & 3); }
template <typename T> __device__ __forceinline__ int rows_half(int group) { return sizeof(T) == 2 ? 0 : (group & 1) * 4; }

// FLAT: for fragments that are not read crossed
template <Order O, bool FLAT = false, typename T> __device__ __forceinline__ T* frag_slot_at(T* s, int row, int k, int chunks)
{
    const int group = frag_group<O>(k & 31), slot = frag_slot<O>(k & 31), index = (row >> 4) * chunks + (k >> 5), lane = (row & 15) + 16 * group;
    if constexpr (FLAT) return s + index * FRAG + turned_rows(lane) * 8 + (slot ^ rows_half<T>(group));
    else return s + index * FRAG_LDS<T> + piece_of<T>(lane) * 8 + (slot ^ half_of<T>(group));
}

// Reads and writes fragments in LDS.
template <typename T> struct Lane {
    typedef typename Op<T>::Frag Frag;
    typedef typename Op<T>::Quad Quad;
    static constexpr bool PAIRS = sizeof(T) == 2;
    int c, g, own, rows, chained, unmixed, mixed, straight[2];

    __device__ __forceinline__ explicit Lane(int lane)
        : c(lane & 15), g(lane >> 4), own(piece_of<T>(lane) * 8 + half_of<T>(g)), rows(turned_rows(lane) * 8 + rows_half<T>(g))
    {
        // Where crossed reads start.  bf16: what this lane reads of the 4 x 16 elements that its 16 lanes exchange, row 4g + c/4, elements 4(c%4) to
        // 4(c%4)+3.  fp32: element c of row 4g; rows 4g+1 to 4g+3 are 17 pieces apart.
        chained = PAIRS ? piece_of<T>(4 * g + (c >> 2) + 16 * (c & 3)) * 8 : piece_of<T>(4 * g + 16 * (c >> 2)) * 8 + (c & 3);
        unmixed = PAIRS ? 0 : half_of<T>(c >> 2);          // the half that is the first
        mixed = unmixed ^ (PAIRS ? c & 1 : (c >> 2) & 1) * 4;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            straight[h] = PAIRS ? piece_of<T>(4 * g + (c >> 2) + 16 * (2 * h + ((c & 3) >> 1))) * 8 + 4 * (c & 1)
                                : piece_of<T>(4 * g + 16 * (2 * h + (c >> 3))) * 8 + ((c & 7) ^ half_of<T>(2 * h + (c >> 3)));
    }
    // A piece whose first half starts at `at`: the other half is on either side.
    static __device__ __forceinline__ Frag piece(const T* s, int at)
    {
        if constexpr (PAIRS) return *reinterpret_cast<const Frag*>(s + at);
        else return __builtin_shufflevector(*reinterpret_cast<const Quad*>(s + at), *reinterpret_cast<const Quad*>(s + (at ^ 4)), 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static __device__ __forceinline__ void put_piece(T* s, int at, const Frag& f)
    {
        if constexpr (PAIRS) *reinterpret_cast<Frag*>(s + at) = f;
        else {
            *reinterpret_cast<Quad*>(s + at) = __builtin_shufflevector(f, f, 0, 1, 2, 3);
            *reinterpret_cast<Quad*>(s + (at ^ 4)) = __builtin_shufflevector(f, f, 4, 5, 6, 7);
        }
    }
    __device__ __forceinline__ Frag get(const T* s, int index) const { return piece(s + index * FRAG_LDS<T>, own); }
    __device__ __forceinline__ void put(T* s, int index, const Frag& f) const { put_piece(s + index * FRAG_LDS<T>, own, f); }
    // of flat fragments: this lane's piece; this group's piece of any row
    __device__ __forceinline__ Frag get_rows(const T* s, int index) const { return piece(s + index * FRAG, rows); }
    __device__ __forceinline__ Frag get_row(const T* s, int index, int row) const { return piece(s + index * FRAG, turned_rows(row + 16 * g) * 8 + rows_half<T>(g)); }
    // eight elements from k on (a multiple of 8) of a row of what lies in the straight order
    static __device__ __forceinline__ void put_straight(T* s, int row, int k, int chunks, const Frag& f)
    {
        const int group = (k & 31) >> 3;
        put_piece(s + ((row >> 4) * chunks + (k >> 5)) * FRAG_LDS<T>, piece_of<T>((row & 15) + 16 * group) * 8 + half_of<T>(group), f);
    }

    // The two halves of a crossed fragment, each of four stored rows: by the transposing read, which gives each of 16 lanes one element from each
    // of four rows, or element by element.
    static __device__ __forceinline__ Frag halves(const T* first, const T* second)
    {
        Frag f;
        if constexpr (PAIRS) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 Shared;
            s16x4 half[2];
            half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Shared*)first);
            half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Shared*)second);
            __builtin_memcpy(&f, half, sizeof f);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = (j < 4 ? first : second)[j % 4 * 136];
        }
        return f;
    }
    // The crossed fragment: its rows are the contraction indices 16*tile to 16*tile+15 of what is stored in order O, its contraction are the stored rows of
    // row blocks `block` and `block`+1 as they lie there, chained; EXCHANGE: with the two blocks exchanged for g = 1, 3, so that rows that were
    // stored mixed come chained.
    template <Order O, bool EXCHANGE = false> __device__ __forceinline__ Frag crossed(const T* s, int block, int chunks, int tile) const
    {
        s += (block * chunks + (tile >> 1)) * FRAG_LDS<T>;
        // (by a choice, not an index: the places stay in registers)
        s += O == STRAIGHT ? (tile & 1 ? straight[1] : straight[0]) : chained + ((O == MIXED ? mixed : unmixed) ^ ((tile & 1) * 4));
        const int second = chunks * FRAG_LDS<T>, turn = EXCHANGE ? (g & 1) * second : 0;
        return halves(s + turn, s + second - turn);
    }
    // The same of a mixed operand whose 32 stored rows are columns of units of 16*N, in the columns' own order (row v of a unit is column
    // (v%16)*N + v/16): the contraction is straight over columns.
    template <int N> __device__ __forceinline__ Frag crossed_columns(const T* s, int block, int chunks, int tile) const
    {
        static_assert(N == 1 || N == 2, "32 columns in two row blocks");
        s += (block * chunks + (tile >> 1)) * FRAG_LDS<T>;
        const int half = mixed ^ ((tile & 1) * 4);
        Frag f;
        if constexpr (PAIRS) {             // this lane's row of the four: column 8g + 4h + r
            const int r = c >> 2;
            const T* from[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = N == 2 ? 4 * g + 2 * h + (r >> 1) : (8 * g + 4 * h + r) & 15;
                from[h] = s + (N == 2 ? r & 1 : g >> 1) * chunks * FRAG_LDS<T> + piece_of<T>(row + 16 * (c & 3)) * 8 + half;
            }
            f = halves(from[0], from[1]);
        } else if constexpr (N == 2) {     // columns of both blocks in turn
            s += chained + half;
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = s[(j >> 1) * 136 + (j & 1) * chunks * FRAG_LDS<T>];
        } else {
            s += (g >> 1) * chunks * FRAG_LDS<T> + (c & 3) + half;
            f = halves(s + piece_of<T>((8 * g & 15) + 16 * (c >> 2)) * 8, s + piece_of<T>((8 * g & 15) + 4 + 16 * (c >> 2)) * 8);
        }
        return f;
    }
};

// FLAT operands whose rows are a block of results' rows and whose contraction, straight, are its columns (dZ for dF1): a lane writes N neighbouring
// indices of rows 4g to 4g+3, and these writes meet all banks.
template <typename T> __device__ __forceinline__ T* rows_slot_at(T* s, int index, int row, int k)
{
    return s + index * FRAG + turned_rows(row + 16 * (k >> 3)) * 8 + ((k & 7) ^ rows_half<T>(k >> 3));
}

// Lays an operand of `rows` x `ks`, element (row, k) at src[k*stride + row], out in fragments, `blocks` x 16 rows and `chunks` x 32 contraction indices
// with zeros outside.  A thread takes 4 rows of 4 indices (four indices of a row stay together in every order).  `vec`: four neighbours can be read at
// once (stride a multiple of 4, address fits).  place(row): the row of the fragments that a row goes to, 0 to 16*blocks-1, each once.
template <Order O, bool FLAT, typename T, class Place>
__device__ __forceinline__ void lay_out(T* dst, const T* __restrict__ src, int rows, int ks, int64_t stride, int blocks, int chunks, bool vec, int tid, int threads, Place place)
{
    typedef typename Op<T>::Quad Quad;
    const int across = blocks * 4;
    for (int i = tid; i < across * chunks * 8; i += threads) {
        const int row = 4 * (i % across), k = 4 * (i / across);
        Quad m[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const T* const from = src + (int64_t)(k + e) * stride + row;
            m[e] = Quad{};
            if (vec && row + 4 <= rows) {
                if (k + e < ks) m[e] = *reinterpret_cast<const Quad*>(from);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (k + e < ks && row + j < rows) m[e][j] = from[j];
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) *reinterpret_cast<Quad*>(frag_slot_at<O, FLAT>(dst, place(row + e), k, chunks)) = Quad{m[0][e], m[1][e], m[2][e], m[3][e]};
    }
}
struct InPlace { __device__ __forceinline__ int operator()(int row) const { return row; } };
struct MixedRows { __device__ __forceinline__ int operator()(int row) const { return mixed_row(row); } };

// A span of memory that is read without branches: what lies past its end, and what is asked for at NOWHERE, reads as zeros.  The
// loads are plain ones otherwise, so they stay in flight until their values are used.
constexpr unsigned NOWHERE = 0x80000000u;
template <typename T> struct Span {
    __amdgpu_buffer_rsrc_t r;
    // `start` has to be the same in all lanes, `elements` * sizeof(T) below 2^31; a span of no or fewer elements has nothing that could be read
    __device__ __forceinline__ Span(const T* start, int elements) : r(__builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(start), 0, max(elements, 0) * (int)sizeof(T), 0x00020000)) {}

    // one element to `at`; nothing is written at NOWHERE
    __device__ __forceinline__ void set(unsigned at, T v) const
    {
        const unsigned o = at == NOWHERE ? NOWHERE : at * (unsigned)sizeof(T);
        if constexpr (sizeof(T) == 2) {
            unsigned short x;
            __builtin_memcpy(&x, &v, 2);
            __builtin_amdgcn_raw_buffer_store_b16(x, r, o, 0, 0);
        } else {
            unsigned x;
            __builtin_memcpy(&x, &v, 4);
            __builtin_amdgcn_raw_buffer_store_b32(x, r, o, 0, 0);
        }
    }
    // element `at`; zero at NOWHERE
    __device__ __forceinline__ T get(unsigned at) const
    {
        const unsigned o = at == NOWHERE ? NOWHERE : at * (unsigned)sizeof(T);
        T v;
        if constexpr (sizeof(T) == 2) {
            const unsigned short x = __builtin_amdgcn_raw_buffer_load_b16(r, o, 0, 0);
            __builtin_memcpy(&v, &x, 2);
        } else {
            const unsigned x = __builtin_amdgcn_raw_buffer_load_b32(r, o, 0, 0);
            __builtin_memcpy(&v, &x, 4);
        }
        return v;
    }
};

// Eight elements of a token's row from element `at` on, in straight order a lane's part of a fragment.  Element addresses are enough (memory is
// read unaligned, 16 bytes at once).  A fragment's places outside P1 x P2 get some other elements of the same row: their
// factor's row is zeros, and what an infinity or NaN there spoils is the token's own results, all of which it is part of anyhow.  So
// there is no choice between loaded values and zeros that would have to wait for them.  `near_end`: some lane may need fewer than eight; it reads the
// row's last eight and moves them down.  WHOLE: no row has fewer than eight elements, as in all classes of factors but the first.  Shorter ones are read
// one by one; `first`: some of a short row may be in this fragment.
template <bool WHOLE, typename T> __device__ __forceinline__ typename Op<T>::Frag eight_of_row(const T* __restrict__ x, int at, bool inside, int total, bool near_end, bool first)
{
    typedef typename Op<T>::Frag Frag;
    Frag f = {};
    if (WHOLE || total >= 8) {
        at = inside ? at : 0;
        const int from = min(at, total - 8);
        __builtin_memcpy(&f, x + from, sizeof f);
        if (near_end) {
            const int over = at - from;
            const Frag z = {};
            Frag m = __builtin_shufflevector(f, z, 4, 5, 6, 7, 8, 9, 10, 11);
            f = over & 4 ? m : f;
            m = __builtin_shufflevector(f, z, 2, 3, 4, 5, 6, 7, 8, 9);
            f = over & 2 ? m : f;
            m = __builtin_shufflevector(f, z, 1, 2, 3, 4, 5, 6, 7, 8);
            f = over & 1 ? m : f;
        }
    } else if (first) {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (inside && at + j < total) f[j] = x[at + j];
    }
    return f;
}

// The activation of a gate and its derivative.  Both activations are z * sigma(v), sigma the logistic function: v = z (SiLU), or
// v = 2c(z + 0.044715 z^3) with c = sqrt(2/pi), which is GELU's form with tanh, since (1 + tanh w)/2 = sigma(2w).  So
// neither end cancels, and v_rcp's last place is enough: exp(-v) overflows to infinity where 1/(1+inf) = 0 is right.  dv stays a number for any z, so that sigma's slope of 0 takes it away.
template <bool GELU> __device__ __forceinline__ float activate(float z, float& slope)
{
    const float c2 = 1.5957691216057308f;
    const float v = GELU ? c2 * z * (1.0f + 0.044715f * z * z) : z, dv = GELU ? c2 * (1.0f + 3.0f * 0.044715f * fminf(z * z, 1e30f)) : 1.0f;
    const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-v));
    slope = s + z * (s * (1.0f - s)) * dv;
    return z * s;
}

// act(z) * u for the forward pass, where SiLU's z comes times log2 e, which the divisor takes back.  u comes last: z * u may be infinite where a closed
// gate makes the result 0.
template <bool GELU> __device__ __forceinline__ float gate(float z, float u)
{
    if constexpr (GELU) {
        float slope;
        return activate<true>(z, slope) * u;
    } else return z * __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_amdgcn_exp2f(-z), LOG2E, LOG2E)) * u;
}

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

enum : int { OP_SILU = 0, OP_GELU = 1, OP_LOSS = 2 };

}  // namespace km
