// Pieces of the gated delta rule's kernels (delta.hip, delta_grad.hip): operands on the matrix cores, tiles in LDS, sequences and chunks.
//
// Products run on the bf16 matrix instruction (16 x 16 x 32) at the precision of 32 bits: a number x is the sum of up to three bf16 pieces
// (x0 = bf16(x), x1 = bf16(x - x0), x2 = bf16(x - x0 - x1): 24 bits), a product of two numbers the sum of the products of pieces i, j with
// i + j < 3.  An input in bf16 is one piece, in f16 two, in f32 three; what the kernels compute is three.  That is 3 instructions for bf16 input
// times a computed operand and 6 for two computed ones, against the 16 that the 32-bit matrix instruction takes in time.
//
// The accumulator of a 16 x 16 tile has, in lane l, column l % 16 and rows 4 (l / 16) .. + 3; an operand of 32 summed elements has, in lane l, row
// (or column) l % 16 and 8 elements.  Since the order of summation is free, the two tiles of rows 32 s .. 32 s + 31 of an accumulator ARE the operand of
// step s, if the other operand takes its 8 elements in the same order: 32 s + 4 (l / 16) .. + 3 and 16 more .. + 3.  Tiles in LDS are kept in that order
// (slot_of), so that no accumulator passes through LDS on its way into the next product.
#pragma once
#include "layer.hpp"
#include "lowp.hpp"

namespace la {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

// What one call works on.  Tensors are [sequences][tokens][heads][size], rows of q, k, v `ld` elements apart per token, the others dense;
// with `offsets` the sequences lie one behind another, sequence n in tokens offsets[n] .. offsets[n + 1] - 1.
struct DeltaArgs {
    const void *q, *k, *v;
    int64_t ldq, ldk, ldv;
    const float *g, *beta;
    const float *state0;    // initial states [sequences][hv][dk][dv], or null
    const int32_t *offsets;
    int64_t batch, tokens;  // tokens of one sequence, of all with `offsets`
    int hk, hv, dk, dv;
    float scale;
    void *o;
    float *state1;  // final states or null
    // by chunk slot and value head: the inverses T [C][C], and for the gradient the state before the chunk [DKP][dvp] and U [C][dvp]
    float *inv, *chunk_state, *chunk_u;
    int64_t slots;
    int dvp;  // dv rounded up to whole tiles
    // gradient
    const void *o_bar;
    const float *state1_bar;
    float *chunk_state_bar, *chunk_z_bar;  // the state's gradient after the chunk, the gradient of Z
    void *q_bar, *k_bar, *v_bar;
    float *g_bar, *beta_bar, *state0_bar;
    int slices;  // blocks over dv
};

template <typename T>
struct DeltaIn;
template <>
struct DeltaIn<bf16_t> {
    static constexpr int NI = 1, C = 64;
};
template <>
struct DeltaIn<f16_t> {
    static constexpr int NI = 2, C = 32;
};
template <>
struct DeltaIn<float> {
    static constexpr int NI = 3, C = 32;
};

constexpr int NX = 3;  // pieces of what is computed

template <int N>
struct Frag {
    bf16x8 p[N];
};

// d += a b, products of the smallest pieces first
template <int NA, int NB>
__device__ __forceinline__ void mma(f32x4 &d, const Frag<NA> &a, const Frag<NB> &b)
{
#pragma unroll
    for (int s = 2; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB)
                d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[s - i], d, 0, 0, 0);
}

template <int N>
__device__ __forceinline__ Frag<N> split(f32x8 x)
{
    Frag<N> f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        f.p[i] = __builtin_convertvector(x, bf16x8);
        if (i + 1 < N)
            x -= __builtin_convertvector(f.p[i], f32x8);
    }
    return f;
}
__device__ __forceinline__ f32x8 join(f32x4 a, f32x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// where element c of a row (or the first of four from a multiple of four) lies in an LDS tile
__device__ __forceinline__ int slot_of(int c)
{
    return (c & ~31) + 8 * ((c & 15) >> 2) + 4 * ((c & 31) >> 4) + (c & 3);
}

// N planes of ROWS x COLS bf16 pieces; 8 elements of padding spread the rows over the banks
template <int N, int ROWS, int COLS>
struct Planes {
    static constexpr int LD = COLS + 8;
    bf16_t e[N][ROWS][LD];
    // the operand of rows r0 .. r0 + 15, summed elements 32 s .. 32 s + 31
    __device__ __forceinline__ Frag<N> frag(int r0, int s) const
    {
        const int lane = threadIdx.x & 63;
        Frag<N> f;
#pragma unroll
        for (int i = 0; i < N; ++i)
            f.p[i] = *reinterpret_cast<const bf16x8 *>(&e[i][r0 + (lane & 15)][32 * s + 8 * (lane >> 4)]);
        return f;
    }
    // four elements c .. c + 3 of row r, c a multiple of four
    __device__ __forceinline__ void put4(int r, int c, f32x4 x)
    {
        const int at = slot_of(c);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bf16x4 h = __builtin_convertvector(x, bf16x4);
            *reinterpret_cast<bf16x4 *>(&e[i][r][at]) = h;
            if (i + 1 < N)
                x -= __builtin_convertvector(h, f32x4);
        }
    }
    __device__ __forceinline__ f32x4 get4(int r, int c) const
    {
        const int at = slot_of(c);
        f32x4 x = {0, 0, 0, 0};
#pragma unroll
        for (int i = N - 1; i >= 0; --i)
            x += __builtin_convertvector(*reinterpret_cast<const bf16x4 *>(&e[i][r][at]), f32x4);
        return x;
    }
};

// 8 elements of a row, those past `n` zero
template <typename T>
__device__ __forceinline__ f32x8 load8(const T *p, int n)
{
    float v[8];
    load_part<T, 8>(p, n, v);
    return f32x8{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
}

// A chunk of q or k: C rows of DKP elements (zeros past `len` rows and `dk` elements), as rows, and turned, summed over the tokens.
template <typename T, int NI, int C, int DKP, bool ROWS, bool TURNED>
__device__ __forceinline__ void stage_chunk(const T *src, int64_t ld, int len, int dk, Planes<NI, C, DKP> *rows, Planes<NI, DKP, C> *turned)
{
    constexpr int UC = DKP / 8, UNITS = (C / 4) * UC;
    for (int u = threadIdx.x; u < UNITS; u += blockDim.x) {
        const int c = 8 * (u % UC), r = 4 * (u / UC);
        f32x8 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[i] = load8<T>(src + (int64_t)(r + i) * ld + c, r + i < len ? dk - c : 0);
        if constexpr (ROWS) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                rows->put4(r + i, c, __builtin_shufflevector(x[i], x[i], 0, 1, 2, 3));
                rows->put4(r + i, c + 4, __builtin_shufflevector(x[i], x[i], 4, 5, 6, 7));
            }
        }
        if constexpr (TURNED) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                turned->put4(c + j, r, f32x4{x[0][j], x[1][j], x[2][j], x[3][j]});
        }
    }
}

// a sequence's first token and length; what `offsets` holds is kept inside the tokens there are
__device__ __forceinline__ void sequence(const DeltaArgs &p, int64_t n, int64_t &t0, int64_t &len)
{
    if (!p.offsets) {
        t0 = n * p.tokens;
        len = p.tokens;
        return;
    }
    const int64_t a = p.offsets[n], b = p.offsets[n + 1];
    t0 = a < 0 ? 0 : a > p.tokens ? p.tokens : a;
    len = (b > p.tokens ? p.tokens : b) - t0;
    len = len < 0 ? 0 : len;
}

// The slot of a sequence's first chunk.  Packed sequences: t0 / C + n, which leaves every sequence the slots it needs without a sum over those before it
// (floor(x) + 1 >= ceil(x)) and stays below tokens / C + sequences.
template <int C>
__device__ __forceinline__ int64_t first_slot(const DeltaArgs &p, int64_t n, int64_t t0)
{
    return p.offsets ? t0 / C + n : n * ((p.tokens + C - 1) / C);
}

// The sequence and chunk of a slot; false where it has none.
template <int C>
__device__ __forceinline__ bool slot_chunk(const DeltaArgs &p, int64_t slot, int64_t &t0, int &len)
{
    int64_t n, all;
    if (!p.offsets) {
        n = slot / ((p.tokens + C - 1) / C);
    } else {
        int64_t lo = 0, hi = p.batch - 1;
        while (lo < hi) {
            const int64_t mid = (lo + hi + 1) / 2;
            sequence(p, mid, t0, all);
            if (first_slot<C>(p, mid, t0) <= slot)
                lo = mid;
            else
                hi = mid - 1;
        }
        n = lo;
    }
    sequence(p, n, t0, all);
    const int64_t c = slot - first_slot<C>(p, n, t0);
    if (c < 0 || c * C >= all)
        return false;
    t0 += c * C;
    const int64_t left = all - c * C;
    len = (int)(left < C ? left : C);
    return true;
}

// Decays of a chunk: b_i the sum of g up to token i in 64 bits (differences of it are exact enough for any decay; g below -1000 counts as -1000, whose
// exponential is zero), and what the products take from it.  Tokens past the end have g = beta = 0.
template <int C>
struct alignas(16) Decays {
    double b[C];
    float in[C], out[C], beta[C];  // exp(b_i), exp(b_last - b_i)
    float all;                     // exp(b_last)
    // by the lanes of one wavefront
    __device__ __forceinline__ void load(const float *g, const float *be, int64_t ld, int len)
    {
        const int i = threadIdx.x & 63;
        double x = i < len ? fmax((double)g[(int64_t)i * ld], -1000.0) : 0.0;
        if (i < len && g[(int64_t)i * ld] != g[(int64_t)i * ld])
            x = g[(int64_t)i * ld];
#pragma unroll
        for (int s = 1; s < C; s *= 2) {
            const double y = __shfl_up(x, s, 64);
            if (i >= s)
                x += y;
        }
        const double last = __shfl(x, C - 1, 64);
        if (i < C) {
            b[i] = x;
            in[i] = expf((float)x);
            out[i] = expf((float)(last - x));
            beta[i] = i < len ? be[(int64_t)i * ld] : 0.0f;
        }
        if (i == 0)
            all = expf((float)last);
    }
    __device__ __forceinline__ float between(int i, int j) const { return expf((float)(b[i] - b[j])); }
    __device__ __forceinline__ f32x4 four(const float *x, int i) const { return *reinterpret_cast<const f32x4 *>(x + i); }
};

}  // namespace la
