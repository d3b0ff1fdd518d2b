// Pieces of the gated delta rule's kernels (delta.hip, delta_grad.hip): operands on the matrix cores, packets of them, sequences and chunks.
//
// Products run on the bf16 matrix instruction (16 x 16 x 32) at the precision of 32 bits: a number x is the sum of up to three bf16 pieces
// (x0 = bf16(x), x1 = bf16(x - x0), x2 = bf16(x - x0 - x1): 24 bits), a product of two numbers the sum of the products of pieces i, j with
// i + j < 3.  An input in bf16 is one piece, in f16 two, in f32 three; what the kernels compute is three.  That is 3 instructions for bf16 input
// times a computed operand and 6 for two computed ones, against the 16 that the 32-bit matrix instruction takes in time.
//
// An operand of 32 summed elements has, in lane l, row (or column) l % 16 and elements 8 (l / 16) .. + 7; the accumulator of a 16 x 16 tile has column
// l % 16 and rows 4 (l / 16) .. + 3.  Which token or key element a tile's row stands for is free, so row 4 x + r of tile 2 s + y is taken to be element
// 32 s + 8 x + 4 y + r: then tiles 2 s and 2 s + 1 of an accumulator ARE the operand of step s, and no accumulator passes through LDS on its way into
// the next product.
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
    int64_t slots;  // chunks
    int dvp;        // dv rounded up to whole steps
    // by chunk slot: packets of operands for every key head and every value head; for the gradient the state before the chunk [DKP][dvp] and U [C][dvp]
    char *pack_k, *pack_v;
    float *chunk_state, *chunk_u;
    // gradient
    const void *o_bar;
    const float *state1_bar;
    float *chunk_state_bar, *chunk_z_bar;  // the state's gradient after the chunk, the gradient of Z
    void *q_bar, *k_bar, *v_bar;
    float *g_bar, *beta_bar, *state0_bar;
    int slices;  // blocks over dv
    int pack_heads;  // value heads of a block of k_delta_pack
    // Few sequences and heads: they are walked in segments of `seg` chunks (0: whole).  By segment slot and value head: the state before it [DKP][dvp], and
    // the matrix [DKP][DKP] by which a segment's last state depends on its first.
    int seg;
    int64_t segs;
    float *seg_state, *seg_map;
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

constexpr int NX = 3;       // pieces of what is computed
constexpr int64_t COMPUTE_UNITS = 256;
constexpr int LDS_BYTES = 160 * 1024;  // of a compute unit
constexpr int UNIT = 1024;  // bytes of an operand of 16 rows, 32 summed elements and one piece, 16 a lane: "a unit"

template <int N>
struct Frag {
    bf16x8 p[N];
};

// d += a b: products of pieces i, j with i + j < LIM, the smallest first
template <int LIM, int NA, int NB>
__device__ __forceinline__ void mma(f32x4 &d, const Frag<NA> &a, const Frag<NB> &b)
{
#pragma unroll
    for (int s = LIM - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB)
                d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[s - i], d, 0, 0, 0);
}

// the same for N tiles with one operand in common, tile after tile: no instruction waits for the one before it
template <int LIM, int N, int NA, int NB>
__device__ __forceinline__ void mma_tiles(f32x4 *d, const Frag<NA> *a, const Frag<NB> &b)
{
#pragma unroll
    for (int s = LIM - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB) {
#pragma unroll
                for (int n = 0; n < N; ++n)
                    d[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[n].p[i], b.p[s - i], d[n], 0, 0, 0);
            }
}
// keeps what is before it (loads of operands) before what follows: the compiler moves loads down to their use, where they would be waited for
__device__ __forceinline__ void issue_point() { __builtin_amdgcn_sched_barrier(0); }

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

// the element that row m of tile i stands for; the first of the four that a lane's accumulator of tile i holds
__device__ __forceinline__ int element_of(int i, int m) { return 32 * (i >> 1) + 8 * (m >> 2) + 4 * (i & 1) + (m & 3); }
__device__ __forceinline__ int first_of(int i) { return 32 * (i >> 1) + 8 * ((threadIdx.x & 63) >> 4) + 4 * (i & 1); }

// Block b runs on die b % 8 of the 8: an order in which the `slices` blocks of a head, which read the same packets, run on the same die and find them in its
// cache, while the heads go round the dies (sequences of like lengths may lie side by side).
__device__ __forceinline__ unsigned block_of_die(unsigned slices)
{
    const unsigned b = blockIdx.x, whole = gridDim.x / slices / 8 * 8 * slices, i = b / 8;
    return b < whole ? (i / slices * 8 + b % 8) * slices + i % slices : b;
}

// Two wavefronts share 16 columns of a walk: wavefront `half` keeps the state's rows and forms the chunk's tokens of its half of the tiles.  What the other one
// needs of it passes through LDS: operands of a step (32 tokens), whose tiles a wavefront has both (RT = 4, step `half`) or one of (RT = 2).
template <int RT>
__device__ __forceinline__ void put_step(char *base, int half, const f32x4 *x)
{
    const int lane = threadIdx.x & 63;
    if constexpr (RT == 4) {
        const Frag<NX> f = split<NX>(join(x[0], x[1]));
#pragma unroll
        for (int i = 0; i < NX; ++i)
            *reinterpret_cast<bf16x8 *>(base + (half * NX + i) * UNIT + 16 * lane) = f.p[i];
    } else {
        f32x4 y = x[0];
#pragma unroll
        for (int i = 0; i < NX; ++i) {
            const bf16x4 h = __builtin_convertvector(y, bf16x4);
            *reinterpret_cast<bf16x4 *>(base + i * UNIT + 16 * lane + 8 * half) = h;
            if (i + 1 < NX)
                y -= __builtin_convertvector(h, f32x4);
        }
    }
}

// Operands of one chunk in units, in the order in which a wavefront reads them.
//   key head:   K (rows tokens, summed over dk), Q, and turned (rows dk, summed over tokens) Kt, for the gradient also Qt
//   value head: decays (2 units), T and P T (lower triangles: steps s <= i / 2 of row tile i), for the gradient also T^T and P^T (s >= i / 2)
template <typename T, int DKP>
struct Pack {
    static constexpr int C = DeltaIn<T>::C, NI = DeltaIn<T>::NI;
    static constexpr int RT = C / 16, KS = DKP / 32, KT = DKP / 16, CS = C / 32;
    static constexpr int NO = NI == 3 ? 3 : 2;  // pieces of what only the answers take: they are rounded to the input's type
    static constexpr int FK = RT * KS, FT = CS == 1 ? 2 : 6;
    // Two blocks of two column groups of the forward walk fit the LDS side by side: always two then, the blocks of sequences of different lengths end more evenly
    // (12 sequences of 1 to 2000 tokens, 12 heads, the whole call: f16 of 72 x 100 295 us with two, 309 with four, f32 of 64 216 and 256; of one length 0.98 to 1.04
    // times as fast; where two do not fit, bf16 of 128, 252 and 222 us; the backward walk of one length is 1 to 5 % slower with two).
    static constexpr bool PAIRED = C == 32 && NI * DKP <= 256;
    static constexpr int K = 0, Q = NI * FK, KTURN = 2 * NI * FK, QTURN = 3 * NI * FK;
    static constexpr int D = 0, TINV = 2, P = TINV + NX * FT, TTURN = P + NO * FT, PTURN = TTURN + NX * FT;
    static constexpr int key_units(bool save) { return (save ? 4 : 3) * NI * FK; }
    static constexpr int value_units(bool save) { return save ? PTURN + NX * FT : TTURN; }
    // unit of row tile i, step s (of piece 0; piece p is p * FK or p * FT further)
    static constexpr __host__ __device__ int row(int i, int s) { return i * KS + s; }
    static constexpr __host__ __device__ int turned(int i, int s) { return i * CS + s; }
    static constexpr __host__ __device__ int lower(int i, int s) { return CS == 1 || i < 2 ? i : 2 * i - 2 + s; }
    static constexpr __host__ __device__ int upper(int i, int s) { return CS == 1 ? i : i < 2 ? 2 * i + s : 2 + i; }
};

// Column groups of 16 of a walk's block, two or four.  A block of two has a SIMD for every wavefront, and a chunk takes it less time: two where four would leave
// half of the compute units idle (2 x 4096 tokens, 32 heads of 128, bf16: the scans of the two passes take 311 and 314 us with two, 365 and 373 with four).
// With more blocks than compute units four share what they load.
inline int walk_groups(int64_t heads, int dv) { return heads * ((dv + 63) / 64) * 2 <= 256 ? 2 : 4; }

// a unit's operand: N pieces, `apart` units from one to the next
template <int N>
__device__ __forceinline__ Frag<N> unit(const char *base, int u, int apart)
{
    Frag<N> f;
#pragma unroll
    for (int i = 0; i < N; ++i)
        f.p[i] = *reinterpret_cast<const bf16x8 *>(base + (u + i * apart) * UNIT + (threadIdx.x & 63) * 16);
    return f;
}
template <int N>
__device__ __forceinline__ void put_unit(char *base, int u, int apart, f32x8 x)
{
    const Frag<N> f = split<N>(x);
#pragma unroll
    for (int i = 0; i < N; ++i)
        *reinterpret_cast<bf16x8 *>(base + (int64_t)(u + i * apart) * UNIT + (threadIdx.x & 63) * 16) = f.p[i];
}

// N units (up to 4) from memory to LDS by one wavefront: a lane's 16 bytes of a unit from `src` (uniform) + 16 lane to LDS address `at` (uniform) + 16 lane.
// Written as assembly because the compiler waits for all loads in flight before it reads any LDS when it knows of one that writes there: who calls this
// waits by wait_loads.  An instruction's offset counts for both addresses.  (The wait states are what a scalar register that a vector instruction has written,
// as the address may be, has to have before a load takes it.)  The warning is about any clobber of m0; without it the compiler takes m0 for unchanged.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int N>
__device__ __forceinline__ void stream_units(const char *src, uint32_t at)
{
    const uint32_t off = (threadIdx.x & 63) * 16;
    static_assert(N >= 1 && N <= 4 && UNIT == 1024, "offsets below 4096");
    if constexpr (N == 1)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(off), "s"(src) : "m0", "memory");
    else if constexpr (N == 2)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2\n\tglobal_load_lds_dwordx4 %1, %2 offset:1024" ::"s"(at), "v"(off),
                     "s"(src)
                     : "m0", "memory");
    else if constexpr (N == 3)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2\n\tglobal_load_lds_dwordx4 %1, %2 offset:1024\n\t"
                     "global_load_lds_dwordx4 %1, %2 offset:2048" ::"s"(at), "v"(off), "s"(src)
                     : "m0", "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2\n\tglobal_load_lds_dwordx4 %1, %2 offset:1024\n\t"
                     "global_load_lds_dwordx4 %1, %2 offset:2048\n\tglobal_load_lds_dwordx4 %1, %2 offset:0xc00" ::"s"(at), "v"(off), "s"(src)
                     : "m0", "memory");
}
#pragma clang diagnostic pop
// A run of units by NW wavefronts, each its part of share(): the last ones' parts overlap where NW does not divide the run, so that all issue as many loads.
template <int UNITS, int NW>
constexpr int share()
{
    return (UNITS + NW - 1) / NW;
}
template <int UNITS, int NW>
__device__ __forceinline__ void stream_run(const char *src, uint32_t at, int wave)
{
    constexpr int EACH = share<UNITS, NW>();
    const int u = wave * EACH < UNITS - EACH ? wave * EACH : UNITS - EACH;
    src += u * UNIT;
    at += u * UNIT;
#pragma unroll
    for (int i = 0; i + 4 <= EACH; i += 4)
        stream_units<4>(src + i * UNIT, at + i * UNIT);
    if constexpr (EACH % 4 != 0)
        stream_units<EACH % 4>(src + EACH / 4 * 4 * UNIT, at + EACH / 4 * 4 * UNIT);
}
// the LDS address of a shared array
__device__ __forceinline__ uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p; }
// the sum over the 16 lanes of a row of lanes, in all of them
__device__ __forceinline__ float row16_sum(float x)
{
#define LA_ROR(n) x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + n, 0xf, 0xf, false))
    LA_ROR(8);
    LA_ROR(4);
    LA_ROR(2);
    LA_ROR(1);
#undef LA_ROR
    return x;
}
// until at most N of this wavefront's loads (and stores) are in flight
template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// A barrier that leaves loads and stores of memory in flight; this wavefront's reads of LDS are done.
__device__ __forceinline__ void block_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// 8 elements of a row, those past `n` zero
template <typename T>
__device__ __forceinline__ f32x8 load8(const T *p, int n)
{
    float v[8];
    load_part<T, 8>(p, n, v);
    return f32x8{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
}

// The walks' rows of v, o and their like pass through LDS, 16 bytes a lane: a wavefront that is alone on its SIMD pays for every instruction, and an access
// of 2 bytes is one as well.  Rows past `rows` and columns past `cols` are not touched; nothing has to be aligned.
// In: 16 NG columns of C rows, by NT lanes; a chunk ahead into registers, then into LDS.
template <typename T, int C, int NG, int NT>
struct RowsIn {
    static constexpr int PE = 16 / sizeof(T), RP = 16 * NG / PE, PACKS = C * RP, PER = (PACKS + NT - 1) / NT;  // elements of a pack, packs of a row, of a lane
    using Pack16 = PackOf<T, 16 / sizeof(T)>;
    typename Pack16::whole x[PER];
    __device__ __forceinline__ void fetch(const T *src, int64_t ld, int rows, int cols)
    {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int u = k * NT + threadIdx.x, row = u < PACKS ? u / RP : rows, c = u % RP * PE;
            const T *at = src + row * ld + c;
            if (row < rows && c + PE <= cols) {
                x[k] = *(typename Pack16::source)at;
            } else {
                at = opaque(at);
#pragma unroll
                for (int e = 0; e < PE; ++e)
                    x[k][e] = row < rows && c + e < cols ? in_memory(at)[e] : (T)0.0f;
            }
        }
    }
    __device__ __forceinline__ void put(char *lds) const
    {
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if (k * NT + (int)threadIdx.x < PACKS)
                *reinterpret_cast<typename Pack16::whole *>(lds + (k * NT + threadIdx.x) * 16) = x[k];
    }
    static __device__ __forceinline__ float at(const char *lds, int row, int col) { return (float)*reinterpret_cast<const T *>(lds + (row * 16 * NG + col) * sizeof(T)); }
};
// Out: a wavefront's 16 columns and N tiles of an accumulator.  Element 4 x + r of tile i is row 8 x + 4 i + r of the 32 that a pair of tiles makes; where N is 1,
// `odd` says which of the two the tile is.
template <typename T, int N>
struct RowsOut {
    static constexpr int ROW = 16 * sizeof(T) + 16, PE = 16 / sizeof(T), RP = sizeof(T);  // bytes of a row with its padding; elements of a pack, packs of a row
    static constexpr int BYTES = 16 * N * ROW, PER = (16 * N * RP + 63) / 64;                     // packs of a lane
    using Pack16 = PackOf<T, 16 / sizeof(T)>;
    using whole = typename Pack16::whole;
    static __device__ __forceinline__ void store(char *buf, T *dst, int64_t ld, const f32x4 *x, int rows, int cols, int odd = 0)
    {
        const int lane = threadIdx.x & 63, col = lane & 15, x4 = lane >> 4;
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)  // (rows in their order; of a tile alone: 4 x + r)
                *reinterpret_cast<T *>(buf + ((N == 1 ? 4 * x4 : 32 * (i >> 1) + 8 * x4 + 4 * (i & 1)) + r) * ROW + col * sizeof(T)) = (T)x[i][r];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        whole y[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k)
            y[k] = *reinterpret_cast<const whole *>(buf + ((k * (64 / RP) + lane / RP) & (16 * N - 1)) * ROW + lane % RP * 16);
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int l = k * (64 / RP) + lane / RP, row = l >= 16 * N ? rows : N == 1 ? 8 * (l >> 2) + 4 * odd + (l & 3) : l, c = lane % RP * PE;
            T *at = dst + row * ld + c;
            if (row < rows && c + PE <= cols) {
                *(typename Pack16::target)at = y[k];
            } else {
                at = opaque(at);
#pragma unroll
                for (int e = 0; e < PE; ++e)
                    if (row < rows && c + e < cols)
                        in_memory(at)[e] = y[k][e];
            }
        }
    }
};
template <int N>
constexpr int rows_out_bytes()
{
    return RowsOut<float, N>::BYTES > RowsOut<bf16_t, N>::BYTES ? RowsOut<float, N>::BYTES : RowsOut<bf16_t, N>::BYTES;
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

// The slot of a sequence's first segment, by first_slot's trick on the chunks' slots.
template <int C>
__device__ __forceinline__ int64_t first_segment(const DeltaArgs &p, int64_t n, int64_t t0)
{
    const int64_t each = (p.tokens + C - 1) / C;
    return p.offsets ? first_slot<C>(p, n, t0) / p.seg + n : n * (each > 0 ? (each + p.seg - 1) / p.seg : 1);
}
// The sequence of a segment's slot (slots between two sequences' belong to the one before).
template <int C>
__device__ __forceinline__ int64_t segment_sequence(const DeltaArgs &p, int64_t sg)
{
    int64_t lo = 0, hi = p.batch - 1, t0, all;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) / 2;
        sequence(p, mid, t0, all);
        if (first_segment<C>(p, mid, t0) <= sg)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// 2^x for x <= 0 in 64 bits: the whole part by the exponent, so that a large x costs no precision
__device__ __forceinline__ float exp2_of(double x)
{
    const double n = rint(x);
    return ldexpf(__builtin_amdgcn_exp2f((float)(x - n)), (int)fmax(n, -1000.0));
}

// Decays of a chunk: b_i the sum of g log2(e) up to token i in 64 bits (differences of it are exact enough for any decay; g below -1000 counts as -1000, whose
// exponential is zero), and what the products take from it.  Tokens past the end have g = beta = 0.  The second unit is what the walks read.
template <int C>
struct alignas(16) Walk {
    float in[C], out[C], beta[C];  // 2^b_i, 2^(b_last - b_i)
    float all;                     // 2^b_last
    char rest[UNIT - (3 * C + 1) * 4];
    static __device__ __forceinline__ f32x4 four(const float *x, int i) { return *reinterpret_cast<const f32x4 *>(x + i); }
};
template <int C>
struct alignas(16) Decays {
    double b[C];
    char rest[UNIT - 8 * C];
    Walk<C> walk;
    // by the lanes of one wavefront
    __device__ __forceinline__ void load(const float *g, const float *be, int64_t ld, int len)
    {
        const int i = threadIdx.x & 63;
        float y = i < len ? g[(int64_t)i * ld] : 0.0f;
        const float gate = i < len ? be[(int64_t)i * ld] : 0.0f;
        y = y < -1000.0f ? -1000.0f : y;
        double x = 1.4426950408889634074 * y;  // log2(e)
#pragma unroll
        for (int s = 1; s < C; s *= 2) {
            const double z = __shfl_up(x, s, 64);
            if (i >= s)
                x += z;
        }
        const double last = __shfl(x, C - 1, 64);
        if (i < C) {
            b[i] = x;
            walk.in[i] = exp2_of(x);
            walk.out[i] = exp2_of(last - x);
            walk.beta[i] = gate;
        }
        if (i == 0)
            walk.all = exp2_of(last);
    }
    __device__ __forceinline__ float between(int i, int j) const { return __builtin_amdgcn_exp2f((float)(b[i] - b[j])); }
};
static_assert(sizeof(Decays<64>) == 2 * UNIT && sizeof(Decays<32>) == 2 * UNIT, "two units");

}  // namespace la
