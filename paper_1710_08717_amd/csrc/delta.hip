// The gated delta rule over whole sequences: state S [dk, dv] of every sequence and value head,
//
//   S_t = a_t S_{t-1} + k_t u_t^T,   a_t = exp(g_t),   u_t = beta_t (v_t - a_t S_{t-1}^T k_t),   o_t = scale S_t^T q_t
//
// by chunks of C tokens.  With b the running sum of g inside the chunk and S0 the state before it, the u_t of a chunk solve a unit
// lower-triangular system:
//
//   A_ij = beta_i exp(b_i - b_j) k_i.k_j (j < i),   T = (I + A)^-1,   Z = beta (V - exp(b) K S0),   U = T Z,
//   P_ij = scale exp(b_i - b_j) q_i.k_j (j <= i),   O = scale exp(b) Q S0 + P U,   S1 = exp(b_last) S0 + K^T exp(b_last - b) U.
//
// k_delta_pack forms T, P T (O = scale exp(b) Q S0 + (P T) Z) and the operands' packets for all chunks at once; k_delta_scan walks a sequence's chunks.
// Everything after T is separate for every column of V, so two wavefronts take 16 columns and keep the state of them in accumulators from the first chunk
// to the last.
#include "delta.hpp"

namespace la {

// ---------------------------------------------------------------------------------
// packets of operands, for all chunks at once
// ---------------------------------------------------------------------------------
// One block a chunk and key head.  K Q and K K^T are formed once and stay in accumulators, the decays of every value head are laid over them.  T is
// formed by blocks: the 16 x 16 blocks of the diagonal by substitution, a column a lane, then twice the lower left block of a 2 x 2 block matrix,
// -T22 (A21 T11), on the 32-bit matrix instruction.  Bound by the packets that it writes and by its steps' latency: 2 x 4096 tokens, 16 key and 32 value heads of
// 128, bf16, everything kept: 127 us.  One block a chunk and value head where there are at most two such blocks a compute unit, which form K K^T and Q K^T
// again: 3 x 333 tokens, 2 key and 6 value heads of 48 x 65, f32: 15 us instead of 22 (the whole call of 1024 tokens, 16 / 32 heads of 128, bf16, 512 such
// blocks: 71 and 77; of 4096 tokens, 4 / 32 heads, 2048 of them: 240 and 237).
template <typename T, int DKP, bool SAVE>
__global__ __launch_bounds__(256) void k_delta_pack(DeltaArgs p)
{
    using G = Pack<T, DKP>;
    constexpr int C = G::C, NI = G::NI, RT = G::RT, LD = C + 4;
    struct Work {
        float A[C][LD], P[C][LD], inv[C][LD];
    };
    union Tiles {
        char units[G::key_units(SAVE) * UNIT];
        Work w;
    };
    __shared__ __align__(16) Tiles m;
    __shared__ Decays<C> d;
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, col = lane & 15, x4 = lane >> 4;
    const int h0 = (int)(blockIdx.x % (p.hv / p.pack_heads)) * p.pack_heads, hk = h0 / (p.hv / p.hk);  // the first value head of this block, their key head
    const bool first = h0 % (p.hv / p.hk) == 0;
    const int64_t slot = blockIdx.x / (p.hv / p.pack_heads);
    if (p.offsets) {  // tokens of no sequence: zeros
        const int64_t a = p.offsets[0], z = p.offsets[p.batch];
        for (int64_t t = slot * C; t < (slot + 1) * C && t < p.tokens; ++t)
            if (t < a || t >= z)
                for (int c = threadIdx.x; c < p.pack_heads * p.dv; c += 256)
                    ((T *)p.o)[(t * p.hv + h0) * p.dv + c] = (T)0.0f;
    }
    int64_t t0;
    int len;
    if (!slot_chunk<C>(p, slot, t0, len))
        return;
    // 8 x 8 blocks of K and Q: as they are and turned
    constexpr int UC = DKP / 8, UNITS = (C / 8) * UC;
    for (int u = threadIdx.x; u < 2 * UNITS; u += 256) {
        const bool isq = u >= UNITS;
        const int c = (u % UNITS) % UC, r = (u % UNITS) / UC;
        const int64_t ld = isq ? p.ldq : p.ldk;
        const T *src = (const T *)(isq ? p.q : p.k) + (t0 + 8 * r) * ld + (int64_t)hk * p.dk + 8 * c;
        f32x8 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = load8<T>(src + i * ld, 8 * r + i < len ? p.dk - 8 * c : 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {  // token 8 r + i: row 4 (r % 4) + i % 4 of tile 2 (r / 4) + i / 4
            const Frag<NI> f = split<NI>(x[i]);
            char *at = m.units + ((isq ? G::Q : G::K) + G::row(2 * (r >> 2) + (i >> 2), c >> 2)) * UNIT + 16 * (16 * (c & 3) + 4 * (r & 3) + (i & 3));
#pragma unroll
            for (int k = 0; k < NI; ++k)
                *reinterpret_cast<bf16x8 *>(at + k * G::FK * UNIT) = f.p[k];
        }
        if (!isq || SAVE) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const Frag<NI> f = split<NI>(f32x8{x[0][j], x[1][j], x[2][j], x[3][j], x[4][j], x[5][j], x[6][j], x[7][j]});
                char *at = m.units + ((isq ? G::QTURN : G::KTURN) + G::turned(2 * (c >> 2) + (j >> 2), r >> 2)) * UNIT +
                           16 * (16 * (r & 3) + 4 * (c & 3) + (j & 3));
#pragma unroll
                for (int k = 0; k < NI; ++k)
                    *reinterpret_cast<bf16x8 *>(at + k * G::FK * UNIT) = f.p[k];
            }
        }
    }
    __syncthreads();
    char *pk = p.pack_k + (slot * p.hk + hk) * (int64_t)G::key_units(SAVE) * UNIT;
    for (int u = first ? wave : G::key_units(SAVE); u < G::key_units(SAVE); u += 4)
        *reinterpret_cast<bf16x8 *>(pk + u * UNIT + 16 * lane) = *reinterpret_cast<const bf16x8 *>(m.units + u * UNIT + 16 * lane);
    // row tile `wave` (of C = 32: tiles 0 and 1 by half of the wavefronts each half of the steps) of K K^T and Q K^T
    constexpr int NT = C == 64 ? RT : 1;  // column tiles of a wavefront
    const int ti = C == 64 ? wave : wave & 1, tj0 = C == 64 ? 0 : wave >> 1;
    f32x4 kk[NT], qk[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        kk[j] = qk[j] = f32x4{0, 0, 0, 0};
        if ((tj0 + j) / 2 <= ti / 2) {
#pragma unroll
            for (int s = 0; s < G::KS; ++s) {
                const Frag<NI> f = unit<NI>(m.units, G::K + G::row(tj0 + j, s), G::FK);
                mma<3>(kk[j], unit<NI>(m.units, G::K + G::row(ti, s), G::FK), f);
                mma<3>(qk[j], unit<NI>(m.units, G::Q + G::row(ti, s), G::FK), f);
            }
        }
    }
    const int i0 = first_of(ti);
    for (int h = h0; h < h0 + p.pack_heads; ++h) {
        __syncthreads();  // the units (or the head before) are read
        if (wave == 0)
            d.load(p.g + t0 * p.hv + h, p.beta + t0 * p.hv + h, p.hv, len);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if ((tj0 + j) / 2 <= ti / 2) {
                const int tj = element_of(tj0 + j, col);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = i0 + r;
                    const float e = d.between(i, tj);
                    m.w.A[i][tj] = tj < i ? d.walk.beta[i] * e * kk[j][r] : 0.0f;
                    m.w.P[i][tj] = tj <= i ? p.scale * e * qk[j][r] : 0.0f;
                }
            }
        }
        __syncthreads();
        char *pv = p.pack_v + (slot * p.hv + h) * (int64_t)G::value_units(SAVE) * UNIT;
        if (wave == 0) {  // the blocks of the diagonal
            const int b0 = 16 * x4;
            if (b0 < C) {
                float t[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float s[2] = {i == col ? 1.0f : 0.0f, 0};
#pragma unroll
                    for (int l = 0; l < i; l += 4) {
                        const f32x4 a = *reinterpret_cast<const f32x4 *>(&m.w.A[b0 + i][b0 + l]);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (l + k < i)
                                s[k & 1] -= a[k] * t[l + k];
                    }
                    t[i] = s[0] + s[1];
                    m.w.inv[b0 + i][b0 + col] = t[i];
                }
            }
        } else {  // the others meanwhile: P^T and the decays out, zeros right of the diagonal
            if constexpr (SAVE) {
                for (int u = wave - 1; u < G::FT; u += 3) {
#pragma unroll
                    for (int i = 0; i < RT; ++i)
#pragma unroll
                        for (int s = 0; s < G::CS; ++s)
                            if (s >= i / 2 && u == G::upper(i, s)) {
                                f32x8 x;
#pragma unroll
                                for (int r = 0; r < 8; ++r)
                                    x[r] = m.w.P[32 * s + 8 * x4 + r][element_of(i, col)];
                                put_unit<NX>(pv, G::PTURN + u, G::FT, x);
                            }
                }
            }
            if (wave < 3)
                *reinterpret_cast<f32x4 *>(pv + (wave - 1) * UNIT + 16 * lane) = *reinterpret_cast<const f32x4 *>((const char *)&d + (wave - 1) * UNIT + 16 * lane);
            else
                for (int b = 0; b < C; b += 32)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        m.w.inv[b + 4 * x4 + r][b + 16 + col] = 0.0f;
        }
        __syncthreads();
        if (wave < C / 32) {
            const int b = 32 * wave;
            f32x4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < 4; ++k)
                x = __builtin_amdgcn_mfma_f32_16x16x4f32(m.w.A[b + 16 + col][b + 4 * k + x4], m.w.inv[b + 4 * k + x4][b + col], x, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                y = __builtin_amdgcn_mfma_f32_16x16x4f32(m.w.inv[b + 16 + col][b + 16 + 4 * x4 + r], x[r], y, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                m.w.inv[b + 16 + 4 * x4 + r][b + col] = -y[r];
        }
        if constexpr (C == 64) {
            __syncthreads();
            const int a1 = wave >> 1, b = 16 * (wave & 1);  // block row of T22, block column of T11
            f32x4 y = {0, 0, 0, 0};
#pragma unroll
            for (int a = 0; a < 2; ++a)
                if (a <= a1) {
                    f32x4 x = {0, 0, 0, 0};
#pragma unroll
                    for (int k = 0; k < 8; ++k)  // (the upper right block of T11 is zero)
                        x = __builtin_amdgcn_mfma_f32_16x16x4f32(m.w.A[32 + 16 * a + col][4 * k + x4], m.w.inv[4 * k + x4][b + col], x, 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        y = __builtin_amdgcn_mfma_f32_16x16x4f32(m.w.inv[32 + 16 * a1 + col][32 + 16 * a + 4 * x4 + r], x[r], y, 0, 0, 0);
                }
#pragma unroll
            for (int r = 0; r < 4; ++r)
                m.w.inv[32 + 16 * a1 + 4 * x4 + r][b + col] = -y[r];
        }
        __syncthreads();
        // P T over A, which is not needed any more: the wavefront's row of 16 x 16 blocks
        if (wave < C / 16) {
#pragma unroll
            for (int j = 0; j < C / 16; ++j) {
                f32x4 x = {0, 0, 0, 0};
                if (j <= wave) {
                    for (int k = j; k <= wave; ++k)
#pragma unroll
                        for (int l = 0; l < 4; ++l)
                            x = __builtin_amdgcn_mfma_f32_16x16x4f32(m.w.P[16 * wave + col][16 * k + 4 * l + x4], m.w.inv[16 * k + 4 * l + x4][16 * j + col], x, 0, 0, 0);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    m.w.A[16 * wave + 4 * x4 + r][16 * j + col] = x[r];
            }
        }
        __syncthreads();
        for (int u = wave; u < (SAVE ? 3 : 2) * G::FT; u += 4) {
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int s = 0; s < G::CS; ++s) {
                    const float *row = &m.w.inv[element_of(i, col)][32 * s + 8 * x4];
                    const float *prow = &m.w.A[element_of(i, col)][32 * s + 8 * x4];
                    if (s <= i / 2 && u == G::lower(i, s))
                        put_unit<NX>(pv, G::TINV + u, G::FT, join(*reinterpret_cast<const f32x4 *>(row), *reinterpret_cast<const f32x4 *>(row + 4)));
                    if (s <= i / 2 && u == G::FT + G::lower(i, s))
                        put_unit<G::NO>(pv, G::P + u - G::FT, G::FT, join(*reinterpret_cast<const f32x4 *>(prow), *reinterpret_cast<const f32x4 *>(prow + 4)));
                    if (SAVE && s >= i / 2 && u == 2 * G::FT + G::upper(i, s)) {
                        f32x8 x;
#pragma unroll
                        for (int r = 0; r < 8; ++r)
                            x[r] = m.w.inv[32 * s + 8 * x4 + r][element_of(i, col)];
                        put_unit<NX>(pv, G::TTURN + u - 2 * G::FT, G::FT, x);
                    }
                }
        }
    }
}

// ---------------------------------------------------------------------------------
// the walk over a sequence's chunks
// ---------------------------------------------------------------------------------
// A block takes NG groups of 16 columns of V, two wavefronts each.  A wavefront sums K S and Q S over its half of the state's rows, for all tokens, takes
// the other half's sums for its half of the tokens, forms Z, U and the answers of those, and with everybody's U its half of the new state.  The packets of
// the next chunk come straight to LDS, into the place of this one's as soon as all have read them.
// Bound by the chain of chunks: 2 x 4096 tokens, 32 heads of 128, bf16, everything kept: 312 us, 64 chunks of 4.9 us with a block on every compute unit.  A wavefront's
// 200 matrix instructions of a chunk are a quarter of that, the rest is splitting into pieces, the exchange and waiting with one wavefront a SIMD.
//
// Where sequences and heads are too few to fill the chip, a sequence is walked in segments side by side.  The state after a segment is M S + N with S the state
// before it: MAP blocks find N (the walk from a state of zeros) and the columns of M (from the unit vectors, with V zero), without answers;
// k_delta_join goes from segment to segment; then every segment is walked from its own state (8192 tokens, 16 heads of 128, bf16: 113, 22 and 80 us).
template <typename T, int DKP, int NG, bool SAVE, bool MAP>
__global__ __launch_bounds__(128 * NG) void k_delta_scan(DeltaArgs p)
{
    using G = Pack<T, DKP>;
    constexpr int C = G::C, NI = G::NI, RT = G::RT, CS = G::CS, FK = G::FK, FT = G::FT, NL = NG;  // NL wavefronts load the packets: those of the first half, which have less to do with T
    constexpr int HT = RT / 2, HK = G::KT / 2, HS = G::KS / 2;  // a wavefront's tiles of tokens and of the state, steps over the state
    constexpr int LQ = NI * FK, LP = NX * FT;
    constexpr int NKQ = (MAP ? 1 : 2) * NI * FK, NTP = (MAP ? NX : NX + G::NO) * FT;
    constexpr int EACH_KQ = share<NKQ, NL>(), EACH_TP = share<NTP, NL>() + 1, EACH_KT = share<NI * FK, NL>();
    using In = RowsIn<T, C, NG, 128 * NG>;
    constexpr int EX1 = 4 * HT * UNIT > CS * NX * UNIT ? 4 * HT * UNIT : CS * NX * UNIT;                                // a group's sums; then its U
    constexpr int EX2 = CS * NX * UNIT > 2 * rows_out_bytes<HT>() ? CS * NX * UNIT : 2 * rows_out_bytes<HT>();  // a group's Z; then rows on their way out
    __shared__ __align__(16) char kq[NKQ * UNIT];
    __shared__ __align__(16) char tp[NTP * UNIT];
    __shared__ __align__(16) char decays[2][UNIT];
    __shared__ __align__(16) char turned[NI * FK * UNIT];
    __shared__ __align__(16) char vin[C * 16 * NG * sizeof(T)];
    __shared__ __align__(16) char ex1_all[NG][EX1], ex2_all[NG][EX2];
    static_assert(!G::PAIRED || (NG == 2 && 2 * (sizeof(kq) + sizeof(tp) + sizeof(decays) + sizeof(turned) + sizeof(vin) + sizeof(ex1_all) + sizeof(ex2_all)) <= LDS_BYTES));
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, col = lane & 15;
    const int half = wave / NG, set = wave % NG;
    const unsigned block = block_of_die(p.slices);
    const int slice = block % p.slices, h = block / p.slices % p.hv;
    const int64_t sg = block / p.slices / p.hv, n = p.seg ? segment_sequence<C>(p, sg) : sg;
    const int vslices = (p.dv + 16 * NG - 1) / (16 * NG);
    const bool unit_columns = MAP && slice >= vslices;
    const int sbase = (unit_columns ? slice - vslices : slice) * 16 * NG, cbase = sbase + set * 16, c0 = cbase + col;  // this lane's column of V (or of M)
    const int width = unit_columns ? p.dk : p.dv;
    const bool live = c0 < width, kept = cbase < p.dvp;
    int64_t t0, len;
    sequence(p, n, t0, len);
    const int hk = h / (p.hv / p.hk);
    const int64_t state_at = (n * p.hv + h) * p.dk * (int64_t)p.dv;
    int64_t slot0 = first_slot<C>(p, n, t0);
    int chunks = (int)((len + C - 1) / C), part = 0;
    bool last = true;
    if (p.seg) {  // chunks seg part .. of the sequence
        part = (int)(sg - first_segment<C>(p, n, t0));
        const int from = part * p.seg;
        if (part < 0 || (part > 0 && from >= chunks))
            return;
        last = from + p.seg >= chunks;
        if (MAP && (last || (part == 0 && unit_columns)))  // (nobody asks for those)
            return;
        chunks = last ? chunks - from : p.seg;
        slot0 += from;
        t0 += (int64_t)from * C;
        len -= (int64_t)from * C;
        len = last ? len : (int64_t)chunks * C;
    }
    const char *pk = p.pack_k + (slot0 * p.hk + hk) * (int64_t)(G::key_units(SAVE) * UNIT), *pv = p.pack_v + (slot0 * p.hv + h) * (int64_t)(G::value_units(SAVE) * UNIT);
    const int64_t key_step = (int64_t)p.hk * (G::key_units(SAVE) * UNIT), value_step = (int64_t)p.hv * (G::value_units(SAVE) * UNIT);
    const uint32_t kq_at = lds_address(kq), tp_at = lds_address(tp), turned_at = lds_address(turned), decays_at = lds_address(decays);
    auto fetch_kq = [&](const char *k) { stream_run<NKQ, NL>(k, kq_at, set); };
    auto fetch_tp = [&](const char *v, int buffer) {
        stream_run<NTP, NL>(v + G::TINV * UNIT, tp_at, set);
        stream_units<1>(v + UNIT, decays_at + buffer * UNIT);  // (by each of them)
    };
    char *ex1 = ex1_all[set], *ex2 = ex2_all[set], *mine = ex2 + half * rows_out_bytes<HT>();
    In V;
    auto fetch_v = [&](int c) {
        V.fetch((const T *)p.v + (t0 + (int64_t)c * C) * p.ldv + (int64_t)h * p.dv + sbase, p.ldv, (int)(len - (int64_t)c * C < C ? len - (int64_t)c * C : C),
                unit_columns ? 0 : p.dv - sbase);
    };
    // rows 16 HT i .. of this wavefront's half of the state
    auto keep_state = [&](int c, const f32x4 *S) {
        if (kept) {
            float *dst = p.chunk_state + (((slot0 + c) * p.hv + h) * DKP + half * (DKP / 2)) * (int64_t)p.dvp + cbase;
            constexpr int N = HT > 1 ? HT : 1;
            if constexpr (N == 1) {
#pragma unroll
                for (int i = 0; i < HK; ++i)
                    RowsOut<float, 1>::store(mine, dst + (int64_t)(i >> 1) * 32 * p.dvp, p.dvp, S + i, 32, 16, i & 1);
            } else {
#pragma unroll
                for (int i = 0; i < HK / 2; ++i)
                    RowsOut<float, 2>::store(mine, dst + (int64_t)i * 32 * p.dvp, p.dvp, S + 2 * i, 32, 16);
            }
        }
    };

    if (half)  // what the others wait for
        __builtin_amdgcn_s_setprio(1);
    f32x4 S[HK];
#pragma unroll
    for (int t = 0; t < HK; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = first_of(half * HK + t) + r;
            if (part == 0 && (MAP || last))
                S[t][r] = p.state0 && live && i < p.dk ? in_memory(p.state0)[state_at + (int64_t)i * p.dv + c0] : 0.0f;
            else if (MAP)
                S[t][r] = unit_columns && i == c0 ? 1.0f : 0.0f;
            else
                S[t][r] = kept ? in_memory(p.seg_state)[((sg * p.hv + h) * DKP + i) * p.dvp + c0] : 0.0f;
        }
    // What the first of several segments is walked from later: by then the last one may have written its state over the initial one's, in place.
    if (MAP && part == 0 && kept) {
        float *to = p.seg_state + (sg * p.hv + h) * DKP * (int64_t)p.dvp;
#pragma unroll
        for (int t = 0; t < HK; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                in_memory(to)[(int64_t)(first_of(half * HK + t) + r) * p.dvp + c0] = S[t][r];
    }
    if (chunks > 0) {
        if (!half) {
            fetch_kq(pk);
            fetch_tp(pv, 0);
        }
        fetch_v(0);
        if constexpr (SAVE && !MAP)
            keep_state(0, S);
        V.put(vin);
        wait_loads<0>();
    }
    for (int c = 0; c < chunks; ++c, pk += key_step, pv += value_step) {
        const bool more = c + 1 < chunks;
        block_barrier();  // K, Q and V are there, all have read what the chunk before left
        if (!half)
            stream_run<NI * FK, NL>(pk + G::KTURN * UNIT, turned_at, set);
        f32x4 X[RT], Y[RT], U[HT], in[HT], out[HT], beta[HT];
#pragma unroll
        for (int i = 0; i < RT; ++i)
            X[i] = Y[i] = f32x4{0, 0, 0, 0};
        Frag<NI> kf[2][RT], qf[2][RT];
        auto rows_of = [&](int s, Frag<NI> *k, Frag<NI> *q) {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                k[i] = unit<NI>(kq, G::row(i, s), FK);
                if constexpr (!MAP)
                    q[i] = unit<NI>(kq, LQ + G::row(i, s), FK);
            }
        };
        rows_of(half * HS, kf[0], qf[0]);
        issue_point();
        Frag<NX> f = split<NX>(join(S[0], S[1]));
#pragma unroll
        for (int s = 0; s < HS; ++s) {
            if (s + 1 < HS)
                rows_of(half * HS + s + 1, kf[~s & 1], qf[~s & 1]);
            issue_point();
            const Frag<NX> now = f;
            if (s + 1 < HS)
                f = split<NX>(join(S[2 * s + 2], S[2 * s + 3]));
            mma_tiles<3, RT>(X, kf[s & 1], now);
            if constexpr (!MAP)
                mma_tiles<G::NO, RT>(Y, qf[s & 1], now);
        }
        // the other half's tokens' sums to the other wavefront; its own sums of this half's
#pragma unroll
        for (int j = 0; j < HT; ++j) {
            *reinterpret_cast<f32x4 *>(ex1 + ((2 * half + 0) * HT + j) * UNIT + 16 * lane) = half ? X[j] : X[HT + j];
            if constexpr (!MAP)
                *reinterpret_cast<f32x4 *>(ex1 + ((2 * half + 1) * HT + j) * UNIT + 16 * lane) = half ? Y[j] : Y[HT + j];
        }
        if (!half)
            wait_loads<EACH_KT>();
        block_barrier();  // (1) sums, T, P T and the decays are there; K and Q are read
        if (more) {
            fetch_v(c + 1);
            if (!half)
                fetch_kq(pk + key_step);
        }
        const Walk<C> &d = *reinterpret_cast<const Walk<C> *>(decays[c & 1]);
        f32x4 Z[HT], O[HT];
        Frag<NX> tf[HT][CS];
        Frag<G::NO> pf[HT][CS];
#pragma unroll
        for (int j = 0; j < HT; ++j) {
            const int i = half * HT + j, first = first_of(i);
            in[j] = d.four(d.in, first);
            out[j] = d.four(d.out, first);
            beta[j] = d.four(d.beta, first);
            X[j] = (half ? X[HT + j] : X[j]) + *reinterpret_cast<const f32x4 *>(ex1 + ((2 * (1 - half) + 0) * HT + j) * UNIT + 16 * lane);
            if constexpr (!MAP)
                Y[j] = (half ? Y[HT + j] : Y[j]) + *reinterpret_cast<const f32x4 *>(ex1 + ((2 * (1 - half) + 1) * HT + j) * UNIT + 16 * lane);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                Z[j][r] = In::at(vin, first + r, 16 * set + col);
        }
#pragma unroll
        for (int j = 0; j < HT; ++j)
#pragma unroll
            for (int s = 0; s < CS; ++s)
                if (CS == 1 || s == 0 || half) {
                    const int u = CS == 1 ? half * HT + j : half ? G::lower(2 + j, s) : j;
                    tf[j][s] = unit<NX>(tp, u, FT);
                    if constexpr (!MAP)
                        pf[j][s] = unit<G::NO>(tp, LP + u, FT);
                }
        const float all = d.all;
#pragma unroll
        for (int j = 0; j < HT; ++j) {
            Z[j] = beta[j] * (Z[j] - in[j] * X[j]);
            O[j] = p.scale * in[j] * Y[j];
            U[j] = f32x4{0, 0, 0, 0};
        }
        put_step<RT>(ex2, half, Z);
#pragma unroll
        for (int i = 0; i < HK; ++i)
            S[i] *= all;
        block_barrier();  // (2) Z is there, the sums are read
        auto token_products = [&](int s) {
            const Frag<NX> z = unit<NX>(ex2, s * NX, 1);
#pragma unroll
            for (int j = 0; j < HT; ++j) {
                mma<3>(U[j], tf[j][s], z);
                if constexpr (!MAP)
                    mma<G::NO>(O[j], pf[j][s], z);
            }
        };
        token_products(0);
        if constexpr (CS > 1)
            if (half)
                token_products(1);
        f32x4 W[HT];
#pragma unroll
        for (int j = 0; j < HT; ++j)
            W[j] = out[j] * U[j];
        put_step<RT>(ex1, half, W);
        if (!half) {
            if (more)
                wait_loads<EACH_KQ>();
            else
                wait_loads<0>();
        }
        block_barrier();  // (3) U and Kt are there; T, P T, V and Z are read
        if (more && !half)
            fetch_tp(pv + value_step, ~c & 1);
        Frag<NI> ktf[CS][HK];
        Frag<NX> w[CS];
#pragma unroll
        for (int s = 0; s < CS; ++s) {
            w[s] = unit<NX>(ex1, s * NX, 1);
#pragma unroll
            for (int i = 0; i < HK; ++i)
                ktf[s][i] = unit<NI>(turned, G::turned(half * HK + i, s), FK);
        }
        issue_point();
#pragma unroll
        for (int s = 0; s < CS; ++s)
            mma_tiles<3, HK>(S, ktf[s], w[s]);
        if (more) {
            if (!half)
                wait_loads<EACH_TP>();  // (before the stores: the next chunk does not wait for them)
            V.put(vin);
        }
        if constexpr (!MAP) {
            const int64_t t = t0 + (int64_t)c * C + (HT > 1 ? 32 * half : 0);
            const int64_t left = len - (int64_t)c * C - (HT > 1 ? 32 * half : 0);
            const int rows = (int)(left < 0 ? 0 : left < 32 ? left : 32);
            RowsOut<T, HT>::store(mine, (T *)p.o + (t * p.hv + h) * p.dv + cbase, (int64_t)p.hv * p.dv, O, rows, p.dv - cbase, half);
        }
        if constexpr (SAVE && !MAP) {
            if (kept)
                RowsOut<float, HT>::store(mine, p.chunk_u + (((slot0 + c) * p.hv + h) * C + (HT > 1 ? 32 * half : 0)) * (int64_t)p.dvp + cbase, p.dvp, U, 32, 16, half);
            if (more)
                keep_state(c + 1, S);
        }
    }
    if constexpr (MAP) {  // N to where the next segment's state will be, or M
        float *to = unit_columns ? p.seg_map + (sg * p.hv + h) * DKP * (int64_t)DKP : p.seg_state + ((sg + 1) * p.hv + h) * DKP * (int64_t)p.dvp;
        const int ld = unit_columns ? DKP : p.dvp;
        if (cbase < ld) {
#pragma unroll
            for (int t = 0; t < HK; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    in_memory(to)[(int64_t)(first_of(half * HK + t) + r) * ld + c0] = S[t][r];
        }
        return;
    }
    if (p.state1 && live && last) {
#pragma unroll
        for (int t = 0; t < HK; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = first_of(half * HK + t) + r;
                if (i < p.dk)
                    in_memory(p.state1)[state_at + (int64_t)i * p.dv + c0] = S[t][r];
            }
    }
}

// From the state before a segment to the one after it, M S + N, over a sequence's segments: 16 columns of one head a block, 32 rows of the state a wavefront, its rows of
// M loaded a segment ahead.  A chain of small products: 22 us over 8 segments of 16 heads of 128.
template <int C, int DKP>
__global__ __launch_bounds__(2 * DKP) void k_delta_join(DeltaArgs p)
{
    constexpr int KS = DKP / 32;
    __shared__ __align__(16) char state[2][KS * NX * UNIT];
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, col = lane & 15, x4 = lane >> 4, slices = p.dvp / 16;
    const int c0 = (int)(blockIdx.x % slices) * 16 + col, h = blockIdx.x / slices % p.hv;
    const int64_t n = blockIdx.x / slices / p.hv;
    int64_t t0, len;
    sequence(p, n, t0, len);
    const int64_t sg = first_segment<C>(p, n, t0);
    const int parts = (int)((len + (int64_t)C * p.seg - 1) / ((int64_t)C * p.seg));
    if (parts < 3)
        return;  // (the state before segment 1 is there)
    f32x4 S[2], N[2];
    f32x8 m[2][KS];
    auto at = [&](int64_t g) { return p.seg_state + ((g * p.hv + h) * DKP) * (int64_t)p.dvp + c0; };
    auto rows_of = [&](int64_t g, f32x4 *x) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                x[i][r] = in_memory(at(g))[(int64_t)(first_of(2 * wave + i) + r) * p.dvp];
    };
    // M's columns are there up to dk, by the 32: rows of the state past dk are zero, and what the workspace holds in their columns of M may be NaN.
    auto map_of = [&](int64_t g) {
        const float *M = p.seg_map + (g * p.hv + h) * DKP * (int64_t)DKP;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int s = 0; s < KS; ++s)
                m[i][s] = 32 * s < p.dk ? load8<float>(M + element_of(2 * wave + i, col) * DKP + 32 * s + 8 * x4, 8) : f32x8{0, 0, 0, 0, 0, 0, 0, 0};
    };
    rows_of(sg + 1, S);
    map_of(sg + 1);
    rows_of(sg + 2, N);
    for (int g = 1; g + 1 < parts; ++g) {
        char *buf = state[g & 1];
        const Frag<NX> own = split<NX>(join(S[0], S[1]));
#pragma unroll
        for (int i = 0; i < NX; ++i)
            *reinterpret_cast<bf16x8 *>(buf + (wave * NX + i) * UNIT + 16 * lane) = own.p[i];
        Frag<NX> f[2][KS];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            S[i] = N[i];
#pragma unroll
            for (int s = 0; s < KS; ++s)
                f[i][s] = split<NX>(m[i][s]);
        }
        if (g + 2 < parts) {
            map_of(sg + g + 1);
            rows_of(sg + g + 2, N);
        }
        block_barrier();
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const Frag<NX> x = unit<NX>(buf, s * NX, 1);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                mma<3>(S[i], f[i][s], x);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                in_memory(at(sg + g + 1))[(int64_t)(first_of(2 * wave + i) + r) * p.dvp] = S[i][r];
    }
}

template <typename T, int DKP, int NG, bool SAVE>
static void walk(DeltaArgs &p, hipStream_t st)
{
    const int vslices = (p.dv + 16 * NG - 1) / (16 * NG);
    if (p.seg) {
        p.slices = vslices + (p.dk + 16 * NG - 1) / (16 * NG);
        LA_LAUNCH((k_delta_scan<T, DKP, NG, SAVE, true>), dim3((unsigned)(p.segs * p.hv * p.slices)), dim3(128 * NG), 0, st, p);
        LA_LAUNCH((k_delta_join<Pack<T, DKP>::C, DKP>), dim3((unsigned)(p.batch * p.hv * (p.dvp / 16))), dim3(2 * DKP), 0, st, p);
    }
    p.slices = vslices;
    LA_LAUNCH((k_delta_scan<T, DKP, NG, SAVE, false>), dim3((unsigned)((p.seg ? p.segs : p.batch) * p.hv * p.slices)), dim3(128 * NG), 0, st, p);
}

template <typename T, int DKP, bool SAVE>
static la_status scan_s(DeltaArgs &p, hipStream_t st)
{
    using G = Pack<T, DKP>;
    p.pack_heads = p.slots * p.hv <= 2 * COMPUTE_UNITS ? 1 : p.hv / p.hk;
    const int groups = G::PAIRED || walk_groups((p.seg ? p.segs : p.batch) * p.hv, p.dv) == 2 ? 2 : 4;
    // (segments are for few heads: their launches are small)
    if (p.slots * (p.hv / p.pack_heads) > most_blocks(256) || p.batch * p.hv * ((p.dv + 16 * groups - 1) / (16 * groups)) > most_blocks(128 * groups))
        return LA_ERR_UNSUPPORTED;
    if (p.slots > 0)
        LA_LAUNCH((k_delta_pack<T, DKP, SAVE>), dim3((unsigned)(p.slots * (p.hv / p.pack_heads))), dim3(256), 0, st, p);
    if (groups == 2)
        walk<T, DKP, 2, SAVE>(p, st);
    else if constexpr (!G::PAIRED)
        walk<T, DKP, 4, SAVE>(p, st);
    return launch_check("delta rule");
}
template <typename T, int DKP>
static la_status scan_t(DeltaArgs &p, bool save, hipStream_t st)
{
    return save ? scan_s<T, DKP, true>(p, st) : scan_s<T, DKP, false>(p, st);
}

la_status launch_delta_rule(la_dtype dt, DeltaArgs p, bool save, hipStream_t st)
{
    const bool half = p.dk <= 64;
    switch (dt) {
    case LA_F32: return half ? scan_t<float, 64>(p, save, st) : scan_t<float, 128>(p, save, st);
    case LA_BF16: return half ? scan_t<bf16_t, 64>(p, save, st) : scan_t<bf16_t, 128>(p, save, st);
    default: return half ? scan_t<f16_t, 64>(p, save, st) : scan_t<f16_t, 128>(p, save, st);
    }
}

// ---------------------------------------------------------------------------------
// one token of every sequence
// ---------------------------------------------------------------------------------
// With s = S^T k and y = S^T q from one read of the state, the new state is a S + k u^T and the answer scale (a y + (q.k) u): the state is read and written
// once, which is what bounds the call (128 sequences, 32 heads of 128 x 128, bf16: 540 MB, 96 us for the kernel by itself, 115 us a call among others, 4.7 TB/s
// where a copy reaches 5.1; one sequence: 4.5 us, a launch and one round trip).  A block takes 32 columns of one state, its lanes packs of VEC columns by rows; all loads of a lane are in
// flight at once.
struct DeltaStepArgs {
    const void *q, *k, *v;
    int64_t ldq, ldk, ldv;
    const float *g, *beta;
    float *state;
    const int32_t *slot;
    int64_t slots;
    int hk, hv, dk, dv, slices;
    float scale;
    void *o;
};

template <typename T>
__global__ __launch_bounds__(256) void k_delta_step(DeltaStepArgs p)
{
    constexpr int VEC = 4, LC = 32 / VEC, RR = 256 / LC, RI = 128 / RR;
    __shared__ float box[4][2][32];
    __shared__ float kq_box[4];
    const int slice = blockIdx.x % p.slices, h = blockIdx.x / p.slices % p.hv;
    const int64_t n = blockIdx.x / p.slices / p.hv;
    const int c = slice * 32 + VEC * (threadIdx.x % LC), r0 = threadIdx.x / LC, wave = threadIdx.x / 64;
    const int left = p.dv - c;  // columns from this lane's first on
    const int hk = h / (p.hv / p.hk);
    const int64_t at = p.slot ? p.slot[n] : n;
    T *o = (T *)p.o + (n * p.hv + h) * p.dv + c;
    if (at < 0 || at >= p.slots) {  // no state of its own: nothing is updated
        const float none[VEC] = {};
        if (r0 == 0)
            store_part<T, VEC>(o, left, none);
        return;
    }
    const T *q = (const T *)p.q + n * p.ldq + (int64_t)hk * p.dk, *k = (const T *)p.k + n * p.ldk + (int64_t)hk * p.dk;
    float *S = p.state + (at * p.hv + h) * p.dk * (int64_t)p.dv + c;
    float x[RI][VEC], kr[RI], qr[RI], v[VEC];
#pragma unroll
    for (int i = 0; i < RI; ++i) {
        const int r = r0 + RR * i;
        load_part<float, VEC>(S + (int64_t)r * p.dv, r < p.dk ? left : 0, x[i]);
        kr[i] = r < p.dk ? (float)k[r] : 0.0f;
        qr[i] = r < p.dk ? (float)q[r] : 0.0f;
    }
    load_part<T, VEC>((const T *)p.v + n * p.ldv + (int64_t)h * p.dv + c, left, v);
    const float a = expf(p.g[n * p.hv + h]), beta = p.beta[n * p.hv + h];
    float ks[VEC] = {}, qs[VEC] = {}, kq = 0;
#pragma unroll
    for (int i = 0; i < RI; ++i) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            ks[j] += kr[i] * x[i][j];
            qs[j] += qr[i] * x[i][j];
        }
        kq += kr[i] * qr[i];
    }
#pragma unroll
    for (int m = LC; m < 64; m *= 2) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            ks[j] += __shfl_xor(ks[j], m, 64);
            qs[j] += __shfl_xor(qs[j], m, 64);
        }
        kq += __shfl_xor(kq, m, 64);
    }
    const int mine = VEC * (threadIdx.x % LC);
    if (threadIdx.x % 64 < LC) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            box[wave][0][mine + j] = ks[j];
            box[wave][1][mine + j] = qs[j];
        }
        kq_box[wave] = kq;
    }
    __syncthreads();
    kq = kq_box[0] + kq_box[1] + kq_box[2] + kq_box[3];
    float u[VEC], y[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        const float s = box[0][0][mine + j] + box[1][0][mine + j] + box[2][0][mine + j] + box[3][0][mine + j];
        const float t = box[0][1][mine + j] + box[1][1][mine + j] + box[2][1][mine + j] + box[3][1][mine + j];
        u[j] = beta * (v[j] - a * s);
        y[j] = p.scale * (a * t + kq * u[j]);
    }
    if (r0 == 0)
        store_part<T, VEC>(o, left, y);
#pragma unroll
    for (int i = 0; i < RI; ++i) {
        const int r = r0 + RR * i;
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            x[i][j] = a * x[i][j] + kr[i] * u[j];
        store_part<float, VEC>(S + (int64_t)r * p.dv, r < p.dk ? left : 0, x[i]);
    }
}

template <typename T>
static la_status step_t(DeltaStepArgs &p, int64_t batch, hipStream_t st)
{
    p.slices = (p.dv + 31) / 32;
    LA_LAUNCH((k_delta_step<T>), dim3((unsigned)(batch * p.hv * p.slices)), dim3(256), 0, st, p);
    return launch_check("delta rule step");
}

// ---------------------------------------------------------------------------------
// sizes and buffers
// ---------------------------------------------------------------------------------
constexpr int DELTA_MAX_DK = 128, DELTA_MAX_DV = 1024;
constexpr int64_t DELTA_MAX_ROW = 1 << 24;  // elements of one token's row of v

struct DeltaSizes {
    int64_t slots = 0, all = 0;  // chunks, tokens of all sequences
    int c = 0, dkp = 0, dvp = 0;
    size_t key[2] = {}, value[2] = {};  // bytes of the packets, without and with what the gradient takes
    size_t state = 0, u = 0;            // of the states and of U by slot and value head
    int seg = 0;                        // chunks of a segment, 0 where sequences are walked whole
    int64_t segs = 0;
    size_t seg_state = 0, seg_map = 0;
    size_t packets(bool save) const { return key[save] + value[save] + seg_state + seg_map; }
    size_t saved() const { return packets(true) + state + u; }
    size_t grad() const { return state + u; }  // the state's gradient, Z's gradient
};

template <typename T, int DKP>
static void packet_sizes(DeltaSizes &z, bool packed, int64_t batch, int64_t tokens, int hk, int hv)
{
    using G = Pack<T, DKP>;
    z.c = G::C;
    z.dkp = DKP;
    z.slots = batch == 0 ? 0 : packed ? tokens / z.c + batch : batch * ((tokens + z.c - 1) / z.c);
    for (int save = 0; save < 2; ++save) {
        z.key[save] = (size_t)z.slots * hk * G::key_units(save) * UNIT;
        z.value[save] = (size_t)z.slots * hv * G::value_units(save) * UNIT;
    }
}

static la_status delta_sizes(la_dtype dt, int64_t batch, int64_t tokens, int hk, int hv, int dk, int dv, bool packed, DeltaSizes &z)
{
    if (unknown_dtype(dt) || batch < 0 || tokens < 0 || hk < 1 || hv < 1 || dk < 1 || dv < 1 || hv % hk)
        return LA_ERR_INVALID_ARG;
    if (dt == LA_F64 || dk > DELTA_MAX_DK || dv > DELTA_MAX_DV)
        return LA_ERR_UNSUPPORTED;
    constexpr int64_t most = 0x7fffffff;
    if (batch > most || tokens > most || (!packed && batch && tokens > most / batch))
        return LA_ERR_UNSUPPORTED;
    const bool half = dk <= 64;
    if (dt == LA_F32)
        half ? packet_sizes<float, 64>(z, packed, batch, tokens, hk, hv) : packet_sizes<float, 128>(z, packed, batch, tokens, hk, hv);
    else if (dt == LA_BF16)
        half ? packet_sizes<bf16_t, 64>(z, packed, batch, tokens, hk, hv) : packet_sizes<bf16_t, 128>(z, packed, batch, tokens, hk, hv);
    else
        half ? packet_sizes<f16_t, 64>(z, packed, batch, tokens, hk, hv) : packet_sizes<f16_t, 128>(z, packed, batch, tokens, hk, hv);
    z.dvp = (dv + 31) / 32 * 32;
    z.all = packed ? tokens : batch * tokens;
    if ((int64_t)hv * dv > DELTA_MAX_ROW)  // lanes address 24 rows by 32 bits
        return LA_ERR_UNSUPPORTED;
    if (z.slots > most / hv || batch > most / hv / ((dv + 15) / 16))  // blocks of one launch
        return LA_ERR_UNSUPPORTED;
    const size_t heads = (size_t)z.slots * hv;
    // Segments where whole sequences would leave three quarters of the compute units idle, as many as fill them, of 8 chunks at least and up to 8 of a
    // sequence of the average length: a sequence of g segments takes the time of about 2 / g of it (heads of 128, bf16, in us with and without: 8192 tokens,
    // 16 heads 250 and 540, 32 heads 530 and 583, 40 heads, which make three segments, 685 and 620; 16 heads, 24 chunks 81 and 99, 16 chunks 71 and 66; of 128
    // chunks of f16 and f32, 16 heads 208 and 347, 244 and 419, 32 heads 376 and 420, 469 and 514; of 24 chunks, 16 heads 70 and 76, 73 and 82; 32 heads of 32
    // chunks are the exception, bf16 140 and 133, f16 116 and 106, f32 125 and 116).  A long sequence among short ones, whose average is below 24, is walked whole.
    const int64_t blocks = batch * hv * ((dv + 63) / 64);
    if (blocks > 0 && blocks * 4 <= COMPUTE_UNITS) {
        const int64_t each = (z.all / batch + z.c - 1) / z.c, most_parts = COMPUTE_UNITS / blocks < 8 ? COMPUTE_UNITS / blocks : 8;
        const int64_t seg = (each + most_parts - 1) / most_parts;
        if (each >= 24) {
            z.seg = (int)(seg < 8 ? 8 : seg);
            z.segs = packed ? z.slots / z.seg + batch : batch * ((each + z.seg - 1) / z.seg);
            z.seg_state = align_up((size_t)(z.segs + 1) * hv * z.dkp * z.dvp * 4);
            z.seg_map = align_up((size_t)z.segs * hv * z.dkp * z.dkp * 4);
        }
    }
    z.state = align_up(heads * z.dkp * z.dvp * 4);
    z.u = align_up(heads * z.c * z.dvp * 4);
    return LA_OK;
}

static void place_packets(DeltaArgs &p, const DeltaSizes &z, void *base, bool save)
{
    p.pack_k = (char *)base;
    p.pack_v = p.pack_k + z.key[save];
    p.seg = z.seg;
    p.segs = z.segs;
    p.seg_state = (float *)(p.pack_v + z.value[save]);
    p.seg_map = (float *)((char *)p.seg_state + z.seg_state);
    if (save) {
        p.chunk_state = (float *)((char *)p.seg_map + z.seg_map);
        p.chunk_u = (float *)((char *)p.chunk_state + z.state);
    }
}

la_status launch_delta_backward(la_dtype dt, DeltaArgs p, hipStream_t st);

}  // namespace la

using namespace la;

extern "C" {

size_t la_delta_rule_workspace_bytes(la_dtype dt, int64_t batch, int64_t tokens, int hk, int hv, int dk, int dv, int packed)
{
    DeltaSizes z;
    return delta_sizes(dt, batch, tokens, hk, hv, dk, dv, packed, z) == LA_OK ? z.packets(false) : 0;
}

size_t la_delta_rule_saved_bytes(la_dtype dt, int64_t batch, int64_t tokens, int hk, int hv, int dk, int dv, int packed)
{
    DeltaSizes z;
    return delta_sizes(dt, batch, tokens, hk, hv, dk, dv, packed, z) == LA_OK ? z.saved() : 0;
}

size_t la_delta_rule_backward_workspace_bytes(la_dtype dt, int64_t batch, int64_t tokens, int hk, int hv, int dk, int dv, int packed, int with_saved)
{
    DeltaSizes z;
    return delta_sizes(dt, batch, tokens, hk, hv, dk, dv, packed, z) == LA_OK ? z.grad() + (with_saved ? 0 : z.saved() + align_up((size_t)z.all * hv * dv * bytes_of(dt))) : 0;
}

la_status la_delta_rule(la_dtype dt, int64_t batch, int64_t tokens, int hk, int hv, int dk, int dv, const int32_t *offsets, const void *q, int64_t ldq,
                        const void *k, int64_t ldk, const void *v, int64_t ldv, const float *g, const float *beta, double scale,
                        const float *initial_state, void *o, float *state, void *saved, size_t saved_bytes, void *workspace, size_t workspace_bytes,
                        void *stream)
{
    DeltaSizes z;
    LA_TRY(delta_sizes(dt, batch, tokens, hk, hv, dk, dv, offsets != nullptr, z));
    if (batch == 0)
        return offsets && z.all ? LA_ERR_INVALID_ARG : LA_OK;
    if (ldq < (int64_t)hk * dk || ldk < (int64_t)hk * dk || ldv < (int64_t)hv * dv)
        return LA_ERR_INVALID_ARG;
    if (ldv > DELTA_MAX_ROW)
        return LA_ERR_UNSUPPORTED;
    const size_t es = bytes_of(dt), ob = (size_t)z.all * hv * dv * es, sb = (size_t)batch * hv * dk * dv * 4;
    if (z.all && (!q || !k || !v || !g || !beta || !o))
        return LA_ERR_INVALID_ARG;
    const size_t qs = z.all ? ((size_t)(z.all - 1) * ldq + (size_t)hk * dk) * es : 0, ks = z.all ? ((size_t)(z.all - 1) * ldk + (size_t)hk * dk) * es : 0,
                 vs = z.all ? ((size_t)(z.all - 1) * ldv + (size_t)hv * dv) * es : 0, gs = (size_t)z.all * hv * 4;
    const size_t fs = offsets ? ((size_t)batch + 1) * 4 : 0;
    if (any_overlap({{q, qs}, {k, ks}, {v, vs}, {g, gs}, {beta, gs}, {offsets, fs}}, {{o, ob}, {state, sb}}) || overlaps(o, ob, initial_state, sb) ||
        (state != initial_state && overlaps(state, sb, initial_state, sb)))
        return LA_ERR_INVALID_ARG;
    DeltaArgs p{q, k, v, ldq, ldk, ldv, g, beta, initial_state, offsets, batch, tokens, hk, hv, dk, dv, (float)scale, o, state};
    p.slots = z.slots;
    p.dvp = z.dvp;
    void *base = saved ? saved : workspace;
    const size_t need = saved ? z.saved() : z.packets(false), given = saved ? saved_bytes : workspace_bytes;
    LA_TRY(check_workspace(base, given, need, saved ? "la_delta_rule_saved_bytes" : "la_delta_rule_workspace_bytes"));
    if (any_overlap({{q, qs}, {k, ks}, {v, vs}, {g, gs}, {beta, gs}, {offsets, fs}, {o, ob}, {state, sb}, {initial_state, sb}}, {{base, need}}))
        return LA_ERR_INVALID_ARG;
    place_packets(p, z, base, saved != nullptr);
    return launch_delta_rule(dt, p, saved != nullptr, (hipStream_t)stream);
}

la_status la_delta_rule_backward(la_dtype dt, int64_t batch, int64_t tokens, int hk, int hv, int dk, int dv, const int32_t *offsets, const void *q,
                                 int64_t ldq, const void *k, int64_t ldk, const void *v, int64_t ldv, const float *g, const float *beta, double scale,
                                 const float *initial_state, const void *o_bar, const float *state_bar, const void *saved, size_t saved_bytes,
                                 void *q_bar, void *k_bar, void *v_bar, float *g_bar, float *beta_bar, float *initial_state_bar, void *workspace,
                                 size_t workspace_bytes, void *stream)
{
    DeltaSizes z;
    LA_TRY(delta_sizes(dt, batch, tokens, hk, hv, dk, dv, offsets != nullptr, z));
    if (batch == 0)
        return offsets && z.all ? LA_ERR_INVALID_ARG : LA_OK;
    if (ldq < (int64_t)hk * dk || ldk < (int64_t)hk * dk || ldv < (int64_t)hv * dv)
        return LA_ERR_INVALID_ARG;
    if (ldv > DELTA_MAX_ROW)
        return LA_ERR_UNSUPPORTED;
    if (z.all && (!q || !k || !v || !g || !beta || !o_bar || !q_bar || !k_bar || !v_bar || !g_bar || !beta_bar))
        return LA_ERR_INVALID_ARG;
    const size_t es = bytes_of(dt), ob = (size_t)z.all * hv * dv * es, qb = (size_t)z.all * hk * dk * es, gb = (size_t)z.all * hv * 4,
                 sb = (size_t)batch * hv * dk * dv * 4;
    const size_t qs = z.all ? ((size_t)(z.all - 1) * ldq + (size_t)hk * dk) * es : 0, ks = z.all ? ((size_t)(z.all - 1) * ldk + (size_t)hk * dk) * es : 0,
                 vs = z.all ? ((size_t)(z.all - 1) * ldv + (size_t)hv * dv) * es : 0;
    const size_t fs = offsets ? ((size_t)batch + 1) * 4 : 0;
    const std::initializer_list<Span> in = {{q, qs}, {k, ks}, {v, vs}, {g, gb}, {beta, gb}, {offsets, fs}, {o_bar, ob}, {initial_state, sb}, {state_bar, sb}, {saved, saved_bytes}},
                                      out = {{q_bar, qb}, {k_bar, qb}, {v_bar, ob}, {g_bar, gb}, {beta_bar, gb}, {initial_state_bar, sb}};
    if (any_overlap(in, out))
        return LA_ERR_INVALID_ARG;
    if (saved) {
        LA_TRY(check_workspace(saved, saved_bytes, z.saved(), "la_delta_rule_saved_bytes"));
    }
    const size_t need = la_delta_rule_backward_workspace_bytes(dt, batch, tokens, hk, hv, dk, dv, offsets != nullptr, saved != nullptr);
    LA_TRY(check_workspace(workspace, workspace_bytes, need, "la_delta_rule_backward_workspace_bytes"));
    if (any_overlap(in, {{workspace, need}}) || any_overlap(out, {{workspace, need}}))
        return LA_ERR_INVALID_ARG;
    hipStream_t st = (hipStream_t)stream;
    DeltaArgs p{q, k, v, ldq, ldk, ldv, g, beta, initial_state, offsets, batch, tokens, hk, hv, dk, dv, (float)scale};
    p.slots = z.slots;
    p.dvp = z.dvp;
    char *at = (char *)workspace;
    p.chunk_state_bar = (float *)at;
    p.chunk_z_bar = (float *)(at + z.state);
    at += z.grad();
    if (saved) {
        place_packets(p, z, (void *)saved, true);
    } else {  // the forward pass again; its answers go to scratch
        place_packets(p, z, at, true);
        p.o = at + z.saved();
        LA_TRY(launch_delta_rule(dt, p, true, st));
    }
    p.o = nullptr;
    p.o_bar = o_bar;
    p.state1_bar = state_bar;
    p.q_bar = q_bar;
    p.k_bar = k_bar;
    p.v_bar = v_bar;
    p.g_bar = g_bar;
    p.beta_bar = beta_bar;
    p.state0_bar = initial_state_bar;
    return launch_delta_backward(dt, p, st);
}

la_status la_delta_rule_step(la_dtype dt, int64_t batch, int hk, int hv, int dk, int dv, const void *q, int64_t ldq, const void *k, int64_t ldk,
                             const void *v, int64_t ldv, const float *g, const float *beta, double scale, float *state, int64_t slots,
                             const int32_t *slot, void *o, void *stream)
{
    DeltaSizes z;
    LA_TRY(delta_sizes(dt, batch, 1, hk, hv, dk, dv, false, z));
    if (slots < 0 || ldq < (int64_t)hk * dk || ldk < (int64_t)hk * dk || ldv < (int64_t)hv * dv)
        return LA_ERR_INVALID_ARG;
    if (batch == 0)
        return LA_OK;
    if (!q || !k || !v || !g || !beta || !o || (slots > 0 && !state) || (!slot && batch > slots))
        return LA_ERR_INVALID_ARG;
    if (batch > most_blocks(256) / hv / ((dv + 31) / 32))
        return LA_ERR_UNSUPPORTED;
    const size_t es = bytes_of(dt), ob = (size_t)batch * hv * dv * es, sb = (size_t)slots * hv * dk * dv * 4, gb = (size_t)batch * hv * 4;
    const size_t qs = ((size_t)(batch - 1) * ldq + (size_t)hk * dk) * es, ks = ((size_t)(batch - 1) * ldk + (size_t)hk * dk) * es,
                 vs = ((size_t)(batch - 1) * ldv + (size_t)hv * dv) * es;
    if (any_overlap({{q, qs}, {k, ks}, {v, vs}, {g, gb}, {beta, gb}, {slot, (size_t)batch * 4}}, {{o, ob}, {state, sb}}))
        return LA_ERR_INVALID_ARG;
    DeltaStepArgs p{q, k, v, ldq, ldk, ldv, g, beta, state, slot, slots, hk, hv, dk, dv, 0, (float)scale, o};
    hipStream_t st = (hipStream_t)stream;
    return dt == LA_F32 ? step_t<float>(p, batch, st) : dt == LA_BF16 ? step_t<bf16_t>(p, batch, st) : step_t<f16_t>(p, batch, st);
}

}  // extern "C"
