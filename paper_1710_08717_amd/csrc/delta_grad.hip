// Gradient of the gated delta rule over whole sequences (delta.hip has the forward pass and its notation).  With bars for gradients, per chunk,
// S0 and S1 the states before and after it:
//
//   U_bar = P^T O_bar + exp(b_last - b) K S1_bar,   Z_bar = T^T U_bar,   V_bar = beta Z_bar,
//   S0_bar = exp(b_last) S1_bar + Q^T scale exp(b) O_bar - K^T exp(b) beta Z_bar
//
// is a walk from the last chunk to the first, separate for every column of V as the forward one is (k_delta_scan_back).  The rest joins those columns
// and is done for all chunks at once (k_delta_grads), with E_ij = exp(b_i - b_j):
//
//   M = scale E (O_bar U^T) (j <= i),   N = -E (Z_bar U^T) (j < i),   H = N K - exp(b) Z_bar S0^T,
//   Q_bar = M K + scale exp(b) O_bar S0^T,
//   K_bar = beta H + (beta N)^T K + M^T Q + exp(b_last - b) U S1_bar^T,
//   beta_bar_i = Z_bar_i.V_i + k_i.H_i,
//   b_bar_i = q_i.Q_bar_i + 2 beta_i k_i.H_i - k_i.K_bar_i,
//   b_bar_last += sum_i exp(b_last - b_i) k_i.(S1_bar u_i) + exp(b_last) <S0, S1_bar>,   g_bar = the sum of b_bar from token i to the chunk's last.
//
// A key head's gradients are summed over the value heads that read it by the block that owns the key head, in their order.
#include "delta.hpp"

namespace la {

// Wavefronts as in the forward walk: the sums of K S1_bar in halves, U_bar and Z_bar of a half of the tokens, a half of the new gradient of the state.
// Bound by its chain as the forward walk is: 2 x 4096 tokens, 32 heads of 128, bf16: 318 us.  Sequences are walked whole, few and long ones too: 8192 tokens of
// 16 heads take the chain of 128 chunks here, where the forward walk takes segments (the gradient 671 us, the forward pass that keeps everything 299).
template <typename T, int DKP, int NG>
__global__ __launch_bounds__(128 * NG) void k_delta_scan_back(DeltaArgs p)
{
    using G = Pack<T, DKP>;
    constexpr int C = G::C, NI = G::NI, RT = G::RT, CS = G::CS, FK = G::FK, FT = G::FT, NL = NG;  // NL wavefronts load the packets: those of the second half, which have less to do with T^T
    constexpr int HT = RT / 2, HK = G::KT / 2, HS = G::KS / 2;
    constexpr int LQ = NI * FK, LP = NX * FT;
    constexpr int EACH_K = share<NI * FK, NL>() + 1, EACH_TP = 2 * share<NX * FT, NL>(), EACH_KT = share<2 * NI * FK, NL>();
    using In = RowsIn<T, C, NG, 128 * NG>;
    constexpr int EX1 = 2 * HT * UNIT > CS * NX * UNIT ? 2 * HT * UNIT : CS * NX * UNIT;                                // a group's sums; then its X_bar
    constexpr int EX2 = CS * NX * UNIT > 2 * rows_out_bytes<HT>() ? CS * NX * UNIT : 2 * rows_out_bytes<HT>();  // a group's U_bar; then rows on their way out
    __shared__ __align__(16) char keys[NI * FK * UNIT];
    __shared__ __align__(16) char tp[2 * NX * FT * UNIT];  // T^T and P^T
    __shared__ __align__(16) char decays[2][UNIT];
    __shared__ __align__(16) char turned[2 * NI * FK * UNIT];  // Kt and Qt
    __shared__ __align__(16) char oin[C * 16 * NG * sizeof(T)];
    __shared__ __align__(16) char ex1_all[NG][EX1], ex2_all[NG][EX2];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, col = lane & 15;
    const int half = wave / NG, set = wave % NG;
    const unsigned block = block_of_die(p.slices);
    const int slice = block % p.slices, h = block / p.slices % p.hv;
    const int64_t n = block / p.slices / p.hv;
    const int cbase = slice * 16 * NG + set * 16, c0 = cbase + col;
    const bool live = c0 < p.dv, kept = cbase < p.dvp;
    int64_t t0, len;
    sequence(p, n, t0, len);
    const int hk = h / (p.hv / p.hk);
    const int64_t state_at = (n * p.hv + h) * p.dk * (int64_t)p.dv, ldo = (int64_t)p.hv * p.dv;
    const int64_t slot0 = first_slot<C>(p, n, t0);
    const int chunks = (int)((len + C - 1) / C);
    const int64_t key_step = (int64_t)p.hk * (G::key_units(true) * UNIT), value_step = (int64_t)p.hv * (G::value_units(true) * UNIT);
    const char *pk = p.pack_k + (slot0 * p.hk + hk) * (int64_t)(G::key_units(true) * UNIT) + (chunks - 1) * key_step,
               *pv = p.pack_v + (slot0 * p.hv + h) * (int64_t)(G::value_units(true) * UNIT) + (chunks - 1) * value_step;
    const uint32_t keys_at = lds_address(keys), tp_at = lds_address(tp), turned_at = lds_address(turned), decays_at = lds_address(decays);
    auto fetch_k = [&](const char *k, const char *v, int buffer) {
        stream_run<NI * FK, NL>(k, keys_at, set);
        stream_units<1>(v + UNIT, decays_at + buffer * UNIT);  // (by each of them)
    };
    auto fetch_tp = [&](const char *v) {
        stream_run<NX * FT, NL>(v + G::TTURN * UNIT, tp_at, set);
        stream_run<NX * FT, NL>(v + G::PTURN * UNIT, tp_at + LP * UNIT, set);
    };
    char *ex1 = ex1_all[set], *ex2 = ex2_all[set], *mine = ex2 + half * rows_out_bytes<HT>();
    In O;
    auto fetch_o = [&](int c) {
        O.fetch((const T *)p.o_bar + ((t0 + (int64_t)c * C) * p.hv + h) * p.dv + slice * 16 * NG, ldo, (int)(len - (int64_t)c * C < C ? len - (int64_t)c * C : C),
                p.dv - slice * 16 * NG);
    };
    auto keep_state = [&](int c, const f32x4 *S) {
        if (kept) {
            float *dst = p.chunk_state_bar + (((slot0 + c) * p.hv + h) * DKP + half * (DKP / 2)) * (int64_t)p.dvp + cbase;
            if constexpr (HT == 1) {
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

    if (!half)  // what the others wait for
        __builtin_amdgcn_s_setprio(1);
    f32x4 S[HK];  // the gradient of the state after the chunk
#pragma unroll
    for (int t = 0; t < HK; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = first_of(half * HK + t) + r;
            S[t][r] = p.state1_bar && live && i < p.dk ? in_memory(p.state1_bar)[state_at + (int64_t)i * p.dv + c0] : 0.0f;
        }
    if (chunks > 0) {
        if (half) {
            fetch_k(pk, pv, (chunks - 1) & 1);
            fetch_tp(pv);
        }
        fetch_o(chunks - 1);
        keep_state(chunks - 1, S);
        O.put(oin);
        wait_loads<0>();
    }
    for (int c = chunks - 1; c >= 0; --c, pk -= key_step, pv -= value_step) {
        block_barrier();  // K, the decays and O_bar are there, all have read what the chunk before left
        if (half)
            stream_run<2 * NI * FK, NL>(pk + G::KTURN * UNIT, turned_at, set);
        const Walk<C> &d = *reinterpret_cast<const Walk<C> *>(decays[c & 1]);
        f32x4 Ob[RT], Y[RT];
        Frag<NI> kf[2][RT];
        auto rows_of = [&](int s, Frag<NI> *k) {
#pragma unroll
            for (int i = 0; i < RT; ++i)
                k[i] = unit<NI>(keys, G::row(i, s), FK);
        };
        rows_of(half * HS, kf[0]);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                Ob[i][r] = In::at(oin, first_of(i) + r, 16 * set + col);
            Y[i] = f32x4{0, 0, 0, 0};
        }
        issue_point();
        Frag<NX> f = split<NX>(join(S[0], S[1]));
#pragma unroll
        for (int s = 0; s < HS; ++s) {
            if (s + 1 < HS)
                rows_of(half * HS + s + 1, kf[~s & 1]);
            issue_point();
            const Frag<NX> now = f;
            if (s + 1 < HS)
                f = split<NX>(join(S[2 * s + 2], S[2 * s + 3]));
            mma_tiles<3, RT>(Y, kf[s & 1], now);
        }
#pragma unroll
        for (int j = 0; j < HT; ++j)
            *reinterpret_cast<f32x4 *>(ex1 + (half * HT + j) * UNIT + 16 * lane) = half ? Y[j] : Y[HT + j];
        if (half)
            wait_loads<EACH_KT>();
        block_barrier();  // (1) sums, T^T and P^T are there; K and O_bar are read
        if (c > 0) {
            fetch_o(c - 1);
            if (half)
                fetch_k(pk - key_step, pv - value_step, ~c & 1);
        }
        // this half's tokens: row tile i = half HT + j, steps s >= i / 2
        f32x4 Ub[HT], Z[HT], out[HT], beta[HT], in[HT];
        Frag<NX> pf[HT][CS], tf[HT][CS];
#pragma unroll
        for (int j = 0; j < HT; ++j) {
            const int first = first_of(half * HT + j);
            Ub[j] = (half ? Y[HT + j] : Y[j]) + *reinterpret_cast<const f32x4 *>(ex1 + ((1 - half) * HT + j) * UNIT + 16 * lane);
            out[j] = d.four(d.out, first);
            in[j] = d.four(d.in, first);
            beta[j] = d.four(d.beta, first);
            Z[j] = f32x4{0, 0, 0, 0};
        }
        auto step_unit = [&](int j, int s) { return CS == 1 ? half * HT + j : half ? G::upper(2 + j, 1) : G::upper(j, s); };
#pragma unroll
        for (int j = 0; j < HT; ++j)
#pragma unroll
            for (int s = 0; s < CS; ++s)
                if (CS == 1 || s == 1 || !half) {
                    pf[j][s] = unit<NX>(tp, LP + step_unit(j, s), FT);
                    tf[j][s] = unit<NX>(tp, step_unit(j, s), FT);
                }
#pragma unroll
        for (int j = 0; j < HT; ++j)
            Ub[j] *= out[j];
#pragma unroll
        for (int s = 0; s < CS; ++s)
            if (CS == 1 || s == 1 || !half) {
                const Frag<NI> o = split<NI>(join(Ob[2 * s], Ob[2 * s + 1]));
#pragma unroll
                for (int j = 0; j < HT; ++j)
                    mma<3>(Ub[j], pf[j][s], o);
            }
        put_step<RT>(ex2, half, Ub);
        const float all = d.all;
#pragma unroll
        for (int i = 0; i < HK; ++i)
            S[i] *= all;
        block_barrier();  // (2) U_bar is there, the sums are read
#pragma unroll
        for (int s = 0; s < CS; ++s)
            if (CS == 1 || s == 1 || !half) {
                const Frag<NX> u = unit<NX>(ex2, s * NX, 1);
#pragma unroll
                for (int j = 0; j < HT; ++j)
                    mma<3>(Z[j], tf[j][s], u);
            }
        // Q^T scale exp(b) O_bar needs nobody else's
        Frag<NX> w[CS];
#pragma unroll
        for (int s = 0; s < CS; ++s)
            w[s] = split<NX>(join(Ob[2 * s] * (p.scale * d.four(d.in, first_of(2 * s))), Ob[2 * s + 1] * (p.scale * d.four(d.in, first_of(2 * s + 1)))));
        f32x4 Vb[HT], Xb[HT];
#pragma unroll
        for (int j = 0; j < HT; ++j) {
            Vb[j] = beta[j] * Z[j];
            Xb[j] = -in[j] * Vb[j];
        }
        put_step<RT>(ex1, half, Xb);
        if (half) {
            if (c > 0)
                wait_loads<EACH_K>();
            else
                wait_loads<0>();
        }
        block_barrier();  // (3) X_bar, Kt and Qt are there; T^T, P^T and U_bar are read
        if (c > 0 && half)
            fetch_tp(pv - value_step);
        auto turned_of = [&](int from, int s, Frag<NI> *k) {
#pragma unroll
            for (int i = 0; i < HK; ++i)
                k[i] = unit<NI>(turned, from + G::turned(half * HK + i, s), FK);
        };
#pragma unroll
        for (int s = 0; s < CS; ++s) {
            Frag<NI> q[HK], k[HK];
            turned_of(LQ, s, q);
            const Frag<NX> x = unit<NX>(ex1, s * NX, 1);
            turned_of(0, s, k);
            issue_point();
            mma_tiles<3, HK>(S, q, w[s]);
            mma_tiles<3, HK>(S, k, x);
        }
        if (c > 0) {
            if (half)
                wait_loads<EACH_TP>();  // (before the stores: the next chunk does not wait for them)
            O.put(oin);
        }
        const int64_t t = t0 + (int64_t)c * C + (HT > 1 ? 32 * half : 0);
        const int64_t left = len - (int64_t)c * C - (HT > 1 ? 32 * half : 0);
        const int rows = (int)(left < 0 ? 0 : left < 32 ? left : 32);
        RowsOut<T, HT>::store(mine, (T *)p.v_bar + (t * p.hv + h) * p.dv + cbase, ldo, Vb, rows, p.dv - cbase, half);
        if (kept)
            RowsOut<float, HT>::store(mine, p.chunk_z_bar + (((slot0 + c) * p.hv + h) * C + (HT > 1 ? 32 * half : 0)) * (int64_t)p.dvp + cbase, p.dvp, Z, 32, 16, half);
        if (c > 0)
            keep_state(c - 1, S);
    }
    if (p.state0_bar && live) {
#pragma unroll
        for (int t = 0; t < HK; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = first_of(half * HK + t) + r;
                if (i < p.dk)
                    in_memory(p.state0_bar)[state_at + (int64_t)i * p.dv + c0] = S[t][r];
            }
    }
}

// One block a chunk and key head, a wavefront for each 16 columns of Q_bar and K_bar over all tokens of the chunk.  The products summed over dv take 128
// columns of O_bar, Z_bar and U through LDS at a time.  M and N go through LDS in 32 bits; their operands, and those turned, are made of that once, in the place of the
// columns, not by every wavefront that reads them.  Bound by LDS, of which a block takes all (bf16): 2 x 4096 tokens, 16 key and 32 value heads of 128: 391 us; with
// the columns split by every wavefront that needs them 510.
template <typename T, int DKP>
__global__ __launch_bounds__(4 * DKP) void k_delta_grads(DeltaArgs p)
{
    using G = Pack<T, DKP>;
    constexpr int C = G::C, NI = G::NI, RT = G::RT, CS = G::CS, FT = G::FT, NW = DKP / 16, NT = 64 * NW;
    constexpr int LZ = NI * RT, LU = LZ + NX * RT, STAGE = LU + NX * RT, WIDE = 4;  // units of 32 columns, and how many of those there are at a time
    constexpr int JM = 0, JN = NX * FT, JMT = 2 * NX * FT, JNT = 3 * NX * FT;  // units of M, N and turned M, beta N
    constexpr bool BOTH = 2 * RT > NW;  // a wavefront forms a row tile of M and of N, else of one of them
    static_assert(4 * FT * NX <= WIDE * STAGE, "M and N take the columns' place");
    __shared__ __align__(16) char stage[WIDE * STAGE * UNIT];
    __shared__ __align__(16) float mn[2][C][C + 4];
    __shared__ Decays<C> d;
    __shared__ __align__(16) float dots[4][NW][C];  // by wavefront: q.Q_bar, k.K_bar, k.H; last: k.(exp(b_last - b) U S1_bar^T)
    __shared__ float zv_box[C];
    __shared__ double state_box[NW];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, col = lane & 15, x4 = lane >> 4;
    const int hk = blockIdx.x % p.hk, group = p.hv / p.hk;
    const int64_t slot = blockIdx.x / p.hk;
    if (p.offsets) {  // tokens of no sequence: zeros
        const int64_t a = p.offsets[0], z = p.offsets[p.batch];
        for (int64_t t = slot * C; t < (slot + 1) * C && t < p.tokens; ++t)
            if (t < a || t >= z) {
                for (int c = threadIdx.x; c < p.dk; c += NT) {
                    ((T *)p.q_bar)[(t * p.hk + hk) * p.dk + c] = (T)0.0f;
                    ((T *)p.k_bar)[(t * p.hk + hk) * p.dk + c] = (T)0.0f;
                }
                for (int c = threadIdx.x; c < group * p.dv; c += NT)
                    ((T *)p.v_bar)[(t * p.hv + hk * group) * p.dv + c] = (T)0.0f;
                for (int c = threadIdx.x; c < group; c += NT)
                    p.g_bar[t * p.hv + hk * group + c] = p.beta_bar[t * p.hv + hk * group + c] = 0.0f;
            }
    }
    int64_t t0;
    int len;
    if (!slot_chunk<C>(p, slot, t0, len))
        return;
    const char *pk = p.pack_k + (slot * p.hk + hk) * (int64_t)(G::key_units(true) * UNIT);
    // the four tokens of tile i that this lane's accumulators hold, of this lane's column of k or q
    auto four_of = [&](const Frag<NI> *f, int i) {
        f32x4 x = {0, 0, 0, 0};
#pragma unroll
        for (int k = NI - 1; k >= 0; --k)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                x[r] += (float)f[i >> 1].p[k][4 * (i & 1) + r];
        return x;
    };
    f32x4 Qs[RT], Ks[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
        Qs[i] = Ks[i] = f32x4{0, 0, 0, 0};
    const int kcol = element_of(wave, col);  // this lane's column
    const bool form_m = BOTH || wave < RT, form_n = BOTH || (wave >= RT && wave < 2 * RT);
    const int tile = wave % RT;

    // 8 columns of a row: of Z_bar and V, or of O_bar and U
    constexpr int ROUNDS = (8 * C + NT - 1) / NT;
    using Pack8 = PackOf<T, 8>;
    struct Row {
        f32x8 computed;              // Z_bar or U
        typename Pack8::whole given;  // V or O_bar
    };
    const int steps = p.dvp / 32;
    auto fetch = [&](Row *in, int h, int s) {
        const int64_t sh = slot * p.hv + h;
#pragma unroll
        for (int k = 0; k < ROUNDS; ++k) {
            in[k] = Row{};  // (or what was there before would be kept for the lanes that load nothing)
            const int u = threadIdx.x + k * NT, r = u / 4 % C, c = 32 * s + 8 * (u % 4);
            if (u < 8 * C) {
                const bool z = u < 4 * C;
                in[k].computed = load8<float>((z ? p.chunk_z_bar : p.chunk_u) + (sh * C + r) * (int64_t)p.dvp + c, 8);
                const T *src = z ? (const T *)p.v + (t0 + r) * p.ldv + (int64_t)h * p.dv : (const T *)p.o_bar + ((t0 + r) * p.hv + h) * p.dv;
                in[k].given = load_raw<T, 8>(src + c, r < len ? p.dv - c : 0);
            }
        }
    };
    for (int h = hk * group; h < (hk + 1) * group; ++h) {
        const int64_t sh = slot * p.hv + h;
        const float *S0 = p.chunk_state + (sh * DKP + kcol) * (int64_t)p.dvp + 8 * x4;
        const float *S1 = p.chunk_state_bar + (sh * DKP + kcol) * (int64_t)p.dvp + 8 * x4;
        if (wave == 0) {
            const char *pv = p.pack_v + sh * (int64_t)(G::value_units(true) * UNIT);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                *reinterpret_cast<f32x4 *>((char *)&d + i * UNIT + 16 * lane) = *reinterpret_cast<const f32x4 *>(pv + i * UNIT + 16 * lane);
        }
        f32x4 pair[BOTH ? 2 : 1][RT];  // M, and N in the last: columns the queries of tile `tile`, rows the keys
        f32x4 a1[RT], a2[RT], a3[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            a1[i] = a2[i] = a3[i] = f32x4{0, 0, 0, 0};
            for (auto &x : pair)
                x[i] = f32x4{0, 0, 0, 0};
        }
        float zv = 0, states = 0;
        f32x8 st0, st1;
        auto fetch_states = [&](int s) {
            st0 = load8<float>(S0 + 32 * s, 8);
            st1 = load8<float>(S1 + 32 * s, 8);
        };
        for (int base = 0; base < steps; base += WIDE) {
            if (base)
                __syncthreads();  // the columns before are read
            // one step's columns are loaded while the one before is put into LDS
            const int until = steps < base + WIDE ? steps : base + WIDE;
            auto put = [&](const Row *in, int s) {
#pragma unroll
                for (int k = 0; k < ROUNDS; ++k) {
                    const int u = threadIdx.x + k * NT, r = u / 4 % C;
                    // token r: row 4 (r / 8 % 4) + r % 4 of tile 2 (r / 32) + r / 4 % 2
                    const int t = 2 * (r >> 5) + ((r >> 2) & 1);
                    char *to = stage + (s - base) * STAGE * UNIT + 16 * (16 * (u % 4) + 4 * ((r >> 3) & 3) + (r & 3));
                    if (u < 8 * C) {
                        const bool z = u < 4 * C;
                        const Frag<NX> f = split<NX>(in[k].computed);
#pragma unroll
                        for (int i = 0; i < NX; ++i)
                            *reinterpret_cast<bf16x8 *>(to + ((z ? LZ : LU) + i * RT + t) * UNIT) = f.p[i];
                        const f32x8 x = __builtin_convertvector(in[k].given, f32x8);
                        if (z) {
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                zv += in[k].computed[i] * x[i];
                        } else {
                            const Frag<NI> o = split<NI>(x);
#pragma unroll
                            for (int i = 0; i < NI; ++i)
                                *reinterpret_cast<bf16x8 *>(to + (i * RT + t) * UNIT) = o.p[i];
                        }
                    }
                }
            };
            Row even[ROUNDS], odd[ROUNDS];
            fetch(even, h, base);
#pragma unroll 1
            for (int s = base; s < until; s += 2) {
                fetch(odd, h, s + 1 < until ? s + 1 : s);
                put(even, s);
                if (s + 1 < until) {
                    fetch(even, h, s + 2 < until ? s + 2 : s);
                    put(odd, s + 1);
                }
            }
            __syncthreads();
            if (base == 0)
                fetch_states(0);
            // M, N: whether this wavefront forms them; HIGH: its queries are in the second half of the tokens
            auto products = [&](auto M, auto N, auto HIGH) {
#pragma unroll 1
                for (int s = base; s < until; ++s) {
                    const char *at = stage + (s - base) * STAGE * UNIT;
                    Frag<NI> ot;
                    Frag<NX> zt;
                    if constexpr (M.value)
                        ot = unit<NI>(at, tile, RT);
                    if constexpr (N.value)
                        zt = unit<NX>(at, LZ + tile, RT);
#pragma unroll
                    for (int i = 0; i < (CS == 1 || HIGH.value ? RT : 2); ++i) {
                        const Frag<NX> u = unit<NX>(at, LU + i, RT);
                        if constexpr (M.value)
                            mma<3>(pair[0][i], u, ot);
                        if constexpr (N.value)
                            mma<3>(pair[BOTH][i], u, zt);
                    }
                }
            };
            using Yes = std::true_type;
            using No = std::false_type;
            auto halves = [&](auto M, auto N) {
                if (CS > 1 && tile >= 2)
                    products(M, N, Yes{});
                else
                    products(M, N, No{});
            };
            if constexpr (BOTH)
                halves(Yes{}, Yes{});
            else if (form_m)
                halves(Yes{}, No{});
            else if (form_n)
                halves(No{}, Yes{});
            if (until == steps) {  // with the decays to LDS
                const int mine = element_of(tile, col);  // this lane's query
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const int x = first_of(i);
                    f32x4 e;
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        e[r] = x + r <= mine ? d.between(mine, x + r) : 0.0f;
                    if (form_m) {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            pair[0][i][r] = e[r] != 0 ? p.scale * e[r] * pair[0][i][r] : 0.0f;
                        *reinterpret_cast<f32x4 *>(&mn[0][mine][x]) = pair[0][i];
                    }
                    if (form_n) {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            pair[BOTH][i][r] = e[r] != 0 && x + r != mine ? -e[r] * pair[BOTH][i][r] : 0.0f;
                        *reinterpret_cast<f32x4 *>(&mn[1][mine][x]) = pair[BOTH][i];
                    }
                }
            }
#pragma unroll 1
            for (int s = base; s < until; ++s) {
                const char *at = stage + (s - base) * STAGE * UNIT;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    states += st0[i] * st1[i];
                const Frag<NX> f0 = split<NX>(st0), f1 = split<NX>(st1);
                fetch_states(s + 1 < steps ? s + 1 : s);
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    mma<3>(a2[i], unit<NX>(at, LZ + i, RT), f0);
                    mma<3>(a3[i], unit<NX>(at, LU + i, RT), f1);
                    mma<3>(a1[i], unit<NI>(at, i, RT), f0);
                }
            }
        }
        Frag<NI> kt[CS], qt[CS];
#pragma unroll
        for (int s = 0; s < CS; ++s) {
            kt[s] = unit<NI>(pk, G::KTURN + G::turned(wave, s), G::FK);
            qt[s] = unit<NI>(pk, G::QTURN + G::turned(wave, s), G::FK);
        }
        __syncthreads();  // the columns are read: the operands take their place
        char *joint = stage;
        for (int u = wave; u < 4 * FT; u += NW) {  // M, N, turned M, turned beta N: FT units of each
            const int which = u / FT, v = u % FT;
            int i = v, s = 0;  // row tile and step of unit v
            if constexpr (CS > 1) {
                i = which < 2 ? (v < 2 ? v : 2 + (v - 2) / 2) : v < 4 ? v / 2 : v - 2;
                s = which < 2 ? (v < 2 ? 0 : v & 1) : v < 4 ? v & 1 : 1;
            }
            const int row = element_of(i, col), at = 32 * s + 8 * x4;
            f32x8 x;
            if (which < 2) {
                const float *from = &mn[which][row][at];
                x = join(*reinterpret_cast<const f32x4 *>(from), *reinterpret_cast<const f32x4 *>(from + 4));
            } else {
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    x[r] = (which == 3 ? d.walk.beta[at + r] : 1.0f) * mn[which - 2][at + r][row];
            }
            put_unit<NX>(joint, which * NX * FT + v, FT, x);
        }
        zv += __shfl_xor(zv, 1, 64);
        zv += __shfl_xor(zv, 2, 64);
        if (threadIdx.x < 4 * C && threadIdx.x % 4 == 0)
            zv_box[threadIdx.x / 4] = zv;
        const double sum = wave_sum((double)states);
        if (lane == 0)
            state_box[wave] = sum;
        auto dot = [&](int which, const f32x4 (&a)[RT], const Frag<NI> (&f)[CS]) {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                f32x4 x = a[i] * four_of(f, i);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    x[r] = row16_sum(x[r]);
                if (col == 0)
                    *reinterpret_cast<f32x4 *>(&dots[which][wave][first_of(i)]) = x;
            }
        };
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const f32x4 in = d.walk.four(d.walk.in, first_of(i));
            a1[i] *= p.scale * in;
            a2[i] *= -in;
            a3[i] *= d.walk.four(d.walk.out, first_of(i));
        }
        dot(3, a3, kt);
        __syncthreads();  // M and N are there
#pragma unroll
        for (int s = 0; s < CS; ++s)
#pragma unroll
            for (int i = 0; i < RT; ++i) {  // row tile i of the results
                if (s <= i / 2) {
                    const Frag<NX> mf = unit<NX>(joint, JM + G::lower(i, s), FT), nf = unit<NX>(joint, JN + G::lower(i, s), FT);
                    mma<3>(a1[i], mf, kt[s]);
                    mma<3>(a2[i], nf, kt[s]);
                }
                if (s >= i / 2) {
                    const Frag<NX> mf = unit<NX>(joint, JMT + G::upper(i, s), FT), nf = unit<NX>(joint, JNT + G::upper(i, s), FT);
                    mma<3>(a3[i], mf, qt[s]);
                    mma<3>(a3[i], nf, kt[s]);
                }
            }
        dot(2, a2, kt);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            a3[i] += d.walk.four(d.walk.beta, first_of(i)) * a2[i];
            Qs[i] += a1[i];
            Ks[i] += a3[i];
        }
        dot(0, a1, qt);
        dot(1, a3, kt);
        __syncthreads();
        if (wave == 0) {
            const int i = lane < C ? lane : C - 1;
            auto whole = [&](int which) {
                double x = 0;
#pragma unroll
                for (int w = 0; w < NW; ++w)
                    x += dots[which][w][i];
                return x;
            };
            const double kh = whole(2);
            double last = lane < C ? whole(3) : 0.0, both = 0;
#pragma unroll
            for (int w = 0; w < NW; ++w)
                both += state_box[w];
            last = wave_sum(last) + d.walk.all * both;
            double x = lane < C ? whole(0) + 2.0 * d.walk.beta[i] * kh - whole(1) : 0.0;
#pragma unroll
            for (int s = 1; s < C; s *= 2) {  // from the chunk's end
                const double y = __shfl_down(x, s, 64);
                if (lane + s < C)
                    x += y;
            }
            if (lane < len) {
                p.g_bar[(t0 + lane) * p.hv + h] = (float)(x + last);
                p.beta_bar[(t0 + lane) * p.hv + h] = (float)(zv_box[i] + kh);
            }
        }
        __syncthreads();  // the next head overwrites what this one reads
    }
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = first_of(i) + r;
            if (row < len && kcol < p.dk) {
                const int64_t at = ((t0 + row) * p.hk + hk) * p.dk + kcol;
                in_memory((T *)p.q_bar)[at] = (T)Qs[i][r];
                in_memory((T *)p.k_bar)[at] = (T)Ks[i][r];
            }
        }
}

template <typename T, int DKP>
static la_status back_t(DeltaArgs &p, hipStream_t st)
{
    const int groups = walk_groups(p.batch * p.hv, p.dv);
    p.slices = (p.dv + 16 * groups - 1) / (16 * groups);
    const int64_t blocks = p.batch * p.hv * p.slices;
    if (blocks > most_blocks(128 * groups) || p.slots * p.hk > most_blocks(4 * DKP))
        return LA_ERR_UNSUPPORTED;
    if (groups == 2)
        LA_LAUNCH((k_delta_scan_back<T, DKP, 2>), dim3((unsigned)blocks), dim3(256), 0, st, p);
    else
        LA_LAUNCH((k_delta_scan_back<T, DKP, 4>), dim3((unsigned)blocks), dim3(512), 0, st, p);
    if (p.slots > 0)
        LA_LAUNCH((k_delta_grads<T, DKP>), dim3((unsigned)(p.slots * p.hk)), dim3(4 * DKP), 0, st, p);
    return launch_check("delta rule backward");
}

la_status launch_delta_backward(la_dtype dt, DeltaArgs p, hipStream_t st)
{
    const bool half = p.dk <= 64;
    switch (dt) {
    case LA_F32: return half ? back_t<float, 64>(p, st) : back_t<float, 128>(p, st);
    case LA_BF16: return half ? back_t<bf16_t, 64>(p, st) : back_t<bf16_t, 128>(p, st);
    default: return half ? back_t<f16_t, 64>(p, st) : back_t<f16_t, 128>(p, st);
    }
}

}  // namespace la
