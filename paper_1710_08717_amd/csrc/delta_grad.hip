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

template <typename T, int DKP, int NW>
__global__ __launch_bounds__(64 * NW) void k_delta_scan_back(DeltaArgs p)
{
    constexpr int C = DeltaIn<T>::C, NI = DeltaIn<T>::NI, RT = C / 16, KT = DKP / 16;
    struct Tiles {
        Planes<NI, C, DKP> K, Q;
        Planes<NI, DKP, C> Kt, Qt;
        Planes<NX, C, C> inv, P;  // T^T and P^T
        Decays<C> d;
    };
    __shared__ __align__(16) Tiles m;
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, col = lane & 15, row4 = 4 * (lane >> 4);
    const int slice = blockIdx.x % p.slices, h = blockIdx.x / p.slices % p.hv;
    const int64_t n = blockIdx.x / p.slices / p.hv;
    const int c0 = (slice * NW + wave) * 16 + col;
    const bool live = c0 < p.dv, kept = c0 < p.dvp;
    int64_t t0, len;
    sequence(p, n, t0, len);
    const int hk = h / (p.hv / p.hk);
    const int64_t state_at = (n * p.hv + h) * p.dk * (int64_t)p.dv;

    f32x4 S[KT];  // the gradient of the state after the chunk
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 16 * t + row4 + r;
            S[t][r] = p.state1_bar && live && i < p.dk ? p.state1_bar[state_at + (int64_t)i * p.dv + c0] : 0.0f;
        }
    for (int i = threadIdx.x; i < C * Planes<NX, C, C>::LD; i += 64 * NW)
        for (int x = 0; x < NX; ++x)
            (&m.P.e[x][0][0])[i] = (bf16_t)0.0f;

    const int64_t chunks = (len + C - 1) / C;
    int64_t slot = first_slot<C>(p, n, t0) + chunks - 1;
    for (int64_t c = chunks - 1; c >= 0; --c, --slot) {
        const int64_t t = t0 + c * C;
        const int left = (int)(len - c * C < C ? len - c * C : C);
        const int64_t sh = slot * p.hv + h;
        __syncthreads();
        stage_chunk<T, NI, C, DKP, true, true>((const T *)p.k + t * p.ldk + (int64_t)hk * p.dk, p.ldk, left, p.dk, &m.K, &m.Kt);
        stage_chunk<T, NI, C, DKP, true, true>((const T *)p.q + t * p.ldq + (int64_t)hk * p.dk, p.ldq, left, p.dk, &m.Q, &m.Qt);
        const float *inv = p.inv + sh * C * C;
        for (int u = threadIdx.x; u < C * C / 16; u += 64 * NW) {
            const int i = 4 * (u / (C / 4)), j = 4 * (u % (C / 4));
            f32x4 x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r)
                x[r] = *reinterpret_cast<const f32x4 *>(inv + (i + r) * C + j);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                m.inv.put4(j + r, i, f32x4{x[0][r], x[1][r], x[2][r], x[3][r]});
        }
        if (wave == 0)
            m.d.load(p.g + t * p.hv + h, p.beta + t * p.hv + h, p.hv, left);
        f32x4 O[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * i + row4 + r;
                O[i][r] = live && row < left ? (float)((const T *)p.o_bar)[((t + row) * p.hv + h) * p.dv + c0] : 0.0f;
            }
        __syncthreads();
        // P^T: lane's column is the key, its four rows the queries
        for (int j = wave; j < RT; j += NW)
            for (int i = j; i < RT; ++i) {
                f32x4 x = {0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < DKP / 32; ++s)
                    mma(x, m.Q.frag(16 * i, s), m.K.frag(16 * j, s));
                const int kj = 16 * j + col;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int qi = 16 * i + row4 + r;
                    x[r] = kj <= qi ? p.scale * m.d.between(qi, kj) * x[r] : 0.0f;
                }
                m.P.put4(kj, 16 * i + row4, x);
            }
        if (kept) {
            float *out = p.chunk_state_bar + sh * DKP * (int64_t)p.dvp + c0;
#pragma unroll
            for (int i = 0; i < KT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    out[(int64_t)(16 * i + row4 + r) * p.dvp] = S[i][r];
        }
        f32x4 Y[RT], Z[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i)
            Y[i] = Z[i] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < DKP / 32; ++s) {
            const Frag<NX> f = split<NX>(join(S[2 * s], S[2 * s + 1]));
#pragma unroll
            for (int i = 0; i < RT; ++i)
                mma(Y[i], m.K.frag(16 * i, s), f);
        }
#pragma unroll
        for (int i = 0; i < RT; ++i)
            Y[i] *= m.d.four(m.d.out, 16 * i + row4);
        __syncthreads();  // P^T is there
        const float all = m.d.all;
#pragma unroll
        for (int i = 0; i < KT; ++i)
            S[i] *= all;
#pragma unroll
        for (int s = 0; s < C / 32; ++s) {
            const Frag<NI> f = split<NI>(join(O[2 * s], O[2 * s + 1]));
#pragma unroll
            for (int j = 0; j < 2 * s + 2; ++j)
                mma(Y[j], m.P.frag(16 * j, s), f);
            const Frag<NX> w = split<NX>(join(O[2 * s] * p.scale * m.d.four(m.d.in, 32 * s + row4), O[2 * s + 1] * p.scale * m.d.four(m.d.in, 32 * s + 16 + row4)));
#pragma unroll
            for (int i = 0; i < KT; ++i)
                mma(S[i], m.Qt.frag(16 * i, s), w);
        }
#pragma unroll
        for (int s = 0; s < C / 32; ++s) {
            const Frag<NX> f = split<NX>(join(Y[2 * s], Y[2 * s + 1]));
#pragma unroll
            for (int j = 0; j < 2 * s + 2; ++j)
                mma(Z[j], m.inv.frag(16 * j, s), f);
        }
        if (kept) {
            float *out = p.chunk_z_bar + sh * C * (int64_t)p.dvp + c0;
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    out[(int64_t)(16 * i + row4 + r) * p.dvp] = Z[i][r];
        }
#pragma unroll
        for (int i = 0; i < RT; ++i)
            Z[i] *= m.d.four(m.d.beta, 16 * i + row4);
        if (live) {
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = 16 * i + row4 + r;
                    if (row < left)
                        ((T *)p.v_bar)[((t + row) * p.hv + h) * p.dv + c0] = (T)Z[i][r];
                }
        }
#pragma unroll
        for (int s = 0; s < C / 32; ++s) {
            const Frag<NX> w = split<NX>(join(-Z[2 * s] * m.d.four(m.d.in, 32 * s + row4), -Z[2 * s + 1] * m.d.four(m.d.in, 32 * s + 16 + row4)));
#pragma unroll
            for (int i = 0; i < KT; ++i)
                mma(S[i], m.Kt.frag(16 * i, s), w);
        }
    }
    if (p.state0_bar && live) {
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * t + row4 + r;
                if (i < p.dk)
                    p.state0_bar[state_at + (int64_t)i * p.dv + c0] = S[t][r];
            }
    }
}

// One block a chunk and key head.  A wavefront owns DKP / 4 columns of Q_bar and K_bar over all tokens of the chunk, and the 16 rows `wave` of M and N.
template <typename T, int DKP>
__global__ __launch_bounds__(256) void k_delta_grads(DeltaArgs p)
{
    constexpr int C = DeltaIn<T>::C, NI = DeltaIn<T>::NI, RT = C / 16, CT = DKP / 64;
    struct Tiles {
        Planes<NI, DKP, C> Kt, Qt;
        Planes<NI, C, 32> O;     // 32 columns of O_bar, Z_bar, U at a time
        Planes<NX, C, 32> Z, U;
        float M[C][C + 4], N[C][C + 4];
        Decays<C> d;
        float dots[4][4][C];  // by wavefront: q.Q_bar, k.K_bar, k.H; last: k.(exp(b_last - b) U S1_bar^T)
        float zv[C];
        double states[4];
    };
    __shared__ __align__(16) Tiles m;
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, col = lane & 15, row4 = 4 * (lane >> 4);
    const int hk = blockIdx.x % p.hk, group = p.hv / p.hk;
    const int64_t slot = blockIdx.x / p.hk;
    if (p.offsets) {  // tokens of no sequence: zeros
        const int64_t a = p.offsets[0], z = p.offsets[p.batch];
        for (int64_t t = slot * C; t < (slot + 1) * C && t < p.tokens; ++t)
            if (t < a || t >= z) {
                for (int c = threadIdx.x; c < p.dk; c += 256) {
                    ((T *)p.q_bar)[(t * p.hk + hk) * p.dk + c] = (T)0.0f;
                    ((T *)p.k_bar)[(t * p.hk + hk) * p.dk + c] = (T)0.0f;
                }
                for (int h = hk * group; h < (hk + 1) * group; ++h) {
                    for (int c = threadIdx.x; c < p.dv; c += 256)
                        ((T *)p.v_bar)[(t * p.hv + h) * p.dv + c] = (T)0.0f;
                    if (threadIdx.x == 0)
                        p.g_bar[t * p.hv + h] = p.beta_bar[t * p.hv + h] = 0.0f;
                }
            }
    }
    int64_t t0;
    int len;
    if (!slot_chunk<C>(p, slot, t0, len))
        return;
    stage_chunk<T, NI, C, DKP, false, true>((const T *)p.k + t0 * p.ldk + (int64_t)hk * p.dk, p.ldk, len, p.dk, (Planes<NI, C, DKP> *)nullptr, &m.Kt);
    stage_chunk<T, NI, C, DKP, false, true>((const T *)p.q + t0 * p.ldq + (int64_t)hk * p.dk, p.ldq, len, p.dk, (Planes<NI, C, DKP> *)nullptr, &m.Qt);
    f32x4 Qs[RT][CT], Ks[RT][CT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int c = 0; c < CT; ++c)
            Qs[i][c] = Ks[i][c] = f32x4{0, 0, 0, 0};
    const int k0 = wave * 16 * CT;  // this wavefront's columns

    for (int h = hk * group; h < (hk + 1) * group; ++h) {
        const int64_t sh = slot * p.hv + h;
        const float *S0 = p.chunk_state + sh * DKP * (int64_t)p.dvp, *S1 = p.chunk_state_bar + sh * DKP * (int64_t)p.dvp;
        const float *Ug = p.chunk_u + sh * C * (int64_t)p.dvp, *Zg = p.chunk_z_bar + sh * C * (int64_t)p.dvp;
        if (wave == 0)
            m.d.load(p.g + t0 * p.hv + h, p.beta + t0 * p.hv + h, p.hv, len);
        f32x4 a1[RT][CT], a2[RT][CT], a3[RT][CT], mp[RT], np[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            mp[i] = np[i] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < CT; ++c)
                a1[i][c] = a2[i][c] = a3[i][c] = f32x4{0, 0, 0, 0};
        }
        float zv = 0;
        double states = 0;
        for (int s = 0; s < p.dvp / 32; ++s) {
            __syncthreads();  // the columns before are read
            if (threadIdx.x < 4 * C) {
                const int r = threadIdx.x / 4, x = 8 * (threadIdx.x % 4), c = 32 * s + x;
                const f32x8 o = load8<T>((const T *)p.o_bar + ((t0 + r) * p.hv + h) * p.dv + c, r < len ? p.dv - c : 0);
                const f32x8 v = load8<T>((const T *)p.v + (t0 + r) * p.ldv + (int64_t)h * p.dv + c, r < len ? p.dv - c : 0);
                const f32x8 z = load8<float>(Zg + (int64_t)r * p.dvp + c, 8), u = load8<float>(Ug + (int64_t)r * p.dvp + c, 8);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    zv += z[i] * v[i];
                m.O.put4(r, x, __builtin_shufflevector(o, o, 0, 1, 2, 3));
                m.O.put4(r, x + 4, __builtin_shufflevector(o, o, 4, 5, 6, 7));
                m.Z.put4(r, x, __builtin_shufflevector(z, z, 0, 1, 2, 3));
                m.Z.put4(r, x + 4, __builtin_shufflevector(z, z, 4, 5, 6, 7));
                m.U.put4(r, x, __builtin_shufflevector(u, u, 0, 1, 2, 3));
                m.U.put4(r, x + 4, __builtin_shufflevector(u, u, 4, 5, 6, 7));
            }
            Frag<NX> f0[CT], f1[CT];
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const int64_t at = (int64_t)(k0 + 16 * c + col) * p.dvp + 32 * s + row4;
                const f32x8 x = join(*reinterpret_cast<const f32x4 *>(S0 + at), *reinterpret_cast<const f32x4 *>(S0 + at + 16));
                const f32x8 y = join(*reinterpret_cast<const f32x4 *>(S1 + at), *reinterpret_cast<const f32x4 *>(S1 + at + 16));
                float sum = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    sum += x[i] * y[i];
                states += sum;
                f0[c] = split<NX>(x);
                f1[c] = split<NX>(y);
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const Frag<NI> o = m.O.frag(16 * i, 0);
                const Frag<NX> z = m.Z.frag(16 * i, 0), u = m.U.frag(16 * i, 0);
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    mma(a1[i][c], o, f0[c]);
                    mma(a2[i][c], z, f0[c]);
                    mma(a3[i][c], u, f1[c]);
                }
                if (wave < RT && i <= wave) {  // rows `wave` of M and N, columns i
                    mma(mp[i], m.O.frag(16 * wave, 0), u);
                    mma(np[i], m.Z.frag(16 * wave, 0), u);
                }
            }
        }
        // M and N
        if (wave < RT) {
#pragma unroll
            for (int j = 0; j < RT; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int qi = 16 * wave + row4 + r, kj = 16 * j + col;
                    const float e = kj <= qi ? m.d.between(qi, kj) : 0.0f;
                    m.M[qi][kj] = kj <= qi ? p.scale * e * mp[j][r] : 0.0f;
                    m.N[qi][kj] = kj < qi ? -e * np[j][r] : 0.0f;
                }
        }
        zv += __shfl_xor(zv, 1, 64);
        zv += __shfl_xor(zv, 2, 64);
        if (threadIdx.x < 4 * C && threadIdx.x % 4 == 0)
            m.zv[threadIdx.x / 4] = zv;
        states = wave_sum(states);
        if (lane == 0)
            m.states[wave] = states;
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const f32x4 in = m.d.four(m.d.in, 16 * i + row4), out = m.d.four(m.d.out, 16 * i + row4);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                a1[i][c] *= p.scale * in;
                a2[i][c] *= -in;
                a3[i][c] *= out;
            }
        }
        auto dots = [&](int which, auto &&a, const Planes<NI, DKP, C> &x) {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                f32x4 d = {0, 0, 0, 0};
#pragma unroll
                for (int c = 0; c < CT; ++c)
                    d += a[i][c] * x.get4(k0 + 16 * c + col, 16 * i + row4);
#pragma unroll
                for (int k = 1; k < 16; k *= 2)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        d[r] += __shfl_xor(d[r], k, 64);
                if (col == 0)
                    *reinterpret_cast<f32x4 *>(&m.dots[which][wave][16 * i + row4]) = d;
            }
        };
        dots(3, a3, m.Kt);
        __syncthreads();  // M and N are there
#pragma unroll
        for (int i = 0; i < RT; ++i) {  // rows i of the results
#pragma unroll
            for (int s = 0; s < C / 32; ++s) {
                const int row = 16 * i + col, at = 32 * s + row4;
                if (2 * s <= i) {
                    const Frag<NX> fm = split<NX>(join(*reinterpret_cast<const f32x4 *>(&m.M[row][at]), *reinterpret_cast<const f32x4 *>(&m.M[row][at + 16])));
                    const Frag<NX> fn = split<NX>(join(*reinterpret_cast<const f32x4 *>(&m.N[row][at]), *reinterpret_cast<const f32x4 *>(&m.N[row][at + 16])));
#pragma unroll
                    for (int c = 0; c < CT; ++c) {
                        const Frag<NI> k = m.Kt.frag(k0 + 16 * c, s);
                        mma(a1[i][c], fm, k);
                        mma(a2[i][c], fn, k);
                    }
                }
                if (2 * s + 1 >= i) {
                    f32x8 x, y;
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        const int t = at + (r & 3) + 16 * (r >> 2);
                        x[r] = m.M[t][row];
                        y[r] = m.d.beta[t] * m.N[t][row];
                    }
                    const Frag<NX> fm = split<NX>(x), fn = split<NX>(y);
#pragma unroll
                    for (int c = 0; c < CT; ++c) {
                        mma(a3[i][c], fm, m.Qt.frag(k0 + 16 * c, s));
                        mma(a3[i][c], fn, m.Kt.frag(k0 + 16 * c, s));
                    }
                }
            }
        }
        dots(2, a2, m.Kt);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const f32x4 beta = m.d.four(m.d.beta, 16 * i + row4);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                a3[i][c] += beta * a2[i][c];
                Qs[i][c] += a1[i][c];
                Ks[i][c] += a3[i][c];
            }
        }
        dots(0, a1, m.Qt);
        dots(1, a3, m.Kt);
        __syncthreads();
        if (wave == 0) {
            const int i = lane < C ? lane : C - 1;
            auto whole = [&](int which) { return (double)m.dots[which][0][i] + m.dots[which][1][i] + m.dots[which][2][i] + m.dots[which][3][i]; };
            const double kh = whole(2);
            double last = lane < C ? whole(3) : 0.0;
            last = wave_sum(last) + m.d.all * (m.states[0] + m.states[1] + m.states[2] + m.states[3]);
            double x = lane < C ? whole(0) + 2.0 * m.d.beta[i] * kh - whole(1) : 0.0;
#pragma unroll
            for (int s = 1; s < C; s *= 2) {  // from the chunk's end
                const double y = __shfl_down(x, s, 64);
                if (lane + s < C)
                    x += y;
            }
            if (lane < len) {
                p.g_bar[(t0 + lane) * p.hv + h] = (float)(x + last);
                p.beta_bar[(t0 + lane) * p.hv + h] = (float)(m.zv[i] + kh);
            }
        }
        __syncthreads();  // the next head overwrites the decays and dots
    }
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * i + row4 + r, k = k0 + 16 * c + col;
                if (row < len && k < p.dk) {
                    const int64_t at = ((t0 + row) * p.hk + hk) * p.dk + k;
                    ((T *)p.q_bar)[at] = (T)Qs[i][c][r];
                    ((T *)p.k_bar)[at] = (T)Ks[i][c][r];
                }
            }
}

template <typename T, int DKP>
static la_status back_t(DeltaArgs &p, hipStream_t st)
{
    constexpr int NW = 4;
    p.slices = (p.dv + 16 * NW - 1) / (16 * NW);
    LA_LAUNCH((k_delta_scan_back<T, DKP, NW>), dim3((unsigned)(p.batch * p.hv * p.slices)), dim3(64 * NW), 0, st, p);
    if (p.slots > 0)
        LA_LAUNCH((k_delta_grads<T, DKP>), dim3((unsigned)(p.slots * p.hk)), dim3(256), 0, st, p);
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
