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
// k_delta_inverse forms T for all chunks at once; k_delta_scan walks a sequence's chunks.  Everything after T is separate for every column of
// V, so a wavefront takes 16 columns and keeps its part of the state in accumulators from the first chunk to the last.
#include "delta.hpp"

namespace la {

// ---------------------------------------------------------------------------------
// T of every chunk and value head
// ---------------------------------------------------------------------------------
template <typename T, int DKP>
__global__ __launch_bounds__(64) void k_delta_inverse(DeltaArgs p)
{
    constexpr int C = DeltaIn<T>::C, NI = DeltaIn<T>::NI;
    __shared__ Planes<NI, C, DKP> K;
    __shared__ __align__(16) float A[C][C + 4];
    __shared__ Decays<C> d;
    const int lane = threadIdx.x, h = blockIdx.x % p.hv;
    const int64_t slot = blockIdx.x / p.hv;
    if (p.offsets) {  // tokens of no sequence: zeros
        const int64_t a = p.offsets[0], z = p.offsets[p.batch];
        for (int64_t t = slot * C; t < (slot + 1) * C && t < p.tokens; ++t)
            if (t < a || t >= z)
                for (int c = lane; c < p.dv; c += 64)
                    ((T *)p.o)[(t * p.hv + h) * p.dv + c] = (T)0.0f;
    }
    int64_t t0;
    int len;
    if (!slot_chunk<C>(p, slot, t0, len))
        return;
    const int hk = h / (p.hv / p.hk);
    const T *k = (const T *)p.k + t0 * p.ldk + (int64_t)hk * p.dk;
    stage_chunk<T, NI, C, DKP, true, false>(k, p.ldk, len, p.dk, &K, nullptr);
    d.load(p.g + t0 * p.hv + h, p.beta + t0 * p.hv + h, p.hv, len);
    __syncthreads();
    const int col = lane & 15, row4 = 4 * (lane >> 4);
#pragma unroll
    for (int ti = 0; ti < C / 16; ++ti)
#pragma unroll
        for (int tj = 0; tj <= ti; ++tj) {
            f32x4 x = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < DKP / 32; ++s)
                mma(x, K.frag(16 * ti, s), K.frag(16 * tj, s));
            const int j = 16 * tj + col;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * ti + row4 + r;
                A[i][j] = j < i ? d.beta[i] * d.between(i, j) * x[r] : 0.0f;
            }
        }
    __syncthreads();
    // column `lane` of T by forward substitution
    float *out = p.inv + (slot * p.hv + h) * C * C;
    float t[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        float s[4] = {i == lane ? 1.0f : 0.0f, 0, 0, 0};
#pragma unroll
        for (int l = 0; l < i; l += 4) {
            const f32x4 a = *reinterpret_cast<const f32x4 *>(&A[i][l]);
#pragma unroll
            for (int m = 0; m < 4; ++m)
                if (l + m < i)
                    s[m] -= a[m] * t[l + m];
        }
        t[i] = (s[0] + s[1]) + (s[2] + s[3]);
        if (lane < C)
            out[i * C + lane] = t[i];
    }
}

// ---------------------------------------------------------------------------------
// the walk over a sequence's chunks
// ---------------------------------------------------------------------------------
template <typename T, int DKP, int NW, bool SAVE>
__global__ __launch_bounds__(64 * NW) void k_delta_scan(DeltaArgs p)
{
    constexpr int C = DeltaIn<T>::C, NI = DeltaIn<T>::NI, RT = C / 16, KT = DKP / 16;
    struct Tiles {
        Planes<NI, C, DKP> K, Q;
        Planes<NI, DKP, C> Kt;
        Planes<NX, C, C> inv, P;
        Decays<C> d;
    };
    __shared__ __align__(16) Tiles m;
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, col = lane & 15, row4 = 4 * (lane >> 4);
    const int slice = blockIdx.x % p.slices, h = blockIdx.x / p.slices % p.hv;
    const int64_t n = blockIdx.x / p.slices / p.hv;
    const int c0 = (slice * NW + wave) * 16 + col;  // this lane's column of V
    const bool live = c0 < p.dv;
    int64_t t0, len;
    sequence(p, n, t0, len);
    const int hk = h / (p.hv / p.hk);
    const int64_t state_at = (n * p.hv + h) * p.dk * (int64_t)p.dv;

    f32x4 S[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 16 * t + row4 + r;
            S[t][r] = p.state0 && live && i < p.dk ? p.state0[state_at + (int64_t)i * p.dv + c0] : 0.0f;
        }
    // the halves of 32-wide steps that lie right of the diagonal stay zero
    for (int i = threadIdx.x; i < C * Planes<NX, C, C>::LD; i += 64 * NW)
        for (int x = 0; x < NX; ++x)
            (&m.P.e[x][0][0])[i] = (bf16_t)0.0f;

    int64_t slot = first_slot<C>(p, n, t0);
    for (int64_t c = 0; c * C < len; ++c, ++slot) {
        const int64_t t = t0 + c * C;
        const int left = (int)(len - c * C < C ? len - c * C : C);
        __syncthreads();  // the tiles of the chunk before are read
        stage_chunk<T, NI, C, DKP, true, true>((const T *)p.k + t * p.ldk + (int64_t)hk * p.dk, p.ldk, left, p.dk, &m.K, &m.Kt);
        stage_chunk<T, NI, C, DKP, true, false>((const T *)p.q + t * p.ldq + (int64_t)hk * p.dk, p.ldq, left, p.dk, &m.Q, nullptr);
        const float *inv = p.inv + (slot * p.hv + h) * C * C;
        for (int u = threadIdx.x; u < C * C / 4; u += 64 * NW)
            m.inv.put4(u / (C / 4), 4 * (u % (C / 4)), *reinterpret_cast<const f32x4 *>(inv + 4 * u));
        if (wave == 0)
            m.d.load(p.g + t * p.hv + h, p.beta + t * p.hv + h, p.hv, left);
        f32x4 V[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * i + row4 + r;
                V[i][r] = live && row < left ? (float)((const T *)p.v)[(t + row) * p.ldv + (int64_t)h * p.dv + c0] : 0.0f;
            }
        __syncthreads();
        // P, turned: lane's column is the query, its four rows the keys
        for (int i = wave; i < RT; i += NW)
            for (int j = 0; j <= i; ++j) {
                f32x4 x = {0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < DKP / 32; ++s)
                    mma(x, m.K.frag(16 * j, s), m.Q.frag(16 * i, s));
                const int qi = 16 * i + col;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int kj = 16 * j + row4 + r;
                    x[r] = kj <= qi ? p.scale * m.d.between(qi, kj) * x[r] : 0.0f;
                }
                m.P.put4(qi, 16 * j + row4, x);
            }
        if constexpr (SAVE) {
            float *out = p.chunk_state + (slot * p.hv + h) * DKP * (int64_t)p.dvp + c0;
            if (c0 < p.dvp) {
#pragma unroll
                for (int i = 0; i < KT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        out[(int64_t)(16 * i + row4 + r) * p.dvp] = S[i][r];
            }
        }
        f32x4 X[RT], Y[RT], U[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i)
            X[i] = Y[i] = U[i] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < DKP / 32; ++s) {
            const Frag<NX> f = split<NX>(join(S[2 * s], S[2 * s + 1]));
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                mma(X[i], m.K.frag(16 * i, s), f);
                mma(Y[i], m.Q.frag(16 * i, s), f);
            }
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const f32x4 in = m.d.four(m.d.in, 16 * i + row4), beta = m.d.four(m.d.beta, 16 * i + row4);
            X[i] = beta * (V[i] - in * X[i]);  // Z
            Y[i] *= p.scale * in;
        }
#pragma unroll
        for (int s = 0; s < C / 32; ++s) {
            const Frag<NX> f = split<NX>(join(X[2 * s], X[2 * s + 1]));
#pragma unroll
            for (int i = 2 * s; i < RT; ++i)
                mma(U[i], m.inv.frag(16 * i, s), f);
        }
        if constexpr (SAVE) {
            float *out = p.chunk_u + (slot * p.hv + h) * C * (int64_t)p.dvp + c0;
            if (c0 < p.dvp) {
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        out[(int64_t)(16 * i + row4 + r) * p.dvp] = U[i][r];
            }
        }
        __syncthreads();  // P is there
        const float all = m.d.all;
#pragma unroll
        for (int i = 0; i < KT; ++i)
            S[i] *= all;
#pragma unroll
        for (int s = 0; s < C / 32; ++s) {
            const Frag<NX> f = split<NX>(join(U[2 * s], U[2 * s + 1]));
#pragma unroll
            for (int i = 2 * s; i < RT; ++i)
                mma(Y[i], m.P.frag(16 * i, s), f);
            const Frag<NX> w = split<NX>(join(U[2 * s] * m.d.four(m.d.out, 32 * s + row4), U[2 * s + 1] * m.d.four(m.d.out, 32 * s + 16 + row4)));
#pragma unroll
            for (int i = 0; i < KT; ++i)
                mma(S[i], m.Kt.frag(16 * i, s), w);
        }
        if (live) {
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = 16 * i + row4 + r;
                    if (row < left)
                        ((T *)p.o)[((t + row) * p.hv + h) * p.dv + c0] = (T)Y[i][r];
                }
        }
    }
    if (p.state1 && live) {
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * t + row4 + r;
                if (i < p.dk)
                    p.state1[state_at + (int64_t)i * p.dv + c0] = S[t][r];
            }
    }
}

template <typename T, int DKP>
static la_status scan_t(DeltaArgs &p, bool save, hipStream_t st)
{
    constexpr int NW = 4;
    if (p.slots > 0)
        LA_LAUNCH((k_delta_inverse<T, DKP>), dim3((unsigned)(p.slots * p.hv)), dim3(64), 0, st, p);
    p.slices = (p.dv + 16 * NW - 1) / (16 * NW);
    const dim3 grid((unsigned)(p.batch * p.hv * p.slices));
    if (save)
        LA_LAUNCH((k_delta_scan<T, DKP, NW, true>), grid, dim3(64 * NW), 0, st, p);
    else
        LA_LAUNCH((k_delta_scan<T, DKP, NW, false>), grid, dim3(64 * NW), 0, st, p);
    return launch_check("delta rule");
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
// once, which is what bounds the call.  A block takes 32 columns of one state, its lanes packs of VEC columns by rows; all loads of a lane are in
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

static int chunk_of(la_dtype dt) { return dt == LA_BF16 ? DeltaIn<bf16_t>::C : dt == LA_F16 ? DeltaIn<f16_t>::C : DeltaIn<float>::C; }

struct DeltaSizes {
    int64_t slots = 0, all = 0;  // chunks, tokens of all sequences
    int c = 0, dkp = 0, dvp = 0;
    size_t inv = 0, state = 0, u = 0;  // bytes of the arrays by slot and value head
    size_t saved() const { return inv + state + u; }
    size_t grad() const { return state + u; }  // the state's gradient, Z's gradient
};

static la_status delta_sizes(la_dtype dt, int64_t batch, int64_t tokens, int hk, int hv, int dk, int dv, bool packed, DeltaSizes &z)
{
    if (unknown_dtype(dt) || batch < 0 || tokens < 0 || hk < 1 || hv < 1 || dk < 1 || dv < 1 || hv % hk)
        return LA_ERR_INVALID_ARG;
    if (dt == LA_F64 || dk > DELTA_MAX_DK || dv > DELTA_MAX_DV)
        return LA_ERR_UNSUPPORTED;
    constexpr int64_t most = 0x7fffffff;
    if (batch > most || tokens > most || (!packed && batch && tokens > most / batch))
        return LA_ERR_UNSUPPORTED;
    z.c = chunk_of(dt);
    z.dkp = dk <= 64 ? 64 : 128;
    z.dvp = (dv + 31) / 32 * 32;
    z.all = packed ? tokens : batch * tokens;
    z.slots = batch == 0 ? 0 : packed ? tokens / z.c + batch : batch * ((tokens + z.c - 1) / z.c);
    if (z.slots > most / hv || batch > most / hv / ((dv + 15) / 16))  // blocks of one launch
        return LA_ERR_UNSUPPORTED;
    const size_t heads = (size_t)z.slots * hv;
    z.inv = align_up(heads * z.c * z.c * 4);
    z.state = align_up(heads * z.dkp * z.dvp * 4);
    z.u = align_up(heads * z.c * z.dvp * 4);
    return LA_OK;
}

static void place_saved(DeltaArgs &p, const DeltaSizes &z, void *base)
{
    char *at = (char *)base;
    p.inv = (float *)at;
    p.chunk_state = (float *)(at + z.inv);
    p.chunk_u = (float *)(at + z.inv + z.state);
}

la_status launch_delta_backward(la_dtype dt, DeltaArgs p, hipStream_t st);

}  // namespace la

using namespace la;

extern "C" {

size_t la_delta_rule_workspace_bytes(la_dtype dt, int64_t batch, int64_t tokens, int hk, int hv, int dk, int dv, int packed)
{
    DeltaSizes z;
    return delta_sizes(dt, batch, tokens, hk, hv, dk, dv, packed, z) == LA_OK ? z.inv : 0;
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
    const size_t es = bytes_of(dt), ob = (size_t)z.all * hv * dv * es, sb = (size_t)batch * hv * dk * dv * 4;
    if (z.all && (!q || !k || !v || !g || !beta || !o))
        return LA_ERR_INVALID_ARG;
    const size_t qs = z.all ? ((size_t)(z.all - 1) * ldq + (size_t)hk * dk) * es : 0, ks = z.all ? ((size_t)(z.all - 1) * ldk + (size_t)hk * dk) * es : 0,
                 vs = z.all ? ((size_t)(z.all - 1) * ldv + (size_t)hv * dv) * es : 0, gs = (size_t)z.all * hv * 4;
    if (overlaps(o, ob, q, qs) || overlaps(o, ob, k, ks) || overlaps(o, ob, v, vs) || overlaps(o, ob, g, gs) || overlaps(o, ob, beta, gs) ||
        overlaps(o, ob, initial_state, sb) || overlaps(o, ob, state, sb) || (state != initial_state && overlaps(state, sb, initial_state, sb)) ||
        overlaps(state, sb, q, qs) || overlaps(state, sb, k, ks) || overlaps(state, sb, v, vs) || overlaps(state, sb, g, gs) || overlaps(state, sb, beta, gs))
        return LA_ERR_INVALID_ARG;
    DeltaArgs p{q, k, v, ldq, ldk, ldv, g, beta, initial_state, offsets, batch, tokens, hk, hv, dk, dv, (float)scale, o, state};
    p.slots = z.slots;
    p.dvp = z.dvp;
    void *base = saved ? saved : workspace;
    const size_t need = saved ? z.saved() : z.inv, given = saved ? saved_bytes : workspace_bytes;
    LA_TRY(check_workspace(base, given, need, saved ? "la_delta_rule_saved_bytes" : "la_delta_rule_workspace_bytes"));
    if (overlaps(base, need, q, qs) || overlaps(base, need, k, ks) || overlaps(base, need, v, vs) || overlaps(base, need, o, ob) ||
        overlaps(base, need, state, sb) || overlaps(base, need, initial_state, sb) || overlaps(base, need, g, gs) || overlaps(base, need, beta, gs))
        return LA_ERR_INVALID_ARG;
    place_saved(p, z, base);
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
    if (z.all && (!q || !k || !v || !g || !beta || !o_bar || !q_bar || !k_bar || !v_bar || !g_bar || !beta_bar))
        return LA_ERR_INVALID_ARG;
    const size_t es = bytes_of(dt), ob = (size_t)z.all * hv * dv * es, qb = (size_t)z.all * hk * dk * es, gb = (size_t)z.all * hv * 4,
                 sb = (size_t)batch * hv * dk * dv * 4;
    const size_t qs = z.all ? ((size_t)(z.all - 1) * ldq + (size_t)hk * dk) * es : 0, ks = z.all ? ((size_t)(z.all - 1) * ldk + (size_t)hk * dk) * es : 0,
                 vs = z.all ? ((size_t)(z.all - 1) * ldv + (size_t)hv * dv) * es : 0;
    const struct {
        const void *p;
        size_t n;
    } in[] = {{q, qs}, {k, ks}, {v, vs}, {g, gb}, {beta, gb}, {o_bar, ob}, {initial_state, sb}, {state_bar, sb}, {saved, saved_bytes}},
      out[] = {{q_bar, qb}, {k_bar, qb}, {v_bar, ob}, {g_bar, gb}, {beta_bar, gb}, {initial_state_bar, sb}};
    for (int i = 0; i < 6; ++i) {
        for (const auto &x : in)
            if (overlaps(out[i].p, out[i].n, x.p, x.n))
                return LA_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (overlaps(out[i].p, out[i].n, out[j].p, out[j].n))
                return LA_ERR_INVALID_ARG;
    }
    if (saved) {
        LA_TRY(check_workspace(saved, saved_bytes, z.saved(), "la_delta_rule_saved_bytes"));
    }
    const size_t need = la_delta_rule_backward_workspace_bytes(dt, batch, tokens, hk, hv, dk, dv, offsets != nullptr, saved != nullptr);
    LA_TRY(check_workspace(workspace, workspace_bytes, need, "la_delta_rule_backward_workspace_bytes"));
    for (const auto &x : in)
        if (overlaps(workspace, need, x.p, x.n))
            return LA_ERR_INVALID_ARG;
    for (const auto &x : out)
        if (overlaps(workspace, need, x.p, x.n))
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
        place_saved(p, z, (void *)saved);
    } else {  // the forward pass again; its answers go to scratch
        place_saved(p, z, at);
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
    if (batch > 0x7fffffff / hv / ((dv + 31) / 32))
        return LA_ERR_UNSUPPORTED;
    const size_t es = bytes_of(dt), ob = (size_t)batch * hv * dv * es, sb = (size_t)slots * hv * dk * dv * 4, gb = (size_t)batch * hv * 4;
    const size_t qs = ((size_t)(batch - 1) * ldq + (size_t)hk * dk) * es, ks = ((size_t)(batch - 1) * ldk + (size_t)hk * dk) * es,
                 vs = ((size_t)(batch - 1) * ldv + (size_t)hv * dv) * es;
    const struct {
        const void *p;
        size_t n;
    } in[] = {{q, qs}, {k, ks}, {v, vs}, {g, gb}, {beta, gb}, {slot, (size_t)batch * 4}};
    for (const auto &x : in)
        if (overlaps(o, ob, x.p, x.n) || overlaps(state, sb, x.p, x.n))
            return LA_ERR_INVALID_ARG;
    if (overlaps(o, ob, state, sb))
        return LA_ERR_INVALID_ARG;
    DeltaStepArgs p{q, k, v, ldq, ldk, ldv, g, beta, state, slot, slots, hk, hv, dk, dv, 0, (float)scale, o};
    hipStream_t st = (hipStream_t)stream;
    return dt == LA_F32 ? step_t<float>(p, batch, st) : dt == LA_BF16 ? step_t<bf16_t>(p, batch, st) : step_t<f16_t>(p, batch, st);
}

}  // extern "C"
