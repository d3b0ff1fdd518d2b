// Layer norm of rows, and its gradient.
//
//   y = h w + c,  h = (x - mean) rstd,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   x_bar = rstd (t - mean(t) - h mean(t h)),  t = y_bar w;   w_bar = sum over rows of y_bar h;   c_bar = sum over rows of y_bar
//
// A row stays in the registers of the lanes that read it, so that the mean, the squares about it and the result cost one read of memory;
// statistics and sums are held in 32 bits (64 for double).  Both kernels are bound by memory.
#include "common.hpp"
#include "layer.hpp"
#include "lowp.hpp"

namespace la {

struct NormArgs {
    const void *x;
    int64_t ldx;
    const void *w, *c;  // weight and bias, or null
    int w32;            // weight and bias are float where x is 16 bits wide
    const void *yb;     // (gradient)
    void *y;            // y, or x_bar
    void *mean, *rstd;  // written by the forward pass (or null), read by the gradient
    void *part;         // (gradient) [blocks][2][n] partial sums of w_bar and c_bar
    int64_t rows;
    int n;
    double eps;
};

// the sum of a and of b over the TPR lanes that share a row; `turn` alternates between calls, so that one barrier a call is enough
template <int TPR, typename A>
__device__ __forceinline__ void row_sums(A &a, A &b, int turn)
{
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (TPR > 64) {
        constexpr int NW = TPR / 64;
        __shared__ A box[2][2][NW];
        const int w = threadIdx.x / 64;
        if (threadIdx.x % 64 == 0) {
            box[turn][0][w] = a;
            box[turn][1][w] = b;
        }
        __syncthreads();
        a = b = A(0);
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            a += box[turn][0][i];
            b += box[turn][1][i];
        }
    }
}

// N elements of the weight or the bias, those past `n` as zeros
template <typename T, int N>
__device__ __forceinline__ void load_weight(const void *w, int w32, int col, int n, acc_of<T> (&v)[N])
{
    if (sizeof(T) == 2 && w32) {
        float f[N];
        load_part<float, N>((const float *)w + col, n, f);
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = f[i];
    } else {
        load_part<T, N>((const T *)w + col, n, v);
    }
}

// TPR lanes a row, R packs of 16 bytes a lane; the row's last pack may be a part of one, and rows may start anywhere.  16384 x 4096, bf16: 268 MB in 57 us, 4.7 TB/s;
// 4099 x 1023, f32, whose rows start on no alignment: 34 MB in 11 us; 16 x 2048, bf16: 4 us, a launch.
template <typename T, int TPR, int R>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_layer_norm(NormArgs p)
{
    using A = acc_of<T>;
    constexpr int NT = TPR < 256 ? 256 : TPR, VEC = 16 / sizeof(T);
    const int lane = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (NT / TPR) + threadIdx.x / TPR;
    if (row >= p.rows)
        return;  // (a whole wavefront: no barrier where a block holds several rows)
    const T *x = (const T *)p.x + row * p.ldx;
    T *y = (T *)p.y + row * p.n;
    A v[R][VEC], sum = 0, none = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int col = (r * TPR + lane) * VEC;
        load_part<T, VEC>(x + col, p.n - col, v[r]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            sum += v[r][i];
    row_sums<TPR>(sum, none, 0);
    const A mean = sum / p.n;
    A sq = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int left = p.n - (r * TPR + lane) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const A d = i < left ? v[r][i] - mean : A(0);
            sq += d * d;
        }
    }
    row_sums<TPR>(sq, none, 1);
    const A rstd = A(1) / sqrt(sq / p.n + (A)p.eps);
    if (lane == 0 && p.mean) {
        ((A *)p.mean)[row] = mean;
        ((A *)p.rstd)[row] = rstd;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int col = (r * TPR + lane) * VEC, left = p.n - col;
        if (left > 0) {
            A w[VEC], c[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                w[i] = 1;
                c[i] = 0;
            }
            if (p.w)
                load_weight<T, VEC>(p.w, p.w32, col, left, w);
            if (p.c)
                load_weight<T, VEC>(p.c, p.w32, col, left, c);
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                v[r][i] = (v[r][i] - mean) * rstd * w[i] + c[i];
            store_part<T, VEC>(y + col, left, v[r]);
        }
    }
}

// A block takes every gridDim.x-th group of rows and keeps its part of w_bar and c_bar in registers: a lane's columns are the same in every row.  The next
// row is loaded before this one's sums are joined.  16384 x 4096, bf16: 403 MB in 87 us, 4.6 TB/s, and 7 us for the parts; 4099 x 1023, f32: 50 MB in 13 us and 5.
template <typename T, int TPR, int R>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_layer_norm_back(NormArgs p)
{
    using A = acc_of<T>;
    constexpr int NT = TPR < 256 ? 256 : TPR, GROUPS = NT / TPR, VEC = 16 / sizeof(T);
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const A inv_n = A(1) / p.n;
    A w[R][VEC], wb[R][VEC], cb[R][VEC];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int col = (r * TPR + lane) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            w[r][i] = 1;
            wb[r][i] = cb[r][i] = 0;
        }
        if (p.w)
            load_weight<T, VEC>(p.w, p.w32, col, p.n - col, w[r]);
    }
    typename PackOf<T, VEC>::whole xr[R], yr[R];
    A mean = 0, rstd = 0;
    auto fetch = [&](int64_t row) {
        const T *x = (const T *)p.x + row * p.ldx, *yb = (const T *)p.yb + row * p.n;
        mean = ((const A *)p.mean)[row];
        rstd = ((const A *)p.rstd)[row];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int col = (r * TPR + lane) * VEC;
            xr[r] = load_raw<T, VEC>(x + col, p.n - col);
            yr[r] = load_raw<T, VEC>(yb + col, p.n - col);
        }
    };
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t row = (int64_t)blockIdx.x * GROUPS + group;
    if (row < p.rows)
        fetch(row);
    int turn = 0;
    for (; row < p.rows; row += step, turn ^= 1) {
        A h[R][VEC], g[R][VEC], s = 0, q = 0;
        const A scale = rstd;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {  // (past the row's end y_bar is zero)
                h[r][i] = ((A)xr[r][i] - mean) * scale;
                g[r][i] = (A)yr[r][i];
            }
        if (row + step < p.rows)
            fetch(row + step);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                wb[r][i] += g[r][i] * h[r][i];
                cb[r][i] += g[r][i];
                g[r][i] *= w[r][i];
                s += g[r][i];
                q += g[r][i] * h[r][i];
            }
        row_sums<TPR>(s, q, turn);
        s *= inv_n;
        q *= inv_n;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int col = (r * TPR + lane) * VEC;
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                g[r][i] = scale * (g[r][i] - s - h[r][i] * q);
            store_part<T, VEC>((T *)p.y + row * p.n + col, p.n - col, g[r]);
        }
    }
    A *part = (A *)p.part + (int64_t)blockIdx.x * 2 * p.n;
    if constexpr (GROUPS > 1) {  // the groups' sums in their order
        __shared__ A box[GROUPS - 1][2][TPR * VEC * R];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (group > 0) {
                    box[group - 1][0][(r * VEC + i) * TPR + lane] = wb[r][i];
                    box[group - 1][1][(r * VEC + i) * TPR + lane] = cb[r][i];
                }
        __syncthreads();
        if (group > 0)
            return;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                for (int k = 0; k < GROUPS - 1; ++k) {
                    wb[r][i] += box[k][0][(r * VEC + i) * TPR + lane];
                    cb[r][i] += box[k][1][(r * VEC + i) * TPR + lane];
                }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int col = (r * TPR + lane) * VEC;
        store_part<A, VEC>(part + col, p.n - col, wb[r]);
        store_part<A, VEC>(part + p.n + col, p.n - col, cb[r]);
    }
}

// w_bar and c_bar from the blocks' parts: 32 columns a block, 32 runs of parts side by side, joined in their order
template <typename A>
__global__ __launch_bounds__(1024) void k_norm_parts(const A *part, int parts, int n, void *wb, void *cb, int type)
{
    __shared__ A box[32][33];
    const int c = threadIdx.x % 32, run = threadIdx.x / 32, col = blockIdx.x * 32 + c;
    void *out = blockIdx.y ? cb : wb;
    if (!out)
        return;
    A s = 0;
    if (col < n) {
        const A *p = part + (int64_t)blockIdx.y * n + col;
#pragma unroll 8
        for (int i = run; i < parts; i += 32)
            s += p[(int64_t)i * 2 * n];
    }
    box[run][c] = s;
    __syncthreads();
    if (run || col >= n)
        return;
#pragma unroll
    for (int k = 1; k < 32; ++k)
        s += box[k][c];
    if (type == LA_BF16)
        ((bf16_t *)out)[col] = (bf16_t)s;
    else if (type == LA_F16)
        ((f16_t *)out)[col] = (f16_t)s;
    else
        ((A *)out)[col] = s;
}

// Rows longer than a block's registers hold: read again for each sum, an element a lane and load.  One block a row.  1024 x 65536, bf16: 206 us, 1.3 TB/s of what the
// formulas need; its gradient, with the columns' sums below: 314 us, 1.3 TB/s.
template <typename T>
__global__ __launch_bounds__(1024) void k_layer_norm_wide(NormArgs p)
{
    using A = acc_of<T>;
    const int64_t row = blockIdx.x;
    const T *x = (const T *)p.x + row * p.ldx;
    A sum = 0, none = 0, sq = 0;
    for (int i = threadIdx.x; i < p.n; i += 1024)
        sum += (A)x[i];
    row_sums<1024>(sum, none, 0);
    const A mean = sum / p.n;
    for (int i = threadIdx.x; i < p.n; i += 1024) {
        const A d = (A)x[i] - mean;
        sq += d * d;
    }
    row_sums<1024>(sq, none, 1);
    const A rstd = A(1) / sqrt(sq / p.n + (A)p.eps);
    if (threadIdx.x == 0 && p.mean) {
        ((A *)p.mean)[row] = mean;
        ((A *)p.rstd)[row] = rstd;
    }
    for (int i = threadIdx.x; i < p.n; i += 1024) {
        A w[1] = {1}, c[1] = {0};
        if (p.w)
            load_weight<T, 1>(p.w, p.w32, i, 1, w);
        if (p.c)
            load_weight<T, 1>(p.c, p.w32, i, 1, c);
        ((T *)p.y)[row * p.n + i] = (T)(((A)x[i] - mean) * rstd * w[0] + c[0]);
    }
}

template <typename T>
__global__ __launch_bounds__(1024) void k_layer_norm_back_wide(NormArgs p)
{
    using A = acc_of<T>;
    const int64_t row = blockIdx.x;
    const T *x = (const T *)p.x + row * p.ldx, *yb = (const T *)p.yb + row * p.n;
    const A mean = ((const A *)p.mean)[row], rstd = ((const A *)p.rstd)[row];
    A s = 0, q = 0;
    for (int i = threadIdx.x; i < p.n; i += 1024) {
        A w[1] = {1};
        if (p.w)
            load_weight<T, 1>(p.w, p.w32, i, 1, w);
        const A t = (A)yb[i] * w[0];
        s += t;
        q += t * (((A)x[i] - mean) * rstd);
    }
    row_sums<1024>(s, q, 0);
    s /= p.n;
    q /= p.n;
    for (int i = threadIdx.x; i < p.n; i += 1024) {
        A w[1] = {1};
        if (p.w)
            load_weight<T, 1>(p.w, p.w32, i, 1, w);
        const A h = ((A)x[i] - mean) * rstd;
        ((T *)p.y)[row * p.n + i] = (T)(rstd * ((A)yb[i] * w[0] - s - h * q));
    }
}

// parts of w_bar and c_bar for wide rows: a lane a column, blockIdx.y a run of rows
template <typename T>
__global__ __launch_bounds__(256) void k_norm_columns_wide(NormArgs p)
{
    using A = acc_of<T>;
    const int col = blockIdx.x * 256 + threadIdx.x;
    if (col >= p.n)
        return;
    A wb = 0, cb = 0;
#pragma unroll 4
    for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
        const A mean = ((const A *)p.mean)[row], rstd = ((const A *)p.rstd)[row];
        const A g = (A)((const T *)p.yb)[row * p.n + col], h = ((A)((const T *)p.x)[row * p.ldx + col] - mean) * rstd;
        wb += g * h;
        cb += g;
    }
    A *part = (A *)p.part + (int64_t)blockIdx.y * 2 * p.n;
    part[col] = wb;
    part[p.n + col] = cb;
}

// Lanes and packs a lane for rows of n elements, by the smallest that holds them.  A wavefront a row needs no barrier, and its rows are many to a block
// (65536 x 1024, bf16, and its gradient: 42 and 60 us, with 256 lanes a row 84 and 99; 16 rows take 4 and 9 us either way).
struct NormShape {
    int tpr, r;
};
static NormShape norm_shape(int n, int size, bool back)
{
    const int vec = 16 / size;
    const int packs = (n + vec - 1) / vec;
    if (packs <= 64)
        return {64, 1};
    if (packs <= 128)
        return {64, 2};
    if (packs <= 256)
        return {256, 1};
    if (packs <= 512)
        return {256, 2};
    if (packs <= 1024)
        return {256, 4};
    // (the gradient holds five numbers for each of a lane's columns: 8 of 16 bits do not fit four times into what 1024 lanes leave each)
    if (packs <= 2048)
        return back ? NormShape{512, 4} : NormShape{1024, 2};
    if (packs <= 4096 && !(back && size == 2))
        return {1024, 4};
    return {0, 0};
}

constexpr int NORM_BLOCKS = 1024;

// Blocks of the gradient's kernel: enough to fill the chip, but 4 rows at least to each, since a block's 2 n sums are written and read once.
static int norm_blocks(int64_t rows, NormShape s)
{
    const int groups = s.tpr && s.tpr < 256 ? 256 / s.tpr : 1;
    const int64_t all = (rows + groups - 1) / groups, most = rows / 4 < 256 ? 256 : rows / 4 < NORM_BLOCKS ? rows / 4 : NORM_BLOCKS;
    return (int)(s.tpr == 0 ? (rows < 64 ? rows : 64) : all < most ? all : most);
}

// A launch has fewer than 2^32 threads: more rows than those serve are taken in pieces, launch(args, blocks) for each.
template <typename T, class F>
static void by_rows(NormArgs p, int rows_of_block, int threads, F &&launch)
{
    const int64_t all = p.rows, most = most_blocks(threads) * rows_of_block;
    const size_t stat = sizeof(acc_of<T>);
    for (int64_t at = 0; at < all; at += most) {
        p.rows = all - at < most ? all - at : most;
        launch(p, (unsigned)((p.rows + rows_of_block - 1) / rows_of_block));
        p.x = (const T *)p.x + most * p.ldx;
        p.y = (T *)p.y + most * p.n;
        p.yb = p.yb ? (const T *)p.yb + most * p.n : nullptr;
        p.mean = p.mean ? (char *)p.mean + most * stat : nullptr;
        p.rstd = p.rstd ? (char *)p.rstd + most * stat : nullptr;
    }
}

template <typename T, int TPR, int R>
static void norm_launch(const NormArgs &p, bool back, hipStream_t st)
{
    constexpr int NT = TPR < 256 ? 256 : TPR, GROUPS = NT / TPR;
    // (what norm_shape gives for one of the two only)
    constexpr bool FORWARD = TPR != 512, BACK = !(TPR == 1024 && (R == 2 || sizeof(T) == 2));
    if constexpr (BACK)
        if (back)
            LA_LAUNCH((k_layer_norm_back<T, TPR, R>), dim3(norm_blocks(p.rows, {TPR, R})), dim3(NT), 0, st, p);
    if constexpr (FORWARD)
        if (!back)
            by_rows<T>(p, GROUPS, NT, [&](const NormArgs &q, unsigned blocks) { LA_LAUNCH((k_layer_norm<T, TPR, R>), dim3(blocks), dim3(NT), 0, st, q); });
}

template <typename T>
static void norm_dispatch(const NormArgs &p, NormShape s, bool back, hipStream_t st)
{
    if (s.tpr == 64 && s.r == 1)
        norm_launch<T, 64, 1>(p, back, st);
    else if (s.tpr == 64)
        norm_launch<T, 64, 2>(p, back, st);
    else if (s.tpr == 256 && s.r == 1)
        norm_launch<T, 256, 1>(p, back, st);
    else if (s.tpr == 256 && s.r == 2)
        norm_launch<T, 256, 2>(p, back, st);
    else if (s.tpr == 256)
        norm_launch<T, 256, 4>(p, back, st);
    else if (s.tpr == 512)
        norm_launch<T, 512, 4>(p, back, st);
    else if (s.r == 2)
        norm_launch<T, 1024, 2>(p, back, st);
    else
        norm_launch<T, 1024, 4>(p, back, st);
}

template <typename T>
static la_status norm_t(const NormArgs &p, bool back, void *wb, void *cb, int wtype, hipStream_t st)
{
    using A = acc_of<T>;
    const NormShape s = norm_shape(p.n, sizeof(T), back);
    int parts = norm_blocks(p.rows, s);
    if (s.tpr) {
        norm_dispatch<T>(p, s, back, st);
    } else if (!back) {
        by_rows<T>(p, 1, 1024, [&](const NormArgs &q, unsigned blocks) { LA_LAUNCH((k_layer_norm_wide<T>), dim3(blocks), dim3(1024), 0, st, q); });
    } else {
        if (wb || cb)  // (first: x_bar may be written over y_bar)
            LA_LAUNCH((k_norm_columns_wide<T>), dim3((p.n + 255) / 256, parts), dim3(256), 0, st, p);
        by_rows<T>(p, 1, 1024, [&](const NormArgs &q, unsigned blocks) { LA_LAUNCH((k_layer_norm_back_wide<T>), dim3(blocks), dim3(1024), 0, st, q); });
    }
    if (back && (wb || cb))
        LA_LAUNCH((k_norm_parts<A>), dim3((p.n + 31) / 32, 2), dim3(1024), 0, st, (const A *)p.part, parts, p.n, wb, cb, wtype);
    return launch_check("layer norm");
}

static la_status norm_any(la_dtype dt, const NormArgs &p, bool back, void *wb, void *cb, int wtype, hipStream_t st)
{
    switch (dt) {
    case LA_F32: return norm_t<float>(p, back, wb, cb, wtype, st);
    case LA_F64: return norm_t<double>(p, back, wb, cb, wtype, st);
    case LA_BF16: return norm_t<bf16_t>(p, back, wb, cb, wtype, st);
    default: return norm_t<f16_t>(p, back, wb, cb, wtype, st);
    }
}

constexpr int64_t NORM_MAX_ROWS = 0x7fffffff;
constexpr int NORM_MAX_N = 1 << 26;            // (columns and the strides over them are int)

static bool norm_sizes_bad(la_dtype dt, la_dtype wdt, int64_t rows, int n, int64_t ldx)
{
    return unknown_dtype(dt) || rows < 0 || n < 0 || ldx < n || !(wdt == dt || (wdt == LA_F32 && small_dtype(dt)));
}

static size_t norm_parts_bytes(la_dtype dt, int64_t rows, int n)
{
    // (the most blocks that any of the shapes above uses)
    const int64_t blocks = rows < NORM_BLOCKS ? rows : NORM_BLOCKS;
    return align_up((size_t)blocks * 2 * n * (dt == LA_F64 ? 8 : 4));
}

}  // namespace la

using namespace la;

extern "C" {

la_status la_layer_norm(la_dtype dt, la_dtype wdt, int64_t rows, int n, int64_t ldx, const void *x, const void *weight, const void *bias, double eps,
                        void *y, void *mean, void *rstd, void *stream)
{
    if (norm_sizes_bad(dt, wdt, rows, n, ldx) || !(eps >= 0))
        return LA_ERR_INVALID_ARG;
    if (rows == 0)
        return LA_OK;
    if (rows > NORM_MAX_ROWS || n > NORM_MAX_N)
        return LA_ERR_UNSUPPORTED;
    if (!mean != !rstd || (n > 0 && (!x || !y)))
        return LA_ERR_INVALID_ARG;
    if (n == 0) {  // rows of nothing
        const size_t b = (size_t)rows * (dt == LA_F64 ? 8 : 4);
        if (overlaps(mean, b, rstd, b))
            return LA_ERR_INVALID_ARG;
        LA_TRY(zero_bytes(mean, b, (hipStream_t)stream));
        return zero_bytes(rstd, b, (hipStream_t)stream);
    }
    const size_t xs = ((size_t)(rows - 1) * ldx + n) * bytes_of(dt), ys = (size_t)rows * n * bytes_of(dt), ws = (size_t)n * bytes_of(wdt),
                 ss = (size_t)rows * (dt == LA_F64 ? 8 : 4);
    if (overlaps(x, xs, y, ys) && !(x == y && ldx == n))
        return LA_ERR_INVALID_ARG;
    if (any_overlap({{weight, ws}, {bias, ws}}, {{y, ys}}) || any_overlap({{x, xs}, {weight, ws}, {bias, ws}, {y, ys}}, {{mean, ss}, {rstd, ss}}))
        return LA_ERR_INVALID_ARG;
    NormArgs p{x, ldx, weight, bias, wdt != dt, nullptr, y, mean, rstd, nullptr, rows, n, eps};
    return norm_any(dt, p, false, nullptr, nullptr, wdt, (hipStream_t)stream);
}

size_t la_layer_norm_backward_workspace_bytes(la_dtype dt, int64_t rows, int n)
{
    if (unknown_dtype(dt) || rows <= 0 || n <= 0 || rows > NORM_MAX_ROWS || n > NORM_MAX_N)
        return 0;
    return norm_parts_bytes(dt, rows, n);
}

la_status la_layer_norm_backward(la_dtype dt, la_dtype wdt, int64_t rows, int n, int64_t ldx, const void *x, const void *y_bar, const void *mean,
                                 const void *rstd, const void *weight, void *x_bar, void *weight_bar, void *bias_bar, void *workspace,
                                 size_t workspace_bytes, void *stream)
{
    if (norm_sizes_bad(dt, wdt, rows, n, ldx))
        return LA_ERR_INVALID_ARG;
    if (n == 0)
        return LA_OK;
    hipStream_t st = (hipStream_t)stream;
    if (rows == 0) {  // empty sums
        LA_TRY(zero_bytes(weight_bar, (size_t)n * bytes_of(wdt), st));
        return zero_bytes(bias_bar, (size_t)n * bytes_of(wdt), st);
    }
    if (rows > NORM_MAX_ROWS || n > NORM_MAX_N)
        return LA_ERR_UNSUPPORTED;
    if (!x || !y_bar || !mean || !rstd || !x_bar)
        return LA_ERR_INVALID_ARG;
    const size_t xs = ((size_t)(rows - 1) * ldx + n) * bytes_of(dt), ys = (size_t)rows * n * bytes_of(dt), ws = (size_t)n * bytes_of(wdt),
                 ss = (size_t)rows * (dt == LA_F64 ? 8 : 4), need = norm_parts_bytes(dt, rows, n);
    if (y_bar != x_bar && overlaps(y_bar, ys, x_bar, ys))
        return LA_ERR_INVALID_ARG;
    if (any_overlap({{x, xs}, {mean, ss}, {rstd, ss}, {weight, ws}}, {{x_bar, ys}, {weight_bar, ws}, {bias_bar, ws}}) ||
        any_overlap({{y_bar, ys}, {x_bar, ys}}, {{weight_bar, ws}, {bias_bar, ws}}))
        return LA_ERR_INVALID_ARG;
    LA_TRY(check_workspace(workspace, workspace_bytes, need, "la_layer_norm_backward_workspace_bytes"));
    if (any_overlap({{x, xs}, {y_bar, ys}, {mean, ss}, {rstd, ss}, {weight, ws}, {x_bar, ys}, {weight_bar, ws}, {bias_bar, ws}}, {{workspace, need}}))
        return LA_ERR_INVALID_ARG;
    NormArgs p{x, ldx, weight, nullptr, wdt != dt, y_bar, x_bar, (void *)mean, (void *)rstd, workspace, rows, n, 0.0};
    return norm_any(dt, p, true, weight_bar, bias_bar, wdt, st);
}

}  // extern "C"
