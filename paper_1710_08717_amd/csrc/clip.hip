// The norm over all gradients of a model, and the gradients scaled to a largest norm.
//
//   norm = sqrt(sum over all tensors of x^2),   out = x min(1, max_norm / norm);  factor 1 where the norm, as it is written out, is not finite (or zero)
//
// Two passes over the data, since the factor is known after the first only: bound by memory.  Squares are summed in 64 bits, which those of float's largest and
// smallest numbers fit (not so in 32); doubles whose squares do not are scaled into sums of their own.  The order of the sums depends on sizes and addresses'
// alignment alone.  A launch takes the pointers of up to
// CLIP_TENSORS tensors among its arguments, so that no table is copied to the device.  290 tensors of 200 million elements, matrices in bf16: the squares of 400 MB
// in 108 us (3.7 TB/s: the conversions to 64 bits stand beside the loads), the scaling of 800 MB in 148 us (5.4 TB/s), each in three launches; 24 tensors of
// 20 thousand elements: 4.2 and 5.5 us.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "layer.hpp"
#include "lowp.hpp"

namespace la {

constexpr int CLIP_TENSORS = 112;     // (the arguments stay below 4096 bytes)
constexpr int CLIP_TILE = 8192;       // elements that a block takes at a time
constexpr int CLIP_BLOCKS = 1024;     // of one launch

struct ClipArgs {
    const void *src[CLIP_TENSORS];
    void *dst[CLIP_TENSORS];
    int64_t n[CLIP_TENSORS];
    uint32_t first[CLIP_TENSORS + 1];  // the first tile of each tensor in this launch; last: their count
    uint8_t type[CLIP_TENSORS];
    int count;
    int parts;       // partial sums of all launches
    double *part;    // the whole array; with `wide` two more behind it, of large and of small doubles
    int wide;        // whether any tensor is of doubles
    int part0;       // where this launch's partial sums start
    double max_norm;
    void *norm;      // written by the first launch of the second pass
    int norm64;
};
static_assert(sizeof(ClipArgs) <= 4096, "kernel arguments");

// (a box for each WHICH: sums one after another need no barrier in between)
template <int WHICH>
__device__ __forceinline__ double block_sum(double x)
{
    __shared__ double box[4];
    x = wave_sum(x);
    if (threadIdx.x % 64 == 0)
        box[threadIdx.x / 64] = x;
    __syncthreads();
    return box[0] + box[1] + box[2] + box[3];
}

// A lane's sum of squares: in `mid` of numbers between 2^-480 and 2^480 and of zeros, so that neither one square nor the sum of 2^63 of them leaves the range; larger
// and smaller ones, doubles only, by 2^-600 and 2^600.  A NaN is in one of them.
struct Squares {
    double mid = 0, large = 0, small = 0;
    __device__ __forceinline__ void add(float x) { mid += (double)x * (double)x; }
    __device__ __forceinline__ void add(double x)
    {
        const double size = fabs(x);
        if (size > 0x1p480)
            large += (x * 0x1p-600) * (x * 0x1p-600);
        else if (size < 0x1p-480)
            small += (x * 0x1p600) * (x * 0x1p600);
        else
            mid += x * x;
    }
    // the root of the sum of all
    __device__ __forceinline__ double norm() const
    {
        if (large != 0)
            return sqrt(large + mid * 0x1p-600 * 0x1p-600) * 0x1p600;
        if (mid != 0)
            return sqrt(mid + small * 0x1p-600 * 0x1p-600);
        return sqrt(small) * 0x1p-600;
    }
};

// The tensor of a tile: the last one whose first tile is not past it.
__device__ __forceinline__ int tensor_of(const ClipArgs &a, uint32_t tile)
{
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (a.first[mid] <= tile)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// One tile of a tensor, f(first, count elements at p) in packs of 16 bytes where they start on one, one element at a time before and after.
// `lead`: elements before the first whole pack of the tensor.
template <typename T>
__device__ __forceinline__ void tile_squares(Squares &s, const T *p, int64_t n, uint32_t tile)
{
    constexpr int VEC = 16 / sizeof(T);
    const int64_t lead = (int64_t)((16 - ((uintptr_t)p & 15)) & 15) / sizeof(T);
    const int64_t from = tile ? lead + (int64_t)tile * CLIP_TILE : 0, to0 = lead + ((int64_t)tile + 1) * CLIP_TILE, to = to0 < n ? to0 : n;
    int64_t at = tile ? from : (lead < n ? lead : n);
    if (!tile && threadIdx.x < at)
        s.add((acc_of<T>)p[threadIdx.x]);
    const int64_t packs = to > at ? (to - at) / VEC : 0;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < packs; i += 256) {
        acc_of<T> v[VEC];
        load_pack<T, VEC>(p + at + i * VEC, v);
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            s.add(v[j]);
    }
    at += packs * VEC;
    if (at + threadIdx.x < to)
        s.add((acc_of<T>)p[at + threadIdx.x]);
}

__global__ __launch_bounds__(256) void k_grad_squares(const ClipArgs a)
{
    Squares s;
    for (uint32_t t = blockIdx.x; t < a.first[a.count]; t += gridDim.x) {
        const int k = tensor_of(a, t);
        const uint32_t tile = t - a.first[k];
        switch (a.type[k]) {
        case LA_F32: tile_squares(s, (const float *)a.src[k], a.n[k], tile); break;
        case LA_F64: tile_squares(s, (const double *)a.src[k], a.n[k], tile); break;
        case LA_BF16: tile_squares(s, (const bf16_t *)a.src[k], a.n[k], tile); break;
        default: tile_squares(s, (const f16_t *)a.src[k], a.n[k], tile); break;
        }
    }
    const int at = a.part0 + blockIdx.x;
    const double mid = block_sum<0>(s.mid);
    if (threadIdx.x == 0)
        a.part[at] = mid;
    if (a.wide) {
        const double large = block_sum<1>(s.large), small = block_sum<2>(s.small);
        if (threadIdx.x == 0) {
            a.part[a.parts + at] = large;
            a.part[2 * a.parts + at] = small;
        }
    }
}

template <typename T>
__device__ __forceinline__ void tile_scale(const ClipArgs &a, const T *p, T *q, int64_t n, uint32_t tile, double factor, double norm)
{
    using A = acc_of<T>;
    constexpr int VEC = 16 / sizeof(T);
    const A f = (A)factor;
    // a factor below A's smallest normal number has few bits in A, and the largest elements times it may not be small: elements divided by 2^100 in 64 bits (which no
    // product above the smallest number of T notices) times the factor times 2^100
    const bool denormal = a.max_norm > 0 && factor < (sizeof(A) == 8 ? 0x1p-1022 : 0x1p-126);
    const int64_t lead = (int64_t)((16 - ((uintptr_t)p & 15)) & 15) / sizeof(T);
    const int64_t to0 = lead + ((int64_t)tile + 1) * CLIP_TILE, to = to0 < n ? to0 : n;
    int64_t at = tile ? lead + (int64_t)tile * CLIP_TILE : 0;
    if (denormal) {
        const double g = a.max_norm / (norm * 0x1p-100);
        for (int64_t i = at + threadIdx.x; i < to; i += 256)
            q[i] = (T)(A)((double)(A)p[i] * 0x1p-100 * g);
        return;
    }
    if (((uintptr_t)p & 15) != ((uintptr_t)q & 15)) {  // no pack starts on 16 bytes in both: by elements (200 million of bf16: 509 us for both passes, else 225)
        for (int64_t i = at + threadIdx.x; i < to; i += 256)
            q[i] = (T)((A)p[i] * f);
        return;
    }
    if (!tile) {
        at = lead < n ? lead : n;
        if (threadIdx.x < at)
            q[threadIdx.x] = (T)((A)p[threadIdx.x] * f);
    }
    const int64_t packs = to > at ? (to - at) / VEC : 0;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < packs; i += 256) {
        A v[VEC];
        load_pack<T, VEC>(p + at + i * VEC, v);
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            v[j] *= f;
        store_pack<T, VEC>(q + at + i * VEC, v);
    }
    at += packs * VEC;
    if (at + threadIdx.x < to)
        q[at + threadIdx.x] = (T)((A)p[at + threadIdx.x] * f);
}

// Every block sums the partial sums itself, in the same order: no launch in between.
__global__ __launch_bounds__(256) void k_grad_scale(const ClipArgs a)
{
    Squares s;
    for (int i = threadIdx.x; i < a.parts; i += 256)
        s.mid += a.part[i];
    s.mid = block_sum<0>(s.mid);
    if (a.wide) {
        for (int i = threadIdx.x; i < a.parts; i += 256) {
            s.large += a.part[a.parts + i];
            s.small += a.part[2 * a.parts + i];
        }
        s.large = block_sum<1>(s.large);
        s.small = block_sum<2>(s.small);
    }
    const double norm = s.norm();
    const double seen = a.norm64 ? norm : (double)(float)norm;  // (what the caller tells by that nothing was scaled)
    const double factor = norm > a.max_norm && seen < INFINITY ? a.max_norm / norm : 1.0;
    if (a.part0 == 0 && blockIdx.x == 0 && threadIdx.x == 0) {
        if (a.norm64)
            *(double *)a.norm = norm;
        else
            *(float *)a.norm = (float)norm;
    }
    for (uint32_t t = blockIdx.x; t < a.first[a.count]; t += gridDim.x) {
        const int k = tensor_of(a, t);
        if (factor == 1.0 && a.src[k] == a.dst[k])
            continue;
        const uint32_t tile = t - a.first[k];
        switch (a.type[k]) {
        case LA_F32: tile_scale(a, (const float *)a.src[k], (float *)a.dst[k], a.n[k], tile, factor, norm); break;
        case LA_F64: tile_scale(a, (const double *)a.src[k], (double *)a.dst[k], a.n[k], tile, factor, norm); break;
        case LA_BF16: tile_scale(a, (const bf16_t *)a.src[k], (bf16_t *)a.dst[k], a.n[k], tile, factor, norm); break;
        default: tile_scale(a, (const f16_t *)a.src[k], (f16_t *)a.dst[k], a.n[k], tile, factor, norm); break;
        }
    }
}

static int64_t tiles_of(int64_t n) { return n > 0 ? (n + CLIP_TILE - 1) / CLIP_TILE : 0; }

// Calls f(tensors [i, j), their tiles) for each launch: up to CLIP_TENSORS tensors and fewer than 2^31 tiles.
template <class F>
static la_status clip_launches(int count, const int64_t *sizes, F &&f)
{
    for (int i = 0; i < count;) {
        int j = i, used = 0;
        int64_t tiles = 0;
        while (j < count && used < CLIP_TENSORS && tiles + tiles_of(sizes[j]) < 0x7fffffff) {
            tiles += tiles_of(sizes[j]);
            used += sizes[j] > 0;
            ++j;
        }
        if (j == i)
            return LA_ERR_UNSUPPORTED;  // (one tensor of 2^31 tiles)
        LA_TRY(f(i, j, tiles));
        i = j;
    }
    return LA_OK;
}

// LA_ERR_INVALID_ARG where an output overlaps another gradient or another output: its elements would be scaled twice, or read by one block after another
// has scaled them.  In order of their addresses, tensors overlap an earlier one where its end lies behind their start.  Outputs and what is only read are put in
// order by themselves, since views of one buffer are so already (290 tensors: 4 us on the host then, 10 in random order).
static la_status clip_overlaps(int count, const la_dtype *types, const int64_t *sizes, const void *const *grads, void *const *out)
{
    struct Tensor {
        uintptr_t from, to;
        bool operator<(const Tensor &t) const { return from < t.from; }
    };
    constexpr int FEW = 64;
    Tensor few[2 * FEW];
    std::unique_ptr<Tensor[]> many;
    if (count > FEW) {
        many.reset(new (std::nothrow) Tensor[2 * (size_t)count]);
        if (!many) {
            set_error_text("clip: no host memory");
            return LA_ERR_RUNTIME;
        }
    }
    Tensor *const written = many ? many.get() : few, *const read = written + count;
    int writes = 0, reads = 0;
    for (int i = 0; i < count; ++i) {
        const size_t b = (size_t)sizes[i] * bytes_of(types[i]);
        if (!b)
            continue;
        written[writes++] = {(uintptr_t)out[i], (uintptr_t)out[i] + b};
        if (grads[i] != out[i])
            read[reads++] = {(uintptr_t)grads[i], (uintptr_t)grads[i] + b};
    }
    if (!std::is_sorted(written, written + writes))
        std::sort(written, written + writes);
    if (!std::is_sorted(read, read + reads))
        std::sort(read, read + reads);
    uintptr_t end_read = 0, end_written = 0;
    for (int w = 0, r = 0; w < writes;) {
        if (r < reads && read[r] < written[w]) {
            if (read[r].from < end_written)
                return LA_ERR_INVALID_ARG;
            end_read = std::max(end_read, read[r++].to);
        } else {
            if (written[w].from < std::max(end_read, end_written))
                return LA_ERR_INVALID_ARG;
            end_written = written[w++].to;
        }
        if (w == writes && r < reads && read[r].from < end_written)
            return LA_ERR_INVALID_ARG;
    }
    return LA_OK;
}

static int clip_blocks(int64_t tiles) { return (int)(tiles < 1 ? 1 : tiles < CLIP_BLOCKS ? tiles : CLIP_BLOCKS); }

}  // namespace la

using namespace la;

extern "C" {

size_t la_clip_gradients_workspace_bytes(int count, const int64_t *sizes)
{
    if (count <= 0 || !sizes)
        return 0;
    size_t parts = 0;
    for (int i = 0; i < count; ++i)
        if (sizes[i] < 0)
            return 0;
    if (clip_launches(count, sizes, [&](int, int, int64_t tiles) {
            parts += clip_blocks(tiles);
            return LA_OK;
        }) != LA_OK)
        return 0;
    return align_up(3 * parts * sizeof(double));  // (the types are not known here)
}

la_status la_clip_gradients(int count, const la_dtype *types, const int64_t *sizes, const void *const *grads, void *const *out, double max_norm,
                            la_dtype norm_type, void *norm, void *workspace, size_t workspace_bytes, void *stream)
{
    if (count < 0 || !(max_norm >= 0) || (norm_type != LA_F32 && norm_type != LA_F64) || !norm)
        return LA_ERR_INVALID_ARG;
    hipStream_t st = (hipStream_t)stream;
    if (count == 0)
        return zero_bytes(norm, bytes_of(norm_type), st);
    if (!types || !sizes || !grads || !out)
        return LA_ERR_INVALID_ARG;
    for (int i = 0; i < count; ++i) {
        if (unknown_dtype(types[i]) || sizes[i] < 0)
            return LA_ERR_INVALID_ARG;
        const size_t b = (size_t)sizes[i] * bytes_of(types[i]);
        if (b && (!grads[i] || !out[i] || (uintptr_t)grads[i] % bytes_of(types[i]) || (uintptr_t)out[i] % bytes_of(types[i]) ||
                  (grads[i] != out[i] && overlaps(grads[i], b, out[i], b)) || overlaps(norm, bytes_of(norm_type), out[i], b) || overlaps(norm, bytes_of(norm_type), grads[i], b)))
            return LA_ERR_INVALID_ARG;
    }
    LA_TRY(clip_overlaps(count, types, sizes, grads, out));
    const size_t need = la_clip_gradients_workspace_bytes(count, sizes);
    if (!need)
        return LA_ERR_UNSUPPORTED;
    LA_TRY(check_workspace(workspace, workspace_bytes, need, "la_clip_gradients_workspace_bytes"));
    for (int i = 0; i < count; ++i)
        if (any_overlap({{grads[i], (size_t)sizes[i] * bytes_of(types[i])}, {out[i], (size_t)sizes[i] * bytes_of(types[i])}, {norm, bytes_of(norm_type)}},
                        {{workspace, need}}))
            return LA_ERR_INVALID_ARG;
    ClipArgs a;
    a.part = (double *)workspace;
    a.max_norm = max_norm;
    a.norm = norm;
    a.norm64 = norm_type == LA_F64;
    a.wide = 0;
    for (int i = 0; i < count; ++i)
        a.wide |= types[i] == LA_F64;
    a.parts = 0;
    LA_TRY(clip_launches(count, sizes, [&](int, int, int64_t tiles) {
        a.parts += clip_blocks(tiles);
        return LA_OK;
    }));
    for (int pass = 0; pass < 2; ++pass) {
        a.part0 = 0;
        LA_TRY(clip_launches(count, sizes, [&](int i, int j, int64_t tiles) {
            a.count = 0;
            uint32_t at = 0;
            for (; i < j; ++i) {
                if (sizes[i] == 0)
                    continue;
                a.src[a.count] = grads[i];
                a.dst[a.count] = out[i];
                a.n[a.count] = sizes[i];
                a.type[a.count] = (uint8_t)types[i];
                a.first[a.count++] = at;
                at += (uint32_t)tiles_of(sizes[i]);
            }
            a.first[a.count] = at;
            const int blocks = clip_blocks(tiles);
            if (pass == 0)
                LA_LAUNCH(k_grad_squares, dim3(blocks), dim3(256), 0, st, a);
            else
                LA_LAUNCH(k_grad_scale, dim3(blocks), dim3(256), 0, st, a);
            a.part0 += blocks;
            return launch_check("clip");
        }));
    }
    return LA_OK;
}

}  // extern "C"
