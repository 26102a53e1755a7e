// Dropout and the root-mean-square norm with its gradients: operators that read and write every row once.
#include "zg_dense.h"

#include <algorithm>
#include <tuple>

namespace zg {
namespace {

constexpr int kRowsBlock = 256;

// ---- dropout --------------------------------------------------------------------------------------------------------------------

struct DropoutArgs {
    Rows rows;
    uint32_t cols, groups; // groups of eight columns to a row
    uint64_t inv;          // ceil(2^32 / groups): e / groups == (e * inv) >> 32 for the small e of a workgroup
    uint32_t per_block;    // rows of a workgroup
    const void *x, *r;
    int64_t ld_x, ld_r;
    void *y;
    int64_t ld_y;
    bool stream;
    Drop drop;
};

// y = m x / (1 - p) + r, eight cells and one Philox call to a lane at a time.  Bound by memory: 285127 x 512 bf16 102 us, 5.7 TB/s (the mask's
// integer instructions take about 90 us of the vector units beside it); 4096 x 601 fp32 with r 7 us, a launch and one way to memory and back.
template <class T> __global__ __launch_bounds__(kRowsBlock) void k_dropout(DropoutArgs a)
{
    const uint32_t live = a.rows.live();
    const uint64_t first = (uint64_t)block_number() * a.per_block;
    if (first >= live) return;
    const uint32_t n = (uint32_t)min((uint64_t)a.per_block, live - first) * a.groups;
    for (uint32_t e = threadIdx.x; e < n; e += kRowsBlock) {
        const uint32_t i = (uint32_t)((e * a.inv) >> 32), g = e - i * a.groups, row = (uint32_t)first + i;
        const int left = (int)(a.cols - 8 * g);
        float v[8];
        load8(static_cast<const T *>(a.x) + row * a.ld_x + 8 * g, left, v);
        if (a.drop.cut) mask8(a.drop, mask_id(a.drop, row), g, a.drop.scale, v);
        if (a.r) {
            float r[8];
            load8(static_cast<const T *>(a.r) + row * a.ld_r + 8 * g, left, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += r[j];
        }
        store8(static_cast<T *>(a.y) + row * a.ld_y + 8 * g, left, v, a.stream);
    }
}

// ---- norm -----------------------------------------------------------------------------------------------------------------------
// A row is held in registers by `PER` lanes, CH groups of eight columns each: by a part of a wavefront, a wavefront, or a workgroup.
// Everything is read once and written once; the sums are trees over the lanes, the same ones whatever the launch.  Bound by memory: 120001 x 1024
// bf16 with residual and dropout 161 us, 6.1 TB/s; 16 x 1024 to 8 bits 4.9 us, a launch and two ways over the lanes.

template <int PER> __device__ __forceinline__ float row_sum(float v, float *lds)
{
#pragma unroll
    for (int m = 1; m < (PER < 64 ? PER : 64); m <<= 1) v += __shfl_xor(v, m);
    if (PER > 64) {
        constexpr int waves = PER / 64;
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < waves; ++w) v += lds[w];
    }
    return v;
}

__device__ __forceinline__ float max_nan(float a, float b) { return a >= b || a != a ? a : b; } // not a number wins

template <int PER> __device__ __forceinline__ float row_max(float v, float *lds)
{
#pragma unroll
    for (int m = 1; m < (PER < 64 ? PER : 64); m <<= 1) v = max_nan(v, __shfl_xor(v, m));
    if (PER > 64) {
        constexpr int waves = PER / 64;
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int w = 1; w < waves; ++w) v = max_nan(v, lds[w]);
    }
    return v;
}

struct NormArgs {
    Rows rows;
    uint32_t cols;
    float inv_cols, eps;
    int32_t out_type;
    bool stream;
    const void *x, *r;
    int64_t ld_x, ld_r;
    const float *gain;
    void *h, *y;
    int64_t ld_h, ld_y;
    float *scale, *rstd;
    Drop drop;
};

// eight values as 8-bit floats, to nearest even; what is beyond 448 becomes 448, not a number stays that
__device__ __forceinline__ void store8_f8(uint8_t *p, int n, const float (&v)[8])
{
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float c[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float x = v[4 * i + j];
            c[j] = x > 448.0f ? 448.0f : x < -448.0f ? -448.0f : x;
        }
        int t = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
        t = __builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], t, true);
        w[i] = (uint32_t)t;
    }
    if (n >= 8) {
        __builtin_memcpy(p, w, 8);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
}

template <class T, int PER, int CH> __global__ __launch_bounds__(PER > kRowsBlock ? PER : kRowsBlock) void k_norm(NormArgs a)
{
    __shared__ float lds[16];
    constexpr int block = PER > kRowsBlock ? PER : kRowsBlock;
    const uint64_t row64 = (uint64_t)block_number() * (block / PER) + threadIdx.x / PER;
    if (row64 >= a.rows.live()) return; // (whole workgroups where lanes of several wavefronts share a row)
    const uint32_t row = (uint32_t)row64, lane = threadIdx.x % PER;
    float v[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = 8 * (c * PER + lane);
        load8(static_cast<const T *>(a.x) + row * a.ld_x + at, (int)a.cols - at, v[c]);
    }
    if (a.drop.cut) {
        const uint32_t id = mask_id(a.drop, row);
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (8 * (c * PER + lane) < a.cols) mask8(a.drop, id, c * PER + lane, a.drop.scale, v[c]);
    }
    if (a.r) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = 8 * (c * PER + lane);
            float r[8];
            load8(static_cast<const T *>(a.r) + row * a.ld_r + at, (int)a.cols - at, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] += r[j];
        }
    }
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = 8 * (c * PER + lane);
        if (a.h) store8(static_cast<T *>(a.h) + row * a.ld_h + at, (int)a.cols - at, v[c], a.stream);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fmaf(v[c][j], v[c][j], sum);
    }
    const float rstd = 1.0f / sqrtf(row_sum<PER>(sum, lds) * a.inv_cols + a.eps);
    if (a.rstd && lane == 0) a.rstd[row] = rstd;
    float top = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = 8 * (c * PER + lane);
        float g[8];
        if (a.gain) load8(a.gain + at, (int)a.cols - at, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[c][j] = a.gain ? v[c][j] * rstd * g[j] : v[c][j] * rstd;
            if (at + j < (int)a.cols) top = max_nan(top, fabsf(v[c][j]));
        }
    }
    if (a.out_type == ZG_F8) {
        float scale = row_max<PER>(top, lds) / 448.0f;
        scale = scale > 0.0f ? scale : 1.0f;
        if (lane == 0) a.scale[row] = scale;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = 8 * (c * PER + lane);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] /= scale;
            store8_f8(static_cast<uint8_t *>(a.y) + row * a.ld_y + at, (int)a.cols - at, v[c]);
        }
        return;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = 8 * (c * PER + lane);
        store8(a.y, a.out_type, row * a.ld_y + at, (int)a.cols - at, v[c], a.stream);
    }
}

struct NormGradArgs {
    Rows rows;
    uint32_t cols;
    float inv_cols;
    const void *dy, *h, *dh;
    int64_t ld_dy, ld_h, ld_dh;
    const float *rstd, *gain;
    void *dx, *dr;
    int64_t ld_dx, ld_dr;
    float *part; // [workgroups, cols] sums of dy h rstd over a workgroup's rows, or null
    bool stream;
    Drop drop;
};

// A workgroup takes every gridDim.x-th group of rows and keeps its columns' sums for the gain in registers; what its wavefronts hold is
// added up in order at the end.  Bound by memory: 131072 x 1024 bf16 212 us, 5.1 TB/s (2048 workgroups 222, 512 340), and 7 to add up the parts.
template <class T, int PER, int CH> __global__ __launch_bounds__(PER > kRowsBlock ? PER : kRowsBlock) void k_norm_grad(NormGradArgs a)
{
    constexpr int block = PER > kRowsBlock ? PER : kRowsBlock, in_block = block / PER;
    __shared__ float lds[16];
    __shared__ float parts[in_block > 1 ? in_block * PER * 8 : 1];
    const uint32_t lane = threadIdx.x % PER, live = a.rows.live();
    float sums[CH][8] = {};
    for (uint64_t first = (uint64_t)blockIdx.x * in_block; first < live; first += (uint64_t)gridDim.x * in_block) {
        const uint64_t row64 = first + threadIdx.x / PER;
        const bool here = row64 < live;
        const uint32_t row = here ? (uint32_t)row64 : live - 1;
        const float rstd = a.rstd[row];
        float gy[CH][8], h[CH][8], dot = 0.0f;
        const auto load = [&](int c, float (&y)[8], float (&x)[8]) {
            const int at = 8 * (c * PER + lane), left = (int)a.cols - at;
            load8(static_cast<const T *>(a.dy) + row * a.ld_dy + at, left, y);
            load8(static_cast<const T *>(a.h) + row * a.ld_h + at, left, x);
        };
        const auto gained = [&](int c, float (&y)[8]) {
            if (!a.gain) return;
            const int at = 8 * (c * PER + lane);
            float g[8];
            load8(a.gain + at, (int)a.cols - at, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] *= g[j];
        };
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float(&y)[8] = gy[c], (&x)[8] = h[c];
            load(c, y, x);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (here) sums[c][j] = fmaf(y[j], x[j] * rstd, sums[c][j]);
            gained(c, y);
#pragma unroll
            for (int j = 0; j < 8; ++j) dot = fmaf(y[j], x[j], dot);
        }
        const float mean = row_sum<PER>(dot, lds) * a.inv_cols * rstd * rstd;
        const uint32_t id = a.drop.cut && here ? mask_id(a.drop, row) : 0u;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = 8 * (c * PER + lane), left = here ? (int)a.cols - at : 0;
            float(&y)[8] = gy[c], (&x)[8] = h[c];
            float d[8] = {};
            if (a.dh) load8(static_cast<const T *>(a.dh) + row * a.ld_dh + at, left, d);
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] += rstd * (y[j] - x[j] * mean);
            if (a.dr) store8(static_cast<T *>(a.dr) + row * a.ld_dr + at, left, d, a.stream);
            if (a.dx) {
                if (a.drop.cut && left > 0) mask8(a.drop, id, c * PER + lane, a.drop.scale, d);
                store8(static_cast<T *>(a.dx) + row * a.ld_dx + at, left, d, a.stream);
            }
        }
    }
    if (!a.part) return;
    float *out = a.part + (uint64_t)blockIdx.x * a.cols;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = 8 * (c * PER + lane);
        if (in_block > 1) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) parts[threadIdx.x * 8 + j] = sums[c][j];
            __syncthreads();
            if (threadIdx.x >= PER) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sums[c][j] = 0.0f;
                for (int k = 0; k < in_block; ++k) sums[c][j] += parts[(k * PER + lane) * 8 + j];
            }
        }
        store8(out + at, (int)a.cols - at, sums[c]);
    }
}

} // namespace

// out[c] = factor * sum over the `n` rows of part[., c], in a fixed order
constexpr int kSumCols = 16, kSumRows = 64;
__global__ __launch_bounds__(kSumCols *kSumRows) void k_column_sums(const float *part, uint32_t n, uint32_t cols, float factor, float *out)
{
    __shared__ float lds[kSumRows][kSumCols + 1];
    const uint32_t tc = threadIdx.x % kSumCols, tr = threadIdx.x / kSumCols, c = blockIdx.x * kSumCols + tc;
    float v = 0.0f;
    if (c < cols)
        for (uint32_t r = tr; r < n; r += kSumRows) v += part[(uint64_t)r * cols + c];
    lds[tr][tc] = v;
    __syncthreads();
    if (tr == 0 && c < cols) {
        v = 0.0f;
        for (int r = 0; r < kSumRows; ++r) v += lds[r][tc];
        out[c] = factor * v;
    }
}

int launch_column_sums(hipStream_t st, const float *part, uint32_t n, uint32_t cols, float factor, float *out)
{
    return launch(st, k_column_sums, dim3((cols + kSumCols - 1) / kSumCols), kSumCols * kSumRows, part, n, cols, factor, out);
}

namespace {

// lanes to a row and groups of eight columns to a lane: as few lanes as hold the row, so that short rows share a wavefront
template <class F> int with_shape(int32_t cols, F &&f)
{
    using std::integral_constant;
    if (cols <= 64) return f(integral_constant<int, 8>(), integral_constant<int, 1>());
    if (cols <= 128) return f(integral_constant<int, 16>(), integral_constant<int, 1>());
    if (cols <= 256) return f(integral_constant<int, 32>(), integral_constant<int, 1>());
    if (cols <= 512) return f(integral_constant<int, 64>(), integral_constant<int, 1>());
    if (cols <= 1024) return f(integral_constant<int, 64>(), integral_constant<int, 2>());
    if (cols <= 2048) return f(integral_constant<int, 256>(), integral_constant<int, 1>());
    if (cols <= 4096) return f(integral_constant<int, 256>(), integral_constant<int, 2>());
    if (cols <= 8192) return f(integral_constant<int, 1024>(), integral_constant<int, 1>());
    return f(integral_constant<int, 1024>(), integral_constant<int, 2>());
}

template <class F> int with_type(int32_t type, F &&f)
{
    if (type == ZG_F32) return f(float());
    if (type == ZG_F16) return f((_Float16)0);
    return f((__bf16)0);
}

constexpr uint32_t kNormGradBlocks = 1024; // workgroups that sum up the gain's gradient

uint32_t norm_grad_blocks(int64_t rows, int per)
{
    const int64_t in_block = per > kRowsBlock ? 1 : kRowsBlock / per;
    return (uint32_t)std::min<int64_t>(kNormGradBlocks, (rows + in_block - 1) / in_block);
}

} // namespace
} // namespace zg

using namespace zg;

extern "C" {

int zg_dropout(const zg_dropout_args *a, void *stream)
{
    return entry([&]() -> int {
        if (!a) return fail(ZG_EINVAL, "null argument");
        ZG_TRY(check_rows(a->rows));
        ZG_TRY(check_width(a->cols));
        if (!wide_type(a->dtype)) return fail(ZG_EINVAL, "dtype is not ZG_F32, ZG_F16 or ZG_BF16");
        ZG_TRY(check_drop(a->drop));
        ZG_TRY(check_vector("d_rows", a->d_rows));
        if (a->rows == 0) return ZG_OK;
        ZG_TRY(check_matrix("d_x", a->d_x, a->ld_x, a->cols, a->dtype));
        if (a->d_r) ZG_TRY(check_matrix("d_r", a->d_r, a->ld_r, a->cols, a->dtype));
        ZG_TRY(check_matrix("d_y", a->d_y, a->ld_y, a->cols, a->dtype));
        ZG_TRY(check_apart(matrix_span("d_y", a->d_y, a->rows, a->ld_y, a->cols, a->dtype), {ids_span(a->drop, a->rows), rows_span(a->d_rows)},
                           {matrix_span("d_x", a->d_x, a->rows, a->ld_x, a->cols, a->dtype), matrix_span("d_r", a->d_r, a->rows, a->ld_r, a->cols, a->dtype)}));
        DropoutArgs k{};
        k.rows = {a->d_rows, (uint32_t)a->rows};
        k.cols = (uint32_t)a->cols;
        k.groups = (k.cols + 7) / 8;
        k.inv = ((uint64_t(1) << 32) + k.groups - 1) / k.groups;
        k.per_block = std::max(1u, 512u / k.groups); // two groups to a lane: 102 us of the largest case, 8.2 of 4096 x 601 (four: 101 and 8.6, one: 112 and 8.0)
        k.stream = a->rows * a->cols * (int64_t)type_size(a->dtype) > kStreamBytes;
        k.x = a->d_x, k.ld_x = a->ld_x, k.r = a->d_r, k.ld_r = a->ld_r, k.y = a->d_y, k.ld_y = a->ld_y;
        k.drop = make_drop(a->drop);
        const uint32_t grid = (uint32_t)((a->rows + k.per_block - 1) / k.per_block);
        return with_type(a->dtype, [&](auto t) { return launch(static_cast<hipStream_t>(stream), k_dropout<decltype(t)>, grid_of(grid), kRowsBlock, k); });
    });
}

int zg_rms_norm(const zg_norm_args *a, void *stream)
{
    return entry([&]() -> int {
        if (!a) return fail(ZG_EINVAL, "null argument");
        ZG_TRY(check_rows(a->rows));
        ZG_TRY(check_width(a->cols, ZG_MAX_NORM_WIDTH));
        if (!wide_type(a->dtype)) return fail(ZG_EINVAL, "dtype is not ZG_F32, ZG_F16 or ZG_BF16");
        if (!wide_type(a->out_dtype) && a->out_dtype != ZG_F8) return fail(ZG_EINVAL, "out_dtype is not ZG_F32, ZG_F16, ZG_BF16 or ZG_F8");
        if (!(a->eps >= 0.0f)) return fail(ZG_EINVAL, "eps is below 0");
        ZG_TRY(check_drop(a->drop));
        ZG_TRY(check_vector("d_rows", a->d_rows));
        ZG_TRY(check_vector("d_gain", a->d_gain));
        ZG_TRY(check_vector("d_scale", a->d_scale));
        ZG_TRY(check_vector("d_rstd", a->d_rstd));
        if (a->rows == 0) return ZG_OK;
        ZG_TRY(check_matrix("d_x", a->d_x, a->ld_x, a->cols, a->dtype));
        if (a->d_r) ZG_TRY(check_matrix("d_r", a->d_r, a->ld_r, a->cols, a->dtype));
        if (a->d_h) ZG_TRY(check_matrix("d_h", a->d_h, a->ld_h, a->cols, a->dtype));
        ZG_TRY(check_matrix("d_y", a->d_y, a->ld_y, a->cols, a->out_dtype));
        if (a->out_dtype == ZG_F8 && !a->d_scale) return fail(ZG_EINVAL, "an 8-bit result needs d_scale");
        {
            const Span x = matrix_span("d_x", a->d_x, a->rows, a->ld_x, a->cols, a->dtype), r = matrix_span("d_r", a->d_r, a->rows, a->ld_r, a->cols, a->dtype);
            const Span h = matrix_span("d_h", a->d_h, a->rows, a->ld_h, a->cols, a->dtype), y = matrix_span("d_y", a->d_y, a->rows, a->ld_y, a->cols, a->out_dtype);
            const Span gain = vector_span("d_gain", a->d_gain, a->cols), rstd = vector_span("d_rstd", a->d_rstd, a->rows);
            const Span scale = vector_span("d_scale", a->out_dtype == ZG_F8 ? a->d_scale : nullptr, a->rows), ids = ids_span(a->drop, a->rows), count = rows_span(a->d_rows);
            ZG_TRY(check_apart(h, {gain, ids, count}, {x, r}));
            ZG_TRY(check_apart(y, {gain, ids, count, h}, {x, r}));
            ZG_TRY(check_apart(rstd, {gain, ids, count, h, y, x, r}));
            ZG_TRY(check_apart(scale, {gain, ids, count, h, y, x, r, rstd}));
        }
        NormArgs k{};
        k.rows = {a->d_rows, (uint32_t)a->rows};
        k.cols = (uint32_t)a->cols;
        k.inv_cols = 1.0f / (float)a->cols;
        k.eps = a->eps;
        k.out_type = a->out_dtype;
        k.stream = a->rows * a->cols * (int64_t)type_size(a->dtype) > kStreamBytes;
        k.x = a->d_x, k.ld_x = a->ld_x, k.r = a->d_r, k.ld_r = a->ld_r, k.gain = a->d_gain;
        k.h = a->d_h, k.ld_h = a->ld_h, k.y = a->d_y, k.ld_y = a->ld_y, k.scale = a->d_scale, k.rstd = a->d_rstd;
        k.drop = make_drop(a->drop);
        return with_type(a->dtype, [&](auto t) {
            return with_shape(a->cols, [&](auto per, auto ch) {
                constexpr int P = decltype(per)::value, block = P > kRowsBlock ? P : kRowsBlock;
                const uint32_t grid = (uint32_t)((a->rows + block / P - 1) / (block / P));
                return launch(static_cast<hipStream_t>(stream), k_norm<decltype(t), P, decltype(ch)::value>, grid_of(grid), block, k);
            });
        });
    });
}

int zg_rms_norm_backward_workspace(const zg_norm_grad_args *a, size_t *bytes)
{
    return entry([&]() -> int {
        if (!a || !bytes) return fail(ZG_EINVAL, "null argument");
        ZG_TRY(check_rows(a->rows));
        ZG_TRY(check_width(a->cols, ZG_MAX_NORM_WIDTH));
        *bytes = 0;
        if (!a->d_dgain) return ZG_OK;
        return with_shape(a->cols, [&](auto per, auto) {
            *bytes = (size_t)norm_grad_blocks(a->rows, decltype(per)::value) * a->cols * sizeof(float);
            return ZG_OK;
        });
    });
}

int zg_rms_norm_backward(const zg_norm_grad_args *a, void *d_workspace, size_t workspace_bytes, void *stream)
{
    return entry([&]() -> int {
        size_t need = 0;
        ZG_TRY(zg_rms_norm_backward_workspace(a, &need));
        if (!wide_type(a->dtype)) return fail(ZG_EINVAL, "dtype is not ZG_F32, ZG_F16 or ZG_BF16");
        ZG_TRY(check_drop(a->drop));
        ZG_TRY(check_vector("d_rows", a->d_rows));
        ZG_TRY(check_vector("d_gain", a->d_gain));
        ZG_TRY(check_vector("d_rstd", a->d_rstd));
        ZG_TRY(check_vector("d_dgain", a->d_dgain));
        ZG_TRY(check_workspace(d_workspace, workspace_bytes, need));
        if (a->rows > 0) {
            ZG_TRY(check_matrix("d_dy", a->d_dy, a->ld_dy, a->cols, a->dtype));
            ZG_TRY(check_matrix("d_h", a->d_h, a->ld_h, a->cols, a->dtype));
            if (!a->d_rstd) return fail(ZG_EINVAL, "d_rstd is null");
            if (a->d_dh) ZG_TRY(check_matrix("d_dh", a->d_dh, a->ld_dh, a->cols, a->dtype));
            if (a->d_dx) ZG_TRY(check_matrix("d_dx", a->d_dx, a->ld_dx, a->cols, a->dtype));
            if (a->d_dr) ZG_TRY(check_matrix("d_dr", a->d_dr, a->ld_dr, a->cols, a->dtype));
            if (!a->d_dx && !a->d_dr) return fail(ZG_EINVAL, "d_dx and d_dr are both null");
            const Span dy = matrix_span("d_dy", a->d_dy, a->rows, a->ld_dy, a->cols, a->dtype), h = matrix_span("d_h", a->d_h, a->rows, a->ld_h, a->cols, a->dtype);
            const Span dh = matrix_span("d_dh", a->d_dh, a->rows, a->ld_dh, a->cols, a->dtype), dx = matrix_span("d_dx", a->d_dx, a->rows, a->ld_dx, a->cols, a->dtype);
            const Span dr = matrix_span("d_dr", a->d_dr, a->rows, a->ld_dr, a->cols, a->dtype), gain = vector_span("d_gain", a->d_gain, a->cols);
            const Span rstd = vector_span("d_rstd", a->d_rstd, a->rows), ids = ids_span(a->drop, a->rows), count = rows_span(a->d_rows);
            ZG_TRY(check_apart(dx, {gain, rstd, ids, count}, {dy, h, dh}));
            ZG_TRY(check_apart(dr, {gain, rstd, ids, count}, {dy, h, dh}));
            ZG_TRY(a->drop.p > 0.0 ? check_apart(dr, {dx}) : check_apart(dr, {}, {dx})); // (without dropout they are the same values)
            ZG_TRY(check_apart(vector_span("d_dgain", a->d_dgain, a->cols), {gain, rstd, ids, count, dy, h, dh, dx, dr}));
        }
        const hipStream_t st = static_cast<hipStream_t>(stream);
        NormGradArgs k{};
        k.rows = {a->d_rows, (uint32_t)a->rows};
        k.cols = (uint32_t)a->cols;
        k.inv_cols = 1.0f / (float)a->cols;
        k.dy = a->d_dy, k.ld_dy = a->ld_dy, k.h = a->d_h, k.ld_h = a->ld_h, k.dh = a->d_dh, k.ld_dh = a->ld_dh;
        k.rstd = a->d_rstd, k.gain = a->d_gain;
        k.dx = a->d_dx, k.ld_dx = a->ld_dx, k.dr = a->d_dr, k.ld_dr = a->ld_dr;
        k.stream = a->rows * a->cols * (int64_t)type_size(a->dtype) > kStreamBytes;
        k.part = a->d_dgain ? static_cast<float *>(d_workspace) : nullptr;
        k.drop = make_drop(a->drop);
        uint32_t grid = 0;
        ZG_TRY(with_type(a->dtype, [&](auto t) {
            return with_shape(a->cols, [&](auto per, auto ch) {
                constexpr int P = decltype(per)::value, block = P > kRowsBlock ? P : kRowsBlock;
                grid = norm_grad_blocks(a->rows, P);
                return launch(st, k_norm_grad<decltype(t), P, decltype(ch)::value>, dim3(grid), block, k);
            });
        }));
        return a->d_dgain ? launch_column_sums(st, k.part, grid, k.cols, 1.0f, a->d_dgain) : ZG_OK;
    });
}

} // extern "C"
