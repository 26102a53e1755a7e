// Products with bias, activation, dropout and residual behind them, and their gradients.
#include "zg_product.h"

namespace zg {
namespace {

// ---- the kernels (how each of them works, and what bounds it, stands at its tile in zg_product.h) -------------------------------------

template <class T, int BM, int BN, bool A_TURNED, bool B_TURNED> __global__ __launch_bounds__(256, 2) void k_product(ProductArgs p)
{
    product_tile<T, BM, BN, A_TURNED, B_TURNED>(p);
}

template <class T, class O, int BM, int BN, int BLOCKS, bool A_TURNED, bool B_TURNED> __global__ __launch_bounds__(256, BLOCKS) void k_chunks(ProductArgs p)
{
    chunks_tile<T, O, BM, BN, A_TURNED, B_TURNED>(p);
}

template <class T, class O, bool A_TURNED, bool B_TURNED> __global__ __launch_bounds__(512, 2) void k_long(ProductArgs p)
{
    long_tiles<T, O, A_TURNED, B_TURNED>(p);
}

template <class T> __global__ __launch_bounds__(256) void k_few(ProductArgs p) { few_tile<T>(p); }

// The sum over the parts, and what happens to it (16 parts of 1024 x 1024: 12 us, 5.6 TB/s; 256 of 256 x 200: 12 us): groups of eight cells, each with `lanes` lanes (a power of two up to 32) that have every so
// manieth part each; then the lanes in order.  One lane, or as many as parts, add them one after the other; beyond 32 parts there are 32 lanes: the order goes by the number of parts alone (dense_join).
struct JoinArgs {
    const float *part;
    uint32_t M, N, splits, lanes;
    Epilogue e;
    Rows rows; // the device's count bounds M
};

__global__ __launch_bounds__(256) void k_join(JoinArgs p)
{
    __shared__ float lds[256][8 + 1];
    const uint32_t groups = (p.N + 7) / 8, in_block = 256 / p.lanes, g = threadIdx.x % in_block, lane = threadIdx.x / in_block;
    const uint64_t i = (uint64_t)block_number() * in_block + g, cells = (uint64_t)p.M * p.N;
    const bool there = i < (uint64_t)min(p.M, p.rows.live()) * groups;
    const uint32_t m = there ? (uint32_t)(i / groups) : 0u, n = there ? (uint32_t)(i % groups) * 8 : 0u;
    float v[8] = {};
    if (there)
        for (uint32_t s = lane; s < p.splits; s += p.lanes) {
            float w[8];
            load8(p.part + s * cells + (uint64_t)m * p.N + n, (int)(p.N - n), w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += w[j];
        }
    if (p.lanes > 1) {
#pragma unroll
        for (int j = 0; j < 8; ++j) lds[threadIdx.x][j] = v[j];
        __syncthreads();
    }
    if (lane || !there) return;
    const Columns c = columns_of(p.e, n, p.N);
    Needs<AnyType, 1> needs;
    needs.ask(p.e, c.n, c.left, m, 1, p.M);
    finish(p.e, c, needs, m, 1, p.M, [&](int, float(&sum)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = v[j];
        for (uint32_t s = 1; s < min(p.splits, p.lanes); ++s)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += lds[s * in_block + g][j];
    });
}

// dZ without dropout's factor (dropped cells 0), and the sums of dZ over a workgroup's rows.  A lane has eight columns.  Bound by memory: 65536 x 1024
// bf16 SiLU with dropout 92 us, 4.4 TB/s; 100000 x 256 fp32 ReLU 51 us, 6.0 TB/s (twice the workgroups: 13 us more for both cases' gradients).
struct SlopeArgs {
    Rows rows;
    uint32_t cols;
    uint32_t lanes; // lanes side by side in a row, a power of two; 256 / lanes rows at a time
    int32_t act;
    const void *dy, *z;
    int64_t ld_dy, ld_z;
    void *dz; // or null: only the sums are wanted
    int64_t ld_dz;
    float *part; // [gridDim.y, cols] or null
    float *tops; // of holds_power: the largest |dZ| of each workgroup, then the power of two that dZ was divided by
    Drop drop;
};

// Whether a dZ of type T, made of a dY of type TO, is held as what is left beside a power of two: fp16's range ends at 65504 above and at 2^-24 below, the
// other types' do not, and the caller of a wider dY may mean either (a mean's gradient over 65536 rows is 2^-16 and less).
template <class TO, class T> constexpr bool holds_power = std::is_same_v<T, _Float16> && !std::is_same_v<TO, _Float16>;

// eight cells of dZ without dropout's factor
template <class TO> __device__ __forceinline__ void slopes8(const SlopeArgs &a, uint64_t r, uint32_t g, int left, float (&v)[8])
{
    load8(static_cast<const TO *>(a.dy) + r * a.ld_dy + 8 * g, left, v);
    if (a.act != ZG_ACT_NONE) {
        float z[8];
        load8(static_cast<const TO *>(a.z) + r * a.ld_z + 8 * g, left, z);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= act_slope(a.act, z[j]);
    }
    if (a.drop.cut) mask8(a.drop, mask_id(a.drop, (uint32_t)r), g, 1.0f, v); // (behind the slope: a dropped cell's may be anything)
}

__device__ __forceinline__ float block_max(float v, float *lds) // of 256 lanes
{
    __syncthreads();
    lds[threadIdx.x] = v;
    __syncthreads();
#pragma unroll
    for (int n = 128; n > 0; n >>= 1) {
        if (threadIdx.x < n) lds[threadIdx.x] = fmaxf(lds[threadIdx.x], lds[threadIdx.x + n]);
        __syncthreads();
    }
    return lds[0];
}

// The largest finite |dZ| of each workgroup, in the grid that k_slope has: 65536 x 1024 of fp32 dY and Z with SiLU 105 us of all gradients' 540.
template <class TO> __global__ __launch_bounds__(256) void k_slope_top(SlopeArgs a)
{
    __shared__ float lds[256];
    const uint32_t live = a.rows.live(), in_block = 256 / a.lanes, g = blockIdx.x * a.lanes + threadIdx.x % a.lanes;
    const int left = (int)a.cols - (int)(8 * g);
    float top = 0.0f;
    for (uint64_t r = (uint64_t)blockIdx.y * in_block + threadIdx.x / a.lanes; r < live && left > 0; r += (uint64_t)gridDim.y * in_block) {
        float v[8];
        slopes8<TO>(a, r, g, left, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fabsf(v[j]) <= 3.402823466e38f ? fmaxf(top, fabsf(v[j])) : top;
    }
    top = block_max(top, lds);
    if (threadIdx.x == 0) a.tops[blockIdx.y * gridDim.x + blockIdx.x] = top;
}

template <class TO, class T> __global__ __launch_bounds__(256) void k_slope(SlopeArgs a)
{
    __shared__ float lds[256 * 8];
    float power = 1.0f;
    if (holds_power<TO, T> && a.dz) {
        const uint32_t n = gridDim.x * gridDim.y;
        float top = 0.0f;
        for (uint32_t i = threadIdx.x; i < n; i += 256) top = fmaxf(top, a.tops[i]);
        top = block_max(top, lds);
        // top 2^e in [2^14, 2^15): the sums of products with other fp16 stay far inside fp32
        const int e = top > 0.0f ? min(15 - __builtin_amdgcn_frexp_expf(top), 126) : 0;
        power = ldexpf(1.0f, e);
        if (threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0) a.tops[n] = ldexpf(1.0f, -e);
        __syncthreads();
    }
    const uint32_t live = a.rows.live(), lane = threadIdx.x % a.lanes, in_block = 256 / a.lanes, mine = threadIdx.x / a.lanes;
    const uint32_t g = blockIdx.x * a.lanes + lane;
    const int left = (int)a.cols - (int)(8 * g);
    float sums[8] = {};
    for (uint64_t r = (uint64_t)blockIdx.y * in_block + mine; r < live && left > 0; r += (uint64_t)gridDim.y * in_block) {
        float v[8];
        slopes8<TO>(a, r, g, left, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[j] += v[j];
        if (holds_power<TO, T>) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= power;
        }
        if (a.dz) store8(static_cast<T *>(a.dz) + r * a.ld_dz + 8 * g, left, v);
    }
    if (!a.part) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) lds[threadIdx.x * 8 + j] = sums[j];
    __syncthreads();
    if (mine != 0 || left <= 0) return;
    for (uint32_t k = 1; k < in_block; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[j] += lds[(k * a.lanes + lane) * 8 + j];
    store8(a.part + (uint64_t)blockIdx.y * a.cols + 8 * g, left, sums);
}

template <class T, class O, bool A_TURNED, bool B_TURNED> int launch_chunks(hipStream_t st, const ProductArgs &p)
{
    if constexpr (std::is_same_v<T, float>) {
        return launch(st, k_chunks<T, O, 128, 128, 3, A_TURNED, B_TURNED>, tile_grid<128, 128>(p), 256, p);
    } else {
        // Two workgroups to a compute unit hide each other's epilogue; one with larger tiles reads less and loses its own.  us with tiles of 256 x 128 /
        // 256 x 256: bf16 65536 x 1024 x 1024 with nothing but a rounding 177 / 162, with GELU, dropout, residual and Z 281 / 292; 262144 x 256 x 256
        // 86 / 97; 4096 x 16384 x 4096 615 / 433; gradients of 65536 x 1024 x 1024 472 / 424.  8 bits, widened as they are multiplied, take the smaller tiles: 65536 x
        // 1024 x 2048 with SiLU 312 / 347, 65536 x 4096 x 2048 906 / 950, 8192 x 8192 x 8192 841 / 868.
        if constexpr (!std::is_same_v<T, uint8_t>) {
            const bool light = p.e.act == ZG_ACT_NONE && !p.e.drop.cut && !p.e.R && !p.e.Z;
            if (tile_blocks<256, 256>(p) >= 256 && (B_TURNED || p.K * sizeof(T) >= (light ? 2048u : 4096u)))
                return launch(st, k_long<T, O, A_TURNED, B_TURNED>, dim3(256), 512, p);
        }
        return launch(st, k_chunks<T, O, 256, 128, 2, A_TURNED, B_TURNED>, tile_grid<256, 128>(p), 256, p);
    }
}

// Operands that lie anyhow, in tiles of tile x tile: the smaller ones where the larger ones would not be two to a compute unit (33333 x 301 x 47 fp16
// 17.6 -> 11.5 us).
template <class T, int tile> int launch_anyhow(hipStream_t st, const ProductArgs &p)
{
    const dim3 grid = tile_grid<tile, tile>(p);
    if constexpr (!std::is_same_v<T, Widened8>) {
        if (p.a.turned) return launch(st, k_product<T, tile, tile, true, true>, grid, 256, p);
        if (p.b.turned) return launch(st, k_product<T, tile, tile, false, true>, grid, 256, p);
    }
    return launch(st, k_product<T, tile, tile, false, false>, grid, 256, p);
}

// the tiles of one product, or of the parts of one, whose results are of type p.e.type
template <class T> int launch_tiles(hipStream_t st, const ProductArgs &p)
{
    const bool chunks = in_chunks<T>(p.a, p.M, p.K) && in_chunks<T>(p.b, p.N, p.K);
    if (few_tiles<T>(p, chunks)) {
        using F = std::conditional_t<std::is_same_v<T, uint8_t>, Widened8, T>;
        return launch(st, k_few<F>, grid_of((uint64_t)((p.M + 31) / 32) * ((p.N + 31) / 32)), 256, p);
    }
    if constexpr (!std::is_same_v<T, Widened8>) {
        if (chunks) {
            if constexpr (!std::is_same_v<T, uint8_t>) {
                if (p.a.turned) return p.e.type == ZG_F32 ? launch_chunks<T, float, true, true>(st, p) : launch_chunks<T, T, true, true>(st, p);
                if (p.b.turned) return launch_chunks<T, T, false, true>(st, p);
            }
            if (p.e.type == ZG_F32) return launch_chunks<T, float, false, false>(st, p);
            if (p.e.type == ZG_F16) return launch_chunks<T, _Float16, false, false>(st, p);
            return launch_chunks<T, __bf16, false, false>(st, p);
        }
    }
    if constexpr (std::is_same_v<T, uint8_t>) return launch_tiles<Widened8>(st, p);
    else return tile_blocks<kTile, kTile>(p) < 512 ? launch_anyhow<T, kTile / 2>(st, p) : launch_anyhow<T, kTile>(st, p);
}

// `part`: room for splits x M x N sums where there are parts
template <class T> int launch_product(hipStream_t st, const ProductArgs &p, float *part)
{
    if (p.splits == 1) return launch_tiles<T>(st, p);
    ProductArgs q = p;
    q.e = Epilogue{};
    q.e.factor = 1.0f;
    q.e.type = ZG_F32;
    q.e.Y = part, q.e.ld_Y = p.N, q.e.part = (int64_t)p.M * p.N;
    ZG_TRY(launch_tiles<T>(st, q));
    return dense_join(st, part, p.M, p.N, p.splits, p.e, {nullptr, p.M});
}

int launch_product(hipStream_t st, int32_t type, const ProductArgs &p, float *part = nullptr)
{
    if (type == ZG_F32) return launch_product<float>(st, p, part);
    if (type == ZG_F16) return launch_product<_Float16>(st, p, part);
    if (type == ZG_BF16) return launch_product<__bf16>(st, p, part);
    return launch_product<uint8_t>(st, p, part);
}

// How the gradients' workspace is laid out.
struct GradPlan {
    bool slopes;       // dZ differs from dY (a slope, a mask or another type): it is written out
    int64_t ld_dz;
    uint32_t lanes, slope_x, slope_y; // of k_slope
    uint32_t splits;   // parts of dW's sum over the rows
    bool power;        // dZ is held beside a power of two
    size_t off_dz, off_tops, off_part, off_dw, total;
};

GradPlan grad_plan(const zg_linear_grad_args &a)
{
    GradPlan g{};
    auto take = [&](size_t bytes) {
        const size_t at = g.total;
        g.total = (g.total + bytes + 255) / 256 * 256;
        return at;
    };
    g.slopes = a.act != ZG_ACT_NONE || a.drop.p > 0.0 || a.dtype != a.out_dtype;
    g.ld_dz = (a.out + 7) / 8 * 8;
    const uint32_t groups = ((uint32_t)a.out + 7) / 8;
    g.lanes = 1;
    while (g.lanes < groups && g.lanes < 64) g.lanes *= 2;
    g.slope_x = (groups + g.lanes - 1) / g.lanes;
    g.slope_y = (uint32_t)std::min<int64_t>(std::max(1u, 1024u / g.slope_x), (a.rows + 256 / g.lanes - 1) / (256 / g.lanes));
    const int64_t tiles = (int64_t)((a.out + kTileM - 1) / kTileM) * ((a.in + kTileN - 1) / kTileN);
    g.splits = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(512 / tiles, (a.rows + 255) / 256));
    if (g.slopes && (a.d_dA || a.d_dW)) g.off_dz = take((size_t)a.rows * g.ld_dz * type_size(a.dtype));
    g.power = g.slopes && (a.d_dA || a.d_dW) && a.dtype == ZG_F16 && a.out_dtype != ZG_F16;
    if (g.power) g.off_tops = take(((size_t)g.slope_x * g.slope_y + 1) * sizeof(float));
    if (a.d_dbias) g.off_part = take((size_t)g.slope_y * a.out * sizeof(float));
    if (a.d_dW && g.splits > 1) g.off_dw = take((size_t)g.splits * a.out * a.in * sizeof(float));
    return g;
}

int check_linear_grad(const zg_linear_grad_args *a)
{
    if (!a) return fail(ZG_EINVAL, "null argument");
    ZG_TRY(check_rows(a->rows));
    ZG_TRY(check_width(a->in));
    ZG_TRY(check_width(a->out));
    if (!wide_type(a->dtype) || !wide_type(a->out_dtype)) return fail(ZG_EINVAL, "dtype or out_dtype is not ZG_F32, ZG_F16 or ZG_BF16");
    if (a->act < ZG_ACT_NONE || a->act > ZG_ACT_GELU) return fail(ZG_EINVAL, "unknown activation");
    return check_drop(a->drop);
}

} // namespace

int dense_product(hipStream_t st, int32_t type, const ProductArgs &p, float *part) { return launch_product(st, type, p, part); }

int dense_join(hipStream_t st, const float *part, uint32_t M, uint32_t N, uint32_t splits, const Epilogue &e, Rows rows)
{
    // One lane, or one for each part (32 beyond that): sums whose order goes by the result's size would give other bits for other sizes.  us with one / each / lanes in between: 2048 x 1024 of 16 parts 23.9 / 28.6,
    // 1024 x 1024 of 16 12.2 / 12.7 / 12.4, 1024 x 512 of 16 8.9 / 9.2 / 7.7, 512 x 512 of 32 13.3 / 10.1 / 7.8, 256 x 256 of 32 11.5 / 6.4.
    const uint64_t groups = (uint64_t)M * ((N + 7) / 8);
    uint32_t lanes = 1;
    while (lanes < 32 && lanes < splits && (splits > 32 || groups < 65536)) lanes *= 2;
    return launch(st, k_join, grid_of((groups * lanes + 255) / 256), 256, JoinArgs{part, M, N, splits, lanes, e, rows});
}

} // namespace zg

using namespace zg;

extern "C" {
int zg_linear(const zg_linear_args *a, void *stream)
{
    return entry([&]() -> int {
        if (!a) return fail(ZG_EINVAL, "null argument");
        ZG_TRY(check_rows(a->rows));
        ZG_TRY(check_width(a->in));
        ZG_TRY(check_width(a->out));
        if (!wide_type(a->dtype) && a->dtype != ZG_F8) return fail(ZG_EINVAL, "dtype is not ZG_F32, ZG_F16, ZG_BF16 or ZG_F8");
        if (!wide_type(a->out_dtype)) return fail(ZG_EINVAL, "out_dtype is not ZG_F32, ZG_F16 or ZG_BF16");
        if (a->act < ZG_ACT_NONE || a->act > ZG_ACT_GELU) return fail(ZG_EINVAL, "unknown activation");
        if (a->dtype != ZG_F8 && (a->d_scale_A || a->d_scale_W)) return fail(ZG_EINVAL, "scales go with operands of type ZG_F8");
        ZG_TRY(check_drop(a->drop));
        ZG_TRY(check_vector("d_rows", a->d_rows));
        ZG_TRY(check_vector("d_bias", a->d_bias));
        ZG_TRY(check_vector("d_scale_A", a->d_scale_A));
        ZG_TRY(check_vector("d_scale_W", a->d_scale_W));
        if (a->rows == 0) return ZG_OK;
        ZG_TRY(check_matrix("d_A", a->d_A, a->ld_A, a->in, a->dtype));
        ZG_TRY(check_matrix("d_W", a->d_W, a->ld_W, a->in, a->dtype));
        ZG_TRY(check_matrix("d_Y", a->d_Y, a->ld_Y, a->out, a->out_dtype));
        if (a->d_R) ZG_TRY(check_matrix("d_R", a->d_R, a->ld_R, a->out, a->out_dtype));
        if (a->d_Z) ZG_TRY(check_matrix("d_Z", a->d_Z, a->ld_Z, a->out, a->out_dtype));
        {
            const Span A = matrix_span("d_A", a->d_A, a->rows, a->ld_A, a->in, a->dtype), W = matrix_span("d_W", a->d_W, a->out, a->ld_W, a->in, a->dtype);
            const Span R = matrix_span("d_R", a->d_R, a->rows, a->ld_R, a->out, a->out_dtype), Y = matrix_span("d_Y", a->d_Y, a->rows, a->ld_Y, a->out, a->out_dtype);
            const Span Z = matrix_span("d_Z", a->d_Z, a->rows, a->ld_Z, a->out, a->out_dtype), bias = vector_span("d_bias", a->d_bias, a->out);
            const Span scale_A = vector_span("d_scale_A", a->d_scale_A, a->rows), scale_W = vector_span("d_scale_W", a->d_scale_W, a->out);
            const Span ids = ids_span(a->drop, a->rows), count = rows_span(a->d_rows);
            ZG_TRY(check_apart(Y, {A, W, Z, bias, scale_A, scale_W, ids, count}, {R}));
            ZG_TRY(check_apart(Z, {A, W, R, bias, scale_A, scale_W, ids, count}));
        }
        ProductArgs p{};
        p.a = {a->d_A, a->ld_A, false, false};
        p.b = {a->d_W, a->ld_W, false, false};
        p.M = (uint32_t)a->rows, p.N = (uint32_t)a->out, p.K = (uint32_t)a->in;
        p.rows = {a->d_rows, p.M};
        p.splits = 1;
        p.e.factor = 1.0f;
        p.e.scale_m = a->d_scale_A, p.e.scale_n = a->d_scale_W, p.e.bias = a->d_bias;
        p.e.act = a->act, p.e.type = a->out_dtype, p.e.drop = make_drop(a->drop);
        p.e.stream = a->rows * a->out * (int64_t)type_size(a->out_dtype) > kStreamBytes;
        p.e.R = a->d_R, p.e.ld_R = a->ld_R, p.e.Y = a->d_Y, p.e.ld_Y = a->ld_Y, p.e.Z = a->d_Z, p.e.ld_Z = a->ld_Z;
        return launch_product(static_cast<hipStream_t>(stream), a->dtype, p);
    });
}

int zg_linear_backward_workspace(const zg_linear_grad_args *a, size_t *bytes)
{
    return entry([&]() -> int {
        ZG_TRY(check_linear_grad(a));
        if (!bytes) return fail(ZG_EINVAL, "null argument");
        *bytes = grad_plan(*a).total;
        return ZG_OK;
    });
}

int zg_linear_backward(const zg_linear_grad_args *a, void *d_workspace, size_t workspace_bytes, void *stream)
{
    return entry([&]() -> int {
        ZG_TRY(check_linear_grad(a));
        ZG_TRY(check_vector("d_rows", a->d_rows));
        ZG_TRY(check_vector("d_dbias", a->d_dbias));
        const GradPlan g = grad_plan(*a);
        ZG_TRY(check_workspace(d_workspace, workspace_bytes, g.total));
        if (a->rows > 0) {
            ZG_TRY(check_matrix("d_dY", a->d_dY, a->ld_dY, a->out, a->out_dtype));
            if (a->act != ZG_ACT_NONE) ZG_TRY(check_matrix("d_Z", a->d_Z, a->ld_Z, a->out, a->out_dtype));
            if (a->d_dA) {
                ZG_TRY(check_matrix("d_dA", a->d_dA, a->ld_dA, a->in, a->dtype));
                ZG_TRY(check_matrix("d_W", a->d_W, a->ld_W, a->in, a->dtype));
            }
            if (a->d_dW) ZG_TRY(check_matrix("d_A", a->d_A, a->ld_A, a->in, a->dtype));
        }
        if (a->d_dW) ZG_TRY(check_matrix("d_dW", a->d_dW, a->ld_dW, a->in, a->dtype));
        {
            const Span dY = matrix_span("d_dY", a->d_dY, a->rows, a->ld_dY, a->out, a->out_dtype);
            const Span Z = matrix_span("d_Z", a->act != ZG_ACT_NONE ? a->d_Z : nullptr, a->rows, a->ld_Z, a->out, a->out_dtype);
            const Span A = matrix_span("d_A", a->d_dW ? a->d_A : nullptr, a->rows, a->ld_A, a->in, a->dtype);
            const Span W = matrix_span("d_W", a->d_dA ? a->d_W : nullptr, a->out, a->ld_W, a->in, a->dtype);
            const Span dA = matrix_span("d_dA", a->d_dA, a->rows, a->ld_dA, a->in, a->dtype), dW = matrix_span("d_dW", a->d_dW, a->out, a->ld_dW, a->in, a->dtype);
            const Span dbias = vector_span("d_dbias", a->d_dbias, a->out), ids = ids_span(a->drop, a->rows), count = rows_span(a->d_rows);
            ZG_TRY(check_apart(dA, {dY, Z, A, W, ids, count}));
            ZG_TRY(check_apart(dW, {dY, Z, A, W, ids, count, dA}));
            ZG_TRY(check_apart(dbias, {dY, Z, A, W, ids, count, dA, dW}));
        }
        const hipStream_t st = static_cast<hipStream_t>(stream);
        char *const ws = static_cast<char *>(d_workspace);
        const Rows rows{a->d_rows, (uint32_t)a->rows};
        const Drop drop = make_drop(a->drop);
        const float factor = a->drop.p > 0.0 ? drop.scale : 1.0f; // (what dropout keeps is multiplied behind the sums)
        const void *dz = a->d_dY;
        int64_t ld_dz = a->ld_dY;
        if (g.slopes && (a->d_dA || a->d_dW)) dz = ws + g.off_dz, ld_dz = g.ld_dz;
        if (dz != a->d_dY || a->d_dbias) {
            SlopeArgs s{};
            s.rows = rows, s.cols = (uint32_t)a->out, s.lanes = g.lanes, s.act = a->act;
            s.dy = a->d_dY, s.ld_dy = a->ld_dY, s.z = a->d_Z, s.ld_z = a->ld_Z;
            s.dz = dz != a->d_dY ? const_cast<void *>(dz) : nullptr, s.ld_dz = ld_dz;
            s.part = a->d_dbias ? reinterpret_cast<float *>(ws + g.off_part) : nullptr;
            s.tops = g.power ? reinterpret_cast<float *>(ws + g.off_tops) : nullptr;
            s.drop = drop;
            const dim3 grid(g.slope_x, g.slope_y);
            if (g.power) ZG_TRY(a->out_dtype == ZG_F32 ? launch(st, k_slope_top<float>, grid, 256, s) : launch(st, k_slope_top<__bf16>, grid, 256, s));
            auto from = [&](auto to) {
                using TO = decltype(to);
                if (a->dtype == ZG_F32) return launch(st, k_slope<TO, float>, grid, 256, s);
                if (a->dtype == ZG_F16) return launch(st, k_slope<TO, _Float16>, grid, 256, s);
                return launch(st, k_slope<TO, __bf16>, grid, 256, s);
            };
            if (a->out_dtype == ZG_F32) ZG_TRY(from(float()));
            else if (a->out_dtype == ZG_F16) ZG_TRY(from((_Float16)0));
            else ZG_TRY(from((__bf16)0));
            if (a->d_dbias) ZG_TRY(launch_column_sums(st, s.part, g.slope_y, s.cols, factor, a->d_dbias));
        }
        ProductArgs p{};
        p.rows = rows;
        p.e.factor = factor;
        if (g.power && a->rows > 0) p.e.power = reinterpret_cast<const float *>(ws + g.off_tops) + (size_t)g.slope_x * g.slope_y;
        p.e.type = a->dtype;
        if (a->d_dA && a->rows > 0) {
            p.a = {dz, ld_dz, false};
            p.b = {a->d_W, a->ld_W, true};
            p.M = (uint32_t)a->rows, p.N = (uint32_t)a->in, p.K = (uint32_t)a->out;
            p.splits = 1;
            p.e.Y = a->d_dA, p.e.ld_Y = a->ld_dA;
            p.e.stream = a->rows * a->in * (int64_t)type_size(a->dtype) > kStreamBytes;
            ZG_TRY(launch_product(st, a->dtype, p));
        }
        if (a->d_dW) {
            p.a = {dz, ld_dz, true};
            p.b = {a->d_A, a->ld_A, true};
            p.M = (uint32_t)a->out, p.N = (uint32_t)a->in, p.K = (uint32_t)a->rows;
            p.rows_are_k = 1;
            p.splits = g.splits;
            p.e.Y = a->d_dW, p.e.ld_Y = a->ld_dW;
            p.e.stream = false;
            ZG_TRY(launch_product(st, a->dtype, p, reinterpret_cast<float *>(ws + g.off_dw)));
        }
        return ZG_OK;
    });
}

} // extern "C"
