// Products with bias, activation, dropout and residual behind them, and their gradients.
#include "zg_dense.h"

#include <algorithm>
#include <tuple>

namespace zg {

int launch_column_sums(hipStream_t st, const float *part, uint32_t n, uint32_t cols, float factor, float *out);

namespace {

// What happens to a product's sums: v = scale_m scale_n sum, z = v + bias, y = R + drop(act(z)).
struct Epilogue {
    float factor;
    const float *scale_m, *scale_n, *bias;
    int32_t act, type; // type of R, Y and Z
    Drop drop;
    const void *R;
    int64_t ld_R;
    void *Y, *Z;
    int64_t ld_Y, ld_Z;
};

__device__ __forceinline__ float load1(const void *p, int32_t type, int64_t at)
{
    if (type == ZG_F32) return static_cast<const float *>(p)[at];
    if (type == ZG_F16) return (float)static_cast<const _Float16 *>(p)[at];
    return (float)static_cast<const __bf16 *>(p)[at];
}

__device__ __forceinline__ void store1(void *p, int32_t type, int64_t at, float v)
{
    if (type == ZG_F32) static_cast<float *>(p)[at] = v;
    else if (type == ZG_F16) static_cast<_Float16 *>(p)[at] = (_Float16)v;
    else static_cast<__bf16 *>(p)[at] = (__bf16)v;
}

__device__ __forceinline__ void finish1(const Epilogue &e, uint32_t m, uint32_t n, float sum)
{
    float v = sum * e.factor;
    if (e.scale_m) v *= e.scale_m[m];
    if (e.scale_n) v *= e.scale_n[n];
    if (e.bias) v += e.bias[n];
    if (e.Z) store1(e.Z, e.type, m * e.ld_Z + n, v);
    v = act_of(e.act, v);
    if (e.drop.cut) {
        uint32_t w[4];
        mask_bits(e.drop, mask_id(e.drop, m), n >> 3, w);
        const uint32_t word = n & 4 ? (n & 2 ? w[3] : w[2]) : (n & 2 ? w[1] : w[0]);
        v = (n & 1 ? word >> 16 : word & 0xFFFFu) >= e.drop.cut ? v * e.drop.scale : 0.0f;
    }
    if (e.R) v += load1(e.R, e.type, m * e.ld_R + n);
    store1(e.Y, e.type, m * e.ld_Y + n, v);
}

// C[m, n] = sum over k of a(m, k) b(n, k); element (i, k) of an operand is p[i * si + k * sk].
struct Operand {
    const void *p;
    int64_t si, sk;
};

struct ProductArgs {
    Operand a, b;
    uint32_t M, N, K;
    Rows rows;
    int32_t rows_are_k; // the device's count bounds K, else M
    uint32_t splits;    // > 1: parts of the sum to part[split][M][N] in place of the epilogue
    float *part;
    Epilogue e;
};

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(_Float16 v) { return (float)v; }
__device__ __forceinline__ float as_float(__bf16 v) { return (float)v; }
__device__ __forceinline__ float as_float(uint8_t v) { return __builtin_amdgcn_cvt_f32_fp8((int)v, 0); }

// A tile of 64 x 64 in registers, 4 x 4 to a lane; 16 of the sum's terms at a time through LDS.
template <class T> __global__ __launch_bounds__(256) void k_product(ProductArgs p)
{
    constexpr int tile = 64, depth = 16;
    __shared__ float la[depth][tile + 1], lb[depth][tile + 1];
    const uint32_t live = p.rows.live();
    const uint32_t M = p.rows_are_k ? p.M : min(p.M, live), K = p.rows_are_k ? min(p.K, live) : p.K;
    const uint32_t m0 = blockIdx.x * tile, n0 = blockIdx.y * tile, split = blockIdx.z;
    if (m0 >= M) return;
    const uint32_t share = ((K + p.splits - 1) / p.splits + depth - 1) / depth * depth;
    const uint32_t k_first = min((uint64_t)K, (uint64_t)share * split), k_last = min((uint64_t)K, (uint64_t)k_first + share);
    const T *a = static_cast<const T *>(p.a.p), *b = static_cast<const T *>(p.b.p);
    float acc[4][4] = {};
    const uint32_t tm = threadIdx.x / 16, tn = threadIdx.x % 16;
    for (uint32_t k0 = k_first; k0 < k_last; k0 += depth) {
        for (uint32_t e = threadIdx.x; e < tile * depth; e += 256) {
            const bool a_k = p.a.sk == 1, b_k = p.b.sk == 1; // (lanes along the dimension whose elements lie side by side)
            const uint32_t ia = a_k ? e / depth : e % tile, ka = a_k ? e % depth : e / tile;
            const uint32_t ib = b_k ? e / depth : e % tile, kb = b_k ? e % depth : e / tile;
            la[ka][ia] = m0 + ia < M && k0 + ka < k_last ? as_float(a[(m0 + ia) * p.a.si + (k0 + ka) * p.a.sk]) : 0.0f;
            lb[kb][ib] = n0 + ib < p.N && k0 + kb < k_last ? as_float(b[(n0 + ib) * p.b.si + (k0 + kb) * p.b.sk]) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < depth; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(la[k][tm * 4 + i], lb[k][tn + 16 * j], acc[i][j]);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t m = m0 + tm * 4 + i, n = n0 + tn + 16 * j;
            if (m >= M || n >= p.N) continue;
            if (p.splits > 1) p.part[((uint64_t)split * p.M + m) * p.N + n] = acc[i][j];
            else finish1(p.e, m, n, acc[i][j]);
        }
}

// the sum over the splits, in order, and what happens to it
__global__ __launch_bounds__(256) void k_join(ProductArgs p)
{
    const uint64_t cells = (uint64_t)p.M * p.N;
    for (uint64_t i = blockIdx.x * 256ull + threadIdx.x; i < cells; i += gridDim.x * 256ull) {
        float v = 0.0f;
        for (uint32_t s = 0; s < p.splits; ++s) v += p.part[s * cells + i];
        finish1(p.e, (uint32_t)(i / p.N), (uint32_t)(i % p.N), v);
    }
}

// dZ without dropout's factor (dropped cells 0), and the sums of dZ over a workgroup's rows.  A lane has eight columns.
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
    Drop drop;
};

template <class TO, class T> __global__ __launch_bounds__(256) void k_slope(SlopeArgs a)
{
    __shared__ float lds[256 * 8];
    const uint32_t live = a.rows.live(), lane = threadIdx.x % a.lanes, in_block = 256 / a.lanes, mine = threadIdx.x / a.lanes;
    const uint32_t g = blockIdx.x * a.lanes + lane;
    const int left = (int)a.cols - (int)(8 * g);
    float sums[8] = {};
    for (uint64_t r = (uint64_t)blockIdx.y * in_block + mine; r < live && left > 0; r += (uint64_t)gridDim.y * in_block) {
        float v[8];
        load8(static_cast<const TO *>(a.dy) + r * a.ld_dy + 8 * g, left, v);
        if (a.drop.cut) mask8(a.drop, mask_id(a.drop, (uint32_t)r), g, 1.0f, v);
        if (a.act != ZG_ACT_NONE) {
            float z[8];
            load8(static_cast<const TO *>(a.z) + r * a.ld_z + 8 * g, left, z);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= act_slope(a.act, z[j]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[j] += v[j];
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

int launch_product(hipStream_t st, int32_t type, const ProductArgs &p)
{
    const dim3 grid((p.M + 63) / 64, (p.N + 63) / 64, p.splits);
    if (type == ZG_F32) ZG_TRY(launch(st, k_product<float>, grid, 256, p));
    else if (type == ZG_F16) ZG_TRY(launch(st, k_product<_Float16>, grid, 256, p));
    else if (type == ZG_BF16) ZG_TRY(launch(st, k_product<__bf16>, grid, 256, p));
    else ZG_TRY(launch(st, k_product<uint8_t>, grid, 256, p));
    if (p.splits == 1) return ZG_OK;
    const uint64_t cells = (uint64_t)p.M * p.N;
    return launch(st, k_join, dim3((unsigned)std::min<uint64_t>(4096, (cells + 255) / 256)), 256, p);
}

// How the gradients' workspace is laid out.
struct GradPlan {
    bool slopes;       // dZ differs from dY (a slope, a mask or another type): it is written out
    int64_t ld_dz;
    uint32_t lanes, slope_x, slope_y; // of k_slope
    uint32_t splits;   // parts of dW's sum over the rows
    size_t off_dz, off_part, off_dw, total;
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
    const int64_t tiles = (int64_t)((a.out + 63) / 64) * ((a.in + 63) / 64);
    g.splits = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(1024 / tiles, (a.rows + 255) / 256));
    if (g.slopes && (a.d_dA || a.d_dW)) g.off_dz = take((size_t)a.rows * g.ld_dz * type_size(a.dtype));
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
        if (a->d_Y == a->d_A || a->d_Z == a->d_A || a->d_Z == a->d_Y || (a->d_Z && a->d_Z == a->d_R))
            return fail(ZG_EINVAL, "an output lies on an input or on the other output");
        ProductArgs p{};
        p.a = {a->d_A, a->ld_A, 1};
        p.b = {a->d_W, a->ld_W, 1};
        p.M = (uint32_t)a->rows, p.N = (uint32_t)a->out, p.K = (uint32_t)a->in;
        p.rows = {a->d_rows, p.M};
        p.splits = 1;
        p.e.factor = 1.0f;
        p.e.scale_m = a->d_scale_A, p.e.scale_n = a->d_scale_W, p.e.bias = a->d_bias;
        p.e.act = a->act, p.e.type = a->out_dtype, p.e.drop = make_drop(a->drop);
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
            s.drop = drop;
            const dim3 grid(g.slope_x, g.slope_y);
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
        p.e.type = a->dtype;
        if (a->d_dA && a->rows > 0) {
            p.a = {dz, ld_dz, 1};
            p.b = {a->d_W, 1, a->ld_W};
            p.M = (uint32_t)a->rows, p.N = (uint32_t)a->in, p.K = (uint32_t)a->out;
            p.splits = 1;
            p.e.Y = a->d_dA, p.e.ld_Y = a->ld_dA;
            ZG_TRY(launch_product(st, a->dtype, p));
        }
        if (a->d_dW) {
            p.a = {dz, 1, ld_dz};
            p.b = {a->d_A, 1, a->ld_A};
            p.M = (uint32_t)a->out, p.N = (uint32_t)a->in, p.K = (uint32_t)a->rows;
            p.rows_are_k = 1;
            p.splits = g.splits;
            p.part = reinterpret_cast<float *>(ws + g.off_dw);
            p.e.Y = a->d_dW, p.e.ld_Y = a->ld_dW;
            ZG_TRY(launch_product(st, a->dtype, p));
        }
        return ZG_OK;
    });
}

} // extern "C"
