// A matrix whose singular values are brought near one by Newton-Schulz products, and the weights' update that uses it.
//
// X = G / (|G| + eps); a step is A = X X^T, B = b A + c A^2, X = a X + B X (on the shorter side; X^T X and X B where G is tall): singular values s become a s + b s^3 + c s^5.
// Between the steps X is held as two fp16 planes (x = high + low: 22 bits) at a power of two, once as G lies (P) and once turned (Q), so that every product's operands lie along their sums:
//   wide:  A = P P^T,  P' = a P + B Q^T        tall:  A = Q Q^T,  P' = a P + P B^T        (B is symmetric)
// and leaves its tile turned beside itself.  A and B are symmetric: only the tiles that reach down to the diagonal are made, and go out mirrored.  A bfloat16 result is made with the high planes as operands
// (one rounding of 2^-12 of each); others with both planes of both operands, three products: high x high, high x low and low x high.
#include "zg_product.h"

namespace zg {
namespace {

typedef _Float16 f16;

// ---- the products -----------------------------------------------------------------------------------------------------------------

// What a product is for: A or B (symmetric), X between two steps (goes out turned, too), or the result.
enum { kSquare, kStep, kResult };

template <int SEGMENTS, int KIND> struct StepArgs : ProductArgs { // v = alpha sum + beta R
    static constexpr bool symmetric = KIND == kSquare;
    static constexpr int segments = SEGMENTS;
    int64_t low_a, low_b; // bytes from the operands' high planes to their low ones
    float alpha, beta;
    const f16 *R, *R_low; // R may be null, R_low too
    int64_t ld_R;
    f16 *H, *L; // v's planes; L may be null
    int64_t ld_H;
    f16 *TH, *TL; // the same turned (of kSquare: H and L); TL may be null
    int64_t ld_T;
    void *O; // kResult: O = v, or O = keep O + v
    int64_t ld_O;
    int32_t type_O;
    bool update;
    float keep;

    // low x high, high x high, high x low
    __device__ __forceinline__ int64_t plane_a(int segment) const { return segment == 0 ? low_a : 0; }
    __device__ __forceinline__ int64_t plane_b(int segment) const { return segment == 2 ? low_b : 0; }
};

// eight cells' planes; zeros behind the first n
__device__ __forceinline__ void put_planes(f16 *h, f16 *l, int64_t at, int n, const float (&v)[8])
{
    f16 high[8], low[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float x = j < n ? v[j] : 0.0f;
        high[j] = (f16)x;
        low[j] = (f16)(x - (float)high[j]);
    }
    __builtin_memcpy(h + at, high, 16);
    if (l) __builtin_memcpy(l + at, low, 16);
}

// cells (m, n .. n + 7) from their sums to where they go; v becomes what they are
template <int SEGMENTS, int KIND> __device__ __forceinline__ void step8(const StepArgs<SEGMENTS, KIND> &p, uint32_t m, uint32_t n, float (&v)[8])
{
    const int left = (int)(p.N - n);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= p.alpha;
    if (p.R) { // (its rows are whole chunks)
        float r[8], l[8] = {};
        load8(p.R + m * p.ld_R + n, r);
        if (p.R_low) load8(p.R_low + m * p.ld_R + n, l);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(p.beta, r[j], fmaf(p.beta, l[j], v[j]));
    }
    if constexpr (KIND == kResult) {
        if (p.update) {
            float w[8];
            load8(p.O, p.type_O, m * p.ld_O + n, left, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = fmaf(p.keep, w[j], v[j]);
        }
        store8(p.O, p.type_O, m * p.ld_O + n, left, v);
    } else {
        put_planes(p.H, p.L, m * p.ld_H + n, left, v);
    }
}

// Through LDS of 4 KB, 32 x 32 cells at a time: four lanes have 32 columns of a row, then four lanes have 32 rows of a column.
template <int SEGMENTS, int KIND, int FM, int FN>
__device__ __forceinline__ void hand_over_step(const StepArgs<SEGMENTS, KIND> &p, f32x16 (&acc)[FM][FN], f32x4 *mine, uint32_t m_wave, uint32_t n_wave)
{
    const uint32_t lane = threadIdx.x & 63, half = lane >> 5, row = lane & 31, g = lane & 3;
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const uint32_t m0 = m_wave + 32 * i, n0 = n_wave + 32 * j;
            if (m0 >= p.M || n0 >= p.N || (KIND == kSquare && m0 < n0)) continue; // (the same in all lanes)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                mine[row * 8 + ((2 * q + half) ^ ((row >> 1) & 7))] = f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            lds_exchange();
            float v[2][8];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t r = (lane >> 2) + 16 * u;
                const f32x4 lo = mine[r * 8 + ((2 * g) ^ ((r >> 1) & 7))], hi = mine[r * 8 + ((2 * g + 1) ^ ((r >> 1) & 7))];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[u][k] = lo[k], v[u][4 + k] = hi[k];
                if (m0 + r < p.M && n0 + 8 * g < p.N) step8(p, m0 + r, n0 + 8 * g, v[u]);
            }
            lds_exchange();
            if (KIND != kResult && !(KIND == kSquare && m0 == n0)) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t r = (lane >> 2) + 16 * u;
                    mine[r * 8 + ((2 * g) ^ ((r >> 1) & 7))] = f32x4{v[u][0], v[u][1], v[u][2], v[u][3]};
                    mine[r * 8 + ((2 * g + 1) ^ ((r >> 1) & 7))] = f32x4{v[u][4], v[u][5], v[u][6], v[u][7]};
                }
                lds_exchange();
                const float *const cells = reinterpret_cast<const float *>(mine);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t c = (lane >> 2) + 16 * u;
                    float t[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const uint32_t r = 8 * g + k;
                        t[k] = cells[(r * 8 + ((c >> 2) ^ ((r >> 1) & 7))) * 4 + (c & 3)];
                    }
                    if (n0 + c < p.N && m0 + 8 * g < p.M) put_planes(p.TH, p.TL, (n0 + c) * p.ld_T + m0 + 8 * g, (int)(p.M - m0 - 8 * g), t);
                }
                lds_exchange();
            }
            __builtin_amdgcn_sched_barrier(0);
        }
}

template <int SEGMENTS, int KIND> struct Out<StepArgs<SEGMENTS, KIND>> {
    using Args = StepArgs<SEGMENTS, KIND>;
    static constexpr bool turns = KIND != kResult;
    template <class O, bool PLAIN, int FM> __device__ __forceinline__ static void wide(const Args &p, f32x16 (&acc)[FM][2], f32x4 *mine, uint32_t m_wave, uint32_t n_wave, uint32_t, uint32_t)
    {
        hand_over_step(p, acc, mine, m_wave, n_wave);
    }
    template <class O, bool PLAIN, int FM, int FN> __device__ __forceinline__ static void narrow(const Args &p, f32x16 (&acc)[FM][FN], f32x4 *mine, uint32_t m_wave, uint32_t n_wave, uint32_t, uint32_t)
    {
        hand_over_step(p, acc, mine, m_wave, n_wave);
    }
    struct Few {
        uint32_t n;
        __device__ __forceinline__ void begin(const Args &, uint32_t, uint32_t at, uint32_t) { n = at; }
        template <class F> __device__ __forceinline__ void end(const Args &p, uint32_t m, uint32_t live, F &&sums, float (&v)[8])
        {
            sums(0, v);
            if (m < live && n < p.N) step8(p, m, n, v);
        }
        template <class F> __device__ __forceinline__ void end(const Args &p, uint32_t m, uint32_t live, F &&sums)
        {
            float v[8];
            end(p, m, live, sums, v);
        }
        __device__ __forceinline__ void turned(const Args &p, uint32_t c, uint32_t m, float (&v)[8])
        {
            if (c < p.N && m < p.M) put_planes(p.TH, p.TL, c * p.ld_T + m, (int)(p.M - m), v);
        }
    };
};

template <int SEGMENTS, int KIND> __global__ __launch_bounds__(256) void k_step_few(StepArgs<SEGMENTS, KIND> p) { few_tile<f16>(p); }
template <int SEGMENTS, int KIND> __global__ __launch_bounds__(256, 3) void k_step_chunks(StepArgs<SEGMENTS, KIND> p) { chunks_tile<f16, f16, 128, 128, false, false>(p); }
template <int SEGMENTS, int KIND> __global__ __launch_bounds__(512, 2) void k_step_long(StepArgs<SEGMENTS, KIND> p) { long_tiles<f16, f16, false, false>(p); }

// ---- what the steps begin with ------------------------------------------------------------------------------------------------------

struct StartArgs {
    uint32_t rows, cols;
    const void *g;
    int64_t ld_g;
    float *m; // null: the matrix is g itself
    int64_t ld_m;
    float momentum;
    bool nesterov;
    double eps;
    double *sums; // [workgroups of k_start_norm]
    uint32_t n_sums;
    float power; // of two, that P and Q are held with
    f16 *P, *P_low, *Q, *Q_low; // Q_low may be null
    int64_t ld_P, ld_Q;
};

// eight elements of the matrix, from the momentum as k_start_norm leaves it
template <class T> __device__ __forceinline__ void start8(const StartArgs &a, uint64_t r, uint32_t c, float (&v)[8])
{
    const int left = (int)(a.cols - c);
    if (!a.m) {
        load8(static_cast<const T *>(a.g) + r * a.ld_g + c, left, v);
        return;
    }
    load8(a.m + r * a.ld_m + c, left, v);
    if (!a.nesterov) return;
    float g[8];
    load8(static_cast<const T *>(a.g) + r * a.ld_g + c, left, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = a.momentum * v[j] + g[j];
}

constexpr int kNormBlocks = 512;

// The momentum, and the sum of the squares of a workgroup's elements, in 64 bits (fp32's squares end at 1.8e19).
template <class T> __global__ __launch_bounds__(256) void k_start_norm(StartArgs a)
{
    __shared__ double lds[256];
    const uint32_t groups = (a.cols + 7) / 8;
    const uint64_t n = (uint64_t)a.rows * groups;
    double sum = 0.0;
    for (uint64_t i = blockIdx.x * 256ull + threadIdx.x; i < n; i += 256ull * gridDim.x) {
        const uint64_t r = i / groups;
        const uint32_t c = (uint32_t)(i - r * groups) * 8;
        float v[8];
        if (a.m) {
            const int left = (int)(a.cols - c);
            float g[8];
            load8(static_cast<const T *>(a.g) + r * a.ld_g + c, left, g);
            load8(a.m + r * a.ld_m + c, left, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = a.momentum * v[j] + g[j];
            store8(a.m + r * a.ld_m + c, left, v);
            if (a.nesterov) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = a.momentum * v[j] + g[j];
            }
        } else {
            start8<T>(a, r, c, v);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += (double)v[j] * (double)v[j];
    }
    lds[threadIdx.x] = sum;
    __syncthreads();
    for (int k = 128; k > 0; k >>= 1) {
        if (threadIdx.x < (unsigned)k) lds[threadIdx.x] += lds[threadIdx.x + k];
        __syncthreads();
    }
    if (threadIdx.x == 0) a.sums[blockIdx.x] = lds[0];
}

// P and Q: 64 x 64 elements to a workgroup, turned through LDS.
template <class T> __global__ __launch_bounds__(256) void k_start_planes(StartArgs a)
{
    __shared__ double sums[256];
    __shared__ float lds[64][65];
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < a.n_sums; i += 256) sum += a.sums[i];
    sums[threadIdx.x] = sum;
    __syncthreads();
    for (int k = 128; k > 0; k >>= 1) {
        if (threadIdx.x < (unsigned)k) sums[threadIdx.x] += sums[threadIdx.x + k];
        __syncthreads();
    }
    const double factor = (double)a.power / (sqrt(sums[0]) + a.eps);
    const uint32_t across = (a.cols + 63) / 64, r0 = block_number() / across * 64, c0 = block_number() % across * 64;
    const uint32_t i = threadIdx.x >> 3, c = 8 * (threadIdx.x & 7);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t r = i + 32 * h;
        float v[8] = {};
        if (r0 + r < a.rows && c0 + c < a.cols) {
            start8<T>(a, r0 + r, c0 + c, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (float)((double)v[j] * factor);
            put_planes(a.P, a.P_low, (uint64_t)(r0 + r) * a.ld_P + c0 + c, (int)(a.cols - c0 - c), v);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) lds[r][c + j] = v[j];
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t q = i + 32 * h; // a column, eight rows of it
        if (c0 + q >= a.cols || r0 + c >= a.rows) continue;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = lds[c + j][q];
        put_planes(a.Q, a.Q_low, (uint64_t)(c0 + q) * a.ld_Q + r0 + c, (int)(a.rows - r0 - c), v);
    }
}

// ---- host side --------------------------------------------------------------------------------------------------------------------

// Singular values of at most `top`: what a step makes of them at most, and B's.  Where the derivative is 0 or at the end.
struct Bounds {
    double x, b;
};

Bounds bounds_of(double top, const float *k)
{
    const double a = k[0], b = k[1], c = k[2], end = top * top;
    Bounds r{0.0, 0.0};
    const auto at = [&](double t) { // t = s^2
        if (!(t >= 0.0 && t <= end)) return;
        r.x = std::max(r.x, std::fabs(std::sqrt(t) * (a + t * (b + t * c))));
        r.b = std::max(r.b, std::fabs(t * (b + t * c)));
    };
    at(end);
    if (c != 0.0) {
        at(-b / (2.0 * c));
        const double under = 9.0 * b * b - 20.0 * a * c;
        if (under >= 0.0) at((-3.0 * b + std::sqrt(under)) / (10.0 * c)), at((-3.0 * b - std::sqrt(under)) / (10.0 * c));
    } else if (b != 0.0) {
        at(-a / (3.0 * b));
    }
    return r;
}

// the exponent that values of at most `top` are held with in fp16, whose range ends at 65504
int exponent_for(double top) { return top > 0.0 ? std::min(24, 14 - (int)std::ceil(std::log2(top))) : 24; }

constexpr double kMostTop = 1024.0; // singular values that a step may reach

struct Common { // of both calls
    int32_t rows, cols, dtype, steps; // dtype: of what is read
    double eps;
    const float *coefficients;
    int32_t type; // of the result
};

int check_steps(const Common &c)
{
    if (c.rows < 1 || c.rows > ZG_MAX_WIDTH || c.cols < 1 || c.cols > ZG_MAX_WIDTH) return fail(ZG_EINVAL, "rows or cols outside 1.." + std::to_string(ZG_MAX_WIDTH));
    if (!wide_type(c.dtype) || !wide_type(c.type)) return fail(ZG_EINVAL, "a type that is not ZG_F32, ZG_F16 or ZG_BF16");
    if (c.steps < 1 || c.steps > ZG_MAX_NEWTON_STEPS) return fail(ZG_EINVAL, "steps outside 1.." + std::to_string(ZG_MAX_NEWTON_STEPS));
    if (!(c.eps >= 0.0 && c.eps <= 3.0e38)) return fail(ZG_EINVAL, "eps is negative or not finite");
    if (!c.coefficients) return fail(ZG_EINVAL, "coefficients is null");
    double top = 1.0;
    for (int s = 0; s < c.steps; ++s) {
        for (int i = 0; i < 3; ++i)
            if (!std::isfinite(c.coefficients[3 * s + i])) return fail(ZG_EINVAL, "a coefficient is not finite");
        const Bounds b = bounds_of(top, c.coefficients + 3 * s);
        top = b.x;
        if (!(top <= kMostTop && b.b <= kMostTop * kMostTop)) return fail(ZG_EINVAL, "the coefficients let singular values grow beyond 1024");
    }
    return ZG_OK;
}

struct StepPlan {
    bool wide, pairs;
    uint32_t small, large; // the sides
    int64_t ld_P, ld_Q, ld_A;
    uint32_t n_sums;
    size_t off_sums, off_P[2], off_Q[2], off_A, off_B, total;
    int64_t plane_P, plane_Q, plane_A; // elements
};

StepPlan step_plan(const Common &c)
{
    StepPlan t{};
    const auto take = [&](size_t bytes) {
        const size_t at = t.total;
        t.total = (t.total + bytes + 255) / 256 * 256;
        return at;
    };
    const auto up = [](int64_t n) { return (n + 7) / 8 * 8; };
    t.wide = c.rows <= c.cols;
    t.small = (uint32_t)std::min(c.rows, c.cols), t.large = (uint32_t)std::max(c.rows, c.cols);
    t.pairs = c.type != ZG_BF16 || t.small < 256 || c.steps > 6;
    t.ld_P = up(c.cols), t.ld_Q = up(c.rows), t.ld_A = up(t.small);
    t.plane_P = c.rows * t.ld_P, t.plane_Q = c.cols * t.ld_Q, t.plane_A = t.small * t.ld_A;
    t.n_sums = (uint32_t)std::min<int64_t>(kNormBlocks, ((int64_t)c.rows * ((c.cols + 7) / 8) + 255) / 256);
    t.off_sums = take(t.n_sums * sizeof(double));
    for (int i = 0; i < 2; ++i) t.off_P[i] = take((size_t)t.plane_P * 2 * sizeof(f16)), t.off_Q[i] = take((size_t)t.plane_Q * (t.pairs ? 2 : 1) * sizeof(f16));
    t.off_A = take((size_t)t.plane_A * 2 * sizeof(f16));
    t.off_B = take((size_t)t.plane_A * 2 * sizeof(f16));
    return t;
}

template <int SEGMENTS, int KIND> int launch_step(hipStream_t st, const StepArgs<SEGMENTS, KIND> &p)
{
    const auto blocks = [&](uint32_t tile) -> uint64_t {
        const uint64_t m = (p.M + tile - 1) / tile, n = (p.N + tile - 1) / tile;
        return KIND == kSquare ? n * (n + 1) / 2 : m * n;
    };
    if (blocks(128) < 128) return launch(st, k_step_few<SEGMENTS, KIND>, grid_of(blocks(32)), 256, p);
    if (blocks(256) < 256) return launch(st, k_step_chunks<SEGMENTS, KIND>, grid_of((blocks(128) + 7) / 8 * 8), 256, p);
    return launch(st, k_step_long<SEGMENTS, KIND>, dim3(256), 512, p);
}

struct Result {
    void *O;
    int64_t ld;
    bool update;
    float keep, factor; // O = keep O + factor X, or factor X
};

template <int SEGMENTS> int run_steps(hipStream_t st, const Common &c, const StepPlan &t, char *ws, const Result &out)
{
    f16 *P[2], *Q[2], *const A = reinterpret_cast<f16 *>(ws + t.off_A), *const B = reinterpret_cast<f16 *>(ws + t.off_B);
    for (int i = 0; i < 2; ++i) P[i] = reinterpret_cast<f16 *>(ws + t.off_P[i]), Q[i] = reinterpret_cast<f16 *>(ws + t.off_Q[i]);
    const bool pairs = SEGMENTS > 1;
    const int64_t low_P = t.plane_P * (int64_t)sizeof(f16), low_Q = t.plane_Q * (int64_t)sizeof(f16), low_A = t.plane_A * (int64_t)sizeof(f16);
    const auto up = [](uint32_t n) { return (n + 7) / 8 * 8; };
    const auto start = [&](auto &p, Operand a, int64_t low_a, Operand b, int64_t low_b, uint32_t M, uint32_t N, uint32_t K) {
        p.a = a, p.b = b, p.low_a = low_a, p.low_b = low_b;
        p.M = M, p.N = N, p.K = up(K);
        p.rows = {nullptr, M};
        p.splits = 1;
    };
    const Operand of_A{A, t.ld_A, false, true}, of_B{B, t.ld_A, false, true};
    double top = 1.0;
    int ex = exponent_for(top);
    for (int s = 0, at = 0; s < c.steps; ++s, at ^= 1) {
        const float *const k = c.coefficients + 3 * s;
        const Bounds next = bounds_of(top, k);
        const int ea = exponent_for(top * top), eb = exponent_for(next.b), en = exponent_for(next.x);
        const Operand of_P{P[at], t.ld_P, false, true}, of_Q{Q[at], t.ld_Q, false, true};
        {
            StepArgs<SEGMENTS, kSquare> p{}; // A = X X^T
            const Operand x = t.wide ? of_P : of_Q;
            start(p, x, t.wide ? low_P : low_Q, x, t.wide ? low_P : low_Q, t.small, t.small, t.large);
            p.alpha = std::ldexp(1.0f, ea - 2 * ex);
            p.H = p.TH = A, p.L = p.TL = pairs ? A + t.plane_A : nullptr, p.ld_H = p.ld_T = t.ld_A;
            ZG_TRY(launch_step(st, p));
        }
        {
            StepArgs<SEGMENTS, kSquare> p{}; // B = b A + c A^2
            start(p, of_A, low_A, of_A, low_A, t.small, t.small, t.small);
            p.alpha = std::ldexp(k[2], eb - 2 * ea), p.beta = std::ldexp(k[1], eb - ea);
            p.R = A, p.R_low = pairs ? A + t.plane_A : nullptr, p.ld_R = t.ld_A;
            p.H = p.TH = B, p.L = p.TL = pairs ? B + t.plane_A : nullptr, p.ld_H = p.ld_T = t.ld_A;
            ZG_TRY(launch_step(st, p));
        }
        const auto last = [&](auto &p, double factor, int exponent) { // a P + B Q^T, or a P + P B^T
            if (t.wide) start(p, of_B, low_A, of_Q, low_Q, (uint32_t)c.rows, (uint32_t)c.cols, t.small);
            else start(p, of_P, low_P, of_B, low_A, (uint32_t)c.rows, (uint32_t)c.cols, t.small);
            p.alpha = (float)std::ldexp(factor, exponent - eb - ex), p.beta = (float)std::ldexp(factor * k[0], exponent - ex);
            p.R = P[at], p.R_low = P[at] + t.plane_P, p.ld_R = t.ld_P;
        };
        if (s + 1 < c.steps) {
            StepArgs<SEGMENTS, kStep> p{};
            last(p, 1.0, en);
            p.H = P[at ^ 1], p.L = P[at ^ 1] + t.plane_P, p.ld_H = t.ld_P;
            p.TH = Q[at ^ 1], p.TL = pairs ? Q[at ^ 1] + t.plane_Q : nullptr, p.ld_T = t.ld_Q;
            ZG_TRY(launch_step(st, p));
        } else {
            StepArgs<SEGMENTS, kResult> p{};
            last(p, out.factor, 0);
            p.O = out.O, p.ld_O = out.ld, p.type_O = c.type, p.update = out.update, p.keep = out.keep;
            ZG_TRY(launch_step(st, p));
        }
        top = next.x, ex = en;
    }
    return ZG_OK;
}

int run(hipStream_t st, const Common &c, StartArgs a, char *ws, const Result &out)
{
    const StepPlan t = step_plan(c);
    a.rows = (uint32_t)c.rows, a.cols = (uint32_t)c.cols;
    a.eps = c.eps, a.sums = reinterpret_cast<double *>(ws + t.off_sums), a.n_sums = t.n_sums;
    a.power = std::ldexp(1.0f, exponent_for(1.0));
    a.P = reinterpret_cast<f16 *>(ws + t.off_P[0]), a.P_low = a.P + t.plane_P, a.ld_P = t.ld_P;
    a.Q = reinterpret_cast<f16 *>(ws + t.off_Q[0]), a.Q_low = t.pairs ? a.Q + t.plane_Q : nullptr, a.ld_Q = t.ld_Q;
    const dim3 planes = grid_of((uint64_t)((c.rows + 63) / 64) * ((c.cols + 63) / 64));
    const auto begin = [&](auto zero) -> int {
        using T = decltype(zero);
        ZG_TRY(launch(st, k_start_norm<T>, dim3(t.n_sums), 256, a));
        return launch(st, k_start_planes<T>, planes, 256, a);
    };
    ZG_TRY(c.dtype == ZG_F32 ? begin(float()) : c.dtype == ZG_F16 ? begin((f16)0) : begin((__bf16)0));
    return t.pairs ? run_steps<3>(st, c, t, ws, out) : run_steps<1>(st, c, t, ws, out);
}

int check_orthogonalize(const zg_orthogonalize_args *a, Common &c)
{
    if (!a) return fail(ZG_EINVAL, "null argument");
    c = {a->rows, a->cols, a->dtype, a->steps, a->eps, a->coefficients, a->out_dtype};
    return check_steps(c);
}

int check_muon(const zg_muon_args *a, Common &c)
{
    if (!a) return fail(ZG_EINVAL, "null argument");
    c = {a->rows, a->cols, a->grad_dtype, a->steps, a->eps, a->coefficients, a->dtype};
    for (const float v : {a->lr, a->momentum, a->decay, a->scale})
        if (!std::isfinite(v)) return fail(ZG_EINVAL, "lr, momentum, decay or scale is not finite");
    return check_steps(c);
}

} // namespace
} // namespace zg

using namespace zg;

extern "C" {
int zg_orthogonalize_workspace(const zg_orthogonalize_args *a, size_t *bytes)
{
    return entry([&]() -> int {
        Common c;
        ZG_TRY(check_orthogonalize(a, c));
        if (!bytes) return fail(ZG_EINVAL, "null argument");
        *bytes = step_plan(c).total;
        return ZG_OK;
    });
}

int zg_orthogonalize(const zg_orthogonalize_args *a, void *d_workspace, size_t workspace_bytes, void *stream)
{
    return entry([&]() -> int {
        Common c;
        ZG_TRY(check_orthogonalize(a, c));
        ZG_TRY(check_matrix("d_G", a->d_G, a->ld_G, a->cols, a->dtype));
        ZG_TRY(check_matrix("d_O", a->d_O, a->ld_O, a->cols, a->out_dtype));
        ZG_TRY(check_apart(matrix_span("d_O", a->d_O, a->rows, a->ld_O, a->cols, a->out_dtype), {}, {matrix_span("d_G", a->d_G, a->rows, a->ld_G, a->cols, a->dtype)}));
        ZG_TRY(check_workspace(d_workspace, workspace_bytes, step_plan(c).total));
        StartArgs s{};
        s.g = a->d_G, s.ld_g = a->ld_G;
        return run(static_cast<hipStream_t>(stream), c, s, static_cast<char *>(d_workspace), {a->d_O, a->ld_O, false, 0.0f, 1.0f});
    });
}

int zg_muon_step_workspace(const zg_muon_args *a, size_t *bytes)
{
    return entry([&]() -> int {
        Common c;
        ZG_TRY(check_muon(a, c));
        if (!bytes) return fail(ZG_EINVAL, "null argument");
        *bytes = step_plan(c).total;
        return ZG_OK;
    });
}

int zg_muon_step(const zg_muon_args *a, void *d_workspace, size_t workspace_bytes, void *stream)
{
    return entry([&]() -> int {
        Common c;
        ZG_TRY(check_muon(a, c));
        ZG_TRY(check_matrix("d_G", a->d_G, a->ld_G, a->cols, a->grad_dtype));
        ZG_TRY(check_matrix("d_M", a->d_M, a->ld_M, a->cols, ZG_F32));
        ZG_TRY(check_matrix("d_W", a->d_W, a->ld_W, a->cols, a->dtype));
        {
            const Span G = matrix_span("d_G", a->d_G, a->rows, a->ld_G, a->cols, a->grad_dtype), M = matrix_span("d_M", a->d_M, a->rows, a->ld_M, a->cols, ZG_F32);
            const Span W = matrix_span("d_W", a->d_W, a->rows, a->ld_W, a->cols, a->dtype);
            ZG_TRY(check_apart(M, {G, W}));
            ZG_TRY(check_apart(W, {G}));
        }
        ZG_TRY(check_workspace(d_workspace, workspace_bytes, step_plan(c).total));
        StartArgs s{};
        s.g = a->d_G, s.ld_g = a->ld_G, s.m = a->d_M, s.ld_m = a->ld_M, s.momentum = a->momentum, s.nesterov = a->nesterov != 0;
        const float keep = (float)(1.0 - (double)a->lr * (double)a->decay), factor = (float)(-(double)a->lr * (double)a->scale);
        return run(static_cast<hipStream_t>(stream), c, s, static_cast<char *>(d_workspace), {a->d_W, a->ld_W, true, keep, factor});
    });
}

} // extern "C"
