// A matrix whose singular values are brought near one by Newton-Schulz products, and the weights' update that uses it.
//
// X = G / (|G| + eps), turned where G is tall; a step is A = X X^T, B = b A + c A^2, X = a X + B X: singular values s become a s + b s^3 + c s^5.
// Between the products X, A and B are held as fp16 planes (x = high + low: 22 bits) at a power of two; X always has both, as it is added to what the products make of it.  A bfloat16 result of large sides is made with the
// high planes as operands (one rounding of 2^-12 of each) where the steps let that be (high_planes_do); others with both planes of both operands, three products: low x high, high x low and high x high.  A and B are symmetric: only
// the tiles that reach down to the diagonal are made, and go out mirrored.  The sums of B X run across the rows of X: tiles of 256 x 256 turn them as they are read from LDS, smaller ones, which that would
// hold up (1024 x 4096: 24 -> 30 us; pairs of 1024 x 2048 in tiles of 64 x 64: 27 -> 48), have X turned beside it.
#include "zg_product.h"

namespace zg {
namespace {

typedef _Float16 f16;

// ---- the products -----------------------------------------------------------------------------------------------------------------

// What a product is for: A or B (symmetric), X between two steps, or the result.
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
    f16 *TH, *TL; // the same turned (kSquare: H and L); TL may be null, of kStep TH, too
    int64_t ld_T;
    void *O; // kResult: O = v, or O = keep O + v, turned where G is tall
    int64_t ld_O;
    int32_t type_O;
    bool update, turn;
    float keep;

    // low x high, high x low, high x high: the sums are small until the last
    __device__ __forceinline__ int64_t plane_a(int segment) const { return segment == 0 ? low_a : 0; }
    __device__ __forceinline__ int64_t plane_b(int segment) const { return segment == 1 ? low_b : 0; }
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

// v of cells (m, n .. n + 7) from their sums
template <class Args> __device__ __forceinline__ void value8(const Args &p, uint32_t m, uint32_t n, float (&v)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= p.alpha;
    if (p.R) { // (its rows are whole chunks)
        float r[8], l[8] = {};
        load8(p.R + m * p.ld_R + n, r);
        if (p.R_low) load8(p.R_low + m * p.ld_R + n, l);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(p.beta, r[j], fmaf(p.beta, l[j], v[j]));
    }
}

// v of eight cells of a row of O, the first `left` of which there are
template <class Args> __device__ __forceinline__ void result8(const Args &p, uint32_t row, uint32_t col, int left, float (&v)[8])
{
    if (p.update) {
        float w[8];
        load8(p.O, p.type_O, row * p.ld_O + col, left, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(p.keep, w[j], v[j]);
    }
    store8(p.O, p.type_O, row * p.ld_O + col, left, v);
}

template <int SEGMENTS, int KIND> __device__ __forceinline__ void straight8(const StepArgs<SEGMENTS, KIND> &p, uint32_t m, uint32_t n, float (&v)[8])
{
    value8(p, m, n, v);
    if constexpr (KIND != kResult) put_planes(p.H, p.L, m * p.ld_H + n, (int)(p.N - n), v);
    else if (!p.turn) result8(p, m, n, (int)(p.N - n), v);
}

// cells (m .. m + 7, n)
template <int SEGMENTS, int KIND> __device__ __forceinline__ void turned8(const StepArgs<SEGMENTS, KIND> &p, uint32_t m, uint32_t n, float (&v)[8])
{
    if constexpr (KIND != kResult) put_planes(p.TH, p.TL, n * p.ld_T + m, (int)(p.M - m), v);
    else result8(p, n, m, (int)(p.M - m), v);
}

template <class Args> __device__ __forceinline__ bool goes_turned(const Args &p) { return p.TH || p.turn; }

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
                if (m0 + r < p.M && n0 + 8 * g < p.N) straight8(p, m0 + r, n0 + 8 * g, v[u]);
            }
            lds_exchange();
            if (KIND == kSquare ? m0 != n0 : goes_turned(p)) {
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
                    if (n0 + c < p.N && m0 + 8 * g < p.M) turned8(p, m0 + 8 * g, n0 + c, t);
                }
                lds_exchange();
            }
            __builtin_amdgcn_sched_barrier(0);
        }
}

template <int SEGMENTS, int KIND> struct Out<StepArgs<SEGMENTS, KIND>> {
    using Args = StepArgs<SEGMENTS, KIND>;
    static constexpr bool turns = true;
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
            if (m < live && n < p.N) straight8(p, m, n, v);
        }
        __device__ __forceinline__ void turned(const Args &p, uint32_t c, uint32_t m, float (&v)[8])
        {
            if (goes_turned(p) && c < p.N && m < p.M) turned8(p, m, c, v);
        }
    };
};

// Tiles of 64 x 64: four wavefronts, three workgroups to a compute unit, or two groups of four that share a tile's sums, one to a compute unit; of 128 x 128: one to a compute unit, four steps of
// 128 bytes on their way, or three with three of 64; of 256 x 256.  (What each is for, and what it takes, stands at time_of.)
template <int SEGMENTS, int KIND> __global__ __launch_bounds__(256) void k_step_few(StepArgs<SEGMENTS, KIND> p) { few_tile<f16>(p); }
template <int SEGMENTS> __global__ __launch_bounds__(512, 1) void k_step_shared(StepArgs<SEGMENTS, kSquare> p) { chunks_tile<f16, f16, 64, 64, false, false, 8, 3, 2>(p); }
template <int SEGMENTS, int KIND> __global__ __launch_bounds__(256, 3) void k_step_64(StepArgs<SEGMENTS, KIND> p) { chunks_tile<f16, f16, 64, 64, false, false, 8, 3>(p); }
template <int SEGMENTS, int KIND> __global__ __launch_bounds__(256, 1) void k_step_128(StepArgs<SEGMENTS, KIND> p) { chunks_tile<f16, f16, 128, 128, false, false, 8, 4>(p); }
template <int SEGMENTS, int KIND> __global__ __launch_bounds__(256, 3) void k_step_dense(StepArgs<SEGMENTS, KIND> p) { chunks_tile<f16, f16, 128, 128, false, false>(p); }
template <int SEGMENTS, int KIND> __global__ __launch_bounds__(512, 2) void k_step_256(StepArgs<SEGMENTS, KIND> p) { long_tiles<f16, f16, false, KIND != kSquare>(p); }

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
    float power; // of two, that the planes are held with
    f16 *P, *P_low, *Q, *Q_low; // the matrix' planes, and those of it turned: any may be null
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

// The planes: 64 x 64 elements to a workgroup, turned through LDS.
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
            if (a.P) put_planes(a.P, a.P_low, (uint64_t)(r0 + r) * a.ld_P + c0 + c, (int)(a.cols - c0 - c), v);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) lds[r][c + j] = v[j];
    }
    if (!a.Q) return;
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

// ---- small matrices, whole ----------------------------------------------------------------------------------------------------------
// Up to 64 x 384 (or turned): one workgroup of eight wavefronts has X, A and B in LDS, planes and all, from the norm to the result: one launch for 2 + 3 steps, each of which would last little more than
// a launch does.  Sums as in the other kernels (the low products apart).  Five steps of 16 x 16 take 21 us, of 64 x 64 27, 64 x 128 33, 47 x 256 46, 64 x 384 65, against 75 in launches; bound by one compute unit's way
// from LDS to the matrix instructions and back.

constexpr uint32_t kWholeSmall = 64, kWholeLarge = 384;

struct WholeArgs {
    StartArgs s; // P, Q and sums are not needed
    uint64_t inv; // ceil(2^32 / cols): e / cols == (e * inv) >> 32 for the elements of a small matrix
    bool tall;
    int32_t steps;
    float scalars[ZG_MAX_NEWTON_STEPS][5]; // A's, B's and X's alpha, B's and X's beta
    void *O;
    int64_t ld_O;
    int32_t type_O;
    bool update;
    float keep;
};

constexpr uint32_t kWholeX = kWholeLarge + 8, kWholeA = kWholeSmall + 8; // elements to a row in LDS: rows start in other banks

struct Pair {
    f16 *high, *low; // in LDS
    __device__ __forceinline__ void put(uint32_t at, float v) const
    {
        high[at] = (f16)v;
        low[at] = (f16)(v - (float)high[at]);
    }
    __device__ __forceinline__ float get(uint32_t at) const { return (float)high[at] + (float)low[at]; }
};

// a lane's eight k of its row, from a plane whose rows lie along k, or across it
__device__ __forceinline__ u32x4 along_k(const f16 *plane, uint32_t ld, uint32_t row, uint32_t k) { return *reinterpret_cast<const u32x4 *>(plane + row * ld + k); }
__device__ __forceinline__ u32x4 across_k(const f16 *plane, uint32_t ld, uint32_t row, uint32_t k)
{
    const uint32_t lane = threadIdx.x & 15, r = (row & ~15u) + 4 * (lane & 3);
    u32x4 v;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint64_t two = __builtin_bit_cast(uint64_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(plane + (k + 4 * h + (lane >> 2)) * ld + r)));
        v[2 * h] = (uint32_t)two, v[2 * h + 1] = (uint32_t)(two >> 32);
    }
    return v;
}

// 32 x 32 cells, k from `first` on, every `stride`th 16 of them: a's rows are the lane's, b's lie side by side
template <bool ACROSS> __device__ __forceinline__ f32x16 whole_product(const Pair &a, uint32_t ld_a, uint32_t row_a, const Pair &b, uint32_t ld_b, uint32_t row_b, uint32_t first, uint32_t end, uint32_t stride)
{
    f32x16 acc = {}, low = {};
    const uint32_t half = (threadIdx.x & 63) >> 5;
#pragma unroll 1
    for (uint32_t k0 = first; k0 < end; k0 += stride) {
        const uint32_t k = k0 + 8 * half;
        const u32x4 x = along_k(a.high, ld_a, row_a, k), lx = along_k(a.low, ld_a, row_a, k);
        const u32x4 y = ACROSS ? across_k(b.high, ld_b, row_b, k) : along_k(b.high, ld_b, row_b, k), ly = ACROSS ? across_k(b.low, ld_b, row_b, k) : along_k(b.low, ld_b, row_b, k);
        multiply((f16)0, y, lx, low);
        multiply((f16)0, ly, x, low);
        multiply((f16)0, y, x, acc);
    }
    return acc + low;
}

template <class T> __global__ __launch_bounds__(512) void k_step_whole(WholeArgs w)
{
    __shared__ f16 lds_x[2][kWholeSmall * kWholeX];
    __shared__ f16 lds_a[2][kWholeSmall * kWholeA];
    __shared__ __attribute__((aligned(16))) f16 lds_b[2][kWholeSmall * kWholeA];
    __shared__ double sums[8];
    static_assert(sizeof lds_b >= 4 * 16 * 64 * sizeof(float), "");
    const Pair X{lds_x[0], lds_x[1]}, A{lds_a[0], lds_a[1]}, B{lds_b[0], lds_b[1]};
    float *const half_sums = reinterpret_cast<float *>(lds_b); // (B is not there yet)
    const StartArgs &s = w.s;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t half = lane >> 5, row = lane & 31;
    const uint32_t small = w.tall ? s.cols : s.rows, large = w.tall ? s.rows : s.cols;
    const uint32_t high = (small + 31) / 32, wide = (large + 31) / 32; // tiles of 32

    // the momentum, the norm, and X; zeros around it.  A lane has every 512th element, all of them on their way at once.
    constexpr int most = kWholeSmall * kWholeLarge / 512;
    const uint32_t cells = s.rows * s.cols;
    const auto row_of = [&](uint32_t e) { return (uint32_t)((e * w.inv) >> 32); };
    float v[most], g[most];
#pragma unroll
    for (int i = 0; i < most; ++i) {
        const uint32_t e = threadIdx.x + 512 * i, r = row_of(e), c = e - r * s.cols;
        v[i] = g[i] = 0.0f;
        if (e >= cells) continue;
        g[i] = (float)static_cast<const T *>(s.g)[r * s.ld_g + c];
        if (s.m) v[i] = s.m[r * s.ld_m + c];
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < most; ++i) {
        const uint32_t e = threadIdx.x + 512 * i, r = row_of(e), c = e - r * s.cols;
        if (s.m) {
            v[i] = s.momentum * v[i] + g[i];
            if (e < cells) s.m[r * s.ld_m + c] = v[i];
            if (s.nesterov) v[i] = s.momentum * v[i] + g[i];
        } else {
            v[i] = g[i];
        }
        sum += (double)v[i] * (double)v[i];
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) sums[wave] = sum;
    for (uint32_t i = threadIdx.x; i < kWholeSmall * kWholeX / 8; i += 512) {
        reinterpret_cast<u32x4 *>(X.high)[i] = u32x4{};
        reinterpret_cast<u32x4 *>(X.low)[i] = u32x4{};
    }
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += sums[i];
    const double factor = (double)s.power / (sqrt(sum) + s.eps);
#pragma unroll
    for (int i = 0; i < most; ++i) {
        const uint32_t e = threadIdx.x + 512 * i, r = row_of(e), c = e - r * s.cols;
        if (e < cells) X.put(w.tall ? c * kWholeX + r : r * kWholeX + c, (float)((double)v[i] * factor));
    }
    __syncthreads();

    for (int step = 0; step < w.steps; ++step) {
        const float *const k = w.scalars[step];
        asm volatile("" : "+v"(half), "+v"(row)); // (or the addresses of all cells would be made, and kept, ahead of the first step)
        const uint32_t ti = (wave >> 1 & 1) * 32, tj = (wave & 1) * 32; // a wavefront's tile of A and B; two share A's sums
        const bool mine = ti < 32 * high && tj < 32 * high;
        f32x16 acc = {};
        if (mine) acc = whole_product<false>(X, kWholeX, ti + row, X, kWholeX, tj + row, (wave >> 2) * 16, 32 * wide, 32);
        if (wave >= 4) {
#pragma unroll
            for (int r = 0; r < 16; ++r) half_sums[((wave - 4) * 16 + r) * 64 + lane] = acc[r];
        }
        __syncthreads();
        if (wave < 4 && mine) {
#pragma unroll
            for (int r = 0; r < 16; ++r) A.put((ti + row) * kWholeA + tj + 8 * (r / 4) + 4 * half + r % 4, k[0] * (acc[r] + half_sums[(wave * 16 + r) * 64 + lane]));
        }
        __syncthreads();
        if (wave < 4 && mine) {
            acc = whole_product<false>(A, kWholeA, ti + row, A, kWholeA, tj + row, 0, 32 * high, 16);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t at = (ti + row) * kWholeA + tj + 8 * (r / 4) + 4 * half + r % 4;
                B.put(at, fmaf(k[3], A.get(at), k[1] * acc[r]));
            }
        }
        __syncthreads();
        const bool last = step + 1 == w.steps;
        float next[3][16];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const uint32_t t = wave + 8 * i, m0 = t % high * 32, n0 = t / high * 32;
            if (n0 >= 32 * wide) continue;
            acc = whole_product<true>(B, kWholeA, m0 + row, X, kWholeX, n0 + row, 0, 32 * high, 16);
#pragma unroll
            for (int r = 0; r < 16; ++r) next[i][r] = fmaf(k[4], X.get((m0 + row) * kWholeX + n0 + 8 * (r / 4) + 4 * half + r % 4), k[2] * acc[r]);
            __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const uint32_t t = wave + 8 * i, m = t % high * 32 + row, n0 = t / high * 32;
            if (n0 >= 32 * wide) continue;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t n = n0 + 8 * (r / 4) + 4 * half + r % 4;
                if (!last) {
                    X.put(m * kWholeX + n, next[i][r]);
                } else if (m < small && n < large) {
                    const int64_t at = w.tall ? n * w.ld_O + m : m * w.ld_O + n;
                    if (w.type_O == ZG_F32) {
                        float *const o = static_cast<float *>(w.O) + at;
                        *o = w.update ? fmaf(w.keep, *o, next[i][r]) : next[i][r];
                    } else if (w.type_O == ZG_F16) {
                        f16 *const o = static_cast<f16 *>(w.O) + at;
                        *o = (f16)(w.update ? fmaf(w.keep, (float)*o, next[i][r]) : next[i][r]);
                    } else {
                        __bf16 *const o = static_cast<__bf16 *>(w.O) + at;
                        *o = (__bf16)(w.update ? fmaf(w.keep, (float)*o, next[i][r]) : next[i][r]);
                    }
                }
            }
        }
        __syncthreads();
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

// The exponent that values of at most `top` are held with in fp16, whose range ends at 65504.  Up to 100 the products' factors, differences of three of these, are numbers of fp32, or of no account beside what they are added to.
int exponent_for(double top) { return top > 0.0 ? std::min(100, 14 - (int)std::ceil(std::log2(top))) : 0; }

constexpr double kMostTop = 1024.0; // singular values that a step may reach (b s^2 + c s^4 is at most 36 times that over what they were, as for any odd polynomial of degree 5 that stays below it)

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
        if (!(top <= kMostTop)) return fail(ZG_EINVAL, "the coefficients let singular values grow beyond 1024");
    }
    return ZG_OK;
}

// How a product is made, and about how long that takes, in us, as measured on an MI355X: `k` terms, a pair's three products being three times as many; small tiles' cost is what they read, once a
// pair's two planes.  fp16, [M, N] x K terms, few / 64 / shared / 128 / dense / 256: symmetric 256 x 256 4.3 / 4.8 / 5.1 / 9 / 9 / 14; 512 x 512 5.4 / 5.9 / 5.9 / 11 / 11 / 20;
// 1024 x 1024 14 / 8.2 / 7.8 / 15 / 16 / 30, over 4096 terms 48 / 21 / 16 / 36 / 41 / 82; 2048 73 / 23 / 30 / 24 / 25 / 49; 4096 557 / 154 / - / 127 / 128 / 101;
// whole 1024 x 2048 x 1024 36 / 14 / 20 / 20 / 21 / 37; 1024 x 4096 x 1024 67 / 27 / 37 / 24 / 24 / 39; 2048 x 2048 x 2048 128 / 41 / 54 / 32 / 33 / 58; 4096 1019 / 314 / - / 211 / 218 / 161.
enum Way { kFew, kShared, k64, k128, kDense, k256, kWays };

uint64_t tiles_of(uint32_t M, uint32_t N, bool symmetric, uint32_t tile)
{
    const uint64_t m = (M + tile - 1) / tile, n = (N + tile - 1) / tile;
    return symmetric ? n * (n + 1) / 2 : m * n;
}

double time_of(Way way, uint32_t M, uint32_t N, uint32_t K, bool symmetric, bool pairs)
{
    const double k = (double)K * (pairs ? 3 : 1);
    const auto tiles = [&](uint32_t tile) { return (double)tiles_of(M, N, symmetric, tile); };
    switch (way) {
    case kFew: return 3.2 + tiles(32) * (1.3e-3 + (tiles(32) > 1024 ? 1.8e-6 : 2.5e-6) * 8.0 * K * (pairs ? 2 : 1));
    case kShared: return symmetric && tiles(64) <= 256 ? 5.0 + 2.9e-3 * k : 1e30;
    case k64: return 5.0 + k * std::max(3.9e-3, 5.0e-3 * tiles(64) / 256);
    case k128: return tiles(128) <= 256 ? 6.0 + k * (7.4e-3 + 7.0e-3 * tiles(128) / 256) : 1e30;
    case kDense: return 6.0 + k * 15.0e-3 * std::max(1.0, tiles(128) / 256);
    default: return 8.0 + k * std::ceil(tiles(256) / 256) * (19.0e-3 + 17.0e-3 * std::min(1.0, tiles(256) / 256));
    }
}

Way way_of(uint32_t M, uint32_t N, uint32_t K, bool symmetric, bool pairs)
{
    Way best = kFew;
    for (int w = kFew + 1; w < kWays; ++w)
        if (time_of((Way)w, M, N, K, symmetric, pairs) < time_of(best, M, N, K, symmetric, pairs)) best = (Way)w;
    return best;
}

// Whether the steps' products may be made of the high planes alone.  What their rounding leaves grows in the steps behind it: an error along a singular value s by the step's slope there, one that turns its direction by
// p(s) / s, whichever is larger, and each step adds about s (3 (b s^2)^2 + 6 (c s^4)^2 + 2 (b s^2 + c s^4)^2)^(1/2) of its own; the square of that is carried from 128 values of s through all steps.  Values above 1/16 are fewer than
// 256, over which errors of the operands spread out: what is left among the few falls with their number's root, s / 16.  The usual triple has 8, 21, 32 and 52 in 3 to 6 steps.  By this arithmetic in 64 bits, some 200 sets of triples
// between 10 and 35, sides of 256 to 600, matrices of noise, of singular values all alike, and both, were off by no more than 1.04e-4 of this (3.5e-3 in all) times the length of as many ones; sets of 75 to 240, made to converge fast,
// by up to 6e-3.  A step that makes small singular values smaller leaves results that an error of that size would hide.
bool high_planes_do(const float *k, int32_t steps)
{
    constexpr int points = 128;
    constexpr float limit = 35.0f, ratio = 0.93003f; // 10^(-4 / 127)
    for (int s = 0; s < steps; ++s)
        if (std::fabs(k[3 * s]) < 1.0f) return false;
    float v[points], off[points] = {};
    v[0] = 1.0f;
    for (int i = 1; i < points; ++i) v[i] = v[i - 1] * ratio;
    for (int s = 0; s < steps; ++s)
        for (int i = 0; i < points; ++i) { // (side by side: 2 us in all)
            const float a = k[3 * s], t = v[i] * v[i], bt = k[3 * s + 1] * t, ct = k[3 * s + 2] * t * t, slope = a + 3.0f * bt + 5.0f * ct, turn = a + bt + ct;
            off[i] = std::max(slope * slope, turn * turn) * off[i] + t * (3.0f * bt * bt + 6.0f * ct * ct + 2.0f * (bt + ct) * (bt + ct));
            v[i] *= turn;
        }
    float from = 1.0f;
    for (int i = 0; i < points; ++i, from *= ratio) {
        const float most = limit * std::max(1.0f, 16.0f * from);
        if (!(off[i] <= most * most)) return false;
    }
    return true;
}

struct StepPlan {
    bool tall, pairs, whole;
    uint32_t small, large; // the sides: X is [small, large]
    Way way_gram, way_square, way_step;
    bool turned; // X is held turned beside itself
    int64_t ld_X, ld_T, ld_A;
    uint32_t n_sums;
    size_t off_sums, off_X[2], off_T[2], off_A, off_B, total;
    int64_t plane_X, plane_T, plane_A; // elements
};

StepPlan plan_of(const Common &c, bool pairs)
{
    StepPlan t{};
    const auto take = [&](size_t bytes) {
        const size_t at = t.total;
        t.total = (t.total + bytes + 255) / 256 * 256;
        return at;
    };
    const auto up = [](int64_t n) { return (n + 7) / 8 * 8; };
    t.tall = c.rows > c.cols;
    t.small = (uint32_t)std::min(c.rows, c.cols), t.large = (uint32_t)std::max(c.rows, c.cols);
    t.pairs = pairs;
    t.whole = t.small <= kWholeSmall && t.large <= kWholeLarge;
    if (t.whole) {
        t.total = 256; // (a workspace of nothing would be refused by who asks for one)
        return t;
    }
    t.way_gram = way_of(t.small, t.small, t.large, true, t.pairs);
    t.way_square = way_of(t.small, t.small, t.small, true, t.pairs);
    t.way_step = way_of(t.small, t.large, t.small, false, t.pairs);
    t.turned = t.way_step != k256;
    t.ld_X = up(t.large), t.ld_T = t.ld_A = up(t.small);
    t.plane_X = t.small * t.ld_X, t.plane_T = t.large * t.ld_T, t.plane_A = t.small * t.ld_A;
    t.n_sums = (uint32_t)std::min<int64_t>(kNormBlocks, ((int64_t)c.rows * ((c.cols + 7) / 8) + 255) / 256);
    t.off_sums = take(t.n_sums * sizeof(double));
    for (int i = 0; i < 2; ++i) {
        t.off_X[i] = take((size_t)t.plane_X * 2 * sizeof(f16));
        if (t.turned) t.off_T[i] = take((size_t)t.plane_T * (t.pairs ? 2 : 1) * sizeof(f16));
    }
    t.off_A = take((size_t)t.plane_A * (t.pairs ? 2 : 1) * sizeof(f16));
    t.off_B = take((size_t)t.plane_A * (t.pairs ? 2 : 1) * sizeof(f16));
    return t;
}

bool may_be_single(const Common &c) { return c.type == ZG_BF16 && std::min(c.rows, c.cols) >= 256; }

StepPlan step_plan(const Common &c) { return plan_of(c, !may_be_single(c) || c.steps > 6 || !high_planes_do(c.coefficients, c.steps)); }

// goes by the matrix, not by the steps
size_t workspace_of(const Common &c)
{
    const size_t pairs = plan_of(c, true).total;
    return may_be_single(c) ? std::max(pairs, plan_of(c, false).total) : pairs;
}

template <int SEGMENTS, int KIND> int launch_step(hipStream_t st, Way way, const StepArgs<SEGMENTS, KIND> &p)
{
    const auto grid = [&](uint32_t tile) { return grid_of((tiles_of(p.M, p.N, KIND == kSquare, tile) + 7) / 8 * 8); };
    if (way == kFew) return launch(st, k_step_few<SEGMENTS, KIND>, grid_of(tiles_of(p.M, p.N, KIND == kSquare, 32)), 256, p);
    if constexpr (KIND == kSquare)
        if (way == kShared) return launch(st, k_step_shared<SEGMENTS>, grid(64), 512, p);
    if (way == k64) return launch(st, k_step_64<SEGMENTS, KIND>, grid(64), 256, p);
    if (way == k128) return launch(st, k_step_128<SEGMENTS, KIND>, grid(128), 256, p);
    if (way == kDense) return launch(st, k_step_dense<SEGMENTS, KIND>, grid(128), 256, p);
    return launch(st, k_step_256<SEGMENTS, KIND>, dim3(256), 512, p);
}

struct Result {
    void *O;
    int64_t ld;
    bool update;
    float keep, factor; // O = keep O + factor X, or factor X
};

template <int SEGMENTS> int run_steps(hipStream_t st, const Common &c, const StepPlan &t, char *ws, const Result &out)
{
    const auto at_ws = [&](size_t off) { return reinterpret_cast<f16 *>(ws + off); };
    f16 *const A = at_ws(t.off_A), *const B = at_ws(t.off_B);
    const bool pairs = SEGMENTS > 1;
    const auto up = [](uint32_t n) { return (n + 7) / 8 * 8; };
    const auto start = [&](auto &p, Operand a, int64_t plane_a, Operand b, int64_t plane_b, uint32_t M, uint32_t N, uint32_t K) {
        p.a = a, p.b = b, p.low_a = plane_a * (int64_t)sizeof(f16), p.low_b = plane_b * (int64_t)sizeof(f16);
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
        f16 *const X = at_ws(t.off_X[at]), *const X_next = at_ws(t.off_X[at ^ 1]);
        const Operand of_X{X, t.ld_X, false, true};
        {
            StepArgs<SEGMENTS, kSquare> p{}; // A = X X^T
            start(p, of_X, t.plane_X, of_X, t.plane_X, t.small, t.small, t.large);
            p.alpha = std::ldexp(1.0f, ea - 2 * ex);
            p.H = p.TH = A, p.L = p.TL = pairs ? A + t.plane_A : nullptr, p.ld_H = p.ld_T = t.ld_A;
            ZG_TRY(launch_step(st, t.way_gram, p));
        }
        {
            StepArgs<SEGMENTS, kSquare> p{}; // B = b A + c A^2
            start(p, of_A, t.plane_A, of_A, t.plane_A, t.small, t.small, t.small);
            p.alpha = std::ldexp(k[2], eb - 2 * ea), p.beta = std::ldexp(k[1], eb - ea);
            p.R = A, p.R_low = pairs ? A + t.plane_A : nullptr, p.ld_R = t.ld_A;
            p.H = p.TH = B, p.L = p.TL = pairs ? B + t.plane_A : nullptr, p.ld_H = p.ld_T = t.ld_A;
            ZG_TRY(launch_step(st, t.way_square, p));
        }
        const auto next_X = [&](auto &p, double factor, int exponent) { // a X + B X
            if (t.turned) {
                start(p, of_B, t.plane_A, Operand{at_ws(t.off_T[at]), t.ld_T, false, true}, t.plane_T, t.small, t.large, t.small);
            } else {
                start(p, of_B, t.plane_A, Operand{X, t.ld_X, true, true}, t.plane_X, t.small, t.large, t.small);
                p.b_short = p.K - t.small;
            }
            p.alpha = (float)std::ldexp(factor, exponent - eb - ex), p.beta = (float)std::ldexp(factor * k[0], exponent - ex);
            p.R = X, p.R_low = X + t.plane_X, p.ld_R = t.ld_X;
        };
        if (s + 1 < c.steps) {
            StepArgs<SEGMENTS, kStep> p{};
            next_X(p, 1.0, en);
            p.H = X_next, p.L = X_next + t.plane_X, p.ld_H = t.ld_X;
            if (t.turned) p.TH = at_ws(t.off_T[at ^ 1]), p.TL = pairs ? p.TH + t.plane_T : nullptr, p.ld_T = t.ld_T;
            ZG_TRY(launch_step(st, t.way_step, p));
        } else {
            StepArgs<SEGMENTS, kResult> p{};
            next_X(p, out.factor, 0);
            p.O = out.O, p.ld_O = out.ld, p.type_O = c.type, p.update = out.update, p.keep = out.keep, p.turn = t.tall;
            ZG_TRY(launch_step(st, t.way_step, p));
        }
        top = next.x, ex = en;
    }
    return ZG_OK;
}

int run_whole(hipStream_t st, const Common &c, const StepPlan &t, const StartArgs &a, const Result &out)
{
    WholeArgs w{};
    w.s = a;
    w.inv = ((uint64_t(1) << 32) + c.cols - 1) / c.cols;
    w.tall = t.tall, w.steps = c.steps;
    double top = 1.0;
    int ex = exponent_for(top);
    for (int s = 0; s < c.steps; ++s) {
        const float *const k = c.coefficients + 3 * s;
        const Bounds next = bounds_of(top, k);
        const bool last = s + 1 == c.steps;
        const double factor = last ? (double)out.factor : 1.0;
        const int ea = exponent_for(top * top), eb = exponent_for(next.b), en = last ? 0 : exponent_for(next.x);
        w.scalars[s][0] = std::ldexp(1.0f, ea - 2 * ex);
        w.scalars[s][1] = std::ldexp(k[2], eb - 2 * ea), w.scalars[s][3] = std::ldexp(k[1], eb - ea);
        w.scalars[s][2] = (float)std::ldexp(factor, en - eb - ex), w.scalars[s][4] = (float)std::ldexp(factor * k[0], en - ex);
        top = next.x, ex = en;
    }
    w.O = out.O, w.ld_O = out.ld, w.type_O = c.type, w.update = out.update, w.keep = out.keep;
    if (c.dtype == ZG_F32) return launch(st, k_step_whole<float>, dim3(1), 512, w);
    if (c.dtype == ZG_F16) return launch(st, k_step_whole<f16>, dim3(1), 512, w);
    return launch(st, k_step_whole<__bf16>, dim3(1), 512, w);
}

int run(hipStream_t st, const Common &c, StartArgs a, char *ws, const Result &out)
{
    const StepPlan t = step_plan(c);
    a.rows = (uint32_t)c.rows, a.cols = (uint32_t)c.cols;
    a.eps = c.eps;
    a.power = std::ldexp(1.0f, exponent_for(1.0));
    if (t.whole) return run_whole(st, c, t, a, out);
    a.sums = reinterpret_cast<double *>(ws + t.off_sums), a.n_sums = t.n_sums;
    f16 *const X = reinterpret_cast<f16 *>(ws + t.off_X[0]), *const T = t.turned ? reinterpret_cast<f16 *>(ws + t.off_T[0]) : nullptr;
    f16 *const X_low = X + t.plane_X, *const T_low = t.turned && t.pairs ? T + t.plane_T : nullptr;
    a.P = t.tall ? T : X, a.P_low = t.tall ? T_low : X_low, a.ld_P = t.tall ? t.ld_T : t.ld_X;
    a.Q = t.tall ? X : T, a.Q_low = t.tall ? X_low : T_low, a.ld_Q = t.tall ? t.ld_X : t.ld_T;
    const dim3 planes = grid_of((uint64_t)((c.rows + 63) / 64) * ((c.cols + 63) / 64));
    const auto begin = [&](auto zero) -> int {
        using T_ = decltype(zero);
        ZG_TRY(launch(st, k_start_norm<T_>, dim3(t.n_sums), 256, a));
        return launch(st, k_start_planes<T_>, planes, 256, a);
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
        *bytes = workspace_of(c);
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
        ZG_TRY(check_workspace(d_workspace, workspace_bytes, workspace_of(c)));
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
        *bytes = workspace_of(c);
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
        ZG_TRY(check_workspace(d_workspace, workspace_bytes, workspace_of(c)));
        StartArgs s{};
        s.g = a->d_G, s.ld_g = a->ld_G, s.m = a->d_M, s.ld_m = a->ld_M, s.momentum = a->momentum, s.nesterov = a->nesterov != 0;
        const float keep = (float)(1.0 - (double)a->lr * (double)a->decay), factor = (float)(-(double)a->lr * (double)a->scale);
        return run(static_cast<hipStream_t>(stream), c, s, static_cast<char *>(d_workspace), {a->d_W, a->ld_W, true, keep, factor});
    });
}

} // extern "C"
