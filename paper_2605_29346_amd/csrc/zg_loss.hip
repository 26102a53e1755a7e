// Softmax cross entropy of a linear layer: the loss over many classes without keeping the logits, and its gradients.
//
// z = A W^T + bias.  The product's tiles keep, of every row of their cells, the largest z and the sum of exp(z - largest) - 8 bytes for 32 or 64 logits -, which a
// second launch joins to lse = log sum exp z.  The gradients make the logits again, a piece of the classes (and of the rows, where there are many) at a time: dZ = f (exp(z - lse) - [class is the label]) leaves the
// product's tiles in the operands' type, f being the row's weight, and goes into the products dW = dZ^T A and dA += dZ W; what all rows have in common (1 / the sum of weights, and what the
// loss' own gradient is) is applied behind the sums.
#include "zg_product.h"

namespace zg {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// what a row counts: its label's class, or kNone
constexpr uint32_t kNone = 0xFFFFFFFFu;

struct Labels {
    const void *p;
    int32_t wide; // int64
    uint32_t classes;
    __device__ __forceinline__ uint32_t of(uint64_t m) const
    {
        const int64_t l = wide ? static_cast<const int64_t *>(p)[m] : static_cast<const int32_t *>(p)[m];
        return l >= 0 && l < (int64_t)classes ? (uint32_t)l : kNone;
    }
};

// ---- the forward product ----------------------------------------------------------------------------------------------------------

struct Top {
    float top, sum; // the largest of some logits of a row, and the sum of exp(z - top)
};

__device__ __forceinline__ float power_of(float v, float top) { return __builtin_amdgcn_exp2f((v - top) * kLog2e); }

// What exponentials are made below: the top, or 0 where that is infinite.  The sum of a row with a +infinity is +infinity then, that of nothing but -infinity 0, and one with a not-a-number stays that.
__device__ __forceinline__ float base_of(float top) { return fabsf(top) == INFINITY ? 0.0f : top; }

// Up to here z log2 e is far inside fp32; beyond, exp(z - top) is made from the difference.
constexpr float kPlainTop = 1e30f;

__device__ __forceinline__ Top join(Top a, Top b)
{
    const float top = fmaxf(a.top, b.top), base = base_of(top);
    return {top, a.sum * power_of(a.top, base) + b.sum * power_of(b.top, base)};
}

struct TopArgs : ProductArgs {
    static constexpr int high = 8;
    Labels labels;
    Top *part;       // [slot][M], a slot being the columns of a wavefront (or of k_loss_top_few's workgroup)
    float *at_label; // [M]: the label's logit
};

// A wavefront's 32 FM x 32 FN cells: half a row's lie side by side in a lane, the other half in the lane 32 further on, so that the row's largest and its sum need one exchange each.
// For each cell the bias, half of a maximum of three, a multiplication and addition in one, an exponential (four times as long) and an addition; the label's cell is looked for only where one of the
// wavefront's 32 rows has it among its columns.
template <int FM, int FN> __device__ __forceinline__ void tops(const TopArgs &p, const f32x16 (&acc)[FM][FN], uint32_t m_wave, uint32_t n_wave, uint32_t M)
{
    const uint32_t lane = threadIdx.x & 63, half = lane >> 5;
    if (n_wave >= p.N) return;
    const bool whole = n_wave + 32 * FN <= p.N;
    float bias[FN][16];
    if (p.e.bias) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t n = n_wave + 32 * j + 8 * q + 4 * half;
                if (whole) {
                    __builtin_memcpy(&bias[j][4 * q], p.e.bias + n, 16);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) bias[j][4 * q + r] = n + r < p.N ? p.e.bias[n + r] : 0.0f;
                }
            }
    }
    Top *const part = p.part + (uint64_t)(n_wave / (32 * FN)) * p.M;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const uint32_t m = m_wave + 32 * i + (lane & 31);
        const uint32_t at = m < M ? p.labels.of(m) - n_wave : kNone; // (kNone - n_wave is beyond the columns, too: classes < 2^25)
        float v[FN][16], top = -INFINITY;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) v[j][r] = acc[i][j][r];
        if (p.e.bias) {
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) v[j][r] += bias[j][r];
        }
        if (!whole) {
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (n_wave + 32 * j + 8 * (r / 4) + 4 * half + r % 4 >= p.N) v[j][r] = -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, v[j][r]);
        top = fmaxf(top, __shfl_xor(top, 32));
        const float base = base_of(top), base2 = base * kLog2e;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f(fmaf(v[j][r], kLog2e, -base2));
        const bool far = fabsf(base) > kPlainTop;
        if (__any(at < 32 * FN || far)) { // what is rare
            float z = 0.0f, below = 0.0f;
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    z = at == 32 * j + 8 * (r / 4) + 4 * half + r % 4 ? v[j][r] : z;
                    below += power_of(v[j][r], base);
                }
            if (at < 32 * FN && (at >> 2 & 1) == half) p.at_label[m] = z;
            sum = far ? below : sum;
        }
        sum += __shfl_xor(sum, 32);
        // base2's rounding, that of a logit of base's size, is a factor of all terms; and one of them is 1
        if (!far) sum *= __builtin_amdgcn_exp2f(fmaf(-base, kLog2e, base2));
        if (fabsf(top) < INFINITY) sum = __builtin_elementwise_maximum(sum, 1.0f);
        if (half == 0 && m < M) part[m] = Top{top, sum};
    }
}

template <> struct Out<TopArgs> {
    static constexpr bool turns = false;
    template <class O, bool PLAIN, int FM> __device__ __forceinline__ static void wide(const TopArgs &p, f32x16 (&acc)[FM][2], f32x4 *, uint32_t m_wave, uint32_t n_wave, uint32_t M, uint32_t)
    {
        tops(p, acc, m_wave, n_wave, M);
    }
    template <class O, bool PLAIN, int FM, int FN> __device__ __forceinline__ static void narrow(const TopArgs &p, f32x16 (&acc)[FM][FN], f32x4 *, uint32_t m_wave, uint32_t n_wave, uint32_t M, uint32_t)
    {
        tops(p, acc, m_wave, n_wave, M);
    }
    struct Few {
        Columns c;
        uint32_t label;
        __device__ __forceinline__ void begin(const TopArgs &p, uint32_t m, uint32_t n, uint32_t live)
        {
            c = columns_of(p.e, n, p.N);
            label = m < live ? p.labels.of(m) : kNone;
        }
        template <class F> __device__ __forceinline__ void end(const TopArgs &p, uint32_t m, uint32_t live, F &&sums)
        {
            float v[8];
            sums(0, v);
            Top t{-INFINITY, 0.0f};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = j < c.left ? v[j] + c.bias[j] : -INFINITY;
                t.top = fmaxf(t.top, v[j]);
            }
            t.top = fmaxf(t.top, __shfl_xor(t.top, 1));
            t.top = fmaxf(t.top, __shfl_xor(t.top, 2));
            const float base = base_of(t.top);
#pragma unroll
            for (int j = 0; j < 8; ++j) t.sum += power_of(v[j], base);
            t.sum += __shfl_xor(t.sum, 1);
            t.sum += __shfl_xor(t.sum, 2);
            if (m >= live) return;
            if ((threadIdx.x & 3) == 0) p.part[(uint64_t)(c.n / 32) * p.M + m] = t;
            const uint32_t at = label - c.n;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (at == (uint32_t)j) p.at_label[m] = v[j];
        }
    };
};

// (bf16 16384 x 1024 x 131072 3610 us, 1220 TFLOP/s, matrix instructions at work 0.63 of the time; 4096 x 256 x 250000 665 us, 790, 0.36: a tile is eight steps there, and its ways in and out are as long; fp32 98765 x 256 x 47 41 us in
// tiles of 64 x 64, 46 in tiles of 128 x 64, 77 of 128 x 128.)
template <class T> __global__ __launch_bounds__(256) void k_loss_top_few(TopArgs p) { few_tile<T>(p); }
template <class T> __global__ __launch_bounds__(256, 2) void k_loss_top_anyhow(TopArgs p) { product_tile<T, 64, 64, false, false>(p); }
template <class T> __global__ __launch_bounds__(256, 2) void k_loss_top_chunks(TopArgs p) { chunks_tile<T, T, 256, 128, false, false>(p); }
template <> __global__ __launch_bounds__(256, 3) void k_loss_top_chunks<float>(TopArgs p) { chunks_tile<float, float, 128, 128, false, false>(p); }
template <class T> __global__ __launch_bounds__(512, 2) void k_loss_top_long(TopArgs p) { long_tiles<T, T, false, false>(p); }

template <class T> __global__ __launch_bounds__(256, 2) void k_loss_top_narrow(TopArgs p) { chunks_tile<T, T, 256, 64, false, false>(p); }
template <> __global__ __launch_bounds__(256, 4) void k_loss_top_narrow<float>(TopArgs p) { chunks_tile<float, float, 64, 64, false, false, 8, 2>(p); }

// A chunk's products, summed in fp32.
template <class T> __device__ __forceinline__ float dot_chunk(u32x4 a, u32x4 b, float sum)
{
    constexpr int K = chunk_k<T>;
    T x[K], y[K];
    __builtin_memcpy(x, &a, 16);
    __builtin_memcpy(y, &b, 16);
#pragma unroll
    for (int k = 0; k < K; ++k) sum = fmaf((float)x[k], (float)y[k], sum);
    return sum;
}

// Up to R rows against all classes, operands in whole chunks, A's rows in LDS: a wavefront has 32 classes, 16 at a time, two to eight lanes, which read lines of 128 bytes of their rows.  Bound by
// memory, which W passes once: 1 x 1024 x 50021 bf16, 102 MB, 21 us, 4.9 TB/s (in tiles of 256 x 128 31, a wavefront to a class 44).
template <class T, int R> __global__ __launch_bounds__(256) void k_loss_top_rows(TopArgs p)
{
    constexpr int K = chunk_k<T>, ahead = R == 1 ? 8 : 4;
    extern __shared__ u32x4 rows[]; // [R][K / chunk_k]
    const uint32_t lane = threadIdx.x & 63, live = min(p.M, p.rows.live()), chunks = p.K / K;
    if (live == 0) return;
    for (uint32_t i = threadIdx.x; i < chunks * R; i += 256) rows[i] = *reinterpret_cast<const u32x4 *>(static_cast<const T *>(p.a.p) + min(i / chunks, live - 1) * p.a.ld + (i % chunks) * K);
    __syncthreads();
    const uint32_t slot = __builtin_amdgcn_readfirstlane(block_number() * 4 + (threadIdx.x >> 6)), n0 = slot * 32;
    if (n0 >= p.N) return;
    float z[R] = {};
#pragma unroll 1
    for (uint32_t c0 = 0; c0 < 32 && n0 + c0 < p.N; c0 += 16) {
        const T *w[2];
        float sum[2][R] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h) w[h] = static_cast<const T *>(p.b.p) + (uint64_t)min(n0 + c0 + 8 * h + (lane >> 3), p.N - 1) * p.b.ld;
        for (uint32_t q0 = lane & 7; q0 < chunks; q0 += 8 * ahead) {
            u32x4 x[ahead][2];
#pragma unroll
            for (int i = 0; i < ahead; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) x[i][h] = q0 + 8 * i < chunks ? *reinterpret_cast<const u32x4 *>(w[h] + (q0 + 8 * i) * K) : u32x4{};
#pragma unroll
            for (int i = 0; i < ahead; ++i)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const u32x4 a = rows[r * chunks + min(q0 + 8 * i, chunks - 1)];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float more = dot_chunk<T>(a, x[i][h], sum[h][r]);
                        sum[h][r] = q0 + 8 * i < chunks ? more : sum[h][r]; // (what A holds in another place may be no number)
                    }
                }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int d = 1; d < 8; d <<= 1) sum[h][r] += __shfl_xor(sum[h][r], d);
                const float there = __shfl(sum[h][r], (lane & 7) * 8); // class lane % 8's
                z[r] = (lane & 31) >> 3 == c0 / 8 + h ? there : z[r];
            }
    }
    const uint32_t n = n0 + (lane & 31);
    const bool there = lane < 32 && n < p.N;
    const float bias = p.e.bias && there ? p.e.bias[n] : 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if ((uint32_t)r >= live) break;
        z[r] = there ? z[r] + bias : -INFINITY;
        float top = z[r];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        float sum = power_of(z[r], base_of(top));
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
        if (lane == 0) p.part[(uint64_t)slot * p.M + r] = Top{top, sum};
        if (there && p.labels.of(r) == n) p.at_label[r] = z[r];
    }
}

// ---- the rows' losses -------------------------------------------------------------------------------------------------------------

struct RowArgs {
    Rows rows;
    uint32_t slots, cap;
    const Top *part;
    const float *at_label, *weight;
    Labels labels;
    float *lse, *row_loss; // row_loss may be null
    double *sums;          // [workgroups][2]: of weight x loss, of the weights
    float *loss, *total;   // total may be null
};

__device__ __forceinline__ void finish_loss(const RowArgs &a, double loss, double total)
{
    *a.loss = total != 0.0 ? (float)(loss / total) : 0.0f;
    if (a.total) *a.total = (float)total;
}

// R rows at a time, G lanes to a row, four of its slots at a time.  Reads what the product's tiles left, 8 bytes for 32 or 64 logits: 16384 x 2048 slots 58 us, 4.6 TB/s, 4096 x 3907 42 us.
template <int R, int G> __global__ __launch_bounds__(R * G) void k_loss_rows(RowArgs a)
{
    __shared__ Top lds[R * G];
    __shared__ double both[2][R];
    const uint32_t live = a.rows.live(), r = threadIdx.x % R, g = threadIdx.x / R;
    double loss = 0.0, total = 0.0;
    for (uint64_t m0 = (uint64_t)blockIdx.x * R; m0 < live; m0 += (uint64_t)gridDim.x * R) {
        const uint64_t m = m0 + r;
        Top t{-INFINITY, 0.0f};
        if (m < live)
            for (uint32_t s = g; s < a.slots; s += 4 * G) {
                Top u[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] = s + i * G < a.slots ? a.part[(uint64_t)(s + i * G) * a.cap + m] : Top{-INFINITY, 0.0f};
                const float top = fmaxf(fmaxf(fmaxf(u[0].top, u[1].top), fmaxf(u[2].top, u[3].top)), t.top), base = base_of(top);
                t.sum *= power_of(t.top, base);
#pragma unroll
                for (int i = 0; i < 4; ++i) t.sum += u[i].sum * power_of(u[i].top, base);
                t.top = top;
            }
        if (G > 1) {
            lds[threadIdx.x] = t;
            __syncthreads();
#pragma unroll
            for (int n = G / 2; n > 0; n >>= 1) {
                if (g < (uint32_t)n) lds[threadIdx.x] = t = join(t, lds[threadIdx.x + n * R]);
                __syncthreads();
            }
        }
        if (g == 0 && m < live) {
            const double lse = (double)t.top + log((double)t.sum);
            a.lse[m] = (float)lse;
            const bool has = a.labels.of(m) != kNone;
            const float w = !has ? 0.0f : a.weight ? a.weight[m] : 1.0f;
            const float each = has ? (float)(lse - (double)a.at_label[m]) : 0.0f;
            if (a.row_loss) a.row_loss[m] = each;
            if (w != 0.0f) {
                loss += (double)w * (double)each;
                total += (double)w;
            }
        }
    }
    if (g == 0) both[0][r] = loss, both[1][r] = total;
    __syncthreads();
#pragma unroll
    for (int n = R / 2; n > 0; n >>= 1) {
        if (threadIdx.x < (unsigned)n) both[0][r] += both[0][r + n], both[1][r] += both[1][r + n];
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        if (gridDim.x == 1) {
            finish_loss(a, both[0][0], both[1][0]);
        } else {
            a.sums[2 * blockIdx.x] = both[0][0];
            a.sums[2 * blockIdx.x + 1] = both[1][0];
        }
    }
}

// the shape of k_loss_rows: few parts to a row need a lane each; many of a few rows as many as a workgroup has
enum RowShape { kRowsOne, kRows8, kRows32, kRowsWide, kRowsAll };
constexpr int rows_of(RowShape s) { return s == kRowsOne ? 1 : s == kRows8 ? 8 : s == kRows32 ? 32 : s == kRowsWide ? 256 : 1024; }

RowShape row_shape(int64_t rows, uint32_t slots)
{
    if (slots <= 4) return rows <= 8192 ? kRowsAll : kRowsWide; // (one workgroup needs no second launch)
    if (rows <= 64) return kRowsOne;
    return rows < 16384 && slots >= 128 ? kRows8 : kRows32;
}

__global__ __launch_bounds__(64) void k_loss_mean(RowArgs a, uint32_t n)
{
    __shared__ double both[2][64];
    double loss = 0.0, total = 0.0;
    for (uint32_t i = threadIdx.x; i < n; i += 64) loss += a.sums[2 * i], total += a.sums[2 * i + 1];
    both[0][threadIdx.x] = loss, both[1][threadIdx.x] = total;
    __syncthreads();
    if (threadIdx.x) return;
    for (int i = 1; i < 64; ++i) loss += both[0][i], total += both[1][i];
    finish_loss(a, loss, total);
}

// ---- dZ ---------------------------------------------------------------------------------------------------------------------------

// what dZ's cells need of their row
struct RowFactor {
    float lse, factor; // factor 0: no gradient, whatever the logits are
    uint32_t label;
};

struct FactorArgs {
    Rows rows;
    const float *lse, *weight, *total, *dloss; // all but lse may be null
    Labels labels;
    const float *tops; // null, or the largest |weight| of each of kWeightBlocks workgroups
    float up;          // a power of two that dZ is held with, where tops is null
    float *power;      // what the products' sums are multiplied by
};

constexpr uint32_t kWeightBlocks = 64; // a wavefront's lanes

// the largest finite |weight| among the rows that count
__global__ __launch_bounds__(256) void k_loss_weight_top(FactorArgs a, float *tops)
{
    __shared__ float lds[256];
    float top = 0.0f;
    const uint32_t live = a.rows.live();
    for (uint64_t m = blockIdx.x * 256ull + threadIdx.x; m < live; m += 256ull * gridDim.x) {
        const float w = fabsf(a.weight[m]);
        if (a.labels.of(m) != kNone && w <= 3.402823466e38f) top = fmaxf(top, w);
    }
    lds[threadIdx.x] = top;
    __syncthreads();
    for (int n = 128; n > 0; n >>= 1) {
        if (threadIdx.x < (unsigned)n) lds[threadIdx.x] = fmaxf(lds[threadIdx.x], lds[threadIdx.x + n]);
        __syncthreads();
    }
    if (threadIdx.x == 0) tops[blockIdx.x] = lds[0];
}

// the power of two that dZ is held with: the largest |dZ| comes into [2^14, 2^15)
__device__ __forceinline__ float up_of(const FactorArgs &a)
{
    if (!a.tops) return a.up;
    float top = a.tops[threadIdx.x & 63];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    return ldexpf(1.0f, top > 0.0f ? min(15 - __builtin_amdgcn_frexp_expf(top), 126) : 0);
}

// by one lane of the first launch that makes dZ, whatever rows there are
__device__ __forceinline__ void put_power(const FactorArgs &a)
{
    if (block_number() != 0 || threadIdx.x >= 64) return;
    const float up = up_of(a), total = a.total ? *a.total : 1.0f;
    if (threadIdx.x == 0) *a.power = total != 0.0f ? (float)((a.dloss ? (double)*a.dloss : 1.0) / (double)total / (double)up) : 0.0f;
}

__device__ __forceinline__ RowFactor factor_of(const FactorArgs &a, uint32_t m, float up)
{
    RowFactor f{a.lse[m], 0.0f, a.labels.of(m)};
    const float w = a.weight ? a.weight[m] : 1.0f;
    if (f.label != kNone && w != 0.0f) f.factor = w * up;
    return f;
}

template <class T> struct DzArgs : ProductArgs {
    static constexpr int high = 8;
    // N = the piece's classes; Y: [M, N rounded up to eight]
    FactorArgs f;
    uint32_t first;   // the piece's first class
    float *bias_part; // null, or [groups of rows][ld_part]: the sums of dZ over a wavefront's rows
    int64_t ld_part;
};

// A probability.  Logits of millions are off by ones, and here they may be added up in another order than for lse: exp(Z - lse) could be any number, and an fp16 dZ infinite.  Not-a-number stays that.
__device__ __forceinline__ float at_most_one(float p) { return __builtin_elementwise_minimum(p, 1.0f); }

// Eight cells of a row; what is beyond the last class is 0.  Mostly a cell takes the bias, a multiplication and addition in one, an exponential, a minimum and the factor; what else there may be, in any row of the
// wavefront, is looked after in a branch of its own.
__device__ __forceinline__ void dz8(const Columns &c, const RowFactor &f, uint32_t first, bool bias, float (&v)[8])
{
    const uint32_t at = f.label - first - c.n;
    if (bias) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += c.bias[j];
    }
    if (__any(at < 8 || f.factor == 0.0f || c.left < 8 || !(fabsf(f.lse) < kPlainTop))) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = f.factor * at_most_one(power_of(v[j], f.lse));
            v[j] -= at == (uint32_t)j ? f.factor : 0.0f;
            v[j] = f.factor != 0.0f && j < c.left ? v[j] : 0.0f;
        }
    } else {
        const float base2 = f.lse * kLog2e; // (its rounding is that of a logit of lse's size)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = f.factor * at_most_one(__builtin_amdgcn_exp2f(fmaf(v[j], kLog2e, -base2)));
    }
}

// dZ is rounded to the operands' type here, once: dW and dA are products of that type's matrix instructions (fp32's have an eighth of the rate), and half the bytes go out and come back.  Off 64 bits that makes bf16 gradients
// 1.84e-3 instead of the 1.66e-3 of their own rounding, fp16 ones 3.0e-4 instead of 2.1e-4.
// The hand-over through LDS of 4 KB, as for other products' cells: 32 x 32 cells at a time, four lanes have 32 columns of a row.  bf16 16384 x 1024 x 16384 634 us, 867 TFLOP/s (the same product's statistics take 450): the way through LDS,
// and 10 vector instructions a cell.
template <class T, int FM, int FN> __device__ __forceinline__ void hand_over_dz(const DzArgs<T> &p, f32x16 (&acc)[FM][FN], f32x4 *mine, uint32_t m_wave, uint32_t n_wave, uint32_t M)
{
    const uint32_t lane = threadIdx.x & 63, half = lane >> 5, row = lane & 31, g = lane & 3;
    if (m_wave >= M) return;
    RowFactor f[FM][2]; // (all at once: a load between the stores would wait for them)
    {
        const float up = up_of(p.f);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u) f[i][u] = factor_of(p.f, min(m_wave + 32 * i + (lane >> 2) + 16 * u, M - 1), up);
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const Columns c = columns_of(p.e, n_wave + 32 * j + 8 * g, p.N);
        float sums[8] = {};
#pragma unroll
        for (int i = 0; i < FM; ++i) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                mine[row * 8 + ((2 * q + half) ^ ((row >> 1) & 7))] = f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            lds_exchange();
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t r = (lane >> 2) + 16 * u, m = m_wave + 32 * i + r;
                const f32x4 lo = mine[r * 8 + ((2 * g) ^ ((r >> 1) & 7))], hi = mine[r * 8 + ((2 * g + 1) ^ ((r >> 1) & 7))];
                float v[8];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = lo[k], v[4 + k] = hi[k];
                if (c.left <= 0 || m >= M) continue;
                dz8(c, f[i][u], p.first, p.e.bias, v);
#pragma unroll
                for (int k = 0; k < 8; ++k) sums[k] += v[k];
                store8(static_cast<T *>(p.e.Y) + m * p.e.ld_Y + c.n, 8, v, p.e.stream);
            }
            lds_exchange();
            __builtin_amdgcn_sched_barrier(0);
        }
        if (p.bias_part) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int d = 4; d < 64; d <<= 1) sums[k] += __shfl_xor(sums[k], d);
            if (lane < 4 && c.left > 0) store8(p.bias_part + m_wave / (32 * FM) * p.ld_part + c.n, 8, sums);
        }
    }
}

template <class T> struct Out<DzArgs<T>> {
    static constexpr bool turns = false;
    template <class O, bool PLAIN, int FM> __device__ __forceinline__ static void wide(const DzArgs<T> &p, f32x16 (&acc)[FM][2], f32x4 *mine, uint32_t m_wave, uint32_t n_wave, uint32_t M, uint32_t)
    {
        hand_over_dz(p, acc, mine, m_wave, n_wave, M);
    }
    template <class O, bool PLAIN, int FM, int FN> __device__ __forceinline__ static void narrow(const DzArgs<T> &p, f32x16 (&acc)[FM][FN], f32x4 *mine, uint32_t m_wave, uint32_t n_wave, uint32_t M, uint32_t)
    {
        hand_over_dz(p, acc, mine, m_wave, n_wave, M);
    }
    struct Few {
        Columns c;
        RowFactor f;
        __device__ __forceinline__ void begin(const DzArgs<T> &p, uint32_t m, uint32_t n, uint32_t live)
        {
            c = columns_of(p.e, n, p.N);
            f = factor_of(p.f, min(m, live - 1), up_of(p.f));
        }
        template <class F> __device__ __forceinline__ void end(const DzArgs<T> &p, uint32_t m, uint32_t live, F &&sums)
        {
            float v[8];
            sums(0, v);
            if (m >= live) f.factor = 0.0f;
            dz8(c, f, p.first, p.e.bias, v);
            if (m < live && c.left > 0) store8(static_cast<T *>(p.e.Y) + m * p.e.ld_Y + c.n, 8, v, p.e.stream);
            if (!p.bias_part) return;
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int d = 4; d < 64; d <<= 1) v[k] += __shfl_xor(v[k], d);
            if ((threadIdx.x & 63) < 4 && m < live && c.left > 0) store8(p.bias_part + m / 16 * p.ld_part + c.n, 8, v); // (m: the wavefront's first row, of the tile's second half there may be none)
        }
    };
};

template <class T> __global__ __launch_bounds__(256) void k_loss_dz_few(DzArgs<T> p) { put_power(p.f); few_tile<T>(p); }
template <class T> __global__ __launch_bounds__(256, 2) void k_loss_dz_anyhow(DzArgs<T> p) { put_power(p.f); product_tile<T, 64, 64, false, false>(p); }
template <class T> __global__ __launch_bounds__(256, 2) void k_loss_dz_chunks(DzArgs<T> p) { put_power(p.f); chunks_tile<T, T, 256, 128, false, false>(p); }
template <> __global__ __launch_bounds__(256, 3) void k_loss_dz_chunks<float>(DzArgs<float> p) { put_power(p.f); chunks_tile<float, float, 128, 128, false, false>(p); }
template <class T> __global__ __launch_bounds__(512, 2) void k_loss_dz_long(DzArgs<T> p) { put_power(p.f); long_tiles<T, T, false, false>(p); }

__global__ __launch_bounds__(64) void k_loss_power(FactorArgs f) { put_power(f); } // (without rows, nobody makes dZ)

template <class T> __global__ __launch_bounds__(256, 2) void k_loss_dz_narrow(DzArgs<T> p) { put_power(p.f); chunks_tile<T, T, 256, 64, false, false>(p); }
template <> __global__ __launch_bounds__(256, 4) void k_loss_dz_narrow<float>(DzArgs<float> p) { put_power(p.f); chunks_tile<float, float, 64, 64, false, false, 8, 2>(p); }

// Parts of dW's sum over the rows for few classes, fp32: 98765 x 47 x 256 35 us, in dense_product's tiles of 128 x 128 61.
__global__ __launch_bounds__(256, 4) void k_loss_part_narrow(ProductArgs p) { chunks_tile<float, float, 64, 128, true, true>(p); }

// Parts of dA's sum over the classes (bf16 16384 x 16384 x 1024 540 us, 1020 TFLOP/s), in fp32: those of one piece, where the tiles of [rows, in] alone would leave compute units idle, and those of the pieces.
template <class T> __global__ __launch_bounds__(256, 2) void k_loss_part_anyhow(ProductArgs p) { product_tile<T, 64, 64, false, true>(p); } // (or of dA itself where that is small)
template <class T> __global__ __launch_bounds__(256, 2) void k_loss_part_chunks(ProductArgs p) { chunks_tile<T, float, 256, 128, false, true>(p); }
template <> __global__ __launch_bounds__(256, 3) void k_loss_part_chunks<float>(ProductArgs p) { chunks_tile<float, float, 128, 128, false, true>(p); }
template <class T> __global__ __launch_bounds__(512, 2) void k_loss_part_long(ProductArgs p) { long_tiles<T, float, false, true>(p); }

// dbias = power x the sum over the groups of rows: C classes to a workgroup, 1024 / C groups side by side, then in order.  `more`: these rows are not the first.
template <int C> __global__ __launch_bounds__(1024) void k_loss_bias(Rows rows, uint32_t group, uint32_t N, const float *part, int64_t ld_part, const float *power, float *out, bool more)
{
    constexpr int G = 1024 / C;
    __shared__ float lds[G][C];
    const uint32_t c = threadIdx.x % C, n = blockIdx.x * C + c, g = threadIdx.x / C, groups = (rows.live() + group - 1) / group;
    float sum = 0.0f;
    if (n < N) {
#pragma unroll 4
        for (uint32_t i = g; i < groups; i += G) sum += part[i * ld_part + n];
    }
    lds[g][c] = sum;
    __syncthreads();
    for (int k = G / 2; k > 0; k >>= 1) {
        if (g < (uint32_t)k) lds[g][c] += lds[g + k][c];
        __syncthreads();
    }
    if (g == 0 && n < N) out[n] = fmaf(lds[0][c], *power, more ? out[n] : 0.0f);
}

// how many rows of each piece of `step` rows there are
__global__ __launch_bounds__(256) void k_row_counts(Rows rows, uint32_t step, uint32_t pieces, uint32_t *counts)
{
    const uint64_t i = (uint64_t)block_number() * 256 + threadIdx.x, first = i * step, live = rows.live();
    if (i < pieces) counts[i] = (uint32_t)(first < live ? min(live - first, (uint64_t)step) : 0);
}

// ---- operands that lie anyhow -----------------------------------------------------------------------------------------------------

// A copy whose rows are whole chunks, zeros behind the columns; `groups` of eight columns to a row.
template <class T> __global__ __launch_bounds__(256) void k_loss_pack(const T *from, int64_t ld_from, Rows rows, uint32_t cols, T *to, uint32_t groups)
{
    const uint64_t i = (uint64_t)block_number() * 256 + threadIdx.x, r = i / groups;
    const uint32_t g = (uint32_t)(i - r * groups);
    if (r >= rows.live()) return;
    float v[8];
    load8(from + r * ld_from + 8 * g, (int)cols - 8 * (int)g, v);
    store8(to + (r * groups + g) * 8, 8, v);
}

// ---- host side --------------------------------------------------------------------------------------------------------------------

enum Kind { kFew, kAnyhow, kChunks, kLong, kNarrow, kRow };

constexpr uint32_t kRowBytes = 16 << 10; // of a row of A, up to four of which k_loss_top_rows has in LDS

// which kernel makes the logits of [M, N], K terms each
template <class T> Kind kind_of(const ProductArgs &p, bool tops)
{
    const bool chunks = in_chunks<T>(p.a, p.M, p.K) && in_chunks<T>(p.b, p.N, p.K);
    if (tops && chunks && p.M <= 4 && p.K * sizeof(T) <= kRowBytes) return kRow;
    if (few_tiles<T>(p, chunks)) return kFew;
    if (!chunks) return kAnyhow;
    if (p.N <= 64) return kNarrow;
    if (sizeof(T) == 4) return kChunks;
    return tile_blocks<256, 256>(p) >= 256 && p.K * sizeof(T) >= 2048 ? kLong : kChunks;
}

constexpr uint32_t slot_width(Kind k) { return k == kChunks || k == kLong ? 64 : 32; } // columns of a Top
constexpr uint32_t group_rows(Kind k, bool f32) { return k == kFew ? 16 : k == kAnyhow || (k == kNarrow && f32) ? 32 : f32 ? 64 : 128; } // rows of a sum for dbias

// Of dZ.  More has it go through memory twice, less makes dA of more parts: 16384 x 1024 x 65536 bf16, all gradients, with 2^27 .. 2^31 bytes 7.5, 7.2, 6.9, 7.0, 7.0 ms.
constexpr int64_t kPieceBytes = int64_t(1) << 29;
constexpr int64_t kPartBytes = int64_t(1) << 30;  // of parts of dA that wait for their join, if more than it takes at least
constexpr int64_t kShareBytes = int64_t(7) << 28; // a workspace that is always fine: the two above and parts of dW and dbias
// Classes to a part of dA's sum, at least: few rows and columns are few tiles, and a part's steps come one behind the other.  The parts' kernel with 1024 / 256 / 128 / 64: f32 1 x 638 x 9054 97 / 32 / 23 / 18 us,
// 771 x 34 x 2012 132 / 23 / 15 / 13, 300 x 256 x 5000 88 / 24 / 18 / 20, bf16 2000 x 64 x 10000 35 / 19 / 19 / 19, 300 x 256 x 5000 39 / 14 / 12 / 16; the join takes 1 to 4 us more with 64 parts than with 8.
constexpr int64_t kPartTerms = 128;
constexpr double kPackFlops = 2e9;                // products from here on are worth a copy of operands that lie anyhow

struct Shape {
    int64_t rows;
    int32_t in, out, dtype;
    const void *A, *W;
    int64_t ld_A, ld_W;
};

// the operands, or where their copies will be
struct Packed {
    bool copy_A = false, copy_W = false;
    uint32_t K = 0; // terms, zeros behind `in` among them
    Operand a, w;
};

template <class Take> Packed packed_plan(const Shape &s, Take &&take, size_t (&off)[2])
{
    Packed r;
    r.K = (uint32_t)s.in;
    r.a = {s.A, s.ld_A, false, false};
    r.w = {s.W, s.ld_W, false, false};
    const auto fits = [&](const Operand &o, int64_t rows) {
        if (s.dtype == ZG_F32) return in_chunks<float>(o, (uint32_t)rows, (uint32_t)s.in);
        return in_chunks<_Float16>(o, (uint32_t)rows, (uint32_t)s.in);
    };
    const bool A = fits(r.a, s.rows), W = fits(r.w, s.out);
    if ((A && W) || 2.0 * s.rows * s.out * s.in < kPackFlops) return r;
    const int64_t ld = (s.in + 7) / 8 * 8;
    if (s.in * type_size(s.dtype) % 16) r.K = (uint32_t)ld; // (else one of the two may be read where it lies)
    if (!A) r.copy_A = true, off[0] = take((size_t)s.rows * ld * type_size(s.dtype)), r.a = {nullptr, ld, false, true};
    if (!W) r.copy_W = true, off[1] = take((size_t)s.out * ld * type_size(s.dtype)), r.w = {nullptr, ld, false, true};
    return r;
}

template <class F> int with_wide_type(int32_t type, F &&f)
{
    if (type == ZG_F32) return f(float());
    if (type == ZG_F16) return f((_Float16)0);
    return f((__bf16)0);
}

int launch_pack(hipStream_t st, int32_t dtype, const void *from, int64_t ld, Rows rows, int32_t cols, void *to)
{
    const uint32_t groups = ((uint32_t)cols + 7) / 8;
    return with_wide_type(dtype, [&](auto t) {
        using T = decltype(t);
        return launch(st, k_loss_pack<T>, grid_of(((uint64_t)rows.cap * groups + 255) / 256), 256, static_cast<const T *>(from), ld, rows, (uint32_t)cols, static_cast<T *>(to), groups);
    });
}

// [rows, in] x [out, in]: the logits' product
ProductArgs logits_product(const Shape &s, const Packed &pk, const uint32_t *d_rows)
{
    ProductArgs p{};
    p.a = pk.a, p.b = pk.w;
    p.M = (uint32_t)s.rows, p.N = (uint32_t)s.out, p.K = pk.K;
    p.rows = {d_rows, p.M};
    p.splits = 1;
    p.e.factor = 1.0f;
    return p;
}

// Addresses only matter for their alignment here: copies' are null.
Kind logits_kind(int32_t dtype, const ProductArgs &p, bool tops) { return (Kind)with_wide_type(dtype, [&](auto t) { return (int)kind_of<decltype(t)>(p, tops); }); }

struct TopPlan {
    Packed pk;
    Kind kind;
    uint32_t slots, row_grid;
    RowShape shape;
    size_t off_pack[2], off_part, off_at, off_sums, total;
};

struct Taker {
    size_t &total;
    size_t operator()(size_t bytes) const
    {
        const size_t at = total;
        total = (total + bytes + 255) / 256 * 256;
        return at;
    }
};

TopPlan top_plan(const Shape &s)
{
    TopPlan t{};
    const Taker take{t.total};
    t.pk = packed_plan(s, take, t.off_pack);
    t.kind = logits_kind(s.dtype, logits_product(s, t.pk, nullptr), true);
    t.slots = ((uint32_t)s.out + slot_width(t.kind) - 1) / slot_width(t.kind);
    t.off_part = take((size_t)t.slots * s.rows * sizeof(Top));
    t.off_at = take((size_t)s.rows * sizeof(float));
    t.shape = row_shape(s.rows, t.slots);
    t.row_grid = t.shape == kRowsAll ? 1 : (uint32_t)std::max<int64_t>(1, std::min<int64_t>(1024, (s.rows + rows_of(t.shape) - 1) / rows_of(t.shape)));
    t.off_sums = take((size_t)t.row_grid * 2 * sizeof(double));
    return t;
}

struct DzPlan {
    Packed pk;
    Kind kind;
    int64_t step, steps, piece, pieces, ld_dz; // rows and classes of a piece of dZ
    uint32_t splits_A, slots_A, splits_W;      // parts of a piece's sum for dA, parts that there is room for, parts of dW's
    size_t off_pack[2], off_power, off_tops, off_counts, off_dz, off_part_A, off_part_W, off_sum_W, off_bias, total;
};

struct Wanted {
    bool dA, dW, dbias, weight;
};

DzPlan dz_layout(const Shape &s, const Wanted &w, int64_t step, int64_t piece)
{
    DzPlan t{};
    const Taker take{t.total};
    const int64_t e = (int64_t)type_size(s.dtype), rows = std::max<int64_t>(1, step);
    Shape some = s;
    some.rows = step;
    t.pk = packed_plan(some, take, t.off_pack);
    t.step = step, t.steps = (std::max<int64_t>(1, s.rows) + rows - 1) / rows;
    t.piece = piece, t.pieces = (s.out + piece - 1) / piece;
    t.ld_dz = (piece + 7) / 8 * 8;
    some.out = (int32_t)piece;
    t.kind = logits_kind(s.dtype, logits_product(some, t.pk, nullptr), false);
    t.off_power = take(sizeof(float));
    if (w.weight) t.off_tops = take(kWeightBlocks * sizeof(float));
    if (t.steps > 1) t.off_counts = take((size_t)t.steps * sizeof(uint32_t));
    t.off_dz = take((size_t)step * t.ld_dz * e);
    const int64_t tiles_A = (rows + 255) / 256 * ((s.in + 127) / 128), tiles_W = (piece + 255) / 256 * ((s.in + 127) / 128);
    // Parts enough for two tiles of 256 x 128 to a compute unit; where tiles of 256 x 256, which would be taken from 256 of them on, were a third empty, fewer than that.
    const int64_t wide_A = (rows + 255) / 256 * ((s.in + 255) / 256), wide_W = (piece + 255) / 256 * ((s.in + 255) / 256);
    const bool narrow = s.dtype != ZG_F32 && (s.in + 255) / 256 * 256 * 3 >= (s.in + 127) / 128 * 128 * 4;
    t.splits_A = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(narrow ? std::min(512 / tiles_A, 255 / wide_A) : 512 / tiles_A, piece / kPartTerms));
    t.splits_W = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(narrow ? std::min(512 / tiles_W, 255 / wide_W) : 512 / tiles_W, (rows + 255) / 256));
    const int64_t parts = t.pieces * t.splits_A, room = kPartBytes / (rows * s.in * (int64_t)sizeof(float));
    t.slots_A = (uint32_t)(parts == 1 ? 0 : std::min(parts, t.splits_A + std::min<int64_t>(4, std::max<int64_t>(1, room - t.splits_A))));
    if (w.dA) t.off_part_A = take((size_t)t.slots_A * step * s.in * sizeof(float));
    if (w.dW && (t.splits_W > 1 || t.steps > 1)) t.off_part_W = take((size_t)t.splits_W * piece * s.in * sizeof(float));
    if (w.dW && t.steps > 1) t.off_sum_W = take((size_t)s.out * s.in * sizeof(float));
    const uint32_t group = group_rows(t.kind, s.dtype == ZG_F32);
    if (w.dbias) t.off_bias = take((size_t)((step + group - 1) / group) * t.ld_dz * sizeof(float));
    return t;
}

// Pieces of the classes, 4096 at least, of all rows; where dZ whole takes less than such a piece and the parts of dA that they leave, whole; and where neither is small, pieces of the rows too, the
// largest that are: then dW is a sum over those, in fp32.
DzPlan dz_plan(const Shape &s, const Wanted &w)
{
    const auto classes = [&](int64_t rows) {
        const int64_t most = kPieceBytes / (std::max<int64_t>(1, rows) * (int64_t)type_size(s.dtype)) / 256 * 256;
        return std::min<int64_t>(s.out, std::max<int64_t>(4096, most));
    };
    DzPlan best = dz_layout(s, w, s.rows, classes(s.rows));
    const auto better = [&](int64_t step, int64_t piece) {
        const DzPlan t = dz_layout(s, w, step, piece);
        if (t.total < best.total) best = t;
    };
    if (best.pieces > 1) better(s.rows, s.out);
    const int64_t whole = kPieceBytes / ((s.out + 7) / 8 * 8 * (int64_t)type_size(s.dtype)) / 256 * 256; // rows of all classes
    for (int64_t step = std::max<int64_t>(65536, whole); step >= 4096 && best.total > (size_t)kShareBytes; step = step > 65536 ? 65536 : step / 2)
        if (step < s.rows) better(step, classes(step));
    return best;
}

int check_labels(const char *what, const void *p, int32_t type)
{
    if (type != ZG_I32 && type != ZG_I64) return fail(ZG_EINVAL, "label_dtype is not ZG_I32 or ZG_I64");
    return reinterpret_cast<uintptr_t>(p) % (type == ZG_I64 ? 8 : 4) ? fail(ZG_EINVAL, std::string(what) + " is not aligned to its elements") : ZG_OK;
}

Span labels_span(const void *p, int64_t rows, int32_t type)
{
    Span s = vector_span("d_labels", p, rows);
    if (type == ZG_I64) s.pitch = s.width = rows * 8, s.size = 8;
    return s;
}

template <class A> int check_common(const A *a)
{
    if (!a) return fail(ZG_EINVAL, "null argument");
    ZG_TRY(check_rows(a->rows));
    ZG_TRY(check_width(a->in));
    ZG_TRY(check_width(a->out, ZG_MAX_CLASSES));
    if (!wide_type(a->dtype)) return fail(ZG_EINVAL, "dtype is not ZG_F32, ZG_F16 or ZG_BF16");
    ZG_TRY(check_labels("d_labels", a->d_labels, a->label_dtype));
    ZG_TRY(check_vector("d_rows", a->d_rows));
    ZG_TRY(check_vector("d_bias", a->d_bias));
    ZG_TRY(check_vector("d_weight", a->d_weight));
    if (a->rows > 0) {
        ZG_TRY(check_matrix("d_A", a->d_A, a->ld_A, a->in, a->dtype));
        ZG_TRY(check_matrix("d_W", a->d_W, a->ld_W, a->in, a->dtype));
        if (!a->d_labels) return fail(ZG_EINVAL, "d_labels is null");
    }
    return ZG_OK;
}

Wanted wanted_of(const zg_linear_cross_entropy_grad_args *a) { return {a->d_dA != nullptr, a->d_dW != nullptr, a->d_dbias != nullptr, a->d_weight != nullptr}; }

template <class A> Shape shape_of(const A *a) { return {a->rows, a->in, a->out, a->dtype, a->d_A, a->d_W, a->ld_A, a->ld_W}; }

// the copies of W, and of the rows of A from `first` on (`rows` of them)
template <class A> int pack_W(hipStream_t st, const A *a, char *ws, const size_t (&off)[2], Packed &pk)
{
    if (!pk.copy_W) return ZG_OK;
    pk.w.p = ws + off[1];
    return launch_pack(st, a->dtype, a->d_W, a->ld_W, Rows{nullptr, (uint32_t)a->out}, a->in, ws + off[1]);
}

template <class A> int pack_A(hipStream_t st, const A *a, char *ws, const size_t (&off)[2], Packed &pk, int64_t first, Rows rows)
{
    const char *const from = static_cast<const char *>(a->d_A) + first * a->ld_A * (int64_t)type_size(a->dtype);
    pk.a.p = pk.copy_A ? ws + off[0] : from;
    return pk.copy_A ? launch_pack(st, a->dtype, from, a->ld_A, rows, a->in, ws + off[0]) : ZG_OK;
}

template <class T> int launch_tops(hipStream_t st, Kind kind, const TopArgs &p)
{
    if (kind == kFew) return launch(st, k_loss_top_few<T>, grid_of((uint64_t)((p.M + 31) / 32) * ((p.N + 31) / 32)), 256, p);
    if (kind == kAnyhow) return launch(st, k_loss_top_anyhow<T>, tile_grid<64, 64>(p), 256, p);
    if (kind == kNarrow) return launch(st, k_loss_top_narrow<T>, sizeof(T) == 4 ? tile_grid<64, 64>(p) : tile_grid<256, 64>(p), 256, p);
    if (kind == kRow) {
        const dim3 grid = grid_of(((uint64_t)p.N + 127) / 128);
        const uint32_t row = p.K * sizeof(T);
        return p.M == 1 ? launch_lds(st, k_loss_top_rows<T, 1>, grid, 256, row, p) : launch_lds(st, k_loss_top_rows<T, 4>, grid, 256, 4 * row, p);
    }
    if constexpr (sizeof(T) == 4) {
        return launch(st, k_loss_top_chunks<T>, tile_grid<128, 128>(p), 256, p);
    } else {
        if (kind == kLong) return launch(st, k_loss_top_long<T>, dim3(256), 512, p);
        return launch(st, k_loss_top_chunks<T>, tile_grid<256, 128>(p), 256, p);
    }
}

template <class T> int launch_dz(hipStream_t st, Kind kind, const DzArgs<T> &p)
{
    if (kind == kFew) return launch(st, k_loss_dz_few<T>, grid_of((uint64_t)((p.M + 31) / 32) * ((p.N + 31) / 32)), 256, p);
    if (kind == kAnyhow) return launch(st, k_loss_dz_anyhow<T>, tile_grid<64, 64>(p), 256, p);
    if (kind == kNarrow) return launch(st, k_loss_dz_narrow<T>, sizeof(T) == 4 ? tile_grid<64, 64>(p) : tile_grid<256, 64>(p), 256, p);
    if constexpr (sizeof(T) == 4) {
        return launch(st, k_loss_dz_chunks<T>, tile_grid<128, 128>(p), 256, p);
    } else {
        if (kind == kLong) return launch(st, k_loss_dz_long<T>, dim3(256), 512, p);
        return launch(st, k_loss_dz_chunks<T>, tile_grid<256, 128>(p), 256, p);
    }
}

// splits parts of [M, N] in fp32, one behind the other from p.e.Y on
template <class T> int launch_parts(hipStream_t st, const ProductArgs &p, bool chunks)
{
    if (!chunks) return launch(st, k_loss_part_anyhow<T>, tile_grid<64, 64>(p), 256, p);
    if constexpr (sizeof(T) == 4) {
        return launch(st, k_loss_part_chunks<T>, tile_grid<128, 128>(p), 256, p);
    } else {
        if (tile_blocks<256, 256>(p) >= 256) return launch(st, k_loss_part_long<T>, dim3(256), 512, p);
        return launch(st, k_loss_part_chunks<T>, tile_grid<256, 128>(p), 256, p);
    }
}

} // namespace
} // namespace zg

using namespace zg;

extern "C" {
int zg_linear_cross_entropy_workspace(const zg_linear_cross_entropy_args *a, size_t *bytes)
{
    return entry([&]() -> int {
        ZG_TRY(check_common(a));
        if (!bytes) return fail(ZG_EINVAL, "null argument");
        *bytes = top_plan(shape_of(a)).total;
        return ZG_OK;
    });
}

int zg_linear_cross_entropy(const zg_linear_cross_entropy_args *a, void *d_workspace, size_t workspace_bytes, void *stream)
{
    return entry([&]() -> int {
        ZG_TRY(check_common(a));
        if (!a->d_loss) return fail(ZG_EINVAL, "d_loss is null");
        if (a->rows > 0 && !a->d_lse) return fail(ZG_EINVAL, "d_lse is null");
        for (const void *v : {(const void *)a->d_loss, (const void *)a->d_total, (const void *)a->d_lse, (const void *)a->d_row_loss}) ZG_TRY(check_vector("an output", v));
        {
            const Span A = matrix_span("d_A", a->d_A, a->rows, a->ld_A, a->in, a->dtype), W = matrix_span("d_W", a->d_W, a->rows ? a->out : 0, a->ld_W, a->in, a->dtype);
            const Span bias = vector_span("d_bias", a->d_bias, a->out), labels = labels_span(a->d_labels, a->rows, a->label_dtype), weight = vector_span("d_weight", a->d_weight, a->rows);
            const Span count = rows_span(a->d_rows), loss = vector_span("d_loss", a->d_loss, 1), total = vector_span("d_total", a->d_total, 1);
            const Span lse = vector_span("d_lse", a->d_lse, a->rows), each = vector_span("d_row_loss", a->d_row_loss, a->rows);
            ZG_TRY(check_apart(loss, {A, W, bias, labels, weight, count, total, lse, each}));
            ZG_TRY(check_apart(total, {A, W, bias, labels, weight, count, lse, each}));
            ZG_TRY(check_apart(lse, {A, W, bias, labels, weight, count, each}));
            ZG_TRY(check_apart(each, {A, W, bias, labels, weight, count}));
        }
        TopPlan t = top_plan(shape_of(a));
        ZG_TRY(check_workspace(d_workspace, workspace_bytes, t.total));
        const hipStream_t st = static_cast<hipStream_t>(stream);
        char *const ws = static_cast<char *>(d_workspace);
        const Labels labels{a->d_labels, a->label_dtype == ZG_I64, (uint32_t)a->out};
        Top *const part = reinterpret_cast<Top *>(ws + t.off_part);
        float *const at = reinterpret_cast<float *>(ws + t.off_at);
        if (a->rows > 0) {
            ZG_TRY(pack_W(st, a, ws, t.off_pack, t.pk));
            ZG_TRY(pack_A(st, a, ws, t.off_pack, t.pk, 0, Rows{a->d_rows, (uint32_t)a->rows}));
            TopArgs p{};
            static_cast<ProductArgs &>(p) = logits_product(shape_of(a), t.pk, a->d_rows);
            p.e.bias = a->d_bias;
            p.labels = labels, p.part = part, p.at_label = at;
            ZG_TRY(with_wide_type(a->dtype, [&](auto v) { return launch_tops<decltype(v)>(st, t.kind, p); }));
        }
        RowArgs r{};
        r.rows = {a->d_rows, (uint32_t)a->rows};
        r.slots = t.slots, r.cap = (uint32_t)a->rows, r.part = part, r.at_label = at, r.weight = a->d_weight, r.labels = labels;
        r.lse = a->d_lse, r.row_loss = a->d_row_loss, r.sums = reinterpret_cast<double *>(ws + t.off_sums), r.loss = a->d_loss, r.total = a->d_total;
        const dim3 grid(t.row_grid);
        switch (t.shape) {
        case kRowsOne: ZG_TRY(launch(st, k_loss_rows<1, 1024>, grid, 1024, r)); break;
        case kRows8: ZG_TRY(launch(st, k_loss_rows<8, 128>, grid, 1024, r)); break;
        case kRows32: ZG_TRY(launch(st, k_loss_rows<32, 32>, grid, 1024, r)); break;
        case kRowsWide: ZG_TRY(launch(st, k_loss_rows<256, 1>, grid, 256, r)); break;
        case kRowsAll: ZG_TRY(launch(st, k_loss_rows<1024, 1>, grid, 1024, r)); break;
        }
        return t.row_grid > 1 ? launch(st, k_loss_mean, dim3(1), 64, r, t.row_grid) : ZG_OK;
    });
}

int zg_linear_cross_entropy_backward_workspace(const zg_linear_cross_entropy_grad_args *a, size_t *bytes)
{
    return entry([&]() -> int {
        ZG_TRY(check_common(a));
        if (!bytes) return fail(ZG_EINVAL, "null argument");
        *bytes = dz_plan(shape_of(a), wanted_of(a)).total;
        return ZG_OK;
    });
}

int zg_linear_cross_entropy_backward(const zg_linear_cross_entropy_grad_args *a, void *d_workspace, size_t workspace_bytes, void *stream)
{
    return entry([&]() -> int {
        ZG_TRY(check_common(a));
        if (a->rows > 0 && !a->d_lse) return fail(ZG_EINVAL, "d_lse is null");
        for (const void *v : {(const void *)a->d_lse, (const void *)a->d_total, (const void *)a->d_dloss, (const void *)a->d_dbias}) ZG_TRY(check_vector("a vector", v));
        if (a->d_dA && a->rows > 0) ZG_TRY(check_matrix("d_dA", a->d_dA, a->ld_dA, a->in, a->dtype));
        if (a->d_dW) ZG_TRY(check_matrix("d_dW", a->d_dW, a->ld_dW, a->in, a->dtype));
        {
            const Span A = matrix_span("d_A", a->d_A, a->rows, a->ld_A, a->in, a->dtype), W = matrix_span("d_W", a->d_W, a->rows ? a->out : 0, a->ld_W, a->in, a->dtype);
            const Span bias = vector_span("d_bias", a->d_bias, a->out), labels = labels_span(a->d_labels, a->rows, a->label_dtype), weight = vector_span("d_weight", a->d_weight, a->rows);
            const Span count = rows_span(a->d_rows), lse = vector_span("d_lse", a->d_lse, a->rows), total = vector_span("d_total", a->d_total, 1), dloss = vector_span("d_dloss", a->d_dloss, 1);
            const Span dA = matrix_span("d_dA", a->d_dA, a->rows, a->ld_dA, a->in, a->dtype), dW = matrix_span("d_dW", a->d_dW, a->out, a->ld_dW, a->in, a->dtype);
            const Span dbias = vector_span("d_dbias", a->d_dbias, a->out);
            ZG_TRY(check_apart(dA, {A, W, bias, labels, weight, count, lse, total, dloss}));
            ZG_TRY(check_apart(dW, {A, W, bias, labels, weight, count, lse, total, dloss, dA}));
            ZG_TRY(check_apart(dbias, {A, W, bias, labels, weight, count, lse, total, dloss, dA, dW}));
        }
        const Wanted want = wanted_of(a);
        DzPlan t = dz_plan(shape_of(a), want);
        ZG_TRY(check_workspace(d_workspace, workspace_bytes, t.total));
        if (!want.dA && !want.dW && !want.dbias) return ZG_OK;
        const hipStream_t st = static_cast<hipStream_t>(stream);
        char *const ws = static_cast<char *>(d_workspace);
        const Rows all{a->d_rows, (uint32_t)a->rows};
        float *const power = reinterpret_cast<float *>(ws + t.off_power);
        if (a->rows > 0) ZG_TRY(pack_W(st, a, ws, t.off_pack, t.pk));
        FactorArgs f{};
        f.rows = all;
        f.lse = a->d_lse, f.weight = a->d_weight, f.total = a->d_total, f.dloss = a->d_dloss;
        f.labels = {a->d_labels, a->label_dtype == ZG_I64, (uint32_t)a->out};
        // fp16's range does not hold a softmax over many classes as it is: |dZ| <= 1 is brought to the top of it.  Weights may be of any size: the largest is brought there, whatever the type.
        f.up = a->dtype == ZG_F16 ? 16384.0f : 1.0f;
        f.power = power;
        if (a->d_weight && a->rows > 0) {
            float *const tops = reinterpret_cast<float *>(ws + t.off_tops);
            f.tops = tops;
            ZG_TRY(launch(st, k_loss_weight_top, dim3(kWeightBlocks), 256, f, tops));
        }
        if (a->rows == 0) ZG_TRY(launch(st, k_loss_power, dim3(1), 64, f));
        uint32_t *const counts = t.steps > 1 && a->d_rows ? reinterpret_cast<uint32_t *>(ws + t.off_counts) : nullptr;
        if (counts) ZG_TRY(launch(st, k_row_counts, grid_of(((uint64_t)t.steps + 255) / 256), 256, all, (uint32_t)t.step, (uint32_t)t.steps, counts));
        const auto run = [&](auto zero) -> int {
            using T = decltype(zero);
            T *const dz = reinterpret_cast<T *>(ws + t.off_dz);
            float *const part_A = reinterpret_cast<float *>(ws + t.off_part_A), *const bias_part = reinterpret_cast<float *>(ws + t.off_bias);
            float *const part_W = reinterpret_cast<float *>(ws + t.off_part_W), *const sum_W = reinterpret_cast<float *>(ws + t.off_sum_W);
            const bool parts_A = t.pieces * t.splits_A > 1;
            Epilogue result_W{};
            result_W.factor = 1.0f, result_W.power = power, result_W.type = a->dtype, result_W.Y = a->d_dW, result_W.ld_Y = a->ld_dW;
            for (int64_t step = 0; step < t.steps; ++step) {
                const int64_t m0 = step * t.step, m = std::min(t.step, a->rows - m0), cells_A = m * a->in;
                const Rows rows{counts ? counts + step : t.steps > 1 ? nullptr : a->d_rows, (uint32_t)m};
                FactorArgs here = f;
                here.lse += m0;
                if (here.weight) here.weight += m0;
                here.labels.p = static_cast<const char *>(f.labels.p) + m0 * (f.labels.wide ? 8 : 4);
                ZG_TRY(pack_A(st, a, ws, t.off_pack, t.pk, m0, rows));
                uint32_t filled = 0; // parts of dA that are there
                for (int64_t first = 0; first < a->out; first += t.piece) {
                    const uint32_t n = (uint32_t)std::min<int64_t>(t.piece, a->out - first), n8 = (n + 7) / 8 * 8;
                    Operand w = t.pk.w;
                    w.p = static_cast<const T *>(w.p) + first * w.ld;
                    if (m > 0) {
                        Shape s = shape_of(a);
                        s.rows = m, s.out = (int32_t)n;
                        DzArgs<T> p{};
                        static_cast<ProductArgs &>(p) = logits_product(s, t.pk, rows.d_rows);
                        p.b = w;
                        p.e.bias = a->d_bias ? a->d_bias + first : nullptr;
                        p.e.Y = dz, p.e.ld_Y = t.ld_dz;
                        p.f = here, p.first = (uint32_t)first;
                        p.bias_part = want.dbias ? bias_part : nullptr, p.ld_part = t.ld_dz;
                        ZG_TRY(launch_dz(st, t.kind, p));
                    }
                    if (want.dbias) {
                        const uint32_t group = group_rows(t.kind, sizeof(T) == 4);
                        if (n < 1024) ZG_TRY(launch(st, k_loss_bias<8>, dim3((n + 7) / 8), 1024, rows, group, n, bias_part, t.ld_dz, power, a->d_dbias + first, step > 0));
                        else ZG_TRY(launch(st, k_loss_bias<32>, dim3((n + 31) / 32), 1024, rows, group, n, bias_part, t.ld_dz, power, a->d_dbias + first, step > 0));
                    }
                    if (want.dW) {
                        ProductArgs p{};
                        p.a = {dz, t.ld_dz, true, true};
                        p.b = t.pk.a, p.b.turned = true;
                        p.M = n, p.N = (uint32_t)a->in, p.K = (uint32_t)m;
                        p.rows = rows, p.rows_are_k = 1;
                        p.splits = t.splits_W;
                        Epilogue to = result_W; // or onto the sums of the rows in front of these
                        to.Y = static_cast<T *>(a->d_dW) + first * a->ld_dW;
                        if (t.steps > 1) {
                            to = Epilogue{};
                            to.factor = 1.0f, to.type = ZG_F32, to.Y = sum_W + first * a->in, to.ld_Y = a->in;
                            if (step > 0) to.R = to.Y, to.ld_R = a->in;
                        }
                        const bool narrow = sizeof(T) == 4 && n <= 64 && p.splits > 1 && in_chunks<T>(p.b, p.N, p.K);
                        if (!narrow && (p.splits > 1 || t.steps == 1)) {
                            p.e = to;
                            ZG_TRY(dense_product(st, a->dtype, p, part_W));
                        } else {
                            p.e.factor = 1.0f, p.e.type = ZG_F32, p.e.Y = part_W, p.e.ld_Y = p.N, p.e.part = (int64_t)p.M * p.N;
                            ZG_TRY(narrow ? launch(st, k_loss_part_narrow, tile_grid<64, 128>(p), 256, static_cast<const ProductArgs &>(p)) : dense_product(st, a->dtype, p));
                            ZG_TRY(dense_join(st, part_W, p.M, p.N, p.splits, to, {nullptr, p.M}));
                        }
                    }
                    if (want.dA && m > 0) {
                        ProductArgs p{};
                        p.a = {dz, t.ld_dz, false, true};
                        p.b = w, p.b.turned = true;
                        p.M = (uint32_t)m, p.N = (uint32_t)a->in;
                        // dZ lies in chunks, and the rows of a tile, 256 or as many as there are, in reach of each other: more than 2^29 bytes of it are there only where a row has 4096 classes, or where all of
                        // them take no more than two rows of dA at 32 bits do, 2^18 bytes.
                        const bool chunks = in_chunks<T>(p.b, p.N, n8);
                        p.K = chunks ? n8 : n, p.b_short = chunks ? n8 - n : 0;
                        p.rows = rows;
                        p.e.factor = 1.0f;
                        if (!parts_A) {
                            p.splits = 1;
                            p.e.power = power, p.e.type = a->dtype;
                            p.e.Y = static_cast<T *>(a->d_dA) + m0 * a->ld_dA, p.e.ld_Y = a->ld_dA;
                            // (bf16 2304 x 256 of 16 terms: 8.6 us in tiles of 256 x 128, 5.6 in tiles of 64 x 64)
                            if (tile_blocks<256, 128>(p) < 128 && p.K <= 256) {
                                p.K = n, p.b_short = 0;
                                ZG_TRY(launch(st, k_loss_part_anyhow<T>, tile_grid<64, 64>(p), 256, p));
                            } else {
                                ZG_TRY(dense_product(st, a->dtype, p));
                            }
                        } else {
                            Epilogue sum{};
                            sum.factor = 1.0f, sum.type = ZG_F32, sum.Y = part_A, sum.ld_Y = a->in;
                            if (filled + t.splits_A > t.slots_A) { // no room: what is there becomes the first part
                                ZG_TRY(dense_join(st, part_A, p.M, p.N, filled, sum, rows));
                                filled = 1;
                            }
                            p.splits = t.splits_A;
                            p.e.type = ZG_F32, p.e.Y = part_A + filled * cells_A, p.e.ld_Y = a->in, p.e.part = cells_A;
                            ZG_TRY(launch_parts<T>(st, p, chunks));
                            filled += t.splits_A;
                        }
                    }
                }
                if (want.dA && parts_A && m > 0) {
                    Epilogue e{};
                    e.factor = 1.0f, e.power = power, e.type = a->dtype, e.Y = static_cast<T *>(a->d_dA) + m0 * a->ld_dA, e.ld_Y = a->ld_dA;
                    ZG_TRY(dense_join(st, part_A, (uint32_t)m, (uint32_t)a->in, filled, e, rows));
                }
            }
            if (want.dW && t.steps > 1) return dense_join(st, sum_W, (uint32_t)a->out, (uint32_t)a->in, 1, result_W, {nullptr, (uint32_t)a->out});
            return ZG_OK;
        };
        return with_wide_type(a->dtype, run);
    });
}

} // extern "C"
