// Products with bias, activation, dropout and residual behind them, and their gradients.
#include "zg_dense.h"

#include <algorithm>
#include <tuple>

namespace zg {

int launch_column_sums(hipStream_t st, const float *part, uint32_t n, uint32_t cols, float factor, float *out);

namespace {

// What happens to a product's sums: v = factor scale_m scale_n sum, z = v + bias, y = R + drop(act(z)).
struct Epilogue {
    float factor;
    const float *power; // null, or a power of two (the device's own) that the sum is multiplied by before all else
    const float *scale_m, *scale_n, *bias;
    int32_t act, type; // type of R, Y and Z
    Drop drop;
    const void *R;
    int64_t ld_R;
    void *Y, *Z;
    int64_t ld_Y, ld_Z;
    bool stream;  // Y and Z go past the caches
    int64_t part; // elements between the parts of a sum that is made in parts (all else is left out then)
};

struct AnyType {}; // the type of R, Y and Z is looked up in the epilogue

// eight elements as they lie in memory (16 bits: two to a register)
template <class O> struct Eight {
    using E = std::conditional_t<std::is_same_v<O, AnyType>, float, O>;
    uint32_t w[2 * sizeof(E)];

    __device__ __forceinline__ float at(int j) const
    {
        if constexpr (sizeof(E) == 4) return __builtin_bit_cast(float, w[j]);
        else return (float)__builtin_bit_cast(E, (uint16_t)(j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xFFFFu));
    }
};

template <class O> __device__ __forceinline__ Eight<O> get8(const void *p, int32_t type, int64_t at, int n)
{
    Eight<O> r;
    if constexpr (std::is_same_v<O, AnyType>) {
        float v[8];
        load8(p, type, at, n, v);
        __builtin_memcpy(r.w, v, sizeof v);
    } else {
        const O *from = static_cast<const O *>(p) + at;
        if (n >= 8) {
            __builtin_memcpy(r.w, from, sizeof r.w);
        } else {
#pragma unroll
            for (auto &w : r.w) w = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j >= n) continue;
                if constexpr (sizeof(O) == 4) r.w[j] = __builtin_bit_cast(uint32_t, from[j]);
                else r.w[j / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, from[j]) << (j & 1 ? 16 : 0);
            }
        }
    }
    return r;
}

template <class O> __device__ __forceinline__ void put8(void *p, int32_t type, int64_t at, int n, const float (&v)[8], bool stream)
{
    if constexpr (std::is_same_v<O, AnyType>) store8(p, type, at, n, v, stream);
    else store8(static_cast<O *>(p) + at, n, v, stream);
}

// what the epilogue has of eight columns, whatever the row
struct Columns {
    uint32_t n;
    int left; // of the eight
    float scale[8], bias[8];
};

__device__ __forceinline__ Columns columns_of(const Epilogue &e, uint32_t n, uint32_t N)
{
    Columns c;
    c.n = n;
    c.left = (int)(N - n);
#pragma unroll
    for (int j = 0; j < 8; ++j) c.scale[j] = 1.0f, c.bias[j] = 0.0f;
    if (n < N) {
        if (e.scale_n) load8(e.scale_n + n, c.left, c.scale);
        if (e.bias) load8(e.bias + n, c.left, c.bias);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) c.scale[j] *= e.factor;
    return c;
}

// Eight columns of ROWS rows, `step` apart: what they need from memory, asked for well before it is used.
template <class O, int ROWS, bool PLAIN = false> struct Needs {
    Eight<O> r[ROWS];
    uint32_t id[ROWS];
    float scale[ROWS];

    __device__ __forceinline__ void ask(const Epilogue &e, uint32_t n, int left, uint32_t m0, uint32_t step, uint32_t M)
    {
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const uint32_t m = m0 + u * step;
            if (PLAIN) continue;
            id[u] = m;
            scale[u] = 1.0f;
            if (m >= M || left <= 0) continue;
            if (e.R) r[u] = get8<O>(e.R, e.type, m * e.ld_R + n, left);
            if (e.drop.ids) id[u] = (uint32_t)e.drop.ids[m];
            if (e.scale_m) scale[u] = e.scale_m[m];
        }
    }
};

// PLAIN: factor and rounding are all there is, as for gradients and parts of sums.
template <class O, int ROWS, bool PLAIN, class F>
__device__ __forceinline__ void finish(const Epilogue &e, const Columns &c, const Needs<O, ROWS, PLAIN> &needs, uint32_t m0, uint32_t step, uint32_t M, F &&sums)
{
    if (c.left <= 0) return;
    constexpr bool gradients = PLAIN || std::is_same_v<O, AnyType>; // (or either)
    const float power = gradients && e.power ? *e.power : 1.0f;
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        const uint32_t m = m0 + u * step;
        if (m >= M) continue;
        float v[8];
        sums(u, v);
        if (gradients && e.power) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= power;
        }
        if constexpr (PLAIN) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= e.factor;
            put8<O>(e.Y, e.type, m * e.ld_Y + c.n, c.left, v, e.stream);
            continue;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(v[j], needs.scale[u] * c.scale[j], c.bias[j]);
        if (e.Z) put8<O>(e.Z, e.type, m * e.ld_Z + c.n, c.left, v, e.stream);
        if (e.act != ZG_ACT_NONE) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = act_of<sizeof(typename Eight<O>::E) == 4>(e.act, v[j]); // (AnyType: for the widest)
        }
        if (e.drop.cut) mask8(e.drop, needs.id[u], c.n >> 3, e.drop.scale, v);
        if (e.R) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += needs.r[u].at(j);
        }
        put8<O>(e.Y, e.type, m * e.ld_Y + c.n, c.left, v, e.stream);
    }
}

// C[m, n] = sum over k of a(m, k) b(n, k); element (i, k) of an operand is p[i * ld + k], or p[k * ld + i] where it is turned.
struct Operand {
    const void *p;
    int64_t ld;
    bool turned;
};

struct ProductArgs {
    Operand a, b;
    uint32_t M, N, K;
    Rows rows;
    int32_t rows_are_k; // the device's count bounds K, else M
    uint32_t splits;    // parts that the sum is made in
    Epilogue e;
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Operands are dealt with in chunks of 16 bytes of one row, 4, 8 or 16 consecutive k.  A matrix instruction takes from a lane's chunk what
// it takes for its half of the wavefront: which k that is does not matter as long as both operands agree.
template <class T> constexpr int chunk_k = 16 / (int)sizeof(T);

// 8-bit operands are multiplied as fp16, which holds each of their values and two of which make an exact product in fp32.  (The matrix instructions
// for 8-bit operands add eight products at a time in a window that ends about 13 bits below the largest of them: one large column in eight takes up
// to 2^-10 of a sum with it, and all of it where the large ones cancel.)  Widened8: operands that are widened on their way to LDS, eight to a chunk;
// uint8_t: operands that lie in LDS as they do in memory, sixteen to a chunk.
struct Widened8 {
    uint8_t v;
};
template <> constexpr int chunk_k<Widened8> = 8;

__device__ __forceinline__ u32x4 widen(uint32_t lo, uint32_t hi) // eight 8-bit values as fp16
{
    const uint32_t r[2] = {lo, hi};
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        w[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(r[i], 1.0f, false));
        w[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(r[i], 1.0f, true));
    }
    return w;
}

// acc += the products over one pair of chunks (a lane's half of the wavefront has one of the two), all 32 x 32 cells.  The first operand's
// rows become the cells that a lane holds side by side.
__device__ __forceinline__ void multiply(float, u32x4 x, u32x4 y, f32x16 &acc)
{
    const f32x4 a = __builtin_bit_cast(f32x4, x), b = __builtin_bit_cast(f32x4, y);
#pragma unroll
    for (int k = 0; k < 4; ++k) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[k], b[k], acc, 0, 0, 0);
}

__device__ __forceinline__ void multiply(_Float16, u32x4 x, u32x4 y, f32x16 &acc)
{
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), acc, 0, 0, 0);
}

__device__ __forceinline__ void multiply(Widened8, u32x4 x, u32x4 y, f32x16 &acc) { multiply((_Float16)0, x, y, acc); }

__device__ __forceinline__ void multiply(__bf16, u32x4 x, u32x4 y, f32x16 &acc)
{
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
}

// Where chunk c of row i lies in an operand's tile in LDS (8 chunks to a row).  Eight rows at one c, eight chunks of one row, and every
// fourth row at one c - what a wavefront reads, writes, and writes of an operand that it turns - each lie in eight different groups of banks.
__device__ __forceinline__ uint32_t slot(uint32_t i, uint32_t c) { return 8 * i + (c ^ ((i ^ (i >> 2)) & 7)); }

// The first n < K elements of a chunk (none where n <= 0), zeros behind them.  Where the row has a chunk's worth of elements up to there
// (`long_row`), the 16 bytes that end with them are read and shifted.
template <class T> __device__ __forceinline__ u32x4 part_of_chunk(const T *from, int n, bool long_row)
{
    constexpr int K = chunk_k<T>;
    uint64_t lo = 0, hi = 0;
    if (n > 0 && long_row) {
        uint64_t w[2] = {};
        __builtin_memcpy(w, from + n - K, K * sizeof(T));
        const int s = (K - n) * (int)sizeof(T) * 8;
        lo = s >= 64 ? w[1] >> (s - 64) : w[0] >> s | w[1] << (64 - s);
        hi = s >= 64 ? 0 : w[1] >> s;
    } else {
#pragma unroll 1
        for (int j = 0; j < n; ++j) {
            uint64_t bits = 0;
            __builtin_memcpy(&bits, from + j, sizeof(T));
            const int s = j * (int)sizeof(T) * 8;
            if (s < 64) lo |= bits << s;
            else hi |= bits << (s - 64);
        }
    }
    return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// One operand's way from memory to LDS: `tile` rows, eight chunks of k.  TURNED: its elements lie side by side along the rows and not
// along k.  What is beyond the last row or k is 0 and not read.
template <class T, int tile, bool TURNED> struct Side {
    static constexpr int K = chunk_k<T>, regs = tile / 32 < 4 && TURNED ? 4 : tile / 32; // chunks of a lane
    static constexpr int groups = tile / 4, patches = 8 * groups;                         // (TURNED: a lane has four at a time)
    const T *p;
    int64_t ld;
    uint32_t first, rows; // the tile's first row; rows of the operand
    u32x4 r[regs];

    __device__ __forceinline__ void load(uint32_t k0, uint32_t k_end)
    {
        if constexpr (!TURNED) {
            if (k0 + 8 * K <= k_end) { // (rows beyond the last one repeat it: their cells are not kept)
#pragma unroll
                for (int c = 0; c < regs; ++c) {
                    const uint32_t e = threadIdx.x + 256 * c;
                    const T *from = p + min(first + e / 8, rows - 1) * ld + k0 + (e % 8) * K;
                    __builtin_memcpy(&r[c], from, K * sizeof(T));
                }
            } else {
#pragma unroll
                for (int c = 0; c < regs; ++c) {
                    const uint32_t e = threadIdx.x + 256 * c, k = k0 + (e % 8) * K;
                    const T *from = p + min(first + e / 8, rows - 1) * ld + k;
                    if (k + K <= k_end) __builtin_memcpy(&r[c], from, K * sizeof(T));
                    else r[c] = part_of_chunk(from, (int)(k_end - k), k_end >= (uint32_t)K);
                }
            }
        } else { // K rows of four elements: four chunks once they are turned
#pragma unroll
            for (int c = 0; c < regs / 4; ++c) {
                const uint32_t e = threadIdx.x + 256 * c, i = first + 4 * (e % groups), k = k0 + (e / groups) * K;
                T t[K][4] = {};
                if (patches < 256 && threadIdx.x >= patches) continue;
                if (k0 + 8 * K <= k_end && first + tile <= rows) {
#pragma unroll
                    for (int j = 0; j < K; ++j) __builtin_memcpy(t[j], p + (k + j) * ld + i, 4 * sizeof(T));
                } else {
#pragma unroll
                    for (int j = 0; j < K; ++j) {
                        if (k + j >= k_end) continue;
                        const T *from = p + (k + j) * ld + i;
                        if (i + 4 <= rows) {
                            __builtin_memcpy(t[j], from, 4 * sizeof(T));
                        } else {
#pragma unroll
                            for (int h = 0; h < 4; ++h)
                                if (i + h < rows) t[j][h] = from[h];
                        }
                    }
                }
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    T u[K];
#pragma unroll
                    for (int j = 0; j < K; ++j) u[j] = t[j][h];
                    __builtin_memcpy(&r[4 * c + h], u, 16);
                }
            }
        }
    }

    __device__ __forceinline__ void store(u32x4 *lds) const
    {
        if constexpr (!TURNED) {
#pragma unroll
            for (int c = 0; c < regs; ++c) {
                const uint32_t e = threadIdx.x + 256 * c;
                if constexpr (std::is_same_v<T, Widened8>) lds[slot(e / 8, e % 8)] = widen(r[c][0], r[c][1]);
                else lds[slot(e / 8, e % 8)] = r[c];
            }
        } else {
#pragma unroll
            for (int c = 0; c < regs / 4; ++c) {
                const uint32_t e = threadIdx.x + 256 * c;
                if (patches < 256 && threadIdx.x >= patches) continue;
#pragma unroll
                for (int h = 0; h < 4; ++h) lds[slot(4 * (e % groups) + h, e / groups)] = r[4 * c + h];
            }
        }
    }
};

// What lanes of a wavefront put into LDS before this, its other lanes read behind it, and what they read before it may be written over behind it.  LDS
// serves a wavefront in order, so no instruction is needed; it holds the compiler to that order.
__device__ __forceinline__ void lds_exchange()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// What a wavefront does with its 32 FM x 64 cells' sums.  Of 32 x 32 cells a lane has row lane % 32, columns 8 q + 4 half + 0..3 in registers
// 4 q + 0..3: they go through LDS (`mine`: 8 KB of the wavefront's own, free from here on), 32 rows at a time, so that eight lanes have 64 columns of a row
// and memory sees whole lines.  Places are 16 bytes, 16 to a row, turned by the row so that neither way meets in a bank.
template <class O, bool PLAIN, int FM> __device__ __forceinline__ void hand_over(const ProductArgs &p, f32x16 (&acc)[FM][2], f32x4 *mine, uint32_t m_wave, uint32_t n_wave, uint32_t M, uint32_t split)
{
    const uint32_t lane = threadIdx.x & 63, half = lane >> 5, row = lane & 31, g = lane & 7;
    const Columns c = columns_of(p.e, n_wave + 8 * g, p.N);
    Epilogue e = p.e;
    if (split) e.Y = static_cast<float *>(e.Y) + split * e.part;
    constexpr int ahead = sizeof(Eight<O>) > 16 ? 0 : 1; // (what fits beside the sums)
    Needs<O, 4, PLAIN> needs[ahead + 1];
    const auto first = [&](int i) { return m_wave + 32 * i + (lane >> 3); };
    if (ahead) needs[0].ask(e, c.n, c.left, first(0), 8, M);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        if (i + ahead < FM) needs[(i + ahead) % (ahead + 1)].ask(e, c.n, c.left, first(i + ahead), 8, M);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                mine[row * 16 + ((8 * j + 2 * q + half) ^ (row & 15))] = f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        lds_exchange();
        finish(e, c, needs[i % (ahead + 1)], first(i), 8, M, [&](int u, float (&v)[8]) {
            const uint32_t r = (lane >> 3) + 8 * u;
            const f32x4 lo = mine[r * 16 + ((2 * g) ^ (r & 15))], hi = mine[r * 16 + ((2 * g + 1) ^ (r & 15))];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = lo[j], v[4 + j] = hi[j];
        });
        lds_exchange();
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The same through 4 KB, 32 x 32 cells at a time: four lanes have 32 columns of a row.  What a part needs from memory is asked for
// ahead.
template <class O, bool PLAIN, int FM, int FN> __device__ __forceinline__ void hand_over_narrow(const ProductArgs &p, f32x16 (&acc)[FM][FN], f32x4 *mine, uint32_t m_wave, uint32_t n_wave, uint32_t M, uint32_t split)
{
    constexpr int parts = FN * FM, ahead = sizeof(Eight<O>) > 16 ? 0 : 2; // (what fits beside the sums)
    const uint32_t lane = threadIdx.x & 63, half = lane >> 5, row = lane & 31, g = lane & 3;
    Epilogue e = p.e;
    if (split) e.Y = static_cast<float *>(e.Y) + split * e.part;
    Columns c;
    const auto ask = [&](Needs<O, 2, PLAIN> &needs, int n) {
        const uint32_t col = n_wave + 32 * (n / FM) + 8 * g;
        needs.ask(e, col, (int)(p.N - col), m_wave + 32 * (n % FM) + (lane >> 2), 16, M);
    };
    Needs<O, 2, PLAIN> needs[ahead + 1];
#pragma unroll
    for (int n = 0; n < ahead && n < parts; ++n) ask(needs[n], n);
#pragma unroll
    for (int n = 0; n < parts; ++n) {
        const int i = n % FM, j = n / FM;
        if (i == 0) c = columns_of(p.e, n_wave + 32 * j + 8 * g, p.N);
        if (n + ahead < parts) ask(needs[(n + ahead) % (ahead + 1)], n + ahead);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            mine[row * 8 + ((2 * q + half) ^ ((row >> 1) & 7))] = f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        lds_exchange();
        finish(e, c, needs[n % (ahead + 1)], m_wave + 32 * i + (lane >> 2), 16, M, [&](int u, float (&v)[8]) {
            const uint32_t r = (lane >> 2) + 16 * u;
            const f32x4 lo = mine[r * 8 + ((2 * g) ^ ((r >> 1) & 7))], hi = mine[r * 8 + ((2 * g + 1) ^ ((r >> 1) & 7))];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = lo[k], v[4 + k] = hi[k];
        });
        lds_exchange();
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The tiles of a product, and the parts of their sums.  Workgroups go to the eight XCDs in turn; each XCD gets a run of tiles, those of one row of
// tiles (of one part of the sum) beside each other, so that what they share is in its L2, and its workgroups take them in turn.
struct Place {
    uint32_t m0, n0, split, k_first, k_end;
};

template <int BM, int BN> struct Tiles {
    uint32_t M, k_all, nt, splits, part_k;
    uint64_t in_part, next, end; // of this workgroup: the next tile, the end of its XCD's run

    __device__ __forceinline__ Tiles(const ProductArgs &p, uint32_t depth)
    {
        const uint32_t live = p.rows.live();
        M = p.rows_are_k ? p.M : min(p.M, live);
        k_all = p.rows_are_k ? min(p.K, live) : p.K;
        nt = (p.N + BN - 1) / BN;
        splits = p.splits;
        in_part = (uint64_t)((M + BM - 1) / BM) * nt;
        part_k = __builtin_amdgcn_readfirstlane(((k_all + splits - 1) / splits + depth - 1) / depth * depth);
        const uint64_t tiles = in_part * splits, share = (tiles + 7) / 8;
        next = blockIdx.x % 8 * share + block_number() / 8; // (a grid's first dimension is a multiple of 8)
        end = min((blockIdx.x % 8 + 1) * share, tiles);
    }
    __device__ __forceinline__ bool take(Place &w)
    {
        if (next >= end) return false;
        // (all of it is the same in every lane: said so, or the divisions would leave it in vector registers)
        const auto same = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane(v); };
        w.split = splits > 1 ? same((uint32_t)(next / in_part)) : 0u;
        const uint32_t t = same((uint32_t)(next - w.split * in_part)), row = same(t / nt);
        w.m0 = row * BM;
        w.n0 = (t - row * nt) * BN;
        w.k_first = same((uint32_t)min((uint64_t)k_all, (uint64_t)part_k * w.split));
        w.k_end = same((uint32_t)min((uint64_t)k_all, (uint64_t)w.k_first + part_k));
        next += gridDim.x / 8;
        return true;
    }
};

// A tile of BM x BN cells: four wavefronts, two by two, matrix instructions of 32 x 32 cells; eight chunks of k at a time through two buffers
// in LDS, the next ones on their way in registers.  The first operand of an instruction is b, so that a lane's cells lie side by side in a
// row of C.  For operands that lie anyhow.  Bound by the dependent steps of loads: 33333 x 301 x 47 fp16, rows of 606 bytes, 11.5 us.
template <class T, int BM, int BN, bool A_TURNED, bool B_TURNED> __global__ __launch_bounds__(256, 2) void k_product(ProductArgs p)
{
    constexpr int K = chunk_k<T>, depth = 8 * K, FM = BM / 64, FN = BN / 64;
    __shared__ u32x4 lds[2][(BM + BN) * 8];
    Tiles<BM, BN> tiles(p, depth);
    Place w;
    if (!tiles.take(w)) return;
    const uint32_t k_end = w.k_end, M = tiles.M;
    Side<T, BM, A_TURNED> a;
    Side<T, BN, B_TURNED> b;
    a.p = static_cast<const T *>(p.a.p), a.ld = p.a.ld, a.first = w.m0, a.rows = M;
    b.p = static_cast<const T *>(p.b.p), b.ld = p.b.ld, b.first = w.n0, b.rows = p.N;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const uint32_t wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2), am = wm + (lane & 31), bn = wn + (lane & 31);
    f32x16 acc[FM][FN] = {};
    if (w.k_first < k_end) {
        a.load(w.k_first, k_end);
        b.load(w.k_first, k_end);
        a.store(lds[0]);
        b.store(lds[0] + BM * 8);
    }
    __syncthreads();
    uint32_t now = 0;
    for (uint32_t k0 = w.k_first; k0 < k_end; k0 += depth, now ^= 1) {
        const bool more = k_end - k0 > (uint32_t)depth;
        if (more) {
            a.load(k0 + depth, k_end);
            b.load(k0 + depth, k_end);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            u32x4 fa[FM], fb[FN];
#pragma unroll
            for (int i = 0; i < FM; ++i) fa[i] = lds[now][slot(am + 32 * i, 2 * s + half)];
#pragma unroll
            for (int j = 0; j < FN; ++j) fb[j] = lds[now][BM * 8 + slot(bn + 32 * j, 2 * s + half)];
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) multiply(T(), fb[j], fa[i], acc[i][j]);
        }
        if (more) {
            a.store(lds[now ^ 1]);
            b.store(lds[now ^ 1] + BM * 8);
        }
        __syncthreads();
    }
    if constexpr (FN == 2) hand_over<AnyType, false>(p, acc, reinterpret_cast<f32x4 *>(lds) + wave * 512, w.m0 + wm, w.n0 + wn, M, w.split);
    else hand_over_narrow<AnyType, false>(p, acc, reinterpret_cast<f32x4 *>(lds) + wave * 256, w.m0 + wm, w.n0 + wn, M, w.split);
}

// ---- operands in whole chunks ---------------------------------------------------------------------------------------------------
// Where both operands' rows start on 16-byte boundaries and are whole chunks long, chunks go from memory to LDS without passing through
// registers, two steps ahead of the one that is multiplied: three buffers, a step being four chunks (64 bytes) of k for every row of the
// tile.  A wavefront has 128 x 64 cells of a workgroup's 256 x 128.

constexpr uint32_t kReach = 0x80000000u; // bytes that what a tile reads in a step may span: offsets from here on read zeros

typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// all but the last n loads of this wavefront are done, and so are its reads of LDS
template <int n> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(n) : "memory"); }

// One operand's buffer in LDS, CH `tile` places of 16 bytes (CH chunks of k a step), and its way there: 64 places side by side are filled by one instruction of a
// wavefront, each lane's from where it says.
template <class T, int tile, int waves, int CH, bool TURNED> struct Feed;

// Along k in memory: place (row i, chunk c) is CH i + (c ^ turn(i)).  LDS serves 16 lanes of a 16-byte read at a time, 0-3, 12-15, 20-23 and 24-27
// first: at one c those rows lie in 16 different groups of banks, as do the others'.
template <class T, int tile, int waves, int CH> struct Feed<T, tile, waves, CH, false> {
    static constexpr int K = 16 / (int)sizeof(T), loads = tile * CH / (64 * waves);
    static_assert(CH == 4 || loads % 4 == 0, "");
    const char *p;
    uint32_t from[loads], chunk;

    __device__ __forceinline__ static uint32_t turn(uint32_t i) { return CH == 4 ? (i >> 2) & 3 : (i ^ (i >> 2)) & 7; }
    // which chunk a lane has in its lth load: the rows of one load are 64 / CH further on than those of the one before
    __device__ __forceinline__ uint32_t chunk_at(int l) const { return CH == 4 ? chunk : chunk ^ (2 * l & 7); }

    __device__ __forceinline__ void start(const Operand &o, uint32_t first, uint32_t rows, uint32_t wave, uint32_t lane)
    {
        const uint64_t ld = (uint64_t)o.ld * sizeof(T);
        p = static_cast<const char *>(o.p) + first * ld;
        chunk = (lane % CH) ^ turn(wave * loads * 64 / CH + lane / CH);
#pragma unroll
        for (int l = 0; l < loads; ++l) {
            const uint32_t i = (wave * loads + l) * (64 / CH) + lane / CH;
            from[l] = first + i < rows ? (uint32_t)(i * ld) + chunk_at(l) * 16 : kReach;
        }
    }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t at(uint32_t k0) const
    {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p) + (uint64_t)k0 * sizeof(T), 0, kReach, 0x00027000);
    }
    // the lth of a step's loads, out of at(k0); zeros where there are no more than `left` k from k0 on
    __device__ __forceinline__ void fetch(int l, __amdgpu_buffer_rsrc_t r, uint32_t left, u32x4 *buffer, uint32_t wave) const
    {
        const uint32_t beyond = (chunk_at(l) + 1) * K <= left ? 0u : kReach;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_u32x4 *)(buffer + (wave * loads + l) * 64), 16, (int)(from[l] | beyond), 0, 0, 0);
    }
    // chunk c of row i
    __device__ __forceinline__ static u32x4 chunk_of(const u32x4 *buffer, uint32_t i, uint32_t c)
    {
        return buffer[CH * i + (c ^ turn(i))];
    }
};

// Along the rows in memory: the buffer holds a row of the tile's `tile` rows for each k, and a lane's chunk is put together as it is read.
template <class T, int tile, int waves, int CH> struct Feed<T, tile, waves, CH, true> {
    static constexpr int K = 16 / (int)sizeof(T), loads = tile * CH / (64 * waves), row = tile / K; // places of one k
    const char *p;
    uint64_t ld;
    uint32_t from[loads], k_of[loads];

    // 16-bit rows of four k that are read together start 64 bytes apart in the banks
    __device__ __forceinline__ static uint32_t turn(uint32_t k) { return sizeof(T) == 2 ? (k & 3) << 2 : 0; }

    __device__ __forceinline__ void start(const Operand &o, uint32_t first, uint32_t rows, uint32_t wave, uint32_t lane)
    {
        ld = (uint64_t)o.ld * sizeof(T);
        p = static_cast<const char *>(o.p) + (uint64_t)first * sizeof(T);
#pragma unroll
        for (int l = 0; l < loads; ++l) {
            const uint32_t s = (wave * loads + l) * 64 + lane, i = ((s % row) ^ turn(s / row)) * K;
            k_of[l] = s / row;
            from[l] = first + i < rows ? (uint32_t)(k_of[l] * ld) + i * (uint32_t)sizeof(T) : kReach;
        }
    }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t at(uint32_t k0) const
    {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p) + k0 * ld, 0, kReach, 0x00027000);
    }
    __device__ __forceinline__ void fetch(int l, __amdgpu_buffer_rsrc_t r, uint32_t left, u32x4 *buffer, uint32_t wave) const
    {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_u32x4 *)(buffer + (wave * loads + l) * 64), 16, (int)(from[l] | (k_of[l] < left ? 0u : kReach)), 0, 0, 0);
    }
    // 16-bit: a group of 16 lanes reads four k of 16 rows, four rows to a lane, and each gets its row's four k (lane 4 k + r / 4 has
    // rows r .. r + 3 of the k-th); i = the lane's row.  fp32: four reads.
    __device__ __forceinline__ static u32x4 chunk_of(const u32x4 *buffer, uint32_t i, uint32_t c)
    {
        if constexpr (sizeof(T) == 2) {
            const uint32_t lane = threadIdx.x & 15, r = (i & ~15u) + 4 * (lane & 3);
            u32x4 v;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t k = 8 * c + 4 * h + (lane >> 2);
                const auto *at = reinterpret_cast<const uint16_t *>(buffer + k * row + ((r / 8) ^ turn(k))) + (r & 4);
                const s16x4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at);
                const uint64_t two = __builtin_bit_cast(uint64_t, t);
                v[2 * h] = (uint32_t)two, v[2 * h + 1] = (uint32_t)(two >> 32);
            }
            return v;
        } else {
            u32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = reinterpret_cast<const uint32_t *>(buffer)[(4 * c + j) * tile + i];
            return v;
        }
    }
};

// A part of a step, a pair of chunks of k: a wavefront's fragments of 32 rows, a chunk of each to a lane.
template <class T, int FM, int FN, int CH> struct Part {
    static constexpr bool widened = std::is_same_v<T, uint8_t>; // a chunk is multiplied in two halves
    static constexpr int parts = CH / 2, products = FM * FN * (widened ? 2 : 1);
    u32x4 a[FM], b[FN];

    template <class A, class B> __device__ __forceinline__ void read(int part, const u32x4 *la, const u32x4 *lb, uint32_t am, uint32_t bn, uint32_t half)
    {
#pragma unroll
        for (int j = 0; j < FN; ++j) b[j] = B::chunk_of(lb, bn + 32 * j, 2 * part + half);
#pragma unroll
        for (int i = 0; i < FM; ++i) a[i] = A::chunk_of(la, am + 32 * i, 2 * part + half);
    }
    // `between(n)` is called behind the nth of `products`
    template <class F> __device__ __forceinline__ void multiply_into(f32x16 (&acc)[FM][FN], F &&between) const
    {
        if constexpr (widened) { // (a's fragments one by one: the registers do not hold all of them)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 wb[FN];
#pragma unroll
                for (int j = 0; j < FN; ++j) wb[j] = widen(b[j][2 * h], b[j][2 * h + 1]);
#pragma unroll
                for (int i = 0; i < FM; ++i) {
                    const u32x4 wa = widen(a[i][2 * h], a[i][2 * h + 1]);
#pragma unroll
                    for (int j = 0; j < FN; ++j) {
                        multiply((_Float16)0, wb[j], wa, acc[i][j]);
                        between((h * FM + i) * FN + j);
                    }
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    multiply(T(), b[j], a[i], acc[i][j]);
                    between(i * FN + j);
                }
        }
    }
};

// The steps of a tile, one after the other, in parts: while the matrix instructions of one part run, the chunks of the next are on their way
// from LDS.  In front of the last part all wavefronts meet: from there on the step's buffer is free - it is asked to be filled with the step that
// comes `stages` later - and the next step's is full.  The loads go out one by one between the products: together, right behind the meeting, those
// of all wavefronts queue up and the products wait behind them; half of them behind the next step's first part.
template <class T, class A, class B, int FM, int FN, int CH, int stages, class Fetch>
__device__ __forceinline__ void multiply_steps(f32x16 (&acc)[FM][FN], const u32x4 *lds, int lb_at, uint32_t stage, uint32_t steps, uint32_t am, uint32_t bn,
                                               uint32_t &now, Fetch &fetch)
{
    using P = Part<T, FM, FN, CH>;
    constexpr int loads = A::loads + B::loads, half_of = loads / 2, products = P::products, last = P::parts - 1;
    const uint32_t half = (threadIdx.x & 63) >> 5;
    P one, two;
    const auto read = [&](P &part, int n) {
        const u32x4 *const la = lds + now * stage;
        part.template read<A, B>(n, la, la + lb_at, am, bn, half);
    };
    // loads first .. end - 1, evenly behind the products of a part
    const auto spread = [&](int m, int first, int end) {
#pragma unroll
        for (int l = 0; l < loads; ++l)
            if (l >= first && l < end && (l - first) * products / (end - first) == m) fetch.load(l);
        __builtin_amdgcn_sched_barrier(0);
    };
    read(one, 0);
    for (uint32_t t = 0; t < steps; ++t) {
#pragma unroll
        for (int n = 0; n < last; ++n) {
            P &cur = n % 2 ? two : one, &nxt = n % 2 ? one : two;
            read(nxt, n + 1);
            __builtin_amdgcn_sched_barrier(0);
            cur.multiply_into(acc, [&](int m) {
                if (n == 0) spread(m, half_of, loads);
            });
            __builtin_amdgcn_sched_barrier(0);
            if (n == 0) fetch.next();
        }
        // this wavefront's share of the next step is there (what was asked for behind it may be on its way), and it has read this step's chunks
        wait_loads<(stages - 2) * loads>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        now = now == stages - 1 ? 0 : now + 1;
        read(one, 0); // (behind the last step, too: nobody looks at it then)
        __builtin_amdgcn_sched_barrier(0);
        fetch.open();
        two.multiply_into(acc, [&](int m) { spread(m, 0, half_of); });
    }
}

// What is asked for of both operands, step by step, into one buffer after the other; `on` moves it to the next tile, if there is one.  Where nothing is
// left it asks for zeros all the same, into buffers that nobody reads: what a wavefront waits for is then the same at every step.
template <class A, class B, int b_at, int step_k, int stage, int stages, class On> struct Fetch {
    A &a;
    B &b;
    u32x4 *lds;
    uint32_t wave, k, k_end;
    On on;
    uint32_t into = 0, left = 0;
    __amdgpu_buffer_rsrc_t ra, rb;

    __device__ __forceinline__ void open()
    {
        left = k < k_end ? k_end - k : 0u;
        ra = a.at(k);
        rb = b.at(k);
    }
    __device__ __forceinline__ void load(int l) const
    {
        u32x4 *const to = lds + into * stage;
        if (l < A::loads) a.fetch(l, ra, left, to, wave);
        else b.fetch(l - A::loads, rb, left, to + b_at, wave);
    }
    __device__ __forceinline__ void next()
    {
        into = into == stages - 1 ? 0 : into + 1;
        if (left == 0) return;
        k += step_k;
        if (k >= k_end) on(*this);
    }
    // the first steps, but for half of the last one's loads; the first is there then
    __device__ __forceinline__ void begin()
    {
        constexpr int loads = A::loads + B::loads;
#pragma unroll
        for (int i = 0; i < stages; ++i) {
            open();
#pragma unroll
            for (int l = 0; l < (i + 1 < stages ? loads : loads / 2); ++l) load(l);
            if (i + 1 < stages) next();
        }
        wait_loads<(stages - 2) * loads + loads / 2>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
};

// Four wavefronts, two by two, BLOCKS workgroups to a compute unit, which hide each other's way in and out; three buffers.  fp32 (128 x 128, three
// to a compute unit): bound by the matrix instructions, 285127 x 256 x 256 with ReLU and Z 370 us, 100 TFLOP/s, 65536 x 1024 x 1024 1005 us, 137.
// 16 and 8 bits (256 x 128, two): by matrix instructions, the epilogue's vector instructions and stores in part beside each other, bf16
// 65537 x 1024 x 1024 with GELU, dropout, residual and Z 266 us, 8 bits 65536 x 1024 x 2048 with SiLU 305 us, 8192 x 8192 x 8192 841 us, 1310 TFLOP/s.
template <class T, class O, int BM, int BN, int BLOCKS, bool A_TURNED, bool B_TURNED> __global__ __launch_bounds__(256, BLOCKS) void k_chunks(ProductArgs p)
{
    using A = Feed<T, BM, 4, 4, A_TURNED>;
    using B = Feed<T, BN, 4, 4, B_TURNED>;
    constexpr int depth = 4 * A::K, FM = BM / 64, FN = BN / 64, stages = 3, stage = (BM + BN) * 4;
    __shared__ u32x4 lds[stages * stage];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2), am = wm + (lane & 31), bn = wn + (lane & 31);
    Tiles<BM, BN> tiles(p, depth);
    Place w;
    if (!tiles.take(w)) return;
    A a;
    B b;
    a.start(p.a, w.m0, tiles.M, wave, lane);
    b.start(p.b, w.n0, p.N, wave, lane);
    const uint32_t steps = (w.k_end - w.k_first + depth - 1) / depth;
    const auto no_more = [](auto &) {};
    Fetch<A, B, BM * 4, depth, stage, stages, decltype(no_more)> fetch{a, b, lds, wave, w.k_first, w.k_end, no_more};
    f32x16 acc[FM][FN] = {};
    uint32_t now = 0;
    if (steps > 0) {
        fetch.begin();
        multiply_steps<T, A, B, FM, FN, 4, stages>(acc, lds, BM * 4, stage, steps, am, bn, now, fetch);
        wait_loads<0>();
    }
    __syncthreads(); // the buffers are free
    hand_over<O, B_TURNED>(p, acc, reinterpret_cast<f32x4 *>(lds) + wave * 512, w.m0 + wm, w.n0 + wn, tiles.M, w.split);
}

// Eight wavefronts, 256 x 256 cells, one workgroup to a compute unit, which takes one tile after the other; two buffers of eight chunks (128 bytes) of k.  For 16-bit types.  The next tile's
// first steps are on their way while this one's cells are handed over, through LDS of their own.  Bound by what is between the matrix
// instructions (counters: they run for 0.38 to 0.43 of the time over 1024 terms): bf16 65536 x 1024 x 1024 162 us, 850 TFLOP/s, 4096 x 16384 x 4096 433 us, 1270.
template <class T, class O, bool A_TURNED, bool B_TURNED> __global__ __launch_bounds__(512, 2) void k_long(ProductArgs p)
{
    constexpr int BM = 256, BN = 256, FM = 4, FN = 2, CH = 8, stages = 2, stage = (BM + BN) * CH;
    using A = Feed<T, BM, 8, CH, A_TURNED>;
    using B = Feed<T, BN, 8, CH, B_TURNED>;
    constexpr int depth = CH * A::K;
    __shared__ u32x4 lds[stages * stage + 8 * 256];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = (wave >> 2) * 128, wn = (wave & 3) * 64, am = wm + (lane & 31), bn = wn + (lane & 31);
    Tiles<BM, BN> tiles(p, depth), ahead = tiles;
    A a{}; // (a workgroup without a tile asks for zeros)
    B b{};
    const auto on = [&](auto &fetch) { // to the next tile that has something to read
        Place h;
        while (ahead.take(h)) {
            if (h.k_first >= h.k_end) continue;
            a.start(p.a, h.m0, tiles.M, wave, lane);
            b.start(p.b, h.n0, p.N, wave, lane);
            fetch.k = h.k_first, fetch.k_end = h.k_end;
            return;
        }
    };
    Fetch<A, B, BM * CH, depth, stage, stages, decltype(on)> fetch{a, b, lds, wave, 0, 0, on};
    on(fetch);
    fetch.begin();
    Place w;
    uint32_t now = 0;
    while (tiles.take(w)) {
        f32x16 acc[FM][FN] = {};
        const uint32_t steps = (w.k_end - w.k_first + depth - 1) / depth;
        if (steps > 0) multiply_steps<T, A, B, FM, FN, CH, stages>(acc, lds, BM * CH, stage, steps, am, bn, now, fetch);
        hand_over_narrow<O, B_TURNED>(p, acc, reinterpret_cast<f32x4 *>(lds) + stages * stage + wave * 256, w.m0 + wm, w.n0 + wn, tiles.M, w.split);
    }
    wait_loads<0>();
}

// ---- few tiles ------------------------------------------------------------------------------------------------------------------
// Where tiles of the sizes above would leave most of the chip idle, or be mostly empty: a workgroup has 32 x 32 cells, its four wavefronts
// every fourth pair of chunks of k each, straight from memory into registers; their sums meet in LDS.  Nothing is shared but what the caches
// hold, and a call lasts little more than one way to memory and back: 1 x 256 x 512 bf16 4 us, 1 x 2048 x 2048 7.1, 512 x 512 x 512 4.5.  Operands
// lie along k, anyhow.
template <class T> struct Along {
    static constexpr int K = chunk_k<T>;
    const T *row;
    uint32_t k_end;
    __device__ __forceinline__ u32x4 at(uint32_t k) const
    {
        u32x4 r = {};
        if (k + K <= k_end) __builtin_memcpy(&r, row + k, K * sizeof(T));
        else if (k < k_end) r = part_of_chunk(row + k, (int)(k_end - k), k_end >= (uint32_t)K);
        if constexpr (std::is_same_v<T, Widened8>) return widen(r[0], r[1]);
        else return r;
    }
};

template <class T> __global__ __launch_bounds__(256) void k_few(ProductArgs p)
{
    constexpr int K = chunk_k<T>, ahead = 4, stride = 36; // floats to a row of LDS: rows start in different groups of banks
    __shared__ float lds[4][32 * stride];
    const uint32_t live = min(p.M, p.rows.live()), nt = (p.N + 31) / 32;
    const uint32_t number = block_number(), m0 = number / nt * 32, n0 = number % nt * 32;
    if (m0 >= live) return;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    Along<T> a, b;
    a.row = static_cast<const T *>(p.a.p) + min(m0 + (lane & 31), live - 1) * p.a.ld;
    b.row = static_cast<const T *>(p.b.p) + min(n0 + (lane & 31), p.N - 1) * p.b.ld;
    a.k_end = b.k_end = p.K;
    const uint32_t row = threadIdx.x >> 2, group = threadIdx.x & 3; // of the lanes that hand the sums over
    const Columns c = columns_of(p.e, n0 + 8 * group, p.N);
    Needs<AnyType, 1> needs;
    if (row < 32) needs.ask(p.e, c.n, c.left, m0 + row, 1, live);
    f32x16 acc = {};
    for (uint32_t k0 = wave * 2 * K; k0 < p.K; k0 += ahead * 8 * K) {
        u32x4 x[ahead], y[ahead];
#pragma unroll
        for (int i = 0; i < ahead; ++i) {
            const uint32_t k = k0 + i * 8 * K + half * K;
            x[i] = a.at(k);
            y[i] = b.at(k);
        }
#pragma unroll
        for (int i = 0; i < ahead; ++i) multiply(T(), y[i], x[i], acc);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4 *>(&lds[wave][(lane & 31) * stride + 8 * q + 4 * half]) = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    __syncthreads();
    if (row >= 32 || c.left <= 0) return;
    finish(p.e, c, needs, m0 + row, 1, live, [&](int, float(&v)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += lds[w][row * stride + 8 * group + j];
    });
}

// The sum over the parts, and what happens to it (16 parts of 1024 x 1024: 19 us, 3.5 TB/s; 256 of 256 x 200: 12 us): eight groups of eight cells to a workgroup, every 32nd part to a lane, then the lanes in order.
struct JoinArgs {
    const float *part;
    uint32_t M, N, splits;
    Epilogue e;
};

__global__ __launch_bounds__(256) void k_join(JoinArgs p)
{
    __shared__ float lds[32][8][8 + 1];
    const uint32_t groups = (p.N + 7) / 8, g = threadIdx.x & 7, lane = threadIdx.x >> 3;
    const uint64_t i = block_number() * 8ull + g, cells = (uint64_t)p.M * p.N;
    const bool there = i < (uint64_t)p.M * groups;
    const uint32_t m = there ? (uint32_t)(i / groups) : 0u, n = there ? (uint32_t)(i % groups) * 8 : 0u;
    float v[8] = {};
    if (there)
        for (uint32_t s = lane; s < p.splits; s += 32) {
            float w[8];
            load8(p.part + s * cells + (uint64_t)m * p.N + n, (int)(p.N - n), w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += w[j];
        }
#pragma unroll
    for (int j = 0; j < 8; ++j) lds[lane][g][j] = v[j];
    __syncthreads();
    if (lane || !there) return;
    const Columns c = columns_of(p.e, n, p.N);
    Needs<AnyType, 1> needs;
    needs.ask(p.e, c.n, c.left, m, 1, p.M);
    finish(p.e, c, needs, m, 1, p.M, [&](int, float(&sum)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
        for (uint32_t s = 0; s < min(p.splits, 32u); ++s)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += lds[s][g][j];
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

constexpr int kTile = 128, kTileM = 256, kTileN = 128; // of operands that lie anyhow, and of those in chunks

template <int BM, int BN> uint64_t tile_blocks(const ProductArgs &p)
{
    const uint64_t tiles = (uint64_t)((p.M + BM - 1) / BM) * ((p.N + BN - 1) / BN) * p.splits;
    return (tiles + 7) / 8 * 8;
}

template <int BM, int BN> dim3 tile_grid(const ProductArgs &p) { return grid_of(tile_blocks<BM, BN>(p)); }

// Whether an operand's rows start on 16-byte boundaries, are whole chunks long, and near enough to each other.
template <class T> bool in_chunks(const Operand &o, uint32_t rows, uint32_t K)
{
    constexpr int tile = 256; // the largest there is
    const uint64_t ld = (uint64_t)o.ld * sizeof(T), along = (uint64_t)(o.turned ? rows : K) * sizeof(T);
    const uint64_t span = o.turned ? ld * (128 / sizeof(T)) + tile * sizeof(T) : ld * tile + 128;
    return reinterpret_cast<uintptr_t>(o.p) % 16 == 0 && ld % 16 == 0 && along % 16 == 0 && span < kReach;
}

// Whether cells of 32 x 32 (k_few) take less time than large tiles, both as measured on an MI355X.  A large tile alone takes 9 us and 0.5 us
// for 64 bytes of k (fp32: 2 us, its instructions' own time; 8 bits, widened: 0.8), 512 of them at a time; k_few 3 us, 1.65 us for a million chunks out of the
// caches (twice that where rows start anywhere) and 1.3 us for a thousand workgroups.  bf16, large tiles / k_few: 1 x 256 x 512 8.1 / 3.0 us,
// 256 x 2048 x 512 40 / 9.7, 4096 x 256 x 256 13.6 / 6.6, 8192 x 256 x 256 13.8 / 11.7, 16384 x 256 x 256 14.7 / 20, 131072 x 64 x 64
// 14.5 / 22; rows of 602 bytes, 32768 x 301 x 47, 13.7 / 22.6; fp32 1024 x 1024 x 1024 135 / 41, 262144 x 128 x 32 84 / 45.
template <class T> bool few_tiles(const ProductArgs &p, bool chunks)
{
    using F = std::conditional_t<std::is_same_v<T, uint8_t>, Widened8, T>;
    if (p.splits > 1 || p.a.turned || p.b.turned) return false;
    const double tiles = std::ceil(p.M / (double)kTileM) * std::ceil(p.N / (double)kTileN), steps = std::ceil(p.K * sizeof(T) / 64.0);
    const double large = (9.0 + (std::is_same_v<T, float> ? 2.0 : sizeof(T) == 1 ? 0.8 : 0.5) * steps) * std::max(1.0, tiles / 512.0);
    const double blocks = std::ceil(p.M / 32.0) * std::ceil(p.N / 32.0), read = blocks * 64.0 * p.K / chunk_k<F>;
    const double few = 3.0 + (chunks ? 1.65e-6 : 3.3e-6) * read + 1.3e-3 * blocks;
    return few < large;
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
    const uint64_t groups = (uint64_t)p.M * ((p.N + 7) / 8);
    return launch(st, k_join, grid_of((groups + 7) / 8), 256, JoinArgs{part, p.M, p.N, p.splits, p.e});
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
        p.a = {a->d_A, a->ld_A, false};
        p.b = {a->d_W, a->ld_W, false};
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
