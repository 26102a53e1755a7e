// What the dense operators share: types and their wide accesses, the dropout mask, activations, argument checks, launches.
#pragma once

#include "zg_internal.h"

#include <cmath>
#include <cstring>
#include <initializer_list>
#include <tuple>

namespace zg {

// ---- host side ------------------------------------------------------------------------------------------------------------------

constexpr int64_t kMaxRows = 0x7FFFFFFF;

inline size_t type_size(int32_t t) { return t == ZG_F32 ? 4 : t == ZG_F16 || t == ZG_BF16 ? 2 : t == ZG_F8 ? 1 : 0; }
inline bool wide_type(int32_t t) { return t == ZG_F32 || t == ZG_F16 || t == ZG_BF16; }

// Nothing of C++ leaves a C entry point.
template <class F> int entry(F &&body) noexcept
{
    try {
        return body();
    } catch (...) {
        return ZG_ENOMEM; // (the only thing that can throw is a message's string)
    }
}

template <class... P, class... A> int launch_lds(hipStream_t st, void (*kernel)(P...), dim3 grid, unsigned block, size_t lds, const A &...given)
{
    if (grid.x == 0 || grid.y == 0 || grid.z == 0) return ZG_OK;
    std::tuple<P...> a{given...};
    void *args[sizeof...(P)];
    std::apply([&](auto &...v) { int i = 0; ((args[i++] = const_cast<void *>(static_cast<const void *>(&v))), ...); }, a);
    // (what the launch returned, and not hipGetLastError: that may be an earlier error of the caller's own)
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, dim3(block), args, lds, st);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        return fail(ZG_EHIP, std::string("hipLaunchKernel: ") + hipGetErrorString(e));
    }
    return ZG_OK;
}

template <class... P, class... A> int launch(hipStream_t st, void (*kernel)(P...), dim3 grid, unsigned block, const A &...given)
{
    return launch_lds(st, kernel, grid, block, 0, given...);
}

// A launch's lanes in one dimension number less than 2^32: beyond 2^21 workgroups the grid has a second one (with workgroups to spare, which
// find no rows).
inline dim3 grid_of(uint64_t blocks)
{
    constexpr uint64_t most = 1 << 21;
    return blocks <= most ? dim3((unsigned)blocks) : dim3((unsigned)most, (unsigned)((blocks + most - 1) / most));
}

inline int check_rows(int64_t rows)
{
    return rows < 0 || rows > kMaxRows ? fail(ZG_EINVAL, "rows outside 0..2^31-1") : ZG_OK;
}

inline int check_width(int32_t width, int32_t most = ZG_MAX_WIDTH)
{
    return width < 1 || width > most ? fail(ZG_EINVAL, "a width outside 1.." + std::to_string(most)) : ZG_OK;
}

inline int check_matrix(const char *what, const void *p, int64_t ld, int32_t width, int32_t type)
{
    if (!p) return fail(ZG_EINVAL, std::string(what) + " is null");
    if (ld < width || ld > (int64_t(1) << 40)) return fail(ZG_EINVAL, std::string("the row stride of ") + what + " is below its width, or above 2^40");
    if (reinterpret_cast<uintptr_t>(p) % type_size(type)) return fail(ZG_EINVAL, std::string(what) + " is not aligned to its elements");
    return ZG_OK;
}

// fp32 and int32 vectors
inline int check_vector(const char *what, const void *p)
{
    return reinterpret_cast<uintptr_t>(p) % 4 ? fail(ZG_EINVAL, std::string(what) + " is not aligned to its elements") : ZG_OK;
}

inline int check_drop(const zg_drop &d)
{
    if (!(d.p >= 0.0 && d.p <= 1.0)) return fail(ZG_EINVAL, "the dropout probability is outside 0..1");
    return check_vector("the dropout's d_ids", d.d_ids);
}

inline int check_workspace(const void *p, size_t have, size_t need)
{
    if (need == 0) return ZG_OK;
    if (!p || reinterpret_cast<uintptr_t>(p) % 256) return fail(ZG_EINVAL, "the workspace is null or not 256-byte aligned");
    return have < need ? fail(ZG_ENOMEM, "the workspace is smaller than the call needs") : ZG_OK;
}

// ---- what lies where ------------------------------------------------------------------------------------------------------------
// Workgroups read and write in no order, so what a call writes must not lie on what it reads; a cell that one lane reads and then writes may be
// the same one.

struct Span {
    const char *what;
    const void *p; // null: nothing is there
    int64_t rows, pitch, width; // bytes from row to row, bytes of a row
    int32_t size;               // of an element
};

inline Span matrix_span(const char *what, const void *p, int64_t rows, int64_t ld, int64_t cols, int32_t type)
{
    const int32_t size = (int32_t)type_size(type);
    return {what, p, rows, rows > 1 ? ld * size : cols * size, cols * size, size};
}

inline Span vector_span(const char *what, const void *p, int64_t n) { return {what, p, 1, n * 4, n * 4, 4}; }

// Whether a byte of `a` is one of `b`.  Where the rows are not equally far apart and only their ranges meet, the caller's word is taken unless the
// first rows meet.
inline bool meet(const Span &a, const Span &b)
{
    if (!a.p || !b.p || a.rows == 0 || b.rows == 0) return false;
    const __int128 d = (__int128) reinterpret_cast<uintptr_t>(b.p) - (__int128) reinterpret_cast<uintptr_t>(a.p); // from a's first byte to b's
    const auto reach = [](const Span &s) { return (__int128)(s.rows - 1) * s.pitch + s.width; };
    if (d >= reach(a) || -d >= reach(b)) return false;
    if (a.rows > 1 && b.rows > 1 && a.pitch != b.pitch) return d < a.width && -d < b.width;
    const __int128 pitch = a.rows > 1 ? a.pitch : b.pitch;
    if (a.rows == 1 && b.rows == 1) return true;
    // row i of a and row i + m of b: m such that b's begins less than a row's width in front of a's, or behind it
    __int128 q = d / pitch;
    if (d % pitch < 0) --q;
    const __int128 behind = d - q * pitch; // of b's first row, from the beginning of row q of a
    const auto rows_meet = [&](__int128 m) { return m <= b.rows - 1 && -m <= a.rows - 1; };
    return (behind < a.width && rows_meet(-q)) || (pitch - behind < b.width && rows_meet(-q - 1));
}

inline bool same_cells(const Span &a, const Span &b) { return a.p == b.p && a.pitch == b.pitch && a.width == b.width && a.size == b.size; }

// `out` lies on none of the first list and, unless cell on cell, on none of the second
inline int check_apart(const Span &out, std::initializer_list<Span> apart, std::initializer_list<Span> apart_or_same = {})
{
    for (const Span &s : apart)
        if (meet(out, s)) return fail(ZG_EINVAL, std::string(out.what) + " lies on " + s.what);
    for (const Span &s : apart_or_same)
        if (meet(out, s) && !same_cells(out, s)) return fail(ZG_EINVAL, std::string(out.what) + " lies on " + s.what + " and is not the same matrix");
    return ZG_OK;
}

inline Span ids_span(const zg_drop &d, int64_t rows) { return vector_span("the dropout's d_ids", d.p > 0.0 ? d.d_ids : nullptr, rows); }
inline Span rows_span(const uint32_t *d_rows) { return vector_span("d_rows", d_rows, 1); }

#define ZG_TRY(call)                                                                                         \
    do {                                                                                                     \
        const int s_ = (call);                                                                               \
        if (s_ != ZG_OK) return s_;                                                                          \
    } while (0)

// ---- the dropout mask -----------------------------------------------------------------------------------------------------------

struct Drop {
    uint32_t cut; // a cell is dropped where its 16 bits are below this; 0: no dropout
    float scale;  // 65536 / (65536 - cut)
    uint32_t key_lo, key_hi, layer;
    const int32_t *ids;
};

inline Drop make_drop(const zg_drop &d)
{
    Drop r{};
    r.cut = (uint32_t)std::floor(d.p * 65536.0 + 0.5);
    r.scale = r.cut < 65536u ? (float)(65536.0 / (65536.0 - r.cut)) : 0.0f;
    r.key_lo = (uint32_t)d.key;
    r.key_hi = (uint32_t)(d.key >> 32);
    r.layer = d.layer;
    r.ids = d.d_ids;
    return r;
}

struct Rows {
    const uint32_t *d_rows;
    uint32_t cap;
    __device__ __forceinline__ uint32_t live() const { return d_rows ? min(*d_rows, cap) : cap; }
};

#ifdef __HIPCC__

// this workgroup's number in a grid_of()
__device__ __forceinline__ uint32_t block_number() { return blockIdx.y * gridDim.x + blockIdx.x; }

__device__ __forceinline__ uint64_t mask_product(uint32_t a, uint32_t b)
{
    uint64_t p;
    asm("v_mad_u64_u32 %0, vcc, %1, %2, 0" : "=v"(p) : "v"(a), "s"(b) : "vcc");
    return p;
}

// Philox4x32-10 (Salmon et al., SC'11) with counter (id, group, layer, 1): the 16 bits of the eight cells 8 group .. 8 group + 7 of a row, two to
// a word.  20 whole products and 20 three-way xors.
__device__ __forceinline__ void mask_bits(const Drop &d, uint32_t id, uint32_t group, uint32_t (&w)[4])
{
    uint32_t c0 = id, c1 = group, c2 = d.layer, c3 = 1u, k0 = d.key_lo, k1 = d.key_hi;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = mask_product(c0, 0xD2511F53u);
        const uint64_t p1 = r == 0 ? (uint64_t)0xCD9E8D57u * c2 : mask_product(c2, 0xCD9E8D57u); // (the first one is the layer's: a scalar)
        c0 = __builtin_amdgcn_bitop3_b32((uint32_t)(p1 >> 32), c1, k0, 0x96);
        c1 = (uint32_t)p1;
        c2 = __builtin_amdgcn_bitop3_b32((uint32_t)(p0 >> 32), c3, k1, 0x96);
        c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    w[0] = c0, w[1] = c1, w[2] = c2, w[3] = c3;
}

__device__ __forceinline__ bool mask_keeps(const Drop &d, const uint32_t (&w)[4], int cell)
{
    return (cell & 1 ? w[cell >> 1] >> 16 : w[cell >> 1] & 0xFFFFu) >= d.cut;
}

__device__ __forceinline__ uint32_t mask_id(const Drop &d, uint32_t row) { return d.ids ? (uint32_t)d.ids[row] : row; }

// eight cells of a row at column 8 group: dropped ones become 0 whatever they are, the others are multiplied by `scale`
__device__ __forceinline__ void mask8(const Drop &d, uint32_t id, uint32_t group, float scale, float (&v)[8])
{
    uint32_t w[4];
    mask_bits(d, id, group, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = mask_keeps(d, w, i) ? v[i] * scale : 0.0f;
}

// ---- eight consecutive elements -------------------------------------------------------------------------------------------------
// Rows may start at any element: wide accesses at any alignment are what global memory on this chip takes.

template <class T> __device__ __forceinline__ void load8(const T *p, float (&v)[8])
{
    T t[8];
    __builtin_memcpy(t, p, sizeof t);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)t[i];
}

// the first `n` of eight elements; 0 for the others
template <class T> __device__ __forceinline__ void load8(const T *p, int n, float (&v)[8])
{
    if (n >= 8) {
        load8(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)p[i] : 0.0f;
    }
}

// 16 bytes past the caches, at any alignment
typedef uint32_t u32x4_anywhere __attribute__((ext_vector_type(4), aligned(1)));

// Results above this size go past the caches (the eight L2s hold 32 MB): norm of 120001 x 1024 bf16 209 -> 161 us, dropout of 285127 x 512
// 129 -> 102 us (each timed alone, nobody reading the result behind it).
constexpr int64_t kStreamBytes = 32 << 20;

template <class T> __device__ __forceinline__ void store8(T *p, int n, const float (&v)[8], bool stream = false)
{
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (T)v[i];
    if (n >= 8) {
        if (stream) {
            u32x4_anywhere w[sizeof t / 16];
            __builtin_memcpy(w, t, sizeof t);
#pragma unroll
            for (unsigned i = 0; i < sizeof t / 16; ++i) __builtin_nontemporal_store(w[i], reinterpret_cast<u32x4_anywhere *>(p) + i);
        } else {
            __builtin_memcpy(p, t, sizeof t);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = t[i];
    }
}

// of a type that is known at run time (ZG_F32, ZG_F16 or ZG_BF16), at element `at`
__device__ __forceinline__ void load8(const void *p, int32_t type, int64_t at, int n, float (&v)[8])
{
    if (type == ZG_F32) load8(static_cast<const float *>(p) + at, n, v);
    else if (type == ZG_F16) load8(static_cast<const _Float16 *>(p) + at, n, v);
    else load8(static_cast<const __bf16 *>(p) + at, n, v);
}

__device__ __forceinline__ void store8(void *p, int32_t type, int64_t at, int n, const float (&v)[8], bool stream = false)
{
    if (type == ZG_F32) store8(static_cast<float *>(p) + at, n, v, stream);
    else if (type == ZG_F16) store8(static_cast<_Float16 *>(p) + at, n, v, stream);
    else store8(static_cast<__bf16 *>(p) + at, n, v, stream);
}

// ---- activations, fp32 ----------------------------------------------------------------------------------------------------------
// PRECISE, where the result is fp32: right to a few units in the last place of each value, and to z^2 / 2 of them in the normal distribution's
// tails.  Otherwise, where the result is rounded to 16 bits: exp(x) as 2^(x log2 e) in one instruction, off by |x| 2^-24 of itself, 1 / x in another,
// and an erf of 1.5e-7.

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// exp(x + rest), |x| <= 150 and rest of x's rounding: what the power's own rounding leaves out goes into a factor
__device__ __forceinline__ float exp_precise(float x, float rest = 0.0f)
{
    constexpr float high = 1.4426950216293335f, low = 1.925963033500011e-8f; // log2 e
    const float power = x * high, left = fmaf(rest, high, fmaf(x, low, fmaf(x, high, -power)));
    return __builtin_amdgcn_exp2f(power) * fmaf(left, 0.69314718f, 1.0f);
}

template <bool PRECISE> __device__ __forceinline__ float sigmoid(float z)
{
    if (!PRECISE) return __builtin_amdgcn_rcpf(1.0f + exp_of(-z));
    return __builtin_amdgcn_rcpf(1.0f + exp_precise(__builtin_amdgcn_fmed3f(-z, -150.0f, 150.0f)));
}

// The normal distribution function and the factor exp(-z^2 / 2) in it.  With x = |z|, its tail is that factor times erfcx(x / sqrt 2) / 2, a polynomial in
// u = c x / (1 + c x), c = 0.34, fitted up to x = 14.5 to 2e-8 of itself (u is 0 where x is, so that its rounding does not count there; beyond 14.5
// the tail is 0 in fp32).
__device__ __forceinline__ float normal_cdf_precise(float z, float &bell)
{
    const float x = fminf(fabsf(z), 14.5f), u = 0.34f * x * __builtin_amdgcn_rcpf(fmaf(0.34f, x, 1.0f)), square = x * x;
    bell = exp_precise(-0.5f * square, -0.5f * fmaf(x, x, -square));
    float s = 0.0281659849f;
    s = fmaf(s, u, -0.103897132f);
    s = fmaf(s, u, 0.11172124f);
    s = fmaf(s, u, -0.0112492209f);
    s = fmaf(s, u, 0.0540692918f);
    s = fmaf(s, u, -0.163854495f);
    s = fmaf(s, u, -0.230821952f);
    s = fmaf(s, u, 0.989227057f);
    s = fmaf(s, u, -1.17335868f);
    s = fmaf(s, u, 0.5f);
    const float tail = s * bell;
    return z < 0.0f ? tail : 1.0f - tail;
}

// For 16-bit results: erf by Abramowitz and Stegun 7.1.26 (a polynomial in 1 / (1 + p x) times exp(-x^2)), half the instructions of the one above.
// z times it is off by 4e-6 of itself for z > -2, 5e-4 from z = -4 on and 4e-3 from -6 on, where it is 6e-9, against 2^-9 and 2^-12 for the
// rounding to 16 bits (and 3e-8, where fp16 ends).
__device__ __forceinline__ float normal_cdf(float z)
{
    const float x = fabsf(z) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.0f));
    const float bell = exp_of(-x * x);
    float s = fmaf(1.061405429f, t, -1.453152027f);
    s = fmaf(s, t, 1.421413741f);
    s = fmaf(s, t, -0.284496736f);
    s = fmaf(s, t, 0.254829592f);
    const float tail = 0.5f * s * t * bell; // (1 - erf(x)) / 2
    return z < 0.0f ? tail : 1.0f - tail;
}

template <bool PRECISE> __device__ __forceinline__ float act_of(int act, float z)
{
    if (act == ZG_ACT_RELU) return z > 0.0f ? z : z != z ? z : 0.0f; // (not a number stays that)
    if (act == ZG_ACT_SILU) return z * sigmoid<PRECISE>(z);
    if (act == ZG_ACT_GELU) {
        float bell;
        return z * (PRECISE ? normal_cdf_precise(z, bell) : normal_cdf(z));
    }
    return z;
}

// precise: a bias' gradient, the sum of slopes, is fp32 whatever the operands are
__device__ __forceinline__ float act_slope(int act, float z)
{
    if (act == ZG_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (act == ZG_ACT_SILU) {
        const float g = sigmoid<true>(z);
        return g * fmaf(z, 1.0f - g, 1.0f);
    }
    if (act == ZG_ACT_GELU) {
        float bell;
        const float c = normal_cdf_precise(z, bell);
        return fmaf(z * bell, 0.39894228040143268f, c);
    }
    return 1.0f;
}

#endif

} // namespace zg
