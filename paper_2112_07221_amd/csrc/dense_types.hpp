// What the dense layers' kernels share: element types, pieces of 16 bytes and less at any alignment, activations and the 8-bit form of
// activations (gfx950, wave64).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace het {

using bf16 = __bf16;
using f16 = _Float16;

template <typename T, int N> using vec = T __attribute__((ext_vector_type(N)));

using f32x4 = vec<float, 4>;
using f32x8 = vec<float, 8>;
using f32x16 = vec<float, 16>;
using i32x4 = vec<int32_t, 4>;

constexpr int CHUNK = 8;             // elements a lane handles at a time in the row-wise kernels
constexpr int PACK_BLOCK = 32;       // values that share a step in the 8-bit form
constexpr uint32_t PACK_NOT_FINITE = 255;

// Which of a row's `per` pieces thread `i` of a launch of a piece a thread has.  (A division of 64 bits is some eighty instructions.)
__device__ __forceinline__ void row_and_piece(int64_t i, int per, int64_t &row, int &piece)
{
    if ((uint64_t)i >> 32) { row = i / per; piece = (int)(i - row * per); }
    else { row = (uint32_t)i / (uint32_t)per; piece = (int)((uint32_t)i - (uint32_t)row * (uint32_t)per); }
}

// ---- pieces of rows at any alignment ------------------------------------------------------------------
// Rows may begin at any element (odd widths, wider matrices), and the vector memory path takes any address: a piece is one load
// of 16 bytes (two for fp32) whatever its alignment, and no second set of kernels is needed for odd strides.

template <typename T>
__device__ __forceinline__ f32x8 load_chunk(const T *p)
{
    vec<T, 8> v;
    __builtin_memcpy(&v, p, sizeof(v));
    return __builtin_convertvector(v, f32x8);
}

template <typename T>
__device__ __forceinline__ void store_chunk(T *p, f32x8 f)
{
    const vec<T, 8> v = __builtin_convertvector(f, vec<T, 8>);
    __builtin_memcpy(p, &v, sizeof(v));
}

// 16 bytes that are not kept in the L2.
template <typename V>
__device__ __forceinline__ void store_past(void *p, V v)
{
    typedef int32_t any16 __attribute__((ext_vector_type(4), aligned(2)));
    static_assert(sizeof(V) == 16, "a piece");
    __builtin_nontemporal_store(__builtin_bit_cast(i32x4, v), static_cast<any16 *>(p));
}
template <typename V>
__device__ __forceinline__ V load_past(const void *p)
{
    typedef int32_t any16 __attribute__((ext_vector_type(4), aligned(2)));
    static_assert(sizeof(V) == 16, "a piece");
    return __builtin_bit_cast(V, __builtin_nontemporal_load(static_cast<const any16 *>(p)));
}

// The first `n` (0 .. 8) of a chunk; the others read as zero and are not written.
template <typename T>
__device__ __forceinline__ f32x8 load_some(const T *p, int n)
{
    if (n >= CHUNK) return load_chunk(p);
    f32x8 f = {};
#pragma unroll
    for (int j = 0; j < CHUNK - 1; ++j) if (j < n) f[j] = (float)p[j];
    return f;
}

template <typename T>
__device__ __forceinline__ void store_some(T *p, f32x8 f, int n)
{
    if (n >= CHUNK) { store_chunk(p, f); return; }
#pragma unroll
    for (int j = 0; j < CHUNK - 1; ++j) if (j < n) p[j] = (T)f[j];
}

// Chunk c of a row of `dim` values, loaded without a branch that lanes take differently, so that the loads of all chunks are under way together.
// WHOLE: rows are whole chunks; a chunk behind the end is zero.  Otherwise the chunk that would cross the end is the row's last eight values, of which the
// first chunk_skip are the chunk before's: they read as zero and are not written.  (Value j of a chunk is column chunk_from + j for all
// that is loaded, whatever its type, so nothing is shifted: 30000 x 300 forward 23 -> 16, backward 38 -> 30 us.)  A row of less than a chunk is its first chunk's first values.
__device__ __forceinline__ int chunk_from(int c, int dim)
{
    const int last = dim < CHUNK ? 0 : dim - CHUNK;
    return min(c * CHUNK, last);
}
__device__ __forceinline__ int chunk_skip(int c, int dim) { return c * CHUNK - chunk_from(c, dim); }
// Whether value j of chunk c is one of its own.
template <bool WHOLE>
__device__ __forceinline__ bool chunk_has(int c, int j, int dim)
{
    if (WHOLE) return c * CHUNK < dim;
    return dim < CHUNK ? c == 0 && j < dim : j >= chunk_skip(c, dim);
}

template <bool WHOLE>
__device__ __forceinline__ f32x8 chunk_only(f32x8 f, int c, int dim)       // zero for the others
{
    if (WHOLE) return c * CHUNK < dim ? f : f32x8{};
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = chunk_has<WHOLE>(c, j, dim) ? f[j] : 0.f;
    return f;
}

template <bool WHOLE, typename T>
__device__ __forceinline__ vec<T, 8> load_raw(const T *row, int c, int dim)
{
    vec<T, 8> v = {};
    if (!WHOLE && dim < CHUNK) {
#pragma unroll
        for (int j = 0; j < CHUNK - 1; ++j) if (j < dim) v[j] = row[j];
        return v;
    }
    __builtin_memcpy(&v, row + chunk_from(c, dim), sizeof(v));
    return v;
}
template <bool WHOLE, typename T>
__device__ __forceinline__ f32x8 raw_values(vec<T, 8> v, int c, int dim)
{
    return chunk_only<WHOLE>(__builtin_convertvector(v, f32x8), c, dim);
}
template <bool WHOLE, typename T>
__device__ __forceinline__ f32x8 load_row(const T *row, int c, int dim) { return raw_values<WHOLE>(load_raw<WHOLE>(row, c, dim), c, dim); }
template <bool WHOLE, bool PAST = false, typename T>
__device__ __forceinline__ void store_row(T *row, int c, int dim, f32x8 f)
{
    const int n = dim - c * CHUNK;
    if (WHOLE ? n > 0 : n >= CHUNK) {
        if constexpr (PAST && sizeof(T) == 2) store_past(row + c * CHUNK, __builtin_convertvector(f, vec<T, 8>));
        else store_chunk(row + c * CHUNK, f);
        return;
    }
    if (WHOLE || n <= 0) return;
    T *at = row + chunk_from(c, dim);
#pragma unroll
    for (int j = 0; j < 8; ++j) if (chunk_has<WHOLE>(c, j, dim)) at[j] = (T)f[j];
}
// The chunk's own values from its first place on, zero behind them.
template <bool WHOLE>
__device__ __forceinline__ f32x8 chunk_own(f32x8 f, int c, int dim)
{
    if (WHOLE || dim < CHUNK) return f;
    const int over = chunk_skip(c, dim);
    if (over >= CHUNK) return f32x8{};
#pragma unroll
    for (int by = 4; by >= 1; by /= 2)
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = over & by ? (j + by < 8 ? f[j + by] : 0.f) : f[j];
    return f;
}

// ---- activations --------------------------------------------------------------------------------------
enum { DENSE_ACT_NONE = 0, DENSE_ACT_RELU = 1, DENSE_ACT_GELU = 2, DENSE_ACT_SILU = 3 };

__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * 1.4426950408889634f); }

// Phi(-|v|), the normal distribution's smaller tail: its logarithm is -v^2 / 2 and a slow function of |v|, for which stands a polynomial of degree 12 (a fit of
// log2(Phi(-x)) + x^2 / 2 log2(e) on [0, 8], by the largest error of x Phi(-x) and a hundredth of its relative one).  The tail is formed itself, not as 1 - erf, which has
// no digits left from v = -5.5 on: x Phi(-x) is off by 4.1e-9 and by 6e-7 of itself up to 8, and by fp32's roundings, 2^-24 times 10 + 3 x^2 + 1.5 2^x of itself at
// most; beyond 8, where it is below 5e-15, the polynomial stays where it is (1.6 %).  In fp32 z Phi(z) is no further from 64 bits than 0.5 z (1 + erf(z / sqrt(2)))
// (root mean square over [-1, 0] 8.2e-9, [-2, -1] 1e-8, [-3, -2] 3.9e-9 against 8.8e-9, 1.9e-8, 2.3e-8).
// Twelve multiply-adds and one exponential: 8192 x 4096 values in bf16, their slopes from z in 8 bits with the bias' gradient 37.0 us (degree 6, whose tail is 6e-4 of itself off at
// -4 and 6e-3 at -5, 35.2; memory's share 31), expanded through gelu 24.9 (21.6); 4096 x 1664 -> 4096 with gelu and z in 8 bits 60.7 (59.1).
__device__ __forceinline__ float normal_tail(float v, float x)           // x: |v|, at most 8
{
    float q = -1.1824052847941857e-10f;
    q = fmaf(q, x, 6.13685413597409e-09f);
    q = fmaf(q, x, -1.416807577925283e-07f);
    q = fmaf(q, x, 1.914204176500789e-06f);
    q = fmaf(q, x, -1.6654646969982423e-05f);
    q = fmaf(q, x, 9.487954230280593e-05f);
    q = fmaf(q, x, -0.0003152537683490664f);
    q = fmaf(q, x, 3.84772865800187e-05f);
    q = fmaf(q, x, 0.006927822716534138f);
    q = fmaf(q, x, -0.05244092270731926f);
    q = fmaf(q, x, 0.2621293067932129f);
    q = fmaf(q, x, -1.1511046886444092f);
    q = fmaf(q, x, -1.0f);
    return __builtin_amdgcn_exp2f(fmaf(v * -0.72134752044448170f, v, q));
}
__device__ __forceinline__ float within_eight(float v) { return __builtin_amdgcn_fmed3f(fabsf(v), 0.f, 8.f); }

__device__ __forceinline__ float act_value(int act, float v)
{
    switch (act) {
    case DENSE_ACT_RELU: return v > 0.f ? v : v == v ? 0.f : v;                       // NaN stays NaN
    case DENSE_ACT_GELU: { const float x = within_eight(v); return fmaf(-x, normal_tail(v, x), fmaxf(v, 0.f)); }      // (8 times the tail of what is beyond)
    case DENSE_ACT_SILU: return v * __builtin_amdgcn_rcpf(1.f + exp_of(-v));
    default: return v;
    }
}

// A sum beyond a 16-bit type's range is kept as an infinity: its slope is the limit, 0 or 1.  So the factor of what vanishes there is held within a range beyond
// which it has vanished in fp32 (infinity times 0 is a NaN); a NaN stays one by the other factors.
__device__ __forceinline__ float act_slope(int act, float v)
{
    switch (act) {
    case DENSE_ACT_RELU: return v > 0.f ? 1.f : v == v ? 0.f : v;
    case DENSE_ACT_GELU: {
        const float tail = normal_tail(v, within_eight(v)), bell = __builtin_amdgcn_exp2f(v * -0.72134752044448170f * v);
        return fmaf(__builtin_amdgcn_fmed3f(v, -16.f, 16.f) * 0.39894228040143268f, bell, v < 0.f ? tail : 1.f - tail);
    }
    case DENSE_ACT_SILU: { const float p = __builtin_amdgcn_rcpf(1.f + exp_of(-v)); return p * (1.f + __builtin_amdgcn_fmed3f(v, -128.f, 128.f) * (1.f - p)); }
    default: return 1.f;
    }
}

// The same for a chunk: one decision for its values.
template <bool SLOPE>
__device__ __forceinline__ f32x8 act_chunk(int act, f32x8 v)
{
#define HET_EACH(A) { for (int j = 0; j < 8; ++j) v[j] = SLOPE ? act_slope(A, v[j]) : act_value(A, v[j]); break; }
    switch (act) {
    case DENSE_ACT_RELU: HET_EACH(DENSE_ACT_RELU)
    case DENSE_ACT_GELU: HET_EACH(DENSE_ACT_GELU)
    case DENSE_ACT_SILU: HET_EACH(DENSE_ACT_SILU)
    default: if (SLOPE) HET_EACH(DENSE_ACT_NONE) break;
    }
#undef HET_EACH
    return v;
}

// ---- the 8-bit form -----------------------------------------------------------------------------------
// A block of 32 values along a row shares a step 2^e; a value is q steps, q whole in [-127, 127] (ties to even).  e is the smallest
// for which the block's largest magnitude rounds to at most 127 steps, so a value is off by at most half a step, 1/127 of that
// magnitude.  The step is a power of two because q 2^e then fits bf16's 8 significant bits: the matrix instructions of the backward
// pass take exactly what was kept.  e is held as the byte e + 127, the exponent field of the float 2^e.  A block with an infinity or a
// NaN has the byte 255 and reads as NaN everywhere: what overflowed is not taken for a number later on.

// Largest magnitude as the bits of a float: as whole numbers they are in the order of the magnitudes, with NaN above infinity.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

struct PackStep {
    uint32_t byte;       // what is stored
    uint32_t finite;     // all ones, or zero
    float inverse;       // 2^-e
};

// most_bits: magnitude() of the block's largest value.  A significand of 127.5 / 64 and above rounds to 128 steps: adding 2^16 (its distance
// from 2) carries into the exponent exactly then.
__device__ __forceinline__ PackStep pack_step(uint32_t most_bits)
{
    PackStep s;
    int e = (int)((most_bits + 0x10000u) >> 23) - 133;
    e = e < -126 ? -126 : e > 122 ? 122 : e;
    s.finite = most_bits < 0x7F800000u ? ~0u : 0u;
    s.byte = s.finite ? (uint32_t)(e + 127) : PACK_NOT_FINITE;
    s.inverse = __uint_as_float((uint32_t)(127 - e) << 23);
    return s;
}

// Four values as bytes.  Adding 3 2^22 leaves the whole number, rounded to even, in the float's low bits: one multiply-add a value and three byte
// permutations for four.  The step is such that no value is beyond 127 of it; at the top of the range alone it is held below 64
// (64 steps of 2^122 would be no float any more).
__device__ __forceinline__ uint32_t pack_four(float a, float b, float c, float d, const PackStep &s)
{
    if (s.byte == 249u) {
        const float most = 63.f / s.inverse;
        a = fminf(fmaxf(a, -most), most); b = fminf(fmaxf(b, -most), most); c = fminf(fmaxf(c, -most), most); d = fminf(fmaxf(d, -most), most);
    }
    const uint32_t p = __float_as_uint(fmaf(a, s.inverse, 12582912.f)), q = __float_as_uint(fmaf(b, s.inverse, 12582912.f));
    const uint32_t r = __float_as_uint(fmaf(c, s.inverse, 12582912.f)), t = __float_as_uint(fmaf(d, s.inverse, 12582912.f));
    return (__builtin_amdgcn_perm(q, p, 0x0C0C0400u) | __builtin_amdgcn_perm(t, r, 0x04000C0Cu)) & s.finite;
}

// 2^e of a stored byte; 255 gives infinity, and 0 times that the NaN the block stands for.
__device__ __forceinline__ float pack_step_of(uint32_t byte) { return __uint_as_float(byte << 23); }

__device__ __forceinline__ f32x8 unpack_chunk(uint64_t q, uint32_t byte)
{
    const float step = pack_step_of(byte);
    f32x8 f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (float)(int8_t)(q >> (8 * j)) * step;
    return f;
}

// The magnitude over the four lanes (aligned) that hold a block of 32 values, eight each.
__device__ __forceinline__ uint32_t quad_max(uint32_t v)
{
    uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false);       // lanes 1 0 3 2
    v = v > o ? v : o;
    o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false);                // lanes 2 3 0 1
    return v > o ? v : o;
}

__device__ __forceinline__ uint32_t chunk_magnitude(f32x8 f)
{
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) { const uint32_t b = magnitude(f[j]); m = m > b ? m : b; }
    return m;
}

// Writes this lane's chunk of a row's 8-bit form and, by the first of a block's four lanes, the block's step.  All four lanes are active; values
// behind the row's end come as zero.  `skip`: chunk_skip's, the first values that are not the chunk's own and come as zero (moving bytes costs an eighth
// of moving values: 30000 x 300 kept 22.3 -> 19.1 us).
__device__ __forceinline__ void pack_chunk(int8_t *q, uint8_t *e, int c, f32x8 f, int skip = 0)
{
    const PackStep s = pack_step(quad_max(chunk_magnitude(f)));
    const uint64_t w = (uint64_t)pack_four(f[4], f[5], f[6], f[7], s) << 32 | pack_four(f[0], f[1], f[2], f[3], s);
    *reinterpret_cast<uint64_t *>(q + (size_t)c * CHUNK) = skip < CHUNK ? w >> (8 * skip) : 0;
    if ((c & 3) == 0) e[c >> 2] = (uint8_t)s.byte;
}

} // namespace het
