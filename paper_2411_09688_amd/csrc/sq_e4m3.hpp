// e4m3 codes with one power-of-two scale per block of tokens and head, as the quantizing kernels write them.
//
// With an exponent of its own in every code, a scale that is a power of two loses no precision against any other scale: it
// only has to keep the largest value of the block in range.  Dividing by it is exact, so a value is rounded once, and a
// block whose scale is raised later (tokens are appended) has its codes shifted, not rounded, unless they become
// subnormal.
#pragma once
#include "sq_common.hpp"

namespace sq {

constexpr int E4M3_EXP_MIN = -64, E4M3_EXP_MAX = 64;      // exponents of a scale
constexpr int KV_BLOCK = 64;                               // keys of the fixed context per scale

typedef float f2v __attribute__((ext_vector_type(2)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));

// What a kernel reads or writes once.  STREAM: past the caches, where the call's data would not stay in them.
template <bool STREAM, typename P>
__device__ __forceinline__ auto load_once(P p)
{
    return STREAM ? __builtin_nontemporal_load(p) : *p;
}
template <bool STREAM, typename T>
__device__ __forceinline__ void store_once(T *p, T v)
{
    if (STREAM) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// The least e with amax <= 448 * 2^e; amax: bits of a float that is finite and not negative.  448 = 1.75 * 2^8, so e is the
// value's own exponent less 8, and one more where its mantissa is over 1.75: 0x1fffff carries exactly then.
__device__ __forceinline__ int scale_exponent(uint32_t amax)
{
    const int e = (int)((amax + 0x1fffffu) >> 23) - 135;
    return min(max(e, E4M3_EXP_MIN), E4M3_EXP_MAX);
}

__device__ __forceinline__ float exp2_int(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// The least e with |scale| <= 2^e, for a scale that stands in a page: of a power of two its own exponent.
__device__ __forceinline__ int exponent_holding(float scale)
{
    const int e = (int)(((__builtin_bit_cast(uint32_t, scale) & 0x7fffffffu) + 0x7fffffu) >> 23) - 127;
    return min(max(e, E4M3_EXP_MIN), E4M3_EXP_MAX);
}

// Eight codes to f16, exact; times a power of two (a normal one, or 0 as some power far below f16's least value), rounded once, past f16's end to
// an infinity.
__device__ __forceinline__ h8 codes_f16(uint32_t lo, uint32_t hi, float scale = 1.0f)
{
    const h2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true);
    const h2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true);
    return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// |x| as bits for a maximum over a block: infinities and NaN count as nothing.
__device__ __forceinline__ uint32_t finite_abs(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}

// Two values to codes: nearest even for |x| <= 448, NaN for NaN and infinities.
template <bool HIGH>
__device__ __forceinline__ uint32_t e4m3_pair(float a, float b, uint32_t old)
{
    return __builtin_amdgcn_cvt_pk_fp8_f32(a, b, old, HIGH);
}

// Eight values to eight codes; scaled first.
__device__ __forceinline__ u2v e4m3_encode8(const float (&x)[8])
{
    const uint32_t lo = e4m3_pair<true>(x[2], x[3], e4m3_pair<false>(x[0], x[1], 0u));
    return u2v{lo, e4m3_pair<true>(x[6], x[7], e4m3_pair<false>(x[4], x[5], 0u))};
}
__device__ __forceinline__ u2v e4m3_encode8(const float (&x)[8], float inv)
{
    const float y[8] = {x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv, x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv};
    return e4m3_encode8(y);
}

// Four codes times a factor, to four codes (exact before the rounding to codes if the factor is a power of two, else rounded in fp32 first:
// a product that 24 bits put onto a border between two codes is off by 2^-24 of itself more than half a step).
__device__ __forceinline__ uint32_t e4m3_rescale4(uint32_t w, float f)
{
    const f2v a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    return e4m3_pair<true>(b.x * f, b.y * f, e4m3_pair<false>(a.x * f, a.y * f, 0u));
}

// x * f in fp32 so that rounding it once more, to 12 significant bits or fewer, gives what rounding the product would have given: where it lies on
// a border of the coarser rounding (its low 12 bits are zero) and is not the product itself, the neighbour on the product's side is taken.  (The
// error e is exact unless the product is near fp32's least values.)
__device__ __forceinline__ float product_unbiased(float x, float f)
{
    const float p = x * f, e = fmaf(x, f, -p);
    const uint32_t b = __builtin_bit_cast(uint32_t, p);
    const uint32_t towards = (__builtin_bit_cast(uint32_t, e) ^ b) >> 31 ? b - 1u : b + 1u;
    return (b & 0xfffu) == 0u && fabsf(e) > 0.0f && (b & 0x7f800000u) != 0x7f800000u ? __builtin_bit_cast(float, towards) : p;
}

// Double to float so that rounding the float once more, to 12 significant bits or fewer, gives what rounding the double
// would have given.  Where the nearest float could lie on a border of the coarser rounding (its low 12 bits are zero) and is
// not the double itself, the neighbour on the double's side is taken.
__device__ __forceinline__ float to_float_unbiased(double x)
{
    float f = (float)x;
    const uint32_t b = __builtin_bit_cast(uint32_t, f);
    if (__builtin_expect((b & 0xfffu) == 0u, 0) && (double)f != x && (b & 0x7f800000u) != 0x7f800000u)
        f = __builtin_bit_cast(float, fabs((double)f) > fabs(x) ? b - 1u : b + 1u);
    return f;
}

}  // namespace sq
