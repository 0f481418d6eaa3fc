// Device helpers of the microscaled operators: types in and out, codes and scales.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mx.h"

namespace fastrack {
namespace mx {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bits_f32(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t f32_bits(float f) { return __builtin_bit_cast(uint32_t, f); }

// The element types as C++ types, by MxType.
template <uint32_t T> struct Elem;
template <> struct Elem<kBf16> { typedef __bf16 type; };
template <> struct Elem<kFp16> { typedef _Float16 type; };
template <> struct Elem<kFp32> { typedef float type; };

// A run-time MxType as the constant T of what follows.
#define MX_TYPE(t, ...)                                                                            \
    do {                                                                                           \
        if ((t) == kBf16) { constexpr uint32_t T = kBf16; __VA_ARGS__; }                           \
        else if ((t) == kFp16) { constexpr uint32_t T = kFp16; __VA_ARGS__; }                      \
        else { constexpr uint32_t T = kFp32; __VA_ARGS__; }                                        \
    } while (0)

// Elements [c, c + 8) of a row as floats, zero past `cols`. A whole unit is loaded 16 bytes at a
// time wherever it starts: the hardware takes any alignment.
template <uint32_t T>
__device__ __forceinline__ void load8(const void *base, uint64_t row_off, uint32_t c, uint32_t cols, float (&v)[8])
{
    typedef typename Elem<T>::type E;
    const E *p = reinterpret_cast<const E *>(base) + row_off + c;
    if (c + 8 <= cols) {
        E e[8];
        __builtin_memcpy(e, p, sizeof e);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = (float)e[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = c + i < cols ? (float)p[i] : 0.0f;
    }
}

// Rounded to the output's type once, to nearest even (what the conversion does).
template <uint32_t T>
__device__ __forceinline__ void store8(void *base, uint64_t row_off, uint32_t c, uint32_t cols, const float (&v)[8])
{
    typedef typename Elem<T>::type E;
    E *p = reinterpret_cast<E *>(base) + row_off + c;
    if (c + 8 <= cols) {
        // As words: the compiler would take eight elements apart again, and join the last of them
        // with the branch below.
        typedef E Ex8 __attribute__((ext_vector_type(8)));
        typedef uint32_t Words __attribute__((ext_vector_type(sizeof(E) * 2)));
        Ex8 e;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            e[i] = (E)v[i];
        const Words w = __builtin_bit_cast(Words, e);
#pragma unroll
        for (int i = 0; i < (int)sizeof(E) / 2; ++i) {
            const u32x4 part = {w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
            __builtin_memcpy(reinterpret_cast<uint8_t *>(p) + 16 * i, &part, 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols)
                p[i] = (E)v[i];
    }
}

// 2^(e - 127) of a scale byte, NaN for 255. 2^-127 (e = 0) is subnormal.
__device__ __forceinline__ float scale_f32(uint32_t e)
{
    return bits_f32((e << 23) | (e - 1u >= 254u ? 0x00400000u : 0u));
}

// What an MX8 code's unit is worth, 2^(e - 133): down to 2^-133, subnormal.
__device__ __forceinline__ float scale8_f32(uint32_t e)
{
    const float s = __builtin_amdgcn_ldexpf(1.0f, (int)e - 133);
    return e == 255u ? bits_f32(0x7FC00000u) : s;
}

// The same for the conversions from and to E2M1, which read the exponent bits alone: 0 is 2^-127
// to them, 255 a NaN.
__device__ __forceinline__ float scale4_f32(uint32_t e) { return bits_f32(e << 23); }

// Eight E2M1 codes as bf16 pairs. Exact: 2 significant bits and any power of two down to
// 2^-128, which bf16 holds as a subnormal.
__device__ __forceinline__ u32x4 decode4_bf16(uint32_t codes, float scale)
{
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}

__device__ __forceinline__ void decode4_f32(uint32_t codes, float scale, float (&v)[8])
{
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0),
                b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1),
                c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2),
                d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
    v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
}

// Eight int8 codes as floats. (The two words are kept apart from each other: taken as one of 64
// bits, each byte is cut out by an instruction of its own before the conversion.)
__device__ __forceinline__ void decode8_f32(u32x2 codes, float scale, float (&v)[8])
{
    uint32_t w[2] = {codes[0], codes[1]};
    asm("" : "+v"(w[0]));
    asm("" : "+v"(w[1]));
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = (float)(int8_t)(w[i / 4] >> (8 * (i % 4))) * scale;
}

// Two of a word's four int8 codes (the lower or the upper ones) as a bf16 pair. Exact: 7
// significant bits and a power of two down to 2^-133, bf16's smallest subnormal.
__device__ __forceinline__ uint32_t decode8_pair(uint32_t word, int upper, float scale)
{
    asm("" : "+v"(word));
    const float a = (float)(int8_t)(word >> (16 * upper)) * scale, b = (float)(int8_t)(word >> (16 * upper + 8)) * scale;
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

__device__ __forceinline__ u32x4 decode8_bf16(u32x2 codes, float scale)
{
    return u32x4{decode8_pair(codes[0], 0, scale), decode8_pair(codes[0], 1, scale), decode8_pair(codes[1], 0, scale),
                 decode8_pair(codes[1], 1, scale)};
}

// The largest magnitude of a block, as the bits of |v| (ordered like the values, infinity and
// then NaN on top), shared by the four lanes that hold 8 of its values each.
__device__ __forceinline__ uint32_t block_top(const float (&v)[8])
{
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        t = max(t, f32_bits(v[i]) & 0x7FFFFFFFu);
    t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0xB1, 0xF, 0xF, true));   // lane ^ 1
    t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x4E, 0xF, 0xF, true));   // lane ^ 2
    return t;
}

// Scale byte of a block: floor(log2 top) - (2 for E2M1, whose largest power is 4), at least
// -127 (a subnormal top has exponent bits 0 and lands there). 255 if the block holds a NaN
// or an infinity, which the codes cannot say.
template <uint32_t FMT>
__device__ __forceinline__ uint32_t block_scale(uint32_t top)
{
    const uint32_t e = top >> 23;
    if (e == 255u)
        return 255u;
    return FMT == kMx8 ? e : (e > 2u ? e - 2u : 0u);
}

// Eight E2M1 codes of v / 2^(e - 127): nearest, ties to the even code, saturated at 6.
__device__ __forceinline__ uint32_t encode4(const float (&v)[8], uint32_t e)
{
    if (e == 255u)
        return 0;
    const float s = scale4_f32(e);
    uint32_t o = 0;
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[0], v[1], s, 0);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[2], v[3], s, 1);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[4], v[5], s, 2);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[6], v[7], s, 3);
    return o;
}

// Eight int8 codes: v / 2^(e - 133) rounded to nearest even, held to +-127. The power goes
// in as 2^(127 - e) and 64, both in range (exact products); adding 1.5 * 2^23 rounds and
// leaves the integer in the low byte.
__device__ __forceinline__ u32x2 encode8(const float (&v)[8], uint32_t e)
{
    if (e == 255u)
        return u32x2{0, 0};
    const float inv = e == 254u ? bits_f32(0x00400000u) : bits_f32((254u - e) << 23);
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = __builtin_amdgcn_fmed3f(v[i] * inv, -1.984375f, 1.984375f);
        b[i] = f32_bits(__builtin_fmaf(t, 64.0f, 12582912.0f)) & 255u;
    }
    return u32x2{b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24, b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24};
}

// The upper halves of eight floats: bf16 values cut, not rounded, so that what is left of each
// (left: v becomes it) has 8 significant bits less and the terms add up to the value, down to
// bf16's smallest, 2^-133.
__device__ __forceinline__ u32x4 upper_halves(const float (&v)[8])
{
    u32x4 h;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        h[i] = __builtin_amdgcn_perm(f32_bits(v[2 * i + 1]), f32_bits(v[2 * i]), 0x07060302u);
    return h;
}

__device__ __forceinline__ void leave_lower(float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] -= bits_f32(f32_bits(v[i]) & 0xFFFF0000u);
}

// The first term of values that have more, and what is left of them. An infinity goes into the
// first term whole (the subtraction alone would leave a NaN; of a NaN it leaves one rightly).
__device__ __forceinline__ u32x4 first_term(float (&v)[8])
{
    const u32x4 h = upper_halves(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float left = v[i] - bits_f32(f32_bits(v[i]) & 0xFFFF0000u);
        v[i] = __builtin_fabsf(v[i]) == __builtin_inff() ? 0.0f : left;
    }
    return h;
}

}  // namespace mx
}  // namespace fastrack
