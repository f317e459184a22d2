// Elements of 4 bits: sixteen values under a scale that 32 of them share, a power of two.
#pragma once
#include <type_traits>

#include "kv_cache.h"

namespace mdsd {

// A scale as the conversions take it, which look at the exponent alone: with all of its bits set every element becomes NaN
__device__ inline float scale_of(uint32_t scale) { return __uint_as_float(scale << 23); }

// Two elements at `kPlace` (a byte of four) times a scale, as T
template <class T, int kPlace>
__device__ inline auto two_of(uint32_t codes, float scale)
{
    if constexpr (std::is_same_v<T, float>)
        return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, kPlace);
    else if constexpr (std::is_same_v<T, __bf16>)
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, kPlace));
    else
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, kPlace));
}
// 16 bytes of T from the codes that hold them: eight elements of four bytes, or four of fp32, the first or the second
template <class T>
__device__ inline u32x4 sixteen_bytes(uint32_t codes, float scale, bool second)
{
    if constexpr (std::is_same_v<T, float>) {
        const f32x2 a = second ? two_of<T, 2>(codes, scale) : two_of<T, 0>(codes, scale);
        const f32x2 b = second ? two_of<T, 3>(codes, scale) : two_of<T, 1>(codes, scale);
        return u32x4{__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(b[0]), __float_as_uint(b[1])};
    } else {
        return u32x4{two_of<T, 0>(codes, scale), two_of<T, 1>(codes, scale), two_of<T, 2>(codes, scale), two_of<T, 3>(codes, scale)};
    }
}

// The scale of elements whose absolute values' bits are `most` at most: the smallest power of two by which the largest is 7 at most, in
// [least, greatest].  7 = 1.75 * 2^2: one less than the exponent's two where the fraction is beyond 1.75.
__device__ inline uint32_t scale_for(uint32_t most, int least, int greatest)
{
    if (most >= 0x7f800000u) return kNoNumber;
    return (uint32_t)max(least, min(greatest, (int)((most + 0x1fffffu) >> 23) - 127 - 2)) + 127;
}
// Eight elements' codes: to the nearest value, ties to even, 6 beyond it
__device__ inline uint32_t codes_of(const float (&x)[8], uint32_t scale)
{
    if (scale == kNoNumber) return 0;
    const float unit = scale_of(scale);
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], unit, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], unit, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], unit, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], unit, 3);
}
// Powers of two under which every value of a block is a number of T: 6 times the largest is finite, half the smallest
// normal, or in fp16 the smallest number there is
template <class T>
constexpr int kLeastScale = std::is_same_v<T, _Float16> ? -23 : -125;
template <class T>
constexpr int kGreatestScale = std::is_same_v<T, _Float16> ? 13 : 125;

// The type that elements of 4 bits are worked on in.  bf16 holds every one of them exactly, and an fp32 number is the sum of
// three of its kind, eight bits each: three products instead of one, each of which costs a sixteenth of fp32's.
template <class T, bool kFour>
using Worked = std::conditional_t<kFour && std::is_same_v<T, float>, __bf16, T>;
template <class T, bool kFour>
constexpr int kPartsOf = kFour && std::is_same_v<T, float> ? 3 : 1;
// the next eight bits of two numbers, cut off, and what is left of these
__device__ inline uint32_t next_parts(float& x, float& y)
{
    const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
    x -= __uint_as_float(a & 0xffff0000u);
    y -= __uint_as_float(b & 0xffff0000u);
    return __builtin_amdgcn_perm(b, a, 0x07060302);
}
// eight numbers in fp32 in three parts
__device__ inline void in_parts(const float* from, u32x4 (&to)[3])
{
    f32x4 x[2] = {*(const f32x4*)from, *(const f32x4*)(from + 4)};
#pragma unroll
    for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) to[p][i] = next_parts(((float*)x)[2 * i], ((float*)x)[2 * i + 1]);
}

// kBytes of codes that a lane has, of one scale.  kAhead: for loops whose loads go from one turn to the next.  A byte that does is
// widened, and so waited for, at the turn's end: the scale comes with the aligned word that it lies in (of the same allocation).
template <int kBytes, bool kAhead>
struct Codes {
    uint32_t code[kBytes / 4];
    uint32_t word, at_bit;

    __device__ void load(const char* codes, const uint8_t* scales, int at)
    {
        if constexpr (kBytes == 16) {
            const u32x4 x = *(const u32x4*)(codes + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) code[i] = x[i];
        } else {
            const u32x2 x = *(const u32x2*)(codes + at);
            code[0] = x[0];
            code[1] = x[1];
        }
        const uint8_t* const scale_at = scales + at / 16;
        if constexpr (kAhead) {
            const uint32_t in_word = (uint32_t)(uintptr_t)scale_at & 3;
            word = *(const uint32_t*)(scale_at - in_word);
            at_bit = in_word * 8;
        } else {
            word = *scale_at;
        }
    }
    __device__ uint32_t scale() const { return kAhead ? word >> at_bit & 255 : word; }
    __device__ void clear(bool all)
    {
#pragma unroll
        for (int i = 0; i < kBytes / 4; ++i) code[i] = all ? 0 : code[i];
        word = all ? kUnitScale : word;
        if (kAhead) at_bit = all ? 0 : at_bit;
    }
    // the i-th 16 bytes of them as T
    template <class T>
    __device__ u32x4 chunk(int i) const
    {
        constexpr int kPer = sizeof(T) / 2;  // chunks of four bytes of codes
        return sixteen_bytes<T>(code[i / kPer], scale_of(scale()), i % kPer);
    }
};

}  // namespace mdsd
