// cache4.cuh -- the 4-bit cache's number format.
//
// A row's channels go in groups of 16 with a scale each.  The scale is an
// unsigned float of 5 exponent and 3 mantissa bits: the f16 of the same value
// without its sign and its low seven bits, so it is read by a shift.  A channel is
// a 4-bit float (sign, 2 exponent bits, 1 mantissa bit; magnitudes 0 0.5 1 1.5 2 3
// 4 6).  A value, code times scale, has at most 2 + 4 significant bits and
// magnitude at most 6 * 10240: exact in f16 and in bf16.  A scale of 255 is a NaN:
// the group held something that is not finite.
//
// The nearest scale and code are found exactly, whatever the rounding of the
// arithmetic here: a bf16 x has 8 significant bits, a scale s at most 4 and the
// border between two codes 3 (between two scales, times 6: 7), so x differs from
// border * s by nothing or by 2^-8 of it at least, far more than the errors below.
#pragma once
#include <cuda_fp16.h>

#include <cstdint>

#include "sm100.cuh"

namespace logo {

constexpr int kC4Group = 16;            // channels that share a scale
constexpr uint32_t kC4MaxScale = 0xe2;  // 10240; 6 times that is the largest multiple below the f16 limit
constexpr uint32_t kC4NaN = 0xff;

// The code of the scale of a group whose largest magnitude has these bf16 bits.
__device__ __forceinline__ uint32_t c4_scale_code(uint32_t amax)
{
    if (amax >= 0x7f80u) return kC4NaN;
    const float s = __fdiv_rn(__uint_as_float(amax << 16), 6.f);
    if (s < 6.103515625e-05f) return __float2int_rn(s * 131072.f);  // below 2^-14: steps of 2^-17
    uint32_t u = __float_as_uint(s);
    u = (u + 0x7ffffu + ((u >> 20) & 1u)) >> 20;  // to nearest, ties to even
    return min(u - ((127u - 15u) << 3), kC4MaxScale);
}

__device__ __forceinline__ float c4_scale(uint32_t code)
{
    return __half2float(__ushort_as_half(static_cast<unsigned short>(code << 7)));
}

// 1 / scale for the quotient of c4_codes; 0 where the codes do not matter.
__device__ __forceinline__ float c4_inverse(uint32_t code)
{
    return code == 0 || code == kC4NaN ? 0.f : __fdividef(1.f, c4_scale(code));
}

// Eight channels (four words of bf16 pairs) -> their codes, the first channel lowest.
// The quotient, off by a few units of fp32's last place, is first rounded to a
// multiple of 2^-13: on a border it comes back to it, beside a border (2^-10 away at
// least) it stays on its side.
__device__ __forceinline__ uint32_t c4_codes(const uint32_t (&x)[4], float inv)
{
    const uint64_t by = f2_pack(inv, inv), up = f2_pack(1536.f, 1536.f), down = f2_pack(-1536.f, -1536.f);
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t q = f2_mul(f2_pack(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u)), by);
        f2_unpack(f2_add(f2_add(q, up), down), y[2 * i], y[2 * i + 1]);
    }
    uint32_t r;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r)
        : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
    return r;
}

// Eight codes -> four f16x2 of their magnitudes and signs, in channel order.
__device__ __forceinline__ void c4_decode(uint32_t codes, uint32_t (&h)[4])
{
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(codes));
}

__device__ __forceinline__ uint32_t h2_mul(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// f16x2 -> bf16x2; exact for a cache's values.
__device__ __forceinline__ uint32_t c4_to_bf16x2(uint32_t h)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(f.y), "f"(f.x));
    return r;
}

}  // namespace logo
