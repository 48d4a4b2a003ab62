// Conversions between fp32 and microscaled 4-bit blocks, shared by the kernels that need them.
#pragma once
#include <stdint.h>

namespace regenvc {

// Scale byte of a block from the largest magnitude's bit pattern: 2^(floor(log2 amax) - 2), so that amax lands in
// [4, 8) where 6 is the largest code; below 2^-125 the smallest scale, 2^-127.  The exponent field is floor(log2) + 127.
// A block that holds an infinity or NaN has no scale: 255.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits) {
    const uint32_t e = amax_bits >> 23;
    return e == 255u ? 255u : (e > 2u ? e - 2u : 0u);
}
// 1 / scale, a power of two (exact products); 0 for a block without a scale, so that its codes are 0 or NaN's (0).
__device__ __forceinline__ float mx_inverse_scale(uint32_t byte) {
    return byte == 255u ? 0.0f : __uint_as_float((254u - byte) << 23);
}
__device__ __forceinline__ float mx_scale_value(uint32_t byte) {
    return byte == 255u ? __uint_as_float(0x7FC00000u) : (byte == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23));
}
// Eight values -> eight e2m1 codes, element i in bits 4i..4i+3; nearest, ties to even, magnitudes above 6 become 6.
__device__ __forceinline__ uint32_t mx_codes8(const float* v) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// Eight codes -> four packed fp16 pairs (every e2m1 value is an fp16 value).
__device__ __forceinline__ void mx_values8(uint32_t codes, uint32_t* h2) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h2[0]), "=r"(h2[1]), "=r"(h2[2]), "=r"(h2[3])
        : "r"(codes));
}

// Eight values -> the e2m1 values nearest to them, as four packed fp16 pairs; by all lanes of a warp.  The two conversions
// must not meet in one thread's registers: ptxas 12.9 from -O1 on makes zeros of mx_values8(mx_codes8(v)) (the same PTX is
// right at ptxas -O0, an empty asm statement between the two changes nothing).  An exchange of each lane with itself keeps
// them apart.
__device__ __forceinline__ void mx_round8(const float* v, uint32_t* h2) {
    mx_values8(__shfl_sync(0xffffffffu, mx_codes8(v), threadIdx.x & 31), h2);
}

}  // namespace regenvc
