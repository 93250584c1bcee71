// pps_q4.cuh -- the cache in 4 bits: a block of 16 channels is 16 e2m1 codes (8 bytes, the even channel of a byte low) and an
// e4m3 scale.
//
//   held:  s = e4m3(min(max |z| / 6, 448)),  code = e2m1(z / s),  to nearest, ties to even;  value = s * code
//
// A value has 6 significant bits and lies between 2^-10 and 2688, so that fp16 holds it exactly: code times scale is one exact
// multiplication of two halves.
#pragma once
#include <cstdint>
#include <cstring>

#include <cuda_fp16.h>

namespace pps {
namespace q4 {

// four bytes of codes -> four pairs (low nibble, high nibble)
__device__ __forceinline__ void widen8(uint32_t codes, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(codes));
}
// the two scales in the low half of `bytes`, as halves
__device__ __forceinline__ uint32_t scales2(uint32_t bytes) {
    uint32_t h;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\t}" : "=r"(h) : "r"(bytes));
    return h;
}
__device__ __forceinline__ uint32_t mul_halves(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float scale_float(uint32_t byte) {
    __half2 h;
    const uint32_t w = scales2(byte & 0xffu);
    memcpy(&h, &w, 4);
    return __low2float(h);
}

__device__ __forceinline__ float max3_abs(float a, float b, float c) {  // NaN if one is
    float y;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(fabsf(a)), "f"(fabsf(b)), "f"(fabsf(c)));
    return y;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t both(float x) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(x));
    return r;
}

// Codes (x: channels 0 to 7, y: 8 to 15) and scale byte of a block of z = x inv, x in pairs of neighbours.  One that is not finite
// throughout has the scale NaN.  z / s is rounded correctly, as a remainder corrects the product with 1 / s (Markstein, IBM J. Res.
// Dev. 34, 1990): next to the middle between two codes its last bit decides.
__device__ __forceinline__ uint2 quantise(const uint64_t (&x)[8], float inv, uint32_t& scale) {
    uint64_t z[8];
    float f[16], top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        z[i] = mul2(x[i], both(inv));
        asm("mov.b64 {%0, %1}, %2;" : "=f"(f[2 * i]), "=f"(f[2 * i + 1]) : "l"(z[i]));
        top = max3_abs(top, f[2 * i], f[2 * i + 1]);
    }
    scale = 0x7fu;
    if (!(top < INFINITY)) return make_uint2(0u, 0u);
    uint16_t two;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(0.0f), "f"(__fdiv_rn(top, 6.0f)));
    scale = two & 0xffu;
    if (scale == 0) return make_uint2(0u, 0u);
    const float s = scale_float(scale), r = __frcp_rn(s);
    const uint64_t r2 = both(r), s2 = both(-s);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint64_t p = mul2(z[i], r2), q = fma2(fma2(p, s2, z[i]), r2, p);
        asm("mov.b64 {%0, %1}, %2;" : "=f"(f[2 * i]), "=f"(f[2 * i + 1]) : "l"(q));
    }
    uint32_t w[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
        asm("{\n\t.reg .b8 a, b, c, d;\n\t"
            "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
            "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
            "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
            "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
            "mov.b32 %0, {a, b, c, d};\n\t}"
            : "=r"(w[k])
            : "f"(f[8 * k]), "f"(f[8 * k + 1]), "f"(f[8 * k + 2]), "f"(f[8 * k + 3]), "f"(f[8 * k + 4]), "f"(f[8 * k + 5]), "f"(f[8 * k + 6]),
              "f"(f[8 * k + 7]));
    return make_uint2(w[0], w[1]);
}

}  // namespace q4
}  // namespace pps
