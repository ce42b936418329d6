// What the kernels that read an 8-bit KV cache share.
#pragma once
#include <stdint.h>

namespace gsd {

// Four codes -> two pairs of fp16, in order.  Exact: a code has four (e4m3) or eight (int8) significant bits.  77 codes a
// cycle and SM together with three integer operations for four codes; by way of bf16 (the least that feeds a bf16
// product) it is 39 for e4m3 and 34 for int8.
template <bool INT8>
__device__ __forceinline__ void widen(uint32_t w, uint32_t& p0, uint32_t& p1) {
    if constexpr (INT8) {
        // 0x6400 | u is 1024 + u for a byte u; u = code + 128
        w ^= 0x80808080u;
        const uint32_t x0 = __byte_perm(w, 0x64646464u, 0x4140), x1 = __byte_perm(w, 0x64646464u, 0x4342);
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(p0) : "r"(x0), "r"(0x64806480u));
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(p1) : "r"(x1), "r"(0x64806480u));
    } else {
        asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}" : "=r"(p0), "=r"(p1) : "r"(w));
    }
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ float two(int e) { return __int_as_float((e + 127) << 23); }     // 2^e, -126 <= e <= 127

// fp16 holds a bf16 row exactly once a power of two has brought its largest magnitude to [2^14, 2^15): what falls below
// 2^-24 then is under 2^-38 of it.
constexpr int kLiftBits = 14;
// The power of two at or below a largest magnitude given as bf16 bits, in the range the lift is formed in.
__device__ __forceinline__ int lift_exp(uint32_t top) { return min(max((int)(top >> 7) - 127, -100), 126); }

}  // namespace gsd
