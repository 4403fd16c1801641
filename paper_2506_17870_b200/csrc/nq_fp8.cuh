// Pieces shared by the e4m3 kernels (quantiser, block norm, product): a group's scale, rounding, packed fp32 arithmetic.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace nq {

constexpr float kE4M3Max = 448.0f;

// The scale of a group from the bits of its largest magnitude, and its inverse; see nq_fp8_quantize in nq.h.  The
// maximum is taken on the bit patterns of |x| as unsigned integers: their order is that of the numbers, infinity
// above all of them and NaN above infinity, so a NaN is never lost.  max() on the float would drop it.
__device__ __forceinline__ void group_scale(uint32_t amax_bits, float& s, float& inv) {
    s = __fdiv_rn(__uint_as_float(amax_bits), kE4M3Max);
    s = s < 1.17549435e-38f ? 1.17549435e-38f : s;        // false for NaN, which stays
    inv = __frcp_rn(s);
}

// Four values to e4m3, `a` in the lowest byte: nearest even, larger magnitudes clamped to 448 (fl(x * inv) can pass 448
// by a rounding), NaN kept.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
        "mov.b32 %0, {lo, hi};\n\t}"
        : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}

// Pairs of fp32 values in one 64-bit register: one instruction works on both (half the issue slots of scalar ones; in the
// product's promotion 536 -> 518 us).
__device__ __forceinline__ uint64_t pack2(uint32_t lo, uint32_t hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
    return r;
}
__device__ __forceinline__ uint64_t pack2f(float lo, float hi) { return pack2(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ uint64_t both(float v) { return pack2f(v, v); }
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ float sum2(uint64_t v) {
    float lo, hi;
    unpack2(v, lo, hi);
    return lo + hi;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint32_t e4m3x4(uint64_t ab, uint64_t cd) {
    float a, b, c, d;
    unpack2(ab, a, b);
    unpack2(cd, c, d);
    return e4m3x4(a, b, c, d);
}
// the largest magnitude; a NaN wins
__device__ __forceinline__ float max_abs(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}
__device__ __forceinline__ float max_abs(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)), "f"(fabsf(c)));
    return r;
}

}  // namespace nq
