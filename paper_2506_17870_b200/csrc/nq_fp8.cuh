// Pieces shared by the kernels that write e4m3 with a scale for each group of 128 (the quantiser and the block norm).
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

// Two values to e4m3, `lo` in the low byte: nearest even, larger magnitudes clamped to 448 (fl(x * inv) can pass 448
// by a rounding), NaN kept.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    return e4m3x2(a, b) | (e4m3x2(c, d) << 16);
}

}  // namespace nq
