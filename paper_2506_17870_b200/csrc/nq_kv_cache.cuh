// Pieces shared by the kernels on the paged key-value cache: the host's checks of a cache, the scale of a row of a head, wide
// accesses.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "nq_fp8.cuh"
#include "nq_internal.cuh"

namespace nq {

inline bool misaligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

// What every entry point that takes a cache checks of it.
inline int check_pages(const nq_kv_pages* c) {
    if (!c || c->pages < 0 || c->page_size <= 0 || c->kv_heads <= 0) return NQ_ERR_INVALID_ARG;
    if (c->dtype != NQ_BF16 && c->dtype != NQ_E4M3 && c->dtype != NQ_I8) return NQ_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128) return NQ_ERR_UNSUPPORTED;
    if ((c->page_size & 15) || c->page_size > 32768 || c->kv_heads > 65536 || c->pages > 0x7fffffffll / c->page_size) return NQ_ERR_UNSUPPORTED;
    if (c->pages > 0) {
        if (!c->k || !c->v || (c->dtype == NQ_BF16) != (c->ks == nullptr) || (c->dtype == NQ_BF16) != (c->vs == nullptr)) return NQ_ERR_INVALID_ARG;
        if (misaligned(c->k, 16) || misaligned(c->v, 16) || misaligned(c->ks, 4) || misaligned(c->vs, 4)) return NQ_ERR_ALIGNMENT;
    }
    return NQ_OK;
}

// A cache as the kernels see it.
struct Pages {
    uint8_t *k, *v;
    float *ks, *vs;
    int pages, page_size, kv_heads;
};
inline Pages pages_of(const nq_kv_pages* c) {
    return {static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), c->ks, c->vs, (int)c->pages, c->page_size, c->kv_heads};
}

// A head's row in a cache: its scale from the bits of its largest magnitude (order of bit patterns = order of magnitudes, NaN
// above infinity above the rest), and its inverse.  As nq_fp8_quantize has it, with 127 in the place of 448 for INT8.
__device__ __forceinline__ void row_scale(uint32_t amax_bits, float most, float& s, float& inv) {
    s = __fdiv_rn(__uint_as_float(amax_bits), most);
    s = s < 1.17549435e-38f ? 1.17549435e-38f : s;        // false for NaN, which stays
    inv = __frcp_rn(s);
}

// Four values to INT8, `a` in the lowest byte: nearest even, a NaN as 0.  (Within +-127.5, as x * inv is, nothing comes out as -128.)
__device__ __forceinline__ uint32_t i8x4(float a, float b, float c, float d) {
    uint32_t w[4], r;
    asm("cvt.rni.sat.s8.f32 %0, %1;" : "=r"(w[0]) : "f"(a));
    asm("cvt.rni.sat.s8.f32 %0, %1;" : "=r"(w[1]) : "f"(b));
    asm("cvt.rni.sat.s8.f32 %0, %1;" : "=r"(w[2]) : "f"(c));
    asm("cvt.rni.sat.s8.f32 %0, %1;" : "=r"(w[3]) : "f"(d));
    asm("{\n\t.reg .b32 x, y;\n\tprmt.b32 x, %1, %2, 0x0040;\n\tprmt.b32 y, %3, %4, 0x0040;\n\tprmt.b32 %0, x, y, 0x5410;\n\t}" : "=r"(r) : "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]));
    return r;
}

// Loads of data that is used once; ordinary ones (not through the read-only path), since they stand behind wait_previous().
__device__ __forceinline__ uint4 load16(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

}  // namespace nq
