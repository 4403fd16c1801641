// What the block norm's forward and backward kernels share: a row in registers, the ring of rows, sums over a row, and the
// host's shapes and checks.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/nq.h"
#include "nq_fp8.cuh"
#include "nq_internal.cuh"
#include "nq_sm100.cuh"

namespace nq {
namespace {

using bf16 = __nv_bfloat16;

constexpr int kMaxCols = 16384;        // 512 threads of 4 pieces of 8 columns

// Where a thread's values of a row lie.  VEC: NV pieces of 8 neighbouring columns (one 16-byte access of bf16, two of
// fp32), threads side by side.  Otherwise (rows that start anywhere, odd lengths): single elements, 32 lanes side by
// side, so that the accesses still coalesce; a warp covers the same 256 columns a piece either way, which keeps the
// 128-column groups of e4m3 inside a warp.
template <int NV, bool VEC>
struct Cols {
    int t, threads, cols;
    __device__ __forceinline__ int col(int k, int j) const {
        return VEC ? (t + k * threads) * 8 + j : k * threads * 8 + (t >> 5) * 256 + j * 32 + (t & 31);
    }
    __device__ __forceinline__ bool has(int k, int j) const { return col(k, VEC ? 0 : j) < cols; }
};

// A thread's values of a row, in pairs.
template <int NV>
using Row = uint64_t[NV][4];

__device__ __forceinline__ uint4 ld16(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void spread(const uint4& w, uint64_t (&v)[4]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = pack2(u[j] << 16, u[j] & 0xffff0000u);
}
__device__ __forceinline__ void spread(const uint4& a, const uint4& b, uint64_t (&v)[4]) {
    v[0] = pack2(a.x, a.y); v[1] = pack2(a.z, a.w); v[2] = pack2(b.x, b.y); v[3] = pack2(b.z, b.w);
}
// a row from global memory; absent columns read as zero
template <int NV, bool VEC>
__device__ __forceinline__ void load_row(const Cols<NV, VEC>& c, const bf16* row, Row<NV>& v) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (VEC) {
            uint4 w = make_uint4(0u, 0u, 0u, 0u);
            if (c.has(k, 0)) w = ld16(row + c.col(k, 0));
            spread(w, v[k]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[k][j] = pack2f(c.has(k, 2 * j) ? __bfloat162float(row[c.col(k, 2 * j)]) : 0.0f,
                                 c.has(k, 2 * j + 1) ? __bfloat162float(row[c.col(k, 2 * j + 1)]) : 0.0f);
        }
    }
}
template <int NV, bool VEC>
__device__ __forceinline__ void load_row(const Cols<NV, VEC>& c, const float* row, Row<NV>& v) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (VEC) {
            uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
            if (c.has(k, 0)) { a = ld16(row + c.col(k, 0)); b = ld16(row + c.col(k, 0) + 4); }
            spread(a, b, v[k]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[k][j] = pack2f(c.has(k, 2 * j) ? row[c.col(k, 2 * j)] : 0.0f, c.has(k, 2 * j + 1) ? row[c.col(k, 2 * j + 1)] : 0.0f);
        }
    }
}
// the same from a row in shared memory
template <int NV>
__device__ __forceinline__ void take_row(const Cols<NV, true>& c, const bf16* row, Row<NV>& v) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        if (c.has(k, 0)) w = *reinterpret_cast<const uint4*>(row + c.col(k, 0));
        spread(w, v[k]);
    }
}
template <int NV>
__device__ __forceinline__ void take_row(const Cols<NV, true>& c, const float* row, Row<NV>& v) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
        if (c.has(k, 0)) {
            a = *reinterpret_cast<const uint4*>(row + c.col(k, 0));
            b = *reinterpret_cast<const uint4*>(row + c.col(k, 0) + 4);
        }
        spread(a, b, v[k]);
    }
}
// ... and, element by element, from one that starts anywhere
template <int NV, typename T>
__device__ __forceinline__ void take_row(const Cols<NV, false>& c, const T* row, Row<NV>& v) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[k][j] = pack2f(c.has(k, 2 * j) ? (float)row[c.col(k, 2 * j)] : 0.0f, c.has(k, 2 * j + 1) ? (float)row[c.col(k, 2 * j + 1)] : 0.0f);
}
// one piece of a parameter vector; `none` where the vector is absent, zero in absent columns of one that is there
template <int NV, bool VEC>
__device__ __forceinline__ void load_param(const Cols<NV, VEC>& c, const float* vec, float none, int k, uint64_t (&v)[4]) {
    if (!vec) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = both(none);
    } else if (VEC) {
        uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
        if (c.has(k, 0)) {
            a = *reinterpret_cast<const uint4*>(vec + c.col(k, 0));
            b = *reinterpret_cast<const uint4*>(vec + c.col(k, 0) + 4);
        }
        spread(a, b, v);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = pack2f(c.has(k, 2 * j) ? vec[c.col(k, 2 * j)] : 0.0f, c.has(k, 2 * j + 1) ? vec[c.col(k, 2 * j + 1)] : 0.0f);
    }
}

__device__ __forceinline__ uint32_t bf16x2(uint64_t v) {
    float lo, hi;
    unpack2(v, lo, hi);
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}
template <int NV, bool VEC>
__device__ __forceinline__ void store_piece(const Cols<NV, VEC>& c, bf16* row, int k, const uint64_t (&v)[4]) {
    if (VEC) {
        if (c.has(k, 0)) *reinterpret_cast<uint4*>(row + c.col(k, 0)) = make_uint4(bf16x2(v[0]), bf16x2(v[1]), bf16x2(v[2]), bf16x2(v[3]));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float lo, hi;
            unpack2(v[j], lo, hi);
            if (c.has(k, 2 * j)) row[c.col(k, 2 * j)] = __float2bfloat16_rn(lo);
            if (c.has(k, 2 * j + 1)) row[c.col(k, 2 * j + 1)] = __float2bfloat16_rn(hi);
        }
    }
}
template <int NV, bool VEC>
__device__ __forceinline__ void store_piece(const Cols<NV, VEC>& c, float* row, int k, const uint64_t (&v)[4]) {
    if (VEC) {
        if (c.has(k, 0)) {
            *reinterpret_cast<ulonglong2*>(row + c.col(k, 0)) = make_ulonglong2(v[0], v[1]);
            *reinterpret_cast<ulonglong2*>(row + c.col(k, 0) + 4) = make_ulonglong2(v[2], v[3]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float lo, hi;
            unpack2(v[j], lo, hi);
            if (c.has(k, 2 * j)) row[c.col(k, 2 * j)] = lo;
            if (c.has(k, 2 * j + 1)) row[c.col(k, 2 * j + 1)] = hi;
        }
    }
}
// eight bytes of a piece, four to a word
template <int NV, bool VEC>
__device__ __forceinline__ void store_bytes8(const Cols<NV, VEC>& c, uint8_t* row, int k, uint32_t lo, uint32_t hi) {
    if (VEC) {
        if (c.has(k, 0)) *reinterpret_cast<uint2*>(row + c.col(k, 0)) = make_uint2(lo, hi);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c.has(k, j)) row[c.col(k, j)] = (uint8_t)((j < 4 ? lo : hi) >> (8 * (j & 3)));
    }
}

// A ring of rows in shared memory, filled by bulk copies that one thread of the block starts several rows ahead, so that the bytes in flight do not depend on how many threads wait for a row's
// sums.  Rows of up to four tensors lie side by side in a stage.  A wait that gives up (see mbar_wait) lets its thread go
// on with what is there: every later wait then returns at once, all threads reach all barriers, and the host finds the
// record.
constexpr int kRingHead = 128;             // barriers and the abort flag, before the stages
constexpr int kMaxStages = 8;
// room for a row in a stage
__host__ __device__ inline int row_slot(int bytes, bool vec) { return vec ? bytes : (bytes + 30) & ~15; }
struct RowRing {
    uint8_t* stages;
    uint64_t* full;
    volatile int* abort_flag;
    unsigned int* status;
    int stage_bytes;
    bool first;                            // this thread starts the copies
    // a __syncthreads has to follow
    __device__ __forceinline__ void init(uint8_t* smem, int n, int bytes, unsigned int* st) {
        full = reinterpret_cast<uint64_t*>(smem);
        abort_flag = reinterpret_cast<volatile int*>(smem + kRingHead - 8);
        stages = smem + kRingHead;
        stage_bytes = bytes;
        status = st;
        first = threadIdx.x == 0;
        if (first) {
            for (int i = 0; i < n; ++i) sm100::mbar_init(sm100::smem_u32(&full[i]), 1);
            *abort_flag = 0;
            sm100::fence_barrier_init();
        }
    }
    __device__ __forceinline__ uint8_t* stage(int s) const { return stages + s * stage_bytes; }
    __device__ __forceinline__ void expect(int s, int bytes) const { sm100::mbar_arrive_expect_tx(sm100::smem_u32(&full[s]), bytes); }
    // Rows that start anywhere are copied as the 16-byte granules that hold them (the granules lie in the same
    // allocation: no allocation starts or ends inside one); the row then starts at its address modulo 16.
    static __device__ __forceinline__ int granules(const void* src, int bytes) {
        const uint64_t a = reinterpret_cast<uint64_t>(src);
        return (int)(((a + bytes + 15) & ~15ull) - (a & ~15ull));
    }
    __device__ __forceinline__ void copy(int s, int offset, const void* src, int bytes) const {
        sm100::bulk_load(sm100::smem_u32(stage(s) + offset), reinterpret_cast<const void*>(reinterpret_cast<uint64_t>(src) & ~15ull), granules(src, bytes),
                         sm100::smem_u32(&full[s]));
    }
    static __device__ __forceinline__ int shift(const void* src) { return (int)(reinterpret_cast<uint64_t>(src) & 15); }
    __device__ __forceinline__ void wait(int s, int parity) const {
        (void)sm100::mbar_wait(sm100::smem_u32(&full[s]), parity, abort_flag, status, 0x400u);
    }
    __device__ __forceinline__ void leave() const {
        if (first && *abort_flag) {                            // let copies in flight land before shared memory is released
            const long long t0 = clock64();
            while (clock64() - t0 < (1ll << 22)) { }
        }
    }
};

// Sums of N values over the threads of a row: a warp (shuffles alone) or the whole block (the warps' sums through shared
// memory; the two halves of `box` alternate, so that one barrier a call is enough).  Every thread adds in the same order,
// so all hold the same bits.
template <int N>
struct TeamSum {
    float (*box)[32][N];
    int threads, half;
    __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) v[n] += __shfl_xor_sync(0xffffffffu, v[n], d);
        if (threads == 32) return;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = threads >> 5;
        if (lane == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) box[half][warp][n] = v[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            v[n] = lane < warps ? box[half][lane][n] : 0.0f;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) v[n] += __shfl_xor_sync(0xffffffffu, v[n], d);
        }
        half ^= 1;
    }
};

// adds `what` to the row's columns; absent ones stay as they are (zero, which sums over the row rely on)
template <int NV, bool VEC>
__device__ __forceinline__ void shift_row(const Cols<NV, VEC>& c, Row<NV>& v, float what) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (VEC) {
                if (c.has(k, 0)) v[k][j] = add2(v[k][j], both(what));
            } else {
                v[k][j] = add2(v[k][j], pack2f(c.has(k, 2 * j) ? what : 0.0f, c.has(k, 2 * j + 1) ? what : 0.0f));
            }
        }
}
template <int NV>
__device__ __forceinline__ float total(const Row<NV>& v) {
    uint64_t s = 0ull;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) s = add2(s, v[k][j]);
    return sum2(s);
}
template <int NV>
__device__ __forceinline__ float dot(const Row<NV>& a, const Row<NV>& b) {
    uint64_t s = 0ull;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) s = fma2(a[k][j], b[k][j], s);
    return sum2(s);
}

// ------------------------------------------------------------------------------------------------------------ host
inline uintptr_t at(const void* p) { return reinterpret_cast<uintptr_t>(p); }

// Threads of a row: 8 * nv columns each.
struct Shape {
    int threads, nv;
};
inline Shape shape_of(int64_t cols, int nv) {
    return Shape{(int)((cols + 256 * nv - 1) / (256 * nv)) * 32, nv};
}
// One piece a thread as far as the block goes: more warps hide more of a row's latencies.
inline Shape wide_shape(int64_t cols, int most_threads) {
    return shape_of(cols, cols <= (int64_t)most_threads * 8 ? 1 : cols <= 512 * 16 ? 2 : 4);
}

// Rows through shared memory: the blocks of an SM, the stages of each and its shared memory.
struct RingPlan {
    int stages, blocks;
    size_t smem;
};
constexpr size_t kRingSmem = 216 * 1024;   // of an SM, for all its blocks
// `fit`: blocks of an SM as far as registers go; fewer where they would leave less than three stages each
inline bool plan_ring(int fit, int64_t stage_bytes, RingPlan& r) {
    const auto stages = [&](int blocks) { return (int)((kRingSmem / blocks - 1024 - kRingHead) / stage_bytes); };
    r.blocks = fit < 1 ? 1 : fit;
    while (r.blocks > 1 && stages(r.blocks) < 3) --r.blocks;
    r.stages = stages(r.blocks);
    if (r.stages > kMaxStages) r.stages = kMaxStages;
    r.smem = kRingHead + (size_t)r.stages * stage_bytes;
    return r.stages >= 2;
}
// the opt-in to large shared memory, once per kernel and device
template <typename K>
bool allow_smem(K kernel, bool (&done)[64]) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
    if (!done[dev]) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingSmem) != cudaSuccess) {
            (void)cudaGetLastError();
            return false;
        }
        done[dev] = true;
    }
    return true;
}

inline bool desc_ok(const nq_block_norm_desc* d) {
    if (!d || d->rows < 0 || d->cols < 1 || d->rows_per_gate < 0 || !(d->eps >= 0.0f)) return false;
    if (d->post < NQ_NORM_NONE || d->post > NQ_NORM_LAYER || d->pre < NQ_NORM_NONE || d->pre > NQ_NORM_LAYER) return false;
    const bool f = d->x_dtype == NQ_F32, b = d->x_dtype == NQ_BF16;
    return (f && (d->y_dtype == NQ_F32 || d->y_dtype == NQ_BF16)) || (b && d->y_dtype == NQ_BF16);
}

// a tensor that may be absent: its pitch, its element alignment, and whether 16-byte accesses fit
inline int check(const void* p, int64_t ld, int esize, const nq_block_norm_desc* d, bool* vec) {
    if (!p) return NQ_OK;
    if (ld < d->cols) return NQ_ERR_INVALID_ARG;
    if (at(p) % esize) return NQ_ERR_ALIGNMENT;
    if ((at(p) & 15) || ((ld * esize) & 15)) *vec = false;
    return NQ_OK;
}
inline int check_vector(const float* p, bool* vec) {
    if (at(p) & 3) return NQ_ERR_ALIGNMENT;
    if (at(p) & 15) *vec = false;
    return NQ_OK;
}

}  // namespace
}  // namespace nq
