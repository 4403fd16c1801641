// Block norm: post-norm, gate, residual sum and pre-norm of a transformer block in one pass, and its backward pass.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/nq.h"
#include "nq_fp8.cuh"
#include "nq_internal.cuh"

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

__device__ __forceinline__ uint4 ld16(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

template <int NV, bool VEC>
__device__ __forceinline__ void load_row(const Cols<NV, VEC>& c, const bf16* row, float (&v)[NV][8]) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (VEC) {
            uint4 w = make_uint4(0u, 0u, 0u, 0u);
            if (c.has(k, 0)) w = ld16(row + c.col(k, 0));
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[k][2 * j] = __uint_as_float(u[j] << 16);
                v[k][2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] = c.has(k, j) ? __bfloat162float(row[c.col(k, j)]) : 0.0f;
        }
    }
}
template <int NV, bool VEC>
__device__ __forceinline__ void load_row(const Cols<NV, VEC>& c, const float* row, float (&v)[NV][8]) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (VEC) {
            uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
            if (c.has(k, 0)) { a = ld16(row + c.col(k, 0)); b = ld16(row + c.col(k, 0) + 4); }
            const uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] = __uint_as_float(u[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] = c.has(k, j) ? row[c.col(k, j)] : 0.0f;
        }
    }
}
// one piece of a parameter vector (cached: every row reads the same one); `none` where it is absent
template <int NV, bool VEC>
__device__ __forceinline__ void load_param(const Cols<NV, VEC>& c, const float* vec, float none, int k, float (&v)[8]) {
    if (!vec) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = none;
    } else if (VEC) {
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
        if (c.has(k, 0)) {
            a = __ldg(reinterpret_cast<const float4*>(vec + c.col(k, 0)));
            b = __ldg(reinterpret_cast<const float4*>(vec + c.col(k, 0) + 4));
        }
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c.has(k, j) ? __ldg(vec + c.col(k, j)) : 0.0f;
    }
}

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}
template <int NV, bool VEC>
__device__ __forceinline__ void store_piece(const Cols<NV, VEC>& c, bf16* row, int k, const float (&v)[8]) {
    if (VEC) {
        if (c.has(k, 0))
            *reinterpret_cast<uint4*>(row + c.col(k, 0)) =
                make_uint4(bf16x2(v[0], v[1]), bf16x2(v[2], v[3]), bf16x2(v[4], v[5]), bf16x2(v[6], v[7]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c.has(k, j)) row[c.col(k, j)] = __float2bfloat16_rn(v[j]);
    }
}
template <int NV, bool VEC>
__device__ __forceinline__ void store_piece(const Cols<NV, VEC>& c, float* row, int k, const float (&v)[8]) {
    if (VEC) {
        if (c.has(k, 0)) {
            *reinterpret_cast<float4*>(row + c.col(k, 0)) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(row + c.col(k, 0) + 4) = make_float4(v[4], v[5], v[6], v[7]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c.has(k, j)) row[c.col(k, j)] = v[j];
    }
}
// the low bytes of q, four to a word
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

// Sums of N values over the threads of a row.  Up to one warp: shuffles alone.  More: the warps' sums through shared
// memory; the two halves of `box` alternate, so that one barrier a call is enough.  Every thread adds in the same
// order, so all hold the same bits.
template <int N>
struct TeamSum {
    float (*box)[32][N];
    int half, warps;
    __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) v[n] += __shfl_xor_sync(0xffffffffu, v[n], d);
        if (warps == 1) return;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
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

struct NormArgs {
    long long rows;
    int cols;
    const void *x, *y;
    void *r, *h;
    float* hs;
    const float *post_weight, *post_bias, *gate, *pre_weight, *pre_bias;
    long long ldx, ldy, ldr, ldh, ldhs, rows_per_gate;
    int h_dtype, post, pre;
    float skip, branch, eps, inv_cols, inv_h_scale;
};

// v -> v^ in place
template <int NV, bool VEC, typename Sum>
__device__ __forceinline__ void standardise(const Cols<NV, VEC>& c, float (&v)[NV][8], int kind, float inv_cols, float eps, Sum& sum) {
    if (kind == NQ_NORM_LAYER) {
        float m[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) m[0] += v[k][j];
        sum(m);
        const float mean = m[0] * inv_cols;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] = c.has(k, j) ? v[k][j] - mean : 0.0f;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) q[0] = fmaf(v[k][j], v[k][j], q[0]);
    sum(q);
    const float inv = rsqrtf(fmaf(q[0], inv_cols, eps));
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[k][j] *= inv;
}

// One row at a time to a team of threads (a warp, or the whole block when a row needs more), the row in registers
// throughout: each tensor is touched once, so the pass is bound by memory.
template <typename TX, typename TY, int NV, bool VEC>
__global__ void __launch_bounds__(512) block_norm_kernel(const NormArgs p, int threads) {
    __shared__ float box[2][32][1];
    const int team = threadIdx.x / threads, teams = blockDim.x / threads;
    const Cols<NV, VEC> c{(int)threadIdx.x - team * threads, threads, p.cols};
    TeamSum<1> sum{box, 0, threads >> 5};
    start_next();
    wait_previous();
    for (long long row = (long long)blockIdx.x * teams + team; row < p.rows; row += (long long)gridDim.x * teams) {
        float r[NV][8];
        load_row(c, static_cast<const TX*>(p.x) + row * p.ldx, r);
        if (p.y) {
            float u[NV][8];
            load_row(c, static_cast<const TY*>(p.y) + row * p.ldy, u);
            if (p.post != NQ_NORM_NONE) standardise(c, u, p.post, p.inv_cols, p.eps, sum);
            const float* gate = p.gate ? p.gate + (p.rows_per_gate ? row / p.rows_per_gate : 0) * p.cols : nullptr;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float w[8], b[8], g[8];
                load_param(c, p.post_weight, 1.0f, k, w);
                load_param(c, p.post_bias, 0.0f, k, b);
                load_param(c, gate, 1.0f, k, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) r[k][j] = fmaf(p.skip, r[k][j], p.branch * g[j] * fmaf(u[k][j], w[j], b[j]));
            }
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) r[k][j] *= p.skip;
        }
        if (p.r) {
#pragma unroll
            for (int k = 0; k < NV; ++k) store_piece(c, static_cast<TX*>(p.r) + row * p.ldr, k, r[k]);
        }
        if (p.pre == NQ_NORM_NONE) continue;
        standardise(c, r, p.pre, p.inv_cols, p.eps, sum);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float w[8], b[8];
            load_param(c, p.pre_weight, 1.0f, k, w);
            load_param(c, p.pre_bias, 0.0f, k, b);
            float h[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = c.has(k, j) ? fmaf(r[k][j], w[j], b[j]) : 0.0f;
            if (p.h_dtype == NQ_BF16) {
                store_piece(c, static_cast<bf16*>(p.h) + row * p.ldh, k, h);
            } else if (p.h_dtype == NQ_F32) {
                store_piece(c, static_cast<float*>(p.h) + row * p.ldh, k, h);
            } else if (p.h_dtype == NQ_I8) {
                uint32_t q[2] = {0u, 0u};
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int i = max(-128, min(127, __float2int_rn(__fmul_rn(h[j], p.inv_h_scale))));
                    q[j / 4] |= (uint32_t)(i & 255) << (8 * (j & 3));
                }
                store_bytes8(c, static_cast<uint8_t*>(p.h) + row * p.ldh, k, q[0], q[1]);
            } else {
                // groups of 128 columns: 16 lanes of 8 neighbours each, or all lanes of four elements each
                uint32_t m[2] = {0u, 0u};
#pragma unroll
                for (int j = 0; j < 8; ++j) m[j / 4] = max(m[j / 4], __float_as_uint(h[j]) & 0x7fffffffu);
                if (VEC) {
                    m[0] = max(m[0], m[1]);
#pragma unroll
                    for (int d = 8; d > 0; d >>= 1) m[0] = max(m[0], __shfl_xor_sync(0xffffffffu, m[0], d));
                    m[1] = m[0];
                } else {
                    m[0] = __reduce_max_sync(0xffffffffu, m[0]);
                    m[1] = __reduce_max_sync(0xffffffffu, m[1]);
                }
                float s[2], inv[2];
                group_scale(m[0], s[0], inv[0]);
                s[1] = s[0]; inv[1] = inv[0];
                if (!VEC) group_scale(m[1], s[1], inv[1]);
                if ((c.t & (VEC ? 15 : 31)) == 0) {
#pragma unroll
                    for (int i = 0; i < (VEC ? 1 : 2); ++i)
                        if (c.has(k, 4 * i)) p.hs[(long long)(c.col(k, 4 * i) >> 7) * p.ldhs + row] = s[i];
                }
                store_bytes8(c, static_cast<uint8_t*>(p.h) + row * p.ldh, k,
                             e4m3x4(h[0] * inv[0], h[1] * inv[0], h[2] * inv[0], h[3] * inv[0]),
                             e4m3x4(h[4] * inv[1], h[5] * inv[1], h[6] * inv[1], h[7] * inv[1]));
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------------- backward
struct BackArgs {
    long long rows;
    int cols;
    const void *r, *y, *dr, *dh;
    void *dx, *dy;
    const float *post_weight, *post_bias, *gate, *pre_weight;
    long long ldr, ldy, lddr, lddh, lddx, lddy;
    long long group_rows, chunk_rows;      // rows that share a gate row, and rows of one work item of theirs
    int chunks;                            // work items of a group
    long long items;
    int post, pre;
    float skip, branch, eps, inv_cols;
    float* gate_part;                      // [items, cols] sums for dgate (dgate itself when chunks == 1), or null
    float* part;                           // [4][blocks][cols]: dpre_weight, dpre_bias, dpost_weight, dpost_bias of each block
};

// Row statistics are computed again from r and y (a row is in registers anyway).  With xh, yh the standardised rows:
//   g  = dr + inv_r * (w dh - mean(w dh) - xh * mean(w dh xh))        (mean(w dh) for NQ_NORM_LAYER only)
//   dx = skip * g;  du = branch * gate * g
//   dy = inv_y * (w du - mean(w du) - yh * mean(w du yh))
// Column sums kept in registers: P = sum dh xh, sum dh (for the pre norm's weight and bias) over all rows of the thread
// block, A = sum g yh, sum g over the rows of one work item, which lie under one gate row: from A follow both
// dgate = branch * (w A0 + b A1) and the item's share branch * gate * A of the post norm's weight and bias.
template <typename TX, typename TY, int NV, bool VEC>
__global__ void __launch_bounds__(512) block_norm_backward_kernel(const BackArgs p) {
    __shared__ float box1[2][32][1];
    __shared__ float box2[2][32][2];
    const int threads = blockDim.x;
    const Cols<NV, VEC> c{(int)threadIdx.x, threads, p.cols};
    TeamSum<1> sum1{box1, 0, threads >> 5};
    TeamSum<2> sum2{box2, 0, threads >> 5};
    const long long plane = (long long)gridDim.x * p.cols, mine = (long long)blockIdx.x * p.cols;

    float P0[NV][8], P1[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) P0[k][j] = P1[k][j] = 0.0f;
    bool first = true;
    start_next();
    wait_previous();

    for (long long item = blockIdx.x; item < p.items; item += gridDim.x) {
        const long long group = item / p.chunks;
        const long long row0 = group * p.group_rows + (item - group * p.chunks) * p.chunk_rows;
        long long row1 = min(row0 + p.chunk_rows, (group + 1) * p.group_rows);
        row1 = min(row1, p.rows);
        const float* gate = p.gate ? p.gate + group * p.cols : nullptr;
        float A0[NV][8], A1[NV][8];
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) A0[k][j] = A1[k][j] = 0.0f;

        for (long long row = row0; row < row1; ++row) {
            float g[NV][8], v[NV][8];
            if (p.dr) {
                load_row(c, static_cast<const TX*>(p.dr) + row * p.lddr, g);
            } else {
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[k][j] = 0.0f;
            }
            if (p.pre != NQ_NORM_NONE) {
                float e[NV][8];
                load_row(c, static_cast<const TX*>(p.r) + row * p.ldr, v);
                load_row(c, static_cast<const TY*>(p.dh) + row * p.lddh, e);
                if (p.pre == NQ_NORM_LAYER) {
                    float m[1] = {0.0f};
#pragma unroll
                    for (int k = 0; k < NV; ++k)
#pragma unroll
                        for (int j = 0; j < 8; ++j) m[0] += v[k][j];
                    sum1(m);
                    const float mean = m[0] * p.inv_cols;
#pragma unroll
                    for (int k = 0; k < NV; ++k)
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[k][j] = c.has(k, j) ? v[k][j] - mean : 0.0f;
                }
                float q[1] = {0.0f};
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) q[0] = fmaf(v[k][j], v[k][j], q[0]);
                sum1(q);
                const float inv = rsqrtf(fmaf(q[0], p.inv_cols, p.eps));
                float d[2] = {0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    float w[8];
                    load_param(c, p.pre_weight, 1.0f, k, w);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        v[k][j] *= inv;
                        P0[k][j] = fmaf(e[k][j], v[k][j], P0[k][j]);
                        P1[k][j] += e[k][j];
                        e[k][j] *= w[j];
                        d[0] = fmaf(e[k][j], v[k][j], d[0]);
                        d[1] += e[k][j];
                    }
                }
                sum2(d);
                const float dot = d[0] * p.inv_cols, mean = p.pre == NQ_NORM_LAYER ? d[1] * p.inv_cols : 0.0f;
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[k][j] = fmaf(inv, e[k][j] - mean - v[k][j] * dot, g[k][j]);
            }
            if (p.dx) {
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    float o[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[j] = p.skip * g[k][j];
                    store_piece(c, static_cast<TX*>(p.dx) + row * p.lddx, k, o);
                }
            }
            if (!p.y) continue;
            load_row(c, static_cast<const TY*>(p.y) + row * p.ldy, v);
            float inv = 1.0f;
            if (p.post == NQ_NORM_LAYER) {
                float m[1] = {0.0f};
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) m[0] += v[k][j];
                sum1(m);
                const float mean = m[0] * p.inv_cols;
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[k][j] = c.has(k, j) ? v[k][j] - mean : 0.0f;
            }
            if (p.post != NQ_NORM_NONE) {
                float q[1] = {0.0f};
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) q[0] = fmaf(v[k][j], v[k][j], q[0]);
                sum1(q);
                inv = rsqrtf(fmaf(q[0], p.inv_cols, p.eps));
            }
            float d[2] = {0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float w[8], gt[8];
                load_param(c, p.post_weight, 1.0f, k, w);
                load_param(c, gate, 1.0f, k, gt);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (!c.has(k, j)) g[k][j] = 0.0f;
                    v[k][j] *= inv;
                    A0[k][j] = fmaf(g[k][j], v[k][j], A0[k][j]);
                    A1[k][j] += g[k][j];
                    g[k][j] *= p.branch * gt[j] * w[j];
                    d[0] = fmaf(g[k][j], v[k][j], d[0]);
                    d[1] += g[k][j];
                }
            }
            if (!p.dy) continue;
            float dot = 0.0f, mean = 0.0f;
            if (p.post != NQ_NORM_NONE) {
                sum2(d);
                dot = d[0] * p.inv_cols;
                if (p.post == NQ_NORM_LAYER) mean = d[1] * p.inv_cols;
            }
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = inv * (g[k][j] - mean - v[k][j] * dot);
                store_piece(c, static_cast<TY*>(p.dy) + row * p.lddy, k, o);
            }
        }
        if (p.y) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float w[8], b[8], gt[8];
                load_param(c, p.post_weight, 1.0f, k, w);
                load_param(c, p.post_bias, 0.0f, k, b);
                load_param(c, gate, 1.0f, k, gt);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (!c.has(k, j)) continue;
                    const int col = c.col(k, j);
                    if (p.gate_part) p.gate_part[item * p.cols + col] = p.branch * fmaf(w[j], A0[k][j], b[j] * A1[k][j]);
                    if (p.post != NQ_NORM_NONE) {
                        float* at = p.part + 2 * plane + mine + col;
                        const float s = p.branch * gt[j];
                        at[0] = fmaf(s, A0[k][j], first ? 0.0f : at[0]);
                        at[plane] = fmaf(s, A1[k][j], first ? 0.0f : at[plane]);
                    }
                }
            }
            first = false;
        }
    }
    if (p.pre != NQ_NORM_NONE) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c.has(k, j)) {
                    p.part[mine + c.col(k, j)] = P0[k][j];
                    p.part[plane + mine + c.col(k, j)] = P1[k][j];
                }
    }
}

// Joins the partial sums: plane z < 4 is one of the four vectors over all blocks, the others are the gate's groups.
struct JoinArgs {
    const float* part;
    const float* gate_part;
    float* out[4];                         // dpre_weight, dpre_bias, dpost_weight, dpost_bias
    float* dgate;
    int cols, col_blocks, blocks, chunks;
    long long groups;
};
constexpr int kJoinCols = 32, kJoinSlices = 8;
__global__ void __launch_bounds__(kJoinCols* kJoinSlices) block_norm_join_kernel(const JoinArgs p) {
    __shared__ float box[kJoinSlices][kJoinCols];
    const int lane = threadIdx.x % kJoinCols, slice = threadIdx.x / kJoinCols;
    const int col = (int)(blockIdx.x % p.col_blocks) * kJoinCols + lane;
    start_next();
    wait_previous();
    for (long long z = blockIdx.x / p.col_blocks; z < 4 + p.groups; z += gridDim.x / p.col_blocks) {
        float* out = z < 4 ? p.out[z] : p.dgate + (z - 4) * p.cols;
        if (!out) continue;                                          // the same for the whole block
        const int n = z < 4 ? p.blocks : p.chunks;
        const float* in = z < 4 ? p.part + z * p.blocks * (long long)p.cols : p.gate_part + (z - 4) * p.chunks * (long long)p.cols;
        float s = 0.0f;
        if (col < p.cols)
            for (int i = slice; i < n; i += kJoinSlices) s += in[(long long)i * p.cols + col];
        box[slice][lane] = s;
        __syncthreads();
        if (slice == 0 && col < p.cols) {
#pragma unroll
            for (int i = 1; i < kJoinSlices; ++i) s += box[i][lane];
            out[col] = s;
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------------------ host
inline uintptr_t at(const void* p) { return reinterpret_cast<uintptr_t>(p); }

struct Shape {
    int threads, nv;
};
// Threads of a row: 8 * nv columns each.
Shape shape_for(int64_t cols) {
    Shape s;
    s.nv = cols <= 512 * 8 ? 1 : cols <= 512 * 16 ? 2 : 4;
    s.threads = (int)((cols + 8 * s.nv - 1) / (8 * s.nv));
    s.threads = (s.threads + 31) / 32 * 32;
    return s;
}

bool desc_ok(const nq_block_norm_desc* d) {
    if (!d || d->rows < 0 || d->cols < 1 || d->rows_per_gate < 0 || !(d->eps >= 0.0f)) return false;
    if (d->post < NQ_NORM_NONE || d->post > NQ_NORM_LAYER || d->pre < NQ_NORM_NONE || d->pre > NQ_NORM_LAYER) return false;
    const bool f = d->x_dtype == NQ_F32, b = d->x_dtype == NQ_BF16;
    return (f && (d->y_dtype == NQ_F32 || d->y_dtype == NQ_BF16)) || (b && d->y_dtype == NQ_BF16);
}

// a tensor that may be absent: its pitch, its element alignment, and whether 16-byte accesses fit
int check(const void* p, int64_t ld, int esize, const nq_block_norm_desc* d, bool* vec) {
    if (!p) return NQ_OK;
    if (ld < d->cols) return NQ_ERR_INVALID_ARG;
    if (at(p) % esize) return NQ_ERR_ALIGNMENT;
    if ((at(p) & 15) || ((ld * esize) & 15)) *vec = false;
    return NQ_OK;
}
int check_vector(const float* p, bool* vec) {
    if (at(p) & 3) return NQ_ERR_ALIGNMENT;
    if (at(p) & 15) *vec = false;
    return NQ_OK;
}

template <typename TX, typename TY>
int launch_norm(const NormArgs& a, bool vec, cudaStream_t stream) {
    const Shape sh = shape_for(a.cols);
    const int teams = sh.threads == 32 ? 4 : 1, block = sh.threads * teams;
    long long grid = (a.rows + teams - 1) / teams;
    const long long most = (long long)sm_count() * (2048 / block);
    if (grid > most) grid = most;
    const auto run = [&](auto kernel) {
        return launch_chained(kernel, (unsigned)grid, block, 0, 1, stream, a, sh.threads);
    };
    if (vec) {
        if (sh.nv == 1) return run(block_norm_kernel<TX, TY, 1, true>);
        if (sh.nv == 2) return run(block_norm_kernel<TX, TY, 2, true>);
        return run(block_norm_kernel<TX, TY, 4, true>);
    }
    if (sh.nv == 1) return run(block_norm_kernel<TX, TY, 1, false>);
    if (sh.nv == 2) return run(block_norm_kernel<TX, TY, 2, false>);
    return run(block_norm_kernel<TX, TY, 4, false>);
}

// Work items of the backward pass: each gate row's rows in equal chunks, about as many items as blocks are wanted.
struct BackPlan {
    Shape shape;
    long long group_rows, groups, chunk_rows, items;
    int chunks, blocks;
};
BackPlan plan_backward(const nq_block_norm_desc* d, bool has_gate) {
    BackPlan p;
    p.shape = shape_for(d->cols);
    p.group_rows = has_gate && d->rows_per_gate > 0 ? d->rows_per_gate : (d->rows > 0 ? d->rows : 1);
    if (p.group_rows > d->rows && d->rows > 0) p.group_rows = d->rows;
    p.groups = (d->rows + p.group_rows - 1) / p.group_rows;
    const int per_sm = 1024 / p.shape.threads < 1 ? 1 : 1024 / p.shape.threads;
    const long long want = (long long)sm_count() * per_sm;
    long long chunks = p.groups ? want / p.groups : 1;
    if (chunks < 1) chunks = 1;
    if (chunks > (p.group_rows + 3) / 4) chunks = (p.group_rows + 3) / 4;       // a few rows each
    p.chunk_rows = (p.group_rows + chunks - 1) / chunks;
    p.chunks = (int)((p.group_rows + p.chunk_rows - 1) / p.chunk_rows);
    p.items = p.groups * p.chunks;
    p.blocks = (int)(p.items < want ? p.items : want);
    return p;
}

template <typename TX, typename TY>
int launch_back(const BackArgs& a, const BackPlan& pl, bool vec, cudaStream_t stream) {
    const auto run = [&](auto kernel) {
        return launch_chained(kernel, (unsigned)pl.blocks, pl.shape.threads, 0, 1, stream, a);
    };
    if (vec) {
        if (pl.shape.nv == 1) return run(block_norm_backward_kernel<TX, TY, 1, true>);
        if (pl.shape.nv == 2) return run(block_norm_backward_kernel<TX, TY, 2, true>);
        return run(block_norm_backward_kernel<TX, TY, 4, true>);
    }
    if (pl.shape.nv == 1) return run(block_norm_backward_kernel<TX, TY, 1, false>);
    if (pl.shape.nv == 2) return run(block_norm_backward_kernel<TX, TY, 2, false>);
    return run(block_norm_backward_kernel<TX, TY, 4, false>);
}

}  // namespace
}  // namespace nq

extern "C" {

int nq_block_norm(const nq_block_norm_desc* d, const void* X, const void* Y, const float* post_weight, const float* post_bias,
                  const float* gate, const float* pre_weight, const float* pre_bias, void* R, void* H, float* Hs, int64_t ldhs,
                  void* stream) {
    using namespace nq;
    if (!desc_ok(d)) return NQ_ERR_INVALID_ARG;
    if (!Y && d->rows > 0 && (gate || d->post != NQ_NORM_NONE)) return NQ_ERR_INVALID_ARG;
    if ((d->post == NQ_NORM_NONE && (post_weight || post_bias)) || (d->pre == NQ_NORM_NONE && (pre_weight || pre_bias || H)))
        return NQ_ERR_INVALID_ARG;
    if (d->h_dtype < NQ_F32 || d->h_dtype > NQ_I8) return NQ_ERR_INVALID_ARG;
    if (d->pre != NQ_NORM_NONE && d->h_dtype == NQ_I8 && !(d->h_scale > 0.0f)) return NQ_ERR_INVALID_ARG;
    if (d->cols > kMaxCols) return NQ_ERR_UNSUPPORTED;
    if (d->rows == 0) return NQ_OK;
    if (!X || (!R && !H) || (d->pre != NQ_NORM_NONE && !H)) return NQ_ERR_INVALID_ARG;
    const bool fp8 = H && d->h_dtype == NQ_E4M3;
    if (fp8 && (!Hs || ldhs < d->rows)) return NQ_ERR_INVALID_ARG;
    const int xs = d->x_dtype == NQ_BF16 ? 2 : 4, ys = d->y_dtype == NQ_BF16 ? 2 : 4;
    const int hs = d->h_dtype == NQ_F32 ? 4 : d->h_dtype == NQ_BF16 ? 2 : 1;
    bool vec = d->cols % 8 == 0, byte_vec = true;
    for (int st : {check(X, d->ldx, xs, d, &vec), check(Y, d->ldy, ys, d, &vec), check(R, d->ldr, xs, d, &vec),
                   check(H, d->ldh, hs, d, hs == 1 ? &byte_vec : &vec), check_vector(post_weight, &vec), check_vector(post_bias, &vec),
                   check_vector(gate, &vec), check_vector(pre_weight, &vec), check_vector(pre_bias, &vec)})
        if (st != NQ_OK) return st;
    if (!byte_vec || (fp8 && (at(Hs) & 3))) return NQ_ERR_ALIGNMENT;
    NormArgs a;
    a.rows = d->rows; a.cols = (int)d->cols; a.x = X; a.y = Y; a.r = R; a.h = H; a.hs = Hs;
    a.post_weight = post_weight; a.post_bias = post_bias; a.gate = gate; a.pre_weight = pre_weight; a.pre_bias = pre_bias;
    a.ldx = d->ldx; a.ldy = d->ldy; a.ldr = d->ldr; a.ldh = d->ldh; a.ldhs = ldhs; a.rows_per_gate = d->rows_per_gate;
    a.h_dtype = d->h_dtype; a.post = d->post; a.pre = d->pre;
    a.skip = d->skip_scale; a.branch = d->branch_scale; a.eps = d->eps;
    a.inv_cols = 1.0f / (float)d->cols;
    a.inv_h_scale = d->h_dtype == NQ_I8 ? 1.0f / d->h_scale : 0.0f;
    const cudaStream_t s = (cudaStream_t)stream;
    if (d->x_dtype == NQ_BF16) return launch_norm<bf16, bf16>(a, vec, s);
    return d->y_dtype == NQ_BF16 ? launch_norm<float, bf16>(a, vec, s) : launch_norm<float, float>(a, vec, s);
}

int64_t nq_block_norm_backward_workspace_bytes(const nq_block_norm_desc* d, int has_gate) {
    using namespace nq;
    if (!desc_ok(d) || d->cols > kMaxCols) return -1;
    const BackPlan pl = plan_backward(d, has_gate != 0);
    return 4 * d->cols * (4ll * pl.blocks + (has_gate && pl.chunks > 1 ? pl.items : 0));
}

int nq_block_norm_backward(const nq_block_norm_desc* d, const void* R, const void* Y, const void* dR, const void* dH,
                           const float* post_weight, const float* post_bias, const float* gate, const float* pre_weight, void* dX,
                           void* dY, float* dgate, float* dpost_weight, float* dpost_bias, float* dpre_weight, float* dpre_bias,
                           void* workspace, int64_t workspace_bytes, void* stream) {
    using namespace nq;
    if (!desc_ok(d)) return NQ_ERR_INVALID_ARG;
    if (!Y && d->rows > 0 && (gate || dY || d->post != NQ_NORM_NONE)) return NQ_ERR_INVALID_ARG;
    if (dgate && !gate) return NQ_ERR_INVALID_ARG;
    if (d->post == NQ_NORM_NONE && (post_weight || post_bias || dpost_weight || dpost_bias)) return NQ_ERR_INVALID_ARG;
    if (d->pre == NQ_NORM_NONE && (pre_weight || dpre_weight || dpre_bias || dH)) return NQ_ERR_INVALID_ARG;
    if (d->cols > kMaxCols) return NQ_ERR_UNSUPPORTED;
    const cudaStream_t s = (cudaStream_t)stream;
    if (d->rows == 0) {                                              // the sums over no rows
        for (float* v : {dpost_weight, dpost_bias, dpre_weight, dpre_bias, d->rows_per_gate == 0 ? dgate : (float*)nullptr})
            if (v && cudaMemsetAsync(v, 0, d->cols * sizeof(float), s) != cudaSuccess) {
                (void)cudaGetLastError();
                return NQ_ERR_CUDA;
            }
        return NQ_OK;
    }
    if ((!dR && !dH) || (d->pre != NQ_NORM_NONE && (!dH || !R))) return NQ_ERR_INVALID_ARG;
    const int xs = d->x_dtype == NQ_BF16 ? 2 : 4, ys = d->y_dtype == NQ_BF16 ? 2 : 4;
    bool vec = d->cols % 8 == 0, any = true;
    for (int st : {check(R, d->ldr, xs, d, &vec), check(dR, d->lddr, xs, d, &vec), check(dX, d->lddx, xs, d, &vec),
                   check(Y, d->ldy, ys, d, &vec), check(dH, d->lddh, ys, d, &vec), check(dY, d->lddy, ys, d, &vec),
                   check_vector(post_weight, &vec), check_vector(post_bias, &vec), check_vector(gate, &vec), check_vector(pre_weight, &vec),
                   check_vector(dgate, &any), check_vector(dpost_weight, &any), check_vector(dpost_bias, &any),
                   check_vector(dpre_weight, &any), check_vector(dpre_bias, &any)})
        if (st != NQ_OK) return st;
    const BackPlan pl = plan_backward(d, gate != nullptr);
    if (!workspace || workspace_bytes < nq_block_norm_backward_workspace_bytes(d, gate != nullptr)) return NQ_ERR_WORKSPACE;
    if (at(workspace) & 15) return NQ_ERR_ALIGNMENT;
    BackArgs a;
    a.rows = d->rows; a.cols = (int)d->cols; a.r = R; a.y = Y; a.dr = dR; a.dh = dH; a.dx = dX; a.dy = dY;
    a.post_weight = post_weight; a.post_bias = post_bias; a.gate = gate; a.pre_weight = pre_weight;
    a.ldr = d->ldr; a.ldy = d->ldy; a.lddr = d->lddr; a.lddh = d->lddh; a.lddx = d->lddx; a.lddy = d->lddy;
    a.group_rows = pl.group_rows; a.chunk_rows = pl.chunk_rows; a.chunks = pl.chunks; a.items = pl.items;
    a.post = d->post; a.pre = d->pre;
    a.skip = d->skip_scale; a.branch = d->branch_scale; a.eps = d->eps; a.inv_cols = 1.0f / (float)d->cols;
    a.part = static_cast<float*>(workspace);
    float* gate_part = a.part + 4ll * pl.blocks * d->cols;
    a.gate_part = !dgate ? nullptr : pl.chunks == 1 ? dgate : gate_part;
    int st;
    if (d->x_dtype == NQ_BF16) st = launch_back<bf16, bf16>(a, pl, vec, s);
    else st = d->y_dtype == NQ_BF16 ? launch_back<float, bf16>(a, pl, vec, s) : launch_back<float, float>(a, pl, vec, s);
    if (st != NQ_OK) return st;
    const bool join_gate = dgate && pl.chunks > 1;
    if (!join_gate && !dpost_weight && !dpost_bias && !dpre_weight && !dpre_bias) return NQ_OK;
    JoinArgs j;
    j.part = a.part; j.gate_part = gate_part; j.dgate = dgate; j.cols = a.cols; j.blocks = pl.blocks; j.chunks = pl.chunks;
    j.out[0] = dpre_weight; j.out[1] = dpre_bias; j.out[2] = dpost_weight; j.out[3] = dpost_bias;
    j.groups = join_gate ? pl.groups : 0;
    const long long planes = 4 + j.groups;
    j.col_blocks = (int)((d->cols + kJoinCols - 1) / kJoinCols);
    return launch_chained(block_norm_join_kernel, (unsigned)(j.col_blocks * (planes < 1024 ? planes : 1024)), kJoinCols * kJoinSlices, 0, 1, s, j);
}

}  // extern "C"
