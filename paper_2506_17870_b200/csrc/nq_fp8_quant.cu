// e4m3 quantiser with a scale for each 1 x 128 group or 128 x 128 block, the matrix and its transpose in one pass.
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/nq.h"
#include "nq_fp8.cuh"
#include "nq_internal.cuh"

namespace nq {
namespace {

constexpr int kTile = 128;
constexpr int kThreads = 256;

struct QuantArgs {
    const void* x;
    long long ldx;
    int rows, cols;
    int col_tiles;
    uint8_t* q;
    long long ldq;
    float* s;
    long long lds;
    uint8_t* qt;
    long long ldqt;
    float* st;
    long long ldst;
};

// 16 values of one row as the thread holds them: bf16 stays packed (8 words), fp32 as it is.
template <typename T>
struct Row16 {
    static constexpr int kWords = sizeof(T) * 4;
    uint32_t w[kWords];
    __device__ __forceinline__ uint32_t abs_bits_max() const {
        if (sizeof(T) == 2) {
            uint32_t m = w[0] & 0x7fff7fffu;
#pragma unroll
            for (int i = 1; i < kWords; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
            return max(m & 0xffff0000u, m << 16);
        }
        uint32_t m = w[0] & 0x7fffffffu;
#pragma unroll
        for (int i = 1; i < kWords; ++i) m = max(m, w[i] & 0x7fffffffu);
        return m;
    }
    __device__ __forceinline__ uint32_t bits(int j) const {
        if (sizeof(T) == 2) return (j & 1) ? (w[j / 2] & 0xffff0000u) : (w[j / 2] << 16);
        return w[j % kWords];
    }
    __device__ __forceinline__ uint64_t pair(int j) const { return pack2(bits(2 * j), bits(2 * j + 1)); }   // columns 2 j, 2 j + 1
};
// Largest magnitudes of a column, or (bf16) of two neighbouring ones in a word.
template <typename T>
__device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) { return sizeof(T) == 2 ? __vmaxu2(a, b) : max(a, b); }
template <typename T>
__device__ __forceinline__ uint32_t abs_word(uint32_t a) { return sizeof(T) == 2 ? a & 0x7fff7fffu : a & 0x7fffffffu; }

__device__ __forceinline__ void ldg_32(const void* p, uint32_t* w) {
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
}

// n (1..16) bytes of v to a 16-byte aligned place
__device__ __forceinline__ void store_bytes(uint8_t* dst, uint4 v, int n) {
    if (n >= 16) {
        *reinterpret_cast<uint4*>(dst) = v;
        return;
    }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < n) dst[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
}

// One thread block per 128 x 128 tile: a tile holds whole groups in both directions, so the matrix is read once
// however many outputs are wanted.  Thread t holds rows 4 * (t / 8) + {0..3}, columns 16 * (t % 8) + {0..15}: 32 (fp32:
// 64) contiguous bytes a row to load, 16 to store, and for the transpose four rows of a column make one 32-bit word.
// 16384 x 8192 bf16 both ways: 87 us replayed from a graph, 6.3 TB/s (0.96 of the measured copy rate), 97 - 98 us by calls that
// each take fresh outputs (0.85); 117 us at first, with scalar products and column maxima by shared-memory atomics; one way
// 61 us.  Bound by HBM.  Rows that start off 32 bytes (!ALIGNED) come element by element: 16384 x 5001 both ways 184 us in fp32
// and 97 us in bf16, against 75 and 50 at HBM rate.
// The transposed tile is put together in shared memory, its 16-byte pieces rotated by column / 16 so that neither
// the word writes (8 column groups x 4 row groups a warp) nor the 16-byte reads meet bank conflicts.
template <typename T, bool BLOCK, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 3 : 4) fp8_quantize_kernel(const QuantArgs p) {
    constexpr int kStagePitch = kTile + 16 / (int)sizeof(T);       // elements; rows 16-byte aligned
    constexpr int kWords = Row16<T>::kWords;
    __shared__ uint32_t s_colmax[kThreads / 32][kTile / 16 * kWords];
    __shared__ __align__(16) float s_colinv[kTile];
    __shared__ uint32_t s_blockmax[kThreads / 32];
    __shared__ __align__(16) uint32_t s_t[kTile * 32];
    extern __shared__ __align__(16) uint8_t s_stage[];             // !ALIGNED: the tile, row pitch kStagePitch elements

    const int tid = threadIdx.x, cg = tid & 7, rg = tid >> 3;
    const int r0 = (int)(blockIdx.x / p.col_tiles) * kTile, c0 = (int)(blockIdx.x % p.col_tiles) * kTile;
    const T* x = static_cast<const T*>(p.x);
    const int rows = min(kTile, p.rows - r0), cols = min(kTile, p.cols - c0);

    start_next();
    wait_previous();

    Row16<T> v[4];
    if (ALIGNED) {
        const int left = cols - 16 * cg;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 4 * rg + i;
#pragma unroll
            for (int w = 0; w < Row16<T>::kWords; ++w) v[i].w[w] = 0;
            if (row >= rows || left <= 0) continue;
            const T* src = x + (long long)(r0 + row) * p.ldx + c0 + 16 * cg;
            if (left >= 16) {
#pragma unroll
                for (int w = 0; w < Row16<T>::kWords; w += 8) ldg_32(reinterpret_cast<const uint8_t*>(src) + 4 * w, v[i].w + w);
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    if (j >= left) break;
                    if (sizeof(T) == 2)
                        v[i].w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(src)[j] << (16 * (j & 1));
                    else
                        v[i].w[j % Row16<T>::kWords] = reinterpret_cast<const uint32_t*>(src)[j];
                }
            }
        }
    } else {
        // rows that start anywhere: single elements, coalesced along the row, through shared memory
        T* stage = reinterpret_cast<T*>(s_stage);
        const int col = tid % kTile;
        const T* src = x + (long long)r0 * p.ldx + c0 + col;
#pragma unroll
        for (int half = 0; half < 4; ++half) {                       // sixteen loads in flight a thread
            T e[kTile * kTile / kThreads / 4];
#pragma unroll
            for (int i = 0; i < kTile * kTile / kThreads / 4; ++i) {
                const int row = half * (kTile / 4) + i * (kThreads / kTile) + tid / kTile;
                e[i] = row < rows && col < cols ? src[(long long)row * p.ldx] : T(0.0f);
            }
#pragma unroll
            for (int i = 0; i < kTile * kTile / kThreads / 4; ++i)
                stage[(half * (kTile / 4) + i * (kThreads / kTile) + tid / kTile) * kStagePitch + col] = e[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4* src = reinterpret_cast<const uint4*>(stage + (4 * rg + i) * kStagePitch + 16 * cg);
#pragma unroll
            for (int w = 0; w < Row16<T>::kWords / 4; ++w) {
                const uint4 t = src[w];
                v[i].w[4 * w] = t.x; v[i].w[4 * w + 1] = t.y; v[i].w[4 * w + 2] = t.z; v[i].w[4 * w + 3] = t.w;
            }
        }
    }

    uint32_t rowmax[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) rowmax[i] = v[i].abs_bits_max();

    float block_inv = 0.0f;
    if (BLOCK) {
        uint32_t m = __reduce_max_sync(0xffffffffu, max(max(rowmax[0], rowmax[1]), max(rowmax[2], rowmax[3])));
        if ((tid & 31) == 0) s_blockmax[tid >> 5] = m;
        __syncthreads();
        m = __reduce_max_sync(0xffffffffu, s_blockmax[tid & 7]);
        float s;
        group_scale(m, s, block_inv);
        if (tid == 0) {
            const long long rb = r0 / kTile, cb = c0 / kTile;
            if (p.s) p.s[cb * p.lds + rb] = s;
            if (p.st) p.st[rb * p.ldst + cb] = s;
        }
    }

    if (p.q) {
        const int left = cols - 16 * cg;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 4 * rg + i;
            float inv = block_inv;
            if (!BLOCK) {
                uint32_t m = rowmax[i];
                m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
                m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
                m = max(m, __shfl_xor_sync(0xffffffffu, m, 4));
                float s;
                group_scale(m, s, inv);
                if (cg == 0 && row < rows) p.s[(long long)(c0 / kTile) * p.lds + r0 + row] = s;
            }
            uint32_t o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = e4m3x4(mul2(v[i].pair(2 * j), both(inv)), mul2(v[i].pair(2 * j + 1), both(inv)));
            if (row < rows && left > 0)
                store_bytes(p.q + (long long)(r0 + row) * p.ldq + c0 + 16 * cg, make_uint4(o[0], o[1], o[2], o[3]), left);
        }
    }

    if (p.qt) {
        if (!BLOCK) {
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
                uint32_t m = abs_word<T>(v[0].w[w]);
#pragma unroll
                for (int i = 1; i < 4; ++i) m = max_word<T>(m, abs_word<T>(v[i].w[w]));
                m = max_word<T>(m, __shfl_xor_sync(0xffffffffu, m, 8));
                m = max_word<T>(m, __shfl_xor_sync(0xffffffffu, m, 16));
                if ((tid & 31) < 8) s_colmax[tid >> 5][kWords * cg + w] = m;
            }
            __syncthreads();
            if (tid < kTile) {
                const int word = sizeof(T) == 2 ? tid >> 1 : tid;
                uint32_t m = s_colmax[0][word];
#pragma unroll
                for (int i = 1; i < kThreads / 32; ++i) m = max_word<T>(m, s_colmax[i][word]);
                if (sizeof(T) == 2) m = (tid & 1) ? m & 0xffff0000u : m << 16;
                float s, inv;
                group_scale(m, s, inv);
                s_colinv[tid] = inv;
                if (tid < cols) p.st[(long long)(r0 / kTile) * p.ldst + c0 + tid] = s;
            }
            __syncthreads();
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int col = 16 * cg + 2 * j;
            const uint64_t inv = BLOCK ? both(block_inv) : *reinterpret_cast<const uint64_t*>(s_colinv + col);
            float lo[4], hi[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) unpack2(mul2(v[i].pair(j), inv), lo[i], hi[i]);
            const int at = (rg + 4 * cg) & 31;
            s_t[col * 32 + at] = e4m3x4(lo[0], lo[1], lo[2], lo[3]);
            s_t[(col + 1) * 32 + at] = e4m3x4(hi[0], hi[1], hi[2], hi[3]);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int col = i * 32 + rg;
            const uint4 o = *reinterpret_cast<const uint4*>(s_t + col * 32 + ((4 * (cg + (col >> 4))) & 31));
            const int left = rows - 16 * cg;
            if (col < cols && left > 0) store_bytes(p.qt + (long long)(c0 + col) * p.ldqt + r0 + 16 * cg, o, left);
        }
    }
}

template <typename T, bool BLOCK, bool ALIGNED>
int launch(const QuantArgs& a, long long tiles, cudaStream_t stream) {
    const int smem = ALIGNED ? 0 : kTile * (kTile + 16 / (int)sizeof(T)) * (int)sizeof(T);
    if (smem > 24 * 1024) {                                          // beside the 17.5 KB of static arrays
        if (cudaFuncSetAttribute(fp8_quantize_kernel<T, BLOCK, ALIGNED>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
            (void)cudaGetLastError();
            return NQ_ERR_CUDA;
        }
    }
    return launch_chained(fp8_quantize_kernel<T, BLOCK, ALIGNED>, (unsigned)tiles, kThreads, smem, 1, stream, a);
}

template <typename T>
int launch_type(const QuantArgs& a, bool block, bool aligned, long long tiles, cudaStream_t s) {
    if (block) return aligned ? launch<T, true, true>(a, tiles, s) : launch<T, true, false>(a, tiles, s);
    return aligned ? launch<T, false, true>(a, tiles, s) : launch<T, false, false>(a, tiles, s);
}

}  // namespace
}  // namespace nq

extern "C" int nq_fp8_quantize(const void* X, int64_t ldx, int x_dtype, int64_t rows, int64_t cols, int block_rows, void* Q,
                               int64_t ldq, float* S, int64_t lds, void* Qt, int64_t ldqt, float* St, int64_t ldst, void* stream) {
    if (rows < 0 || cols < 0 || (x_dtype != NQ_F32 && x_dtype != NQ_BF16) || (block_rows != 1 && block_rows != 128)) return NQ_ERR_INVALID_ARG;
    if ((Q == nullptr) != (S == nullptr) || (Qt == nullptr) != (St == nullptr)) return NQ_ERR_INVALID_ARG;
    if (rows >= 0x7fffff80ll || cols >= 0x7fffff80ll) return NQ_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return NQ_OK;
    if (!X || (!Q && !Qt) || ldx < cols) return NQ_ERR_INVALID_ARG;
    const int64_t row_tiles = (rows + 127) / 128, col_tiles = (cols + 127) / 128;
    if (Q && (ldq < cols || lds < (block_rows == 1 ? rows : row_tiles))) return NQ_ERR_INVALID_ARG;
    if (Qt && (ldqt < rows || ldst < (block_rows == 1 ? cols : col_tiles))) return NQ_ERR_INVALID_ARG;
    const int esize = x_dtype == NQ_BF16 ? 2 : 4;
    const auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
    if ((at(X) & (esize - 1)) || (at(S) & 3) || (at(St) & 3) || (at(Q) & 15) || (at(Qt) & 15)) return NQ_ERR_ALIGNMENT;
    if ((Q && (ldq & 15)) || (Qt && (ldqt & 15))) return NQ_ERR_ALIGNMENT;
    if (row_tiles * col_tiles > 0x7fffffffll) return NQ_ERR_UNSUPPORTED;
    nq::QuantArgs a;
    a.x = X; a.ldx = ldx; a.rows = (int)rows; a.cols = (int)cols; a.col_tiles = (int)col_tiles;
    a.q = static_cast<uint8_t*>(Q); a.ldq = ldq; a.s = S; a.lds = lds;
    a.qt = static_cast<uint8_t*>(Qt); a.ldqt = ldqt; a.st = St; a.ldst = ldst;
    const bool aligned = (at(X) & 31) == 0 && ((ldx * esize) & 31) == 0;
    const cudaStream_t s = (cudaStream_t)stream;
    return x_dtype == NQ_BF16 ? nq::launch_type<__nv_bfloat16>(a, block_rows == 128, aligned, row_tiles * col_tiles, s)
                              : nq::launch_type<float>(a, block_rows == 128, aligned, row_tiles * col_tiles, s);
}
