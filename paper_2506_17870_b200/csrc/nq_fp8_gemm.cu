// Product of e4m3 matrices with a scale for each block of 128: kernels and the entry point.
//
//   Y[m, n] = sum_g sa[g, m] * sb[g, n] * D_g[m, n] (+ bias[n]),   D_g = the 128-long inner products of group g
//
// tcgen05.mma (kind::f8f6f4) computes each D_g afresh in tensor memory; the epilogue warps read it, scale it and add it to
// accumulators that stay in registers for the whole of K ("promotion").  Two or more D buffers let the tensor core
// compute group g + 1 while group g is promoted.
//
// fp8_tile_kernel<NT>: one CTA per 128 (rows of B) x NT (rows of A) tile, K split over a cluster of up to 8 CTAs that join
//   their sums through distributed shared memory.  For few rows of A (the weights stream through shared memory once,
//   as the MMA's 128-row operand, so a single token wastes no bandwidth) and for outputs too small to fill the machine.
// fp8_pair_kernel<ROW_SCALES>: persistent CTA pairs (cta_group::2) on 256 x 256 tiles, for everything larger.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/nq.h"
#include "nq_fp8.cuh"
#include "nq_internal.cuh"
#include "nq_sm100.cuh"

namespace nq {
namespace {

using namespace sm100;

constexpr int kGroup = 128;              // K values of a scale group = bytes of a shared-memory row

struct Fp8Args {
    int M, N, k_blocks;
    const float* sa;
    const float* sb;
    long long ldsa, ldsb;
    int b_shift;                         // log2 of the rows of B that share a scale: 0 or 7
    const float* bias;
    void* y;
    long long ldy;
    int y_is_bf16, accumulate;
    unsigned int* status;
    int m_tiles, n_tiles;                // in tiles of the kernel that runs
    int split;                           // tile kernel: CTAs of a cluster, which share K
    int group_m;                         // pair kernel: M-tiles that share a band of N-tiles
    int y_tma;                           // pair kernel: Y is written with tile stores
};

__device__ __forceinline__ void store_out(const Fp8Args& p, long long m, int n, float v) {
    if (p.bias) v += p.bias[n];
    const long long at = m * p.ldy + n;
    if (p.y_is_bf16) {
        static_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(v);
    } else {
        float* y = static_cast<float*>(p.y) + at;
        *y = p.accumulate ? *y + v : v;
    }
}

__device__ __forceinline__ float half_of(uint64_t v, int which) {
    float lo, hi;
    unpack2(v, lo, hi);
    return which ? hi : lo;
}

// ------------------------------------------------------------------------------------------------------ tile kernel
constexpr int kTileThreads = 192;        // warp 0 TMA, warp 1 MMA and TMEM, warps 2-5 promotion (a 32-lane quarter each)
// Bound by latencies: 1 x 4096 x 4096 takes 7.2 us of which the weights' 17 MB are 2.6 at HBM rate (6.1 with the weights in L2),
// 37 x 8192 x 4096 11.7 us (5.2; 11.0 from L2), in a graph: launch, tensor memory, the first loads, and the two cluster barriers
// of the join.
template <int NT>
struct TileShape {
    static constexpr int kStageBytes = (128 + NT) * kGroup;
    static constexpr int kStages = NT == 16 ? 6 : NT == 32 ? 5 : 4;                     // two CTAs an SM: about 100 KB each
    static constexpr int kBufs = 4;                                                     // D buffers: 64 .. 256 TMEM columns
    static constexpr int kSmem = kStages * kStageBytes + 4 * 2 * NT * 4 + 512 + 1024;
    static_assert(NT * 128 * 4 <= kStages * kStageBytes, "the joined tile lies where the stages were");
};

template <int NT>
__global__ void __launch_bounds__(kTileThreads, 2)
fp8_tile_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const Fp8Args p) {
    using S = TileShape<NT>;
    constexpr int STAGES = S::kStages, BUFS = S::kBufs;
    constexpr uint32_t COLS = BUFS * NT;
    constexpr uint32_t IDESC = idesc_e4m3(128, NT);
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sW = smem;                                       // [STAGES][128 rows of B][128 B]
    uint8_t* sX = sW + STAGES * 128 * kGroup;                 // [STAGES][NT rows of A][128 B]
    float* sScale = reinterpret_cast<float*>(sX + STAGES * NT * kGroup);     // [4 warps][2][NT]
    uint64_t* full = reinterpret_cast<uint64_t*>(sScale + 4 * 2 * NT);
    uint64_t* empty = full + STAGES;
    uint64_t* tfull = empty + STAGES;
    uint64_t* tempty = tfull + BUFS;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tempty + BUFS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)(blockIdx.x % (unsigned)p.split);
    const int tile = (int)(blockIdx.x / (unsigned)p.split);
    const int n0 = (tile % p.n_tiles) * 128, m0 = (tile / p.n_tiles) * NT;
    const int kb0 = (int)((long long)p.k_blocks * rank / p.split), kb1 = (int)((long long)p.k_blocks * (rank + 1) / p.split);

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(smem_u32(&full[s]), 1); mbar_init(smem_u32(&empty[s]), 1); }
        for (int b = 0; b < BUFS; ++b) { mbar_init(smem_u32(&tfull[b]), 1); mbar_init(smem_u32(&tempty[b]), 4); }
        *abort_flag = 0;
        fence_barrier_init();
        prefetch_tensormap(&tmA);
        prefetch_tensormap(&tmB);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), COLS);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    start_next();
    wait_previous();

    uint64_t acc[NT / 2];                                      // pairs of neighbouring rows of A
#pragma unroll
    for (int c = 0; c < NT / 2; ++c) acc[c] = 0ull;
    const int quarter = warp & 3;
    const int nl = quarter * 32 + lane;                        // this lane's row of the B tile (promotion warps)

    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                const uint32_t s = it % STAGES, use = it / STAGES;
                if (!(ok = mbar_wait(smem_u32(&empty[s]), (use & 1) ^ 1, abort_flag, p.status, 0x210u))) break;
                const uint32_t bar = smem_u32(&full[s]);
                mbar_arrive_expect_tx(bar, S::kStageBytes);
                tma_load_2d(smem_u32(sW + s * 128 * kGroup), &tmB, kb * kGroup, n0, bar);
                tma_load_2d(smem_u32(sX + s * NT * kGroup), &tmA, kb * kGroup, m0, bar);
            }
            if (!ok) {
                const long long t0 = clock64();                // let copies in flight land before shared memory is released
                while (clock64() - t0 < (1ll << 22)) { }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            uint32_t it = 0;
            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                const uint32_t s = it % STAGES, use = it / STAGES, b = it % BUFS, buse = it / BUFS;
                if (!mbar_wait(smem_u32(&tempty[b]), (buse & 1) ^ 1, abort_flag, p.status, 0x220u)) break;
                if (!mbar_wait(smem_u32(&full[s]), use & 1, abort_flag, p.status, 0x221u)) break;
                tc_fence_after_sync();
                const uint64_t dw = smem_desc_sw128(smem_u32(sW + s * 128 * kGroup));
                const uint64_t dx = smem_desc_sw128(smem_u32(sX + s * NT * kGroup));
#pragma unroll
                for (int k = 0; k < kGroup / 32; ++k) mma_e4m3(tmem_base + b * NT, dw + 2 * k, dx + 2 * k, IDESC, k != 0);
                mma_commit(smem_u32(&empty[s]));
                mma_commit(smem_u32(&tfull[b]));
            }
        }
    } else {
        // Promotion: this lane holds one row of B against the NT rows of A.  The scales of A's rows are needed by every
        // lane: each warp keeps a group's NT of them in shared memory, fetched one group ahead.
        float* mine = sScale + (warp - 2) * 2 * NT;
        constexpr int PER = (NT + 31) / 32;
        const long long sb_row = (n0 + nl < p.N) ? (long long)((n0 + nl) >> p.b_shift) : -1;
        float next_b = 0.0f, next_a[PER];
        const auto fetch = [&](int kb) {
            next_b = sb_row >= 0 ? p.sb[(long long)kb * p.ldsb + sb_row] : 0.0f;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int c = i * 32 + lane;
                next_a[i] = (c < NT && m0 + c < p.M) ? p.sa[(long long)kb * p.ldsa + m0 + c] : 0.0f;
            }
        };
        if (kb0 < kb1) fetch(kb0);
        uint32_t it = 0;
        for (int kb = kb0; kb < kb1; ++kb, ++it) {
            const uint32_t b = it % BUFS, buse = it / BUFS;
            float* sc = mine + (it & 1) * NT;
            const uint64_t scale_b = both(next_b);
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (i * 32 + lane < NT) sc[i * 32 + lane] = next_a[i];
            __syncwarp();
            if (kb + 1 < kb1) fetch(kb + 1);
            bool ok = mbar_wait(smem_u32(&tfull[b]), buse & 1, abort_flag, p.status, 0x230u);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after_sync();
            const uint32_t from = tmem_base + b * NT + ((uint32_t)(quarter * 32) << 16);
            constexpr int PIECES = NT / 16;
            uint32_t d[2][16];
            tmem_ld_32x16(from, d[0]);
            if (PIECES > 1) tmem_ld_32x16(from + 16, d[1]);
#pragma unroll
            for (int c = 0; c < PIECES; ++c) {                 // two loads in flight, waited for in pairs
                if ((c & 1) == 0) {
                    tmem_ld_wait();
                    tmem_arrived(d[0]);
                    if (PIECES > 1) tmem_arrived(d[1]);
                    if (c + 2 >= PIECES) {                     // all have arrived
                        tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&tempty[b]));
                    }
                }
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(sc + c * 16 + 2 * j);
                    acc[c * 8 + j] = fma2(mul2(pack2(d[c & 1][2 * j], d[c & 1][2 * j + 1]), w.x), scale_b, acc[c * 8 + j]);
                    acc[c * 8 + j + 1] = fma2(mul2(pack2(d[c & 1][2 * j + 2], d[c & 1][2 * j + 3]), w.y), scale_b, acc[c * 8 + j + 1]);
                }
                if (c + 2 < PIECES) tmem_ld_32x16(from + (c + 2) * 16, d[c & 1]);
            }
        }
        if (p.split == 1) {
            if (n0 + nl < p.N)
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    if (m0 + c < p.M) store_out(p, m0 + c, n0 + nl, half_of(acc[c / 2], c & 1));
        } else {
            // every stage has been read by then: the last group's MMAs are complete, and so are all before them
            float* red = reinterpret_cast<float*>(smem);
#pragma unroll
            for (int c = 0; c < NT; ++c) red[c * 128 + nl] = half_of(acc[c / 2], c & 1);
        }
    }

    __syncwarp();
    if (p.split > 1) {
        cluster_sync_all();
        if (warp >= 2) {
            // CTA `rank` joins its share of the tile's rows of A, adding the ranks in order; a lane takes four neighbouring
            // columns, and four rows' loads from all ranks are on their way at once (a load from another CTA takes about a
            // microsecond: joined value by value, 37 tokens took 15.9 us)
            const int c0 = NT * rank / p.split, c1 = min(NT * (rank + 1) / p.split, p.M - m0);
            const uint32_t red = smem_u32(smem) + lane * 16;
            const int n = n0 + lane * 4;
            const bool vec = (p.ldy & 3) == 0 && (reinterpret_cast<uintptr_t>(p.y) & 15) == 0 && n + 4 <= p.N && !p.accumulate;
            float4 bias = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (p.bias && vec) bias = make_float4(p.bias[n], p.bias[n + 1], p.bias[n + 2], p.bias[n + 3]);
            for (int first = c0 + warp - 2; first < c1; first += 16) {
                float4 v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                for (int r = 0; r < p.split; ++r) {
                    const uint32_t from = map_to_cta(red, r);
                    float4 t[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (first + 4 * i < c1)
                            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(t[i].x), "=f"(t[i].y), "=f"(t[i].z), "=f"(t[i].w)
                                         : "r"(from + (first + 4 * i) * 512));
                        else
                            t[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                    for (int i = 0; i < 4; ++i) { v[i].x += t[i].x; v[i].y += t[i].y; v[i].z += t[i].z; v[i].w += t[i].w; }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = first + 4 * i;
                    if (c >= c1) break;
                    const long long m = m0 + c;
                    if (vec && p.y_is_bf16) {
                        const __nv_bfloat162 lo = __floats2bfloat162_rn(v[i].x + bias.x, v[i].y + bias.y), hi = __floats2bfloat162_rn(v[i].z + bias.z, v[i].w + bias.w);
                        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.y) + m * p.ldy + n) =
                            make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
                    } else if (vec) {
                        *reinterpret_cast<float4*>(static_cast<float*>(p.y) + m * p.ldy + n) =
                            make_float4(v[i].x + bias.x, v[i].y + bias.y, v[i].z + bias.z, v[i].w + bias.w);
                    } else {
                        if (n < p.N) store_out(p, m, n, v[i].x);
                        if (n + 1 < p.N) store_out(p, m, n + 1, v[i].y);
                        if (n + 2 < p.N) store_out(p, m, n + 2, v[i].z);
                        if (n + 3 < p.N) store_out(p, m, n + 3, v[i].w);
                    }
                }
            }
        }
        __syncwarp();
        cluster_sync_all();                                    // nobody leaves while its sums are being read
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, COLS);
    }
}

// ------------------------------------------------------------------------------------------------------ pair kernel
// 256 x 256 tiles on CTA pairs, in two halves of 128 columns: a CTA stages its 128 rows of A and half of the rows of each
// half of B (32 KB a group of K) and gets 128 x 128 sums a half; four such buffers fill its tensor memory.  What bounds the
// rate is the hand-over of a buffer -- commit, promotion warps in BOTH CTAs read it, their signal travels to the
// leader's MMA thread: about a thousand cycles, against 512 in which the tensor core computes a group of 256 x 256.  With
// two buffers of 256 columns the tensor core waited for it every group (735 us for 8192^3, in a kernel that had neither the
// promotion warps of a half, nor two issuing threads, nor packed arithmetic yet; not tried again with them); with four of 128
// it has three others to fill meanwhile, at the price of reading A from shared memory twice.
// Eight promotion warps, two to a scheduler, one for each half: a warp reads 32 rows x 128 columns in four loads of 32, two in
// flight, and adds them to 128 accumulators a thread.  The two warps of a scheduler work half a group apart, so that the
// FMAs of one fall into the waits of the other (both on the same half, 64 columns each, they waited together: 8192^3 took
// 656 us; sixteen warps of 64 accumulators have no registers to take in what they add: 637 us).
// Measured: 8192^3 545 - 590 us one call at a time (1.9 - 2.0 PFLOP/s), 612 - 622 us back to back, where the power limit holds the
// clock near 1.5 GHz; 4096 x 4096 x 12608 with row scales 378 us in a graph, 400 - 405 by calls.  When 8192^3 took 520 - 536 us as
// a burst, the kernel without the FMAs took 430, and 430 without reading tensor memory either, where the products alone should
// take 339: that part is the tensor side's own, probably A read twice, and the rest the promotion's, 256 FMA cycles a
// scheduler and group (512 with row scales, which multiply twice) plus the waits that two warps cannot cover.  Adding to what Y
// holds (accumulate) goes by ordinary loads and stores: 4096 x 4096 x 12608 606 us, 768 x 768 x 2048 12.3 against 9.2.
// Barriers (at the same offsets in both CTAs): full[s] in the leader counts the bytes of both CTAs' loads; done[s][h], in
// each CTA, is arrived on by the commit of half h of the group in stage s: it hands the sums to the promotion warps, and
// both halves together free the stage for the producer (a waiter is never more than one phase behind: the next use of the
// stage needs the buffers back first); tempty[b] in the leader: the half's four promotion warps of both CTAs arrive;
// sfull[s] / sempty[s], private to a CTA (ROW_SCALES): the ring of column scales, filled by warp 2 with asynchronous copies.
constexpr int kPairThreads = 384;        // warp 0 TMA, warps 1 and 3 MMA (1 also TMEM), warp 2 column scales, warps 4-11 promotion
constexpr int kPairWarps = 8;
constexpr int kPairStages = 4;           // six are no faster; the room goes to the output
constexpr int kPairStageBytes = 2 * 128 * kGroup;
constexpr int kOutPiece = 32 * 64;       // 32 rows x 64 bytes of output, in the 64-byte swizzle
template <bool ROW_SCALES>
struct PairShape {
    static constexpr int kPieces = 4;                                                    // output pieces a warp fills before it hands them over
    static constexpr int kScales = ROW_SCALES ? 256 : 0;                                 // of a group: rows of B
    static constexpr int kSmem = kPairStages * (kPairStageBytes + kScales * 4) + kPairWarps * (kPieces * kOutPiece + 128 * 4) + 512 + 1024;
};

// one scale (or bias) to shared memory, asynchronously; zero where there is none (`any`: some readable address)
__device__ __forceinline__ void copy_scale(uint32_t dst, const float* src, bool present, const float* any) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(present ? src : any), "r"(present ? 4 : 0) : "memory");
}

// Tiles in groups of M-tiles that share a band of N-tiles, so that a group's rows of A stay in L2 while B goes by.
__device__ __forceinline__ void pair_tile(int tile, const Fp8Args& p, int& mt, int& nt) {
    const int per_group = p.group_m * p.n_tiles;
    const int first = tile / per_group * p.group_m;
    const int local = tile - first * p.n_tiles;
    const int height = min(p.group_m, p.m_tiles - first);
    nt = local / height;
    mt = first + local - nt * height;
}

// 32 rows x 64 bytes of finished values into a piece of shared memory, in the 64-byte swizzle.
__device__ __forceinline__ void fill_piece(uint8_t* piece, const uint32_t (&w)[16], int lane) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
        *reinterpret_cast<uint4*>(piece + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)) = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
}
// `count` filled pieces, side by side from column col0, to the output: by tile stores, or by ordinary ones that coalesce
// along the rows.
__device__ __forceinline__ void store_pieces(const Fp8Args& p, const CUtensorMap* tmY, uint8_t* pieces, int count, long long row0, int col0, int lane) {
    const int width = p.y_is_bf16 ? 32 : 16;                   // columns of a piece
    if (p.y_tma) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            for (int i = 0; i < count && col0 + i * width < p.N; ++i)
                tma_store_4d(tmY, smem_u32(pieces + i * kOutPiece), (col0 + i * width) * (p.y_is_bf16 ? 2 : 4), (int)row0, 0, 0);
            bulk_commit_group();
        }
        return;
    }
    __syncwarp();
    const long long rows = p.M - row0;
    for (int i = 0; i < count; ++i) {
        const uint8_t* piece = pieces + i * kOutPiece;
        const int col = col0 + i * width;
        if (p.y_is_bf16) {
            if (col + lane < p.N)
#pragma unroll 8
                for (int r = 0; r < 32; ++r)
                    if (r < rows)
                        static_cast<uint16_t*>(p.y)[(row0 + r) * p.ldy + col + lane] =
                            *reinterpret_cast<const uint16_t*>(piece + r * 64 + (((lane >> 3) ^ ((r >> 1) & 3)) << 4) + (lane & 7) * 2);
        } else {
            const int c = lane & 15;
            if (col + c < p.N)
#pragma unroll 8
                for (int k = 0; k < 16; ++k) {
                    const int r = 2 * k + (lane >> 4);
                    if (r < rows) {
                        float* y = static_cast<float*>(p.y) + (row0 + r) * p.ldy + col + c;
                        const float v = *reinterpret_cast<const float*>(piece + r * 64 + (((c >> 2) ^ ((r >> 1) & 3)) << 4) + (c & 3) * 4);
                        *y = p.accumulate ? *y + v : v;
                    }
                }
        }
    }
    __syncwarp();                                              // the pieces may be written again
}

template <bool ROW_SCALES>
__global__ void __launch_bounds__(kPairThreads, 1)
fp8_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmY,
                const Fp8Args p) {
    using S = PairShape<ROW_SCALES>;
    constexpr int STAGES = kPairStages;
    constexpr uint32_t IDESC = idesc_e4m3(256, 128);
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sA = smem;
    uint8_t* sB = sA + STAGES * 128 * kGroup;
    uint8_t* sOut = sB + STAGES * 128 * kGroup;
    float* sScale = reinterpret_cast<float*>(sOut + kPairWarps * S::kPieces * kOutPiece);
    float* sBias = sScale + STAGES * S::kScales;              // [8 warps][128]
    uint64_t* full = reinterpret_cast<uint64_t*>(sBias + kPairWarps * 128);
    uint64_t* done = full + STAGES;
    uint64_t* sfull = done + 2 * STAGES;
    uint64_t* sempty = sfull + STAGES;
    uint64_t* tempty = sempty + STAGES;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tempty + 4);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
    const int num_tiles = p.m_tiles * p.n_tiles;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(smem_u32(&full[s]), 1);
            mbar_init(smem_u32(&sfull[s]), 32);
            mbar_init(smem_u32(&sempty[s]), kPairWarps);
        }
        for (int s = 0; s < 2 * STAGES; ++s) mbar_init(smem_u32(&done[s]), 1);
        for (int b = 0; b < 4; ++b) mbar_init(smem_u32(&tempty[b]), kPairWarps);
        *abort_flag = 0;
        fence_barrier_init();
        prefetch_tensormap(&tmA);
        prefetch_tensormap(&tmB);
        if (p.y_tma) prefetch_tensormap(&tmY);
    }
    if (warp == 1) {
        tmem_alloc_pair(smem_u32(tmem_slot), 512);
        tmem_relinquish_pair();
    }
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync_all();                                        // both CTAs' barriers exist before anyone signals across
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    start_next();
    wait_previous();
    // 384 threads are launched with 168 registers each (64512); the promotion warps take 232 (256 x 232 = 59392), the
    // other four 40 (128 x 40 = 5120): together what was launched.
    if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");

    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            for (int tile = pair; ok && tile < num_tiles; tile += num_pairs) {
                int mt, nt;
                pair_tile(tile, p, mt, nt);
                const int row = mt * 256 + (int)rank * 128, brow = nt * 256 + (int)rank * 64;
                for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                    const uint32_t s = it % STAGES, use = it / STAGES;
                    if (!(ok = mbar_wait(smem_u32(&done[2 * s]), (use & 1) ^ 1, abort_flag, p.status, 0x310u))) break;
                    if (!(ok = mbar_wait(smem_u32(&done[2 * s + 1]), (use & 1) ^ 1, abort_flag, p.status, 0x311u))) break;
                    const uint32_t bar = map_to_cta(smem_u32(&full[s]), 0);
                    if (rank == 0) mbar_arrive_expect_tx(smem_u32(&full[s]), 2 * kPairStageBytes);
                    tma_load_2d_pair(smem_u32(sA + s * 128 * kGroup), &tmA, kb * kGroup, row, bar);
                    tma_load_2d_pair(smem_u32(sB + s * 128 * kGroup), &tmB, kb * kGroup, brow, bar);
                    tma_load_2d_pair(smem_u32(sB + s * 128 * kGroup + 64 * kGroup), &tmB, kb * kGroup, brow + 128, bar);
                }
            }
            if (!ok) {
                const long long t0 = clock64();                // let copies in flight land before shared memory is released
                while (clock64() - t0 < (1ll << 22)) { }
            }
        }
    } else if (warp == 1 || warp == 3) {
        // One thread issues the first halves, another the second: what a thread pays between two batches (a probe of a
        // barrier that is ready costs about 115 cycles, a commit 70) passes while the other's products are computed.
        if (lane == 0 && rank == 0) {
            const int h = warp >> 1;
            uint32_t it = 0;
            bool ok = true;
            for (int tile = pair; ok && tile < num_tiles; tile += num_pairs) {
                for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                    const uint32_t s = it % STAGES, use = it / STAGES, b = (2 * it + h) & 3;
                    if (!(ok = mbar_wait(smem_u32(&full[s]), use & 1, abort_flag, p.status, 0x321u))) break;
                    if (!(ok = mbar_wait(smem_u32(&tempty[b]), ((it >> 1) & 1) ^ 1, abort_flag, p.status, 0x320u))) break;
                    tc_fence_after_sync();
                    const uint64_t da = smem_desc_sw128(smem_u32(sA + s * 128 * kGroup));
                    const uint64_t db = smem_desc_sw128(smem_u32(sB + s * 128 * kGroup + h * 64 * kGroup));
#pragma unroll
                    for (int k = 0; k < kGroup / 32; ++k) mma_e4m3_pair(tmem_base + b * 128, da + 2 * k, db + 2 * k, IDESC, k != 0);
                    mma_commit_pair(smem_u32(&done[2 * s + h]));
                }
            }
        }
    } else if (warp == 2) {
        // column scales of each group, as many groups ahead as there are stages; outside the matrix they read as zero
        uint32_t it = 0;
        bool ok = true;
        for (int tile = pair; ROW_SCALES && ok && tile < num_tiles; tile += num_pairs) {
            int mt, nt;
            pair_tile(tile, p, mt, nt);
            const int col = nt * 256 + lane;
            for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                const uint32_t s = it % STAGES, use = it / STAGES;
                ok = mbar_wait(smem_u32(&sempty[s]), (use & 1) ^ 1, abort_flag, p.status, 0x340u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint32_t to = smem_u32(sScale + s * S::kScales + lane);
                const float* from = p.sb + (long long)kb * p.ldsb + col;
#pragma unroll
                for (int i = 0; i < 8; ++i) copy_scale(to + 128 * i, from + 32 * i, col + 32 * i < p.N, p.sb);
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&sfull[s])) : "memory");
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp >= 4) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        const int quarter = warp & 3, h = (warp - 4) >> 2;     // 32 rows of one half
        const uint32_t tmem_mine = tmem_base + h * 128 + ((uint32_t)(quarter * 32) << 16);
        uint8_t* pieces = sOut + (warp - 4) * S::kPieces * kOutPiece;
        float* my_bias = sBias + (warp - 4) * 128;
        // this row's scales and (blocks) the column block's, one group ahead
        const float *from_a = nullptr, *from_b = nullptr;
        float next_a = 0.0f, next_b = 1.0f;
        const auto fetch = [&]() {
            next_a = *from_a;
            from_a += p.ldsa;
            if (!ROW_SCALES) {
                next_b = *from_b;
                from_b += p.ldsb;
            }
        };
        const auto fetch_first = [&](int mt, int nt) {
            const long long row = (long long)mt * 256 + rank * 128 + quarter * 32 + lane;
            const int col = nt * 256 + h * 128;
            from_a = p.sa + (row < p.M ? row : 0);
            from_b = p.sb + (col < p.N ? col >> 7 : 0);
            fetch();
        };
        // whether this warp's part of a tile holds anything of Y
        const auto inside = [&](int m, int n) {
            return (long long)m * 256 + rank * 128 + quarter * 32 < p.M && n * 256 + h * 128 < p.N;
        };
        uint32_t it = 0;
        bool ok = true;
        int mt = 0, nt = 0;
        if (pair < num_tiles) {
            pair_tile(pair, p, mt, nt);
            fetch_first(mt, nt);
        }
        for (int tile = pair; ok && tile < num_tiles; tile += num_pairs) {
            // Needed at the tile's end; asynchronous, so it costs no registers.  A warp without anything to store starts no
            // copies: it would not wait for them, and copies of two tiles to one place are not ordered.
            if (p.bias && inside(mt, nt)) {
                __syncwarp();                                  // the last tile's have been read
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = nt * 256 + h * 128 + 32 * i + lane;
                    copy_scale(smem_u32(my_bias + 32 * i + lane), p.bias + c, c < p.N, p.bias);
                }
            }
            uint64_t acc[64];                                  // pairs of neighbouring columns
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = 0ull;
            for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                const uint32_t s = it % STAGES, parity = (it / STAGES) & 1;
                const float* col_scales = sScale + s * S::kScales + h * 128;
                const float scale = ROW_SCALES ? next_a : next_a * next_b;
                const uint64_t scale2 = pack2(__float_as_uint(scale), __float_as_uint(scale));
                if (kb + 1 < p.k_blocks) fetch();
                uint32_t d[2][32];
                const auto add = [&](int c) {
#pragma unroll
                    for (int j = 0; j < 16; j += 2) {
                        uint64_t v0 = pack2(d[c & 1][2 * j], d[c & 1][2 * j + 1]), v1 = pack2(d[c & 1][2 * j + 2], d[c & 1][2 * j + 3]);
                        if (ROW_SCALES) {
                            const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(col_scales + c * 32 + 2 * j);
                            v0 = mul2(v0, w.x);
                            v1 = mul2(v1, w.y);
                        }
                        acc[c * 16 + j] = fma2(v0, scale2, acc[c * 16 + j]);
                        acc[c * 16 + j + 1] = fma2(v1, scale2, acc[c * 16 + j + 1]);
                    }
                };
                const uint32_t b = (2 * it) & 3, from = tmem_mine + b * 128;
                ok = mbar_wait(smem_u32(&done[2 * s + h]), parity, abort_flag, p.status, 0x330u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after_sync();
                tmem_ld_32x32(from, d[0]);
                tmem_ld_32x32(from + 32, d[1]);
                if (ROW_SCALES) {
                    ok = mbar_wait(smem_u32(&sfull[s]), parity, abort_flag, p.status, 0x331u);
                    ok = __all_sync(0xffffffffu, ok);          // together again: what follows is for the whole warp
                }
                tmem_ld_wait();
                tmem_arrived(d[0]);
                tmem_arrived(d[1]);
                add(0);
                tmem_ld_32x32(from + 64, d[0]);
                add(1);
                tmem_ld_32x32(from + 96, d[1]);
                tmem_ld_wait();
                tmem_arrived(d[0]);
                tmem_arrived(d[1]);
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) {                               // the buffer goes back before its last sums are added
                    const uint32_t to = smem_u32(&tempty[b + h]);
                    if (rank == 0) mbar_arrive(to);
                    else mbar_arrive_cluster_relaxed(map_to_cta(to, 0));
                }
                add(2);
                add(3);
                if (ROW_SCALES) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&sempty[s]));
                    if (!ok) break;
                }
            }
            if (!ok) break;
            const long long row0 = (long long)mt * 256 + rank * 128 + quarter * 32;
            const int col = nt * 256 + h * 128;
            const bool empty = !inside(mt, nt);
            if (tile + num_pairs < num_tiles) {
                pair_tile(tile + num_pairs, p, mt, nt);
                fetch_first(mt, nt);
            }
            if (empty) continue;
            if (p.bias) {
                asm volatile("cp.async.wait_all;" ::: "memory");
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 64; i += 2) {
                    const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(my_bias + 2 * i);
                    acc[i] = add2(acc[i], v.x);
                    acc[i + 1] = add2(acc[i + 1], v.y);
                }
            }
            if (p.y_tma) {                                     // the pieces' last stores have read them
                if (lane == 0) bulk_wait_read_all();
                __syncwarp();
            }
            if (p.y_is_bf16) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float lo, hi;
                        unpack2(acc[c * 16 + j], lo, hi);
                        const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
                        w[j] = *reinterpret_cast<const uint32_t*>(&t);
                    }
                    fill_piece(pieces + c * kOutPiece, w, lane);
                }
                store_pieces(p, &tmY, pieces, 4, row0, col, lane);
            } else {
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    if (c == 4 && p.y_tma) {
                        if (lane == 0) bulk_wait_read_all();
                        __syncwarp();
                    }
                    uint32_t w[16];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        w[2 * j] = (uint32_t)acc[c * 8 + j];
                        w[2 * j + 1] = (uint32_t)(acc[c * 8 + j] >> 32);
                    }
                    fill_piece(pieces + (c & 3) * kOutPiece, w, lane);
                    if (c == 3) store_pieces(p, &tmY, pieces, 4, row0, col, lane);
                    if (c == 7) store_pieces(p, &tmY, pieces, 4, row0, col + 64, lane);
                }
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");       // nothing to wait for, unless a wait above gave up
        if (lane == 0) bulk_wait_all();                        // this lane's tile stores are done before the block leaves
    }

    tc_fence_before_sync();
    __syncthreads();
    cluster_sync_all();          // the partner's shared memory and TMEM stay alive until both CTAs are done
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc_pair(tmem_base, 512);
    }
}

// K == 0: no groups
__global__ void fp8_empty_kernel(const Fp8Args p) {
    start_next();
    wait_previous();
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (i < (long long)p.M * p.N) store_out(p, i / p.N, (int)(i % p.N), 0.0f);
}

// ------------------------------------------------------------------------------------------------------------ host
// How K is split: while that still adds CTAs that run at once (two fit on an SM), a CTA keeping two groups at least.
int tile_split(long long tiles, int k_blocks) {
    int split = 1;
    while (split < 8 && tiles * split * 2 <= 2 * sm_count() && k_blocks >= 4 * split) split *= 2;
    return split;
}

template <int NT>
int launch_tile(const CUtensorMap& tmB, const void* A, int64_t lda, int64_t K, Fp8Args& a, cudaStream_t stream) {
    a.m_tiles = (a.M + NT - 1) / NT;
    a.n_tiles = (a.N + 127) / 128;
    const long long tiles = (long long)a.m_tiles * a.n_tiles;
    const int split = tile_split(tiles, a.k_blocks);
    a.split = split;
    if (tiles * split > 0x7fffffffll) return NQ_ERR_UNSUPPORTED;
    CUtensorMap tmA;
    const int st = encode_tensor_map_2d(&tmA, A, (uint64_t)K, (uint64_t)a.M, (uint64_t)lda, kGroup, NT, 128);
    if (st != NQ_OK) return st;
    static int configured[64] = {0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return NQ_ERR_CUDA;
    if (!configured[dev]) {
        if (cudaFuncSetAttribute(fp8_tile_kernel<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, TileShape<NT>::kSmem) != cudaSuccess) {
            (void)cudaGetLastError();
            return NQ_ERR_CUDA;
        }
        configured[dev] = 1;
    }
    return launch_chained(fp8_tile_kernel<NT>, (unsigned)(tiles * split), kTileThreads, TileShape<NT>::kSmem, (unsigned)split, stream, tmA, tmB, a);
}

template <bool ROW_SCALES>
int launch_pair(const CUtensorMap& tmA, const CUtensorMap& tmB, const CUtensorMap& tmY, const Fp8Args& a, cudaStream_t stream) {
    using S = PairShape<ROW_SCALES>;
    static int configured[64] = {0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return NQ_ERR_CUDA;
    if (!configured[dev]) {
        if (cudaFuncSetAttribute(fp8_pair_kernel<ROW_SCALES>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem) != cudaSuccess) {
            (void)cudaGetLastError();
            return NQ_ERR_CUDA;
        }
        configured[dev] = 1;
    }
    const long long tiles = (long long)a.m_tiles * a.n_tiles;
    const int max_pairs = sm_count() / 2;
    return launch_chained(fp8_pair_kernel<ROW_SCALES>, (unsigned)(2 * (tiles < max_pairs ? tiles : max_pairs)), kPairThreads, S::kSmem, 2u, stream, tmA, tmB, tmY, a);
}

int run_fp8_gemm(const void* A, int64_t lda, const void* B, int64_t ldb, int64_t K, Fp8Args& a, cudaStream_t stream) {
    CUtensorMap tmB;
    const long long pair_tiles = (long long)((a.M + 255) / 256) * ((a.N + 255) / 256);
    // Which kernel: by the time each would take in microseconds, (rounds of tiles over the machine) x (groups of K a tile and
    // round x t + c), with t and c fitted to measurements from 128 x 128 to 8192 x 8192 outputs and K of 768 to 16384 that they
    // meet within a sixth:
    //   pair      t 0.55 (1.0 with row scales), c 1.5, and 5 once     512 x 4096 x 4096: 22.3,  4096^3: 78,  300 x 300 x 16384: 137
    //   64 rows   t 0.55, c 7.4                                                         26.6          177                     15.9
    //   32 rows   t 0.465, c 4.8                                                        39.7          274                     12.3
    // (128 rows a tile spill their sums: 33 us for 128 x 8192 x 4096 against 16.5 with 64.)
    const auto tile_cost = [&](int nt, double t, double c) {
        const long long tiles = (long long)((a.M + nt - 1) / nt) * ((a.N + 127) / 128);
        const int split = tile_split(tiles, a.k_blocks);
        return (double)((tiles * split + 2 * sm_count() - 1) / (2 * sm_count())) * (((a.k_blocks + split - 1) / split) * t + c);
    };
    const double cost32 = tile_cost(32, 0.465, 4.8), cost64 = tile_cost(64, 0.55, 7.4);
    const long long pairs = sm_count() / 2;
    const double cost_pair = 5.0 + (double)((pair_tiles + pairs - 1) / pairs) * (a.k_blocks * (a.b_shift ? 0.55 : 1.0) + 1.5);
    if (a.M > 64 && cost_pair <= cost32 && cost_pair <= cost64) {
        if (pair_tiles > 0x3fffffffll) return NQ_ERR_UNSUPPORTED;
        CUtensorMap tmA, tmY;
        int st = encode_tensor_map_2d(&tmA, A, (uint64_t)K, (uint64_t)a.M, (uint64_t)lda, kGroup, 128, 128);
        if (st != NQ_OK) return st;
        st = encode_tensor_map_2d(&tmB, B, (uint64_t)K, (uint64_t)a.N, (uint64_t)ldb, kGroup, 64, 128);
        if (st != NQ_OK) return st;
        a.m_tiles = (a.M + 255) / 256;
        a.n_tiles = (a.N + 255) / 256;
        // a group's rows of A stay within about 32 MB of L2
        a.group_m = 16;
        while (a.group_m > 4 && 256.0 * a.group_m * (double)K > 34.0e6) a.group_m /= 2;
        tmY = tmA;
        const uint64_t esize = a.y_is_bf16 ? 2 : 4, pitch = (uint64_t)a.ldy * esize;
        a.y_tma = !a.accumulate && (reinterpret_cast<uintptr_t>(a.y) & 15) == 0 && (pitch & 15) == 0 && pitch < (1ull << 40) &&
                  encode_tensor_map_out(&tmY, a.y, (uint64_t)a.N * esize, pitch, (uint64_t)a.M, 1, 1, 32, 1, 1, 64) == NQ_OK;
        return a.b_shift == 0 ? launch_pair<true>(tmA, tmB, tmY, a, stream) : launch_pair<false>(tmA, tmB, tmY, a, stream);
    }
    const int st = encode_tensor_map_2d(&tmB, B, (uint64_t)K, (uint64_t)a.N, (uint64_t)ldb, kGroup, 128, 128);
    if (st != NQ_OK) return st;
    if (a.M <= 16) return launch_tile<16>(tmB, A, lda, K, a, stream);
    return a.M <= 32 || cost32 < cost64 ? launch_tile<32>(tmB, A, lda, K, a, stream) : launch_tile<64>(tmB, A, lda, K, a, stream);
}

}  // namespace
}  // namespace nq

extern "C" int nq_fp8_gemm(const void* A, int64_t lda, const float* SA, int64_t ldsa, const void* B, int64_t ldb, const float* SB,
                           int64_t ldsb, int b_block_rows, const float* bias, int64_t M, int64_t N, int64_t K, void* Y, int64_t ldy,
                           int y_dtype, int accumulate, void* stream) {
    if (M < 0 || N < 0 || K < 0 || (y_dtype != NQ_F32 && y_dtype != NQ_BF16) || (b_block_rows != 1 && b_block_rows != 128))
        return NQ_ERR_INVALID_ARG;
    if (accumulate && y_dtype != NQ_F32) return NQ_ERR_UNSUPPORTED;
    if (M >= (1ll << 29) || N >= (1ll << 29) || K >= (1ll << 29)) return NQ_ERR_UNSUPPORTED;     // byte coordinates fit 32 bits
    if (M == 0 || N == 0) return NQ_OK;
    if (!Y || ldy < N) return NQ_ERR_INVALID_ARG;
    const auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
    if (at(Y) % (y_dtype == NQ_BF16 ? 2 : 4) || (at(bias) & 3)) return NQ_ERR_ALIGNMENT;
    nq::Fp8Args a{};
    a.M = (int)M; a.N = (int)N; a.k_blocks = (int)((K + 127) / 128);
    a.sa = SA; a.sb = SB; a.ldsa = ldsa; a.ldsb = ldsb; a.b_shift = b_block_rows == 128 ? 7 : 0;
    a.bias = bias; a.y = Y; a.ldy = ldy; a.y_is_bf16 = y_dtype == NQ_BF16; a.accumulate = accumulate != 0;
    const cudaStream_t s = (cudaStream_t)stream;
    if (K == 0) {
        if ((M * N + 255) / 256 > 0x7fffffffll) return NQ_ERR_UNSUPPORTED;
        return nq::launch_chained(nq::fp8_empty_kernel, (unsigned)((M * N + 255) / 256), 256, 0, 1, s, a);
    }
    if (!A || !B || !SA || !SB || lda < K || ldb < K || ldsa < M || ldsb < (b_block_rows == 128 ? (N + 127) / 128 : N)) return NQ_ERR_INVALID_ARG;
    if ((at(A) & 15) || (at(B) & 15) || (lda & 15) || (ldb & 15) || (at(SA) & 3) || (at(SB) & 3)) return NQ_ERR_ALIGNMENT;
    a.status = nq::status_word();
    if (!a.status) return NQ_ERR_CUDA;
    return nq::run_fp8_gemm(A, lda, B, ldb, K, a, s);
}
