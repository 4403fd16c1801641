// Attention of one new token a sequence over the paged key-value cache.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/nq.h"
#include "nq_kv_cache.cuh"
#include "nq_ranges.cuh"

namespace nq {
namespace {

// The cache is read once, 16 or 32 tokens of one kv head (a "step") at a time by one warp, straight into the registers of the matrix
// instruction: no shared memory, no barrier, nothing between warps until they have their sums.  Both products have the tokens or
// the head's channels as their 16 rows and the query heads of the kv head as their 8 columns:
//   S^T [16 tokens, 8 heads] = K Q^T       a lane's 16-byte pieces of two tokens are the operand as they come: the channels are
//                                          summed over, so any order of them will do as long as Q has the same
//   O^T [16 channels, 8 heads] += V^T P^T  a lane holds a piece of four tokens; a byte permutation puts two tokens' values of a
//                                          channel side by side; P^T is S^T's fragment, transposed in 8 x 8 blocks
// Heads as columns need half of the instructions and accumulators that heads as 16 rows would (a group has 1 to 8 heads, or 16).
// The sequences' steps (of all kv heads) lie in one long row that is cut evenly over the warps of a full GPU, however the
// lengths fall.  What a warp has of a sequence and head, if not all of it, is joined in its thread block, and over thread blocks by
// a second kernel, in a fixed order.
// The matrix instruction cuts products off 25 bits below the running sum that they are added to, towards zero: a warp's sum over n tokens of values of
// one sign loses n 2^-27.  Cut over 1184 warps or more, that stays under half a bf16 step up to a cache of some 6 10^8 tokens times heads.
// Bound by HBM: 64 sequences of up to 8192 tokens, 32 / 8 heads of 128, bf16 193 us (0.97 of the copy rate), e4m3 120 (0.80); one of 131072 e4m3 tokens
// 58 (0.72: some 11 us go to the cut, the first loads and the joins); one of 1501 INT8 tokens 10.5, all latency (15 with a search for the
// place, a block's parts weighed one after the other, and a join that asked for maxima, weights and values in turn).
constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr float kRescale = 8.0f;         // the running maximum moves when a score passes it by 2^8 (fp32 sums have room)
// 8-bit caches: what is rounded to f16 is a weight times its value's scale, times a power of two of the column's own (`held`): the largest such
// product so far is 2^7 to 2^8 when that power is set and may rise to 2^15 before it is set anew, so f16 is normal down to 2^-21 of it, and what is
// lost is under 2^-32 of it.  (In units of the largest scale, whatever its weight, one token of a large value and no weight took the bits of
// all others.)  When the running maximum moves, by 2^8 or more, the power moves against it, and the sums grow by 2 at most.  It is at most
// 2^125, so that its inverse is a normal number (products under 2^-118 are then held to 2^-150), and weights are at most 1 (2^-8 for the one that
// moved the maximum), so that no scale takes a product past fp32.  (One sequence of 131072 e4m3 tokens 58.1 us, in units of the largest scale 57.5; 64
// of up to 8192 120 - 128 against 131.)
constexpr float kLift = 8.0f, kMostHeld = 32768.0f;
constexpr int kHeld = 7, kMostPower = 125;

// Tokens of a step: as many as bring 8 KB (4 KB of 8-bit heads of 64) to a warp.  Two groups of 16 at once also halve what a step costs
// beside its products (e4m3, 131072 tokens of 8 heads of 128, 16 at once: 79 us).
__host__ __device__ constexpr int step_tokens(int dim, int cache) { return dim == 128 && cache == NQ_BF16 ? 16 : 32; }

struct TokenArgs {
    Pages c;
    const __nv_bfloat16* q;
    long long ldq;
    int q_heads, group, head_blocks;     // query heads of a kv head, and how many blocks of columns they make
    const int* table;
    long long ld_table;
    int table_tokens;                    // what the table's columns can hold
    const int* lengths;
    int seqs, window;
    float scale2;                        // score scale * log2(e)
    __nv_bfloat16* y;
    long long ldy;
    int4* records;                       // [blocks]: a sequence and head that begins in this block and goes on: its number, head, last block
    float* slots;                        // [blocks][2]: what the block has of the one it goes on with (0) and of that one (1)
};

template <int D, int NT>
constexpr int kSlotFloats = 8 * NT * (D + 2);      // sums [heads][D], maxima [heads], weights' sums [heads]

__device__ __forceinline__ float exp2a(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// of a positive normal number: the exponent of the power of two at or below it; and back
__device__ __forceinline__ int log2_of(float x) { return (__float_as_int(x) >> 23) - 127; }
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t s) {
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(s));
    return r;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
template <bool HALF>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (HALF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two e4m3 codes (in the low 16 bits) to f16 exactly.
__device__ __forceinline__ uint32_t codes2(uint32_t two) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)two));
    return h;
}
// Four codes to two words of f16, in their order.  INT8: code + 128 as the low bits of 1024 + (code + 128), less 1152.
template <int CACHE>
__device__ __forceinline__ void codes4(uint32_t w, uint32_t& lo, uint32_t& hi) {
    if (CACHE == NQ_E4M3) {
        lo = codes2(w);
        hi = codes2(w >> 16);
    } else {
        const uint32_t u = w ^ 0x80808080u;
        const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
        const uint32_t a = prmt(u, 0x64646464u, 0x4140), b = prmt(u, 0x64646464u, 0x4342);
        const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), off), y = __hsub2(*reinterpret_cast<const __half2*>(&b), off);
        lo = *reinterpret_cast<const uint32_t*>(&x);
        hi = *reinterpret_cast<const uint32_t*>(&y);
    }
}

// Steps of a sequence, its tokens and the number of its first step (behind a window it is not 0).
template <int TOKENS>
__device__ __forceinline__ int steps_of(const TokenArgs& a, int seq, int& length, int& first) {
    length = min(a.lengths[seq], a.table_tokens);
    first = a.window > 0 && length > a.window ? (length - a.window) / TOKENS : 0;
    return length <= 0 ? 0 : (length - 1) / TOKENS + 1 - first;
}

// (a 64-bit division takes several hundred cycles; what fits takes the short one)
__device__ __forceinline__ long long divide(long long a, long long b) {
    return ((unsigned long long)a | (unsigned long long)b) >> 32 ? a / b : (long long)((unsigned)a / (unsigned)b);
}

// Where a warp is in the long row.
template <int TOKENS>
struct Place {
    int seq, head, block, step;              // sequence, kv head, block of columns, step among the sequence's
    int steps, length, first;                // of the sequence
    __device__ __forceinline__ void next(const TokenArgs& a) {
        if (++step < steps) return;
        step = 0;
        if (++block < a.head_blocks) return;
        block = 0;
        if (++head < a.c.kv_heads) return;
        head = 0;
        do {
            if (++seq >= a.seqs) return;
            steps = steps_of<TOKENS>(a, seq, length, first);
        } while (steps == 0);
    }
};

__device__ __forceinline__ void zero_row(const TokenArgs& a, int seq, int columns) {
    uint4* to = reinterpret_cast<uint4*>(a.y + seq * a.ldy);
    for (int i = threadIdx.x; i < columns / 8; i += kThreads) to[i] = make_uint4(0, 0, 0, 0);
}

// Four channels: sums over the sum of weights, zeros where nothing was seen.
__device__ __forceinline__ void store_row4(__nv_bfloat16* to, const float4& sum, float weights) {
    const __nv_bfloat162 lo = weights == 0.0f ? __floats2bfloat162_rn(0.0f, 0.0f) : __floats2bfloat162_rn(sum.x / weights, sum.y / weights);
    const __nv_bfloat162 hi = weights == 0.0f ? __floats2bfloat162_rn(0.0f, 0.0f) : __floats2bfloat162_rn(sum.z / weights, sum.w / weights);
    *reinterpret_cast<uint2*>(to) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}

template <int D, int CACHE, int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 && !(D == 128 && CACHE != NQ_BF16) ? 3 : 2) token_kernel(const TokenArgs a) {
    constexpr bool kCodes = CACHE != NQ_BF16;
    constexpr int kRow = D * (kCodes ? 1 : 2);                       // bytes of a token's head
    constexpr int kKPieces = kRow / 64;                              // 16-byte pieces of a K row in a lane (4 lanes a row)
    constexpr int kVBytes = kRow / 8 > 16 ? 16 : kRow / 8;           // piece of a V row in a lane (8 lanes a row)
    constexpr int kVPieces = kRow / 8 / kVBytes, kVWords = kVBytes / 4;
    constexpr int kSteps = D / 16;                                   // matrix instructions of 16 channels
    constexpr int kSub = step_tokens(D, CACHE) / 16, kTokens = 16 * kSub;
    constexpr int kSlot = kSlotFloats<D, NT>;
    extern __shared__ __align__(16) float s_parts[];                 // [2 * kWarps][kSlot]
    __shared__ __align__(16) long long s_before[kThreads + 1];
    __shared__ long long s_warp[kWarps];
    __shared__ float s_factor[2 * kWarps][8 * NT], s_total[8 * NT];
    __shared__ int4 s_meta[2 * kWarps];                              // of each part: sequence (-1: none), unit, whether it holds the first (1) and the last (2) step

    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = lane >> 2, j = lane & 3;
    const int units = a.c.kv_heads * a.head_blocks;
    wait_previous();

    // ---- the long row: steps before each chunk of sequences
    const int chunk = (a.seqs + kThreads - 1) / kThreads;
    long long mine = 0;
    for (int s = threadIdx.x * chunk; s < min(a.seqs, (int)(threadIdx.x + 1) * chunk); ++s) {
        int length, first;
        mine += steps_of<kTokens>(a, s, length, first);
    }
    long long sum = mine;
#pragma unroll
    for (int m = 1; m < 32; m *= 2) {
        const long long o = __shfl_up_sync(0xffffffffu, sum, m);
        if (lane >= m) sum += o;
    }
    if (lane == 31) s_warp[warp] = sum;
    if (threadIdx.x < 2 * kWarps) s_meta[threadIdx.x] = make_int4(-1, 0, 0, 0);
    __syncthreads();
    for (int w = 0; w < warp; ++w) sum += s_warp[w];
    s_before[threadIdx.x + 1] = sum;
    if (threadIdx.x == 0) s_before[0] = 0;
    __syncthreads();
    const long long total = s_before[kThreads] * units;
    for (int s = blockIdx.x; s < a.seqs; s += gridDim.x)
        if (a.lengths[s] <= 0 || a.table_tokens == 0) zero_row(a, s, a.q_heads * D);

    // ---- this block's and this warp's part of it
    const long long blocks = min((long long)gridDim.x, (total + kWarps - 1) / kWarps);
    const long long per = blocks > 0 ? divide(total, blocks) : 0, more = total - per * blocks;           // the first `more` blocks have one more
    const long long begin = per * blockIdx.x + min((long long)blockIdx.x, more), end = blockIdx.x < blocks ? begin + per + (blockIdx.x < more) : begin;
    const long long from = begin + (end - begin) * warp / kWarps;
    int left = (int)(begin + (end - begin) * (warp + 1) / kWarps - from);
    int part = 2 * warp;                                             // next part to fill
    if (left > 0) {
        Place<kTokens> at;
        {
            // the last chunk that starts at or before `from`
            int lo = 0;
#pragma unroll
            for (int x = 0; x < kThreads / 32; ++x) lo += s_before[kThreads / 32 * lane + x] * units <= from;
            lo = __reduce_add_sync(0xffffffffu, lo) - 1;
            long long rest = from - s_before[lo] * units;
            at.seq = lo * chunk;
            at.steps = steps_of<kTokens>(a, at.seq, at.length, at.first);
            while (rest >= (long long)at.steps * units) {
                rest -= (long long)at.steps * units;
                at.steps = steps_of<kTokens>(a, ++at.seq, at.length, at.first);
            }
            const int unit = (int)divide(rest, at.steps);
            at.step = (int)(rest - (long long)unit * at.steps);
            at.head = a.head_blocks == 1 ? unit : unit / a.head_blocks;
            at.block = unit - at.head * a.head_blocks;
        }
        const int per_page = a.c.page_size >> 4;
        const long long page_rows = (long long)a.c.kv_heads * a.c.page_size;

        uint4 kw[kSub][2][kKPieces];                                 // K of tokens i, i + 8 of 16
        uint32_t vw[kSub][4][kVPieces][kVWords];                     // V of tokens 2 j, 2 j + 1, 2 j + 8, 2 j + 9 of 16
        float ks[kSub][2], vs[kSub][2];                              // scales of tokens i, i + 8
        long long row[kSub];                                         // of the first of 16 tokens in the cache, -1: no such page
        long long my_row = -1;                                       // lane's page of 16 tokens number pages_from + lane: its first row for head 0, -1: none
        int pages_seq = -1, pages_from = 0;

        auto find_rows = [&](const Place<kTokens>& p) {
            const int number = (p.first + p.step) * kSub;
            if (p.seq != pages_seq || number < pages_from || number + kSub > pages_from + 32) {
                pages_seq = p.seq;
                pages_from = number;
                const int n = number + lane;
                my_row = -1;
                if (group_in(n, p.length)) {
                    const int nth = n / per_page, page = a.table[p.seq * a.ld_table + nth];
                    if (page >= 0 && page < a.c.pages) my_row = page * page_rows + (n - nth * per_page) * 16;
                }
            }
#pragma unroll
            for (int u = 0; u < kSub; ++u) {
                const long long r = __shfl_sync(0xffffffffu, my_row, number + u - pages_from);
                row[u] = r < 0 ? -1 : r + (long long)p.head * a.c.page_size;
            }
        };
        auto load_k = [&] {
#pragma unroll
            for (int u = 0; u < kSub; ++u)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const uint8_t* src = a.c.k + (row[u] + i + 8 * t) * kRow + 16 * j;
#pragma unroll
                    for (int p = 0; p < kKPieces; ++p) kw[u][t][p] = row[u] < 0 ? make_uint4(0, 0, 0, 0) : load16(src + 64 * p);
                    if (kCodes && row[u] >= 0) ks[u][t] = a.c.ks[row[u] + i + 8 * t];
                }
        };
        auto load_v = [&] {
#pragma unroll
            for (int u = 0; u < kSub; ++u) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const uint8_t* src = a.c.v + (row[u] + 2 * j + (t & 1) + 8 * (t >> 1)) * kRow + kVBytes * i;
#pragma unroll
                    for (int p = 0; p < kVPieces; ++p) {
                        if (row[u] < 0) {
#pragma unroll
                            for (int w = 0; w < kVWords; ++w) vw[u][t][p][w] = 0;
                        } else if (kVWords == 4) {
                            const uint4 v = load16(src + 8 * kVBytes * p);
                            vw[u][t][p][0] = v.x; vw[u][t][p][1] = v.y; vw[u][t][p][2 % kVWords] = v.z; vw[u][t][p][3 % kVWords] = v.w;
                        } else {
                            asm volatile("ld.global.L1::no_allocate.v2.b32 {%0, %1}, [%2];" : "=r"(vw[u][t][p][0]), "=r"(vw[u][t][p][1]) : "l"(src) : "memory");
                        }
                    }
                }
                if (kCodes && row[u] >= 0) {
                    vs[u][0] = a.c.vs[row[u] + i];
                    vs[u][1] = a.c.vs[row[u] + i + 8];
                }
            }
        };

        uint32_t qf[NT][kSteps][2];
        float q_scale[NT][2];                                        // of heads 2 j, 2 j + 1: what a product of codes is multiplied by
        float o[NT][kSteps][4], top[NT][2], weight[NT][2];
        float held[NT][2];                                           // of heads 2 j, 2 j + 1: what a weight times its value's scale is multiplied by
        int begun = 0;

        find_rows(at);
        load_k();
        load_v();
        bool fresh = true;
        while (left > 0) {
            const Place<kTokens> cur = at;
            bool there[kSub];
#pragma unroll
            for (int u = 0; u < kSub; ++u) there[u] = row[u] >= 0;
            const int block = cur.block, kv_head = cur.head;
            if (fresh) {                                             // another sequence or head
                fresh = false;
                begun = cur.step == 0;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int h = (block * NT + n) * 8 + i;
                    const bool live = h < a.group;
                    const __nv_bfloat16* src = a.q + cur.seq * a.ldq + (long long)(kv_head * a.group + (live ? h : 0)) * D;
                    top[n][0] = top[n][1] = -INFINITY;
                    weight[n][0] = weight[n][1] = 0.0f;
                    held[n][0] = held[n][1] = 1.0f;
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) o[n][s][0] = o[n][s][1] = o[n][s][2] = o[n][s][3] = 0.0f;
                    if (!kCodes) {
#pragma unroll
                        for (int p = 0; p < kKPieces; ++p) {
                            const uint4 v = live ? load16(src + 8 * (j + 4 * p)) : make_uint4(0, 0, 0, 0);
                            qf[n][2 * p][0] = v.x; qf[n][2 * p][1] = v.y; qf[n][2 * p + 1][0] = v.z; qf[n][2 * p + 1][1] = v.w;
                        }
                        q_scale[n][0] = q_scale[n][1] = a.scale2;
                    } else {
                        // bf16 to f16, times a power of two that puts the head's largest into [1, 2): exact but for values below 2^-17 of it,
                        // whose 8 bits go under f16's last, 2^-24
                        uint4 v[2 * kKPieces];
                        uint32_t m = 0;
#pragma unroll
                        for (int p = 0; p < kKPieces; ++p) {
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const uint4 x = live ? load16(src + 16 * (j + 4 * p) + 8 * half) : make_uint4(0, 0, 0, 0);
                                v[2 * p + half] = x;
                                m = __vmaxu2(m, __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu)));
                            }
                        }
                        m = max(m >> 16, m & 0xffffu);
                        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
                        m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
                        const int e = min(max((int)(m >> 7), 1), 253);               // 254: [2, 4); 255 (infinity, NaN): no finite number in f16 either
                        const float up = __int_as_float((254 - e) << 23), down = __int_as_float(e << 23);
#pragma unroll
                        for (int w = 0; w < 8 * kKPieces; ++w) {
                            const uint4 x = v[w / 4];
                            const uint32_t u = w % 4 == 0 ? x.x : w % 4 == 1 ? x.y : w % 4 == 2 ? x.z : x.w;
                            const __half2 h2 = __floats2half2_rn(__uint_as_float(u << 16) * up, __uint_as_float(u & 0xffff0000u) * up);
                            qf[n][w / 2][w & 1] = *reinterpret_cast<const uint32_t*>(&h2);
                        }
#pragma unroll
                        for (int c = 0; c < 2; ++c) q_scale[n][c] = __shfl_sync(0xffffffffu, down, 4 * (2 * j + c)) * a.scale2;
                    }
                }
            }

            // ---- scores
            float sc[kSub][NT][4];
#pragma unroll
            for (int u = 0; u < kSub; ++u)
#pragma unroll
                for (int n = 0; n < NT; ++n) sc[u][n][0] = sc[u][n][1] = sc[u][n][2] = sc[u][n][3] = 0.0f;
#pragma unroll
            for (int p = 0; p < kKPieces; ++p)
#pragma unroll
                for (int u = 0; u < kSub; ++u) {
                    const uint4 x = kw[u][0][p], y = kw[u][1][p];
                    const uint32_t w0[4] = {x.x, x.y, x.z, x.w}, w1[4] = {y.x, y.y, y.z, y.w};
                    if (!kCodes) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int n = 0; n < NT; ++n) mma<false>(sc[u][n], w0[2 * h], w1[2 * h], w0[2 * h + 1], w1[2 * h + 1], qf[n][2 * p + h][0], qf[n][2 * p + h][1]);
                    } else {
#pragma unroll
                        for (int h = 0; h < 4; ++h) {
                            uint32_t a0, a1, a2, a3;
                            codes4<CACHE>(w0[h], a0, a2);
                            codes4<CACHE>(w1[h], a1, a3);
#pragma unroll
                            for (int n = 0; n < NT; ++n) mma<true>(sc[u][n], a0, a1, a2, a3, qf[n][4 * p + h][0], qf[n][4 * p + h][1]);
                        }
                    }
                }
            float kscale[kSub][2], vscale[kSub][2];
#pragma unroll
            for (int u = 0; u < kSub; ++u)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    kscale[u][t] = kCodes ? ks[u][t] + (ks[u][t] - ks[u][t]) : 1.0f;                 // an infinite scale's values are no numbers
                    vscale[u][t] = kCodes ? vs[u][t] + (vs[u][t] - vs[u][t]) : 1.0f;
                }
            --left;
            at.next(a);
            const bool closes = left == 0 || at.step == 0;           // the warp's last step of this sequence and head
            if (left > 0) {
                find_rows(at);
                load_k();
            }
            // ---- masks: only a sequence's first and last steps have any
            const int length = cur.length, token0 = (cur.first + cur.step) * kTokens;
            const int lo = a.window > 0 ? length - a.window : 0;
            bool edge = length - token0 < kTokens || token0 < lo;       // (token0 + kTokens may pass 32 bits)
#pragma unroll
            for (int u = 0; u < kSub; ++u) edge |= !there[u];
            bool seen[kSub][2];
#pragma unroll
            for (int u = 0; u < kSub; ++u) seen[u][0] = seen[u][1] = true;
            if (edge) {
#pragma unroll
                for (int u = 0; u < kSub; ++u) {
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const int token = token0 + 16 * u + i + 8 * t;
                        seen[u][t] = there[u] && token < length && token >= lo;
                        if (!seen[u][t]) vscale[u][t] = 0.0f;
                    }
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const int token = token0 + 16 * u + 2 * j + (t & 1) + 8 * (t >> 1);
                        if (there[u] && token < length && token >= lo) continue;
#pragma unroll
                        for (int p = 0; p < kVPieces; ++p)
#pragma unroll
                            for (int w = 0; w < kVWords; ++w) vw[u][t][p][w] = 0;
                    }
                }
            }
            // ---- weights
            bool move = false;
#pragma unroll
            for (int u = 0; u < kSub; ++u)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float s = sc[u][n][e] * q_scale[n][e & 1];
                        if (kCodes) s *= kscale[u][e >> 1];
                        s = seen[u][e >> 1] ? s : -INFINITY;
                        sc[u][n][e] = s;
                        move |= s > top[n][e & 1] + (kCodes ? 0.0f : kRescale);
                    }
            if (__any_sync(0xffffffffu, move)) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float by[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float m = top[n][c];
#pragma unroll
                        for (int u = 0; u < kSub; ++u) m = fmaxf(m, fmaxf(sc[u][n][c], sc[u][n][2 + c]));
#pragma unroll
                        for (int x = 4; x < 32; x *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
                        if (kCodes) m = m > top[n][c] ? m + kLift : m;
                        const float d = top[n][c] == -INFINITY ? -INFINITY : top[n][c] - m;
                        by[c] = exp2a(d);
                        top[n][c] = m;
                        weight[n][c] *= by[c];
                        if (kCodes) {
                            const float up = fminf(ceilf(-d), (float)(kMostPower - log2_of(held[n][c])));
                            by[c] = exp2a(d + up);
                            held[n][c] = power_of_two(log2_of(held[n][c]) + (int)up);
                        }
                    }
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        o[n][s][0] *= by[0]; o[n][s][1] *= by[1]; o[n][s][2] *= by[0]; o[n][s][3] *= by[1];
                    }
                }
            }
            bool grow = false;
#pragma unroll
            for (int u = 0; u < kSub; ++u)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float m = top[n][e & 1], p = exp2a(sc[u][n][e] - (m == -INFINITY ? 0.0f : m));
                        weight[n][e & 1] += p;
                        sc[u][n][e] = kCodes ? p * vscale[u][e >> 1] : p;
                        if (kCodes) grow |= fabsf(sc[u][n][e]) * held[n][e & 1] > kMostHeld;
                    }
            if (kCodes && __any_sync(0xffffffffu, grow)) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float by[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float m = 0.0f;
#pragma unroll
                        for (int u = 0; u < kSub; ++u) m = fmaxf(m, fmaxf(fabsf(sc[u][n][c]), fabsf(sc[u][n][2 + c])));
#pragma unroll
                        for (int x = 4; x < 32; x *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
                        by[c] = 1.0f;
                        if (m * held[n][c] > kMostHeld) {
                            const int old = log2_of(held[n][c]), now = kHeld - log2_of(m);
                            by[c] = exp2a((float)(now - old));
                            held[n][c] = power_of_two(now);
                        }
                    }
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        o[n][s][0] *= by[0]; o[n][s][1] *= by[1]; o[n][s][2] *= by[0]; o[n][s][3] *= by[1];
                    }
                }
            }
            uint32_t pf[kSub][NT][2];
#pragma unroll
            for (int u = 0; u < kSub; ++u)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float (&p)[4] = sc[u][n];
                    if (kCodes) {
                        const __half2 x = __floats2half2_rn(p[0] * held[n][0], p[1] * held[n][1]), y = __floats2half2_rn(p[2] * held[n][0], p[3] * held[n][1]);
                        pf[u][n][0] = transpose8x8(*reinterpret_cast<const uint32_t*>(&x));
                        pf[u][n][1] = transpose8x8(*reinterpret_cast<const uint32_t*>(&y));
                    } else {
                        // bf16 has fp32's range: a weight is off by at most 2^-8 of itself
                        const __nv_bfloat162 x = __floats2bfloat162_rn(p[0], p[1]), y = __floats2bfloat162_rn(p[2], p[3]);
                        pf[u][n][0] = transpose8x8(*reinterpret_cast<const uint32_t*>(&x));
                        pf[u][n][1] = transpose8x8(*reinterpret_cast<const uint32_t*>(&y));
                    }
                }
            // ---- values
#pragma unroll
            for (int u = 0; u < kSub; ++u) {
                const uint32_t (&v)[4][kVPieces][kVWords] = vw[u];
                if (!kCodes) {
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        // two pieces of 8 channels: rows 0-7 of tile s are channel s of piece i, rows 8-15 of piece i + 8; one piece: channels 2 s, 2 s + 1
                        const int w = kVPieces == 2 ? s / 2 : s;
                        const uint32_t lo0 = kVPieces == 2 ? ((s & 1) ? 0x7632u : 0x5410u) : 0x5410u, hi0 = kVPieces == 2 ? lo0 : 0x7632u;
                        const uint32_t a0 = prmt(v[0][0][w], v[1][0][w], lo0), a1 = prmt(v[0][kVPieces - 1][w], v[1][kVPieces - 1][w], hi0);
                        const uint32_t a2 = prmt(v[2][0][w], v[3][0][w], lo0), a3 = prmt(v[2][kVPieces - 1][w], v[3][kVPieces - 1][w], hi0);
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma<false>(o[n][s], a0, a1, a2, a3, pf[u][n][0], pf[u][n][1]);
                    }
                } else {
#pragma unroll
                    for (int w = 0; w < kVWords; ++w) {              // four channels: two tiles, channels 2 s, 2 s + 1 of the lane's piece
                        uint32_t x[4], y[4];
                        codes4<CACHE>(prmt(v[0][0][w], v[1][0][w], 0x5140), x[0], x[1]);
                        codes4<CACHE>(prmt(v[0][0][w], v[1][0][w], 0x7362), x[2], x[3]);
                        codes4<CACHE>(prmt(v[2][0][w], v[3][0][w], 0x5140), y[0], y[1]);
                        codes4<CACHE>(prmt(v[2][0][w], v[3][0][w], 0x7362), y[2], y[3]);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            mma<true>(o[n][2 * w], x[0], x[1], y[0], y[1], pf[u][n][0], pf[u][n][1]);
                            mma<true>(o[n][2 * w + 1], x[2], x[3], y[2], y[3], pf[u][n][0], pf[u][n][1]);
                        }
                    }
                }
            }
            if (left > 0) load_v();

            if (closes) {
                fresh = true;
                const int ended = cur.step + 1 == cur.steps;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int x = 4; x < 32; x *= 2) weight[n][c] += __shfl_xor_sync(0xffffffffu, weight[n][c], x);
                // a lane's channels of a head: kVPieces runs of 8 (bf16), or one run of 2 * kSteps
                float* slot = s_parts + part * kSlot;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int column = n * 8 + 2 * j + c, h = block * NT * 8 + column;
                        // (the two factors one after the other: their product can be too small a number)
                        const float by = begun && ended ? (weight[n][c] > 0.0f || weight[n][c] != weight[n][c] ? 1.0f / weight[n][c] : 0.0f) : 1.0f;
                        const float back = kCodes ? power_of_two(-log2_of(held[n][c])) : 1.0f;
                        constexpr int kRuns = !kCodes && kVPieces == 2 ? 2 : 1, kRun = D / 8 / kRuns;
#pragma unroll
                        for (int r = 0; r < kRuns; ++r) {
                            const int channel = kRun * (i + 8 * r);
                            float v[kRun];
#pragma unroll
                            for (int x = 0; x < kRun; ++x) v[x] = by == 0.0f ? 0.0f : by * (kRuns == 2 ? o[n][x % kSteps][2 * r + c] : o[n][x / 2][2 * (x & 1) + c]) * back;
                            if (begun && ended) {
                                if (h < a.group) {
                                    __nv_bfloat16* to = a.y + cur.seq * a.ldy + (long long)(kv_head * a.group + h) * D + channel;
#pragma unroll
                                    for (int x = 0; x < kRun; x += 8) {
                                        uint32_t w4[4];
#pragma unroll
                                        for (int y = 0; y < 4; ++y) {
                                            const __nv_bfloat162 b2 = __floats2bfloat162_rn(v[x + 2 * y], v[x + 2 * y + 1]);
                                            w4[y] = *reinterpret_cast<const uint32_t*>(&b2);
                                        }
                                        *reinterpret_cast<uint4*>(to + x) = make_uint4(w4[0], w4[1], w4[2], w4[3]);
                                    }
                                }
                            } else {
#pragma unroll
                                for (int x = 0; x < kRun; x += 4) *reinterpret_cast<float4*>(slot + column * D + channel + x) = make_float4(v[x], v[x + 1], v[x + 2], v[x + 3]);
                            }
                        }
                        if (!(begun && ended) && i == 0) {
                            slot[8 * NT * D + column] = top[n][c];
                            slot[8 * NT * (D + 1) + column] = weight[n][c];
                        }
                    }
                }
                if (!(begun && ended)) {
                    if (lane == 0) s_meta[part] = make_int4(cur.seq, cur.head * a.head_blocks + cur.block, begun + 2 * ended, cur.steps - 1 - cur.step);
                    ++part;
                }
            }
        }
    }
    start_next();
    __syncthreads();

    // ---- the block's parts: neighbours of one sequence and head are joined; all of it: out; otherwise to the block's slots
    int4 record = make_int4(-1, 0, 0, 0);
    const int4 meta = lane < 2 * kWarps ? s_meta[lane] : make_int4(-1, 0, 0, 0);
    const auto of = [](int v, int from) { return __shfl_sync(0xffffffffu, v, from); };
    for (unsigned parts = __ballot_sync(0xffffffffu, meta.x >= 0); parts;) {
        const int p = __ffs(parts) - 1;
        const int4 first = make_int4(of(meta.x, p), of(meta.y, p), of(meta.z, p), 0);
        const unsigned these = __ballot_sync(0xffffffffu, meta.x == first.x && meta.y == first.y);
        const int rest = of(meta.w, 31 - __clz(these));
        const bool ends = __any_sync(0xffffffffu, (these >> lane & 1u) && (meta.z & 2));
        parts &= ~these;
        const bool begins = first.z & 1;
        const int kv_head = a.head_blocks == 1 ? first.y : first.y / a.head_blocks, block = first.y - kv_head * a.head_blocks;
        float* slot = a.slots + (2ll * blockIdx.x + (begins ? 1 : 0)) * kSlot;
        if (threadIdx.x < 8 * NT * 2 * kWarps) {                     // what each part counts for, by column: eight parts side by side
            const int column = threadIdx.x / (2 * kWarps), x = threadIdx.x % (2 * kWarps);
            const bool one = these >> x & 1u;
            const float t = one ? s_parts[x * kSlot + 8 * NT * D + column] : -INFINITY;
            float m = t;
#pragma unroll
            for (int y = 1; y < 2 * kWarps; y *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, y));
            const float by = t == -INFINITY && m == -INFINITY ? 1.0f : exp2a(t - m);
            float sum_w = one ? by * s_parts[x * kSlot + 8 * NT * (D + 1) + column] : 0.0f;
#pragma unroll
            for (int y = 1; y < 2 * kWarps; y *= 2) sum_w += __shfl_xor_sync(0xffffffffu, sum_w, y);
            s_factor[x][column] = by;
            if (x == 0) {
                s_total[column] = sum_w;
                if (!(begins && ends)) {
                    slot[8 * NT * D + column] = m;
                    slot[8 * NT * (D + 1) + column] = sum_w;
                }
            }
        }
        if (threadIdx.x == kThreads - 1 && begins && !ends) {
            // the last step of it is `rest` steps behind this block's end
            const long long x = end - 1 + rest, large = more * (per + 1);
            record = make_int4(first.x, first.y, (int)(x < large ? divide(x, per + 1) : more + divide(x - large, per)), 0);
        }
        __syncthreads();
        for (int e = threadIdx.x; e < 8 * NT * D / 4; e += kThreads) {
            const int column = e / (D / 4), h = block * NT * 8 + column;
            float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int x = 0; x < 2 * kWarps; ++x) {
                if (!(these >> x & 1u)) continue;
                const float4 v = *reinterpret_cast<const float4*>(s_parts + x * kSlot + 4 * e);
                const float by = s_factor[x][column];
                sum.x += by * v.x; sum.y += by * v.y; sum.z += by * v.z; sum.w += by * v.w;
            }
            if (!(begins && ends)) *reinterpret_cast<float4*>(slot + 4 * e) = sum;
            else if (h < a.group) store_row4(a.y + first.x * a.ldy + (long long)(kv_head * a.group + h) * D + 4 * (e % (D / 4)), sum, s_total[column]);
        }
        __syncthreads();
    }
    if (threadIdx.x == kThreads - 1) a.records[blockIdx.x] = record;
}

// A sequence and head that begins in block blockIdx.x and goes on in others: their parts joined, blockIdx.y: four columns of it.  What each
// part counts for first, then D / 4 threads a column and 256 / D parts at once.
// (Little shared memory: with 20 KB a block, the kernel that follows found its room divided otherwise, and 64 sequences back to back took
// 285 us against 200.)
constexpr int kJoin = 256;
template <int D, int NT>
__global__ void __launch_bounds__(kJoin) join_kernel(const TokenArgs a) {
    constexpr int kSlot = kSlotFloats<D, NT>, kAtOnce = kJoin / D;
    __shared__ __align__(16) float4 s_warp[kJoin / 32], s_sums[kJoin];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, column0 = 4 * blockIdx.y;
    wait_previous();
    start_next();
    const int4 rec = a.records[blockIdx.x];
    if (rec.x < 0) return;
    const int block = rec.y % a.head_blocks, kv_head = rec.y / a.head_blocks;
    if (block * NT * 8 + column0 >= a.group) return;
    const int n = rec.z - (int)blockIdx.x + 1;                       // parts: slot 1 of this block, slot 0 of the others
    const auto part = [&](int x) { return a.slots + (2ll * (blockIdx.x + x) + (x == 0)) * kSlot; };
    const auto over_block = [&](float4 v, bool largest) {            // the largest, or the sum, of all threads' values
        const auto join = [&](float p, float q) { return largest ? fmaxf(p, q) : p + q; };
#pragma unroll
        for (int s = 1; s < 32; s *= 2) {
            v.x = join(v.x, __shfl_xor_sync(0xffffffffu, v.x, s)); v.y = join(v.y, __shfl_xor_sync(0xffffffffu, v.y, s));
            v.z = join(v.z, __shfl_xor_sync(0xffffffffu, v.z, s)); v.w = join(v.w, __shfl_xor_sync(0xffffffffu, v.w, s));
        }
        __syncthreads();
        if (lane == 0) s_warp[warp] = v;
        __syncthreads();
        v = s_warp[0];
        for (int w = 1; w < kJoin / 32; ++w) {
            const float4 o = s_warp[w];
            v.x = join(v.x, o.x); v.y = join(v.y, o.y); v.z = join(v.z, o.z); v.w = join(v.w, o.w);
        }
        return v;
    };
    const int column = threadIdx.x / (D / 4) % 4, piece = threadIdx.x % (D / 4), first = threadIdx.x / D;
    // all that a thread needs at first, asked for at once: a part's maximum and weights, and its values of kEarly parts
    constexpr int kEarly = 8;
    const float4 none = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    const auto top_of = [&](int x) { return *reinterpret_cast<const float4*>(part(x) + 8 * NT * D + column0); };
    const auto weight_of = [&](int x) { return *reinterpret_cast<const float4*>(part(x) + 8 * NT * (D + 1) + column0); };
    const auto value_of = [&](int x) { return *reinterpret_cast<const float4*>(part(x) + (column0 + column) * D + 4 * piece); };
    float4 m = none, sum_w = make_float4(0.0f, 0.0f, 0.0f, 0.0f), early[kEarly];
    float early_top[kEarly];
    if (threadIdx.x < n) {
        m = top_of(threadIdx.x);
        sum_w = weight_of(threadIdx.x);
    }
#pragma unroll
    for (int e = 0; e < kEarly; ++e)
        if (first + e * kAtOnce < n) {
            early[e] = value_of(first + e * kAtOnce);
            early_top[e] = part(first + e * kAtOnce)[8 * NT * D + column0 + column];
        }
    const float4 mine = m;
    for (int x = threadIdx.x + kJoin; x < n; x += kJoin) {
        const float4 t = top_of(x);
        m = make_float4(fmaxf(m.x, t.x), fmaxf(m.y, t.y), fmaxf(m.z, t.z), fmaxf(m.w, t.w));
    }
    m = over_block(m, true);
    const auto by = [](float t, float top) { return t == -INFINITY && top == -INFINITY ? 1.0f : exp2a(t - top); };
    if (threadIdx.x < n) {
        sum_w.x *= by(mine.x, m.x); sum_w.y *= by(mine.y, m.y); sum_w.z *= by(mine.z, m.z); sum_w.w *= by(mine.w, m.w);
    }
    for (int x = threadIdx.x + kJoin; x < n; x += kJoin) {
        const float4 t = top_of(x), w = weight_of(x);
        sum_w.x += by(t.x, m.x) * w.x; sum_w.y += by(t.y, m.y) * w.y; sum_w.z += by(t.z, m.z) * w.z; sum_w.w += by(t.w, m.w) * w.w;
    }
    sum_w = over_block(sum_w, false);
    const float top = column == 0 ? m.x : column == 1 ? m.y : column == 2 ? m.z : m.w;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int e = 0; e < kEarly; ++e)
        if (first + e * kAtOnce < n) {
            const float f = by(early_top[e], top);
            sum.x += f * early[e].x; sum.y += f * early[e].y; sum.z += f * early[e].z; sum.w += f * early[e].w;
        }
#pragma unroll 8
    for (int x = first + kEarly * kAtOnce; x < n; x += kAtOnce) {
        const float4 v = value_of(x);
        const float f = by(part(x)[8 * NT * D + column0 + column], top);
        sum.x += f * v.x; sum.y += f * v.y; sum.z += f * v.z; sum.w += f * v.w;
    }
    s_sums[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x >= D) return;
    for (int x = 1; x < kAtOnce; ++x) {
        const float4 o = s_sums[threadIdx.x + x * D];
        sum.x += o.x; sum.y += o.y; sum.z += o.z; sum.w += o.w;
    }
    const int h = block * NT * 8 + column0 + column;
    if (h < a.group)
        store_row4(a.y + rec.x * a.ldy + (long long)(kv_head * a.group + h) * D + 4 * piece, sum, column == 0 ? sum_w.x : column == 1 ? sum_w.y : column == 2 ? sum_w.z : sum_w.w);
}

int tiles(int group) { return group <= 8 ? 1 : 2; }

// Thread blocks: as many as the GPU holds at once, no more than there can be work for.
int64_t block_count(const nq_kv_pages* c, int64_t q_heads, int64_t seqs, int64_t table_cols) {
    const int group = (int)(q_heads / c->kv_heads), nt = tiles(group);
    const int64_t per = (group + 8 * nt - 1) / (8 * nt) * c->kv_heads * ((table_cols * c->page_size + step_tokens(c->head_dim, c->dtype) - 1) / step_tokens(c->head_dim, c->dtype));     // steps of the longest sequence
    const int64_t most = (nt == 1 && !(c->head_dim == 128 && c->dtype != NQ_BF16) ? 3 : 2) * (int64_t)sm_count();
    if (per >= most * kWarps || seqs >= most * kWarps) return most;
    const int64_t need = (per * seqs + kWarps - 1) / kWarps;
    return need < 1 ? 1 : need < most ? need : most;
}
int64_t slot_floats(const nq_kv_pages* c, int64_t q_heads) { return 8ll * tiles((int)(q_heads / c->kv_heads)) * (c->head_dim + 2); }

int check_call(const nq_kv_pages* c, int64_t q_heads, int64_t seqs, int64_t table_cols) {
    const int bad = check_pages(c);
    if (bad != NQ_OK) return bad;
    if (q_heads <= 0 || q_heads % c->kv_heads || seqs < 0 || table_cols < 0) return NQ_ERR_INVALID_ARG;
    if (q_heads > 65536 || seqs >= 1 << 30 || table_cols > 0x7fffffffll / c->page_size) return NQ_ERR_UNSUPPORTED;
    return NQ_OK;
}

template <int D, int CACHE, int NT>
int launch_token(const TokenArgs& a, unsigned blocks, cudaStream_t s) {
    const int smem = 2 * kWarps * kSlotFloats<D, NT> * (int)sizeof(float);
    if (smem > 48 * 1024 - 2048 && cudaFuncSetAttribute(token_kernel<D, CACHE, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
        (void)cudaGetLastError();
        return NQ_ERR_CUDA;
    }
    const int st = launch_chained(token_kernel<D, CACHE, NT>, blocks, kThreads, smem, 1, s, a);
    if (st != NQ_OK || blocks == 1) return st;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks, 2 * NT, 1);
    cfg.blockDim = dim3(kJoin, 1, 1);
    cfg.stream = s;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, join_kernel<D, NT>, a) != cudaSuccess) {
        (void)cudaGetLastError();
        return NQ_ERR_CUDA;
    }
    return NQ_OK;
}
template <int D, int CACHE>
int launch_tiles(const TokenArgs& a, unsigned blocks, cudaStream_t s) {
    return tiles(a.group) == 1 ? launch_token<D, CACHE, 1>(a, blocks, s) : launch_token<D, CACHE, 2>(a, blocks, s);
}
template <int D>
int launch_cache(const TokenArgs& a, int cache, unsigned blocks, cudaStream_t s) {
    return cache == NQ_BF16 ? launch_tiles<D, NQ_BF16>(a, blocks, s) : cache == NQ_E4M3 ? launch_tiles<D, NQ_E4M3>(a, blocks, s) : launch_tiles<D, NQ_I8>(a, blocks, s);
}

}  // namespace
}  // namespace nq

extern "C" int64_t nq_paged_attention_workspace_bytes(const nq_kv_pages* cache, int64_t q_heads, int64_t seqs, int64_t table_cols) {
    if (nq::check_call(cache, q_heads, seqs, table_cols) != NQ_OK) return -1;
    return nq::block_count(cache, q_heads, seqs, table_cols) * (int64_t)(sizeof(int4) + 2 * sizeof(float) * nq::slot_floats(cache, q_heads));
}

extern "C" int nq_paged_attention(const nq_kv_pages* cache, const void* Q, int64_t ldq, int64_t q_heads, const int32_t* table, int64_t ld_table,
                                  int64_t table_cols, const int32_t* lengths, int64_t seqs, int window, float scale, void* Y, int64_t ldy,
                                  void* workspace, int64_t workspace_bytes, void* stream) {
    using nq::misaligned;
    const int bad = nq::check_call(cache, q_heads, seqs, table_cols);
    if (bad != NQ_OK) return bad;
    if (window < 0 || !(scale > 0.0f) || !(scale - scale == 0.0f)) return NQ_ERR_INVALID_ARG;
    if (seqs == 0) return NQ_OK;
    const int64_t width = q_heads * cache->head_dim;
    if (!Q || !Y || !lengths || (table_cols > 0 && (!table || ld_table < table_cols)) || ldq < width || ldy < width) return NQ_ERR_INVALID_ARG;
    if (misaligned(Q, 16) || misaligned(Y, 16) || (ldq & 7) || (ldy & 7) || misaligned(table, 4) || misaligned(lengths, 4) || misaligned(workspace, 16)) return NQ_ERR_ALIGNMENT;
    const int64_t blocks = nq::block_count(cache, q_heads, seqs, table_cols);
    if (!workspace || workspace_bytes < nq_paged_attention_workspace_bytes(cache, q_heads, seqs, table_cols)) return NQ_ERR_WORKSPACE;
    nq::TokenArgs a = {};
    a.c = nq::pages_of(cache);
    a.q = static_cast<const __nv_bfloat16*>(Q); a.ldq = ldq; a.q_heads = (int)q_heads; a.group = (int)(q_heads / cache->kv_heads);
    a.head_blocks = (a.group + 8 * nq::tiles(a.group) - 1) / (8 * nq::tiles(a.group));
    a.table = table; a.ld_table = ld_table; a.table_tokens = (int)(table_cols * cache->page_size);
    a.lengths = lengths; a.seqs = (int)seqs; a.window = window; a.scale2 = scale * 1.44269504088896341f;
    a.y = static_cast<__nv_bfloat16*>(Y); a.ldy = ldy;
    a.records = static_cast<int4*>(workspace);
    a.slots = reinterpret_cast<float*>(a.records + blocks);
    const cudaStream_t s = (cudaStream_t)stream;
    return cache->head_dim == 64 ? nq::launch_cache<64>(a, cache->dtype, (unsigned)blocks, s) : nq::launch_cache<128>(a, cache->dtype, (unsigned)blocks, s);
}
