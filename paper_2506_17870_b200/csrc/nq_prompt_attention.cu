// Attention over whole prompts of different lengths, packed behind one another.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/nq.h"
#include "nq_fp8.cuh"
#include "nq_internal.cuh"
#include "nq_ranges.cuh"
#include "nq_sm100.cuh"
#include "nq_sm100_bf16.cuh"

namespace nq {
namespace {

using namespace sm100;

// A unit of work is two tiles of 128 rows of queries that read the same keys: 256 rows of a head, or 128 of two heads; a thread block works
// through units, one block an SM.
// For each 64 keys ("step") and tile:  S = Q K^T into one of the tile's two score buffers in tensor memory (64 columns), the tile's four
// softmax warps read a row a thread, keep its maximum and sum, write the weights back as bf16 over S, and O += P V takes them from there
// (P as the operand in tensor memory, V as it lies, N-major).  A tile's products go  PV(j - 2)  QK(j)  into the same buffer, while the
// softmax is at step j - 1 in the other.  (Steps of 128 keys and one buffer, tiles taking turns: each waits out the other's round trip,
// 16384 tokens of 8 heads 552 us.)
// Measured: 16384 tokens, 8 / 2 heads of 128, causal: 421 us as a burst, 1.31 PFLOP/s (0.78 of the measured bf16 rate), some 520 back to back under
// the power limit; tensor pipe, exponentials and issue are each about half busy, what bounds a step is the round trip.
// The running maximum moves only when a score passes it by 2^8, so the sums in tensor memory are seldom rescaled (by the softmax warps:
// S(j) being there says that PV(j - 2) is complete, for the tensor core works in order; PV(j - 1) has a barrier).
// A warp looks after V where a step has hidden keys (the last of a sequence, the diagonal, a window's edge): rows of V behind the
// sequence are zeroed, since 0 x NaN is NaN in the product, and where the sequence's own rows hold infinities or NaN, the tiles that
// hide some of the step take their weights times V by themselves, only what each row sees.
constexpr int kThreads = 384;            // warp 0 TMA and units, warps 1 and 2 MMA of the tiles (1 also TMEM), warp 3 looks after V, warps 4-7 and 8-11 softmax of the tiles
constexpr int kTile = 128, kKeys = 64;   // rows of a tile, keys of a step
constexpr float kRescale = 8.0f;
// The tensor core cuts each product off some 25 bits below the running sum that it is added to, towards zero: over n keys whose values have one sign
// that takes n 2^-27 of a sum (measured: 0.8 % of 2^20 keys, 10 % of 2^24).  So every kFold steps (a part: 2^16 keys) a row's sums go to fp32 sums of
// the thread's own, in local memory, and start anew; its sum of weights likewise.
constexpr int kFold = 1024;              // (a power of two)

template <int D>
struct Shape {
    static constexpr int kTileBytes = kTile * D * 2, kStageBytes = kKeys * D * 2;
    static constexpr int kStages = D == 128 ? 4 : 8;          // of K, and of V
    static constexpr int kOut = 2048;                         // a softmax warp's rows on their way out: 32 of 64 bytes
    static constexpr int kSmem = 2 * kTileBytes + 2 * kStages * kStageBytes + 8 * kOut + 1024 + 1024;
    static constexpr int kSlabQ = kTile * 128, kSlab = kKeys * 128;      // 64 values of all rows of a tile, of a stage
};

struct PromptArgs {
    const int *starts_q, *starts_k;
    int seqs, rows_q, rows_k, group, causal, window;
    int heads;                           // query heads, or pairs of them: what a unit is made for
    int per_unit, span, next_row;        // a unit is 128 rows (`span`) of two heads that share their keys, or 256 of one, whose second tile starts next_row on
    float scale2;                        // score scale * log2(e)
    __nv_bfloat16* y;
    long long ldy;
    unsigned int* status;
};

struct Unit {
    int q0, k0;                          // rows of the tensors: the sequence's first query and key
    int lq, lk;                          // its lengths
    int row[2], head[2];                 // of each tile: its first row in the sequence, and its query head
    int lo[2], hi[2];                    // steps of each tile (hi <= lo: none)
    int all_lo[2], all_hi[2];            // keys that all rows of the tile see
    int begin, end;                      // steps of either
    __device__ __forceinline__ bool takes(int t, int j) const { return j >= lo[t] && j < hi[t]; }
    __device__ __forceinline__ bool hides(int t, int j) const { return takes(t, j) && (j * kKeys < all_lo[t] || (j + 1) * kKeys > all_hi[t]); }
};

__device__ __forceinline__ int clamp_start(int v, int low, int high) { return min(max(v, low), high); }

// `before`: units (of one head) before each chunk of sequences
__device__ __forceinline__ void unit_of(const PromptArgs& a, const int* before, int chunk, int index, Unit& u) {
    const int pair = before[kThreads] - 1 - index / a.heads;       // the longest rows of a causal prompt first
    const int head = index % a.heads * a.per_unit;
    int lo = 0, hi = kThreads;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (before[mid] <= pair) lo = mid; else hi = mid;
    }
    int rest = pair - before[lo], s = lo * chunk;
    for (;; ++s) {
        u.q0 = clamp_start(a.starts_q[s], 0, a.rows_q);
        u.lq = clamp_start(a.starts_q[s + 1], u.q0, a.rows_q) - u.q0;
        const int n = (u.lq + a.span - 1) / a.span;
        if (rest < n) break;
        rest -= n;
    }
    u.k0 = clamp_start(a.starts_k[s], 0, a.rows_k);
    u.lk = clamp_start(a.starts_k[s + 1], u.k0, a.rows_k) - u.k0;
    const int off = u.lk - u.lq;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        u.row[t] = rest * a.span + t * a.next_row;
        u.head[t] = head + t * (a.per_unit - 1);
        const int a0 = u.row[t], b0 = min(a0 + kTile, u.lq);                       // rows [a0, b0)
        u.lo[t] = u.hi[t] = u.all_lo[t] = u.all_hi[t] = 0;
        if (a0 >= b0) continue;
        const int seen_hi = a.causal ? min(u.lk, b0 + off) : u.lk, seen_lo = window_start(a.window, a0 + off + 1);
        u.all_hi[t] = a.causal ? min(u.lk, a0 + off + 1) : u.lk;
        u.all_lo[t] = window_start(a.window, b0 + off);
        if (seen_hi > seen_lo) {
            u.lo[t] = seen_lo / kKeys;
            u.hi[t] = (seen_hi + kKeys - 1) / kKeys;
        }
    }
    const bool one = u.hi[0] > u.lo[0], two = u.hi[1] > u.lo[1];
    u.begin = one && two ? min(u.lo[0], u.lo[1]) : one ? u.lo[0] : u.lo[1];
    u.end = one && two ? max(u.hi[0], u.hi[1]) : one ? u.hi[0] : u.hi[1];
}

__device__ __forceinline__ float exp2a(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));       // a NaN shows
    return r;
}
// Asks for a thread block of this grid that has not begun: its launch is cancelled, and 16 bytes that name it (or say that there is none)
// arrive at `to` and are counted on `bar`.
__device__ __forceinline__ void cancel_next(uint32_t to, uint32_t bar) {
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(to), "r"(bar) : "memory");
}
// The block's number, -1 where there was none.
__device__ __forceinline__ int cancelled(uint32_t from) {
    int index;
    asm volatile(
        "{\n\t.reg .pred P;\n\t.reg .b128 h;\n\t"
        "ld.shared.b128 h, [%1];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 P, h;\n\t"
        "mov.b32 %0, -1;\n\t"
        "@P clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, h;\n\t}"
        : "=r"(index) : "r"(from) : "memory");
    return index;
}
// scores of the columns outside [lo, hi) to -infinity
__device__ __forceinline__ void hide(uint32_t (&s)[32], int lo, int hi) {
    const uint32_t below = lo <= 0 ? 0u : lo >= 32 ? ~0u : (1u << lo) - 1u, under = hi <= 0 ? 0u : hi >= 32 ? ~0u : (1u << hi) - 1u;
    const uint32_t keep = under & ~below;
#pragma unroll
    for (int c = 0; c < 32; ++c) s[c] = (keep >> c) & 1u ? s[c] : 0xff800000u;
}

// Weights 2^(s scale + minus) of 32 scores, their sum, and as pairs of bf16 (a weight is off by at most 2^-8 of itself).
// The exponential unit takes 4 a cycle and scheduler, which alone would be as long as both products.  So 3 of 8 come from the other
// pipes: 2^y = 2^n 2^f, n = y rounded (y + 1.5 * 2^23 holds it in its low bits), f in [-1/2, 1/2] by a polynomial of degree 3, fitted
// to 2^f for the least relative error on that interval: 7.5e-5 (2^-13.7), where a weight's rounding is 2^-8.  y under -127 counts as that,
// whose 2^n is made as 0; a NaN stays one.  (16384 tokens of 8 heads: none 492 us, one of 8 476, one of 4 428, 3 of 8 421.)
__device__ __forceinline__ void weights_of(const uint32_t (&s)[32], float scale, float minus, uint64_t& sum, uint32_t (&p)[16]) {
    constexpr float kBig = 12582912.0f;
#pragma unroll
    for (int c = 0; c < 32; c += 2) {
        const uint64_t y = fma2(pack2(s[c], s[c + 1]), both(scale), both(minus));
        float e0, e1;
        unpack2(y, e0, e1);
        uint64_t e;
        if ((c / 2) % 8 >= 5) {
            const uint64_t z = pack2f(max3(e0, e0, -127.0f), max3(e1, e1, -127.0f));
            const uint64_t big = add2(z, both(kBig)), f = fma2(add2(big, both(-kBig)), both(-1.0f), z);
            const uint64_t q = fma2(fma2(fma2(both(0.0551716793f), f, both(0.2426111685f)), f, both(0.6932609878f)), f, both(0.9999280708f));
            float n0, n1;
            unpack2(big, n0, n1);
            e = mul2(q, pack2((__float_as_uint(n0) << 23) + 0x3f800000u, (__float_as_uint(n1) << 23) + 0x3f800000u));
        } else {
            e = pack2f(exp2a(e0), exp2a(e1));
        }
        sum = add2(sum, e);
        unpack2(e, e0, e1);
        p[c / 2] = bf16x2(e0, e1);
    }
}

// A row's sums in tensor memory and those of its parts so far (none: !more), the latter times `then`, together: to the parts, or back.  (A function
// of its own: in the place of its calls it slowed down every step, 16384 tokens of 8 heads 433 -> 443 us and, at a step's end, 467.)
template <int D>
__device__ __noinline__ void fold(uint32_t o_at, float* far, bool more, float then, bool back) {
#pragma unroll 1
    for (int c0 = 0; c0 < D; c0 += 32) {
        uint32_t o[32];
        tmem_ld_32x32(o_at + c0, o);
        tmem_ld_wait();
        tmem_arrived(o);
#pragma unroll
        for (int c = 0; c < 32; ++c) {
            const float x = __uint_as_float(o[c]) + (more ? far[c0 + c] * then : 0.0f);
            if (back) o[c] = __float_as_uint(x); else far[c0 + c] = x;
        }
        if (back) tmem_st_32x32(o_at + c0, o);
    }
    tmem_st_wait();
}

// LONG: a sequence may have more than kFold steps of keys.
template <int D, bool LONG>
__global__ void __launch_bounds__(kThreads, 1)
prompt_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const PromptArgs a) {
    using P = Shape<D>;
    constexpr int ST = P::kStages;
    constexpr uint32_t kS = 0, kO = 256;                       // tensor memory columns: S of tile t at kS + 128 t (two buffers of 64), O at kO + D t
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    // shared-memory addresses: tiles of Q [2], stages of K [ST] and of V [ST], rows on their way out [8 warps], then barriers
    const uint32_t sQ = smem_u32(smem), sK = sQ + 2 * P::kTileBytes, sV = sK + ST * P::kStageBytes, bars = sV + ST * P::kStageBytes + 8 * P::kOut;
    const uint32_t q_full = bars, q_empty = bars + 8, s_full = bars + 16, p_full = bars + 48, o_full = bars + 80;       // one, one, [2 tiles][2 buffers] each
    const uint32_t k_full = bars + 112, k_empty = k_full + 8 * ST, v_full = k_empty + 8 * ST, v_empty = v_full + 8 * ST, v_ok = v_empty + 8 * ST;   // [ST]
    const uint32_t u_full = v_ok + 8 * ST, u_empty = u_full + 16, c_full = u_empty + 16;                                // [2], [2], one
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + 2 * P::kTileBytes + 2 * ST * P::kStageBytes + 8 * P::kOut + 112 + 40 * ST + 40);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    volatile int* v_odd = abort_flag + 1;                      // [ST]: whether the step's V holds what is no number
    __shared__ int s_before[kThreads + 1];
    __shared__ int s_warp[kThreads / 32];
    __shared__ Unit s_unit[2];
    __shared__ __align__(16) uint4 s_cancelled;

    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;      // (the compiler then knows that a warp shares it)
    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        mbar_init(q_empty, 2);
        for (int t = 0; t < 4; ++t) {
            mbar_init(s_full + 8 * t, 1);
            mbar_init(p_full + 8 * t, 4);
            mbar_init(o_full + 8 * t, 1);
        }
        for (int s = 0; s < ST; ++s) {
            mbar_init(k_full + 8 * s, 1);
            mbar_init(k_empty + 8 * s, 2);
            mbar_init(v_full + 8 * s, 1);
            mbar_init(v_empty + 8 * s, 3);                     // both tiles' products, and the warp that looks after V
            mbar_init(v_ok + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) { mbar_init(u_full + 8 * s, 1); mbar_init(u_empty + 8 * s, 11); }       // warps 1 to 3, softmax
        mbar_init(c_full, 1);
        *abort_flag = 0;
        fence_barrier_init();
        prefetch_tensormap(&tmQ);
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    start_next();
    wait_previous();

    // units of one head (or pair) before each chunk of sequences
    const int chunk = (a.seqs + kThreads - 1) / kThreads;
    {
        int sum = 0;
        for (int s = threadIdx.x * chunk; s < min(a.seqs, (int)(threadIdx.x + 1) * chunk); ++s) {
            const int from = clamp_start(a.starts_q[s], 0, a.rows_q);
            sum += (clamp_start(a.starts_q[s + 1], from, a.rows_q) - from + a.span - 1) / a.span;
        }
#pragma unroll
        for (int m = 1; m < 32; m *= 2) {
            const int o = __shfl_up_sync(0xffffffffu, sum, m);
            if (lane >= m) sum += o;
        }
        if (lane == 31) s_warp[warp] = sum;
        __syncthreads();
        for (int w = 0; w < warp; ++w) sum += s_warp[w];
        s_before[threadIdx.x + 1] = sum;
        if (threadIdx.x == 0) s_before[0] = 0;
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    const int units = s_before[kThreads] * a.heads;          // the host has checked that it fits

    // The grid has a block for each unit that there can be; a block that is done with its own takes one that has not begun (it
    // cancels that block's launch), so that all SMs end together however the units differ.  Warp 0 does this, one unit ahead of the
    // tensor core, and hands what it has worked out to the others.
    // The n-th unit of this block, for a whole warp until it gives it back; null: no more of them, or given up.  `idle`: steps of the unit before
    // that this warp had no part in.
    const auto take = [&](uint32_t n, int idle) -> const Unit* {
        const bool ok = mbar_wait(u_full + 8 * (n & 1), (n >> 1) & 1, abort_flag, a.status, 0x301u, wait_limit(kWaitLimitCycles, idle));
        return __all_sync(0xffffffffu, ok) && s_unit[n & 1].lq > 0 ? &s_unit[n & 1] : nullptr;
    };
    const auto give_back = [&](uint32_t n) {
        __syncwarp();
        if (lane == 0) mbar_arrive(u_empty + 8 * (n & 1));
    };

    // 128 x 72 + 256 x 216 registers, all of the 384 x 168 that the block was launched with
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == 0) {
            if (lane == 0) {
                uint32_t it = 0, used = 0, asks = 0;               // steps, units with any step, cancellations so far
                bool ok = true;
                int index = blockIdx.x;                            // -1: no more
                const uint32_t answer = smem_u32(&s_cancelled);
                const auto ask = [&] {
                    mbar_arrive_expect_tx(c_full, 16);
                    cancel_next(answer, c_full);
                };
                const auto answered = [&] {
                    ok = mbar_wait(c_full, asks++ & 1, abort_flag, a.status, 0x313u);
                    index = ok ? cancelled(answer) : -1;
                    fence_proxy_async_smem();
                };
                for (uint32_t n = 0;; ++n) {
                    while (index >= units) {                       // (the host knows no more than how many units there can be)
                        ask();
                        answered();
                    }
                    if (!ok || !(ok = mbar_wait(u_empty + 8 * (n & 1), ((n >> 1) & 1) ^ 1, abort_flag, a.status, 0x314u))) break;
                    Unit& u = s_unit[n & 1];
                    if (index >= 0) unit_of(a, s_before, chunk, index, u);
                    else u.lq = 0;
                    mbar_arrive(u_full + 8 * (n & 1));
                    if (index < 0) break;
                    const int begin = u.begin, end = u.end;
                    if (end > begin) {
                        if (!(ok = mbar_wait(q_empty, (used & 1) ^ 1, abort_flag, a.status, 0x310u))) break;
                        ++used;
                        const bool one = u.hi[0] > u.lo[0], two = u.hi[1] > u.lo[1];
                        const int kv_head = u.head[0] / a.group, k0 = u.k0;
                        mbar_arrive_expect_tx(q_full, (one + two) * P::kTileBytes);
#pragma unroll
                        for (int h = 0; h < D / 64; ++h) {
                            if (one) tma_load_3d(sQ + h * P::kSlabQ, &tmQ, 64 * h, u.head[0], u.q0 + u.row[0], q_full);
                            if (two) tma_load_3d(sQ + P::kTileBytes + h * P::kSlabQ, &tmQ, 64 * h, u.head[1], u.q0 + u.row[1], q_full);
                        }
                        for (int j = begin; j < end; ++j, ++it) {
                            const uint32_t s = it % ST, use = it / ST;
                            // the next unit is asked for as late as its answer still comes in time: asked for at this one's start, a
                            // long unit's block takes a second one that others would begin earlier (8192 tokens of 8 heads 165 -> 208 us)
                            if (j == end - 1) ask();
                            if (!(ok = mbar_wait(k_empty + 8 * s, (use & 1) ^ 1, abort_flag, a.status, 0x311u))) break;
                            mbar_arrive_expect_tx(k_full + 8 * s, P::kStageBytes);
#pragma unroll
                            for (int h = 0; h < D / 64; ++h)
                                tma_load_3d(sK + s * P::kStageBytes + h * P::kSlab, &tmK, 64 * h, kv_head, k0 + j * kKeys, k_full + 8 * s);
                            if (!(ok = mbar_wait(v_empty + 8 * s, (use & 1) ^ 1, abort_flag, a.status, 0x312u))) break;
                            mbar_arrive_expect_tx(v_full + 8 * s, P::kStageBytes);
#pragma unroll
                            for (int h = 0; h < D / 64; ++h)
                                tma_load_3d(sV + s * P::kStageBytes + h * P::kSlab, &tmV, 64 * h, kv_head, k0 + j * kKeys, v_full + 8 * s);
                        }
                    }
                    if (!ok) break;
                    if (end <= begin) ask();
                    answered();
                }
                if (!ok) {
                    const long long t0 = clock64();                // let copies in flight land before shared memory is released
                    while (clock64() - t0 < (1ll << 22)) { }
                }
            }
        } else if (warp < 3) {
            // A tile's products, in a warp of their own: while one waits for a barrier, which takes a few hundred cycles even if it has long
            // been arrived on, the tensor core has the other's to do.  The whole warp goes through this together, and one thread issues: where
            // one thread alone runs the loop, the compiler does not know an instruction's operands to be the warp's, and each takes some
            // 100 cycles to issue (16384 tokens of 8 heads, both tiles from one thread: 888 us; from one warp: 682).
            constexpr uint32_t kQK = idesc_bf16(kTile, kKeys, false), kPV = idesc_bf16(kTile, D, true);
            const int t = warp - 1;
            const bool leader = elect_one();
            const auto same = [](int v) { return __shfl_sync(0xffffffffu, v, 0); };
            // A barrier's answer takes 100 cycles and more to come, so those of a step are asked together.  (Each of them holds its phase until
            // this warp has gone on.)
            const auto wait = [&](uint32_t b0, uint32_t p0, uint32_t b1, uint32_t p1, uint32_t b2, uint32_t p2, unsigned code) {
                bool all = mbar_try_wait(b0, p0);
                all &= mbar_try_wait(b1, p1);
                all &= mbar_try_wait(b2, p2);
                if (__all_sync(0xffffffffu, all)) return true;
                all = mbar_wait(b0, p0, abort_flag, a.status, code) && mbar_wait(b1, p1, abort_flag, a.status, code + 1) && mbar_wait(b2, p2, abort_flag, a.status, code + 2);
                return (bool)__all_sync(0xffffffffu, all);
            };
            const uint64_t dq = smem_desc_sw128(sQ + t * P::kTileBytes), dk0 = smem_desc_sw128(sK), dv0 = smem_desc_mn_sw128(sV, P::kSlab);
            const uint32_t sums = tmem + kO + t * D;
            uint32_t it = 0, used = 0, weights = 0;                // steps, units with any, a phase bit for each buffer
            bool ok = true;
            for (uint32_t n = 0; ok; ++n) {
                const Unit* u = take(n, 0);
                if (!u) break;
                const int first = same(u->begin), last = same(u->end), lo = same(u->lo[t]), hi = same(u->hi[t]), all_lo = same(u->all_lo[t]), all_hi = same(u->all_hi[t]);
                give_back(n);
                if (last <= first) continue;
                if (!(ok = wait(q_full, used & 1, q_full, used & 1, q_full, used & 1, 0x320u))) break;
                ++used;
                // step j's scores, and the sums of step j - 2, whose weights are where those scores go
                for (int j = first; j < last + 2; ++j) {
                    const uint32_t i = it + (j - first), s = i % ST, sp = (i - 2) % ST, parity = ((i - 2) / ST) & 1, buffer = j & 1;
                    const uint32_t scores = tmem + kS + t * kTile + buffer * kKeys;
                    const bool sums_due = j - 2 >= lo && j - 2 < hi, scores_due = j >= lo && j < hi;
                    bool by_hand = false;
                    // the step's keys, and the values and weights of step j - 2, each where there is such a step
                    const bool keys = j < last, values = j >= first + 2;
                    const uint32_t kb = k_full + 8 * s, kp = (i / ST) & 1, vb = v_full + 8 * sp;
                    if (sums_due) {                            // (then there are values)
                        if (!(ok = wait(p_full + 16 * t + 8 * buffer, (weights >> buffer) & 1, vb, parity, keys ? kb : vb, keys ? kp : parity, 0x323u))) break;
                        weights ^= 1u << buffer;
                        if ((j - 2) * kKeys < all_lo || (j - 1) * kKeys > all_hi) {
                            const uint32_t ob = v_ok + 8 * sp;
                            if (!(ok = wait(ob, parity, ob, parity, ob, parity, 0x326u))) break;
                            by_hand = v_odd[sp];
                        }
                    } else if (keys || values) {
                        if (!(ok = wait(keys ? kb : vb, keys ? kp : parity, values ? vb : kb, values ? parity : kp, keys ? kb : vb, keys ? kp : parity, 0x329u))) break;
                    }
                    tc_fence_after_sync();
                    if (leader) {
                        if (sums_due && !by_hand) {
                            const uint64_t dv = dv0 + sp * (P::kStageBytes / 16);
#pragma unroll
                            for (int k = 0; k < kKeys / 16; ++k) mma_bf16_ts(sums, scores + 8 * k, dv + k * (16 * 128 / 16), kPV, k > 0 || (LONG ? ((j - 2 - lo) & (kFold - 1)) != 0 : j - 2 > lo));
                        }
                        if (scores_due) {
                            const uint64_t dk = dk0 + s * (P::kStageBytes / 16);
#pragma unroll
                            for (int k = 0; k < D / 16; ++k)
                                mma_bf16(scores, dq + (k % 4) * 2 + (k / 4) * (P::kSlabQ / 16), dk + (k % 4) * 2 + (k / 4) * (P::kSlab / 16), kQK, k > 0);
                            mma_commit(s_full + 16 * t + 8 * buffer);
                        }
                        if (sums_due) mma_commit(o_full + 16 * t + 8 * buffer);
                        if (j >= first + 2) mma_commit(v_empty + 8 * sp);
                        if (j < last) mma_commit(k_empty + 8 * s);
                        if (j == last - 1) mma_commit(q_empty);
                    }
                    __syncwarp();
                }
                it += last - first;
            }
        } else {
            // V where a step hides something.  Every step is waited for and confirmed, for a wait must not be more than one phase behind its
            // barrier.
            uint32_t it = 0;
            bool ok = true;
            for (uint32_t n = 0; ok; ++n) {
                const Unit* u = take(n, 0);
                if (!u) break;
                for (int j = u->begin; j < u->end; ++j, ++it) {
                    const uint32_t s = it % ST;
                    ok = mbar_wait(v_full + 8 * s, (it / ST) & 1, abort_flag, a.status, 0x330u);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    if (u->hides(0, j) || u->hides(1, j)) {
                        const int live = u->lk - j * kKeys;        // rows of the sequence
                        uint8_t* v0 = smem + 2 * P::kTileBytes + (ST + s) * P::kStageBytes + (lane >> 3) * 128 + (lane & 7) * 16;
                        // a lane takes a 16-byte piece of every fourth row: 8 lanes are a row of 64 values
                        for (int x = max(0, live) & ~3; x < kKeys; x += 4)
                            if (x + (lane >> 3) >= live)
#pragma unroll
                                for (int h = 0; h < D / 64; ++h) *reinterpret_cast<uint4*>(v0 + h * P::kSlab + x * 128) = make_uint4(0, 0, 0, 0);
                        uint32_t odd = 0;
                        if (a.causal || a.window) {                // (otherwise all that is left is seen by all)
#pragma unroll 16
                            for (int x = 0; x < D; x += 4) {       // rows x % 64 of slab x / 64
                                const uint4 v = *reinterpret_cast<const uint4*>(v0 + x / 64 * P::kSlab + x % 64 * 128);
                                odd |= ((v.x & 0x7f807f80u) + 0x00800080u) | ((v.y & 0x7f807f80u) + 0x00800080u) | ((v.z & 0x7f807f80u) + 0x00800080u) |
                                       ((v.w & 0x7f807f80u) + 0x00800080u);
                            }
                        }
                        const bool any = __any_sync(0xffffffffu, (odd & 0x80008000u) != 0);
                        fence_proxy_async_smem();
                        if (lane == 0) v_odd[s] = any;
                    }
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(v_ok + 8 * s);
                        mbar_arrive(v_empty + 8 * s);
                    }
                }
                give_back(n);
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int t = (warp - 4) >> 2, quarter = warp & 3;         // a row a thread
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const uint32_t o_at = tmem + kO + t * D + lanes;
        uint32_t it = 0, phases = 0;                               // steps of all, a phase bit for each buffer
        bool ok = true;
        // PV(j) of the last step but one or the last so far is complete.  (The one before it with this buffer is known to be: S(j + 2), or the
        // end of the unit before, said so; a barrier is never two phases ahead of one who waits for it.)
        const auto sums_of = [&](int j) {
            return mbar_wait(o_full + 16 * t + 8 * (j & 1), ((phases >> (j & 1)) & 1) ^ 1, abort_flag, a.status, 0x342u);
        };
        // A tile without rows (the second one of a head's last rows) is done at once, and its warps wait for the next unit as long as the
        // other tile has steps: with 10^8 keys that is longer than a step's limit.
        int idle = 0;
        float far[LONG ? D + 2 : 1];                               // sums of the parts so far, the maximum that they go with, the sum of their weights
        for (uint32_t n = 0; ok; ++n, give_back(n - 1)) {
            const Unit* u = take(n, idle);
            if (!u) break;
            const int lo_t = u->lo[t], hi_t = u->hi[t], all_lo = u->all_lo[t], all_hi = u->all_hi[t];
            const int row = u->row[t] + quarter * 32 + lane;
            // of the keys, this row sees no more than the first `reach`, and of those the last `window`; rows behind the last one must not
            // get in the way
            const int reach = u->lk - (u->lq - 1 - min(row, u->lq - 1));
            const int see_hi = a.causal ? min(u->lk, reach) : u->lk, see_lo = window_start(a.window, reach);
            const uint32_t it0 = it - u->begin;                    // steps before step 0
            it += u->end - u->begin;
            float top = -INFINITY, total = 0.0f;
            bool there = false;                                    // the next step's scores, as far as is known
            int from, upto = lo_t;                                 // steps of the sums in tensor memory
            do {
                from = upto;
                upto = LONG ? min(from + kFold, hi_t) : hi_t;
                for (int j = from; j < upto; ++j) {
                    const uint32_t s_at = tmem + kS + t * kTile + (j & 1) * kKeys + lanes;
                    if (!__all_sync(0xffffffffu, there)) {
                        ok = mbar_wait(s_full + 16 * t + 8 * (j & 1), (phases >> (j & 1)) & 1, abort_flag, a.status, 0x340u);
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) break;
                    }
                    phases ^= 1u << (j & 1);
                    tc_fence_after_sync();
                    const bool hides = j * kKeys < all_lo || (j + 1) * kKeys > all_hi;
                    const int lo = see_lo - j * kKeys, hi = see_hi - j * kKeys;                  // columns that this row sees
                    uint32_t s[2][32];
                    tmem_ld_32x32(s_at, s[0]);
                    tmem_ld_32x32(s_at + 32, s[1]);
                    tmem_ld_wait();
                    float m = -INFINITY, m1 = -INFINITY, m2 = -INFINITY, m3 = -INFINITY;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        tmem_arrived(s[x]);
                        if (hides) hide(s[x], lo - 32 * x, hi - 32 * x);
                    }
#pragma unroll
                    for (int c = 0; c < 32; c += 4) {
                        m = max3(m, __uint_as_float(s[0][c]), __uint_as_float(s[0][c + 1]));
                        m1 = max3(m1, __uint_as_float(s[0][c + 2]), __uint_as_float(s[0][c + 3]));
                        m2 = max3(m2, __uint_as_float(s[1][c]), __uint_as_float(s[1][c + 1]));
                        m3 = max3(m3, __uint_as_float(s[1][c + 2]), __uint_as_float(s[1][c + 3]));
                    }
                    m = max3(m, m1, max3(m2, m2, m3)) * a.scale2;
                    const bool move = m > top + kRescale;
                    if (__any_sync(0xffffffffu, move)) {
                        const float to = fmaxf(top, m), by = top == -INFINITY ? 0.0f : exp2a(top - to);
                        top = to;
                        total *= by;
                        if (j > from) {
                            // (that S(j) is there says that PV(j - 2) is complete)
                            ok = sums_of(j - 1);
                            ok = __all_sync(0xffffffffu, ok);
                            if (!ok) break;
                            tc_fence_after_sync();
#pragma unroll 1
                            for (int c0 = 0; c0 < D; c0 += 32) {
                                uint32_t o[32];
                                tmem_ld_32x32(o_at + c0, o);
                                tmem_ld_wait();
                                tmem_arrived(o);
#pragma unroll
                                for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * by);
                                tmem_st_32x32(o_at + c0, o);
                            }
                        }
                    }
                    const float minus = top == -INFINITY ? 0.0f : -top;
                    uint64_t sum = 0;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        uint32_t p[16];
                        weights_of(s[x], a.scale2, minus, sum, p);
                        tmem_st_32x16(s_at + 16 * x, p);
                    }
                    total += sum2(sum);
                    there = j + 1 < hi_t && mbar_try_wait(s_full + 16 * t + 8 * ((j + 1) & 1), (phases >> ((j + 1) & 1)) & 1);
                    tmem_st_wait();
                    if (hides) {
                        const uint32_t sl = (it0 + j) % ST;
                        ok = mbar_wait(v_ok + 8 * sl, ((it0 + j) / ST) & 1, abort_flag, a.status, 0x341u);
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) break;
                        if (v_odd[sl]) {
                            // some of V is no number, and this tile hides some of it: the product by hand, of what each row sees
                            if (j > from) {
                                ok = sums_of(j - 1);
                                ok = __all_sync(0xffffffffu, ok);
                                if (!ok) break;
                                tc_fence_after_sync();
                            }
#pragma unroll 1
                            for (int c0 = 0; c0 < D; c0 += 32) {
                                uint32_t o[32];
                                if (j > from) {
                                    tmem_ld_32x32(o_at + c0, o);
                                    tmem_ld_wait();
                                    tmem_arrived(o);
                                } else {
#pragma unroll
                                    for (int c = 0; c < 32; ++c) o[c] = 0;
                                }
#pragma unroll 1
                                for (int k = 0; k < kKeys; ++k) {
                                    uint32_t two = tmem_ld_32x1(s_at + k / 2);
                                    tmem_ld_wait();
                                    asm volatile("" : "+r"(two));
                                    const float w = __uint_as_float((k & 1) ? two & 0xffff0000u : two << 16);
                                    const bool seen = k >= lo && k < hi;
                                    const uint8_t* v = smem + 2 * P::kTileBytes + (ST + sl) * P::kStageBytes + (c0 / 64) * P::kSlab + k * 128;
#pragma unroll
                                    for (int x = 0; x < 4; ++x) {
                                        const uint4 q = *reinterpret_cast<const uint4*>(v + ((((c0 % 64) / 8 + x) ^ (k & 7)) << 4));
                                        const uint32_t words[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                                        for (int y = 0; y < 4; ++y) {
                                            float& e0 = reinterpret_cast<float&>(o[8 * x + 2 * y]);
                                            float& e1 = reinterpret_cast<float&>(o[8 * x + 2 * y + 1]);
                                            e0 = seen ? fmaf(w, __uint_as_float(words[y] << 16), e0) : e0;
                                            e1 = seen ? fmaf(w, __uint_as_float(words[y] & 0xffff0000u), e1) : e1;
                                        }
                                    }
                                }
                                tmem_st_32x32(o_at + c0, o);
                            }
                            tmem_st_wait();
                        }
                    }
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full + 16 * t + 8 * (j & 1));
                }
                if (!ok) break;
                if (LONG && upto < hi_t) {
                    ok = sums_of(upto - 1);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const bool more = from > u->lo[t];             // (asked again: kept in a register, it slows the steps down by 2.5 %)
                    const float then = more && far[D] != -INFINITY ? exp2a(far[D] - top) : 0.0f;
                    fold<D>(o_at, far, more, then, false);
                    far[D + 1] = total + (more ? far[D + 1] * then : 0.0f);
                    far[D] = top;
                    total = 0.0f;
                }
            } while (LONG && upto < hi_t);
            if (!ok) break;
            if (u->row[t] >= u->lq) {                     // the whole tile
                idle = u->end - u->begin;
                continue;
            }
            idle = 0;
            const bool any = hi_t > lo_t;
            if (any) {
                ok = sums_of(hi_t - 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after_sync();
            }
            if (LONG && from > u->lo[t]) {
                const float then = far[D] != -INFINITY ? exp2a(far[D] - top) : 0.0f;
                total += far[D + 1] * then;
                fold<D>(o_at, far, true, then, true);
            }
            const float by = total == 0.0f ? 0.0f : 1.0f / total;
            // 32 channels at once go through shared memory, so that four lanes write 64 bytes of a row (a row a lane, 16 bytes at once, took
            // 3500 cycles of 64 channels' unit).  Pieces are rotated by row / 2, so that neither way meets bank conflicts.
            uint8_t* stage = smem + 2 * P::kTileBytes + 2 * ST * P::kStageBytes + (warp - 4) * P::kOut;
            const int rows = min(32, u->lq - u->row[t] - quarter * 32), piece = lane & 3;
            __nv_bfloat16* to = a.y + (long long)(u->q0 + u->row[t] + quarter * 32) * a.ldy + u->head[t] * D + 8 * piece;
#pragma unroll 1
            for (int c0 = 0; c0 < D; c0 += 32) {
                uint32_t o[32];
                if (any) {
                    tmem_ld_32x32(o_at + c0, o);
                    tmem_ld_wait();
                    tmem_arrived(o);
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    uint32_t w[4];
#pragma unroll
                    for (int y = 0; y < 4; ++y) w[y] = by == 0.0f ? 0u : bf16x2(__uint_as_float(o[8 * x + 2 * y]) * by, __uint_as_float(o[8 * x + 2 * y + 1]) * by);
                    *reinterpret_cast<uint4*>(stage + lane * 64 + ((x + (lane >> 1)) & 3) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                }
                __syncwarp();
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int r = 8 * x + (lane >> 2);
                    const uint4 v = *reinterpret_cast<const uint4*>(stage + r * 64 + ((piece + (r >> 1)) & 3) * 16);
                    if (r < rows) *reinterpret_cast<uint4*>(to + (long long)r * a.ldy + c0) = v;
                }
                __syncwarp();
            }
            tc_fence_before_sync();                                // the next unit's first PV comes after this warp's next p_full
        }
    }

    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Heads of bf16 values as a 3-D tensor (values, heads, tokens), a token `pitch` elements after the other: boxes of 64 values of one head
// x box_tokens tokens in the 128-byte swizzle.
int encode_heads(CUtensorMap* map, const void* base, int64_t dim, int64_t heads, int64_t tokens, int64_t pitch, int box_tokens) {
    const EncodeFn fn = reinterpret_cast<EncodeFn>(tensor_map_encoder());
    if (!fn) return NQ_ERR_CUDA;
    const cuuint64_t dims[3] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)(tokens > 0 ? tokens : 1)}, strides[2] = {(cuuint64_t)dim * 2, (cuuint64_t)pitch * 2};
    const cuuint32_t box[3] = {64, 1, (cuuint32_t)box_tokens}, each[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? NQ_OK : NQ_ERR_CUDA;
}

template <int D>
int launch_prompt(const nq_prompt_desc* d, const void* Q, const void* K, const void* V, const PromptArgs& a, int64_t most, cudaStream_t s) {
    CUtensorMap tmQ, tmK, tmV;
    int st = encode_heads(&tmQ, Q, D, d->q_heads, d->rows_q, d->ldq, kTile);
    // (no keys at all: nothing is loaded, but a map needs an address)
    if (st == NQ_OK) st = encode_heads(&tmK, d->rows_k > 0 ? K : Q, D, d->kv_heads, d->rows_k, d->rows_k > 0 ? d->ldk : d->kv_heads * (int64_t)D, kKeys);
    if (st == NQ_OK) st = encode_heads(&tmV, d->rows_k > 0 ? V : Q, D, d->kv_heads, d->rows_k, d->rows_k > 0 ? d->ldv : d->kv_heads * (int64_t)D, kKeys);
    if (st != NQ_OK) return st;
    // No sequence has more keys than there are rows of them: up to one part there is nothing to fold (64 images of heads of 64 41.2 us, with the code
    // for it 42.2; 64 queries of 32 heads of 128 behind 131072 keys 1671 us, without it 1655).
    const auto kernel = d->rows_k > kFold * kKeys ? prompt_kernel<D, true> : prompt_kernel<D, false>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<D>::kSmem) != cudaSuccess) {
        (void)cudaGetLastError();
        return NQ_ERR_CUDA;
    }
    return launch_chained(kernel, (unsigned)most, kThreads, Shape<D>::kSmem, 1, s, tmQ, tmK, tmV, a);
}

}  // namespace
}  // namespace nq

extern "C" int nq_prompt_attention(const nq_prompt_desc* d, const void* Q, const void* K, const void* V, const int32_t* starts_q, const int32_t* starts_k,
                                   void* Y, void* stream) {
    if (!d || d->seqs < 0 || d->rows_q < 0 || d->rows_k < 0 || d->q_heads <= 0 || d->kv_heads <= 0 || d->q_heads % d->kv_heads || d->window < 0) return NQ_ERR_INVALID_ARG;
    if (!(d->scale > 0.0f) || !(d->scale - d->scale == 0.0f)) return NQ_ERR_INVALID_ARG;
    if (d->head_dim != 64 && d->head_dim != 128) return NQ_ERR_UNSUPPORTED;
    const int64_t most_rows = 0x7fffffffll - 4096;
    if (d->rows_q > most_rows || d->rows_k > most_rows || d->seqs >= 1 << 30 || d->q_heads > 65536) return NQ_ERR_UNSUPPORTED;
    if (d->seqs == 0 || d->rows_q == 0) return NQ_OK;
    const int64_t wide = (int64_t)d->q_heads * d->head_dim, narrow = (int64_t)d->kv_heads * d->head_dim;
    if (!Q || !Y || (d->rows_k > 0 && (!K || !V)) || !starts_q || !starts_k) return NQ_ERR_INVALID_ARG;
    if (d->ldq < wide || d->ldy < wide || (d->rows_k > 0 && (d->ldk < narrow || d->ldv < narrow))) return NQ_ERR_INVALID_ARG;
    const auto off = [](const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; };
    if (off(Q, 16) || off(Y, 16) || (d->ldq & 7) || (d->ldy & 7) || off(starts_q, 4) || off(starts_k, 4)) return NQ_ERR_ALIGNMENT;
    if (d->rows_k > 0 && (off(K, 16) || off(V, 16) || (d->ldk & 7) || (d->ldv & 7))) return NQ_ERR_ALIGNMENT;
    // Heads that share keys go in pairs where there is an even number of them: both tiles of a unit then see the same keys, and short
    // prompts fill both (the five packed ones: 144 us with 256 rows of a head).
    const bool paired = d->q_heads / d->kv_heads % 2 == 0;
    const int64_t heads = paired ? d->q_heads / 2 : d->q_heads;
    const int64_t most = (d->rows_q / (paired ? 128 : 256) + (d->seqs < d->rows_q ? d->seqs : d->rows_q)) * heads;      // units
    if (most > 0x7fff0000ll || d->ldq >= 1ll << 38 || d->ldk >= 1ll << 38 || d->ldv >= 1ll << 38) return NQ_ERR_UNSUPPORTED;
    nq::PromptArgs a = {};
    a.starts_q = starts_q; a.starts_k = starts_k; a.seqs = (int)d->seqs; a.rows_q = (int)d->rows_q; a.rows_k = (int)d->rows_k;
    a.heads = (int)heads; a.per_unit = paired ? 2 : 1; a.span = paired ? 128 : 256; a.next_row = paired ? 0 : 128; a.group = d->q_heads / d->kv_heads; a.causal = d->causal != 0; a.window = d->window;
    a.scale2 = d->scale * 1.44269504088896341f;
    a.y = static_cast<__nv_bfloat16*>(Y); a.ldy = d->ldy;
    a.status = nq::status_word();
    if (!a.status) return NQ_ERR_CUDA;
    const cudaStream_t s = (cudaStream_t)stream;
    return d->head_dim == 64 ? nq::launch_prompt<64>(d, Q, K, V, a, most, s) : nq::launch_prompt<128>(d, Q, K, V, a, most, s);
}
