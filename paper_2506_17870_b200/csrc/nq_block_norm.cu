// Block norm: post-norm, gate, residual sum and pre-norm of a transformer block in one pass, and its backward pass.
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
    int ring, stage_bytes;                 // RING: stages and their size
    unsigned int* status;
};

// Centres v for a layer norm and returns 1 / sqrt(mean of squares + eps); 1 for no norm.  The variance is that of the
// centred values, from registers: no cancellation however large the mean.
template <int NV, bool VEC, typename Sum>
__device__ __forceinline__ float norm_factor(const Cols<NV, VEC>& c, Row<NV>& v, int kind, float inv_cols, float eps, Sum& sum) {
    if (kind == NQ_NORM_NONE) return 1.0f;
    if (kind == NQ_NORM_LAYER) {
        float m[1] = {total<NV>(v)};
        sum(m);
        shift_row(c, v, -m[0] * inv_cols);
    }
    float q[1] = {dot<NV>(v, v)};
    sum(q);
    return rsqrtf(fmaf(q[0], inv_cols, eps));
}

// A team of threads (a warp, or as many warps as a row needs) walks its share of the rows, neighbours one after the other,
// with the row in registers throughout: each tensor is touched once, so the pass should be bound by memory.  What it
// competes with is the instruction issue -- at HBM speed an SM has 38 issue slots for 32 columns of bf16 in, bf16 and e4m3
// out -- and the latency of a row's two to four joins.  So arithmetic is on pairs, and where blocks work through many
// rows (RING) they come through a ring in shared memory; the parameters stay in registers, the post norm's weight, the gate
// and the branch scale as one factor that changes only with the gate's row.  Otherwise rows are loaded when their turn
// comes.  16384 x 8192, bf16 to e4m3: 475 us without all that, 398 with a ring, 229 with all (4.1 TB/s).  Tried: parameters in
// shared memory and several teams of 16 columns a thread in a block: no room for rows enough (514 us).
// BIAS: one of the norms has a bias.
template <typename TX, typename TY, int NV, bool VEC, bool RING, bool BIAS>
__global__ void __launch_bounds__(NV == 1 ? 1024 : 512) block_norm_kernel(const NormArgs p, int threads) {
    constexpr bool HOLD = NV <= 2;
    __shared__ float box[2][32][1];
    extern __shared__ __align__(16) uint8_t ring_smem[];
    // several teams in a block only without RING, each a warp
    const int team = RING ? 0 : threadIdx.x / threads, teams = RING ? 1 : blockDim.x / threads;
    const Cols<NV, VEC> c{(int)threadIdx.x - team * threads, threads, p.cols};
    TeamSum<1> sum{box, threads, 0};
    RowRing ring;
    const int x_bytes = p.cols * (int)sizeof(TX), y_bytes = p.cols * (int)sizeof(TY), at_y = row_slot(x_bytes, VEC);
    const auto start = [&](int s, long long row) {             // one thread
        const TX* x = static_cast<const TX*>(p.x) + row * p.ldx;
        const TY* y = static_cast<const TY*>(p.y) + row * p.ldy;
        ring.expect(s, RowRing::granules(x, x_bytes) + (p.y ? RowRing::granules(y, y_bytes) : 0));
        ring.copy(s, 0, x, x_bytes);
        if (p.y) ring.copy(s, at_y, y, y_bytes);
    };
    if (RING) {
        ring.init(ring_smem, p.ring, p.stage_bytes, p.status);
        __syncthreads();
    }
    start_next();
    wait_previous();
    const long long share = (long long)blockIdx.x * teams + team, shares = (long long)gridDim.x * teams;
    const long long row0 = p.rows * share / shares, row1 = p.rows * (share + 1) / shares;
    if (RING && ring.first)
        for (int s = 0; s < p.ring && row0 + s < row1; ++s) start(s, row0 + s);

    // u enters r as fma(u, factor * inv, offset), h is fma(r^, weight, shift)
    Row<HOLD ? NV : 1> factor, offset, weight, shift;
    const auto load_post = [&](const float* gate, int k, uint64_t (&f)[4], uint64_t (&o)[4]) {
        uint64_t g[4];
        load_param(c, p.post_weight, 1.0f, k, f);
        load_param(c, gate, 1.0f, k, g);
        if (BIAS) load_param(c, p.post_bias, 0.0f, k, o);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            g[j] = mul2(g[j], both(p.branch));
            f[j] = mul2(f[j], g[j]);
            if (BIAS) o[j] = mul2(o[j], g[j]);
        }
    };
    const auto load_pre = [&](int k, uint64_t (&w)[4], uint64_t (&b)[4]) {
        load_param(c, p.pre_weight, 1.0f, k, w);
        if (BIAS) load_param(c, p.pre_bias, 0.0f, k, b);
    };
    if (HOLD && p.pre != NQ_NORM_NONE) {
#pragma unroll
        for (int k = 0; k < NV; ++k) load_pre(k, weight[HOLD ? k : 0], shift[HOLD ? k : 0]);
    }
    long long gate_until = row0;                               // first row that needs another gate row
    const float* gate = p.gate;
    int stage = 0, parity = 0;
    for (long long row = row0; row < row1; ++row) {
        if (p.y && row == gate_until) {
            gate_until = row1;
            if (p.gate && p.rows_per_gate) {
                const long long g = row / p.rows_per_gate;
                gate = p.gate + g * p.cols;
                gate_until = (g + 1) * p.rows_per_gate;
            }
            if (HOLD) {
#pragma unroll
                for (int k = 0; k < NV; ++k) load_post(gate, k, factor[HOLD ? k : 0], offset[HOLD ? k : 0]);
            }
        }
        const auto refill = [&]() {                            // after a barrier: every thread has taken its part
            if (RING && ring.first && row + p.ring < row1) start(stage, row + p.ring);
        };
        Row<NV> r;
        if constexpr (RING) {
            ring.wait(stage, parity);
            take_row(c, reinterpret_cast<const TX*>(ring.stage(stage) + (VEC ? 0 : RowRing::shift(static_cast<const TX*>(p.x) + row * p.ldx))), r);
        } else {
            load_row(c, static_cast<const TX*>(p.x) + row * p.ldx, r);
        }
        if (p.y) {
            Row<NV> u;
            if constexpr (RING)
                take_row(c, reinterpret_cast<const TY*>(ring.stage(stage) + at_y + (VEC ? 0 : RowRing::shift(static_cast<const TY*>(p.y) + row * p.ldy))), u);
            else load_row(c, static_cast<const TY*>(p.y) + row * p.ldy, u);
            const float inv = norm_factor(c, u, p.post, p.inv_cols, p.eps, sum);
            if (p.post != NQ_NORM_NONE) refill();
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                uint64_t f[4], o[4];
                if (!HOLD) load_post(gate, k, f, o);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint64_t fj = HOLD ? factor[HOLD ? k : 0][j] : f[j];
                    r[k][j] = BIAS ? fma2(r[k][j], both(p.skip), HOLD ? offset[HOLD ? k : 0][j] : o[j]) : mul2(r[k][j], both(p.skip));
                    r[k][j] = fma2(u[k][j], mul2(fj, both(inv)), r[k][j]);
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) r[k][j] = mul2(r[k][j], both(p.skip));
        }
        if (p.r) {
#pragma unroll
            for (int k = 0; k < NV; ++k) store_piece(c, static_cast<TX*>(p.r) + row * p.ldr, k, r[k]);
        }
        const float inv = norm_factor(c, r, p.pre, p.inv_cols, p.eps, sum);
        if (RING) {
            if (p.post == NQ_NORM_NONE) {
                if (p.pre == NQ_NORM_NONE) __syncthreads();
                refill();
            }
            if (++stage == p.ring) { stage = 0; parity ^= 1; }
        }
        if (p.pre == NQ_NORM_NONE) continue;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            uint64_t w[4], b[4], h[4];
            if (!HOLD) load_pre(k, w, b);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint64_t t = mul2(r[k][j], both(inv)), wj = HOLD ? weight[HOLD ? k : 0][j] : w[j];
                h[j] = BIAS ? fma2(t, wj, HOLD ? shift[HOLD ? k : 0][j] : b[j]) : mul2(t, wj);
            }
            if (p.h_dtype == NQ_BF16) {
                store_piece(c, static_cast<bf16*>(p.h) + row * p.ldh, k, h);
            } else if (p.h_dtype == NQ_F32) {
                store_piece(c, static_cast<float*>(p.h) + row * p.ldh, k, h);
            } else {
                float e[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) unpack2(h[j], e[2 * j], e[2 * j + 1]);
                if (p.h_dtype == NQ_I8) {
                    uint32_t q[2] = {0u, 0u};
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int i = max(-128, min(127, __float2int_rn(__fmul_rn(e[j], p.inv_h_scale))));
                        q[j / 4] |= (uint32_t)(i & 255) << (8 * (j & 3));
                    }
                    store_bytes8(c, static_cast<uint8_t*>(p.h) + row * p.ldh, k, q[0], q[1]);
                } else {
                    // groups of 128 columns: 16 lanes of 8 neighbours each, or all lanes of four elements each
                    float m[2], s[2], i[2];
                    m[0] = max_abs(max_abs(e[0], e[1], e[2]), e[3]);
                    m[1] = max_abs(max_abs(e[4], e[5], e[6]), e[7]);
                    if (VEC) {
                        m[0] = max_abs(m[0], m[1]);
#pragma unroll
                        for (int d = 8; d > 0; d >>= 1) m[0] = max_abs(m[0], __shfl_xor_sync(0xffffffffu, m[0], d));
                        group_scale(__float_as_uint(m[0]), s[0], i[0]);
                        s[1] = s[0]; i[1] = i[0];
                    } else {
#pragma unroll
                        for (int n = 0; n < 2; ++n)
                            group_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(m[n]) & 0x7fffffffu), s[n], i[n]);
                    }
                    if ((c.t & (VEC ? 15 : 31)) == 0) {
#pragma unroll
                        for (int n = 0; n < (VEC ? 1 : 2); ++n)
                            if (c.has(k, 4 * n)) p.hs[(long long)(c.col(k, 4 * n) >> 7) * p.ldhs + row] = s[n];
                    }
                    store_bytes8(c, static_cast<uint8_t*>(p.h) + row * p.ldh, k, e4m3x4(mul2(h[0], both(i[0])), mul2(h[1], both(i[0]))),
                                 e4m3x4(mul2(h[2], both(i[1])), mul2(h[3], both(i[1]))));
                }
            }
        }
    }
    if (RING) ring.leave();
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
    int ring, stage_bytes;
    unsigned int* status;
};

// Row statistics are computed again from r and y.  With v, t the rows r and y (centred for a layer norm), e = w_pre dh,
// f = branch * gate * w_post * g, and means over the row:
//   g  = dr + inv_r * (e - mean(e) - v inv_r * mean(e v) inv_r);   dx = skip * g       (mean(e), mean(f) for a layer norm only)
//   dy = inv_y * (f - mean(f) - t inv_y * mean(f t inv_y))
// Sums over a row are joined across the block together: [r, y, e] if a norm needs means, [v^2, e v, t^2], then [f t, f]
// -- two or three joins a row, not one for each sum.  Tensors are read again from the ring instead of being held.
// Column sums stay in registers: P = sum dh v inv_r, sum dh (for the pre norm's weight and bias) over all rows of the thread
// block, A = sum g t inv_y, sum g over the rows of one work item, which lie under one gate row: from A follow both
// dgate = branch * (w A0 + b A1) and the item's share branch * gate * A of the post norm's weight and bias.
template <typename TX, typename TY, int NV, bool VEC, bool RING, bool BIAS>
__global__ void __launch_bounds__(512) block_norm_backward_kernel(const BackArgs p, int threads) {
    constexpr bool HOLD = NV <= 2;
    __shared__ float box3[2][32][3];
    __shared__ float box2[2][32][2];
    extern __shared__ __align__(16) uint8_t ring_smem[];
    const Cols<NV, VEC> c{(int)threadIdx.x, threads, p.cols};
    TeamSum<3> sum3{box3, threads, 0};
    TeamSum<2> sum2v{box2, threads, 0};
    const long long plane = (long long)gridDim.x * p.cols, mine = (long long)blockIdx.x * p.cols;
    const bool has_pre = p.pre != NQ_NORM_NONE;

    // a stage: r, dh (pre norm), dr, y, as far as they are there
    RowRing ring;
    const int x_bytes = p.cols * (int)sizeof(TX), y_bytes = p.cols * (int)sizeof(TY);
    const int x_slot = row_slot(x_bytes, VEC), y_slot = row_slot(y_bytes, VEC);
    const int at_dh = has_pre ? x_slot : 0, at_dr = at_dh + (has_pre ? y_slot : 0), at_y = at_dr + (p.dr ? x_slot : 0);
    const auto start = [&](int s, long long row) {
        const TX *r = static_cast<const TX*>(p.r) + row * p.ldr, *dr = static_cast<const TX*>(p.dr) + row * p.lddr;
        const TY *dh = static_cast<const TY*>(p.dh) + row * p.lddh, *y = static_cast<const TY*>(p.y) + row * p.ldy;
        ring.expect(s, (has_pre ? RowRing::granules(r, x_bytes) + RowRing::granules(dh, y_bytes) : 0) + (p.dr ? RowRing::granules(dr, x_bytes) : 0) +
                           (p.y ? RowRing::granules(y, y_bytes) : 0));
        if (has_pre) {
            ring.copy(s, 0, r, x_bytes);
            ring.copy(s, at_dh, dh, y_bytes);
        }
        if (p.dr) ring.copy(s, at_dr, dr, x_bytes);
        if (p.y) ring.copy(s, at_y, y, y_bytes);
    };
    if (RING) {
        ring.init(ring_smem, p.ring, p.stage_bytes, p.status);
        __syncthreads();
    }
    start_next();
    wait_previous();

    Row<NV> P0, P1;
    Row<HOLD ? NV : 1> weight, factor;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) P0[k][j] = P1[k][j] = 0ull;
    if (HOLD && has_pre) {
#pragma unroll
        for (int k = 0; k < NV; ++k) load_param(c, p.pre_weight, 1.0f, k, weight[HOLD ? k : 0]);
    }
    bool first = true;
    int stage = 0, parity = 0;

    for (long long item = blockIdx.x; item < p.items; item += gridDim.x) {
        const long long group = item / p.chunks;
        const long long row0 = group * p.group_rows + (item - group * p.chunks) * p.chunk_rows;
        long long row1 = min(row0 + p.chunk_rows, (group + 1) * p.group_rows);
        row1 = min(row1, p.rows);
        const float* gate = p.gate ? p.gate + group * p.cols : nullptr;
        const auto load_factor = [&](int k, uint64_t (&f)[4]) {
            uint64_t g[4];
            load_param(c, p.post_weight, 1.0f, k, f);
            load_param(c, gate, 1.0f, k, g);
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = mul2(f[j], mul2(g[j], both(p.branch)));
        };
        if (HOLD && p.y) {
#pragma unroll
            for (int k = 0; k < NV; ++k) load_factor(k, factor[HOLD ? k : 0]);
        }
        Row<NV> A0, A1;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) A0[k][j] = A1[k][j] = 0ull;
        if (RING && ring.first)                                // the ring is empty between items
            for (int i = 0, s = stage; i < p.ring && row0 + i < row1; ++i, s = s + 1 == p.ring ? 0 : s + 1) start(s, row0 + i);

        for (long long row = row0; row < row1; ++row) {
            const uint8_t* here = RING ? ring.stage(stage) : nullptr;
            const auto get_x = [&](const void* base, long long ld, int offset, Row<NV>& v) {
                if constexpr (RING) take_row(c, reinterpret_cast<const TX*>(here + offset + (VEC ? 0 : RowRing::shift(static_cast<const TX*>(base) + row * ld))), v);
                else load_row(c, static_cast<const TX*>(base) + row * ld, v);
            };
            const auto get_y = [&](const void* base, long long ld, int offset, Row<NV>& v) {
                if constexpr (RING) take_row(c, reinterpret_cast<const TY*>(here + offset + (VEC ? 0 : RowRing::shift(static_cast<const TY*>(base) + row * ld))), v);
                else load_row(c, static_cast<const TY*>(base) + row * ld, v);
            };
            if (RING) ring.wait(stage, parity);
            Row<NV> v, e, t;
            float s[3] = {0.0f, 0.0f, 0.0f};
            if (has_pre) {
                get_x(p.r, p.ldr, 0, v);
                get_y(p.dh, p.lddh, at_dh, e);
            }
            if (p.y) get_y(p.y, p.ldy, at_y, t);
            const auto weigh = [&](int k, int j, uint64_t d) {
                if (HOLD) return mul2(d, weight[HOLD ? k : 0][j]);
                uint64_t w[4];
                load_param(c, p.pre_weight, 1.0f, k, w);
                return mul2(d, w[j]);
            };
            float mean_e = 0.0f;
            if (p.pre == NQ_NORM_LAYER || p.post == NQ_NORM_LAYER) {
                if (has_pre) {
                    uint64_t a = 0ull;
#pragma unroll
                    for (int k = 0; k < NV; ++k)
#pragma unroll
                        for (int j = 0; j < 4; ++j) a = add2(a, weigh(k, j, e[k][j]));
                    s[0] = total<NV>(v);
                    s[1] = sum2(a);
                }
                if (p.y) s[2] = total<NV>(t);
                sum3(s);
                if (p.pre == NQ_NORM_LAYER) {
                    shift_row(c, v, -s[0] * p.inv_cols);
                    mean_e = s[1] * p.inv_cols;
                }
                if (p.post == NQ_NORM_LAYER) shift_row(c, t, -s[2] * p.inv_cols);
            }
            const float y_total = s[2];
            if (has_pre || p.post != NQ_NORM_NONE) {
                s[0] = s[1] = s[2] = 0.0f;
                if (has_pre) {
                    uint64_t a = 0ull;
#pragma unroll
                    for (int k = 0; k < NV; ++k)
#pragma unroll
                        for (int j = 0; j < 4; ++j) a = fma2(v[k][j], weigh(k, j, e[k][j]), a);
                    s[0] = dot<NV>(v, v);
                    s[1] = sum2(a);
                }
                if (p.post != NQ_NORM_NONE) s[2] = dot<NV>(t, t);
                sum3(s);
            }
            const float inv_y = p.post != NQ_NORM_NONE ? rsqrtf(fmaf(s[2], p.inv_cols, p.eps)) : 1.0f;
            Row<NV> g;
            if (p.dr) {
                get_x(p.dr, p.lddr, at_dr, g);
            } else {
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) g[k][j] = 0ull;
            }
            if (has_pre) {
                const float inv = rsqrtf(fmaf(s[0], p.inv_cols, p.eps));
                const uint64_t inv2 = both(inv), back = both(-(s[1] * p.inv_cols * inv) * inv);
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint64_t xh = mul2(v[k][j], inv2);
                        P0[k][j] = fma2(e[k][j], xh, P0[k][j]);
                        if (BIAS) P1[k][j] = add2(P1[k][j], e[k][j]);
                        g[k][j] = fma2(weigh(k, j, e[k][j]), inv2, g[k][j]);
                        g[k][j] = fma2(xh, back, g[k][j]);
                    }
                if (p.pre == NQ_NORM_LAYER) shift_row(c, g, -inv * mean_e);
            }
            if (p.dx) {
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    uint64_t o[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[j] = mul2(g[k][j], both(p.skip));
                    store_piece(c, static_cast<TX*>(p.dx) + row * p.lddx, k, o);
                }
            }
            if (p.y) {
                get_y(p.y, p.ldy, at_y, t);                    // again: cheaper than holding it
                if (p.post == NQ_NORM_LAYER) shift_row(c, t, -y_total * p.inv_cols);
                const uint64_t inv2 = both(inv_y);
                uint64_t ft = 0ull, fs = 0ull;
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    uint64_t f[4];
                    if (!HOLD) load_factor(k, f);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint64_t fj = HOLD ? factor[HOLD ? k : 0][j] : f[j];
                        t[k][j] = mul2(t[k][j], inv2);
                        A0[k][j] = fma2(g[k][j], t[k][j], A0[k][j]);
                        if (BIAS) A1[k][j] = add2(A1[k][j], g[k][j]);
                        g[k][j] = mul2(g[k][j], fj);
                        ft = fma2(g[k][j], t[k][j], ft);
                        fs = add2(fs, g[k][j]);
                    }
                }
                float d[2] = {0.0f, 0.0f};
                if (p.post != NQ_NORM_NONE) {
                    d[0] = sum2(ft);
                    d[1] = p.post == NQ_NORM_LAYER ? sum2(fs) : 0.0f;
                    sum2v(d);
                }
                if (p.dy) {
                    const uint64_t back = both(-(d[0] * p.inv_cols) * inv_y), less = both(-inv_y * (d[1] * p.inv_cols));
#pragma unroll
                    for (int k = 0; k < NV; ++k) {
                        uint64_t o[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            o[j] = fma2(g[k][j], inv2, less);
                            if (p.post != NQ_NORM_NONE) o[j] = fma2(t[k][j], back, o[j]);
                        }
                        store_piece(c, static_cast<TY*>(p.dy) + row * p.lddy, k, o);
                    }
                }
            }
            if (RING) {
                // the last reads of the stage lie before the last join; without a post norm there is none after them
                if (p.post == NQ_NORM_NONE) __syncthreads();
                if (ring.first && row + p.ring < row1) start(stage, row + p.ring);
                if (++stage == p.ring) { stage = 0; parity ^= 1; }
            }
        }
        if (p.y) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                uint64_t w[4], b[4], gt[4];
                load_param(c, p.post_weight, 1.0f, k, w);
                load_param(c, p.post_bias, 0.0f, k, b);
                load_param(c, gate, 1.0f, k, gt);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (!c.has(k, j)) continue;
                    const int col = c.col(k, j);
                    const auto pick = [&](uint64_t v) {
                        float lo, hi;
                        unpack2(v, lo, hi);
                        return j & 1 ? hi : lo;
                    };
                    const float a0 = pick(A0[k][j / 2]), a1 = pick(A1[k][j / 2]);
                    if (p.gate_part) p.gate_part[item * p.cols + col] = p.branch * fmaf(pick(w[j / 2]), a0, pick(b[j / 2]) * a1);
                    if (p.post != NQ_NORM_NONE) {
                        float* at = p.part + 2 * plane + mine + col;
                        const float s = p.branch * pick(gt[j / 2]);
                        at[0] = fmaf(s, a0, first ? 0.0f : at[0]);
                        if (BIAS) at[plane] = fmaf(s, a1, first ? 0.0f : at[plane]);
                    }
                }
            }
            first = false;
        }
    }
    if (has_pre) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c.has(k, j)) {
                    float lo, hi;
                    unpack2(P0[k][j / 2], lo, hi);
                    p.part[mine + c.col(k, j)] = j & 1 ? hi : lo;
                    if (BIAS) {
                        unpack2(P1[k][j / 2], lo, hi);
                        p.part[plane + mine + c.col(k, j)] = j & 1 ? hi : lo;
                    }
                }
    }
    if (RING) ring.leave();
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
constexpr int kJoinCols = 32, kJoinSlices = 16;
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
#pragma unroll 8
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

// Threads of a row: 8 * nv columns each.
struct Shape {
    int threads, nv;
};
Shape shape_of(int64_t cols, int nv) {
    return Shape{(int)((cols + 256 * nv - 1) / (256 * nv)) * 32, nv};
}
// One piece a thread as far as the block goes: more warps hide more of a row's latencies.
Shape wide_shape(int64_t cols, int most_threads) {
    return shape_of(cols, cols <= (int64_t)most_threads * 8 ? 1 : cols <= 512 * 16 ? 2 : 4);
}

// Rows through shared memory: the blocks of an SM, the stages of each and its shared memory.
struct RingPlan {
    int stages, blocks;
    size_t smem;
};
constexpr size_t kRingSmem = 216 * 1024;   // of an SM, for all its blocks
// `fit`: blocks of an SM as far as registers go; fewer where they would leave less than three stages each
bool plan_ring(int fit, int64_t stage_bytes, RingPlan& r) {
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

template <typename TX, typename TY, int NV, bool VEC, bool BIAS>
int launch_norm_ring(NormArgs& a, const Shape& sh, const RingPlan& r, cudaStream_t stream) {
    const auto kernel = block_norm_kernel<TX, TY, NV, VEC, true, BIAS>;
    static bool done[64] = {false};
    if (!allow_smem(kernel, done)) return NQ_ERR_CUDA;
    a.ring = r.stages;
    return launch_chained(kernel, (unsigned)(r.blocks * sm_count()), (unsigned)sh.threads, r.smem, 1, stream, a, sh.threads);
}
template <typename TX, typename TY, int NV, bool BIAS>
int launch_norm_plain(const NormArgs& a, const Shape& sh, bool vec, cudaStream_t stream) {
    const int teams = sh.threads == 32 ? 4 : 1, block = sh.threads * teams;
    long long grid = (a.rows + teams - 1) / teams;
    const long long most = (long long)sm_count() * (2048 / block);
    if (grid > most) grid = most;
    return vec ? launch_chained(block_norm_kernel<TX, TY, NV, true, false, BIAS>, (unsigned)grid, block, 0, 1, stream, a, sh.threads)
               : launch_chained(block_norm_kernel<TX, TY, NV, false, false, BIAS>, (unsigned)grid, block, 0, 1, stream, a, sh.threads);
}
template <typename TX, typename TY, bool BIAS>
int launch_norm_bias(NormArgs& a, bool vec, cudaStream_t stream) {
    const Shape wide = wide_shape(a.cols, 1024);
    // The ring is worth filling from two rows a block on; a warp to a row (up to 256) has enough loads in flight by itself
    // (50000 x 200: 27 us).
    if (wide.threads > 32) {
        a.stage_bytes = row_slot(a.cols * (int)sizeof(TX), vec) + (a.y ? row_slot(a.cols * (int)sizeof(TY), vec) : 0);
        // both instantiations are bound to the registers that fill an SM: 64 at 1024 threads, 128 at 512
        RingPlan r;
        if (plan_ring((wide.nv == 1 ? 1024 : 512) / wide.threads, a.stage_bytes, r) && a.rows >= 2ll * r.blocks * sm_count())
            return wide.nv == 1 ? (vec ? launch_norm_ring<TX, TY, 1, true, BIAS>(a, wide, r, stream) : launch_norm_ring<TX, TY, 1, false, BIAS>(a, wide, r, stream))
                                : (vec ? launch_norm_ring<TX, TY, 4, true, BIAS>(a, wide, r, stream) : launch_norm_ring<TX, TY, 4, false, BIAS>(a, wide, r, stream));
    }
    return wide.nv == 1 ? launch_norm_plain<TX, TY, 1, BIAS>(a, wide, vec, stream) : launch_norm_plain<TX, TY, 4, BIAS>(a, wide, vec, stream);
}
template <typename TX, typename TY>
int launch_norm(NormArgs& a, bool vec, cudaStream_t stream) {
    return a.post_bias || a.pre_bias ? launch_norm_bias<TX, TY, true>(a, vec, stream) : launch_norm_bias<TX, TY, false>(a, vec, stream);
}

// Work items of the backward pass: each gate row's rows in equal chunks, about as many items as blocks are wanted.
struct BackPlan {
    Shape shape;
    RingPlan ring;
    bool use_ring;
    long long group_rows, groups, chunk_rows, items;
    int chunks, blocks, stage_bytes;
};
// The workspace is sized before the pointers are known, so the plan goes by the shape and types alone (stages have room
// for rows that start anywhere).
BackPlan plan_backward(const nq_block_norm_desc* d, bool has_gate) {
    BackPlan p;
    p.group_rows = has_gate && d->rows_per_gate > 0 ? d->rows_per_gate : (d->rows > 0 ? d->rows : 1);
    if (p.group_rows > d->rows && d->rows > 0) p.group_rows = d->rows;
    p.groups = (d->rows + p.group_rows - 1) / p.group_rows;
    p.shape = wide_shape(d->cols, 512);
    const int xs = d->x_dtype == NQ_BF16 ? 2 : 4, ys = d->y_dtype == NQ_BF16 ? 2 : 4;
    p.stage_bytes = 2 * (row_slot((int)d->cols * xs, false) + row_slot((int)d->cols * ys, false));     // at most: r, dr and y, dh
    p.use_ring = p.shape.threads > 32 && plan_ring(512 / p.shape.threads, p.stage_bytes, p.ring) &&
                 d->rows >= 4ll * p.ring.blocks * sm_count();
    const int per_sm = p.use_ring ? p.ring.blocks : 1024 / p.shape.threads;
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

template <typename TX, typename TY, int NV, bool VEC, bool BIAS>
int launch_back_ring(BackArgs& a, const BackPlan& pl, cudaStream_t stream) {
    const auto kernel = block_norm_backward_kernel<TX, TY, NV, VEC, true, BIAS>;
    static bool done[64] = {false};
    if (!allow_smem(kernel, done)) return NQ_ERR_CUDA;
    a.ring = pl.ring.stages;
    const int x = row_slot(a.cols * (int)sizeof(TX), VEC), y = row_slot(a.cols * (int)sizeof(TY), VEC);
    a.stage_bytes = (a.pre != NQ_NORM_NONE ? x + y : 0) + (a.dr ? x : 0) + (a.y ? y : 0);
    return launch_chained(kernel, (unsigned)pl.blocks, (unsigned)pl.shape.threads, pl.ring.smem, 1, stream, a, pl.shape.threads);
}
template <typename TX, typename TY, int NV, bool BIAS>
int launch_back_plain(const BackArgs& a, const BackPlan& pl, bool vec, cudaStream_t stream) {
    return vec ? launch_chained(block_norm_backward_kernel<TX, TY, NV, true, false, BIAS>, (unsigned)pl.blocks, pl.shape.threads, 0, 1, stream, a, pl.shape.threads)
               : launch_chained(block_norm_backward_kernel<TX, TY, NV, false, false, BIAS>, (unsigned)pl.blocks, pl.shape.threads, 0, 1, stream, a, pl.shape.threads);
}
template <typename TX, typename TY, bool BIAS>
int launch_back_bias(BackArgs& a, const BackPlan& pl, bool vec, cudaStream_t stream) {
    if (pl.use_ring) {
        if (pl.shape.nv == 1) return vec ? launch_back_ring<TX, TY, 1, true, BIAS>(a, pl, stream) : launch_back_ring<TX, TY, 1, false, BIAS>(a, pl, stream);
        if (pl.shape.nv == 2) return vec ? launch_back_ring<TX, TY, 2, true, BIAS>(a, pl, stream) : launch_back_ring<TX, TY, 2, false, BIAS>(a, pl, stream);
        return vec ? launch_back_ring<TX, TY, 4, true, BIAS>(a, pl, stream) : launch_back_ring<TX, TY, 4, false, BIAS>(a, pl, stream);
    }
    if (pl.shape.nv == 1) return launch_back_plain<TX, TY, 1, BIAS>(a, pl, vec, stream);
    if (pl.shape.nv == 2) return launch_back_plain<TX, TY, 2, BIAS>(a, pl, vec, stream);
    return launch_back_plain<TX, TY, 4, BIAS>(a, pl, vec, stream);
}
template <typename TX, typename TY>
int launch_back(BackArgs& a, const BackPlan& pl, bool bias, bool vec, cudaStream_t stream) {
    return bias ? launch_back_bias<TX, TY, true>(a, pl, vec, stream) : launch_back_bias<TX, TY, false>(a, pl, vec, stream);
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
    a.ring = 0; a.stage_bytes = 0;
    a.status = status_word();
    if (!a.status) return NQ_ERR_CUDA;
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
    a.ring = 0; a.stage_bytes = 0;
    a.status = status_word();
    if (!a.status) return NQ_ERR_CUDA;
    const bool bias = post_bias || dpost_bias || dpre_bias;    // the sums of g and dh are wanted
    int st;
    if (d->x_dtype == NQ_BF16) st = launch_back<bf16, bf16>(a, pl, bias, vec, s);
    else st = d->y_dtype == NQ_BF16 ? launch_back<float, bf16>(a, pl, bias, vec, s) : launch_back<float, float>(a, pl, bias, vec, s);
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
