// Block norm: post-norm, gate, residual sum and pre-norm of a transformer block in one pass.
#include "nq_block_norm.cuh"

namespace nq {
namespace {

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
// comes.  16384 x 8192, bf16 to e4m3: 475 us without all that, 398 with a ring, 223 with all (4.2 TB/s).  16384 x 4096, bf16 to
// e4m3 114 us, to INT8 110, to bf16 97, to fp32 124; 12608 x 768, fp32 stream, layer norms, a gate row for 197 rows, to INT8 32.
// Tried: parameters in shared memory and several teams of 16 columns a thread in a block: no room for rows enough (514 us).
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

// ------------------------------------------------------------------------------------------------------------ host
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
    // The ring is worth filling from two rows a block on (us with / without, bf16 to e4m3, in a graph: 768 columns, 740 rows
    // 4.1 / 3.7, 1480 4.7 / 5.0, 2960 -- two rows a block -- 7.2 / 8.8, 5920 12.2 / 15.3; 4096 columns, 148 rows 4.3 / 4.1,
    // 296 4.5 / 5.1, 592 -- two a block -- 6.8 / 9.5, 2368 20.7 / 24.5); a warp to a row (up to 256) has enough loads in flight
    // by itself (50000 x 200: 27 us).
    if (wide.threads > 32) {
        a.stage_bytes = row_slot(a.cols * (int)sizeof(TX), vec) + (a.y ? row_slot(a.cols * (int)sizeof(TY), vec) : 0);
        // both instantiations are bound to the registers that fill an SM: 64 at 1024 threads, 128 at 512
        RingPlan r;
        if (plan_ring((wide.nv == 1 ? 1024 : 512) / wide.threads, a.stage_bytes, r) && a.rows >= 2ll * r.blocks * sm_count())
            return wide.nv == 1 ? (vec ? launch_norm_ring<TX, TY, 1, true, BIAS>(a, wide, r, stream) : launch_norm_ring<TX, TY, 1, false, BIAS>(a, wide, r, stream))
                                : (vec ? launch_norm_ring<TX, TY, 4, true, true>(a, wide, r, stream) : launch_norm_ring<TX, TY, 4, false, true>(a, wide, r, stream));
    }
    return wide.nv == 1 ? launch_norm_plain<TX, TY, 1, BIAS>(a, wide, vec, stream) : launch_norm_plain<TX, TY, 4, true>(a, wide, vec, stream);
}
template <typename TX, typename TY>
int launch_norm(NormArgs& a, bool vec, cudaStream_t stream) {
    return a.post_bias || a.pre_bias ? launch_norm_bias<TX, TY, true>(a, vec, stream) : launch_norm_bias<TX, TY, false>(a, vec, stream);
}

}  // namespace
}  // namespace nq

extern "C" int nq_block_norm(const nq_block_norm_desc* d, const void* X, const void* Y, const float* post_weight, const float* post_bias,
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
