// Backward pass of the block norm.
#include "nq_block_norm.cuh"

namespace nq {
namespace {

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
// Measured: 16384 x 4096 bf16 218 us (3.7 TB/s; 524 with one join for each sum and no ring), 12608 x 768 fp32 stream 74 us,
// 10 of them joining the blocks' sums.  Bound by issue and by the joins: half of the issue slots are used at four warps a
// scheduler, which the accumulators' registers allow.  (Parameters read for each row instead of held: 330 - 380 us.)
// Short groups: 12608 x 768 with a gate row for each row 262 us, for 8 rows 104, for 64 92 (the ring starts anew with each item,
// and an item's share of the post norm's sums goes to memory).
// Wide rows do not fit the registers, of which a thread has 128: at 2 pieces a thread (4097 to 8192 columns) a frame of 112 - 320
// bytes is spilled, at 4 pieces, whose four accumulators alone take 128, 0.7 KB (rows that start anywhere: 1.4).  bf16, RMS /
// layer norm: 16384 x 5000 401 / 657 us (150 at HBM rate), 16384 x 8192 474 / 759 (246), 8192 x 16384 1495 / 1718 (246).
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
// The ring from four rows a block on, and four rows an item at least, measured in a graph with one gate row (us):
//   768 columns, layer norms, fp32 stream
//     with / without the ring: 1024 rows 26.2 / 29.2, 2048 31.7 / 34.4, 2960 (four a block) 43.6 / 38.6, 4096 39.7 / 57.9, 8192 54 / 82
//     items of 1 / 2 / 4 / 8 rows: 64 rows 12.9 / 13.5 / 15.9 / 22.9, 256 19.3 / 17.5 / 20.6 / 29.3, 1024 39.8 / 28.3 / 29.2 / 36.9
//   4096 columns, RMS, bf16
//     with / without the ring: 32 rows 19.8 / 22.6, 296 23.4 / 29.3, 592 (four a block) 25.3 / 30.5, 1184 32.4 / 55.3
//     items of 1 / 2 / 4 / 8 rows: 32 rows 15.7 / 17.5 / 22.5 / 32.1, 128 19.0 / 21.7 / 26.9 / 39.8, 296 33.2 / 23.4 / 29.1 / 41.9
// The ring gains below that too with wide rows, and two rows an item are up to a quarter faster up to some hundred rows: the
// bounds are on the safe side of that, not at the best place for each width.
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
        return vec ? launch_back_ring<TX, TY, 4, true, true>(a, pl, stream) : launch_back_ring<TX, TY, 4, false, true>(a, pl, stream);
    }
    if (pl.shape.nv == 1) return launch_back_plain<TX, TY, 1, BIAS>(a, pl, vec, stream);
    if (pl.shape.nv == 2) return launch_back_plain<TX, TY, 2, BIAS>(a, pl, vec, stream);
    return launch_back_plain<TX, TY, 4, true>(a, pl, vec, stream);
}
template <typename TX, typename TY>
int launch_back(BackArgs& a, const BackPlan& pl, bool bias, bool vec, cudaStream_t stream) {
    return bias ? launch_back_bias<TX, TY, true>(a, pl, vec, stream) : launch_back_bias<TX, TY, false>(a, pl, vec, stream);
}

}  // namespace
}  // namespace nq

extern "C" {

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
