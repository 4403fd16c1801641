// Heads of queries, keys and values on their way to attention: norm and position rotation of each head, keys and values into
// the paged cache (quantised as they are written), and a cache's tokens back as dense rows.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/nq.h"
#include "nq_kv_cache.cuh"

namespace nq {
namespace {

constexpr int kThreads = 256;

struct HeadsArgs {
    const void *q, *k, *v;             // sources; a token's heads are dense behind one another
    long long ldq, ldk, ldv;           // pitches of tokens, in elements
    int q_heads, kv_heads;             // heads that are read of q, and of each of k and v
    int q_turns, kv_turns, turns;      // turns of a warp for a token's queries, for its keys, and in all (with the values, where they are wanted)
    long long tokens;
    int parts, per_part;               // warps of a token, and turns of each of them
    int rms, rotary, neighbours;
    float eps;
    const float *q_weight, *k_weight, *angles;
    const int* positions;
    int angle_rows;
    void *q_out, *k_out;
    long long ldqo, ldko;
    Pages c;
    const int* slots;                  // NULL: no cache
};

// 8 neighbouring values of a head
template <typename T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
    uint4 a;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = load16(p); }
    __device__ __forceinline__ void to(uint64_t* f) const {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = pack2(w[i] << 16, w[i] & 0xffff0000u);
    }
};
template <>
struct Eight<float> {
    uint4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = load16(p);
        b = load16(p + 4);
    }
    __device__ __forceinline__ void to(uint64_t* f) const {
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = pack2(w[2 * i], w[2 * i + 1]);
    }
};

__device__ __forceinline__ uint32_t bf16x2(uint64_t v) {
    float lo, hi;
    unpack2(v, lo, hi);
    const __nv_bfloat162 r = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&r);
}
template <typename Y>
__device__ __forceinline__ void store8(Y* p, const uint64_t* f);
template <>
__device__ __forceinline__ void store8(__nv_bfloat16* p, const uint64_t* f) {
    *reinterpret_cast<uint4*>(p) = make_uint4(bf16x2(f[0]), bf16x2(f[1]), bf16x2(f[2]), bf16x2(f[3]));
}
template <>
__device__ __forceinline__ void store8(float* p, const uint64_t* f) {
    reinterpret_cast<ulonglong2*>(p)[0] = make_ulonglong2(f[0], f[1]);
    reinterpret_cast<ulonglong2*>(p)[1] = make_ulonglong2(f[2], f[3]);
}
__device__ __forceinline__ uint32_t i8x4(uint64_t ab, uint64_t cd) {
    float a, b, c, d;
    unpack2(ab, a, b);
    unpack2(cd, c, d);
    return nq::i8x4(a, b, c, d);
}

// A lane holds 16 values of a head, as two chunks of eight that the rotation by halves pairs with each other: chunks p and
// p + rotary / 16 of the rotated part, and of the rest (`free` lanes of it) chunk p + rotary / 16 and the one (D - rotary) / 16 on.
// So a pair of values never leaves its lane, for either order of pairs, and D / 16 lanes are a head.  A token's angles stay in
// registers for all the heads that a warp takes; heads are dealt to 32 / (D / 16) lane groups in turn.
// Four turns (two in fp32) are on their way to a warp at any time.  16384 tokens of 32 + 8 heads of 128 67 us (0.78 of the copy rate), 88 into
// an e4m3 cache; 87 with a head's kind looked up lane by lane, all loads waited for together and scalar products.  Bound by the latency
// of the loads and by issue in about equal parts (16 warps of 128 registers); for few tokens a token is cut into `parts` warps, so that a
// turn or two of loads is all a warp does (3 tokens 3 us).
template <typename T, typename Y, int D, int CACHE, bool PLAIN>
__global__ void __launch_bounds__(kThreads) heads_kernel(const HeadsArgs a) {
    constexpr int kLanes = D / 16, kGroups = 32 / kLanes, kTurns = sizeof(T) == 2 ? 4 : 2;
    const int lane = threadIdx.x & 31, p = lane % kLanes, group = lane / kLanes;
    const long long warp = (long long)blockIdx.x * (kThreads / 32) + __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0);    // (known to be the warp's)
    const long long token = warp / a.parts;
    const int turn0 = (int)(warp - token * a.parts) * a.per_part;
    if (token >= a.tokens) return;
    start_next();
    wait_previous();

    const int r16 = PLAIN ? 0 : a.rotary / 16;
    const bool turned = !PLAIN && p < r16;
    const int c0 = turned ? p : r16 + p, c1 = turned ? p + r16 : p + D / 16;
    // (not rotated: the rest starts at chunk 2 * r16, lane p is its number p - r16, and (D - rotary) / 16 = D / 16 - r16)
    // A turn is one head for each group of lanes, all of one kind: queries, keys or values.
    const int end = min(a.turns, turn0 + a.per_part);
    const auto kind_of = [&](int turn) { return turn < a.q_turns ? 0 : turn < a.q_turns + a.kv_turns ? 1 : 2; };
    const auto head_of = [&](int turn, int kind) { return (turn - (kind == 0 ? 0 : kind == 1 ? a.q_turns : a.q_turns + a.kv_turns)) * kGroups + group; };
    const T* const from[3] = {static_cast<const T*>(a.q) + token * a.ldq, static_cast<const T*>(a.k) + token * a.ldk, static_cast<const T*>(a.v) + token * a.ldv};
    Eight<T> raw[kTurns][2];
    const auto load = [&](Eight<T> (&to)[2], int turn) {
        const int kind = kind_of(turn), h = head_of(turn, kind);
        // (behind the last head: that one again, which nobody stores)
        const T* src = (kind == 0 ? from[0] : kind == 1 ? from[1] : from[2]) + min(h, (kind == 0 ? a.q_heads : a.kv_heads) - 1) * D;
        to[0].load(src + 8 * c0);
        to[1].load(src + 8 * c1);
    };
    const int position = turned ? a.positions[token] : 0, slot = CACHE >= 0 ? a.slots[token] : 0;
#pragma unroll
    for (int u = 0; u < kTurns; ++u)                                 // on their way while the position's angles come
        if (turn0 + u < end) load(raw[u], turn0 + u);
    uint64_t cosine[4], sine[4];                                     // of pairs 2 e, 2 e + 1
    if (turned) {
        const int half = a.rotary / 2;
        const bool inside = position >= 0 && position < a.angle_rows;
        const float* row = a.angles + (long long)(inside ? position : 0) * a.rotary;
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
            const int from = a.neighbours ? 4 * (e == 0 ? c0 : c1) : 8 * p + 2 * e;
            const ulonglong2 c = *reinterpret_cast<const ulonglong2*>(row + from), s = *reinterpret_cast<const ulonglong2*>(row + half + from);
            cosine[e] = c.x; cosine[e + 1] = c.y;
            sine[e] = s.x; sine[e + 1] = s.y;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (!inside) cosine[e] = both(__int_as_float(0x7fffffff));
    }
    long long page = -1;
    int within = 0;
    if (CACHE >= 0 && slot >= 0 && slot / a.c.page_size < a.c.pages) {
        page = slot / a.c.page_size;
        within = slot - (int)page * a.c.page_size;
    }
    uint64_t weight[8];
    int weight_of = -1;                                              // 0 queries, 1 keys

    for (int first = turn0; first < end; first += kTurns) {
#pragma unroll
        for (int u = 0; u < kTurns; ++u) {
            const int turn = first + u;
            if (turn >= end) break;
            const int kind = kind_of(turn), h = head_of(turn, kind);
            const bool live = h < (kind == 0 ? a.q_heads : a.kv_heads);
            uint64_t f[8];
            raw[u][0].to(f);
            raw[u][1].to(f + 4);
            if (turn + kTurns < end) load(raw[u], turn + kTurns);    // kTurns turns are on their way at any time
            if (!PLAIN) {
                if (a.rms && kind < 2) {
                    uint64_t squares = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) squares = fma2(f[e], f[e], squares);
                    float ss = sum2(squares);
#pragma unroll
                    for (int m = 1; m < kLanes; m *= 2) ss += __shfl_xor_sync(0xffffffffu, ss, m);
                    {
                        const float* w = kind == 0 ? a.q_weight : a.k_weight;
                        if (w && weight_of != kind) {
                            weight_of = kind;
#pragma unroll
                            for (int e = 0; e < 8; e += 2) {
                                const ulonglong2 g = *reinterpret_cast<const ulonglong2*>(w + 8 * (e < 4 ? c0 : c1) + 2 * (e & 3));
                                weight[e] = g.x; weight[e + 1] = g.y;
                            }
                        }
                        const uint64_t inv = both(rsqrtf(fmaf(ss, 1.0f / D, a.eps)));
#pragma unroll
                        for (int e = 0; e < 8; ++e) f[e] = w ? mul2(mul2(f[e], inv), weight[e]) : mul2(f[e], inv);
                    }
                }
                if (turned && kind < 2) {
                    if (a.neighbours) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {                // (x, y) (c, c) + (y, x) (-s, s)
                            float x, y, c[2], s[2];
                            unpack2(f[e], x, y);
                            unpack2(cosine[e / 2], c[0], c[1]);
                            unpack2(sine[e / 2], s[0], s[1]);
                            f[e] = pack2f(x * c[e & 1] - y * s[e & 1], y * c[e & 1] + x * s[e & 1]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint64_t x = f[e], y = f[4 + e];
                            f[e] = fma2(x, cosine[e], mul2(y, sine[e]) ^ 0x8000000080000000ull);
                            f[4 + e] = fma2(y, cosine[e], mul2(x, sine[e]));
                        }
                    }
                }
                if (live && kind == 0) {
                    Y* to = static_cast<Y*>(a.q_out) + token * a.ldqo + h * D;
                    store8(to + 8 * c0, f);
                    store8(to + 8 * c1, f + 4);
                }
                if (live && kind == 1 && a.k_out) {
                    Y* to = static_cast<Y*>(a.k_out) + token * a.ldko + h * D;
                    store8(to + 8 * c0, f);
                    store8(to + 8 * c1, f + 4);
                }
            }
            if (CACHE < 0) continue;
            const bool keep = live && kind > 0 && page >= 0;
            const long long at = (page * a.c.kv_heads + h) * a.c.page_size + within;      // row of the cache
            uint8_t* rows = kind == 1 ? a.c.k : a.c.v;
            if (CACHE == NQ_BF16) {
                if (keep) {
                    __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(rows) + at * D;
                    store8(to + 8 * c0, f);
                    store8(to + 8 * c1, f + 4);
                }
            } else {
                float most = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float x, y;
                    unpack2(f[e], x, y);
                    most = max_abs(most, x, y);
                }
                uint32_t top = __float_as_uint(most) & 0x7fffffffu;
#pragma unroll
                for (int m = 1; m < kLanes; m *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, m));
                if (keep) {
                    float s, inv;
                    row_scale(top, CACHE == NQ_E4M3 ? kE4M3Max : 127.0f, s, inv);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = mul2(f[e], both(inv));
                    uint2 lo, hi;
                    if (CACHE == NQ_E4M3) {
                        lo = make_uint2(e4m3x4(f[0], f[1]), e4m3x4(f[2], f[3]));
                        hi = make_uint2(e4m3x4(f[4], f[5]), e4m3x4(f[6], f[7]));
                    } else {
                        lo = make_uint2(i8x4(f[0], f[1]), i8x4(f[2], f[3]));
                        hi = make_uint2(i8x4(f[4], f[5]), i8x4(f[6], f[7]));
                    }
                    *reinterpret_cast<uint2*>(rows + at * D + 8 * c0) = lo;
                    *reinterpret_cast<uint2*>(rows + at * D + 8 * c1) = hi;
                    if (p == 0) (kind == 1 ? a.c.ks : a.c.vs)[at] = s;
                }
            }
        }
    }
}

// How many warps a token's turns are cut into: one where the tokens alone give each SM 16 warps or more, otherwise as many as
// fill that, down to one turn a warp.
void cut(HeadsArgs& a, int dim, bool values) {
    const int groups = 32 / (dim / 16);
    a.q_turns = (a.q_heads + groups - 1) / groups;
    a.kv_turns = (a.kv_heads + groups - 1) / groups;
    const int turns = a.turns = a.q_turns + (values ? 2 : 1) * a.kv_turns;
    const long long want = (16ll * sm_count() + a.tokens - 1) / a.tokens;
    const int parts = (int)(want < turns ? want : turns);
    a.per_part = (turns + parts - 1) / parts;
    a.parts = (turns + a.per_part - 1) / a.per_part;
}

template <typename T, typename Y, int D, int CACHE, bool PLAIN>
int launch_heads(const HeadsArgs& a, cudaStream_t s) {
    const long long blocks = (a.tokens * a.parts * 32 + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffffll) return NQ_ERR_UNSUPPORTED;
    return launch_chained(heads_kernel<T, Y, D, CACHE, PLAIN>, (unsigned)blocks, kThreads, 0, 1, s, a);
}
template <typename T, typename Y, int D, bool PLAIN>
int launch_cache(const HeadsArgs& a, int cache, cudaStream_t s) {
    switch (cache) {
        case NQ_BF16: return launch_heads<T, Y, D, NQ_BF16, PLAIN>(a, s);
        case NQ_E4M3: return launch_heads<T, Y, D, NQ_E4M3, PLAIN>(a, s);
        case NQ_I8: return launch_heads<T, Y, D, NQ_I8, PLAIN>(a, s);
        default: break;
    }
    if constexpr (PLAIN) return NQ_ERR_INVALID_ARG;
    else return launch_heads<T, Y, D, -1, PLAIN>(a, s);
}
template <typename T, typename Y, bool PLAIN>
int launch_dim(const HeadsArgs& a, int dim, int cache, cudaStream_t s) {
    return dim == 64 ? launch_cache<T, Y, 64, PLAIN>(a, cache, s) : launch_cache<T, Y, 128, PLAIN>(a, cache, s);
}

// ------------------------------------------------------------------------------------------------------- reading back
struct ReadArgs {
    Pages c;
    const int *table, *starts;
    long long ld_table;
    int table_cols, seqs;
    long long rows;
    void *k, *v;
    long long ldk, ldv;
    int tokens;                               // rows of a warp,
    int parts, per_part;                      // or warps of a row and turns of each of them
};

// The sequence that a packed row belongs to: the last one that starts at or before it (empty ones share a start with the next);
// -1 where it lies outside all of them.
__device__ __forceinline__ int sequence_of(const int* starts, int seqs, long long row) {
    int lo = 0, hi = seqs;                                    // starts[lo] <= row < starts[hi]
    if (row < starts[0] || row >= starts[seqs]) return -1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= row) lo = mid; else hi = mid;
    }
    return lo;
}

// 16 values of a row, times its scale
template <int CACHE>
__device__ __forceinline__ void dequantise16(const uint4* w, float s, uint64_t* f) {
    if (CACHE == NQ_BF16) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) f[4 * i + j] = pack2(u[j] << 16, u[j] & 0xffff0000u);
        }
        return;
    }
    const uint32_t u[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            float lo, hi;
            if (CACHE == NQ_E4M3) {
                uint32_t h;
                asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)(u[j] >> (16 * b))));
                asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}" : "=f"(lo), "=f"(hi) : "r"(h));
            } else {
                lo = (float)(int8_t)(u[j] >> (16 * b));
                hi = (float)(int8_t)(u[j] >> (16 * b + 8));
            }
            f[2 * j + b] = mul2(pack2f(lo, hi), both(s));
        }
    }
}

// A warp takes `tokens` packed rows one after the other and the heads of each in turn, D / 16 lanes a head: 16 neighbouring values a lane,
// which are 16 bytes of an 8-bit cache and 32 of a bf16 one.  Where a row's sequence and page are, three loads that wait for one another,
// is looked up again only where it changes.  Two rows a warp: 16 e4m3 sequences of up to 8192 tokens 75 us (0.82 of the copy rate), one 85;
// eight 82, for then neighbouring tokens, which lie behind one another in the cache, are read further apart in time.
template <typename Y, int D, int CACHE>
__global__ void __launch_bounds__(kThreads, 3) read_kernel(const ReadArgs a) {
    constexpr int kLanes = D / 16, kGroups = 32 / kLanes, kSize = CACHE == NQ_BF16 ? 2 : 1, kTurns = 4;
    const int lane = threadIdx.x & 31, p = lane % kLanes, group = lane / kLanes;
    const long long warp = ((long long)blockIdx.x * kThreads + threadIdx.x) >> 5;
    const long long first = warp / a.parts * a.tokens, end = min(a.rows, first + a.tokens);
    if (first >= a.rows) return;
    start_next();
    wait_previous();
    const int turn0 = (int)(warp % a.parts) * a.per_part, last = min(2 * a.c.kv_heads, (turn0 + a.per_part) * kGroups);
    long long from = 0, to = 0;                               // rows of the sequence
    int seq = -1, nth = -1, page = -1;
    struct Batch {
        uint4 w[kTurns][kSize];
        float s[kTurns];
        long long row;
        int r0;
    };
    // The next batch of heads: of the same row, or of the next that belongs to a sequence; false: there is none.
    long long row = first - 1;
    int r0 = last;
    const auto load = [&](Batch& b) {
        r0 += kTurns * kGroups;
        if (r0 - group >= last) {
            r0 = turn0 * kGroups + group;
            for (;;) {
                if (++row >= end) return false;
                if (row < to) break;
                seq = sequence_of(a.starts, a.seqs, row);
                nth = -1;
                if (seq < 0) continue;
                from = a.starts[seq];
                to = a.starts[seq + 1];
                break;
            }
        }
        const long long t = row - from;                       // (a start far below 0 leaves no page: all tokens of a table have numbers under 2^31)
        const int of = t > 0x7fffffffll ? 0x7fffffff : (int)t / a.c.page_size, within = t > 0x7fffffffll ? 0 : (int)t - of * a.c.page_size;
        if (of != nth) {
            nth = of;
            page = of < a.table_cols ? a.table[seq * a.ld_table + of] : -1;
        }
        const bool there = page >= 0 && page < a.c.pages;
        b.row = row;
        b.r0 = r0;
#pragma unroll
        for (int u = 0; u < kTurns; ++u) {
            const int r = r0 + u * kGroups, head = r < a.c.kv_heads ? r : r - a.c.kv_heads;
            b.s[u] = 0.0f;
#pragma unroll
            for (int i = 0; i < kSize; ++i) b.w[u][i] = make_uint4(0, 0, 0, 0);
            if (r >= last || !there) continue;
            const long long at = ((long long)page * a.c.kv_heads + head) * a.c.page_size + within;
            const uint8_t* src = (r < a.c.kv_heads ? a.c.k : a.c.v) + (at * D + 16 * p) * kSize;
#pragma unroll
            for (int i = 0; i < kSize; ++i) b.w[u][i] = load16(src + 16 * i);
            if (CACHE != NQ_BF16) b.s[u] = (r < a.c.kv_heads ? a.c.ks : a.c.vs)[at];
        }
        return true;
    };
    const auto store = [&](const Batch& b) {
#pragma unroll
        for (int u = 0; u < kTurns; ++u) {
            const int r = b.r0 + u * kGroups;
            if (r >= last) continue;
            uint64_t f[8];
            dequantise16<CACHE>(b.w[u], b.s[u], f);
            Y* out = (r < a.c.kv_heads ? static_cast<Y*>(a.k) + b.row * a.ldk + r * D : static_cast<Y*>(a.v) + b.row * a.ldv + (r - a.c.kv_heads) * D) + 16 * p;
            store8(out, f);
            store8(out + 8, f + 4);
        }
    };
    Batch b;                                                  // (two in turn, one on its way while the other is written, leave room for fewer warps: 89 us)
    while (load(b)) store(b);
}

template <typename Y, int D>
int launch_read(const ReadArgs& a, int cache, cudaStream_t s) {
    const long long blocks = ((a.rows + a.tokens - 1) / a.tokens * a.parts * 32 + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffffll) return NQ_ERR_UNSUPPORTED;
    switch (cache) {
        case NQ_BF16: return launch_chained(read_kernel<Y, D, NQ_BF16>, (unsigned)blocks, kThreads, 0, 1, s, a);
        case NQ_E4M3: return launch_chained(read_kernel<Y, D, NQ_E4M3>, (unsigned)blocks, kThreads, 0, 1, s, a);
        default: return launch_chained(read_kernel<Y, D, NQ_I8>, (unsigned)blocks, kThreads, 0, 1, s, a);
    }
}

}  // namespace
}  // namespace nq

extern "C" int nq_qk_norm_rotate(const nq_qk_desc* d, const void* X, const float* q_weight, const float* k_weight, const float* angles,
                                 const int32_t* positions, void* Q, void* K, const nq_kv_pages* cache, const int32_t* slots, void* stream) {
    using nq::misaligned;
    if (!d || d->tokens < 0 || d->q_heads < 0 || d->kv_heads < 0 || d->angle_rows < 0 || d->rotary_dim < 0 || !(d->eps >= 0.0f)) return NQ_ERR_INVALID_ARG;
    if ((d->x_dtype != NQ_F32 && d->x_dtype != NQ_BF16) || (d->y_dtype != NQ_F32 && d->y_dtype != NQ_BF16)) return NQ_ERR_INVALID_ARG;
    if (d->norm != NQ_NORM_NONE && d->norm != NQ_NORM_RMS) return NQ_ERR_INVALID_ARG;
    if (d->norm == NQ_NORM_NONE && (q_weight || k_weight)) return NQ_ERR_INVALID_ARG;
    if ((cache == nullptr) != (slots == nullptr) && d->tokens > 0) return NQ_ERR_INVALID_ARG;
    if (d->head_dim != 64 && d->head_dim != 128) return NQ_ERR_UNSUPPORTED;
    if ((d->rotary_dim & 15) || d->rotary_dim > d->head_dim || d->q_heads > 65536 || d->kv_heads > 65536) return NQ_ERR_UNSUPPORTED;
    if (cache) {
        const int bad = nq::check_pages(cache);
        if (bad != NQ_OK) return bad;
        if (cache->kv_heads != d->kv_heads || cache->head_dim != d->head_dim) return NQ_ERR_INVALID_ARG;
    }
    if (d->tokens >= 1ll << 40 || d->angle_rows >= 1ll << 31) return NQ_ERR_UNSUPPORTED;
    if (d->tokens == 0 || d->q_heads + d->kv_heads == 0) return NQ_OK;
    const int64_t dim = d->head_dim;
    if (!X || (d->q_heads > 0 && !Q) || (d->kv_heads > 0 && !K && !cache)) return NQ_ERR_INVALID_ARG;
    if (d->ldx < (d->q_heads + (cache ? 2 : 1) * d->kv_heads) * dim || (Q && d->ldq < d->q_heads * dim) || (K && d->ldk < d->kv_heads * dim)) return NQ_ERR_INVALID_ARG;
    if (d->rotary_dim > 0 && (!positions || !angles || d->angle_rows == 0)) return NQ_ERR_INVALID_ARG;
    if (misaligned(X, 16) || misaligned(Q, 16) || misaligned(K, 16) || misaligned(q_weight, 16) || misaligned(k_weight, 16) || misaligned(angles, 16)) return NQ_ERR_ALIGNMENT;
    if (misaligned(positions, 4) || misaligned(slots, 4)) return NQ_ERR_ALIGNMENT;
    const int xsize = d->x_dtype == NQ_BF16 ? 2 : 4, ysize = d->y_dtype == NQ_BF16 ? 2 : 4;
    if ((d->ldx * xsize & 15) || (Q && (d->ldq * ysize & 15)) || (K && (d->ldk * ysize & 15))) return NQ_ERR_ALIGNMENT;
    nq::HeadsArgs a = {};
    const uint8_t* x = static_cast<const uint8_t*>(X);
    a.q = x;
    a.k = x + d->q_heads * dim * xsize;
    a.v = x + (d->q_heads + (int64_t)d->kv_heads) * dim * xsize;
    a.ldq = a.ldk = a.ldv = d->ldx;
    a.q_heads = d->q_heads; a.kv_heads = d->kv_heads;
    a.tokens = d->tokens;
    a.rms = d->norm == NQ_NORM_RMS; a.rotary = d->rotary_dim; a.neighbours = d->neighbours != 0; a.eps = d->eps;
    a.q_weight = q_weight; a.k_weight = k_weight; a.angles = angles; a.positions = positions; a.angle_rows = (int)d->angle_rows;
    a.q_out = Q; a.k_out = K; a.ldqo = d->ldq; a.ldko = d->ldk;
    if (cache) a.c = nq::pages_of(cache);
    a.slots = slots;
    nq::cut(a, (int)dim, cache != nullptr);
    const int kind = cache ? cache->dtype : -1;
    const cudaStream_t s = (cudaStream_t)stream;
    using bf16 = __nv_bfloat16;
    if (d->x_dtype == NQ_BF16)
        return d->y_dtype == NQ_BF16 ? nq::launch_dim<bf16, bf16, false>(a, (int)dim, kind, s) : nq::launch_dim<bf16, float, false>(a, (int)dim, kind, s);
    return d->y_dtype == NQ_BF16 ? nq::launch_dim<float, bf16, false>(a, (int)dim, kind, s) : nq::launch_dim<float, float, false>(a, (int)dim, kind, s);
}

extern "C" int nq_kv_cache_write(const nq_kv_pages* cache, const void* K, int64_t ldk, const void* V, int64_t ldv, int x_dtype,
                                 const int32_t* slots, int64_t tokens, void* stream) {
    using nq::misaligned;
    if (tokens < 0 || (x_dtype != NQ_F32 && x_dtype != NQ_BF16)) return NQ_ERR_INVALID_ARG;
    const int bad = nq::check_pages(cache);
    if (bad != NQ_OK) return bad;
    if (tokens >= 1ll << 40) return NQ_ERR_UNSUPPORTED;
    if (tokens == 0) return NQ_OK;
    const int64_t width = (int64_t)cache->kv_heads * cache->head_dim;
    if (!K || !V || !slots || ldk < width || ldv < width) return NQ_ERR_INVALID_ARG;
    const int size = x_dtype == NQ_BF16 ? 2 : 4;
    if (misaligned(K, 16) || misaligned(V, 16) || misaligned(slots, 4) || (ldk * size & 15) || (ldv * size & 15)) return NQ_ERR_ALIGNMENT;
    nq::HeadsArgs a = {};
    a.k = K; a.v = V; a.ldk = ldk; a.ldv = ldv;
    a.kv_heads = cache->kv_heads; a.tokens = tokens;
    a.c = nq::pages_of(cache); a.slots = slots;
    nq::cut(a, cache->head_dim, true);
    const cudaStream_t s = (cudaStream_t)stream;
    return x_dtype == NQ_BF16 ? nq::launch_dim<__nv_bfloat16, __nv_bfloat16, true>(a, cache->head_dim, cache->dtype, s)
                              : nq::launch_dim<float, float, true>(a, cache->head_dim, cache->dtype, s);
}

extern "C" int nq_kv_cache_read(const nq_kv_pages* cache, const int32_t* table, int64_t ld_table, int64_t table_cols, const int32_t* starts,
                                int64_t seqs, void* K, int64_t ldk, void* V, int64_t ldv, int y_dtype, int64_t rows, void* stream) {
    using nq::misaligned;
    if (rows < 0 || seqs < 0 || table_cols < 0 || (y_dtype != NQ_F32 && y_dtype != NQ_BF16)) return NQ_ERR_INVALID_ARG;
    const int bad = nq::check_pages(cache);
    if (bad != NQ_OK) return bad;
    if (rows >= 1ll << 31 || seqs >= 1ll << 30 || table_cols >= 1ll << 31) return NQ_ERR_UNSUPPORTED;
    if (rows == 0 || seqs == 0) return NQ_OK;
    const int64_t width = (int64_t)cache->kv_heads * cache->head_dim;
    if (!K || !V || !starts || (table_cols > 0 && (!table || ld_table < table_cols)) || ldk < width || ldv < width) return NQ_ERR_INVALID_ARG;
    const int size = y_dtype == NQ_BF16 ? 2 : 4;
    if (misaligned(K, 16) || misaligned(V, 16) || misaligned(table, 4) || misaligned(starts, 4) || (ldk * size & 15) || (ldv * size & 15)) return NQ_ERR_ALIGNMENT;
    nq::ReadArgs a = {};
    a.c = nq::pages_of(cache);
    a.table = table; a.starts = starts; a.ld_table = ld_table; a.table_cols = (int)table_cols; a.seqs = (int)seqs;
    a.rows = rows; a.k = K; a.v = V; a.ldk = ldk; a.ldv = ldv;
    const int groups = 32 / (cache->head_dim / 16), turns = (2 * cache->kv_heads + groups - 1) / groups;
    const long long want = (16ll * nq::sm_count() + rows - 1) / rows;
    const int parts = (int)(want < turns ? want : turns);
    a.per_part = (turns + parts - 1) / parts;
    a.parts = (turns + a.per_part - 1) / a.per_part;
    // two rows a warp, as long as each SM gets 64 warps or more
    const long long each = rows / (64ll * nq::sm_count());
    a.tokens = a.parts > 1 || each < 2 ? 1 : 2;
    const cudaStream_t s = (cudaStream_t)stream;
    using bf16 = __nv_bfloat16;
    if (cache->head_dim == 64)
        return y_dtype == NQ_BF16 ? nq::launch_read<bf16, 64>(a, cache->dtype, s) : nq::launch_read<float, 64>(a, cache->dtype, s);
    return y_dtype == NQ_BF16 ? nq::launch_read<bf16, 128>(a, cache->dtype, s) : nq::launch_read<float, 128>(a, cache->dtype, s);
}
