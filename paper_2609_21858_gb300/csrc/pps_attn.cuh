// pps_attn.cuh -- what the attention kernels over paged caches share: the work's line and its shares, tree masks, and the
// joining of partial results.
//
// Key tiles of all (sequence, key head, row block) items, plus AttnPlan::fix per item for its start and end, lie on one line that
// is cut into equal shares, one per CTA, whatever the lengths are; a cut that would leave a few tiles of an item alone moves to
// the item's end.  An item cut between CTAs leaves one partial result (maximum, sum, fp32 O) per CTA, at most two per CTA, and a
// second launch joins them in order: the same call gives the same bits.  Lengths are read on the device; nothing waits for the host.
#pragma once
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pps.h"
#include "pps_internal.h"
#include "pps_tc.cuh"

namespace pps {
namespace {

constexpr int kTileRows = 128, kTileKeys = 128;

// a cut item: nsplit partial results of a block of ntok tokens from tok0 on, in slot 2 cta + 1 and slots 2 (cta + k),
// k = 1 .. nsplit - 1
struct Cut {
    int32_t nsplit, ntok, tok0, vh;
};

struct AttnPlan {
    int group, gs, nsub, tt;  // heads of a key head; those taken at a time, in nsub turns; tokens per tile
    int bt, fix;        // tokens per row block (one tile or two); key tiles that an item's start and end cost
    int cap_rows, page_log2;
    float shift;        // log2 of a factor on all weights
    int64_t cap_keys;   // what a row of the page table holds, at most whole tiles of an int's range
    float sc;           // |scale| log2 e
    uint32_t s_and, s_xor;  // on scores: a negative scale turns their signs, a zero one clears them
    Cut* cuts;          // [gridDim.x]
    float* part_o;      // [2 gridDim.x][cap_rows][DC]
    float2* part_ml;    // [2 gridDim.x][cap_rows] (maximum, sum)
};

struct Seq {
    int off, n, len;  // first token, tokens, keys
};

__device__ __forceinline__ Seq load_seq(const AttnArgs& a, const AttnPlan& P, int s, bool flag) {
    Seq q;
    q.off = __ldg(a.q_off + s);
    const int end = __ldg(a.q_off + s + 1), len = __ldg(a.kv_len + s);
    q.n = end - q.off;
    q.len = (int)min((int64_t)max(len, 0), P.cap_keys);
    const bool bad = q.off < 0 || end < q.off || end > a.n_tok;
    if (bad) q.n = 0;
    if (flag && a.status && (bad || q.len != len)) atomicOr(a.status, PPS_FLAG_INDEX);
    return q;
}

// key tiles of row block `blk`: those its last token sees
__device__ __forceinline__ int block_tiles(const AttnArgs& a, const AttnPlan& P, const Seq& q, int blk) {
    int vis = q.len;
    const int i0 = blk * P.bt;
    if (a.mask == nullptr) vis = max(0, q.len - q.n + i0 + min(q.n - i0, P.bt));
    return (vis + kTileKeys - 1) / kTileKeys;
}
__device__ __forceinline__ int n_blocks(const AttnPlan& P, const Seq& q) {
    return (int)(((uint32_t)q.n + (uint32_t)P.bt - 1u) / (uint32_t)P.bt);
}
__device__ __forceinline__ int64_t head_cost(const AttnArgs& a, const AttnPlan& P, const Seq& q) {
    const int nb = n_blocks(P, q);
    if (nb == 1 || a.mask != nullptr) return (int64_t)nb * (block_tiles(a, P, q, 0) + P.fix);
    int64_t c = 0;
#pragma unroll 1
    for (int b = 0; b < nb; ++b) c += block_tiles(a, P, q, b) + P.fix;
    return c;
}
__device__ __forceinline__ int64_t divide(int64_t x, int64_t y) {  // of non-negative numbers, most of them small
    return (x | y) >> 32 ? x / y : (int64_t)((uint32_t)x / (uint32_t)y);
}

// key tiles of a block of T before the cut that the line makes after x of them: pieces have `least` tiles or more
__device__ __forceinline__ int cut_at(int64_t x, int T, int least) {
    return x < least ? 0 : x > T - least ? T : (int)x;
}

// where a share starts
struct Start {
    int64_t base;  // the block's start on the line
    int s, vh, blk;
    Seq q;
};

// A CTA's items in order; every warp walks them by itself.
struct Walk {
    int64_t x, x1, base;  // where the walk is, the share's end, the next block's start
    int least;            // key tiles of a cut item's piece
    int s, vh, blk, nb;   // the next block: sequence, turn of a key head (key head x nsub + turn), number; blocks of the sequence
    Seq q;
    // the segment: key tiles t0 .. t1 - 1 of T of a block that starts at `from` on the line, with tokens i0 .. i0 + ntok - 1
    int64_t from;
    int t0, t1, T, i0, ntok;
    int heads;  // the segment's vh

    __device__ __forceinline__ Walk(const AttnPlan& P, const Start& st, int64_t c0, int64_t c1, int least_)
        : x(c0), x1(c1), base(st.base), least(least_), s(st.s), vh(st.vh), blk(st.blk), nb(n_blocks(P, st.q)), q(st.q) {}
    __device__ __forceinline__ bool next(const AttnArgs& a, const AttnPlan& P) {
        while (x < x1) {
            while (blk >= nb) {  // the next turn of heads, or the next sequence with tokens
                blk = 0;
                if (nb == 0 || ++vh == a.c.n_kv_heads * P.nsub) {
                    vh = 0;
                    if (++s >= a.n_seq) return false;
                    q = load_seq(a, P, s, false);
                    nb = n_blocks(P, q);
                }
            }
            T = block_tiles(a, P, q, blk);
            i0 = blk * P.bt;
            ntok = min(q.n - i0, P.bt);
            t0 = cut_at(x - base, T, least);
            t1 = cut_at(x1 - base, T, least);
            const bool none = T == 0 && x == base;
            from = base;
            heads = vh;
            base += T + P.fix;
            x = base;
            ++blk;
            if (t0 < t1 || none) return true;
        }
        return false;
    }
};

// The CTA's share [c0, c1) of the line of costs, and where on it the share starts (s_start, where the share is not empty; the
// caller synchronises the CTA before it is read).  Returns the length of the shares.  s_sum: a number per warp.
template <int THREADS>
__device__ __forceinline__ int64_t find_share(const AttnArgs& a, const AttnPlan& P, int64_t* s_sum, Start* s_start, int64_t& c0,
                                              int64_t& c1) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    Seq own = {0, 0, 0};
    if (tid < a.n_seq) own = load_seq(a, P, tid, cta == 0);
    if (tid == 0) P.cuts[cta].nsplit = 0;
    const int n_vh = a.c.n_kv_heads * P.nsub;
    auto cost = [&](const Seq& q) { return q.n > 0 ? head_cost(a, P, q) * n_vh : (int64_t)0; };
    auto block_scan = [&](int64_t v, int64_t& total) {  // inclusive
        int64_t w = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t t = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += t;
        }
        __syncthreads();
        if (lane == 31) s_sum[warp] = w;
        __syncthreads();
        total = 0;
        for (int i = 0; i < THREADS / 32; ++i) {
            const int64_t t = s_sum[i];
            if (i < warp) w += t;
            total += t;
        }
        return w;
    };
    const int64_t mine = cost(own);
    int64_t more = 0;
    for (int64_t s = tid + THREADS; s < a.n_seq; s += THREADS) more += cost(load_seq(a, P, (int)s, cta == 0));
    int64_t U, U0;
    int64_t at = block_scan(mine, U0);
    U = U0;
    if (a.n_seq > THREADS) {
        block_scan(more, U);
        U += U0;
    }
    const int64_t share = max(divide(U + gridDim.x - 1, gridDim.x), (int64_t)1);
    c0 = min(cta * share, U);
    c1 = min(c0 + share, U);
    if (c0 < c1) {
        int64_t before = 0, v = mine;
        for (int64_t b = 0;; b += THREADS) {
            if (c0 >= before + at - v && c0 < before + at) {  // one thread: its sequence holds the start
                Start st;
                st.s = (int)(b + tid);
                st.q = own;
                const int64_t per = divide(v, n_vh);
                int64_t rem = c0 - (before + at - v);
                st.vh = (int)divide(rem, per);
                rem -= st.vh * per;
                st.blk = 0;
#pragma unroll 1
                for (int c; rem >= (c = block_tiles(a, P, own, st.blk) + P.fix); ++st.blk) rem -= c;
                st.base = c0 - rem;
                *s_start = st;
            }
            before += U0;
            if (before > c0) break;  // CTA-uniform
            own.n = 0;
            if (b + THREADS + tid < a.n_seq) own = load_seq(a, P, (int)(b + THREADS + tid), false);
            v = cost(own);
            at = block_scan(v, U0);
        }
    }
    return share;
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

template <typename T>
struct Half;
template <>
struct Half<__nv_bfloat16> {
    static constexpr uint32_t kType = 1;    // of an operand in the instruction descriptor
    static constexpr float kShift = 0.0f;   // log2 of a factor on all weights
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
};
template <>
struct Half<__half> {
    static constexpr uint32_t kType = 0;
    // weights up to 2^(kLazy + kShift) = 2^14 stay below fp16's largest value, and those down to 2^-20 of the largest
    // are normal numbers
    static constexpr float kShift = 6.0f;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
};

// Of each four lanes, lane q gets the q-th 16-byte unit of every lane: u[k] = unit q of lane k.  A warp that holds a row per
// lane so writes 64 bytes of 8 rows at a time instead of 16 of 32, a quarter of the lines.
__device__ __forceinline__ uint4 shfl4(const uint4& v, int mask) {
    return make_uint4(__shfl_xor_sync(0xffffffffu, v.x, mask), __shfl_xor_sync(0xffffffffu, v.y, mask),
                      __shfl_xor_sync(0xffffffffu, v.z, mask), __shfl_xor_sync(0xffffffffu, v.w, mask));
}
__device__ __forceinline__ uint4 pick(bool first, const uint4& a, const uint4& b) {
    return make_uint4(first ? a.x : b.x, first ? a.y : b.y, first ? a.z : b.z, first ? a.w : b.w);
}
__device__ __forceinline__ void quad_transpose(uint4 (&u)[4], int q) {
    const bool odd = q & 1, high = q & 2;
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
        const uint4 r = shfl4(pick(odd, u[k], u[k + 1]), 1);
        u[k] = pick(odd, r, u[k]);
        u[k + 1] = pick(odd, u[k + 1], r);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint4 r = shfl4(pick(high, u[k], u[k + 2]), 2);
        u[k] = pick(high, r, u[k]);
        u[k + 2] = pick(high, u[k + 2], r);
    }
}

// bits c of a tile's 32 columns from key k0 on that a row sees: those below vis, and of its tree's tokens (from key
// `prefix` on) those of its mask
__device__ __forceinline__ uint32_t seen_bits(int k0, int vis, int prefix, const uint32_t* mask, int words) {
    const int n = vis - k0;
    uint32_t m = n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u;
    if (mask != nullptr) {
        const int rel = k0 - prefix;
        if (rel > -32) {
            const int w = rel >> 5, sh = rel & 31;
            const uint32_t lo = w < 0 ? 0xffffffffu : w < words ? __ldg(mask + w) : 0u;
            const uint32_t hi = w + 1 < words ? __ldg(mask + w + 1) : 0u;
            m &= __funnelshift_r(lo, hi, sh);
        }
    }
    return m;
}

// Joins the partial results of the items that are cut between CTAs.  A row has one warp (its lanes the channels), or up
// to eight that share its parts where there are many (a long sequence's few rows); four parts are read at a time.
template <typename T, int DC>
__global__ void __launch_bounds__(256, 4) join_kernel(const AttnArgs a, const AttnPlan P) {
    using H = Half<T>;
    constexpr int VW = DC / 32;
    __shared__ float s_o[8][DC];
    __shared__ float2 s_x[8];
    pdl_wait();
    const int4 cut = __ldcg(reinterpret_cast<const int4*>(P.cuts + blockIdx.x));
    const int nsplit = cut.x, ntok = cut.y, tok0 = cut.z, vh = cut.w;
    if (nsplit == 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = a.c.head_dim;
    const int wpr = nsplit <= 4 ? 1 : nsplit <= 8 ? 2 : nsplit <= 16 ? 4 : 8, rpb = 8 / wpr;  // warps per row, rows at a time
    const int kvh = vh / P.nsub, sub = vh - kvh * P.nsub, gs = min(P.gs, P.group - sub * P.gs);
    const int64_t first = (int64_t)(2 * blockIdx.x + 1) * P.cap_rows, rest = (int64_t)2 * blockIdx.x * P.cap_rows;
    auto put = [&](int i, float M, float l, const float (&o)[VW]) {
        const float inv = l > 0.0f ? 1.0f / l : l;
        const int t = i / gs, tok = tok0 + t, head = kvh * P.group + sub * P.gs + (i - t * gs);
        if (lane * VW < D) {
            T* out = static_cast<T*>(a.out.p) + (int64_t)tok * a.out.tok + head * a.out.head + lane * VW;
            if constexpr (VW == 4)
                *reinterpret_cast<uint2*>(out) = make_uint2(H::pack(o[0] * inv, o[1] * inv), H::pack(o[2] * inv, o[3] * inv));
            else
                *reinterpret_cast<uint32_t*>(out) = H::pack(o[0] * inv, o[1] * inv);
        }
        if (lane == 0 && a.lse)
            a.lse[(int64_t)tok * a.n_heads + head] = l == 0.0f ? -INFINITY : (M + log2f(l) - P.shift) * 0.69314718055994531f;
    };
    if (nsplit == 2) {  // the usual cut of a batch: four rows of two parts in flight
        const int step = 8 * gridDim.y;
        for (int i0 = blockIdx.y * 8 + warp; i0 < ntok * gs; i0 += 4 * step) {
            float2 x[4][2];
            float v[4][2][VW];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = min(i0 + u * step, ntok * gs - 1), t = i / gs;
                const int row = t < P.tt ? t * P.gs + (i - t * gs) : kTileRows + (t - P.tt) * P.gs + (i - t * gs);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int64_t at = (k == 0 ? first : rest + (int64_t)2 * P.cap_rows) + row;
                    x[u][k] = __ldcg(P.part_ml + at);
                    const float* p = P.part_o + at * DC + lane * VW;
                    if constexpr (VW == 4)
                        *reinterpret_cast<float4*>(v[u][k]) = __ldcg(reinterpret_cast<const float4*>(p));
                    else
                        *reinterpret_cast<float2*>(v[u][k]) = __ldcg(reinterpret_cast<const float2*>(p));
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (i0 + u * step >= ntok * gs) break;
                const float M = fmaxf(x[u][0].x, x[u][1].x);
                const float f0 = x[u][0].x == -INFINITY ? 0.0f : ex2(x[u][0].x - M), f1 = x[u][1].x == -INFINITY ? 0.0f : ex2(x[u][1].x - M);
                float o[VW];
#pragma unroll
                for (int e = 0; e < VW; ++e)  // a part without weight may hold anything
                    o[e] = (f0 != 0.0f ? v[u][0][e] * f0 : 0.0f) + (f1 != 0.0f ? v[u][1][e] * f1 : 0.0f);
                put(i0 + u * step, M, x[u][0].y * f0 + x[u][1].y * f1, o);
            }
        }
        return;
    }
    for (int i0 = blockIdx.y * rpb; i0 < ntok * gs; i0 += rpb * gridDim.y) {
        const int i = i0 + warp / wpr;
        float M = -INFINITY, l = 0.0f, o[VW] = {};
        if (i < ntok * gs) {
            const int t = i / gs, row = t < P.tt ? t * P.gs + (i - t * gs) : kTileRows + (t - P.tt) * P.gs + (i - t * gs);
            for (int k0 = warp % wpr; k0 < nsplit; k0 += 4 * wpr) {
                float2 x[4];
                float v[4][VW];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int k = k0 + u * wpr;
                    const int64_t at = (k == 0 ? first : rest + (int64_t)2 * k * P.cap_rows) + row;
                    x[u] = make_float2(-INFINITY, 0.0f);
                    if (k < nsplit) {
                        x[u] = __ldcg(P.part_ml + at);
                        const float* p = P.part_o + at * DC + lane * VW;
                        if constexpr (VW == 4)
                            *reinterpret_cast<float4*>(v[u]) = __ldcg(reinterpret_cast<const float4*>(p));
                        else
                            *reinterpret_cast<float2*>(v[u]) = __ldcg(reinterpret_cast<const float2*>(p));
                    }
                }
                const float N = fmaxf(fmaxf(fmaxf(x[0].x, x[1].x), fmaxf(x[2].x, x[3].x)), M);
                if (N == -INFINITY) continue;
                const float g = ex2(M - N);
                l *= g;
#pragma unroll
                for (int e = 0; e < VW; ++e) o[e] *= g;
                M = N;
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (x[u].x != -INFINITY) {
                        const float f = ex2(x[u].x - N);
                        l = fmaf(x[u].y, f, l);
#pragma unroll
                        for (int e = 0; e < VW; ++e) o[e] = fmaf(v[u][e], f, o[e]);
                    }
            }
        }
        if (wpr == 1) {
            if (i < ntok * gs) put(i, M, l, o);
            continue;
        }
        __syncthreads();  // the last rows are read
        if (lane == 0) s_x[warp] = make_float2(M, l);
#pragma unroll
        for (int e = 0; e < VW; ++e) s_o[warp][lane * VW + e] = o[e];
        __syncthreads();
        if (warp % wpr == 0 && i < ntok * gs) {
            float N = M;
            for (int k = 1; k < wpr; ++k) N = fmaxf(N, s_x[warp + k].x);
            const float g = N == -INFINITY ? 0.0f : ex2(M - N);
            l *= g;
#pragma unroll
            for (int e = 0; e < VW; ++e) o[e] *= g;
            for (int k = 1; k < wpr; ++k) {
                const float2 x = s_x[warp + k];
                if (x.x == -INFINITY) continue;
                const float f = ex2(x.x - N);
                l = fmaf(x.y, f, l);
#pragma unroll
                for (int e = 0; e < VW; ++e) o[e] = fmaf(s_o[warp + k][lane * VW + e], f, o[e]);
            }
            put(i, N, l, o);
        }
    }
}

inline int channel_class(int head_dim) { return head_dim <= 64 ? 64 : 128; }
// of shares of `ctas` CTAs, of row blocks of `rows` rows
inline size_t cut_bytes(int ctas) { return sizeof(Cut) * (size_t)ctas; }
inline size_t ml_bytes(int ctas, int rows) { return sizeof(float2) * 2 * (size_t)ctas * (size_t)rows; }
inline size_t part_bytes(int ctas, int rows, int head_dim) {
    return cut_bytes(ctas) + ml_bytes(ctas, rows) + sizeof(float) * 2 * (size_t)ctas * (size_t)rows * channel_class(head_dim);
}
inline void carve(AttnPlan& P, void* ws, int ctas) {
    char* w = static_cast<char*>(ws);
    P.cuts = reinterpret_cast<Cut*>(w);
    w += cut_bytes(ctas);
    P.part_ml = reinterpret_cast<float2*>(w);
    w += ml_bytes(ctas, P.cap_rows);
    P.part_o = reinterpret_cast<float*>(w);
}
// what follows from the cache and the scale alone
inline void plan_common(AttnPlan& P, const AttnArgs& a) {
    P.page_log2 = 0;
    while ((1 << P.page_log2) < a.c.page_size) ++P.page_log2;
    P.cap_keys = std::min<int64_t>((int64_t)a.max_pages * a.c.page_size, INT32_MAX - (kTileKeys - 1));
    const float scale = a.scale;
    P.sc = scale == 0.0f ? 1.0f : (float)((double)(scale < 0.0f ? -scale : scale) * 1.4426950408889634074);
    P.s_and = scale == 0.0f ? 0u : 0xffffffffu;
    P.s_xor = scale < 0.0f ? 0x80000000u : 0u;
}
// blocks of a cut's join: for its mean number of rows (a block takes 8 of them, or one of many parts); 32 for each of the 152 cost
// 8 us where most have nothing to do
inline int join_blocks(const AttnArgs& a, const AttnPlan& P) {
    const int64_t mean = (a.n_tok + a.n_seq - 1) / a.n_seq * P.gs;
    return (int)std::min<int64_t>(std::min<int64_t>(mean, P.cap_rows), 16);
}

}  // namespace
}  // namespace pps
