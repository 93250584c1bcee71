// pps_attention.cu -- attention of the newest tokens of each sequence over a paged cache (tcgen05, sm_103a).
//
//   out[i] = sum_j w_j v_j / sum_j w_j,   w_j = exp(scale q_i . k_j)   over the keys j that row i sees,
//
// with the running maximum and sum of an online softmax, so that every key and value is read once per row block.
//
// Rows.  The tokens of a sequence and the heads that share a key head (group; taken gs <= 128 at a time) are packed
// into rows, token after token, so that a decoding step's few rows read their keys once.  A tile is 128 rows (tensor
// memory's lanes) of which tt gs are used, tt = 128 / gs whole tokens: one TMA box of queries.  A row block is two
// tiles, or one where its tokens fit into one.  Keys are taken 128 at a time.
//
// Two streams.  Each of two softmax warpgroups drives one stream: scores S = Q K^T into its own 128 columns of
// tensor memory, weights P written over them in 16 bits, O += P V into its own accumulator (P is read from tensor
// memory).  A block of two tiles gives each stream a tile and both the same keys; a block of one tile gives
// both streams the same rows and every other key tile, and their results are merged at the end.  Either way the tensor
// cores work for one stream while the other is in its softmax.
//
// Softmax.  A thread owns a row.  O is rescaled only when a row's maximum has risen by more than 2^kLazy since the
// maximum in use (then by its own warpgroup, in place): the weights may pass 1 by that factor, which neither
// the fp32 sums nor the 16-bit types' ranges feel.  Weights are rounded to the cache's type for the second product
// (up to 2^-8 of each in bf16, 2^-11 in fp16, as the result's own rounding); their sum is formed before rounding.  The largest
// weight of a row is 2^kShift and loses nothing as long as its score is the maximum in use; below a later, larger one (by less than
// kLazy) it is any number, so a row with one key that matters may be off by one such rounding more.  Against 64 bits the error is 1.4 times
// that of a result formed in fp32 and rounded once (bf16 2.3e-3 to 1.7e-3, fp16 2.8e-4 to 2.1e-4): weights of 32 bits would double the products.
//
// Work split.  Key tiles of all (sequence, key head, row block) items, plus kFix per item for its start and end, lie
// on one line that is cut into equal shares, one per SM, whatever the lengths are; a cut that would leave a few tiles
// of an item alone moves to the item's end.  An item cut between CTAs leaves
// one partial result (maximum, sum, fp32 O) per CTA, at most two per CTA, and a second launch joins them in
// order: the same call gives the same bits.  Lengths are read on the device; nothing waits for the host.
//
// Every wait gives up after tc::kWaitLimit polls and raises PPS_FLAG_TIMEOUT.
//
// Measured (bf16, 32 heads over 8 key heads of 128 channels unless said; a copy moves 6.78 TB/s, library products run
// at 1936 TFLOP/s):
//   64 sequences, a token each, up to 8000 keys      216 us = 6.1 TB/s, 0.91 of the copy's: bound by HBM
//   one sequence of 130001 keys, 28 over 4 heads      55 us = 4.8 TB/s: one segment per CTA, of which 8 us of start, end, join
//   64 trees of 41 nodes, up to 4100 keys            180 to 183 us = 4.0 TB/s: a key tile takes 3200 clocks (164 rows padded to 256), and
//                                                    CTAs go through 3.8 segments, 10000 clocks of start and end each
//   8192 tokens after 8192                          1030 to 1050 us = 1600 TFLOP/s, 0.82 of the library's rate: a key tile of two row tiles
//                                                    takes 2880 clocks, 2048 of them tensor work; the rest is the softmax's latency.
//                                                    Over seconds 1120 us = 1480 TFLOP/s, 0.86 of the library's sustained rate: the power
//                                                    limit (1.38 kW) takes the clock from 2070 to 1935 MHz
//   7 chunks of up to 777 tokens, 14 over 2 x 64      51 us = 380 TFLOP/s: 64 channels halve the products, not the softmax (2650 clocks)
//   one sequence of 900 keys                          13 us: some 6 us from the launch to the first scores, of which most is
//                                                    fetching each role's instructions; 4 us for the join
// Code size is speed here: with the wait loops unrolled by the compiler (198 KB of code, now 110) the long sequence took 66 us.
//
// Built and measured slower: P apart from S at 64 channels, so that the next scores need not wait for O += P V (3 to 5 percent: the
// softmax, not the products' latency, is what a tile takes); the next segment's page table read ahead by the loaders (1 percent);
// the plan made by every warp for itself (3 to 8 percent: more code at the start); four softmax warpgroups, half of a row's keys each
// (28 percent: a vote per tile on the common maximum, 96 registers, so that some scores are read twice); shares of at least 2, 4 or 8 key tiles (short
// contexts up to 45 percent).
#include <algorithm>
#include <atomic>
#include <cfloat>
#include <climits>
#include <cstdint>
#include <cstring>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pps.h"
#include "pps_internal.h"
#include "pps_tc.cuh"

namespace pps {
namespace {

using namespace tc;

constexpr int kTileRows = 128, kTileKeys = 128;
constexpr int kAttnThreads = 384;  // two softmax warpgroups; warps that load keys, values, issue products, load queries
constexpr int kLoadWarp = 8, kMmaWarp = 10, kQueryWarp = 11;
static_assert(32 * (kQueryWarp + 1) == kAttnThreads, "the last warp loads the queries");
constexpr int kMaxCtas = 160;      // shares of the work (one per SM)
// Key tiles that an item's start and end cost.  (2, 3, 4: decoding batches and ragged chunks 1 to 3 percent faster, trees 3 to 11
// and one long sequence 4 to 6 percent slower.)
constexpr int kFix = 6;
constexpr int kLeast = 3;          // of a cut item's key tiles, at most, for a cut to move to the item's end
constexpr float kLazy = 8.0f;      // log2 of the rise of a maximum that O is not rescaled for
constexpr uint32_t kColO = 256;    // tensor memory columns: S/P of streams 0, 1; O of streams 0, 1

// what depends on the channels' class DC: 64 (head_dim <= 64) or 128
template <int DC>
struct Cfg {
    static constexpr int kBlock = 128 * 128;                 // 128 rows of 64 channels, 128-byte swizzle
    static constexpr int kTile = kBlock * (DC / 64);         // 16 or 32 KB: a tile of Q, K or V
    static constexpr int kStages = (224 * 1024 - 2 * kTile) / kTile;  // 5 (or 12) tiles of K and V in flight
    static constexpr int kSmem = (2 + kStages) * kTile + 320 /* barriers */ + 224 /* plan */ + 2048 /* maxima and sums */;
    static_assert(8 * (2 * kStages + 13) <= 320 && kSmem <= 227 * 1024, "barriers and shared memory fit");
};

// a cut item: nsplit partial results of a block of ntok tokens from tok0 on, in slot 2 cta + 1 and slots 2 (cta + k),
// k = 1 .. nsplit - 1
struct Cut {
    int32_t nsplit, ntok, tok0, vh;
};

struct AttnPlan {
    int group, gs, nsub, tt;  // heads of a key head; those taken at a time, in nsub turns; tokens per tile
    int cap_rows, page_log2;
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
    const int i0 = blk * 2 * P.tt;
    if (a.mask == nullptr) vis = max(0, q.len - q.n + i0 + min(q.n - i0, 2 * P.tt));
    return (vis + kTileKeys - 1) / kTileKeys;
}
__device__ __forceinline__ int n_blocks(const AttnPlan& P, const Seq& q) {
    return (int)(((uint32_t)q.n + 2u * P.tt - 1u) / (2u * P.tt));
}
__device__ __forceinline__ int64_t head_cost(const AttnArgs& a, const AttnPlan& P, const Seq& q) {
    const int nb = n_blocks(P, q);
    if (nb == 1 || a.mask != nullptr) return (int64_t)nb * (block_tiles(a, P, q, 0) + kFix);
    int64_t c = 0;
#pragma unroll 1
    for (int b = 0; b < nb; ++b) c += block_tiles(a, P, q, b) + kFix;
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
            i0 = blk * 2 * P.tt;
            ntok = min(q.n - i0, 2 * P.tt);
            t0 = cut_at(x - base, T, least);
            t1 = cut_at(x1 - base, T, least);
            const bool none = T == 0 && x == base;
            from = base;
            heads = vh;
            base += T + kFix;
            x = base;
            ++blk;
            if (t0 < t1 || none) return true;
        }
        return false;
    }
};

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

__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int* abort) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort));
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

template <typename T, int DC>
__global__ void __launch_bounds__(kAttnThreads, 1)
    attention_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                     const __grid_constant__ CUtensorMap tmV, const AttnArgs a, const AttnPlan P) {
    using C = Cfg<DC>;
    using H = Half<T>;
    extern __shared__ __align__(1024) uint8_t attn_smem[];
    const uint32_t base = smem_u32(attn_smem);
    const uint32_t ring = base + 2 * C::kTile;
    const uint32_t bars = ring + C::kStages * C::kTile;
    auto bar = [&](uint32_t i) { return bars + 8u * i; };
    auto full = [&](uint32_t s) { return bar(s); };
    auto empty = [&](uint32_t s) { return bar(C::kStages + s); };
    auto sfull = [&](uint32_t w) { return bar(2 * C::kStages + w); };
    auto pready = [&](uint32_t w, uint32_t half) { return bar(2 * C::kStages + (half ? 11 : 2) + w); };  // a barrier per half: no warp may count twice
    auto odone = [&](uint32_t w) { return bar(2 * C::kStages + 4 + w); };
    auto qfull = [&](uint32_t t) { return bar(2 * C::kStages + 6 + t); };
    auto qfree = [&](uint32_t t) { return bar(2 * C::kStages + 8 + t); };
    const uint32_t segbar = bar(2 * C::kStages + 10);
    uint8_t* tail = attn_smem + (2 + C::kStages) * C::kTile + 320;
    volatile int* abort = reinterpret_cast<volatile int*>(tail);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tail + 4);
    int64_t* s_sum = reinterpret_cast<int64_t*>(tail + 16);          // [12] warp sums
    Start* s_start = reinterpret_cast<Start*>(tail + 16 + 12 * 8);
    float2* s_ml = reinterpret_cast<float2*>(tail + 224);            // [2][128]
    static_assert(16 + 12 * 8 + sizeof(Start) <= 224, "plan fits");

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    if (tid == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(sfull(w), 1);
            mbar_init(pready(w, 0), 4);  // the weights of a tile's first 64 keys
            mbar_init(pready(w, 1), 4);  // of the others
            mbar_init(odone(w), 1);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(qfull(t), 1);
            mbar_init(qfree(t), 1);
        }
        mbar_init(segbar, 8);
        *abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kLoadWarp && lane == 0) {
        tma_prefetch_map(&tmQ);
        tma_prefetch_map(&tmK);
        tma_prefetch_map(&tmV);
    }
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    pdl_wait();  // what comes before this runs while the stream's last kernel ends
    pdl_launch_dependents();
    Seq own = {0, 0, 0};
    if (tid < a.n_seq) own = load_seq(a, P, tid, cta == 0);
    if (tid == 0) P.cuts[cta].nsplit = 0;

    // the share: [c0, c1) of the line of costs, and where on it the share starts
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
        for (int i = 0; i < kAttnThreads / 32; ++i) {
            const int64_t t = s_sum[i];
            if (i < warp) w += t;
            total += t;
        }
        return w;
    };
    const int64_t mine = cost(own);
    int64_t more = 0;
    for (int64_t s = tid + kAttnThreads; s < a.n_seq; s += kAttnThreads) more += cost(load_seq(a, P, (int)s, cta == 0));
    int64_t U, U0;
    int64_t at = block_scan(mine, U0);
    U = U0;
    if (a.n_seq > kAttnThreads) {
        block_scan(more, U);
        U += U0;
    }
    const int64_t share = max(divide(U + gridDim.x - 1, gridDim.x), (int64_t)1);
    const int64_t c0 = min(cta * share, U), c1 = min(c0 + share, U);
    if (c0 < c1) {
        int64_t before = 0, v = mine;
        for (int64_t b = 0;; b += kAttnThreads) {
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
                for (int c; rem >= (c = block_tiles(a, P, own, st.blk) + kFix); ++st.blk) rem -= c;
                st.base = c0 - rem;
                *s_start = st;
            }
            before += U0;
            if (before > c0) break;  // CTA-uniform
            own.n = 0;
            if (b + kAttnThreads + tid < a.n_seq) own = load_seq(a, P, (int)(b + kAttnThreads + tid), false);
            v = cost(own);
            at = block_scan(v, U0);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    if (c0 >= c1 || (base & 1023u) != 0) {  // no work (or a base that the swizzled tiles cannot have)
        if (c0 < c1 && tid == 0 && a.status) atomicOr(a.status, PPS_FLAG_TIMEOUT);
        if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
        return;
    }
    const int least = (int)min(max(share / 8, (int64_t)1), (int64_t)kLeast);
    Walk W(P, *s_start, c0, c1, least);
    const int D = a.c.head_dim;

    // registers: 384 x 168 at launch = 256 x 216 + 128 x 72
    if (warp >= kLoadWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp < kMmaWarp) {
            // ---- one warp loads the keys' tiles, one the values'.  The ring holds them in the order of their use: K of
            // the first tile (or two, one per stream), then V_j and the next K in turn.
            const bool is_v = warp != kLoadWarp;
            const int box = min(kTileKeys, a.c.page_size), boxes = kTileKeys / box, box_log2 = 31 - __clz(boxes);
            // the segment's first place in the ring; one past the last place this warp filled, and which it filled before it
            uint32_t ring0 = 0, last = 0, filled = 0;
            bool ok = true;
            while (ok && W.next(a, P)) {
                const int n = W.t1 - W.t0, ahead = W.ntok <= P.tt ? 2 : 1, len = W.q.len, kvh = W.heads / P.nsub;
                const int32_t* table = a.pages + (int64_t)W.s * a.pages_stride;
                // pages of 32 boxes at a time, one per lane; the next 32 are on their way
                const int per = 32 >> box_log2;  // tiles of 32 boxes
                auto pages_from = [&](int j) {
                    const int64_t k = (int64_t)(W.t0 + j) * kTileKeys + lane * box;
                    return k < len && j < n ? __ldg(table + (k >> P.page_log2)) : 0;
                };
                int cur = pages_from(0), nxt = pages_from(per);
                for (int j = 0; j < n; ++j) {
                    if (j > 0 && (j & (per - 1)) == 0) {
                        cur = nxt;
                        nxt = pages_from(j + per);
                    }
                    const uint32_t it = ring0 + (is_v ? (j + ahead < n ? ahead + 2 * j : n + j) : j < ahead ? j : 2 * j - ahead + 1);
                    const uint32_t s = it % C::kStages;
                    if (!(ok = wait_warp(empty(s), ((it / C::kStages) & 1u) ^ 1u, abort))) break;
                    filled = (filled << (it + 1 - last)) | 1u;
                    last = it + 1;
                    const int k0 = (W.t0 + j) * kTileKeys, need = (min(kTileKeys, len - k0) + box - 1) / box;
                    const uint32_t dst = ring + s * C::kTile;
                    int page = __shfl_sync(0xffffffffu, cur, ((j & (per - 1)) << box_log2) + (lane & (boxes - 1)));
                    if (lane == 0) mbar_expect_tx(full(s), (uint32_t)(need * box * 128 * (DC / 64)));
                    __syncwarp();
                    if (lane < need) {
                        if (page < 0 || page >= a.c.n_pages) {  // reads as zeros past the last page
                            if (a.status) atomicOr(a.status, PPS_FLAG_INDEX);
                            page = (int)a.c.n_pages;
                        }
                        const int in_page = (k0 + lane * box) & (a.c.page_size - 1);
#pragma unroll
                        for (int b = 0; b < DC / 64; ++b)
                            if (is_v)
                                tma_load_4d(dst + b * C::kBlock + lane * box * 128, &tmV, full(s), b * 64, in_page, kvh, page);
                            else
                                tma_load_4d(dst + b * C::kBlock + lane * box * 128, &tmK, full(s), b * 64, in_page, kvh, page);
                    }
                }
                ring0 += 2 * n;
            }
            // copies in flight when the CTA gives up: wait (bounded) for each
            for (uint32_t j = 0; j < (uint32_t)C::kStages && *abort; ++j)
                if (filled >> j & 1u)
                    for (uint32_t n = 0, i = last - 1 - j; n < kWaitLimit && !mbar_try_wait(full(i % C::kStages), (i / C::kStages) & 1u); ++n) {
                    }
        } else if (warp == kMmaWarp) {
            // ---- products (one thread): per stream S = Q K^T, then O += P V as its weights arrive
            // Straight-line products of the class's full width (channels past head_dim are zeros): in a loop they issue at
            // 100 cycles each, so at the tensor core's 64.  No product stands under a condition of its own.
            if (elect_one()) {
                constexpr uint32_t id_qk = (1u << 4) | (H::kType << 7) | (H::kType << 10) | ((kTileKeys / 8u) << 17) | ((kTileRows / 16u) << 24);
                constexpr uint32_t id_pv = (1u << 4) | (H::kType << 7) | (H::kType << 10) | (1u << 16) | ((DC / 8u) << 17) | ((kTileRows / 16u) << 24);
                uint32_t it = 0, np0 = 0, np1 = 0, nq0 = 0, nq1 = 0, turn = 0;
                auto stage = [&](uint32_t i) { return ring + (i % C::kStages) * C::kTile; };
                auto landed = [&](uint32_t i) {
                    const bool ok = mbar_wait(full(i % C::kStages), (i / C::kStages) & 1u, abort);
                    tc_fence_after();
                    return ok;
                };
                auto scores = [&](uint32_t w, uint32_t tile, uint32_t k, bool last) {  // last: the segment needs the queries no more
                    const uint64_t qd = sw128_desc(base + tile * C::kTile), kd = sw128_desc(stage(k));
#pragma unroll
                    for (uint32_t c = 0; c < DC / 16; ++c) {
                        const uint64_t o = ((c >> 2) * C::kBlock + (c & 3u) * 32u) >> 4;
                        tc_mma(tmem + w * 128u, qd + o, kd + o, id_qk, c != 0);
                    }
                    tc_commit(sfull(w));
                    if (last) tc_commit(qfree(tile));
                };
                // O += P V in two halves, each as soon as its weights are there
                auto values = [&](uint32_t w, uint32_t v, bool first) {
                    const uint64_t vd = sw128_desc_mn(stage(v), C::kBlock);
                    const uint32_t o = tmem + kColO + w * 128u, p = tmem + w * 128u, at = w ? np1 : np0;
                    ++(w ? np1 : np0);
                    if (!mbar_wait(pready(w, 0), at & 1u, abort)) return false;
                    tc_fence_after();
#pragma unroll
                    for (uint32_t c = 0; c < kTileKeys / 32; ++c) tc_mma_ts(o, p + c * 8u, vd + c * (2048u >> 4), id_pv, !first || c != 0);
                    if (!mbar_wait(pready(w, 1), at & 1u, abort)) return false;
                    tc_fence_after();
#pragma unroll
                    for (uint32_t c = kTileKeys / 32; c < kTileKeys / 16; ++c) tc_mma_ts(o, p + c * 8u, vd + c * (2048u >> 4), id_pv, 1u);
                    tc_commit(odone(w));
                    return true;
                };
                bool ok = true;
                while (ok && W.next(a, P)) {
                    const int n = W.t1 - W.t0;
                    if (n == 0) continue;
                    if (W.ntok > P.tt) {  // a tile per stream, the same keys
                        ok = mbar_wait(qfull(0), nq0++ & 1u, abort) && mbar_wait(qfull(1), nq1++ & 1u, abort) && landed(it);
                        if (!ok) break;
                        scores(0, 0, it, n == 1);
                        scores(1, 1, it, n == 1);
                        tc_commit(empty(it % C::kStages));
                        ++it;
                        for (int j = 0; j < n && ok; ++j) {
                            const uint32_t v = it, k = it + 1;
                            const bool more_keys = j + 1 < n;
                            ok = landed(v);
                            for (uint32_t w = 0; w < 2 && ok; ++w) {
                                ok = values(w, v, j == 0);
                                if (!ok) break;
                                if (w == 1) tc_commit(empty(v % C::kStages));
                                if (more_keys) {
                                    if (w == 0) ok = landed(k);
                                    if (!ok) break;
                                    scores(w, w, k, j + 2 == n);
                                    if (w == 1) tc_commit(empty(k % C::kStages));
                                }
                            }
                            it += more_keys ? 2 : 1;
                        }
                    } else {  // one tile, every other key tile per stream: S of tile j + 2 follows O += P V of tile j
                        const uint32_t tile = turn;
                        turn ^= 1u;
                        ok = mbar_wait(qfull(tile), (tile ? nq1++ : nq0++) & 1u, abort);
#pragma unroll 1
                        for (int j = -2; j < n && ok; ++j) {
                            const uint32_t w = (uint32_t)j & 1u;
                            if (j >= 0) {
                                if (!(ok = landed(it) && values(w, it, j < 2))) break;
                                tc_commit(empty(it % C::kStages));
                                ++it;
                            }
                            if (j + 2 < n) {
                                if (!(ok = landed(it))) break;
                                scores(w, tile, it, j + 3 == n);
                                tc_commit(empty(it % C::kStages));
                                ++it;
                            }
                        }
                    }
                }
            }
            __syncwarp();
        } else {
            // ---- queries: both tiles of a block of two, or the tile that the last block of one did not use
            uint32_t n0 = 0, n1 = 0, turn = 0;
            bool ok = true;
            while (ok && W.next(a, P)) {
                if (W.t0 == W.t1) continue;
                const bool two = W.ntok > P.tt;
                const int kvh = W.heads / P.nsub, sub = W.heads - kvh * P.nsub;
                for (uint32_t i = 0; i < (two ? 2u : 1u) && ok; ++i) {
                    const uint32_t tile = two ? i : turn;
                    ok = wait_warp(qfree(tile), ((tile ? n1 : n0) & 1u) ^ 1u, abort);
                    if (!ok) break;
                    if (tile) ++n1; else ++n0;
                    if (lane == 0) {
                        mbar_expect_tx(qfull(tile), (uint32_t)(P.gs * P.tt * 128 * (DC / 64)));
#pragma unroll
                        for (int b = 0; b < DC / 64; ++b)
                            tma_load_4d(base + tile * C::kTile + b * C::kBlock, &tmQ, qfull(tile), b * 64, sub * P.gs,
                                        W.q.off + W.i0 + (int)i * P.tt, kvh);
                    }
                    __syncwarp();
                }
                if (!two) turn ^= 1u;
            }
            // copies in flight when the CTA gives up: wait (bounded) for each
            for (uint32_t tile = 0; tile < 2 && *abort; ++tile) {
                const uint32_t u = tile ? n1 : n0;
                for (uint32_t n = 0; u > 0 && n < kWaitLimit && !mbar_try_wait(qfull(tile), (u - 1) & 1u); ++n) {
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // ---- softmax: warpgroup w drives stream w, thread = row r of its tile
        const uint32_t w = warp >> 2, q4 = warp & 3;
        const int r = (int)(q4 * 32) + lane;
        const int row_tok = r / P.gs, row_head = r - row_tok * P.gs;  // the row's token in its tile, its head of the turn
        const uint32_t lanes = (q4 * 32u) << 16;
        const uint32_t tS = tmem + lanes + w * 128u, tO = tmem + lanes + kColO;
        uint32_t done = 0, done_other = 0;  // tiles of this stream and of the other one so far
        uint32_t it = 0, syncs = 0;
        auto seg_sync = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(segbar);
            return wait_warp(segbar, syncs++ & 1u, abort);
        };
        bool ok = true;
        const bool odd_scale = P.s_xor != 0 || P.s_and == 0;
        while (ok && W.next(a, P)) {
            const bool two = W.ntok > P.tt;  // a tile per stream
            const int n = W.t1 - W.t0;
            const int kvh = W.heads / P.nsub, in_group = (W.heads - kvh * P.nsub) * P.gs + row_head;
            const int in_tok = (two ? (int)w * P.tt : 0) + row_tok;  // in the block
            const bool valid = row_tok < P.tt && in_tok < W.ntok && in_group < P.group;
            const bool busy = __any_sync(0xffffffffu, valid);
            const int tok = W.i0 + min(in_tok, W.ntok - 1), head = kvh * P.group + in_group;
            const int in_block = (two ? (int)w * kTileRows : 0) + r;
            const int prefix = W.q.len - W.q.n;
            const uint32_t* mask = a.mask ? a.mask + (int64_t)(W.q.off + tok) * a.mask_words : nullptr;
            const int vis = mask ? W.q.len : prefix + tok + 1;
            const int plain = mask ? prefix : vis;  // keys below it are seen by the row
            float m = -INFINITY, l = 0.0f;
            int i = 0;  // tiles of the stream in this segment
            for (int j = two ? 0 : (int)w; j < n; j += two ? 1 : 2, ++i) {
                const int k0 = (W.t0 + j) * kTileKeys;
                const bool partly = __any_sync(0xffffffffu, k0 + kTileKeys > plain) || odd_scale;  // not all as it stands
                if (!(ok = wait_warp(sfull(w), (done + i) & 1u, abort))) break;
                // values past the sequence's end (in its last tile): whatever the pages hold there becomes zero before any
                // weight is handed over
                if (k0 + kTileKeys > W.q.len && (w == 0 || !two)) {
                    const uint32_t v = it + 2 * n - 1;  // the segment's last value tile
                    if (!(ok = wait_warp(full(v % C::kStages), (v / C::kStages) & 1u, abort))) break;
                    const uint32_t from = ring + (v % C::kStages) * C::kTile + (W.q.len - k0) * 128;
                    const uint32_t bytes = (k0 + kTileKeys - W.q.len) * 128;
#pragma unroll
                    for (int b = 0; b < DC / 64; ++b)
                        for (uint32_t o = r * 16; o < bytes; o += 128 * 16)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(from + b * C::kBlock + o), "r"(0) : "memory");
                    fence_async_smem();
                }
                tc_fence_after();
                if (busy) {
                    uint32_t v[4][32];
                    tmem_ld32(tS, v[0]);
                    tmem_ld32(tS + 32, v[1]);
                    tmem_wait_ld();
                    tmem_landed(v[0]);
                    tmem_landed(v[1]);
                    tmem_ld32(tS + 64, v[2]);
                    tmem_ld32(tS + 96, v[3]);
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    auto highest = [&](int c) {  // of 32 scores, in four chains
#pragma unroll
                        for (int e = 0; e < 32; e += 2)
                            mx[(e >> 1) & 3] = max3(mx[(e >> 1) & 3], __uint_as_float(v[c][e]), __uint_as_float(v[c][e + 1]));
                    };
                    highest(0);
                    highest(1);
                    tmem_wait_ld();
                    tmem_landed(v[2]);
                    tmem_landed(v[3]);
                    highest(2);
                    highest(3);
                    if (partly) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) mx[c] = -INFINITY;
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t bits = seen_bits(k0 + 32 * c, vis, prefix, mask, a.mask_words);
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                v[c][e] = (v[c][e] & P.s_and) ^ P.s_xor;
                                if (!(bits & (1u << e))) v[c][e] = 0xff800000u;  // -inf
                            }
                            highest(c);
                        }
                    }
                    const float top = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]);
                    if (__any_sync(0xffffffffu, valid && (top - m) * P.sc > kLazy)) {
                        const float M = fmaxf(m, top), f = m == M ? 1.0f : ex2((m - M) * P.sc);
                        m = M;
                        l *= f;
                        if (i > 0) {
                            if (!(ok = wait_warp(odone(w), (done + i - 1) & 1u, abort))) break;
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < D; c += 16) {  // few columns: the scores stay in registers
                                uint32_t o[16];
                                tmem_ld16(tO + w * 128u + c, o);
                                tmem_wait_ld();
                                tmem_landed(o);
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_st16(tO + w * 128u + c, o);
                            }
                        }
                    }
                    const float neg = (m == -INFINITY ? 0.0f : -m * P.sc) + H::kShift;
                    const uint64_t sc2 = pack2(P.sc, P.sc), neg2 = pack2(neg, neg);
                    uint64_t sum[2] = {0, 0};
                    auto weights = [&](int c) {  // of 32 keys, into tensor memory
                        uint32_t pk[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float x0, x1;
                            unpack2(fma2(pack2(__uint_as_float(v[c][2 * e]), __uint_as_float(v[c][2 * e + 1])), sc2, neg2), x0, x1);
                            x0 = ex2(x0);
                            x1 = ex2(x1);
                            sum[e & 1] = add2(sum[e & 1], pack2(x0, x1));
                            pk[e] = H::pack(x0, x1);
                        }
                        tmem_st16(tS + c * 16, pk);
                    };
                    weights(0);
                    weights(1);
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(pready(w, 0));
                    weights(2);
                    weights(3);
                    float s0, s1;
                    unpack2(add2(sum[0], sum[1]), s0, s1);
                    l += s0 + s1;
                    tmem_wait_st();
                } else {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(pready(w, 0));
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pready(w, 1));
            }
            if (!ok) break;
            // ---- the segment's result
            const bool whole = W.t0 == 0 && W.t1 == W.T;
            const int slot = 2 * cta + (W.t0 == 0 ? 1 : 0);
            if (tid == 0 && W.t0 == 0 && !whole) {
                Cut c;
                c.nsplit = (int)divide(W.from + W.T - least, share) - cta + 1;  // the cuts that leave `least` tiles on both sides
                c.ntok = W.ntok;
                c.tok0 = W.q.off + W.i0;
                c.vh = W.heads;
                P.cuts[cta] = c;
            }
            const uint32_t tiles = i, tiles_other = n + (two ? n : 0) - i;
            if (tiles > 0) ok = wait_warp(odone(w), (done + tiles - 1) & 1u, abort);
            if (!ok) break;
            m = fmaxf(m * P.sc, -INFINITY);  // log2 of the largest weight (-inf stays, whatever the scale)
            if (l != l) m = INFINITY;  // a score that is not a number, or infinite: so is the row, whatever it is joined with
            float f = 1.0f, f1 = 0.0f;  // factors of the first accumulator (the stream's own) and, of one tile, the second
            if (!two) {
                s_ml[w * 128 + r] = make_float2(m, l);
                if (!(ok = seg_sync())) break;
                if (tiles_other > 0 && !(ok = wait_warp(odone(w ^ 1u), (done_other + tiles_other - 1) & 1u, abort))) break;
                const float2 x = s_ml[r], y = s_ml[128 + r];
                m = fmaxf(x.x, y.x);
                f = x.x == -INFINITY ? 0.0f : ex2(x.x - m);
                f1 = y.x == -INFINITY ? 0.0f : ex2(y.x - m);
                l = x.y * f + y.y * f1;
            }
            tc_fence_after();
            if (busy) {
                if (whole) {
                    const float inv = l > 0.0f ? 1.0f / l : l;  // (l: zero, or not a number)
                    f *= inv;
                    f1 *= inv;
                }
                const uint32_t first = two ? w : 0u;
                const int from = two ? 0 : (int)w * (DC / 2), to = two ? DC : from + DC / 2;
                // the quad's rows: where they go, which of them are there
                const unsigned long long out = reinterpret_cast<unsigned long long>(
                    static_cast<T*>(a.out.p) + (int64_t)(W.q.off + tok) * a.out.tok + head * a.out.head);
                unsigned long long out4[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) out4[k] = __shfl_sync(0xffffffffu, out, (lane & ~3) + k);
                const uint32_t rows4 = __ballot_sync(0xffffffffu, valid) >> (lane & ~3) & 15u;
                float* part = P.part_o + ((int64_t)slot * P.cap_rows + in_block) * DC;
                if (valid && (two || w == 0)) {
                    if (!whole)
                        P.part_ml[(int64_t)slot * P.cap_rows + in_block] = make_float2(m, l);
                    else if (a.lse)
                        a.lse[(int64_t)(W.q.off + tok) * a.n_heads + head] =
                            l == 0.0f ? -INFINITY : (m + log2f(l) - H::kShift) * 0.69314718055994531f;
                }
                int kind = (whole ? 1 : 0) | (!two && n > 1 ? 2 : 0);
#pragma unroll 1
                for (int c = from; c < to && c < D; c += 32) {
                    asm volatile("" : "+r"(kind));  // one body for all kinds: the compiler would make a loop of each
                    uint32_t o[32];
                    if (n > 0) {
                        tmem_ld32(tO + first * 128u + c, o);
                        tmem_wait_ld();
                        tmem_landed(o);
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        o[e] = n > 0 && f != 0.0f ? __float_as_uint(__uint_as_float(o[e]) * f) : 0u;
                    if (kind & 2) {
                        uint32_t o1[32];
                        tmem_ld32(tO + 128u + c, o1);
                        tmem_wait_ld();
                        tmem_landed(o1);
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (f1 != 0.0f) o[e] = __float_as_uint(fmaf(__uint_as_float(o1[e]), f1, __uint_as_float(o[e])));
                    }
                    const int q = lane & 3;
                    if (kind & 1) {
                        uint4 u[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t* x = o + 8 * e;
                            u[e] = make_uint4(H::pack(__uint_as_float(x[0]), __uint_as_float(x[1])), H::pack(__uint_as_float(x[2]), __uint_as_float(x[3])),
                                              H::pack(__uint_as_float(x[4]), __uint_as_float(x[5])), H::pack(__uint_as_float(x[6]), __uint_as_float(x[7])));
                        }
                        quad_transpose(u, q);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if ((rows4 >> k & 1u) && c + 8 * q < D)
                                *reinterpret_cast<uint4*>(reinterpret_cast<T*>(out4[k]) + c + 8 * q) = u[k];
                    } else {
#pragma unroll
                        for (int b = 0; b < 32; b += 16) {
                            uint4 u[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) u[e] = make_uint4(o[b + 4 * e], o[b + 4 * e + 1], o[b + 4 * e + 2], o[b + 4 * e + 3]);
                            quad_transpose(u, q);
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (rows4 >> k & 1u) *reinterpret_cast<uint4*>(part + (k - q) * DC + c + b + 4 * q) = u[k];
                        }
                    }
                    __syncwarp();
                }
            }
            done += tiles;
            done_other += tiles_other;
            it += 2 * n;
            tc_fence_before();
            ok = seg_sync();  // the accumulators, queries and s_ml are free
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (tid == 0 && *abort && a.status) atomicOr(a.status, PPS_FLAG_TIMEOUT);
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
            a.lse[(int64_t)tok * a.n_heads + head] = l == 0.0f ? -INFINITY : (M + log2f(l) - H::kShift) * 0.69314718055994531f;
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

// ---------------------------------------------------------------- host side

// the heads of a key head taken at a time, the tokens of a tile, the rows of a block
struct Rows {
    int nsub, gs, tt, cap;
    Rows(int64_t n_tok, int group) {
        nsub = (group + kTileRows - 1) / kTileRows;
        gs = (group + nsub - 1) / nsub;
        tt = kTileRows / gs;
        cap = n_tok > tt ? 2 * kTileRows : (int)((n_tok * gs + 31) / 32 * 32);
    }
};
int channel_class(int head_dim) { return head_dim <= 64 ? 64 : 128; }
size_t cut_bytes() { return sizeof(Cut) * kMaxCtas; }
size_t ml_bytes(int rows) { return sizeof(float2) * 2 * kMaxCtas * (size_t)rows; }

// one half of the cache as [page, head, token, channel], loaded in boxes of up to 128 tokens x 64 channels
bool cache_map(CUtensorMap* m, const void* ptr, const CacheView& c, int dtype) {
    EncodeTiledFn f = encode_fn();
    if (f == nullptr) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_size, (cuuint64_t)c.n_kv_heads,
                                (cuuint64_t)std::max<int64_t>(c.n_pages, 1)};
    // the stride of a dimension of one is never used, but has to be a multiple of 16 bytes
    const cuuint64_t strides[3] = {(cuuint64_t)c.tok * 2, c.n_kv_heads > 1 ? (cuuint64_t)c.head * 2 : 256,
                                   c.n_pages > 1 ? (cuuint64_t)c.page * 2 : 256};
    const cuuint32_t box[4] = {64, (cuuint32_t)std::min(kTileKeys, c.page_size), 1, 1}, es[4] = {1, 1, 1, 1};
    // What a miss brings into L2: no more than the rows fill, since their neighbours are other heads' and are read much later.
    // 35 sequences decoding over 20 / 4 heads, pages token by token, with 256 -> 64 bytes: 64 channels 133 -> 104 us, 80 203 -> 145,
    // 96 208 -> 153 (128 bytes: 177); rows that follow one another (pages head by head), of 72 channels: 256 180, 128 145, 64 150;
    // 128 channels: no difference.
    const auto fetch = c.head_dim % 128 == 0 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B
                       : c.tok == c.head_dim    ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B
                                                : CU_TENSOR_MAP_L2_PROMOTION_L2_64B;
    return f(m, dtype == PPS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
             const_cast<void*>(ptr), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, fetch,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// the queries as [key head, token, head of the group, channel], loaded in boxes of tt tokens x gs heads x 64 channels
bool query_map(CUtensorMap* m, const AttnArgs& a, const AttnPlan& P, int dtype) {
    EncodeTiledFn f = encode_fn();
    if (f == nullptr) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)a.c.head_dim, (cuuint64_t)P.group, (cuuint64_t)a.n_tok, (cuuint64_t)a.c.n_kv_heads};
    const cuuint64_t strides[3] = {P.group > 1 ? (cuuint64_t)a.q.head * 2 : 256, a.n_tok > 1 ? (cuuint64_t)a.q.tok * 2 : 256,
                                   a.c.n_kv_heads > 1 ? (cuuint64_t)a.q.head * P.group * 2 : 256};
    const cuuint32_t box[4] = {64, (cuuint32_t)P.gs, (cuuint32_t)P.tt, 1}, es[4] = {1, 1, 1, 1};
    return f(m, dtype == PPS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, a.q.p, dims, strides,
             box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int DC>
cudaError_t launch(const AttnArgs& a, int dtype, cudaStream_t st) {
    AttnPlan P;
    P.group = a.n_heads / a.c.n_kv_heads;
    const Rows rows(a.n_tok, P.group);
    P.nsub = rows.nsub;
    P.gs = rows.gs;
    P.tt = rows.tt;
    P.cap_rows = rows.cap;
    P.page_log2 = 0;
    while ((1 << P.page_log2) < a.c.page_size) ++P.page_log2;
    P.cap_keys = std::min<int64_t>((int64_t)a.max_pages * a.c.page_size, INT32_MAX - (kTileKeys - 1));
    const float scale = a.scale;
    P.sc = scale == 0.0f ? 1.0f : (float)((double)(scale < 0.0f ? -scale : scale) * 1.4426950408889634074);
    P.s_and = scale == 0.0f ? 0u : 0xffffffffu;
    P.s_xor = scale < 0.0f ? 0x80000000u : 0u;
    char* w = static_cast<char*>(a.ws);
    P.cuts = reinterpret_cast<Cut*>(w);
    w += cut_bytes();
    P.part_ml = reinterpret_cast<float2*>(w);
    w += ml_bytes(P.cap_rows);
    P.part_o = reinterpret_cast<float*>(w);
    CUtensorMap tmQ, tmK, tmV;
    // an empty cache has nothing to read: any mapped memory will do for its maps
    if (!query_map(&tmQ, a, P, dtype) || !cache_map(&tmK, a.c.n_pages > 0 ? a.c.k : a.ws, a.c, dtype) || !cache_map(&tmV, a.c.n_pages > 0 ? a.c.v : a.ws, a.c, dtype))
        return cudaErrorInvalidValue;
    static std::atomic<uint64_t> ready{0};
    cudaError_t e = allow_smem(ready, (const void*)attention_kernel<T, DC>, Cfg<DC>::kSmem);
    if (e != cudaSuccess) return e;
    const int ctas = std::min(device_sm_count(), kMaxCtas);
    e = launch_pdl(attention_kernel<T, DC>, dim3(ctas), dim3(kAttnThreads), Cfg<DC>::kSmem, st, tmQ, tmK, tmV, a, P);
    if (e != cudaSuccess) return e;
    // blocks for a cut's mean number of rows (a block takes 8 of them, or one of many parts); 32 for each of the 152 cost
    // 8 us where most have nothing to do
    const int64_t mean = (a.n_tok + a.n_seq - 1) / a.n_seq * P.gs;
    const int per_cut = (int)std::min<int64_t>(std::min<int64_t>(mean, P.cap_rows), 16);
    return launch_pdl(join_kernel<T, DC>, dim3(ctas, per_cut), dim3(256), 0, st, a, P);
}

template <typename T>
cudaError_t by_channels(const AttnArgs& a, int dtype, cudaStream_t st) {
    return channel_class(a.c.head_dim) == 64 ? launch<T, 64>(a, dtype, st) : launch<T, 128>(a, dtype, st);
}

}  // namespace

size_t attention_workspace_bytes(int64_t n_tok, int n_heads, int n_kv_heads, int head_dim) {
    const int rows = Rows(n_tok, (n_heads + n_kv_heads - 1) / n_kv_heads).cap;
    return cut_bytes() + ml_bytes(rows) + sizeof(float) * 2 * kMaxCtas * (size_t)rows * channel_class(head_dim);
}

cudaError_t launch_attention(const AttnArgs& a, int dtype, cudaStream_t stream) {
    return dtype == PPS_BF16 ? by_channels<__nv_bfloat16>(a, dtype, stream) : by_channels<__half>(a, dtype, stream);
}

}  // namespace pps
