// pps_chain.cu -- verification of drafted chains by the token-level maximal coupling (Alg. 1).
//
// With P = softmax(p / T) and Q = softmax(q / T), the drafted token x of a node is accepted iff
// u Q(x) < P(x); at the first rejection the emitted token is argmax_i max(P(i) - Q(i), 0) / E(i), past
// the chain argmax_i P(i) / E(i).  exp2 of c (l - max) with c = log2(e) / T stands for exp(l / T) throughout;
// a logit equal to its row's maximum counts as 1 also where both are infinite.
//
// Two launches, both bound by HBM.  stats_kernel (which also writes zeros for the acceptance of all rows) reads every logit once: the rows' 16-byte vectors lie on one line
// that is cut into equal shares, one per CTA, and a CTA leaves (max, sum of exponentials) of each row it meets.
// finish_kernel runs slices x sequences: each CTA joins the parts of its chain's rows, finds the first rejection and races
// its slice of the one row (pair) that matters; the CTA that arrives last at the sequence's ticket joins the slices in
// order and writes the outputs.  In both a warp of its own copies chunks to shared memory (cp.async.bulk), several
// ahead, and eight warps compute: with the next vectors in registers instead, the registers of 32 warps an SM did not
// hold enough of them (64 sequences of V = 128256: 66 to 70 us).  The copies take whole 16-byte vectors inside a row;
// the few tokens at its unaligned ends are read one by one.
//
// Measured (in a graph; launched one by one 1.5 to 2 us more): 64 chains of 5, V = 128256, bf16: 47.5 us, 4.5 TB/s over both passes (0.66 of a copy's 6.78): the statistics 35 us (2.5
// of 4 issue slots: exponentials and maxima of 8 logits per vector), the race 23 of which a part runs beside them.  16 ragged chains
// of up to 8, V = 152063, fp32: 31.7 us, 3.2 TB/s.  One chain, V = 32000: 13 to 14 us, two launches and their chains of dependent
// loads (offsets, rows, tokens, logits; sums, acceptance, the row, the ticket).
#include <algorithm>
#include <climits>
#include <cstdint>

#include <cuda_bf16.h>

#include "pps.h"
#include "pps_internal.h"
#include "pps_tc.cuh"

namespace pps {
namespace {

using namespace tc;

constexpr int kThreads = 256;    // that compute; a warp more copies
constexpr int kStatCtas = 2;     // per SM
constexpr int kVecs = 4;         // 16-byte vectors per thread of a chunk
constexpr int kStatChunk = kVecs * kThreads * 16;  // bytes
constexpr int kStatStages = 3;
constexpr int kStatSmem = kStatStages * kStatChunk;
constexpr int kRaceTok = 8;      // tokens per thread of a chunk
constexpr int kRaceChunk = kRaceTok * kThreads;
constexpr int kRaceStages = 4;
template <typename T>
struct RaceSmem {  // a stage: the chunk of the target's row, of the drafter's, of the noise, from the vector that holds its first token
    static constexpr int kRow = kRaceChunk * (int)sizeof(T) + 16, kNoise = kRaceChunk * 4 + 16;
    static constexpr int kStage = 2 * kRow + kNoise, kBytes = kRaceStages * kStage;
    static constexpr int kCtas = sizeof(T) == 2 ? 3 : 2;  // per SM
};
// The first CTA of finish_kernel on an SM fits beside the two of stats_kernel (shared memory, registers): it starts early, and
// its chain of dependent loads (offsets, rows, tokens, logits) is over when the sums are there.
constexpr int kMaxParts = 1024;  // CTAs of stats_kernel
constexpr int kMaxSlices = 64;   // of the final row
constexpr int kMaxChain = 64;    // gamma

struct Stat {
    float m, s;  // the largest logit (-inf: none) and the sum of exp2(c (l - m))
};
struct Best {
    float v;
    int i;  // INT_MAX: none
};

struct ChainPlan {
    int64_t nv, share;  // 16-byte vectors of a row (with room for any alignment), of a CTA's share of rows x nv
    int race_slices;    // of the final row
    int race_len;       // its tokens per slice
    int margin;         // tokens at a row's ends that may lie in vectors it shares
    Stat* stats;        // part of row r by CTA c: [r + c]
    Best* best;         // [n_seq][race_slices]
    uint32_t* ticket;   // [n_seq]
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// the same in one instruction, below 2^-126 zero: for sums, and for races (some token has a probability of 1 / V)
__device__ __forceinline__ float ex2z(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// exp2(c (l - m)), 1 at the maximum itself
__device__ __forceinline__ float weight(float l, float m, float c) { return l == m ? 1.0f : ex2(c * (l - m)); }
__device__ __forceinline__ float usable(float l) { return l != l ? -INFINITY : l; }

__device__ __forceinline__ int64_t divide(int64_t x, int64_t y) {  // of non-negative numbers, most of them small
    return (x | y) >> 32 ? x / y : (int64_t)((uint32_t)x / (uint32_t)y);
}

__device__ __forceinline__ void join(float& m, float& s, float om, float os, float c) {
    const float M = fmaxf(m, om);
    if (M == -INFINITY) return;
    s = s * weight(m, M, c) + os * weight(om, M, c);
    m = M;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
template <typename T>
struct Elem;
template <>
struct Elem<float> {
    static constexpr int kVW = 4;
    static __device__ __forceinline__ float at(const uint4& v, int e) {
        return __uint_as_float(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w);
    }
    static __device__ __forceinline__ float get(const float* p) { return __ldg(p); }
    static __device__ __forceinline__ float value(float x) { return x; }
    template <int N>
    static __device__ __forceinline__ float largest(const uint4 (&x)[N], float m) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            m = max3(m, at(x[j], 0), at(x[j], 1));
            m = max3(m, at(x[j], 2), at(x[j], 3));
        }
        return m;
    }
};
template <>
struct Elem<__nv_bfloat16> {
    static constexpr int kVW = 8;
    static __device__ __forceinline__ float at(const uint4& v, int e) {
        const uint32_t w = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
        return __uint_as_float((e & 1) ? (w & 0xffff0000u) : (w << 16));
    }
    static __device__ __forceinline__ float get(const __nv_bfloat16* p) { return __bfloat162float(__ldg(p)); }
    static __device__ __forceinline__ float value(__nv_bfloat16 x) { return __bfloat162float(x); }
    // the largest logit of N vectors, and m; NaN is passed by
    template <int N>
    static __device__ __forceinline__ float largest(const uint4 (&x)[N], float m) {
        uint32_t h[2] = {0xff80ff80u, 0xff80ff80u};  // -inf
#pragma unroll
        for (int j = 0; j < N; ++j) {
            h[j & 1] = max2(max2(h[j & 1], x[j].x), x[j].y);
            h[j & 1] = max2(max2(h[j & 1], x[j].z), x[j].w);
        }
        h[0] = max2(h[0], h[1]);
        return max3(m, __uint_as_float(h[0] << 16), __uint_as_float(h[0] & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
};

__device__ __forceinline__ uint64_t pack2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// exp2(c (x - m)) of two logits.  (One product c x - c m would round c m: 6e-6 of the sum at logits of 100.)
__device__ __forceinline__ void weights2(float x0, float x1, uint64_t cc, uint64_t mm, float& w0, float& w1) {
    unpack2(mul2(add2(pack2(x0, x1), mm), cc), w0, w1);
    w0 = ex2z(w0);
    w1 = ex2z(w1);
}

// adds the logits of kVecs vectors to a running (max, sum)
template <typename T>
__device__ __forceinline__ void add_logits(const uint4 (&x)[kVecs], float& m, float& s, float c) {
    using E = Elem<T>;
    const float bm = E::largest(x, m);
    if (bm == -INFINITY) return;
    uint64_t sum[2] = {0, 0};
    const uint64_t cc = pack2(c, c), mm = pack2(-bm, -bm);
#pragma unroll
    for (int j = 0; j < kVecs; ++j)
#pragma unroll
        for (int e = 0; e < E::kVW; e += 2) {
            float w0, w1;
            weights2(E::at(x[j], e), E::at(x[j], e + 1), cc, mm, w0, w1);
            sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], pack2(w0, w1));
        }
    float bs, b1;
    unpack2(add2(sum[0], sum[1]), bs, b1);
    bs += b1;
    if (bs != bs) {  // NaN among the logits, or an infinite maximum
        bs = 0.0f;
#pragma unroll
        for (int j = 0; j < kVecs; ++j)
#pragma unroll
            for (int e = 0; e < E::kVW; ++e) bs += weight(usable(E::at(x[j], e)), bm, c);
    }
    s = fmaf(s, weight(m, bm, c), bs);
    m = bm;
}

// A part of a row as vectors: al, the aligned vector that holds its first token, `lead` tokens into it; vectors v0 .. v1 - 1 of
// it are a CTA's, of which lo .. hi - 1 lie wholly inside the row.
template <typename T>
struct RowPart {
    const T* al;
    int64_t row, end;  // end: in tokens from al
    int lead;
    int32_t v0, v1, lo, hi;
    __device__ __forceinline__ RowPart(const ChainArgs& a, const ChainPlan& P, int64_t x, int64_t x1) {
        constexpr int VW = Elem<T>::kVW;
        row = divide(x, P.nv);
        v0 = (int32_t)(x - row * P.nv);
        v1 = (int32_t)min(v0 + (x1 - x), P.nv);
        const T* base = row < a.n_nodes ? static_cast<const T*>(a.p) + row * a.p_stride
                                        : static_cast<const T*>(a.q) + (row - a.n_nodes) * a.q_stride;
        lead = (int)((reinterpret_cast<uintptr_t>(base) & 15) / sizeof(T));
        al = base - lead;
        end = a.V + lead;
        lo = max(v0, lead > 0 ? 1 : 0);
        hi = min(v1, (int32_t)(end / VW));
    }
};

template <typename T>
__global__ void __launch_bounds__(kThreads + 32, kStatCtas + 1) stats_kernel(const ChainArgs a, const ChainPlan P) {
    using E = Elem<T>;
    constexpr int VW = E::kVW, kChunkVecs = kVecs * kThreads;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ Stat sh[2][kThreads / 32];
    __shared__ __align__(8) uint64_t s_bar[2 * kStatStages];
    __shared__ volatile int s_abort;
    const uint32_t ring = smem_u32(smem), bars = smem_u32(s_bar);
    auto full = [&](uint32_t s) { return bars + 8u * s; };
    auto empty = [&](uint32_t s) { return bars + 8u * (kStatStages + s); };
    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStatStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), kThreads / 32);
        }
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < a.n_seq; i += kThreads + 32) P.ticket[i] = 0;
    if (a.out_prob)  // for the rows that no chain names; finish_kernel writes the others once this grid has ended
        for (int64_t i = (int64_t)blockIdx.x * (kThreads + 32) + threadIdx.x; i < a.n_draft; i += (int64_t)gridDim.x * (kThreads + 32))
            a.out_prob[i] = 0.0f;
    __syncthreads();
    const int64_t x1 = min((blockIdx.x + 1) * P.share, (a.n_nodes + a.n_draft) * P.nv);
    uint32_t it = 0;
    if (threadIdx.x >= kThreads) {
        if (threadIdx.x == kThreads) {
            for (int64_t x = blockIdx.x * P.share; x < x1;) {
                const RowPart<T> R(a, P, x, x1);
                x += R.v1 - R.v0;
                for (int32_t v = R.lo; v < R.hi && !s_abort; v += kChunkVecs, ++it) {
                    const uint32_t s = it % kStatStages, bytes = 16u * (uint32_t)min(R.hi - v, kChunkVecs);
                    if (!mbar_wait(empty(s), ((it / kStatStages) & 1u) ^ 1u, &s_abort)) break;
                    mbar_expect_tx(full(s), bytes);
                    bulk_load(ring + s * kStatChunk, R.al + (int64_t)v * VW, bytes, full(s));
                }
            }
            // copies in flight when the CTA gives up: wait (bounded) for each
            for (uint32_t i = it > (uint32_t)kStatStages ? it - kStatStages : 0u; i < it && s_abort; ++i)
                for (uint32_t n = 0; n < kDrainLimit && !mbar_try_wait(full(i % kStatStages), (i / kStatStages) & 1u); ++n) {
                }
        }
    } else {
        int turn = 0;
        for (int64_t x = blockIdx.x * P.share; x < x1; turn ^= 1) {  // (a wait that gives up leaves the order of barriers as it is)
            const RowPart<T> R(a, P, x, x1);
            x += R.v1 - R.v0;
            float m = -INFINITY, s = 0.0f;
            for (int32_t v = R.lo; v < R.hi; v += kChunkVecs, ++it) {
                const uint32_t st = it % kStatStages, n = (uint32_t)min(R.hi - v, kChunkVecs);
                mbar_wait(full(st), (it / kStatStages) & 1u, &s_abort);
                uint4 y[kVecs];
#pragma unroll
                for (int k = 0; k < kVecs; ++k) {
                    const uint32_t i = threadIdx.x + k * kThreads;
                    constexpr uint32_t none = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;  // -inf
                    y[k] = make_uint4(none, none, none, none);
                    if (i < n) y[k] = *reinterpret_cast<const uint4*>(smem + st * kStatChunk + i * 16);
                }
                __syncwarp();
                if ((threadIdx.x & 31) == 0) mbar_arrive(empty(st));
                add_logits<T>(y, m, s, a.c);
            }
            // the row's ends that are not whole vectors: at most two, a token per thread
            if (threadIdx.x < 2 * VW) {
                const int64_t v = threadIdx.x < VW ? 0 : R.end / VW, tok = v * VW + threadIdx.x % VW;
                const bool whole = threadIdx.x < VW ? R.lead == 0 && R.end >= VW : R.end % VW == 0 || R.end < VW;  // (of one vector: the first's)
                if (!whole && v >= R.v0 && v < R.v1 && tok >= R.lead && tok < R.end) join(m, s, usable(E::get(R.al + tok)), 1.0f, a.c);
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const float om = __shfl_xor_sync(0xffffffffu, m, o), os = __shfl_xor_sync(0xffffffffu, s, o);
                join(m, s, om, os, a.c);
            }
            if ((threadIdx.x & 31) == 0) sh[turn][threadIdx.x >> 5] = {m, s};
            asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
            if (threadIdx.x == 0) {
                for (int w = 1; w < kThreads / 32; ++w) join(m, s, sh[turn][w].m, sh[turn][w].s, a.c);
                P.stats[R.row + blockIdx.x] = {m, s};
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && s_abort && a.status) atomicOr(a.status, PPS_FLAG_TIMEOUT);
}

// a row's (max, sum), by one warp, in the same order for every reader
__device__ __forceinline__ Stat row_stat(const ChainPlan& P, int64_t row, float c, int lane) {
    float m = -INFINITY, s = 0.0f;
    const int64_t from = divide(row * P.nv, P.share), to = divide((row + 1) * P.nv - 1, P.share);
    for (int64_t j = from + lane; j <= to; j += 32) {
        const Stat t = P.stats[row + j];
        join(m, s, t.m, t.s, c);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float om = __shfl_xor_sync(0xffffffffu, m, o), os = __shfl_xor_sync(0xffffffffu, s, o);
        join(m, s, om, os, c);
    }
    return {m, s};
}

__device__ __forceinline__ void better(Best& b, float v, int i) {
    if (v > b.v || (v == b.v && i < b.i)) b = {v, i};
}
template <class Sync>
__device__ __forceinline__ Best block_best(Best b, Best* sh, Sync sync) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float v = __shfl_xor_sync(0xffffffffu, b.v, o);
        const int i = __shfl_xor_sync(0xffffffffu, b.i, o);
        better(b, v, i);
    }
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = b;
    sync();
    b = sh[0];
    for (int w = 1; w < kThreads / 32; ++w) better(b, sh[w].v, sh[w].i);
    sync();
    return b;
}

// One token's score max(P - Q, 0) / E from its logits (drafter: whether there is one) and noise
struct Law {
    Stat p, q;
    float c, ip, iq;
    bool drafter, finite;  // finite: both rows' maxima are
    __device__ __forceinline__ Law(const Stat& sp, const Stat& sq, bool has, float c_)
        : p(sp), q(sq), c(c_), ip(sp.s > 0.0f ? 1.0f / sp.s : 0.0f), iq(sq.s > 0.0f ? 1.0f / sq.s : 0.0f), drafter(has),
          finite(fabsf(sp.m) < INFINITY && (!has || fabsf(sq.m) < INFINITY)) {}
    // max(P - Q, 0) is the positive part of this
    __device__ __forceinline__ void excess(float (&x)[kRaceTok], const float (&y)[kRaceTok]) const {
        if (!finite) {
#pragma unroll
            for (int k = 0; k < kRaceTok; ++k) x[k] = excess(x[k], y[k]);
            return;
        }
        const uint64_t cc = pack2(c, c), mp = pack2(-p.m, -p.m), mq = pack2(-q.m, -q.m);
#pragma unroll
        for (int k = 0; k < kRaceTok; k += 2) {
            weights2(x[k], x[k + 1], cc, mp, x[k], x[k + 1]);
            x[k] *= ip;
            x[k + 1] *= ip;
            if (drafter) {
                float w0, w1;
                weights2(fmaxf(y[k], -INFINITY), fmaxf(y[k + 1], -INFINITY), cc, mq, w0, w1);
                x[k] = fmaf(w0, -iq, x[k]);
                x[k + 1] = fmaf(w1, -iq, x[k + 1]);
            }
        }
    }
    __device__ __forceinline__ float excess(float x, float y) const {
        if (!finite) {
            const float d = weight(usable(x), p.m, c) * ip;
            return drafter ? d - weight(usable(y), q.m, c) * iq : d;
        }
        const float d = ex2z((x - p.m) * c) * ip;  // NaN logits of the target's never win, those of the drafter's count as -inf
        return drafter ? fmaf(ex2z((fmaxf(y, -INFINITY) - q.m) * c), -iq, d) : d;
    }
};
// 8 consecutive values of a row in shared memory, the j-th 8
__device__ __forceinline__ void load8(float (&x)[kRaceTok], const uint8_t* row, int j, float) {
    *reinterpret_cast<float4*>(x) = reinterpret_cast<const float4*>(row)[2 * j];
    *reinterpret_cast<float4*>(x + 4) = reinterpret_cast<const float4*>(row)[2 * j + 1];
}
__device__ __forceinline__ void load8(float (&x)[kRaceTok], const uint8_t* row, int j, __nv_bfloat16) {
    const uint4 v = reinterpret_cast<const uint4*>(row)[j];
#pragma unroll
    for (int k = 0; k < kRaceTok; ++k) x[k] = Elem<__nv_bfloat16>::at(v, k);
}
// offers a token: it is looked at closely (the quotient, ties) only if it is not clearly below the best so far
__device__ __forceinline__ void offer(Best& b, float d, float z, int64_t tok) {
    if (d > 0.0f && d >= b.v * 0.999999f * z) better(b, d / z, (int)tok);
}

template <typename T>
__global__ void __launch_bounds__(kThreads + 32) finish_kernel(const ChainArgs a, const ChainPlan P) {
    using E = Elem<T>;
    using S = RaceSmem<T>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int s_row[kMaxChain], s_tok[kMaxChain], s_ok[kMaxChain];
    __shared__ Stat s_p[kMaxChain + 1], s_q[kMaxChain];
    __shared__ Best s_best[kThreads / 32];
    __shared__ int s_last, s_node, s_fr;
    __shared__ __align__(8) uint64_t s_bar[2 * kRaceStages];
    __shared__ volatile int s_abort;
    __shared__ volatile uint32_t s_high;  // bits of the best score any thread has seen (scores are not negative)
    const uint32_t ring = smem_u32(smem), bars = smem_u32(s_bar);
    auto full = [&](uint32_t s) { return bars + 8u * s; };
    auto empty = [&](uint32_t s) { return bars + 8u * (kRaceStages + s); };
    const int seq = (int)(blockIdx.x / (unsigned)P.race_slices), slice = (int)(blockIdx.x % (unsigned)P.race_slices);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, j = threadIdx.x;
    const int n0 = __ldg(a.seq_off + seq), n1 = __ldg(a.seq_off + seq + 1);
    if (n0 < 0 || n1 <= n0 || n1 > a.n_nodes) {  // CTA-uniform: nothing of the sequence can be read
        pdl_wait();  // a grid without one CTA that waits may end before the statistics do, whose workspace is then another's
        if (slice == 0 && j == 0) {
            a.out_acc[seq] = 0;
            a.out_ne[seq] = 0;
            for (int i = 0; i <= a.gamma; ++i) a.out_em[(int64_t)seq * (a.gamma + 1) + i] = -1;
            if (a.status) atomicOr(a.status, PPS_FLAG_INDEX);
        }
        return;
    }
    if (j == 0) {
        for (int s = 0; s < kRaceStages; ++s) {
            mbar_init(full(s), 2);  // the noise, the rows
            mbar_init(empty(s), kThreads / 32);
        }
        s_abort = 0;
        s_high = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    // The slice's tokens t0 .. t1 - 1; of them those from ta to tb - 1 lie in whole vectors of all three rows, whatever
    // rows of the logits these will be (their first and last 16 bytes are left out if any may be unaligned).
    const float* noise = a.noise + seq * a.noise_stride;
    const int64_t t0 = (int64_t)slice * P.race_len, t1 = min(t0 + P.race_len, a.V);
    const int64_t ta = max(t0, (int64_t)P.margin), tb = max(min(t1, a.V - P.margin), ta);
    const uint32_t chunks = (uint32_t)((tb - ta + kRaceChunk - 1) / kRaceChunk);
    // copies tokens t .. t + n - 1 of a row, from the vector that holds the first
    auto copy = [&](uint32_t dst, const void* row, uint32_t size, int64_t t, uint32_t n, uint32_t bar) {
        const uintptr_t from = (reinterpret_cast<uintptr_t>(row) + t * size) & ~(uintptr_t)15;
        const uintptr_t to = (reinterpret_cast<uintptr_t>(row) + (t + n) * size + 15) & ~(uintptr_t)15;
        bulk_load(dst, reinterpret_cast<const void*>(from), (uint32_t)(to - from), bar);
    };
    auto span = [&](const void* row, uint32_t size, int64_t t, uint32_t n) {
        const uintptr_t from = (reinterpret_cast<uintptr_t>(row) + t * size) & ~(uintptr_t)15;
        return (uint32_t)(((reinterpret_cast<uintptr_t>(row) + (t + n) * size + 15) & ~(uintptr_t)15) - from);
    };
    auto length = [&](uint32_t i) { return (uint32_t)min(tb - (ta + (int64_t)i * kRaceChunk), (int64_t)kRaceChunk); };
    if (threadIdx.x >= kThreads) {
        auto copy_noise = [&](uint32_t i) {
            const uint32_t s = i % kRaceStages;
            const int64_t t = ta + (int64_t)i * kRaceChunk;
            mbar_expect_tx(full(s), span(noise, 4, t, length(i)));
            copy(ring + s * S::kStage + 2 * S::kRow, noise, 4, t, length(i), full(s));
        };
        // the noise does not wait for the rows' sums
        if (lane == 0)
            for (uint32_t i = 0; i < min(chunks, (uint32_t)kRaceStages); ++i) copy_noise(i);
        __syncwarp();
        asm volatile("bar.sync 2, %0;" ::"n"(kThreads + 32) : "memory");  // the rows are known
        if (lane == 0) {
            const T* p = static_cast<const T*>(a.p) + s_node * a.p_stride;
            const T* q = s_fr >= 0 ? static_cast<const T*>(a.q) + s_fr * a.q_stride : nullptr;
            uint32_t rows = 0;
            for (; rows < chunks && !s_abort; ++rows) {
                const uint32_t s = rows % kRaceStages, n = length(rows);
                const int64_t t = ta + (int64_t)rows * kRaceChunk;
                if (rows >= (uint32_t)kRaceStages) {
                    if (!mbar_wait(empty(s), ((rows / kRaceStages) & 1u) ^ 1u, &s_abort)) break;
                    copy_noise(rows);
                }
                mbar_expect_tx(full(s), span(p, sizeof(T), t, n) + (q != nullptr ? span(q, sizeof(T), t, n) : 0u));
                copy(ring + s * S::kStage, p, sizeof(T), t, n, full(s));
                if (q != nullptr) copy(ring + s * S::kStage + S::kRow, q, sizeof(T), t, n, full(s));
            }
            // copies in flight when the CTA gives up: wait (bounded) for each
            for (uint32_t i = rows > (uint32_t)kRaceStages ? rows - kRaceStages : 0u; i < rows && s_abort; ++i)
                for (uint32_t n = 0; n < kDrainLimit && !mbar_try_wait(full(i % kRaceStages), (i / kRaceStages) & 1u); ++n) {
                }
        }
    } else {
        // the chain's tokens and their logits do not wait for the sums either
        const int longest = min(n1 - n0 - 1, a.gamma);
        int r = -1;
        float u = 0.0f, lp = -INFINITY, lq = -INFINITY;
        if (j < longest) {
            r = __ldg(a.node_draft_row + n0 + j);
            bool bad = r >= a.n_draft;
            if (r < 0 || bad) r = -1;
            int tok = -1;
            if (r >= 0) {
                tok = __ldg(a.draft_tok + r);
                u = __ldg(a.u + r);
                if (tok < 0 || tok >= a.V)
                    bad = true;
                else {
                    lp = usable(E::get(static_cast<const T*>(a.p) + (n0 + j) * a.p_stride + tok));
                    lq = usable(E::get(static_cast<const T*>(a.q) + r * a.q_stride + tok));
                }
            }
            s_row[j] = r;
            s_tok[j] = tok;
            if (bad && slice == 0 && a.status) atomicOr(a.status, PPS_FLAG_INDEX);
        }
        auto sync = [] { asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory"); };
        sync();
        pdl_wait();
        for (int i = warp; i < 2 * longest + 1; i += kThreads / 32) {  // the chain's rows, the drafter's after the target's
            const bool is_q = i > longest;
            const int64_t row = is_q ? (s_row[i - longest - 1] >= 0 ? a.n_nodes + s_row[i - longest - 1] : -1) : (int64_t)n0 + i;
            const Stat st = row >= 0 ? row_stat(P, row, a.c, lane) : Stat{-INFINITY, 0.0f};
            if (lane == 0) (is_q ? s_q[i - longest - 1] : s_p[i]) = st;
        }
        sync();
        if (j < longest) {
            // a token out of range has no logit: it counts as impossible under both laws
            const Stat sp = s_p[j], sq = s_q[j];
            const float px = lp > -INFINITY && sp.s > 0.0f ? weight(lp, sp.m, a.c) / sp.s : 0.0f;
            const float qx = lq > -INFINITY && sq.s > 0.0f ? weight(lq, sq.m, a.c) / sq.s : 0.0f;
            s_ok[j] = r >= 0 && u * qx < px;
            if (r >= 0 && slice == 0 && a.out_prob) a.out_prob[r] = px > 0.0f ? (px < qx ? px / qx : 1.0f) : 0.0f;
        }
        sync();
        int acc = 0;
        while (acc < longest && s_ok[acc]) ++acc;
        const int node = n0 + acc;
        int fr = acc < longest ? s_row[acc] : -1;
        if (fr >= 0 && !(s_q[acc].s > 0.0f)) fr = -1;  // a drafter without mass
        if (j == 0) {
            s_node = node;
            s_fr = fr;
        }
        asm volatile("bar.sync 2, %0;" ::"n"(kThreads + 32) : "memory");
        const Law law(s_p[acc], fr >= 0 ? s_q[acc] : Stat{0.0f, 0.0f}, fr >= 0, a.c);
        const T* p = static_cast<const T*>(a.p) + node * a.p_stride;
        const T* q = static_cast<const T*>(a.q) + (fr >= 0 ? fr : 0) * a.q_stride;
        Best b = {0.0f, INT_MAX};  // only positive scores count; a row without mass has none
        const uint32_t skip_p = (uint32_t)((reinterpret_cast<uintptr_t>(p + ta) & 15) / sizeof(T));
        const uint32_t skip_q = (uint32_t)((reinterpret_cast<uintptr_t>(q + ta) & 15) / sizeof(T));
        const uint32_t skip_z = (uint32_t)((reinterpret_cast<uintptr_t>(noise + ta) & 15) / 4);
        for (uint32_t i = 0; i < chunks; ++i) {
            const uint32_t s = i % kRaceStages, n = length(i);
            const int64_t t = ta + (int64_t)i * kRaceChunk;
            mbar_wait(full(s), (i / kRaceStages) & 1u, &s_abort);
            const uint8_t* stage = smem + s * S::kStage;
            const T* xs = reinterpret_cast<const T*>(stage) + skip_p;
            const T* ys = reinterpret_cast<const T*>(stage + S::kRow) + skip_q;
            const float* zs = reinterpret_cast<const float*>(stage + 2 * S::kRow) + skip_z;
            if (law.p.s > 0.0f) {
                // All scores side by side, then one test for any that comes near the CTA's best so far (a thread's own best is
                // beaten too often: some lane of a warp would divide in every chunk).  Thread j has tokens 8 j .. 8 j + 7 of
                // an aligned chunk, else j, j + 256 and so on.
                float x[kRaceTok], y[kRaceTok], z[kRaceTok];
                const bool wide = P.margin == 0 && n == (uint32_t)kRaceChunk;  // CTA-uniform
                if (wide) {
                    load8(x, stage, j, T());
                    if (law.drafter) load8(y, stage + S::kRow, j, T());
                    load8(z, stage + 2 * S::kRow, j, 0.0f);
                } else {
#pragma unroll
                    for (int k = 0; k < kRaceTok; ++k) {
                        const uint32_t e = (uint32_t)j + k * kThreads;
                        x[k] = -INFINITY;
                        y[k] = z[k] = 0.0f;
                        if (e < n) {
                            x[k] = E::value(xs[e]);
                            if (law.drafter) y[k] = E::value(ys[e]);
                            z[k] = zs[e];
                        }
                    }
                }
                law.excess(x, y);
                const float low = fmaxf(b.v, __uint_as_float(s_high)) * 0.999999f;
                bool near = false;
#pragma unroll
                for (int k = 0; k < kRaceTok; ++k) near = near || x[k] >= low * z[k];
                if (near) {
#pragma unroll
                    for (int k = 0; k < kRaceTok; ++k)
                        if (x[k] > 0.0f && x[k] >= low * z[k]) better(b, x[k] / z[k], (int)(t + (wide ? kRaceTok * j + k : j + k * kThreads)));
                    atomicMax(const_cast<uint32_t*>(&s_high), __float_as_uint(b.v));
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty(s));
        }
        // the slice's tokens outside the whole vectors
        auto single = [&](int64_t t) { offer(b, law.excess(E::get(p + t), law.drafter ? E::get(q + t) : 0.0f), __ldg(noise + t), t); };
        if (law.p.s > 0.0f) {
            if (t0 + j < min(ta, t1)) single(t0 + j);
            if (max(tb, t0) + j < t1 && max(tb, t0) + j >= ta) single(max(tb, t0) + j);
        }
        b = block_best(b, s_best, sync);
        if (j == 0) {
            __stcg(reinterpret_cast<float2*>(P.best + (int64_t)seq * P.race_slices + slice), make_float2(b.v, __int_as_float(b.i)));
            __threadfence();
            s_last = atomicAdd(P.ticket + seq, 1u) == (unsigned)P.race_slices - 1;
        }
        sync();
        if (s_last) {
            __threadfence();
            b = {0.0f, INT_MAX};
            if (j < P.race_slices) {
                const float2 o = __ldcg(reinterpret_cast<const float2*>(P.best + (int64_t)seq * P.race_slices + j));
                b = {o.x, __float_as_int(o.y)};
            }
            b = block_best(b, s_best, sync);
            if (b.i == INT_MAX && law.drafter && law.p.s > 0.0f) {  // the residual is zero everywhere (CTA-uniform): P itself
                const Law whole(law.p, law.q, false, a.c);
                for (int64_t t = j; t < a.V; t += kThreads) offer(b, whole.excess(E::get(p + t), 0.0f), __ldg(noise + t), t);
                b = block_best(b, s_best, sync);
            }
            if (j <= a.gamma)
                a.out_em[(int64_t)seq * (a.gamma + 1) + j] = j < acc ? s_tok[j] : j == acc && b.i != INT_MAX ? b.i : -1;
            if (j == 0) {
                a.out_acc[seq] = acc;
                a.out_ne[seq] = acc + (b.i != INT_MAX);
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && s_abort && a.status) atomicOr(a.status, PPS_FLAG_TIMEOUT);
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

template <typename T>
cudaError_t launch(const ChainArgs& a, cudaStream_t st) {
    ChainPlan P;
    const int64_t rows = a.n_nodes + a.n_draft;
    const int sms = device_sm_count();
    P.nv = (a.V + Elem<T>::kVW - 1) / Elem<T>::kVW + 1;
    // every CTA resident at once, of a vector a thread at least
    const int64_t most = std::min<int64_t>(kMaxParts, (int64_t)kStatCtas * sms);
    P.share = std::max<int64_t>((rows * P.nv + most - 1) / most, kThreads);
    const unsigned ctas = (unsigned)((rows * P.nv + P.share - 1) / P.share);
    // the final rows: every CTA resident at once, of a chunk at least (64 sequences, V = 128256: 61 us with one CTA per SM, 51
    // with two, 47.5 with three)
    using S = RaceSmem<T>;
    const int64_t n = std::min<int64_t>((a.V + kRaceChunk - 1) / kRaceChunk, std::max<int64_t>(1, S::kCtas * sms / a.n_seq));
    P.race_slices = (int)std::min<int64_t>(std::max<int64_t>(n, 1), kMaxSlices);
    P.race_len = (int)(((a.V + P.race_slices - 1) / P.race_slices + 7) / 8 * 8);
    const uint64_t bits = reinterpret_cast<uintptr_t>(a.p) | reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.noise) |
                          (uint64_t)(a.p_stride | a.q_stride | a.V) * sizeof(T) | (uint64_t)(a.noise_stride | a.V) * 4;
    P.margin = bits % 16 == 0 ? 0 : 8;
    char* w = static_cast<char*>(a.ws);
    P.stats = reinterpret_cast<Stat*>(w);
    w += align256(sizeof(Stat) * (size_t)(rows + kMaxParts));
    P.best = reinterpret_cast<Best*>(w);
    w += align256(sizeof(Best) * (size_t)a.n_seq * kMaxSlices);
    P.ticket = reinterpret_cast<uint32_t*>(w);
    if ((int64_t)a.n_seq * P.race_slices > INT32_MAX) return cudaErrorInvalidValue;
    static std::atomic<uint64_t> stats_ready{0}, finish_ready{0};
    cudaError_t e = allow_smem(stats_ready, (const void*)stats_kernel<T>, kStatSmem);
    if (e != cudaSuccess) return e;
    e = allow_smem(finish_ready, (const void*)finish_kernel<T>, S::kBytes);
    if (e != cudaSuccess) return e;
    stats_kernel<T><<<ctas, kThreads + 32, kStatSmem, st>>>(a, P);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_pdl(finish_kernel<T>, dim3((unsigned)(a.n_seq * P.race_slices)), dim3(kThreads + 32), S::kBytes, st, a, P);
}

}  // namespace

size_t chain_workspace_bytes(int64_t n_nodes, int64_t n_draft, int n_seq) {
    return align256(sizeof(Stat) * (size_t)(n_nodes + n_draft + kMaxParts)) +
           align256(sizeof(Best) * (size_t)n_seq * kMaxSlices) + align256(sizeof(uint32_t) * (size_t)n_seq);
}

cudaError_t launch_chain(const ChainArgs& a, int dtype, cudaStream_t stream) {
    return dtype == PPS_BF16 ? launch<__nv_bfloat16>(a, stream) : launch<float>(a, stream);
}

}  // namespace pps
