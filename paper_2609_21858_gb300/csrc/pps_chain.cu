// pps_chain.cu -- verification of drafted chains by the token-level maximal coupling (Alg. 1).
//
// With P = softmax(p / T) and Q = softmax(q / T), the drafted token x of a node is accepted iff
// u Q(x) < P(x); at the first rejection the emitted token is argmax_i max(P(i) - Q(i), 0) / E(i), past
// the chain argmax_i P(i) / E(i).  exp2 of c (l - max) with c = log2(e) / T stands for exp(l / T) throughout;
// a logit equal to its row's maximum counts as 1 also where both are infinite.
//
// Two launches, both bound by HBM.  stats_kernel reads every logit once: the rows' 16-byte vectors lie on one line
// that is cut into equal shares, one per CTA, and a CTA leaves (max, sum of exponentials) of each row it meets.  A thread
// takes kVecs vectors at a time, the next ones on their way: their maximum first, then their exponentials against it.
// finish_kernel runs slices x sequences: each CTA joins the parts of its chain's rows, finds the first rejection and races
// its slice of the one row (pair) that matters; the CTA that arrives last at the sequence's ticket joins the slices in
// order and writes the outputs.
#include <algorithm>
#include <climits>
#include <cstdint>

#include <cuda_bf16.h>

#include "pps.h"
#include "pps_internal.h"

namespace pps {
namespace {

constexpr int kStatThreads = 256, kStatCtas = 4;  // CTAs per SM
constexpr int kVecs = 4;         // 16-byte vectors per thread and turn
constexpr int kRaceThreads = 256, kRaceCtas = 4;
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

__device__ __forceinline__ void join(float& m, float& s, float om, float os, float c) {
    const float M = fmaxf(m, om);
    if (M == -INFINITY) return;
    s = s * weight(m, M, c) + os * weight(om, M, c);
    m = M;
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
};
template <>
struct Elem<__nv_bfloat16> {
    static constexpr int kVW = 8;
    static __device__ __forceinline__ float at(const uint4& v, int e) {
        const uint32_t w = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
        return __uint_as_float((e & 1) ? (w & 0xffff0000u) : (w << 16));
    }
    static __device__ __forceinline__ float get(const __nv_bfloat16* p) { return __bfloat162float(__ldg(p)); }
};

__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
// c (x0 - m) and c (x1 - m) at once.  (One product c x - c m would round c m: 6e-6 of the sum at logits of 100.)
__device__ __forceinline__ void scale2(float& x0, float& x1, float c, float m) {
    uint64_t x, cc, mm;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(x0), "f"(x1));
    asm("mov.b64 %0, {%1, %1};" : "=l"(cc) : "f"(c));
    asm("mov.b64 %0, {%1, %1};" : "=l"(mm) : "f"(-m));
    asm("add.rn.f32x2 %0, %0, %1;" : "+l"(x) : "l"(mm));
    asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(x) : "l"(cc));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x0), "=f"(x1) : "l"(x));
}

// one vector of a row seen as the aligned 16-byte vectors that cover it (al: the first one); its first and last one may
// hold tokens of no concern, and are read token by token
template <typename T>
__device__ __forceinline__ uint4 row_vec(const T* al, int64_t v, int lead, int64_t end) {
    using E = Elem<T>;
    constexpr int VW = E::kVW;
    if (v * VW >= lead && (v + 1) * VW <= end) return __ldg(reinterpret_cast<const uint4*>(al) + v);
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;  // -inf
#pragma unroll
    for (int e = 0; e < VW; ++e) {
        const int64_t t = v * VW + e;
        if (t >= lead && t < end) {
            const uint32_t f = __float_as_uint(E::get(al + t));
            if constexpr (sizeof(T) == 2)
                w[e >> 1] = (e & 1) ? ((w[e >> 1] & 0xffffu) | (f & 0xffff0000u)) : ((w[e >> 1] & 0xffff0000u) | (f >> 16));
            else
                w[e] = f;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// adds the logits of kVecs vectors to a running (max, sum)
template <typename T>
__device__ __forceinline__ void add_logits(const uint4 (&x)[kVecs], float& m, float& s, float c) {
    using E = Elem<T>;
    float bm = m;
#pragma unroll
    for (int j = 0; j < kVecs; ++j)
#pragma unroll
        for (int e = 0; e < E::kVW; e += 2) bm = max3(bm, E::at(x[j], e), E::at(x[j], e + 1));  // NaN is passed by
    if (bm == -INFINITY) return;
    float bs = 0.0f, b1 = 0.0f;
#pragma unroll
    for (int j = 0; j < kVecs; ++j)
#pragma unroll
        for (int e = 0; e < E::kVW; e += 2) {
            float x0 = E::at(x[j], e), x1 = E::at(x[j], e + 1);
            scale2(x0, x1, c, bm);
            bs += ex2z(x0);
            b1 += ex2z(x1);
        }
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

template <typename T>
__global__ void __launch_bounds__(kStatThreads, kStatCtas) stats_kernel(const ChainArgs a, const ChainPlan P) {
    constexpr int VW = Elem<T>::kVW;
    __shared__ Stat sh[2][kStatThreads / 32];
    pdl_launch_dependents();
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < a.n_seq; i += kStatThreads) P.ticket[i] = 0;
    int64_t x = blockIdx.x * P.share;
    const int64_t x1 = min(x + P.share, (a.n_nodes + a.n_draft) * P.nv);
    for (int turn = 0; x < x1; turn ^= 1) {  // one row, or a part of it, at a time
        const int64_t row = x / P.nv, v0 = x - row * P.nv, v1 = min(v0 + (x1 - x), P.nv);
        x += v1 - v0;
        const T* base = row < a.n_nodes ? static_cast<const T*>(a.p) + row * a.p_stride
                                        : static_cast<const T*>(a.q) + (row - a.n_nodes) * a.q_stride;
        const int lead = (int)((reinterpret_cast<uintptr_t>(base) & 15) / sizeof(T));  // tokens of the first vector before the row
        const T* al = base - lead;
        const int64_t end = a.V + lead;  // in tokens from al
        const int64_t last = min(v1, (end + VW - 1) / VW);
        auto fetch = [&](uint4 (&y)[kVecs], int64_t b) {
#pragma unroll
            for (int j = 0; j < kVecs; ++j) {
                const int64_t v = b + j * kStatThreads;
                y[j] = v < last ? row_vec<T>(al, v, lead, end) : make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
                if (sizeof(T) == 4 && v >= last) y[j] = make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u);
            }
        };
        float m = -INFINITY, s = 0.0f;
        uint4 cur[kVecs], nxt[kVecs];
        int64_t b = v0 + threadIdx.x;
        fetch(cur, b);
        for (; b < last; b += kVecs * kStatThreads) {
            fetch(nxt, b + kVecs * kStatThreads);
            add_logits<T>(cur, m, s, a.c);
#pragma unroll
            for (int j = 0; j < kVecs; ++j) cur[j] = nxt[j];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float om = __shfl_xor_sync(0xffffffffu, m, o), os = __shfl_xor_sync(0xffffffffu, s, o);
            join(m, s, om, os, a.c);
        }
        if ((threadIdx.x & 31) == 0) sh[turn][threadIdx.x >> 5] = {m, s};
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kStatThreads / 32; ++w) join(m, s, sh[turn][w].m, sh[turn][w].s, a.c);
            P.stats[row + blockIdx.x] = {m, s};
        }
    }
}

// a row's (max, sum), by one warp, in the same order for every reader
__device__ __forceinline__ Stat row_stat(const ChainPlan& P, int64_t row, float c, int lane) {
    float m = -INFINITY, s = 0.0f;
    const int64_t from = row * P.nv / P.share, to = ((row + 1) * P.nv - 1) / P.share;
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
__device__ __forceinline__ Best block_best(Best b, Best* sh) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float v = __shfl_xor_sync(0xffffffffu, b.v, o);
        const int i = __shfl_xor_sync(0xffffffffu, b.i, o);
        better(b, v, i);
    }
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = b;
    __syncthreads();
    b = sh[0];
    for (int w = 1; w < kRaceThreads / 32; ++w) better(b, sh[w].v, sh[w].i);
    __syncthreads();
    return b;
}

// the 8 tokens from t of a row, widest loads its address allows; past the end: -inf (or 0)
template <typename T>
__device__ __forceinline__ void load8(float (&x)[8], const T* row, int64_t t, int64_t V, float none) {
    using E = Elem<T>;
    const T* p = row + t;
    if (t + 8 <= V && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll
        for (int k = 0; k < 8 / E::kVW; ++k) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(p) + k);
#pragma unroll
            for (int e = 0; e < E::kVW; ++e) x[k * E::kVW + e] = E::at(v, e);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = t + e < V ? E::get(p + e) : none;
    }
}

// the best of tokens [t0, t1) of max(P - Q, 0) / E (q == nullptr: P / E), as this thread's share; z: the noise of its first 8
template <typename T>
__device__ __forceinline__ Best race(const T* p, const T* q, const float* noise, float (&z)[8], Stat sp, Stat sq, float c,
                                     int64_t t0, int64_t t1, int64_t V) {
    Best b = {0.0f, INT_MAX};  // only positive scores count
    const float ip = sp.s > 0.0f ? 1.0f / sp.s : 0.0f, iq = sq.s > 0.0f ? 1.0f / sq.s : 0.0f;
    const bool finite = fabsf(sp.m) < INFINITY && (q == nullptr || fabsf(sq.m) < INFINITY);  // CTA-uniform
    float x[8], y[8];
    int64_t t = t0 + 8 * threadIdx.x;
    if (t < t1) {
        load8(x, p, t, V, -INFINITY);
        if (q != nullptr) load8(y, q, t, V, -INFINITY);
    }
    while (t < t1) {
        float xn[8], yn[8], zn[8], d[8];
        const int64_t tn = t + 8 * kRaceThreads;
        if (tn < t1) {
            load8(xn, p, tn, V, -INFINITY);
            if (q != nullptr) load8(yn, q, tn, V, -INFINITY);
            load8(zn, noise, tn, V, 1.0f);
        }
        if (finite) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                scale2(x[e], x[e + 1], c, sp.m);
                d[e] = ex2z(x[e]) * ip;
                d[e + 1] = ex2z(x[e + 1]) * ip;
                if (q != nullptr) {
                    scale2(y[e], y[e + 1], c, sq.m);
                    d[e] = fmaf(ex2z(fmaxf(y[e], -INFINITY)), -iq, d[e]);  // a NaN logit of the drafter's counts as -inf
                    d[e + 1] = fmaf(ex2z(fmaxf(y[e + 1], -INFINITY)), -iq, d[e + 1]);
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                d[e] = weight(usable(x[e]), sp.m, c) * ip;
                if (q != nullptr) d[e] -= weight(usable(y[e]), sq.m, c) * iq;
            }
        }
        // a token is looked at closely (the quotient, ties) only if it is not clearly below the best so far
        const float low = b.v * 0.999999f;
        uint32_t near = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (d[e] > 0.0f && !(d[e] < low * z[e])) near |= 1u << e;
        if (near)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if ((near >> e & 1u) && t + e < t1) better(b, d[e] / z[e], (int)(t + e));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = xn[e];
            y[e] = yn[e];
            z[e] = zn[e];
        }
        t = tn;
    }
    return b;
}

template <typename T>
__global__ void __launch_bounds__(kRaceThreads, kRaceCtas) finish_kernel(const ChainArgs a, const ChainPlan P) {
    using E = Elem<T>;
    __shared__ int s_row[kMaxChain], s_tok[kMaxChain], s_ok[kMaxChain];
    __shared__ Stat s_p[kMaxChain + 1], s_q[kMaxChain];
    __shared__ Best s_best[kRaceThreads / 32];
    __shared__ int s_last;
    const int seq = (int)(blockIdx.x / (unsigned)P.race_slices), slice = (int)(blockIdx.x % (unsigned)P.race_slices);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, j = threadIdx.x;
    const int64_t t0 = (int64_t)slice * P.race_len, t1 = min(t0 + P.race_len, a.V);
    const float* noise = a.noise + seq * a.noise_stride;
    // what does not wait for the rows' sums: the slice's first noise, the chain's tokens and their logits
    float z[8];
    if (t0 + 8 * j < t1) load8(z, noise, t0 + 8 * j, a.V, 1.0f);
    const int n0 = __ldg(a.seq_off + seq), n1 = __ldg(a.seq_off + seq + 1);
    if (n0 < 0 || n1 <= n0 || n1 > a.n_nodes) {  // CTA-uniform: nothing of the sequence can be read
        if (slice == 0 && j == 0) {
            a.out_acc[seq] = 0;
            a.out_ne[seq] = 0;
            for (int i = 0; i <= a.gamma; ++i) a.out_em[(int64_t)seq * (a.gamma + 1) + i] = -1;
            if (a.status) atomicOr(a.status, PPS_FLAG_INDEX);
        }
        return;
    }
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
    __syncthreads();
    pdl_wait();
    for (int i = warp; i < 2 * longest + 1; i += kRaceThreads / 32) {  // the chain's rows, the drafter's after the target's
        const bool is_q = i > longest;
        const int64_t row = is_q ? (s_row[i - longest - 1] >= 0 ? a.n_nodes + s_row[i - longest - 1] : -1) : (int64_t)n0 + i;
        const Stat st = row >= 0 ? row_stat(P, row, a.c, lane) : Stat{-INFINITY, 0.0f};
        if (lane == 0) (is_q ? s_q[i - longest - 1] : s_p[i]) = st;
    }
    __syncthreads();
    if (j < longest) {
        // a token out of range has no logit: it counts as impossible under both laws
        const Stat sp = s_p[j], sq = s_q[j];
        const float px = lp > -INFINITY && sp.s > 0.0f ? weight(lp, sp.m, a.c) / sp.s : 0.0f;
        const float qx = lq > -INFINITY && sq.s > 0.0f ? weight(lq, sq.m, a.c) / sq.s : 0.0f;
        s_ok[j] = r >= 0 && u * qx < px;
        if (r >= 0 && slice == 0 && a.out_prob) a.out_prob[r] = px > 0.0f ? (px < qx ? px / qx : 1.0f) : 0.0f;
    }
    __syncthreads();
    int acc = 0;
    while (acc < longest && s_ok[acc]) ++acc;
    const int node = n0 + acc, fr = acc < longest ? s_row[acc] : -1;
    const Stat sp = s_p[acc], sq = fr >= 0 ? s_q[acc] : Stat{0.0f, 0.0f};
    const T* p = static_cast<const T*>(a.p) + node * a.p_stride;
    const T* q = fr >= 0 && sq.s > 0.0f ? static_cast<const T*>(a.q) + fr * a.q_stride : nullptr;
    Best b = {0.0f, INT_MAX};
    if (sp.s > 0.0f) b = race(p, q, noise, z, sp, sq, a.c, t0, t1, a.V);
    b = block_best(b, s_best);
    if (threadIdx.x == 0) {
        __stcg(reinterpret_cast<float2*>(P.best + (int64_t)seq * P.race_slices + slice), make_float2(b.v, __int_as_float(b.i)));
        __threadfence();
        s_last = atomicAdd(P.ticket + seq, 1u) == (unsigned)P.race_slices - 1;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    b = {0.0f, INT_MAX};
    if (j < P.race_slices) {
        const float2 o = __ldcg(reinterpret_cast<const float2*>(P.best + (int64_t)seq * P.race_slices + j));
        b = {o.x, __float_as_int(o.y)};
    }
    b = block_best(b, s_best);
    if (b.i == INT_MAX && q != nullptr && sp.s > 0.0f) {  // the residual is zero everywhere (CTA-uniform)
        if (8 * j < a.V) load8(z, noise, 8 * j, a.V, 1.0f);
        b = block_best(race<T>(p, nullptr, noise, z, sp, sq, a.c, 0, a.V, a.V), s_best);
    }
    if (j <= a.gamma)
        a.out_em[(int64_t)seq * (a.gamma + 1) + j] = j < acc ? s_tok[j] : j == acc && b.i != INT_MAX ? b.i : -1;
    if (j == 0) {
        a.out_acc[seq] = acc;
        a.out_ne[seq] = acc + (b.i != INT_MAX);
    }
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
    P.share = std::max<int64_t>((rows * P.nv + most - 1) / most, kStatThreads);
    const unsigned ctas = (unsigned)((rows * P.nv + P.share - 1) / P.share);
    // the final rows: every CTA resident at once, of 8 tokens a thread at least
    const int64_t n = std::min<int64_t>((a.V + 8 * kRaceThreads - 1) / (8 * kRaceThreads), std::max<int64_t>(1, kRaceCtas * sms / a.n_seq));
    P.race_slices = (int)std::min<int64_t>(std::max<int64_t>(n, 1), kMaxSlices);
    P.race_len = (int)(((a.V + P.race_slices - 1) / P.race_slices + 7) / 8 * 8);
    char* w = static_cast<char*>(a.ws);
    P.stats = reinterpret_cast<Stat*>(w);
    w += align256(sizeof(Stat) * (size_t)(rows + kMaxParts));
    P.best = reinterpret_cast<Best*>(w);
    w += align256(sizeof(Best) * (size_t)a.n_seq * kMaxSlices);
    P.ticket = reinterpret_cast<uint32_t*>(w);
    if ((int64_t)a.n_seq * P.race_slices > INT32_MAX) return cudaErrorInvalidValue;
    stats_kernel<T><<<ctas, kStatThreads, 0, st>>>(a, P);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_pdl(finish_kernel<T>, dim3((unsigned)(a.n_seq * P.race_slices)), dim3(kRaceThreads), 0, st, a, P);
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
