// pps_chain.cu -- verification of drafted chains by the token-level maximal coupling (Alg. 1).
//
// With P = softmax(p / T) and Q = softmax(q / T), the drafted token x of a node is accepted iff
// u Q(x) < P(x); at the first rejection the emitted token is argmax_i max(P(i) - Q(i), 0) / E(i), past
// the chain argmax_i P(i) / E(i).  exp2 of c (l - max) with c = log2(e) / T stands for exp(l / T) throughout;
// a logit equal to its row's maximum counts as 1 also where both are infinite.
//
// Two launches.  stats_kernel reads every logit once: a CTA takes one slice of one row, each thread up to
// kVecs 16-byte vectors in registers, their maximum first and then their sum of exponentials, and the
// CTA leaves (max, sum).  finish_kernel runs slices x sequences: each CTA merges the sums of its chain's rows (a
// warp a row), finds the first rejection, and races its slice of the one row (pair) that matters; the CTA
// that arrives last at the sequence's ticket joins the slices in order and writes the outputs.  Both are
// bound by HBM: all logits once, then one row pair and the noise per sequence.
#include <algorithm>
#include <climits>
#include <cstdint>

#include <cuda_bf16.h>

#include "pps.h"
#include "pps_internal.h"

namespace pps {
namespace {

constexpr int kStatThreads = 256;
constexpr int kVecs = 8;         // 16-byte vectors per thread of a slice
constexpr int kMaxSlices = 64;   // of a row
constexpr int kRaceThreads = 256;
constexpr int kMaxChain = 64;    // gamma

struct Stat {
    float m, s;  // the slice's largest logit (-inf: none) and its sum of exp2(c (l - m))
};
struct Best {
    float v;
    int i;  // INT_MAX: none
};

struct ChainPlan {
    int slices;       // of a row in stats_kernel
    int vecs;         // 16-byte vectors per slice
    int race_slices;  // of the final row
    int race_len;     // its tokens per slice
    Stat* stats;      // [n_nodes + n_draft][slices]
    Best* best;       // [n_seq][race_slices]
    uint32_t* ticket; // [n_seq]
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
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

// (max, sum) of one slice of one row.  The row is seen as the aligned 16-byte vectors that cover it; its first
// and last one may hold tokens of no concern, and are read token by token.
template <typename T>
__global__ void __launch_bounds__(kStatThreads) stats_kernel(const ChainArgs a, const ChainPlan P) {
    using E = Elem<T>;
    constexpr int VW = E::kVW;
    __shared__ float sm[kStatThreads / 32], ss[kStatThreads / 32];
    const int64_t row = blockIdx.x / (unsigned)P.slices;
    const int slice = (int)(blockIdx.x % (unsigned)P.slices);
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < a.n_seq; i += kStatThreads) P.ticket[i] = 0;
    const T* base = row < a.n_nodes ? static_cast<const T*>(a.p) + row * a.p_stride
                                    : static_cast<const T*>(a.q) + (row - a.n_nodes) * a.q_stride;
    const int lead = (int)((reinterpret_cast<uintptr_t>(base) & 15) / sizeof(T));  // tokens of the first vector before the row
    const T* al = base - lead;
    const int64_t end = a.V + lead;  // in tokens from al
    const int64_t v0 = (int64_t)slice * P.vecs, v1 = min(v0 + P.vecs, (end + VW - 1) / VW);
    float m = -INFINITY, s = 0.0f;
    for (int64_t b = v0; b < v1; b += kVecs * kStatThreads) {  // one turn, unless the row has more than kMaxSlices full slices
        uint4 x[kVecs];
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int64_t v = b + threadIdx.x + j * kStatThreads;
            if (v < v1 && v * VW >= lead && (v + 1) * VW <= end)
                x[j] = __ldg(reinterpret_cast<const uint4*>(al) + v);
            else {
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;  // -inf
                if (v < v1) {
#pragma unroll
                    for (int e = 0; e < VW; ++e) {
                        const int64_t t = v * VW + e;
                        if (t >= lead && t < end) {
                            const uint32_t f = __float_as_uint(E::get(al + t));
                            if constexpr (sizeof(T) == 2)
                                w[e >> 1] = (e & 1) ? ((w[e >> 1] & 0xffffu) | (f & 0xffff0000u))
                                                    : ((w[e >> 1] & 0xffff0000u) | (f >> 16));
                            else
                                w[e] = f;
                        }
                    }
                }
                x[j] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        float bm = -INFINITY;
#pragma unroll
        for (int j = 0; j < kVecs; ++j)
#pragma unroll
            for (int e = 0; e < VW; ++e) bm = fmaxf(bm, E::at(x[j], e));  // fmaxf passes NaN by
        if (bm == -INFINITY) continue;
        float bs = 0.0f;
#pragma unroll
        for (int j = 0; j < kVecs; ++j)
#pragma unroll
            for (int e = 0; e < VW; ++e) bs += weight(usable(E::at(x[j], e)), bm, a.c);
        join(m, s, bm, bs, a.c);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float om = __shfl_xor_sync(0xffffffffu, m, o), os = __shfl_xor_sync(0xffffffffu, s, o);
        join(m, s, om, os, a.c);
    }
    if ((threadIdx.x & 31) == 0) {
        sm[threadIdx.x >> 5] = m;
        ss[threadIdx.x >> 5] = s;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kStatThreads / 32; ++w) join(m, s, sm[w], ss[w], a.c);
        P.stats[row * P.slices + slice] = {m, s};
    }
}

// a row's (max, sum), by one warp, in the same order for every reader
__device__ __forceinline__ Stat row_stat(const ChainPlan& P, int64_t row, float c, int lane) {
    float m = -INFINITY, s = 0.0f;
    for (int j = lane; j < P.slices; j += 32) {
        const Stat t = P.stats[row * P.slices + j];
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

// the best of tokens [t0, t1) of max(P - Q, 0) / E (q == nullptr: P / E), as this thread's share
template <typename T>
__device__ __forceinline__ Best race(const T* p, const T* q, const float* noise, Stat sp, Stat sq, float c, int64_t t0,
                                     int64_t t1, int64_t V) {
    Best b = {0.0f, INT_MAX};  // only positive scores count
    const float ip = sp.s > 0.0f ? 1.0f / sp.s : 0.0f, iq = sq.s > 0.0f ? 1.0f / sq.s : 0.0f;
    for (int64_t t = t0 + 8 * threadIdx.x; t < t1; t += 8 * kRaceThreads) {
        float x[8], y[8], z[8];
        load8(x, p, t, V, -INFINITY);
        if (q != nullptr) load8(y, q, t, V, -INFINITY);
        load8(z, noise, t, V, 1.0f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float d = weight(usable(x[e]), sp.m, c) * ip;
            if (q != nullptr) d -= weight(usable(y[e]), sq.m, c) * iq;
            if (t + e < t1 && d > 0.0f) better(b, d / z[e], (int)(t + e));
        }
    }
    return b;
}

template <typename T>
__global__ void __launch_bounds__(kRaceThreads) finish_kernel(const ChainArgs a, const ChainPlan P) {
    using E = Elem<T>;
    __shared__ int s_row[kMaxChain], s_tok[kMaxChain], s_ok[kMaxChain];
    __shared__ Best s_best[kRaceThreads / 32];
    __shared__ Stat s_stat[2];
    __shared__ int s_last;
    pdl_wait();
    const int seq = (int)(blockIdx.x / (unsigned)P.race_slices), slice = (int)(blockIdx.x % (unsigned)P.race_slices);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n0 = __ldg(a.seq_off + seq), n1 = __ldg(a.seq_off + seq + 1);
    if (n0 < 0 || n1 <= n0 || n1 > a.n_nodes) {  // CTA-uniform: nothing of the sequence can be read
        if (slice == 0 && threadIdx.x == 0) {
            a.out_acc[seq] = 0;
            a.out_ne[seq] = 0;
            for (int j = 0; j <= a.gamma; ++j) a.out_em[(int64_t)seq * (a.gamma + 1) + j] = -1;
            if (a.status) atomicOr(a.status, PPS_FLAG_INDEX);
        }
        return;
    }
    const int longest = min(n1 - n0 - 1, a.gamma);
    for (int j = warp; j < longest; j += kRaceThreads / 32) {
        const int node = n0 + j, r = __ldg(a.node_draft_row + node);
        const bool has = r >= 0 && r < a.n_draft;
        int tok = has ? __ldg(a.draft_tok + r) : -1, ok = 0;
        bool bad = r >= a.n_draft;
        if (has) {
            const Stat sp = row_stat(P, node, a.c, lane), sq = row_stat(P, a.n_nodes + r, a.c, lane);
            float px = 0.0f, qx = 0.0f;
            if (tok < 0 || tok >= a.V)
                bad = true;
            else {
                const float lp = usable(E::get(static_cast<const T*>(a.p) + node * a.p_stride + tok));
                const float lq = usable(E::get(static_cast<const T*>(a.q) + r * a.q_stride + tok));
                if (sp.s > 0.0f) px = weight(lp, sp.m, a.c) / sp.s;
                if (sq.s > 0.0f) qx = weight(lq, sq.m, a.c) / sq.s;
            }
            ok = __ldg(a.u + r) * qx < px;
            if (slice == 0 && lane == 0 && a.out_prob)
                a.out_prob[r] = px > 0.0f ? (px < qx ? px / qx : 1.0f) : 0.0f;
        }
        if (lane == 0) {
            s_row[j] = has ? r : -1;
            s_tok[j] = tok;
            s_ok[j] = ok;
            if (bad && slice == 0 && a.status) atomicOr(a.status, PPS_FLAG_INDEX);
        }
    }
    __syncthreads();
    int acc = 0;
    while (acc < longest && s_ok[acc]) ++acc;
    const int node = n0 + acc, r = acc < longest ? s_row[acc] : -1;
    if (warp < 2) {
        const Stat st = warp == 0 ? row_stat(P, node, a.c, lane) : r >= 0 ? row_stat(P, a.n_nodes + r, a.c, lane) : Stat{0.0f, 0.0f};
        if (lane == 0) s_stat[warp] = st;
    }
    __syncthreads();
    const Stat sp = s_stat[0], sq = s_stat[1];
    const T* p = static_cast<const T*>(a.p) + node * a.p_stride;
    const T* q = r >= 0 && sq.s > 0.0f ? static_cast<const T*>(a.q) + r * a.q_stride : nullptr;
    const float* noise = a.noise + seq * a.noise_stride;
    const int64_t t0 = (int64_t)slice * P.race_len, t1 = min(t0 + P.race_len, a.V);
    Best b = {0.0f, INT_MAX};
    if (sp.s > 0.0f) b = race(p, q, noise, sp, sq, a.c, t0, t1, a.V);
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
    for (int j = threadIdx.x; j < P.race_slices; j += kRaceThreads) {
        const float2 o = __ldcg(reinterpret_cast<const float2*>(P.best + (int64_t)seq * P.race_slices + j));
        better(b, o.x, __float_as_int(o.y));
    }
    b = block_best(b, s_best);
    if (b.i == INT_MAX && q != nullptr && sp.s > 0.0f)  // the residual is zero everywhere (CTA-uniform)
        b = block_best(race<T>(p, nullptr, noise, sp, sq, a.c, 0, a.V, a.V), s_best);
    for (int j = threadIdx.x; j <= a.gamma; j += kRaceThreads)
        a.out_em[(int64_t)seq * (a.gamma + 1) + j] = j < acc ? s_tok[j] : j == acc && b.i != INT_MAX ? b.i : -1;
    if (threadIdx.x == 0) {
        a.out_acc[seq] = acc;
        a.out_ne[seq] = acc + (b.i != INT_MAX);
    }
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

template <typename T>
cudaError_t launch(const ChainArgs& a, cudaStream_t st) {
    ChainPlan P;
    const int64_t rows = a.n_nodes + a.n_draft, nv = (a.V + Elem<T>::kVW - 1) / Elem<T>::kVW + 1;
    const int sms = device_sm_count();
    // slices of at most kVecs vectors a thread (one turn), of fewer where rows alone leave SMs idle
    const int64_t full = kVecs * kStatThreads;
    int64_t n = std::max<int64_t>((nv + full - 1) / full, std::min<int64_t>((nv + kStatThreads - 1) / kStatThreads, 4 * sms / rows));
    P.slices = (int)std::min<int64_t>(std::max<int64_t>(n, 1), kMaxSlices);
    P.vecs = (int)((nv + P.slices - 1) / P.slices);
    // the final rows: a turn of 8 tokens a thread at least
    n = std::min<int64_t>((a.V + 8 * kRaceThreads - 1) / (8 * kRaceThreads), std::max<int64_t>(1, 8 * sms / a.n_seq));
    P.race_slices = (int)std::min<int64_t>(std::max<int64_t>(n, 1), kMaxSlices);
    P.race_len = (int)(((a.V + P.race_slices - 1) / P.race_slices + 7) / 8 * 8);
    char* w = static_cast<char*>(a.ws);
    P.stats = reinterpret_cast<Stat*>(w);
    w += align256(sizeof(Stat) * (size_t)rows * kMaxSlices);
    P.best = reinterpret_cast<Best*>(w);
    w += align256(sizeof(Best) * (size_t)a.n_seq * kMaxSlices);
    P.ticket = reinterpret_cast<uint32_t*>(w);
    if (rows * P.slices > INT32_MAX || (int64_t)a.n_seq * P.race_slices > INT32_MAX) return cudaErrorInvalidValue;
    stats_kernel<T><<<(unsigned)(rows * P.slices), kStatThreads, 0, st>>>(a, P);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_pdl(finish_kernel<T>, dim3((unsigned)(a.n_seq * P.race_slices)), dim3(kRaceThreads), 0, st, a, P);
}

}  // namespace

size_t chain_workspace_bytes(int64_t n_nodes, int64_t n_draft, int n_seq) {
    return align256(sizeof(Stat) * (size_t)(n_nodes + n_draft) * kMaxSlices) +
           align256(sizeof(Best) * (size_t)n_seq * kMaxSlices) + align256(sizeof(uint32_t) * (size_t)n_seq);
}

cudaError_t launch_chain(const ChainArgs& a, int dtype, cudaStream_t stream) {
    return dtype == PPS_BF16 ? launch<__nv_bfloat16>(a, stream) : launch<float>(a, stream);
}

}  // namespace pps
