// pps_adjust.cu -- penalties for repeated tokens, biases and grammar masks on logits.
//
// Row r of sequence s, token i; c: how often i stands in the sequence's output and on the row's path through its draft tree, said:
// c > 0, or i stands in the prompt:
//   y = said ? (x > 0 ? x / repetition : x * repetition) : x
//   y = y - frequency c - presence [c > 0] + bias_i,   -inf where the mask has no bit;   in 32 bits, rounded once.
//
// Every logit is read and written once, whatever the texts are, so the pass is bound by HBM.  A CTA has a slice of the vocabulary
// of one sequence: it counts the text's tokens that fall into the slice in shared memory (and which entry of the bias list is
// a token's last) and lists the tokens that anything is known of, in order.  Its warps then take pieces of the sequence's rows: a piece
// is copied, but for the mask; then its listed tokens are formed from their logits, which the copy has left as they were (also in
// place); last the tokens of the row's path, a handful, whose values were formed before.  (Formed within the copy, with a look at each vector, they
// cost 400 us where this takes 250: of 32 vectors nearly always one has such a token, and all wait for it.)
#include <algorithm>
#include <climits>
#include <cstdint>
#include <cstring>

#include <cuda_bf16.h>

#include "pps.h"
#include "pps_internal.h"

namespace pps {
namespace {

constexpr int kAdjustThreads = 256, kAdjustWarps = kAdjustThreads / 32;
constexpr int kSlice = 4096;       // tokens
constexpr int kPiece = 1024;       // tokens that a warp takes of a row at a time
constexpr int kPath = 64;          // nodes of a path
constexpr uint32_t kPrompt = 1u << 31;

template <typename T>
struct Logit;
template <>
struct Logit<float> {
    static __device__ __forceinline__ float get(float x) { return x; }
    static __device__ __forceinline__ float put(float x) { return x; }
};
template <>
struct Logit<__nv_bfloat16> {
    static __device__ __forceinline__ float get(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 put(float x) { return __float2bfloat16_rn(x); }
};

struct Law {
    float rep, freq, pres;
    __device__ __forceinline__ float operator()(float x, uint32_t count, bool prompt, float bias, bool allowed) const {
        if (count > 0 || prompt) x = x > 0.0f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
        x = __fsub_rn(x, __fmul_rn(freq, (float)count));
        if (count > 0) x = __fsub_rn(x, pres);
        x = __fadd_rn(x, bias);
        return allowed ? x : -INFINITY;
    }
};

// N bits of `words` from bit i on; a second word is read only where they reach into it
template <int N>
__device__ __forceinline__ uint32_t bits_at(const uint32_t* words, int i) {
    const uint32_t lo = words[i >> 5], hi = (i & 31) > 32 - N ? words[(i >> 5) + 1] : 0u;
    return __funnelshift_r(lo, hi, i & 31) & ((1u << N) - 1u);
}

template <typename T, bool COUNTS, bool BIAS>
__global__ void __launch_bounds__(kAdjustThreads, 4) adjust_kernel(const AdjustArgs a) {
    constexpr int VN = 16 / sizeof(T);
    __shared__ __align__(16) uint32_t s_count[COUNTS ? kSlice : 4];
    __shared__ __align__(16) int s_bias[BIAS ? kSlice : 4];   // 1 + the last entry for the token
    __shared__ uint32_t s_known[kSlice / 32];
    __shared__ uint16_t s_list[COUNTS || BIAS ? kSlice : 2];  // the slice's known tokens, in order
    __shared__ int s_from[kSlice / kPiece + 1];               // where those of a piece begin
    __shared__ int s_warp[kAdjustWarps];
    __shared__ int s_path[kAdjustWarps][kPath];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int seq = blockIdx.y;
    const int t0 = blockIdx.x * kSlice, tn = (int)min((int64_t)kSlice, a.V - t0);
    int first = __ldg(a.seq_off + seq), end = __ldg(a.seq_off + seq + 1);
    if (first < 0 || end < first || end > a.n_rows) {
        if (tid == 0 && a.status) atomicOr(a.status, PPS_FLAG_INDEX);
        return;
    }
    if (first == end) return;
    const int n_rows = end - first;
    bool bad = false;
    Law law = {1.0f, 0.0f, 0.0f};
    if constexpr (COUNTS || BIAS) {
        for (int i = tid; i < kSlice / 32; i += kAdjustThreads) s_known[i] = 0;
        if constexpr (COUNTS)
            for (int i = tid; i < kSlice / 4; i += kAdjustThreads) reinterpret_cast<uint4*>(s_count)[i] = make_uint4(0, 0, 0, 0);
        if constexpr (BIAS)
            for (int i = tid; i < kSlice / 4; i += kAdjustThreads) reinterpret_cast<int4*>(s_bias)[i] = make_int4(0, 0, 0, 0);
        __syncthreads();
        if constexpr (COUNTS) {
            if (a.rep) law.rep = __ldg(a.rep + seq);
            if (a.freq) law.freq = __ldg(a.freq + seq);
            if (a.pres) law.pres = __ldg(a.pres + seq);
            if (a.text) {
                const int said = __ldg(a.text_len + seq), len = min(max(said, 0), a.text_cap);
                const int prompt = a.prompt_len ? min(max(__ldg(a.prompt_len + seq), 0), len) : 0;
                bad |= said != len;
                const int32_t* text = a.text + seq * a.text_stride;
                for (int i0 = tid; i0 < len; i0 += 4 * kAdjustThreads) {
                    int tok[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) tok[k] = i0 + k * kAdjustThreads < len ? __ldg(text + i0 + k * kAdjustThreads) : INT_MIN;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int i = i0 + k * kAdjustThreads, at = tok[k] - t0;
                        if (i >= len) break;
                        bad |= tok[k] < 0 || tok[k] >= a.V;
                        if (tok[k] < 0 || at < 0 || at >= tn) continue;
                        if (i < prompt)
                            atomicOr(&s_count[at], kPrompt);
                        else
                            atomicAdd(&s_count[at], 1u);
                        atomicOr(&s_known[at >> 5], 1u << (at & 31));
                    }
                }
            }
        }
        if constexpr (BIAS) {
            const int b0 = __ldg(a.bias_off + seq), b1 = __ldg(a.bias_off + seq + 1);
            const bool off = b0 < 0 || b1 < b0 || b1 > a.n_bias;
            bad |= off;
            if (!off)
                for (int i = b0 + tid; i < b1; i += kAdjustThreads) {
                    const int tok = __ldg(a.bias_tok + i), at = tok - t0;
                    bad |= tok < 0 || tok >= a.V;
                    if (tok < 0 || at < 0 || at >= tn) continue;
                    atomicMax(&s_bias[at], i + 1);
                    atomicOr(&s_known[at >> 5], 1u << (at & 31));
                }
        }
        __syncthreads();
        static_assert(kSlice / 32 <= kAdjustThreads && kPiece % 32 == 0, "a thread per word, whole words in a piece");
        uint32_t word = tid < kSlice / 32 ? s_known[tid] : 0u;
        int before = __popc(word);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, before, o);
            if (lane >= o) before += y;
        }
        if (lane == 31) s_warp[warp] = before;
        __syncthreads();
        before -= __popc(word);
        for (int w = 0; w < warp; ++w) before += s_warp[w];
        if (tid < kSlice / 32 && tid % (kPiece / 32) == 0) s_from[tid / (kPiece / 32)] = before;
        if (tid == kSlice / 32 - 1) s_from[kSlice / kPiece] = before + __popc(word);
        for (; word != 0; word &= word - 1) s_list[before++] = (uint16_t)(32 * tid + __ffs(word) - 1);
        __syncthreads();
    }
    auto adjusted = [&](float x, int at, uint32_t more, bool allowed) {
        uint32_t c = 0;
        if constexpr (COUNTS) c = s_count[at];
        float bias = 0.0f;
        if constexpr (BIAS)
            if (const int e = s_bias[at]) bias = __ldg(a.bias_val + e - 1);
        return law(x, (c & ~kPrompt) + more, (c & kPrompt) != 0, bias, allowed);
    };

    // items: pieces of rows
    const int pieces = (tn + kPiece - 1) / kPiece;
    for (int item = warp; item < n_rows * pieces; item += kAdjustWarps) {
        const int i = item / pieces, p0 = (item - i * pieces) * kPiece, p1 = min(p0 + kPiece, tn);
        const int64_t row = first + i;
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride + t0;
        T* out = static_cast<T*>(a.out) + row * a.out_stride + t0;
        const uint32_t* allowed = a.allowed ? a.allowed + row * a.allowed_stride : nullptr;
        // the path's tokens: the row's own and its ancestors'
        int n_path = 0;
        float fixed[2];
        int fixed_at[2] = {-1, -1};
        if (COUNTS && a.node_tok) {
            const int words = a.node_mask ? min(a.mask_words, (n_rows + 31) >> 5) : (i >> 5) + 1;
            for (int w = 0; w < words; ++w) {
                const int node = 32 * w + lane;
                const bool on = node < n_rows && (a.node_mask ? (__ldg(a.node_mask + row * a.mask_words + w) >> lane & 1u) != 0 : node <= i);
                const uint32_t who = __ballot_sync(0xffffffffu, on);
                if (on) {
                    const int tok = __ldg(a.node_tok + first + node), to = n_path + __popc(who & ((1u << lane) - 1u));
                    if (to < kPath) s_path[warp][to] = tok;
                    bad |= to >= kPath || tok < 0 || tok >= a.V;
                }
                n_path = min(n_path + __popc(who), kPath);
            }
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int me = lane + 32 * k;
                if (me >= n_path) continue;
                const int tok = s_path[warp][me], at = tok - t0;
                if (tok < 0 || at < p0 || at >= p1) continue;
                uint32_t n = 0;
                bool again = false;
                for (int j = 0; j < n_path; ++j)
                    if (s_path[warp][j] == tok) {
                        ++n;
                        again |= j < me;
                    }
                if (again) continue;
                fixed_at[k] = at;
                fixed[k] = adjusted(Logit<T>::get(x[at]), at, n, !allowed || (allowed[tok >> 5] >> (tok & 31) & 1u));
            }
            __syncwarp();  // (in place: the logits are read)
        }
        auto one = [&](int at) {
            const int tok = t0 + at;
            const bool ok = !allowed || (__ldg(allowed + (tok >> 5)) >> (tok & 31) & 1u);
            out[at] = ok ? x[at] : Logit<T>::put(-INFINITY);
        };
        // whole vectors where input and output lie alike, what is before and behind them one by one
        const int lies = (int)((reinterpret_cast<uintptr_t>(x + p0) & 15) / sizeof(T));
        const bool alike = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
        const int v0 = alike ? min(p0 + (lies ? VN - lies : 0), p1) : p1, nv = (p1 - v0) / VN;
        for (int at = p0 + lane; at < v0; at += 32) one(at);
        for (int at = v0 + nv * VN + lane; at < p1; at += 32) one(at);
        constexpr uint32_t all = (1u << VN) - 1u;
        constexpr int kBatch = 4;  // vectors on their way
        for (int j0 = lane; j0 < nv; j0 += 32 * kBatch) {
            uint4 raw[kBatch];
            uint32_t ok[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) ok[k] = allowed && j0 + 32 * k < nv ? bits_at<VN>(allowed, t0 + v0 + (j0 + 32 * k) * VN) : all;
#pragma unroll
            for (int k = 0; k < kBatch; ++k)  // what is not allowed need not be read
                if (j0 + 32 * k < nv && ok[k] != 0) raw[k] = __ldcs(reinterpret_cast<const uint4*>(x + v0) + j0 + 32 * k);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int j = j0 + 32 * k, at = v0 + j * VN;
                if (j >= nv) break;
                if (ok[k] != all) {
                    T v[VN];
                    memcpy(v, &raw[k], 16);
#pragma unroll
                    for (int e = 0; e < VN; ++e)
                        if (!(ok[k] >> e & 1u)) v[e] = Logit<T>::put(-INFINITY);
                    memcpy(&raw[k], v, 16);
                }
                __stcs(reinterpret_cast<uint4*>(out + at), raw[k]);
            }
        }
        if constexpr (COUNTS || BIAS) {
            __syncwarp();
            const int from = s_from[p0 / kPiece], to = s_from[p0 / kPiece + 1];
            for (int e0 = from + lane; e0 < to; e0 += 64) {  // two on their way
                int at[2];
                T v[2];
                bool ok[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int e = e0 + 32 * k;
                    at[k] = e < to ? s_list[e] : -1;
                    ok[k] = at[k] >= 0 && (!allowed || (allowed[(t0 + at[k]) >> 5] >> ((t0 + at[k]) & 31) & 1u));
                    if (ok[k]) v[k] = x[at[k]];
                }
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (ok[k]) out[at[k]] = Logit<T>::put(adjusted(Logit<T>::get(v[k]), at[k], 0, true));
            }
        }
        if (COUNTS && a.node_tok) {
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (fixed_at[k] >= 0) out[fixed_at[k]] = Logit<T>::put(fixed[k]);
        }
    }
    if (bad && a.status) atomicOr(a.status, PPS_FLAG_INDEX);
}

template <typename T>
cudaError_t by_parts(const AdjustArgs& a, cudaStream_t st) {
    const bool counts = a.text != nullptr || a.node_tok != nullptr, bias = a.bias_tok != nullptr;
    auto kernel = counts ? (bias ? adjust_kernel<T, true, true> : adjust_kernel<T, true, false>)
                         : (bias ? adjust_kernel<T, false, true> : adjust_kernel<T, false, false>);
    const int64_t slices = (a.V + kSlice - 1) / kSlice;
    for (int s0 = 0; s0 < a.n_seq; s0 += 65535) {  // (a grid's second dimension)
        AdjustArgs part = a;
        const int n = std::min(a.n_seq - s0, 65535);
        part.n_seq = n;
        part.seq_off += s0;
        if (part.text) part.text += s0 * a.text_stride;
        if (part.text_len) part.text_len += s0;
        if (part.prompt_len) part.prompt_len += s0;
        if (part.rep) part.rep += s0;
        if (part.freq) part.freq += s0;
        if (part.pres) part.pres += s0;
        if (part.bias_off) part.bias_off += s0;
        kernel<<<dim3((unsigned)slices, (unsigned)n), kAdjustThreads, 0, st>>>(part);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_adjust(const AdjustArgs& a, int dtype, cudaStream_t stream) {
    return dtype == PPS_BF16 ? by_parts<__nv_bfloat16>(a, stream) : by_parts<float>(a, stream);
}

}  // namespace pps
