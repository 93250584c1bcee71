// pps_adjust.cu -- penalties for repeated tokens, biases and grammar masks on logits.
//
// Row r of sequence s, token i; c: how often i stands in the sequence's output and on the row's path through its draft tree, said:
// c > 0, or i stands in the prompt:
//   y = said ? (x > 0 ? x / repetition : x * repetition) : x
//   y = y - frequency c - presence [c > 0] + bias_i,   -inf where the mask has no bit;   in 32 bits, rounded once.
//
// Every logit is read and written once, whatever the texts are, so the pass is bound by HBM.  A CTA has a slice of the vocabulary
// of one sequence: it counts the text's tokens that fall into the slice in shared memory (and which entry of the bias list is
// a token's last), with a bit per token that anything is known of.  Its warps take pieces of the sequence's rows: vectors are copied
// through registers, and a vector's known tokens, by their bits, formed there one at a time.  (All elements of such a vector at once:
// 423 us for 64 x 41 rows of 128256 where this took 249, and takes 229 now; listed and formed in memory after the copy, 295 to 320: a read and a write of 32 bytes for each, of what
// has left L2 in part.)  Tokens of a row's path, a handful, are formed before its piece (which may be written in place) and written
// after it.
#include <algorithm>
#include <climits>
#include <cstdint>
#include <cstring>
#include <type_traits>

#include <cuda_bf16.h>

#include "pps.h"
#include "pps_internal.h"

namespace pps {
namespace {

constexpr int kAdjustThreads = 256, kAdjustWarps = kAdjustThreads / 32;
constexpr int kSlice = 4096;       // tokens
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

// element e of a 16-byte vector that stays in registers
template <typename T>
struct Pick;
template <>
struct Pick<float> {
    static __device__ __forceinline__ float get(const uint4& v, int e) { return __uint_as_float(e & 2 ? (e & 1 ? v.w : v.z) : (e & 1 ? v.y : v.x)); }
    static __device__ __forceinline__ void set(uint4& v, int e, float f) {
        const uint32_t x = __float_as_uint(f);
        v.x = e == 0 ? x : v.x;
        v.y = e == 1 ? x : v.y;
        v.z = e == 2 ? x : v.z;
        v.w = e == 3 ? x : v.w;
    }
};
template <>
struct Pick<__nv_bfloat16> {
    static __device__ __forceinline__ float get(const uint4& v, int e) {
        const uint32_t w = e & 4 ? (e & 2 ? v.w : v.z) : (e & 2 ? v.y : v.x);
        return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
    }
    static __device__ __forceinline__ void set(uint4& v, int e, float f) {
        const uint32_t x = __bfloat16_as_ushort(__float2bfloat16_rn(f)), how = e & 1 ? 0x5410u : 0x3254u;  // (of x, w: w's low half and x; x and w's high half)
        v.x = e >> 1 == 0 ? __byte_perm(v.x, x, how) : v.x;
        v.y = e >> 1 == 1 ? __byte_perm(v.y, x, how) : v.y;
        v.z = e >> 1 == 2 ? __byte_perm(v.z, x, how) : v.z;
        v.w = e >> 1 == 3 ? __byte_perm(v.w, x, how) : v.w;
    }
};

struct Law {
    float rep, freq, pres;
    __device__ __forceinline__ float operator()(float x, uint32_t count, bool prompt, float bias) const {
        if (count > 0 || prompt) x = x > 0.0f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
        x = __fsub_rn(x, __fmul_rn(freq, (float)count));
        if (count > 0) x = __fsub_rn(x, pres);
        return __fadd_rn(x, bias);
    }
};

// N bits of `words` from bit i on; a second word is read only where they reach into it
template <int N>
__device__ __forceinline__ uint32_t bits_at(const uint32_t* words, int i) {
    const uint32_t lo = words[i >> 5], hi = (i & 31) > 32 - N ? words[(i >> 5) + 1] : 0u;
    return __funnelshift_r(lo, hi, i & 31) & ((1u << N) - 1u);
}

// PIECE: tokens that a warp takes of a row at a time
template <typename T, bool COUNTS, bool BIAS, bool MASK, int PIECE>
__global__ void __launch_bounds__(kAdjustThreads, 4) adjust_kernel(const AdjustArgs a) {
    constexpr int VN = 16 / sizeof(T);
    // vectors of a lane on their way (64 x 41 rows: eight 231 us, four 238; beside biases or masks eight do not fit in the 64 registers)
    constexpr int kBatch = PIECE == 2048 && !BIAS && !MASK ? 8 : 4;
    __shared__ __align__(16) uint32_t s_count[COUNTS ? kSlice : 4];
    __shared__ __align__(16) int s_bias[BIAS ? kSlice : 4];   // 1 + the last entry for the token
    __shared__ uint32_t s_known[kSlice / 32];
    __shared__ int s_path[kAdjustWarps][kPath];
    constexpr int kWords = PIECE / 32;
    __shared__ uint32_t s_may[MASK ? kAdjustWarps : 1][kWords];  // a piece's part of the mask
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int seq = blockIdx.y;
    const int t0 = blockIdx.x * kSlice, tn = (int)min((int64_t)kSlice, a.V - t0);
    pdl_wait();
    pdl_launch_dependents();
    int first = __ldg(a.seq_off + seq), end = __ldg(a.seq_off + seq + 1);
    if (first < 0 || end < first || end > a.n_rows) {
        if (tid == 0 && a.status) atomicOr(a.status, PPS_FLAG_INDEX);
        return;
    }
    if (first == end) return;
    const int n_rows = end - first;
    bool bad = COUNTS && a.node_mask && n_rows > 32ll * a.mask_words;  // rows that no mask has a bit for
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
            if (a.text_len) {
                const int said = __ldg(a.text_len + seq), len = min(max(said, 0), a.text_cap);
                const int given = a.prompt_len ? __ldg(a.prompt_len + seq) : 0, prompt = min(max(given, 0), len);
                bad |= said != len || given != prompt;
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
    }
    auto adjusted = [&](float x, int at, uint32_t more) {
        uint32_t c = 0;
        if constexpr (COUNTS) c = s_count[at];
        float bias = 0.0f;
        if constexpr (BIAS)
            if (const int e = s_bias[at]) bias = __ldg(a.bias_val + e - 1);
        return law(x, (c & ~kPrompt) + more, (c & kPrompt) != 0, bias);
    };

    // items: pieces of rows
    const int pieces = (tn + PIECE - 1) / PIECE;
    // the next piece's part of the mask, on its way while this piece's logits are: read when it is needed, it is one more latency before
    // theirs (16 x 9 rows of 152063 in fp32: 41 us, 44 without)
    uint32_t next[kWords / 32];
    auto mask_of = [&](int item) {
        const int i = item / pieces, p0 = (item - i * pieces) * PIECE, words = item < n_rows * pieces ? (tn - p0 + 31) >> 5 : 0;
        const uint32_t* from = a.allowed + (first + i) * a.allowed_stride + ((t0 + p0) >> 5);
#pragma unroll
        for (int j = 0; j < kWords / 32; ++j) next[j] = 32 * j + lane < words ? __ldg(from + 32 * j + lane) : 0u;
    };
    if constexpr (MASK) mask_of(warp);
    for (int item = warp; item < n_rows * pieces; item += kAdjustWarps) {
        const int i = item / pieces, p0 = (item - i * pieces) * PIECE, p1 = min(p0 + PIECE, tn);
        const int64_t row = first + i;
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride + t0;
        T* out = static_cast<T*>(a.out) + row * a.out_stride + t0;
        if constexpr (MASK) {
            __syncwarp();
#pragma unroll
            for (int j = 0; j < kWords / 32; ++j) s_may[warp][32 * j + lane] = next[j];
            __syncwarp();
            mask_of(item + kAdjustWarps);
        }
        auto may = [&](int at) { return !MASK || (s_may[warp][(at - p0) >> 5] >> (at & 31) & 1u); };
        // the path's tokens: the row's own and its ancestors'
        float fixed[2];
        int fixed_at[2] = {-1, -1};
        if (COUNTS && a.node_tok) {
            int n_path = 0;
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
                if (again || !may(at)) continue;
                fixed_at[k] = at;
                fixed[k] = adjusted(Logit<T>::get(x[at]), at, n);
            }
            __syncwarp();  // (in place: the logits are read)
        }
        // whole vectors where input and output lie alike, what is before and behind them one by one
        const int lies = (int)((reinterpret_cast<uintptr_t>(x + p0) & 15) / sizeof(T));
        const bool alike = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
        const int v0 = alike ? min(p0 + (lies ? VN - lies : 0), p1) : p1, nv = (p1 - v0) / VN;
        auto one = [&](int at) {
            const bool known = (COUNTS || BIAS) && (s_known[at >> 5] >> (at & 31) & 1u);
            const T v = x[at];
            out[at] = !may(at) ? Logit<T>::put(-INFINITY) : known ? Logit<T>::put(adjusted(Logit<T>::get(v), at, 0)) : v;
        };
        for (int at = p0 + lane; at < v0; at += 32) one(at);
        for (int at = v0 + nv * VN + lane; at < p1; at += 32) one(at);
        const uint4* from = reinterpret_cast<const uint4*>(x + v0);
        uint4* to = reinterpret_cast<uint4*>(out + v0);
        constexpr uint32_t all = (1u << VN) - 1u;
        for (int j0 = lane; j0 < nv; j0 += 32 * kBatch) {
            uint4 raw[kBatch];
            uint32_t ok[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                ok[k] = j0 + 32 * k < nv ? all : 0u;
                if (MASK && ok[k]) ok[k] = bits_at<VN>(s_may[warp], v0 - p0 + (j0 + 32 * k) * VN);
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k)  // what is not allowed need not be read
                if (ok[k] != 0) raw[k] = __ldcs(from + j0 + 32 * k);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (j0 + 32 * k >= nv) break;
                const int at = v0 + (j0 + 32 * k) * VN;
                if constexpr (COUNTS || BIAS) {
                    // a known token at a time: of 32 vectors nearly always one has one, rarely one has two
                    for (uint32_t known = bits_at<VN>(s_known, at) & ok[k]; known != 0; known &= known - 1) {
                        const int e = __ffs(known) - 1;
                        Pick<T>::set(raw[k], e, adjusted(Pick<T>::get(raw[k], e), at + e, 0));
                    }
                }
                if (MASK && ok[k] != all) {
                    T v[VN];
                    memcpy(v, &raw[k], 16);
#pragma unroll
                    for (int e = 0; e < VN; ++e)
                        if (!(ok[k] >> e & 1u)) v[e] = Logit<T>::put(-INFINITY);
                    memcpy(&raw[k], v, 16);
                }
                __stcs(to + j0 + 32 * k, raw[k]);
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
    const bool counts = a.text_len != nullptr || a.node_tok != nullptr, bias = a.bias_tok != nullptr;
    // Pieces of 2048 tokens, or of 1024 where a sequence has few rows (measured on an earlier form: 64 x 41 rows 249 and 276 us, 16 x 9
    // rows 46 and 44, one row 7.1 and 6.1).  What a piece is, and whether there is a mask, are compile-time choices: each as a variable
    // made the call of 64 x 41 rows, which has no mask, 16 to 25 percent slower.
    const bool many = a.n_rows / 16 >= a.n_seq;
    auto sized = [&](auto c, auto b, auto m) {
        return many ? adjust_kernel<T, c.value, b.value, m.value, 2048> : adjust_kernel<T, c.value, b.value, m.value, 1024>;
    };
    auto masked = [&](auto c, auto b) { return a.allowed ? sized(c, b, std::true_type()) : sized(c, b, std::false_type()); };
    auto biased = [&](auto c) { return bias ? masked(c, std::true_type()) : masked(c, std::false_type()); };
    auto kernel = counts ? biased(std::true_type()) : biased(std::false_type());
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
        const cudaError_t e = launch_pdl(kernel, dim3((unsigned)slices, (unsigned)n), dim3(kAdjustThreads), 0, st, part);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_adjust(const AdjustArgs& a, int dtype, cudaStream_t stream) {
    return dtype == PPS_BF16 ? by_parts<__nv_bfloat16>(a, stream) : by_parts<float>(a, stream);
}

}  // namespace pps
