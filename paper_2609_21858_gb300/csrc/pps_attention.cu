// pps_attention.cu -- attention of the newest tokens of each sequence over a paged cache.
//
// One warp per (token, head): lane l holds channels 4l .. 4l+3 of the query and of the running output; keys are
// taken one at a time with the running maximum and sum of an online softmax.
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pps.h"
#include "pps_internal.h"

namespace pps {
namespace {

__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }

template <typename T>
__global__ void __launch_bounds__(128) attention_kernel(const AttnArgs a) {
    const int64_t gw = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31, D = a.c.head_dim;
    const int64_t tok = gw / a.n_heads;
    const int h = (int)(gw % a.n_heads), kh = h / (a.n_heads / a.c.n_kv_heads);
    if (tok >= a.n_tok) return;
    if (gw == 0 && lane == 0 && a.status)
        for (int i = 0; i < a.n_seq; ++i)
            if (a.q_off[i] < 0 || a.q_off[i + 1] > a.n_tok || a.q_off[i + 1] < a.q_off[i]) atomicOr(a.status, PPS_FLAG_INDEX);
    int s = -1;
    for (int i = 0; i < a.n_seq; ++i)
        if (a.q_off[i] >= 0 && a.q_off[i + 1] <= a.n_tok && a.q_off[i] <= tok && tok < a.q_off[i + 1]) s = i;
    if (s < 0) return;
    const int n = a.q_off[s + 1] - a.q_off[s], i = (int)tok - a.q_off[s];
    const int64_t cap = (int64_t)a.max_pages * a.c.page_size;
    const int64_t L = min((int64_t)max(a.kv_len[s], 0), cap);
    if (lane == 0 && a.status && L != a.kv_len[s]) atomicOr(a.status, PPS_FLAG_INDEX);
    const T* qp = static_cast<const T*>(a.q.p) + tok * a.q.tok + h * a.q.head;
    float q[4], o[4] = {0, 0, 0, 0}, m = -INFINITY, sum = 0.0f;
    for (int e = 0; e < 4; ++e) q[e] = 4 * lane + e < D ? to_f(qp[4 * lane + e]) * a.scale : 0.0f;
    for (int64_t j = 0; j < L; ++j) {
        const int64_t rel = j - (L - n);
        const bool sees = a.mask ? rel < 0 || (rel < 32 * a.mask_words && (a.mask[tok * a.mask_words + rel / 32] >> (rel % 32) & 1))
                                 : rel <= i;
        if (!sees) continue;
        const int page = a.pages[s * a.pages_stride + j / a.c.page_size];
        const bool in = page >= 0 && page < a.c.n_pages;
        if (!in && lane == 0 && a.status) atomicOr(a.status, PPS_FLAG_INDEX);
        const int64_t at = page * a.c.page + (j % a.c.page_size) * a.c.tok + kh * a.c.head + 4 * lane;
        float d = 0.0f, v[4] = {0, 0, 0, 0};
        if (in)
            for (int e = 0; e < 4; ++e)
                if (4 * lane + e < D) {
                    d += q[e] * to_f(static_cast<const T*>(a.c.k)[at + e]);
                    v[e] = to_f(static_cast<const T*>(a.c.v)[at + e]);
                }
        for (int w = 16; w > 0; w >>= 1) d += __shfl_xor_sync(0xffffffffu, d, w);
        const float M = fmaxf(m, d), r = m == M ? 1.0f : expf(m - M), x = d == M ? 1.0f : expf(d - M);
        sum = sum * r + x;
        for (int e = 0; e < 4; ++e) o[e] = o[e] * r + x * v[e];
        m = M;
    }
    T* op = static_cast<T*>(a.out.p) + tok * a.out.tok + h * a.out.head;
    for (int e = 0; e < 4; ++e)
        if (4 * lane + e < D) op[4 * lane + e] = from_f<T>(sum > 0.0f ? o[e] / sum : 0.0f);
    if (lane == 0 && a.lse) a.lse[tok * a.n_heads + h] = sum > 0.0f ? m + logf(sum) : -INFINITY;
}

}  // namespace

size_t attention_workspace_bytes(int64_t, int, int, int) { return 256; }

cudaError_t launch_attention(const AttnArgs& a, int dtype, cudaStream_t stream) {
    const unsigned blocks = (unsigned)((a.n_tok * a.n_heads + 3) / 4);
    if (dtype == PPS_BF16)
        attention_kernel<__nv_bfloat16><<<blocks, 128, 0, stream>>>(a);
    else
        attention_kernel<__half><<<blocks, 128, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace pps
