// pps_append.cu -- norming, rotation and paged-cache append of new tokens' heads.
//
// Per head x of a query or key (channels c < D):
//   y = x / sqrt(mean x^2 + eps) * w                        (where a weight is given)
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t)        (the first rot channels, in pairs)
// in fp32, rounded once; values are copied.  Each of the (n_heads + 2 n_kv_heads) D channels of a token
// is read once and written once, so the pass is bound by HBM; norm and rotation are some ten
// operations a channel.
//
// Layout.  A group of lanes holds one head: lane l has unit l, two vectors of VW channels, the two
// halves of VW (or, interleaved, 2 x VW / 2) rotation pairs, so that no channel leaves its lane but
// for the norm's sum (log2(group) shuffles).  A warp's item is kAhead heads of each lane group, of one token.  Warps
// stay and take items in turn, slots and positions two items ahead, channels and the table's row one ahead: a
// position has to arrive before the row's address is known, and each wait is an item long.
#include <algorithm>
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pps.h"
#include "pps_internal.h"

namespace pps {
namespace {

constexpr int kAppendWarps = 4;  // per CTA
constexpr int kAhead = 2;        // heads of a lane group in an item
constexpr int kAppendCtas = 4;   // per SM

struct AppendPlan {
    int lg;          // log2 of the lanes per head
    int parts;       // items per token
    int units;       // units per head
    int pair_units;  // of which rotated
    float inv_d;
};

template <int VW>
struct RawVec;
template <>
struct RawVec<8> { using type = uint4; };
template <>
struct RawVec<4> { using type = uint2; };
template <>
struct RawVec<1> { using type = uint16_t; };

__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }

template <typename T, int VW>
union Vec {
    typename RawVec<VW>::type raw;
    T e[VW];
    __device__ __forceinline__ Vec() {}
    __device__ __forceinline__ Vec(const Vec& o) : raw(o.raw) {}
    __device__ __forceinline__ Vec& operator=(const Vec& o) {
        raw = o.raw;
        return *this;
    }
};

template <typename T, int VW>
__device__ __forceinline__ void load(Vec<T, VW>& x, const T* p) {
    x.raw = *reinterpret_cast<const typename RawVec<VW>::type*>(p);
}
template <typename T, int VW>
__device__ __forceinline__ void store(T* p, const Vec<T, VW>& x) {
    *reinterpret_cast<typename RawVec<VW>::type*>(p) = x.raw;
}

// what an item needs from memory
template <typename T, int VW, int NU>
struct Item {
    Vec<T, VW> x[kAhead][NU][2];
    float cs[NU][VW], sn[NU][VW];
};

// NU: units per lane (more than one only for VW = 1).  NORM: whether queries or keys have a norm (its sums and weights in the
// loop, although skipped, cost a pass without norm 4 to 17 percent: 8192 tokens of (32 + 2 x 8) x 128 37.6 -> 35.8 us, with norm 48.5)
template <typename T, int VW, int NU, bool NORM>
__global__ void __launch_bounds__(32 * kAppendWarps, kAppendCtas) append_kernel(const AppendArgs a, const AppendPlan P) {
    const int lane = threadIdx.x & 31;
    const int D = a.c.head_dim, half = a.rot >> 1;
    const int l = lane & ((1 << P.lg) - 1), hp = 32 >> P.lg, group = lane >> P.lg;
    const int n_kv = a.c.n_kv_heads, n_qk = a.n_heads + n_kv, H = n_qk + n_kv;
    const uint32_t items = (uint32_t)a.n_tok * P.parts, stride = gridDim.x * kAppendWarps;
    uint32_t it = blockIdx.x * kAppendWarps + (threadIdx.x >> 5);
    if (it >= items) return;  // warp-uniform

    // the lane's units: channel starts of their two vectors
    int c0[NU], c1[NU];
#pragma unroll
    for (int n = 0; n < NU; ++n) {
        const int u = l + (n << P.lg);
        if (u < P.pair_units) {
            c0[n] = a.interleaved ? 2 * u * VW : u * VW;
            c1[n] = a.interleaved ? c0[n] + VW : half + u * VW;
        } else {
            c0[n] = u < P.units ? a.rot + (u - P.pair_units) * 2 * VW : D;
            c1[n] = c0[n] + VW;
        }
    }
    auto fetch_x = [&](Item<T, VW, NU>& y, int64_t tok, int part) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int h = (part * kAhead + j) * hp + group;
            if (h >= H) break;
            const bool is_q = h < a.n_heads, is_k = h < n_qk;
            const HeadsView& s = is_q ? a.q : is_k ? a.k : a.v;
            const T* src = static_cast<const T*>(s.p) + tok * s.tok + (h - (is_q ? 0 : is_k ? a.n_heads : n_qk)) * s.head;
#pragma unroll
            for (int n = 0; n < NU; ++n) {
                if (c0[n] < D) load(y.x[j][n][0], src + c0[n]);
                if (c1[n] < D) load(y.x[j][n][1], src + c1[n]);
            }
        }
    };
    auto fetch_rope = [&](Item<T, VW, NU>& y, int pos) {
        if (half == 0) return;
        const float* table = a.rope + min(max((int64_t)pos, (int64_t)0), a.max_pos - 1) * a.rot;
#pragma unroll
        for (int n = 0; n < NU; ++n) {
            const int u = l + (n << P.lg);
            if (u >= P.pair_units) continue;
            if constexpr (VW == 1) {
                y.cs[n][0] = __ldg(table + u);
                y.sn[n][0] = __ldg(table + half + u);
            } else {
#pragma unroll
                for (int e = 0; e < VW; e += 4) {
                    *reinterpret_cast<float4*>(&y.cs[n][e]) = __ldg(reinterpret_cast<const float4*>(table + u * VW + e));
                    *reinterpret_cast<float4*>(&y.sn[n][e]) = __ldg(reinterpret_cast<const float4*>(table + half + u * VW + e));
                }
            }
        }
    };

    Item<T, VW, NU> cur, nxt;
    uint32_t tok = it / (uint32_t)P.parts, tok1 = (it + stride) / (uint32_t)P.parts;
    fetch_x(cur, tok, (int)(it - tok * P.parts));
    int64_t slot = __ldg(a.slot + tok), slot1 = -1;
    int pos = half > 0 ? __ldg(a.pos + tok) : 0, pos1 = 0;
    if (it + stride < items) {
        slot1 = __ldg(a.slot + tok1);
        if (half > 0) pos1 = __ldg(a.pos + tok1);
    }
    fetch_rope(cur, pos);
    while (true) {
        const int part = (int)(it - tok * P.parts);
        const bool more = it + stride < items;
        const uint32_t tok2 = (it + 2 * stride) / (uint32_t)P.parts;
        int64_t slot2 = -1;
        int pos2 = 0;
        if (more) {
            fetch_x(nxt, tok1, (int)(it + stride - tok1 * P.parts));
            if (items - it > 2 * stride) {
                slot2 = __ldg(a.slot + tok2);
                if (half > 0) pos2 = __ldg(a.pos + tok2);
            }
            fetch_rope(nxt, pos1);
        }

        int64_t page = 0;
        int in_page = 0;
        bool kept = slot >= 0;
        if (kept) {
            page = (slot >> 32) != 0 ? slot / a.c.page_size : (int64_t)((uint32_t)slot / (uint32_t)a.c.page_size);
            in_page = (int)(slot - page * a.c.page_size);
            kept = page < a.c.n_pages;
        }
        if (((slot >= 0 && !kept) || (half > 0 && (pos < 0 || pos >= a.max_pos))) && part == 0 && lane == 0 && a.status)
            atomicOr(a.status, PPS_FLAG_INDEX);

#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if ((part * kAhead + j) * hp >= H) break;  // warp-uniform
            const int h = (part * kAhead + j) * hp + group;
            const bool is_q = h < a.n_heads, turned = h < n_qk;  // queries; queries and keys
            T* dst = nullptr;
            if (is_q)
                dst = static_cast<T*>(a.out.p) + tok * a.out.tok + h * a.out.head;
            else if (h < H && kept)
                dst = static_cast<T*>(turned ? a.c.k : a.c.v) + page * a.c.page + in_page * a.c.tok +
                      (h - (turned ? a.n_heads : n_qk)) * a.c.head;
            const T* w = static_cast<const T*>(is_q ? a.q_norm : a.k_norm);
            if (!turned || dst == nullptr) w = nullptr;
            float r = 1.0f;
            Vec<T, VW> wv[NU][2];
            if constexpr (NORM) {  // uniform: every lane takes part in the shuffles
                float ss = 0.0f;
                if (w != nullptr) {
#pragma unroll
                    for (int n = 0; n < NU; ++n)
#pragma unroll
                        for (int v = 0; v < 2; ++v)
                            if ((v ? c1[n] : c0[n]) < D) {
                                load(wv[n][v], w + (v ? c1[n] : c0[n]));
#pragma unroll
                                for (int e = 0; e < VW; ++e) {
                                    const float f = to_f(cur.x[j][n][v].e[e]);
                                    ss = fmaf(f, f, ss);
                                }
                            }
                }
                for (int o = (1 << P.lg) >> 1; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
                r = rsqrtf(fmaf(ss, P.inv_d, a.eps));
            }
            if (dst == nullptr) continue;
#pragma unroll
            for (int n = 0; n < NU; ++n) {
                if (c0[n] >= D) continue;
                if (turned) {
                    float f[2][VW];
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
                        if ((v ? c1[n] : c0[n]) >= D) continue;
#pragma unroll
                        for (int e = 0; e < VW; ++e) f[v][e] = to_f(cur.x[j][n][v].e[e]);
                        if (NORM && w != nullptr)
#pragma unroll
                            for (int e = 0; e < VW; ++e) f[v][e] *= r * to_f(wv[n][v].e[e]);
                    }
                    if (c0[n] < a.rot) {
                        if (VW > 1 && a.interleaved) {
#pragma unroll
                            for (int v = 0; v < 2; ++v)
#pragma unroll
                                for (int e = 0; e + 1 < VW; e += 2) {
                                    const float c = cur.cs[n][(v * VW + e) >> 1], s = cur.sn[n][(v * VW + e) >> 1];
                                    const float p = f[v][e], q = f[v][e + 1];
                                    f[v][e] = p * c - q * s;
                                    f[v][e + 1] = p * s + q * c;
                                }
                        } else {
#pragma unroll
                            for (int e = 0; e < VW; ++e) {
                                const float p = f[0][e], q = f[1][e];
                                f[0][e] = p * cur.cs[n][e] - q * cur.sn[n][e];
                                f[1][e] = p * cur.sn[n][e] + q * cur.cs[n][e];
                            }
                        }
                    }
#pragma unroll
                    for (int v = 0; v < 2; ++v)
                        if ((v ? c1[n] : c0[n]) < D)
#pragma unroll
                            for (int e = 0; e < VW; ++e) cur.x[j][n][v].e[e] = from_f<T>(f[v][e]);
                }
                store(dst + c0[n], cur.x[j][n][0]);
                if (c1[n] < D) store(dst + c1[n], cur.x[j][n][1]);
            }
        }
        if (!more) break;
        it += stride;
        cur = nxt;
        tok = tok1;
        tok1 = tok2;
        slot = slot1;
        slot1 = slot2;
        pos = pos1;
        pos1 = pos2;
    }
}

template <typename T, int VW, int NU>
cudaError_t launch(const AppendArgs& a, cudaStream_t st) {
    AppendPlan P;
    P.pair_units = a.rot / (2 * VW);
    P.units = P.pair_units + (a.c.head_dim - a.rot + 2 * VW - 1) / (2 * VW);
    P.lg = 0;
    while (P.lg < 5 && (1 << P.lg) < P.units) ++P.lg;
    const int H = a.n_heads + 2 * a.c.n_kv_heads;
    const int per_item = kAhead * (32 >> P.lg);  // heads
    P.parts = (H + per_item - 1) / per_item;
    P.inv_d = 1.0f / (float)a.c.head_dim;
    const int64_t items = a.n_tok * P.parts, most = (int64_t)device_sm_count() * kAppendCtas;
    if (items > INT32_MAX) return cudaErrorInvalidValue;
    const int64_t blocks = std::min((items + kAppendWarps - 1) / kAppendWarps, most);
    if (a.q_norm != nullptr || a.k_norm != nullptr)
        append_kernel<T, VW, NU, true><<<(unsigned)blocks, 32 * kAppendWarps, 0, st>>>(a, P);
    else
        append_kernel<T, VW, NU, false><<<(unsigned)blocks, 32 * kAppendWarps, 0, st>>>(a, P);
    return cudaGetLastError();
}

template <typename T>
cudaError_t by_width(const AppendArgs& a, cudaStream_t st) {
    // the widest vectors that every address and the rotation's halves allow
    uint64_t bits = 0;  // byte addresses and element strides, doubled to bytes
    for (const HeadsView* h : {&a.q, &a.k, &a.v, &a.out})
        bits |= reinterpret_cast<uintptr_t>(h->p) | (uint64_t)h->tok * 2 | (uint64_t)h->head * 2;
    bits |= reinterpret_cast<uintptr_t>(a.c.k) | reinterpret_cast<uintptr_t>(a.c.v);
    bits |= (uint64_t)(a.c.page | a.c.tok | a.c.head) * 2;
    bits |= reinterpret_cast<uintptr_t>(a.q_norm) | reinterpret_cast<uintptr_t>(a.k_norm);
    const bool table = a.rot == 0 || (reinterpret_cast<uintptr_t>(a.rope) & 15) == 0;
    if (table && bits % 16 == 0 && a.rot % 16 == 0) return launch<T, 8, 1>(a, st);
    if (table && bits % 8 == 0 && a.rot % 8 == 0) return launch<T, 4, 1>(a, st);
    return launch<T, 1, 4>(a, st);
}

}  // namespace

cudaError_t launch_kv_append(const AppendArgs& a, int dtype, cudaStream_t stream) {
    return dtype == PPS_BF16 ? by_width<__nv_bfloat16>(a, stream) : by_width<__half>(a, stream);
}

}  // namespace pps
