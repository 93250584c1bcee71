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
// stay and take tokens in turn, always the same heads, so that what belongs to a head (where it comes from and goes to, its
// kind, its norm's weights) is found once; slots and positions are read two tokens ahead, channels and the table's row one
// ahead: a position has to arrive before the row's address is known, and each wait is an item long.
//
// Measured: with every item's addresses formed anew a pass issued 14 instructions per channel of a lane and was bound by
// issuing them (norm: 24); now 9 and 15.  8192 tokens of (32 + 2 x 8) heads of 128 channels take 35.9 us, 5.7 TB/s (85 percent
// of a copy's), with norm 43.7; of (14 + 2 x 2) x 64 11.5 and 15.3; of (20 + 2 x 4) x 80, where 5 of 8 lanes have a unit, 19.9 and 28.4
// (rot 40, 8-byte vectors: 28.1 and 38.8).  With a norm neither the issue slots (1.7 of 4 a clock) nor HBM (20 percent at 2624
// tokens) are full: the 16 warps of an SM, as many as their 124 registers allow, wait for loads and for their own last results.  A few tokens: 2.5 to 2.8 us
// in a graph, 4.1 launched one by one.  Tried: one head
// ahead and more CTAs, weights held or read before the shuffles (registers, 10 percent slower), one body of the loop
// that copies the next item's registers (10 percent slower).
#include <algorithm>
#include <cstdint>
#include <cstring>

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
    int tok_step;    // tokens in work at a time: tok_step x parts warps
    int page_log2;   // -1: not a power of two
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
    uint32_t w[VW > 1 ? VW / 2 : 1];
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

// two channels at a time
__device__ __forceinline__ uint64_t pack2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t sub2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
template <typename T>
__device__ __forceinline__ uint64_t widen(uint32_t w);
template <>
__device__ __forceinline__ uint64_t widen<__nv_bfloat16>(uint32_t w) {
    return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <>
__device__ __forceinline__ uint64_t widen<__half>(uint32_t w) {
    __half2 h;
    memcpy(&h, &w, 4);
    const float2 f = __half22float2(h);
    return pack2(f.x, f.y);
}
template <typename T>
__device__ __forceinline__ uint32_t narrow(uint64_t v);
template <>
__device__ __forceinline__ uint32_t narrow<__nv_bfloat16>(uint64_t v) {
    float a, b;
    unpack2(v, a, b);
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
}
template <>
__device__ __forceinline__ uint32_t narrow<__half>(uint64_t v) {
    float a, b;
    unpack2(v, a, b);
    const __half2 h = __floats2half2_rn(a, b);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
}

// what an item needs from memory
template <typename T, int VW, int NU>
struct Item {
    Vec<T, VW> x[kAhead][NU][2];
    float cs[NU][VW], sn[NU][VW];
};

// A unit's channels in fp32: in pairs of neighbours (VW > 1), or one of each half
template <typename T, int VW>
struct Wide {
    static constexpr int kN = VW > 1 ? VW / 2 : 1;
    uint64_t f[2][kN];
    __device__ __forceinline__ Wide(const Vec<T, VW> (&x)[2]) {
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int i = 0; i < kN; ++i) f[v][i] = VW > 1 ? widen<T>(x[v].w[i]) : pack2(to_f(x[v].e[0]), 0.0f);
    }
    __device__ __forceinline__ float squares() const {
        uint64_t s[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            s[0] = fma2(f[0][i], f[0][i], s[0]);
            s[1] = fma2(f[1][i], f[1][i], s[1]);
        }
        float a, b;
        unpack2(add2(s[0], s[1]), a, b);
        return a + b;
    }
    __device__ __forceinline__ void scale(float r, const Vec<T, VW> (&w)[2]) {
        const uint64_t rr = pack2(r, r);
        const Wide<T, VW> y(w);
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int i = 0; i < kN; ++i) f[v][i] = mul2(f[v][i], mul2(rr, y.f[v][i]));
    }
    __device__ __forceinline__ void rotate(bool interleaved, const float (&cs)[VW], const float (&sn)[VW]) {
        if (VW > 1 && interleaved) {
#pragma unroll
            for (int v = 0; v < 2; ++v)
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    const float c = cs[(v * kN + i) % VW], s = sn[(v * kN + i) % VW];
                    float p, q;
                    unpack2(f[v][i], p, q);
                    f[v][i] = pack2(p * c - q * s, p * s + q * c);
                }
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                const uint64_t c = pack2(cs[2 * i], cs[(2 * i + 1) % VW]), s = pack2(sn[2 * i], sn[(2 * i + 1) % VW]);
                const uint64_t p = f[0][i], q = f[1][i];
                f[0][i] = sub2(mul2(p, c), mul2(q, s));
                f[1][i] = fma2(p, s, mul2(q, c));
            }
        }
    }
    __device__ __forceinline__ void round(Vec<T, VW> (&x)[2]) const {
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                if constexpr (VW > 1) {
                    x[v].w[i] = narrow<T>(f[v][i]);
                } else {
                    float a, b;
                    unpack2(f[v][i], a, b);
                    x[v].e[0] = from_f<T>(a);
                }
            }
    }
};

// NU: units per lane (more than one only for VW = 1).  NORM: whether queries or keys have a norm (its sums and weights in the
// loop, although skipped, cost a pass without norm 4 to 17 percent: 8192 tokens of (32 + 2 x 8) x 128 37.6 -> 35.8 us)
template <typename T, int VW, int NU, bool NORM>
__global__ void __launch_bounds__(32 * kAppendWarps, kAppendCtas) append_kernel(const AppendArgs a, const AppendPlan P) {
    const int lane = threadIdx.x & 31;
    const int D = a.c.head_dim, half = a.rot >> 1;
    const int l = lane & ((1 << P.lg) - 1), hp = 32 >> P.lg, group = lane >> P.lg;
    const int n_kv = a.c.n_kv_heads, n_qk = a.n_heads + n_kv, H = n_qk + n_kv;
    const uint32_t me = blockIdx.x * kAppendWarps + (threadIdx.x >> 5), n = (uint32_t)a.n_tok, step = (uint32_t)P.tok_step;
    uint32_t tok = me / (uint32_t)P.parts;
    const int part = (int)(me - tok * P.parts);
    if (tok >= min(n, step)) return;  // warp-uniform

    // the lane's units: channel starts of their two vectors
    int c0[NU], c1[NU];
#pragma unroll
    for (int k = 0; k < NU; ++k) {
        const int u = l + (k << P.lg);
        if (u < P.pair_units) {
            c0[k] = a.interleaved ? 2 * u * VW : u * VW;
            c1[k] = a.interleaved ? c0[k] + VW : half + u * VW;
        } else {
            c0[k] = u < P.units ? a.rot + (u - P.pair_units) * 2 * VW : D;
            c1[k] = c0[k] + VW;
        }
    }
    // the lane's heads: where their channels of the next token are, and where they go but for the token's or slot's offset
    const T* src[kAhead];
    int64_t src_step[kAhead];
    T* dst[kAhead];
    bool is_q[kAhead], turned[kAhead], there[kAhead];  // queries; queries and keys
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        const int h = (part * kAhead + j) * hp + group;
        is_q[j] = h < a.n_heads;
        turned[j] = h < n_qk;
        there[j] = h < H;
        const HeadsView& s = is_q[j] ? a.q : turned[j] ? a.k : a.v;
        const int in_kind = h - (is_q[j] ? 0 : turned[j] ? a.n_heads : n_qk);
        src[j] = static_cast<const T*>(s.p) + tok * s.tok + in_kind * s.head;
        src_step[j] = step * s.tok;
        dst[j] = is_q[j] ? static_cast<T*>(a.out.p) + h * a.out.head
                         : static_cast<T*>(turned[j] ? a.c.k : a.c.v) + in_kind * a.c.head;
    }
    auto fetch_x = [&](Item<T, VW, NU>& y) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (there[j])
#pragma unroll
                for (int k = 0; k < NU; ++k) {
                    if (c0[k] < D) load(y.x[j][k][0], src[j] + c0[k]);
                    if (c1[k] < D) load(y.x[j][k][1], src[j] + c1[k]);
                }
            src[j] += src_step[j];
        }
    };
    auto fetch_rope = [&](Item<T, VW, NU>& y, int pos) {
        if (half == 0) return;
        const float* table = a.rope + min(max((int64_t)pos, (int64_t)0), a.max_pos - 1) * a.rot;
#pragma unroll
        for (int k = 0; k < NU; ++k) {
            const int u = l + (k << P.lg);
            if (u >= P.pair_units) continue;
            if constexpr (VW == 1) {
                y.cs[k][0] = __ldg(table + u);
                y.sn[k][0] = __ldg(table + half + u);
            } else {
#pragma unroll
                for (int e = 0; e < VW; e += 4) {
                    *reinterpret_cast<float4*>(&y.cs[k][e]) = __ldg(reinterpret_cast<const float4*>(table + u * VW + e));
                    *reinterpret_cast<float4*>(&y.sn[k][e]) = __ldg(reinterpret_cast<const float4*>(table + half + u * VW + e));
                }
            }
        }
    };

    Item<T, VW, NU> even, odd;
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
#pragma unroll
        for (int k = 0; k < NU; ++k)
#pragma unroll
            for (int v = 0; v < 2; ++v)  // channels that are never read count as zeros in a norm
                even.x[j][k][v].raw = odd.x[j][k][v].raw = typename RawVec<VW>::type{};
    fetch_x(even);
    int64_t slot = __ldg(a.slot + tok), slot1 = -1;
    int pos = half > 0 ? __ldg(a.pos + tok) : 0, pos1 = 0;
    if (n - tok > step) {
        slot1 = __ldg(a.slot + tok + step);
        if (half > 0) pos1 = __ldg(a.pos + tok + step);
    }
    fetch_rope(even, pos);
    auto item = [&](Item<T, VW, NU>& cur, Item<T, VW, NU>& nxt) {  // whether there is another
        const bool more = n - tok > step;
        int64_t slot2 = -1;
        int pos2 = 0;
        if (more) {
            fetch_x(nxt);
            if (n - tok > 2 * step) {
                slot2 = __ldg(a.slot + tok + 2 * step);
                if (half > 0) pos2 = __ldg(a.pos + tok + 2 * step);
            }
            fetch_rope(nxt, pos1);
        }

        int64_t in_cache = 0;
        bool kept = slot >= 0;
        if (kept) {
            const int64_t page = P.page_log2 >= 0 ? slot >> P.page_log2
                                 : (slot >> 32) != 0 ? slot / a.c.page_size : (int64_t)((uint32_t)slot / (uint32_t)a.c.page_size);
            kept = page < a.c.n_pages;
            if (kept) in_cache = page * a.c.page + (int)(slot - page * a.c.page_size) * a.c.tok;
        }
        if (((slot >= 0 && !kept) || (half > 0 && (pos < 0 || pos >= a.max_pos))) && part == 0 && lane == 0 && a.status)
            atomicOr(a.status, PPS_FLAG_INDEX);
        const int64_t in_out = tok * a.out.tok;

#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if ((part * kAhead + j) * hp >= H) break;  // warp-uniform
            T* to = dst[j] + (is_q[j] ? in_out : in_cache);
            const bool goes = is_q[j] || (there[j] && kept);
            auto put = [&](int k) {
                store(to + c0[k], cur.x[j][k][0]);
                if (c1[k] < D) store(to + c1[k], cur.x[j][k][1]);
            };
            if ((part * kAhead + j) * hp >= n_qk) {  // values only: copied
#pragma unroll
                for (int k = 0; k < NU; ++k)
                    if (goes && c0[k] < D) put(k);
                continue;
            }
            const T* w = static_cast<const T*>(is_q[j] ? a.q_norm : a.k_norm);
            float r = 0.0f;
            if constexpr (NORM) {  // every lane takes part in the shuffles
#pragma unroll
                for (int k = 0; k < NU; ++k) r += Wide<T, VW>(cur.x[j][k]).squares();
#pragma unroll
                for (int o = 0; o < 5; ++o)
                    if (o < P.lg) r += __shfl_xor_sync(0xffffffffu, r, 1 << o);
                r = rsqrtf(fmaf(r, P.inv_d, a.eps));
            }
            if (!goes) continue;
#pragma unroll
            for (int k = 0; k < NU; ++k) {
                if (c0[k] >= D) continue;
                if (turned[j]) {
                    Wide<T, VW> f(cur.x[j][k]);
                    if (NORM && w != nullptr) {
                        Vec<T, VW> wv[2];
                        load(wv[0], w + c0[k]);
                        load(wv[1], w + (c1[k] < D ? c1[k] : c0[k]));
                        f.scale(r, wv);
                    }
                    if (c0[k] < a.rot) f.rotate(a.interleaved != 0, cur.cs[k], cur.sn[k]);
                    f.round(cur.x[j][k]);
                }
                put(k);
                // A vector that is never read (only one of 8 channels can be) stays zero: a norm that is not finite, or a weight,
                // would make it NaN, and with it the sums of all heads that these lanes take later.
                if constexpr (NORM && VW == 8)
                    if (c1[k] >= D) cur.x[j][k][1].raw = typename RawVec<VW>::type{};
            }
        }
        tok += step;
        slot = slot1;
        slot1 = slot2;
        pos = pos1;
        pos1 = pos2;
        return more;
    };
    while (item(even, odd) && item(odd, even)) {
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
    P.page_log2 = -1;
    for (int i = 0; i < 31; ++i)
        if (a.c.page_size == 1 << i) P.page_log2 = i;
    const int64_t items = a.n_tok * P.parts, most = (int64_t)device_sm_count() * kAppendCtas * kAppendWarps;
    if (items > INT32_MAX) return cudaErrorInvalidValue;
    P.tok_step = (int)std::max<int64_t>(std::min(items, most) / P.parts, 1);
    const int64_t blocks = ((int64_t)P.tok_step * P.parts + kAppendWarps - 1) / kAppendWarps;
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
