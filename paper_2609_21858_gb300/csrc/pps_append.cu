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
//
// Into 4 bits (pps_q4.cuh).  A block's scale needs all its 16 channels, which lie in two to sixteen lanes, so a warp's keys and values go
// through shared memory as floats: lanes spread their channels there, then each lane takes a block or two, finds the scale, forms the
// codes and writes 8 bytes and 1.  A warp whose heads are all queries has none of that.  The next item's channels come through
// shared memory too (16-byte vectors): in registers they made the compiler spill, 68.8 us where an earlier form of this took 59.7 (20 warps an SM
// at 96 registers: 99).  16384 tokens of (28 + 2 x 4) heads of 128: 59.2 us (its bytes: 42; 16 bits 52.7), bound by the latency of
// 16 warps an SM (1.9 of 4 issue slots, DRAM at 52 percent).  Eight tokens with a norm: 3.7 us in a graph, a chain of loads and the division.
// The codes' way back (read_kernel) takes 10.7 us for 16 thousand slots, of 6: the slot's division, its codes and its stores stand one behind the other.
#include <algorithm>
#include <cstdint>
#include <cstring>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pps.h"
#include "pps_internal.h"
#include "pps_q4.cuh"

namespace pps {
namespace {

constexpr int kAppendWarps = 4;  // per CTA
constexpr int kAhead = 2;        // heads of a lane group in an item
constexpr int kAppendCtas = 4;   // per SM
constexpr int kRing = 2;         // items of a warp in shared memory (below; 3: 62.1 us where 2 take 59.3)
// What an item with keys or values takes where they become 4 bits, to one of queries alone.  16384 tokens of (28 + 2 x 4) heads of 128
// channels: 62.0 us at 1.1, 59.3 at 1.2, 60.4 at 1.3, 62.5 at 1.4 (52.7 into a cache of 16 bits).  No other shape was measured.
constexpr double kHeavy = 1.2;
// a block's 16 channels in shared memory, 80 bytes apart: eight lanes' 16-byte reads touch all banks
constexpr int kBlockFloats = 20;

struct AppendPlan {
    int lg;          // log2 of the lanes per head
    int parts;       // items per token
    int tok_step;    // tokens in work at a time: tok_step x parts warps
    int light, light_step;  // of 4 bits: the first parts, of queries alone, and their tokens in work at a time (else 0)
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
    // FUSED: a product's rounding may be left out of a sum.  Never of what becomes 4 bits, where a last bit can decide a code: the
    // values are those of products and sums rounded one by one, and so operations of one channel, as the compiler joins packed products
    // and sums of the same rounding (16384 tokens of (28 + 2 x 4) heads of 128 channels in fp16: one query's channel in 8500 was a bit off).
    template <bool FUSED>
    __device__ __forceinline__ void rotate(bool interleaved, const float (&cs)[VW], const float (&sn)[VW]) {
        if (VW > 1 && interleaved) {
#pragma unroll
            for (int v = 0; v < 2; ++v)
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    const float c = cs[(v * kN + i) % VW], s = sn[(v * kN + i) % VW];
                    float p, q;
                    unpack2(f[v][i], p, q);
                    f[v][i] = FUSED ? pack2(p * c - q * s, p * s + q * c)
                                    : pack2(__fsub_rn(__fmul_rn(p, c), __fmul_rn(q, s)), __fadd_rn(__fmul_rn(p, s), __fmul_rn(q, c)));
                }
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                const uint64_t c = pack2(cs[2 * i], cs[(2 * i + 1) % VW]), s = pack2(sn[2 * i], sn[(2 * i + 1) % VW]);
                const uint64_t p = f[0][i], q = f[1][i];
                if constexpr (FUSED) {
                    f[0][i] = sub2(mul2(p, c), mul2(q, s));
                    f[1][i] = fma2(p, s, mul2(q, c));
                } else {
                    float x[2], y[2], cc[2], ss[2], a[2], b[2];
                    unpack2(p, x[0], x[1]);
                    unpack2(q, y[0], y[1]);
                    unpack2(c, cc[0], cc[1]);
                    unpack2(s, ss[0], ss[1]);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        a[e] = __fsub_rn(__fmul_rn(x[e], cc[e]), __fmul_rn(y[e], ss[e]));
                        b[e] = __fadd_rn(__fmul_rn(x[e], ss[e]), __fmul_rn(y[e], cc[e]));
                    }
                    f[0][i] = pack2(a[0], a[1]);
                    f[1][i] = pack2(b[0], b[1]);
                }
            }
        }
    }
    // in 32 bits to a head's blocks of 16 in shared memory, from channel c0 and channel c1 on
    __device__ __forceinline__ void spread(float* head, int c0, int c1, bool both) const {
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            if (v == 1 && !both) break;
            const int c = v ? c1 : c0;
            float* to = head + (c >> 4) * kBlockFloats + (c & 15);
            float x[VW > 1 ? VW : 2];
#pragma unroll
            for (int i = 0; i < kN; ++i) unpack2(f[v][i], x[2 * i], x[2 * i + 1]);
            if constexpr (VW == 1)
                *to = x[0];
            else
#pragma unroll
                for (int i = 0; i < VW; i += 4) *reinterpret_cast<float4*>(to + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
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
// Q4: keys and values go to a cache in 4 bits.  An item's keys and values pass through shared memory in 32 bits, whatever the
// rotation's pairs are, and lanes then have a block of 16 channels each: its scale, its codes, an 8-byte store of codes.
template <typename T, int VW, int NU, bool NORM, bool Q4>
__global__ void __launch_bounds__(32 * kAppendWarps, kAppendCtas) append_kernel(const AppendArgs a, const AppendPlan P) {
    constexpr int kBlocks = 64;  // of an item: 32 lanes x 16 channels x kAhead
    __shared__ __align__(16) float s_x[Q4 ? kAppendWarps : 1][Q4 ? kBlocks * kBlockFloats : 4];
    // of 4 bits, channels come through shared memory, a lane's own sixteen bytes at a time: an item in use and kRing - 1 on their way
    constexpr bool RING = Q4 && VW == 8;
    __shared__ uint4 s_ring[RING ? kAppendWarps : 1][RING ? kRing : 1][2 * kAhead][RING ? 32 : 1];
    const int lane = threadIdx.x & 31;
    const int D = a.c.head_dim, half = a.rot >> 1;
    const int l = lane & ((1 << P.lg) - 1), hp = 32 >> P.lg, group = lane >> P.lg;
    const int n_kv = a.c.n_kv_heads, n_qk = a.n_heads + n_kv, H = n_qk + n_kv;
    const uint32_t me = blockIdx.x * kAppendWarps + (threadIdx.x >> 5), n = (uint32_t)a.n_tok;
    // the warp's first token, how many tokens further its next one is, and its part of all of them
    const uint32_t light = Q4 ? (uint32_t)(P.light * P.light_step) : 0u, of = Q4 && me < light ? (uint32_t)P.light : (uint32_t)(P.parts - P.light);
    const uint32_t step = Q4 && me < light ? (uint32_t)P.light_step : (uint32_t)P.tok_step, mine = Q4 && me >= light ? me - light : me;
    uint32_t tok = mine / of;
    const int part = (int)(mine - tok * of) + (Q4 && me >= light ? P.light : 0);
    if constexpr (Q4) {
        pdl_wait();
        pdl_launch_dependents();
    }
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
    // the lane's blocks of an item's keys and values: where their codes and scales go but for the slot's offset
    const int n_blk = Q4 ? D / 16 : 0;
    uint8_t *codes[2] = {}, *scales[2] = {};
    float inv[2] = {};
    float* const spread_at = s_x[Q4 ? threadIdx.x >> 5 : 0];
    const bool holds = Q4 && (part + 1) * kAhead * hp > a.n_heads;  // warp-uniform: keys or values among the item's heads
    if constexpr (Q4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int b = lane + 32 * i, hs = b / n_blk, h = part * kAhead * hp + hs;
            if (hs >= kAhead * hp || h < a.n_heads || h >= H) continue;
            const bool key = h < n_qk;
            const int in_kind = h - (key ? a.n_heads : n_qk), blk = b - hs * n_blk;
            codes[i] = static_cast<uint8_t*>(key ? a.c.k : a.c.v) + in_kind * a.c.head + 8 * blk;
            scales[i] = (key ? a.q4.ks : a.q4.vs) + in_kind * a.q4.head + blk;
            const float* unit = key ? a.q4.k_unit : a.q4.v_unit;
            inv[i] = unit ? __frcp_rn(__ldg(unit + in_kind)) : 1.0f;
        }
    }
    uint4(*const ring)[2 * kAhead][RING ? 32 : 1] = s_ring[RING ? threadIdx.x >> 5 : 0];
    uint32_t to_fill = 0, to_use = 0;
    auto fetch_ring = [&](bool more) {  // the channels of the next item that is not on its way; a group of copies in any case
        if (more) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (there[j])
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
                        const int c = v ? c1[0] : c0[0];
                        if (c < D)
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(&ring[to_fill][2 * j + v][lane])),
                                         "l"(src[j] + c)
                                         : "memory");
                    }
                src[j] += src_step[j];
            }
            to_fill = to_fill + 1 == kRing ? 0 : to_fill + 1;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto take_ring = [&](Item<T, VW, NU>& y) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 2) : "memory");
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
#pragma unroll
            for (int v = 0; v < 2; ++v)
                *reinterpret_cast<uint4*>(&y.x[j][0][v]) = there[j] && (v ? c1[0] : c0[0]) < D ? ring[to_use][2 * j + v][lane] : make_uint4(0, 0, 0, 0);
        to_use = to_use + 1 == kRing ? 0 : to_use + 1;
    };
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
    if constexpr (RING) {
#pragma unroll
        for (int i = 0; i < kRing - 1; ++i) fetch_ring(n - tok > i * step);
    } else
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
        if constexpr (RING) {
            take_ring(cur);
            fetch_ring(n - tok > (kRing - 1) * step);
        }
        if (more) {
            if constexpr (!RING) fetch_x(nxt);
            if (n - tok > 2 * step) {
                slot2 = __ldg(a.slot + tok + 2 * step);
                if (half > 0) pos2 = __ldg(a.pos + tok + 2 * step);
            }
            fetch_rope(nxt, pos1);
        }

        int64_t in_cache = 0, in_scales = 0;
        bool kept = slot >= 0;
        if (kept) {
            const int64_t page = P.page_log2 >= 0 ? slot >> P.page_log2
                                 : (slot >> 32) != 0 ? slot / a.c.page_size : (int64_t)((uint32_t)slot / (uint32_t)a.c.page_size);
            kept = page < a.c.n_pages;
            if (kept) {
                const int in_page = (int)(slot - page * a.c.page_size);
                in_cache = page * a.c.page + in_page * a.c.tok;
                if constexpr (Q4) in_scales = page * a.q4.page + in_page * a.q4.tok;
            }
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
                    if (goes && c0[k] < D) {
                        if constexpr (Q4)
                            Wide<T, VW>(cur.x[j][k]).spread(spread_at + (j * hp + group) * n_blk * kBlockFloats, c0[k], c1[k], c1[k] < D);
                        else
                            put(k);
                    }
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
                    if (c0[k] < a.rot) f.template rotate<!Q4>(a.interleaved != 0, cur.cs[k], cur.sn[k]);
                    if (!Q4 || is_q[j])
                        f.round(cur.x[j][k]);
                    else
                        f.spread(spread_at + (j * hp + group) * n_blk * kBlockFloats, c0[k], c1[k], c1[k] < D);
                } else if constexpr (Q4)
                    Wide<T, VW>(cur.x[j][k]).spread(spread_at + (j * hp + group) * n_blk * kBlockFloats, c0[k], c1[k], c1[k] < D);
                if (!Q4 || is_q[j]) put(k);
                // A vector that is never read (only one of 8 channels can be) stays zero: a norm that is not finite, or a weight,
                // would make it NaN, and with it the sums of all heads that these lanes take later.
                if constexpr (NORM && VW == 8)
                    if (c1[k] >= D) cur.x[j][k][1].raw = typename RawVec<VW>::type{};
            }
        }
        if constexpr (Q4) {
            if (holds) {
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (kept && codes[i] != nullptr) {
                        const float* x = spread_at + (lane + 32 * i) * kBlockFloats;
                        uint64_t z[8];
#pragma unroll
                        for (int e = 0; e < 8; e += 2) *reinterpret_cast<ulonglong2*>(z + e) = *reinterpret_cast<const ulonglong2*>(x + 2 * e);
                        uint32_t scale;
                        const uint2 c = q4::quantise(z, inv[i], scale);
                        *reinterpret_cast<uint2*>(codes[i] + in_cache) = c;
                        scales[i][in_scales] = (uint8_t)scale;
                    }
                __syncwarp();
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
    P.light = P.light_step = 0;
    const bool norm = a.q_norm != nullptr || a.k_norm != nullptr, bits4 = a.q4.ks != nullptr;
    if (bits4) {  // parts with keys or values take longer than those of queries alone: more warps have them
        P.light = a.n_heads / per_item;
        const double heavy = kHeavy * (P.parts - P.light);
        P.light_step = (int)std::min<int64_t>(std::max<int64_t>((int64_t)((double)most / (P.light + heavy)), 1), a.n_tok);
        P.tok_step = (int)std::min<int64_t>(std::max<int64_t>((int64_t)(kHeavy * (double)most / (P.light + heavy)), 1), a.n_tok);
    }
    const int64_t blocks = ((int64_t)P.tok_step * (P.parts - P.light) + (int64_t)P.light * P.light_step + kAppendWarps - 1) / kAppendWarps;
    auto kernel = bits4 ? (norm ? append_kernel<T, VW, NU, true, true> : append_kernel<T, VW, NU, false, true>)
                        : (norm ? append_kernel<T, VW, NU, true, false> : append_kernel<T, VW, NU, false, false>);
    // A few CTAs may come while what is before them ends.  Many may not: they would find SMs whose shared memory is divided for that
    // other kernel, and the one wave that they are would become two (append, then read of 16384 tokens, on an earlier form: 72 us, 80 to 91 that way).
    if (bits4 && blocks <= device_sm_count()) return launch_pdl(kernel, dim3((unsigned)blocks), dim3(32 * kAppendWarps), 0, st, a, P);
    kernel<<<(unsigned)blocks, 32 * kAppendWarps, 0, st>>>(a, P);
    return cudaGetLastError();
}

template <typename T>
cudaError_t by_width(const AppendArgs& a, cudaStream_t st) {
    // the widest vectors that every address and the rotation's halves allow
    uint64_t bits = 0;  // byte addresses and element strides, doubled to bytes
    for (const HeadsView* h : {&a.q, &a.k, &a.v, &a.out})
        bits |= reinterpret_cast<uintptr_t>(h->p) | (uint64_t)h->tok * 2 | (uint64_t)h->head * 2;
    if (a.q4.ks == nullptr) {
        bits |= reinterpret_cast<uintptr_t>(a.c.k) | reinterpret_cast<uintptr_t>(a.c.v);
        bits |= (uint64_t)(a.c.page | a.c.tok | a.c.head) * 2;
    }
    bits |= reinterpret_cast<uintptr_t>(a.q_norm) | reinterpret_cast<uintptr_t>(a.k_norm);
    const bool table = a.rot == 0 || (reinterpret_cast<uintptr_t>(a.rope) & 15) == 0;
    if (table && bits % 16 == 0 && a.rot % 16 == 0) return launch<T, 8, 1>(a, st);
    if (table && bits % 8 == 0 && a.rot % 8 == 0) return launch<T, 4, 1>(a, st);
    return launch<T, 1, 4>(a, st);
}

// Values of cache slots: a thread has a block of 16 channels of a head, of keys and of values, in every step-th slot.
template <typename T>
__global__ void __launch_bounds__(256) read_kernel(const ReadArgs a, int per_slot, int step) {
    const int n_blk = a.c.head_dim / 16;
    const int in_cta = 256 / per_slot, sl = threadIdx.x / per_slot, task = threadIdx.x - sl * per_slot;
    // per_slot: blocks of a slot that a CTA takes at a time; blockIdx.y: which of them
    const int b = blockIdx.y * per_slot + task, head = b / n_blk, blk = b - head * n_blk;
    pdl_wait();
    pdl_launch_dependents();
    if (sl >= in_cta || head >= a.c.n_kv_heads) return;
    const float ku = a.q4.k_unit ? __ldg(a.q4.k_unit + head) : 1.0f, vu = a.q4.v_unit ? __ldg(a.q4.v_unit + head) : 1.0f;
    for (int64_t i = (int64_t)blockIdx.x * in_cta + sl; i < a.n; i += step) {
        const int64_t slot = __ldg(a.slot + i), page = slot < 0 ? -1 : slot / a.c.page_size;
        const bool there = page >= 0 && page < a.c.n_pages;
        if (page >= a.c.n_pages && b == 0 && a.status) atomicOr(a.status, PPS_FLAG_INDEX);
        const int in_page = there ? (int)(slot - page * a.c.page_size) : 0;
        const int64_t at = page * a.c.page + in_page * a.c.tok + head * a.c.head + 8 * blk;
        const int64_t st = page * a.q4.page + in_page * a.q4.tok + head * a.q4.head + blk;
        uint2 c[2] = {};
        uint32_t s[2] = {};
        if (there) {
            c[0] = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.c.k) + at);
            c[1] = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.c.v) + at);
            s[0] = a.q4.ks[st];
            s[1] = a.q4.vs[st];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float su = q4::scale_float(s[h]) * (h ? vu : ku);
            const uint64_t su2 = pack2(su, su);
            uint32_t w[8], o[8];
            uint32_t(&w0)[4] = *reinterpret_cast<uint32_t(*)[4]>(w);
            uint32_t(&w1)[4] = *reinterpret_cast<uint32_t(*)[4]>(w + 4);
            q4::widen8(c[h].x, w0);
            q4::widen8(c[h].y, w1);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = narrow<T>(mul2(widen<__half>(w[e]), su2));
            const HeadsView& out = h ? a.v : a.k;
            uint4* to = reinterpret_cast<uint4*>(static_cast<T*>(out.p) + i * out.tok + head * out.head + 16 * blk);
            to[0] = make_uint4(o[0], o[1], o[2], o[3]);
            to[1] = make_uint4(o[4], o[5], o[6], o[7]);
        }
    }
}

}  // namespace

cudaError_t launch_kv_read(const ReadArgs& a, int dtype, cudaStream_t stream) {
    const int64_t blocks = (int64_t)a.c.n_kv_heads * (a.c.head_dim / 16);
    const int per_slot = (int)std::min<int64_t>(blocks, 256), in_cta = 256 / per_slot;
    const int64_t rounds = (blocks + per_slot - 1) / per_slot;
    if (rounds > 65535) return cudaErrorInvalidValue;
    const int64_t ctas = std::min<int64_t>((a.n + in_cta - 1) / in_cta, std::max<int64_t>((int64_t)device_sm_count() * 8 / rounds, 1));
    const dim3 grid((unsigned)ctas, (unsigned)rounds);
    const int step = (int)(ctas * in_cta);
    return launch_pdl(dtype == PPS_BF16 ? read_kernel<__nv_bfloat16> : read_kernel<__half>, grid, dim3(256), 0, stream, a, per_slot, step);
}

cudaError_t launch_kv_append(const AppendArgs& a, int dtype, cudaStream_t stream) {
    return dtype == PPS_BF16 ? by_width<__nv_bfloat16>(a, stream) : by_width<__half>(a, stream);
}

}  // namespace pps
