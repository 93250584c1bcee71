// pps_attention_q4.cu -- attention of the newest tokens of each sequence over a paged cache held in 4 bits (pps_q4.cuh), sm_103a.
//
//   out[i] = v_unit sum_j w_j v_j / sum_j w_j,   w_j = exp(scale k_unit q_i . k_j)   over the keys j that row i sees
//
// Rows.  The tokens of a sequence and the heads that share a key head are packed into rows, token after token; a row block has
// R = 8 NT of them (NT 1 or 2).
//
// Few rows.  A key's 128 channels are 72 bytes, and what a decoding step has to do per byte of them is to widen it: both
// products run on registers, without a way through shared memory for what was widened.  A warp takes 64 keys at a time, 16 by 16:
//   S^T = K Q^T  (m16n8k16, m: keys, n: rows).  Lane (g, t) of the warp reads a quarter of key g's codes, t-th from the left, and
//                takes them as the operand's elements whatever channels these are: the queries are read in the same order;
//   O^T += V^T P^T (m: channels, n: rows, k: keys).  Lane (g, t) reads the g-th eighth of the codes of keys 2t, 2t + 1; nibbles of
//                two keys are put together into bytes, which become pairs of halves along the keys; a transposing move turns S^T into
//                the operand P^T.
// Codes times scales are exact halves.  Queries in bf16 are brought to halves by a power of two per row, exactly but for
// channels below 2^-31 of the row's largest.  Weights are rounded to halves (2^-11 of each); sums are formed before rounding,
// in 32 bits, and the softmax is the running one with the rescaling left out while a maximum rises by less than 2^kLazy4.
// The warps of a CTA take the units of a segment in turn, each through a ring of its own (a unit on its way while one is in use),
// and join at its end.
// What bounds it: with many keys the latency of those conversions and products in 12 warps an SM (64 sequences of 2000 to 8000 keys: 80 us, 4.7
// TB/s, 61 percent of DRAM's time and 2.1 instructions a clock of 4; the first form, 32 keys at a time with codes by lanes' copies, took 98), with few the start,
// the plan and the join's launch (one sequence of 900 keys: 9.6 us).  Three CTAs of four warps to an SM leave 168 registers.
// A wait that gives up ends its CTA: its warps' copies on their way are waited for, and nothing more is written.
//
// Many rows (trees, chunks).  The 128-row tiles of pps_attn_tiles.cuh on the 5th-generation tensor cores: six warps copy a tile's codes
// and scales into shared memory ahead of the products, widen them (64 conversions and as many multiplications a lane for 32 keys of
// 128 channels) and write the halves where TMA would have put them.  Queries in bf16 become halves in a launch before it, at the same
// power of two per row.  64 trees of 41 nodes: 220 us, of which that launch is some 8; a cache of 16 bits takes 180.  As there, what bounds it is
// the softmax's latency: two warps a scheduler, each with whole rows, whose steps (wait, load, maximum, exponentials, store) stand one
// behind the other.  The tensor cores are busy 37 percent of the time and 1.4 instructions issue a clock of 4; which part of the
// difference the widening warps make has not been measured.
//
// Work split.  The line of pps_attn.cuh.
#include <atomic>
#include <cstring>

#include "pps_attn_tiles.cuh"

namespace pps {
namespace {

constexpr int kWarps4 = 4, kThreads4 = 32 * kWarps4;
constexpr int kUnit = 64;         // keys that a warp takes at a time
constexpr int kGroups = kUnit / 16;
constexpr int kStages4 = 2;       // units of a warp, on their way or in use
constexpr int few_ctas(int nt) { return nt == 1 ? 3 : 2; }  // per SM: 168 or 255 registers
constexpr int kMaxCtas4 = 640;
constexpr auto kFetch4 = CU_TENSOR_MAP_L2_PROMOTION_L2_64B;  // what a miss brings into L2: a row (520000 keys: 68 us, 128 bytes 70, 256 71)
// Key tiles that an item's start and end cost: few rows (seven batches of 8 to 256 sequences, 1500 to 30000 keys: 4 is 1 to 5 percent
// faster than 2, and equal to 3, 5 and 6 within 3), and tiles, which take longer each than those of 16 bits (six of trees, four of chunks: 3
// is 3 to 5 percent faster than 6, within 1 of 4; 64 trees 220 us, 2: 238).
constexpr int kFix4 = 4, kFixTiles4 = 3;
constexpr int kLeast4 = 1;
constexpr float kLazy4 = 8.0f;    // log2 of the rise of a maximum that nothing is rescaled for
constexpr float kShift4 = 6.0f;   // log2 of a factor on all weights: 2^(8 + 6) is below fp16's largest number
constexpr int kQBits = 14;        // a bf16 row's largest channel lies in [2^14, 2^15) as a half
// Rows of a sequence and key head, on average, up to which the kernel of few rows takes a call (64 sequences of 1000 to 4000 keys, 32
// over 8 heads: 8 rows 54 us against 149 on tiles, 16 rows 78 against 150, 32 rows 138 against 152, 48 rows 197 against 157).  All of these are batches
// of one kind.  Of a batch of both kinds one gets the wrong kernel, whatever the mean says: 63 single tokens (63 us alone) with a chunk
// of 300 (48 alone) take 183 us here, with a chunk of 2048 (139 alone) 381 on tiles; two calls take the sum.
constexpr int kFewRows = 32;

// The power of two that brings a row in bf16 whose largest finite magnitude has the bits `top` to halves.
__device__ __forceinline__ int halving(uint32_t top) { return top == 0 ? 0 : min(kQBits + 127 - (int)(top >> 7), 126); }
__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float((uint32_t)(127 + k) << 23); }

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {  // c = a b
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// A warp's ring in shared memory: stages of kUnit keys, each their codes, the values' codes, and the scales of both, row after row.
template <int DC>
struct Stage {
    static constexpr int kRow = DC / 2, kScales = DC / 16;  // bytes of a key
    static constexpr int kV = kUnit * kRow, kKs = 2 * kV, kVs = kKs + kUnit * kScales, kBytes = kVs + kUnit * kScales;
};

// How a cache lies.  kByHead: all DC channels are there, 16 keys in a row share their page, and a page's rows of a head follow one
// another, from 16-byte boundaries on (a page laid out head by head): a stage's codes are eight bulk copies, its scales sixteen bytes a
// lane.  kByToken: the same, but rows are apart: the copies are boxes of 16 rows, scales a row a lane.  kAnyHow: anything else; four
// lanes copy a row of codes and a lane a row's scales, each with a look at the key's page and length.  (One sequence of 130001 and 520000
// keys over 4 heads of 128, back to back in a graph: 25 and 65 us head by head, 27 and 68 token by token, which kAnyHow reads in 34 and 104.)
enum Lie { kAnyHow, kByToken, kByHead };

template <typename T, int DC, int NT, Lie LIE>
__global__ void __launch_bounds__(kThreads4, few_ctas(NT)) few_rows_kernel(const __grid_constant__ CUtensorMap tmK,
                                                                           const __grid_constant__ CUtensorMap tmV, const AttnArgs a, const Q4View z,
                                                                           const AttnPlan P) {
    constexpr bool DENSE = LIE != kAnyHow;
    using S = Stage<DC>;
    constexpr int R = 8 * NT, RS = DC + 4;  // a row's floats in shared memory: 4 modulo 16, so that lanes (g, t) touch all banks
    __shared__ int64_t s_sum[kWarps4];
    __shared__ Start s_start;
    __shared__ float2 s_ml[kWarps4][R];
    __shared__ float2 s_tot[R];
    __shared__ uint64_t s_bar[kWarps4][kStages4];
    __shared__ int s_abort;
    extern __shared__ __align__(128) uint8_t s_ring[];  // [kWarps4][kStages4] stages; between segments:
    float* const s_o = reinterpret_cast<float*>(s_ring);  // [kWarps4][R][RS]
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x, g = lane >> 2, t = lane & 3;
    if (DENSE && tid == 0) {
        for (int i = 0; i < kWarps4 * kStages4; ++i) mbar_init(smem_u32(&s_bar[0][0] + i), 1);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();
    pdl_launch_dependents();
    int64_t c0, c1;
    const int64_t share = find_share<kThreads4>(a, P, s_sum, &s_start, c0, c1);
    __syncthreads();
    if (c0 >= c1) return;
    const int least = (int)min(max(share / 8, (int64_t)1), (int64_t)kLeast4);
    Walk W(P, s_start, c0, c1, least);
    const int D = DENSE ? DC : a.c.head_dim;
    // what of the lane's scale bytes counts
    const bool k_there = DENSE || t * (DC / 4) < D, k_half = DENSE || t * (DC / 4) + 16 < D, v_there = DENSE || g * (DC / 8) < D;
    const uint32_t k_mask = (k_there ? 0xffu : 0u) | (DC == 128 && k_half ? 0xff00u : 0u), v_mask = v_there ? 0xffu : 0u;
    uint8_t* const my_ring = s_ring + warp * kStages4 * S::kBytes;
    const uint32_t ring_at = smem_u32(my_ring), bar_at = smem_u32(&s_bar[warp][0]);
    const bool wide = ((reinterpret_cast<uintptr_t>(a.c.k) | reinterpret_cast<uintptr_t>(a.c.v) | (uintptr_t)a.c.page | (uintptr_t)a.c.tok |
                        (uintptr_t)a.c.head | (uintptr_t)(D / 2)) & 15) == 0;
    // of a bulk copy, lane 2 G + kind (keys, values): the codes of the G-th 16 keys; scales come sixteen bytes a lane
    const int kind = lane & 1, G16 = lane >> 1 & (kGroups - 1);
    const uint8_t* const part = static_cast<const uint8_t*>(kind ? a.c.v : a.c.k);
    const uint32_t part_at = (kind ? S::kV : 0) + 16 * G16 * S::kRow;
    constexpr int kScaleLanes = 16 * S::kScales / 16;  // of 16 keys
    const int Gs = lane / kScaleLanes & (kGroups - 1);
    // key by key: four lanes copy a row of codes; a lane has the scales of keys lane, + 32
    const int64_t quarter = (lane >> 2) * a.c.tok + (lane & 3) * (DC / 8);
    const bool q_there = (lane & 3) * (DC / 4) < D, q_half = (lane & 3) * (DC / 4) + 16 < D;
    uint32_t to_fill = 0, to_use = 0, phase = 0;  // the stage that is filled next, used next, and the phase of the latter's barrier

    while (W.next(a, P)) {
        const int kvh = W.heads / P.nsub, sub = W.heads - kvh * P.nsub;
        const int gs = min(P.gs, P.group - sub * P.gs);
        const int head0 = kvh * P.group + sub * P.gs;
        const int len = W.q.len, prefix = len - W.q.n;
        const float ku = z.k_unit ? __ldg(z.k_unit + kvh) : 1.0f, vu = z.v_unit ? __ldg(z.v_unit + kvh) : 1.0f;
        const int plain = a.mask ? prefix : prefix + W.i0 + 1;  // keys below it are seen by every row
        const int end = a.mask ? len : prefix + W.i0 + W.ntok;  // keys from it on by none
        const int first = W.t0 * kTileKeys, last = min(W.t1 * kTileKeys, end);
        const int32_t* table = a.pages + (int64_t)W.s * a.pages_stride;

        // the lane's page of the unit from key k0 on: of 16 keys G16, or of eight keys, lane modulo 8
        auto page_of = [&](int k0) {
            const int k = k0 + (DENSE ? 16 * G16 : 8 * (lane & 7));
            return k < last ? __ldg(table + (k >> P.page_log2)) : 0;
        };
        const uint8_t* const my_part = part + kvh * a.c.head;
        const int64_t my_scales = kvh * z.head + 16 * (lane % kScaleLanes);
        uint32_t paged = 0;  // a bit per 16 keys of the units on their way, the newest lowest: their page is there
        auto fill = [&](int k0, int page) {
            const uint32_t to = ring_at + to_fill * S::kBytes, full = bar_at + 8 * to_fill;
            to_fill = to_fill + 1 == kStages4 ? 0 : to_fill + 1;
            if constexpr (DENSE) {
                const int k = k0 + 16 * G16, in_page = k & (a.c.page_size - 1);
                const bool key = k < last, good = key && (uint32_t)page < (uint32_t)a.c.n_pages;  // (a missing page reads as zeros)
                if (key && !good && a.status) atomicOr(a.status, PPS_FLAG_INDEX);
                const uint32_t who = __ballot_sync(0xffffffffu, good && kind == 0) & ((1u << 2 * kGroups) - 1u);
                paged = paged << 2 * kGroups | who;
                if (lane == 0) {
                    if (who)
                        mbar_expect_tx(full, __popc(who) * (16 * 2 * S::kRow));
                    else
                        mbar_arrive(full);
                }
                __syncwarp();
                if constexpr (LIE == kByHead) {
                    if (lane < 2 * kGroups && good) bulk_load(to + part_at, my_part + page * a.c.page + in_page * S::kRow, 16 * S::kRow, full);
                    const int p = __shfl_sync(0xffffffffu, page, 2 * Gs);
                    if (lane < kGroups * kScaleLanes && (who >> 2 * Gs & 1u)) {
                        const int64_t at = p * z.page + ((k0 + 16 * Gs) & (a.c.page_size - 1)) * S::kScales + my_scales;
                        copy_async<16>(to + S::kKs + 16 * lane, z.ks + at);
                        copy_async<16>(to + S::kVs + 16 * lane, z.vs + at);
                    }
                } else {
                    if (lane < 2 * kGroups && good) tma_load_4d(to + part_at, kind ? &tmV : &tmK, full, 0, in_page, kvh, page);
#pragma unroll
                    for (int i = 0; i < kUnit / 32; ++i) {
                        const int G = 2 * i + (lane >> 4), p = __shfl_sync(0xffffffffu, page, 2 * G);
                        if (!(who >> 2 * G & 1u)) continue;
                        const int64_t at = p * z.page + ((k0 + 32 * i + lane) & (a.c.page_size - 1)) * z.tok + kvh * z.head;
                        const uint32_t scales = to + S::kKs + (32 * i + lane) * S::kScales;
                        copy_async<S::kScales>(scales, z.ks + at);
                        copy_async<S::kScales>(scales + S::kVs - S::kKs, z.vs + at);
                    }
                }
            } else {
                if (k0 + 8 * (lane & 7) < last && (uint32_t)page >= (uint32_t)a.c.n_pages) {  // reads as zeros
                    if (a.status) atomicOr(a.status, PPS_FLAG_INDEX);
                    page = -1;
                }
#pragma unroll
                for (int i = 0; i < kUnit / 8; ++i) {  // codes
                    const int p = __shfl_sync(0xffffffffu, page, i), k = k0 + 8 * i, in_page = k & (a.c.page_size - 1);
                    if (p < 0 || k + (lane >> 2) >= last || !q_there) continue;
                    const int64_t at = p * a.c.page + in_page * a.c.tok + kvh * a.c.head + quarter;
                    const uint32_t row = to + (8 * i + (lane >> 2)) * S::kRow + (lane & 3) * (DC / 8);
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
                        const uint8_t* src = static_cast<const uint8_t*>(v ? a.c.v : a.c.k) + at;
                        if (DC == 128 && wide)
                            copy_async<16>(row + v * S::kV, src);
                        else {
                            copy_async<8>(row + v * S::kV, src);
                            if (DC == 128 && q_half) copy_async<8>(row + v * S::kV + 8, src + 8);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < kUnit / 32; ++i) {
                    const int key = lane + 32 * i, k = k0 + key, p = __shfl_sync(0xffffffffu, page, key >> 3);
                    const uint32_t scales = to + S::kKs + key * S::kScales;
                    if (k < last && p >= 0) {
                        const int64_t at = p * z.page + (k & (a.c.page_size - 1)) * z.tok + kvh * z.head;
#pragma unroll
                        for (int c = 0; c < DC / 64; ++c)
                            if (64 * c < D) {
                                copy_async<4>(scales + 4 * c, z.ks + at + 4 * c);
                                copy_async<4>(scales + S::kVs - S::kKs + 4 * c, z.vs + at + 4 * c);
                            }
                    } else {
#pragma unroll
                        for (int c = 0; c < DC / 64; ++c) {  // scales of zero, whatever the codes
                            asm volatile("st.shared.b32 [%0], %1;" ::"r"(scales + 4 * c), "r"(0) : "memory");
                            asm volatile("st.shared.b32 [%0], %1;" ::"r"(scales + S::kVs - S::kKs + 4 * c), "r"(0) : "memory");
                        }
                    }
                }
            }
        };
        auto close = [&]() {  // a group of copies per unit, with or without any
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        constexpr int kStep = kUnit * kWarps4, kAhead4 = kStages4 - 1;
        int k0 = first + warp * kUnit;
        const int k_start = k0;
        int pages = k0 < last ? page_of(k0) : 0;
#pragma unroll
        for (int i = 0; i < kAhead4; ++i) {
            const int k = k_start + i * kStep, p = pages;
            pages = page_of(k + kStep);
            if (k < last)
                fill(k, p);
            else
                paged <<= 2 * kGroups;
            close();
        }
        // ---- queries: row 8 nt + g, the channels of quarter t, as halves
        uint32_t qf[NT][DC / 8];
        float row_sc[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = 8 * nt + g, tok = row / P.gs, h = row - tok * P.gs;
            const bool valid = tok < W.ntok && h < gs;
            const T* src = static_cast<const T*>(a.q.p) + (int64_t)(W.q.off + W.i0 + tok) * a.q.tok + (head0 + h) * a.q.head + t * (DC / 4);
            uint4 raw[DC / 32];
#pragma unroll
            for (int i = 0; i < DC / 32; ++i) {
                raw[i] = make_uint4(0, 0, 0, 0);
                if (valid && t * (DC / 4) + 8 * i < D) raw[i] = __ldg(reinterpret_cast<const uint4*>(src) + i);
            }
            const uint32_t* x = reinterpret_cast<const uint32_t*>(raw);
            row_sc[nt] = P.sc * ku;  // (kept from zero: scores of zero, equal weights, are what the smallest normal number gives too)
            if constexpr (Half<T>::kType == 0) {
#pragma unroll
                for (int i = 0; i < DC / 8; ++i) qf[nt][i] = x[i];
            } else {
                uint32_t top = 0;  // the largest finite magnitude
#pragma unroll
                for (int i = 0; i < DC / 8; ++i) {
                    const uint32_t lo = x[i] & 0x7fffu, hi = x[i] >> 16 & 0x7fffu;
                    top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
                }
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const int k = halving(top);
                const float f = power_of_two(k);
                row_sc[nt] = fminf(row_sc[nt] * power_of_two(-k), FLT_MAX);
#pragma unroll
                for (int i = 0; i < DC / 8; ++i)
                    qf[nt][i] = Half<__half>::pack(__uint_as_float(x[i] << 16) * f, __uint_as_float(x[i] & 0xffff0000u) * f);
            }
        }
        // of the lane's rows 8 nt + 2t, + 1 (an odd index: the second)
        // m: maximum in use; limit: a score past it raises it; neg: what is added to a score times sc
        float sc[2 * NT], m[2 * NT], l[2 * NT], limit[2 * NT], neg[2 * NT];
#pragma unroll
        for (int r = 0; r < 2 * NT; ++r) {
            sc[r] = fmaxf(__shfl_sync(0xffffffffu, row_sc[r >> 1], 4 * (2 * t + (r & 1))), FLT_MIN);
            m[r] = limit[r] = -INFINITY;
            l[r] = 0.0f;
            neg[r] = kShift4;
        }
        float o[NT][DC / 16][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < DC / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][i][e] = 0.0f;

        bool ok = true;
#pragma unroll 1
        for (; k0 < last; k0 += kStep) {
            const int key0 = k0, ahead = k0 + kAhead4 * kStep, page = pages;
            pages = page_of(ahead + kStep);
            __syncwarp();  // the stage that is filled now has been read
            if (ahead < last)
                fill(ahead, page);
            else
                paged <<= 2 * kGroups;
            close();
            if constexpr (DENSE)
                if (!(ok = wait_warp(bar_at + 8 * to_use, phase, &s_abort))) break;
            asm volatile("cp.async.wait_group %0;" ::"n"(kAhead4) : "memory");
            __syncwarp();
            uint8_t* const unit = my_ring + to_use * S::kBytes;
            if (++to_use == kStages4) {
                to_use = 0;
                phase ^= 1u;
            }
            if constexpr (DENSE) {  // keys that are not there, or lie on a missing page, get scales of zero
                const uint32_t who = paged >> (2 * kGroups * kAhead4) & ((1u << 2 * kGroups) - 1u);
                if (k0 + kUnit > last || who != (0x5555u & ((1u << 2 * kGroups) - 1u))) {
#pragma unroll
                    for (int key = lane; key < kUnit; key += 32)
                        if (k0 + key >= last || !(who >> (2 * (key >> 4)) & 1u)) {
#pragma unroll
                            for (int i = 0; i < S::kScales; i += 4) {
                                *reinterpret_cast<uint32_t*>(unit + S::kKs + key * S::kScales + i) = 0;
                                *reinterpret_cast<uint32_t*>(unit + S::kVs + key * S::kScales + i) = 0;
                            }
                        }
                    fence_async_smem();  // (before the stage's next copies)
                    __syncwarp();
                }
            }
            float s[NT][kGroups][4];
#pragma unroll
            for (int G = 0; G < kGroups; ++G) {
                uint32_t h[2][DC / 8];  // the quarter of keys 16 G + g and 16 G + 8 + g
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int key = 16 * G + 8 * j + g;
                    uint32_t c[DC / 32];
                    if constexpr (DC == 128)
                        *reinterpret_cast<uint4*>(c) = *reinterpret_cast<const uint4*>(unit + key * S::kRow + 16 * t);
                    else
                        *reinterpret_cast<uint2*>(c) = *reinterpret_cast<const uint2*>(unit + key * S::kRow + 8 * t);
                    const uint8_t* sp = unit + S::kKs + key * S::kScales + t * (DC / 64);
                    uint32_t sb = DC == 128 ? *reinterpret_cast<const uint16_t*>(sp) : *sp;
                    if (!DENSE) sb &= k_mask;
                    const uint32_t s2 = q4::scales2(sb);
                    const uint32_t lo = __byte_perm(s2, 0, 0x1010), hi = __byte_perm(s2, 0, 0x3232);
#pragma unroll
                    for (int i = 0; i < DC / 32; ++i) {
                        uint32_t w[4];
                        q4::widen8(c[i], w);
#pragma unroll
                        for (int e = 0; e < 4; ++e) h[j][4 * i + e] = q4::mul_halves(w[e], i < 2 ? lo : hi);
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int i = 0; i < DC / 16; ++i) {
                        const uint32_t A[4] = {h[0][2 * i], h[1][2 * i], h[0][2 * i + 1], h[1][2 * i + 1]};
                        if (i == 0)
                            mma16816_first(s[nt][G], A, qf[nt][0], qf[nt][1]);
                        else
                            mma16816(s[nt][G], A, qf[nt][2 * i], qf[nt][2 * i + 1]);
                    }
                }
            }
            // scores of the lane: keys 16 G + 8 (e >> 1) + g, rows 8 nt + 2t + (e & 1)
            const bool odd_scale = P.s_xor != 0 || P.s_and == 0;
            if (key0 + kUnit > plain || odd_scale) {
#pragma unroll
                for (int r = 0; r < 2 * NT; ++r) {
                    const int row = 8 * (r >> 1) + 2 * t + (r & 1), tok = W.i0 + min(row / P.gs, W.ntok - 1);
                    const uint32_t* mask = a.mask ? a.mask + (int64_t)(W.q.off + tok) * a.mask_words : nullptr;
#pragma unroll
                    for (int h = 0; h < kUnit / 32; ++h) {
                        const uint32_t bits = seen_bits(key0 + 32 * h, mask ? len : prefix + tok + 1, prefix, mask, a.mask_words) >> g;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float& y = s[r >> 1][2 * h + (e >> 1)][2 * (e & 1) + (r & 1)];
                            y = bits >> (8 * e) & 1u ? __uint_as_float((__float_as_uint(y) & P.s_and) ^ P.s_xor) : -INFINITY;
                        }
                    }
                }
            }
            float top[2 * NT];
            bool rises = false;
#pragma unroll
            for (int r = 0; r < 2 * NT; ++r) {
                const float(&y)[kGroups][4] = s[r >> 1];
                top[r] = fmaxf(y[0][r & 1], y[0][2 + (r & 1)]);
#pragma unroll
                for (int G = 1; G < kGroups; ++G) top[r] = max3(top[r], y[G][r & 1], y[G][2 + (r & 1)]);
                rises |= top[r] > limit[r];
            }
            if (__any_sync(0xffffffffu, rises)) {
#pragma unroll
                for (int r = 0; r < 2 * NT; ++r) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], d));
                    const float M = fmaxf(m[r], top[r]), f = m[r] == M ? 1.0f : ex2((m[r] - M) * sc[r]);
                    m[r] = M;
                    l[r] *= f;
                    limit[r] = M == -INFINITY ? M : M + kLazy4 / sc[r];
                    neg[r] = (M == -INFINITY ? 0.0f : -M * sc[r]) + kShift4;
#pragma unroll
                    for (int i = 0; i < DC / 16; ++i) {
                        o[r >> 1][i][r & 1] *= f;
                        o[r >> 1][i][2 + (r & 1)] *= f;
                    }
                }
            }
            uint32_t p[NT][2 * kGroups];  // the operand P^T: rows 8 nt + g, keys 8 e + 2t, + 1
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int e = 0; e < 2 * kGroups; ++e) {
                    const float x0 = ex2(fmaf(s[nt][e >> 1][2 * (e & 1)], sc[2 * nt], neg[2 * nt]));
                    const float x1 = ex2(fmaf(s[nt][e >> 1][2 * (e & 1) + 1], sc[2 * nt + 1], neg[2 * nt + 1]));
                    l[2 * nt] += x0;
                    l[2 * nt + 1] += x1;
                    p[nt][e] = transpose8x8(Half<__half>::pack(x0, x1));
                }
            }
#pragma unroll
            for (int G = 0; G < kGroups; ++G) {
                uint32_t c[2][2][DC / 64], s2[2];  // of keys 16 G + 8 j + 2t, + 1
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uint32_t sb[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int key = 16 * G + 8 * j + 2 * t + i;
                        const uint8_t* src = unit + S::kV + key * S::kRow + g * (DC / 16);
                        if constexpr (DC == 128)
                            *reinterpret_cast<uint2*>(c[j][i]) = *reinterpret_cast<const uint2*>(src);
                        else
                            c[j][i][0] = *reinterpret_cast<const uint32_t*>(src);
                        sb[i] = unit[S::kVs + key * S::kScales + (DC == 128 ? g : g >> 1)];
                        if (!DENSE) sb[i] &= v_mask;
                    }
                    s2[j] = q4::scales2(sb[0] | sb[1] << 8);
                }
#pragma unroll
                for (int w = 0; w < DC / 64; ++w) {
                    uint32_t lo[2][4], hi[2][4];  // the word's even and odd channels of two keys
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t x0 = c[j][0][w], x1 = c[j][1][w];
                        q4::widen8((x0 & 0x0f0f0f0fu) | (x1 << 4 & 0xf0f0f0f0u), lo[j]);
                        q4::widen8((x0 >> 4 & 0x0f0f0f0fu) | (x1 & 0xf0f0f0f0u), hi[j]);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t A[4] = {q4::mul_halves(lo[0][e], s2[0]), q4::mul_halves(hi[0][e], s2[0]),
                                               q4::mul_halves(lo[1][e], s2[1]), q4::mul_halves(hi[1][e], s2[1])};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma16816(o[nt][4 * w + e], A, p[nt][2 * G], p[nt][2 * G + 1]);
                    }
                }
            }
        }

        if (DENSE && !ok) {  // the warp gave up: its copies on their way are waited for (bounded)
            asm volatile("cp.async.wait_all;" ::: "memory");
            for (int i = 0; i <= kAhead4 && k0 + i * kStep < last; ++i) {
                const uint32_t at = to_use + i, bar = bar_at + 8 * (at % kStages4), parity = phase ^ (at / kStages4 & 1u);
                for (uint32_t n = 0; n < kDrainLimit && !mbar_try_wait(bar, parity); ++n) {
                }
            }
        }

        // ---- the segment's result: the warps' parts, joined
#pragma unroll
        for (int r = 0; r < 2 * NT; ++r) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], d);
            m[r] = m[r] == -INFINITY ? -INFINITY : m[r] * sc[r];  // log2 of the largest weight
            if (l[r] != l[r]) m[r] = INFINITY;  // a score that is not a number, or infinite: so is the row, whatever it is joined with
            if (g == 0) s_ml[warp][8 * (r >> 1) + 2 * t + (r & 1)] = make_float2(m[r], l[r]);
        }
        if (__syncthreads_or(!ok)) break;  // (the rings are read; or a warp gave up: nothing of this segment or a later one is written)
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
#pragma unroll
        for (int r = 0; r < 2 * NT; ++r) {
            const int row = 8 * (r >> 1) + 2 * t + (r & 1);
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps4; ++w) M = fmaxf(M, s_ml[w][row].x);
            const float f = m[r] == -INFINITY ? 0.0f : ex2(m[r] - M);
            float* to = s_o + ((size_t)warp * R + row) * RS + 2 * g;
#pragma unroll
            for (int i = 0; i < DC / 16; ++i) {  // channels g DC / 8 + 2i, + 1 (a part without weight may hold anything)
                const float x = o[r >> 1][i][r & 1], y = o[r >> 1][i][2 + (r & 1)];
                *reinterpret_cast<float2*>(to + 16 * i) = f != 0.0f ? make_float2(x * f, y * f) : make_float2(0.0f, 0.0f);
            }
        }
        if (tid < R) {
            float M = -INFINITY, L = 0.0f;
            for (int w = 0; w < kWarps4; ++w) M = fmaxf(M, s_ml[w][tid].x);
            for (int w = 0; w < kWarps4; ++w)
                if (s_ml[w][tid].x != -INFINITY) L = fmaf(s_ml[w][tid].y, ex2(s_ml[w][tid].x - M), L);
            s_tot[tid] = make_float2(M, L);
        }
        __syncthreads();
        for (int i = tid; i < R * (DC / 2); i += kThreads4) {
            const int row = i / (DC / 2), at = i - row * (DC / 2);  // pair `at` of the row: pair at / 8 of the eighth at % 8
            const int tok = row / P.gs, h = row - tok * P.gs, c = (at & 7) * (DC / 8) + 2 * (at >> 3);
            if (tok >= W.ntok || h >= gs || c >= D) continue;
            float2 x = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < kWarps4; ++w) {
                const float2 y = *reinterpret_cast<const float2*>(s_o + ((size_t)w * R + row) * RS + 2 * at);
                x.x += y.x;
                x.y += y.y;
            }
            const float2 ml = s_tot[row];
            const int token = W.q.off + W.i0 + tok, head = head0 + h;
            if (whole) {
                const float inv = (ml.y > 0.0f ? 1.0f / ml.y : ml.y) * vu;  // (the sum: zero, or not a number)
                *reinterpret_cast<uint32_t*>(static_cast<T*>(a.out.p) + (int64_t)token * a.out.tok + head * a.out.head + c) =
                    Half<T>::pack(x.x * inv, x.y * inv);
                if (at == 0 && a.lse)
                    a.lse[(int64_t)token * a.n_heads + head] = ml.y == 0.0f ? -INFINITY : (ml.x + log2f(ml.y) - kShift4) * 0.69314718055994531f;
            } else {
                const int64_t to = (int64_t)slot * P.cap_rows + row;
                *reinterpret_cast<float2*>(P.part_o + to * DC + c) = make_float2(x.x * vu, x.y * vu);
                if (at == 0) P.part_ml[to] = ml;
            }
        }
        fence_async_smem();
        __syncthreads();  // s_ml, s_tot and the rings are free
    }
    if (DENSE && tid == 0 && *static_cast<volatile int*>(&s_abort) && a.status) atomicOr(a.status, PPS_FLAG_TIMEOUT);
}

// Whether a cache lies as kByToken has it; its maps in boxes of 16 rows, [page, head, token, byte].
bool by_token_maps(CUtensorMap (&m)[2], const AttnArgs& a, const Q4View& z, int dc) {
    const CacheView& c = a.c;
    const uintptr_t codes = reinterpret_cast<uintptr_t>(c.k) | reinterpret_cast<uintptr_t>(c.v) | (uintptr_t)c.page | (uintptr_t)c.tok | (uintptr_t)c.head;
    const uintptr_t scales = reinterpret_cast<uintptr_t>(z.ks) | reinterpret_cast<uintptr_t>(z.vs) | (uintptr_t)z.page | (uintptr_t)z.tok | (uintptr_t)z.head;
    if (c.head_dim != dc || c.page_size < 16 || c.n_pages < 1 || codes % 16 != 0 || scales % (dc / 16) != 0) return false;
    EncodeTiledFn f = encode_fn();
    if (f == nullptr) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)dc / 2, (cuuint64_t)c.page_size, (cuuint64_t)c.n_kv_heads, (cuuint64_t)c.n_pages};
    // the stride of a dimension of one is never used, but has to be a multiple of 16 bytes
    const cuuint64_t strides[3] = {(cuuint64_t)c.tok, c.n_kv_heads > 1 ? (cuuint64_t)c.head : 256, c.n_pages > 1 ? (cuuint64_t)c.page : 256};
    const cuuint32_t box[4] = {(cuuint32_t)dc / 2, 16, 1, 1}, es[4] = {1, 1, 1, 1};
    for (int i = 0; i < 2; ++i)
        if (f(&m[i], CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, i ? c.v : c.k, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
              kFetch4, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return false;
    return true;
}
// Whether it lies as kByHead has it, and CopyKeys dense.
bool is_by_head(const AttnArgs& a, const Q4View& z, int dc) {
    const uintptr_t bits = reinterpret_cast<uintptr_t>(a.c.k) | reinterpret_cast<uintptr_t>(a.c.v) | reinterpret_cast<uintptr_t>(z.ks) |
                           reinterpret_cast<uintptr_t>(z.vs) | (uintptr_t)a.c.page | (uintptr_t)a.c.head | (uintptr_t)z.page | (uintptr_t)z.head;
    return a.c.head_dim == dc && a.c.page_size >= 16 && a.c.tok == dc / 2 && z.tok == dc / 16 && bits % 16 == 0;
}

// the rows of a block, the heads taken at a time, the tokens of a block: by the mean number of tokens of a sequence
struct Rows4 {
    int nt, nsub, gs, tt;
    Rows4(int64_t n_tok, int64_t n_seq, int group) {
        const int64_t mean = n_seq > 0 ? (n_tok + n_seq - 1) / n_seq : n_tok;
        nt = mean * group <= 8 ? 1 : 2;
        nsub = (group + 8 * nt - 1) / (8 * nt);
        gs = (group + nsub - 1) / nsub;
        tt = 8 * nt / gs;
    }
};

template <typename T, int DC, int NT>
cudaError_t launch_few(const AttnArgs& a, const Q4View& z, const Rows4& rows, cudaStream_t st) {
    AttnPlan P;
    std::memset(&P, 0, sizeof(P));
    P.group = a.n_heads / a.c.n_kv_heads;
    P.nsub = rows.nsub;
    P.gs = rows.gs;
    P.tt = P.bt = rows.tt;
    P.fix = kFix4;
    P.cap_rows = 8 * NT;
    P.shift = kShift4;
    plan_common(P, a);
    carve(P, a.ws, kMaxCtas4);
    constexpr int kSmem = std::max(kWarps4 * 8 * NT * (DC + 4) * 4, kWarps4 * kStages4 * Stage<DC>::kBytes);
    CUtensorMap maps[2] = {};
    const Lie lie = is_by_head(a, z, DC) ? kByHead : by_token_maps(maps, a, z, DC) ? kByToken : kAnyHow;
    auto kernel = lie == kByHead ? few_rows_kernel<T, DC, NT, kByHead>
                                 : lie == kByToken ? few_rows_kernel<T, DC, NT, kByToken> : few_rows_kernel<T, DC, NT, kAnyHow>;
    static std::atomic<uint64_t> ready[3] = {};
    cudaError_t e = allow_smem(ready[lie], (const void*)kernel, kSmem);
    if (e != cudaSuccess) return e;
    const int ctas = std::min(device_sm_count() * few_ctas(NT), kMaxCtas4);
    e = launch_pdl(kernel, dim3(ctas), dim3(kThreads4), kSmem, st, maps[0], maps[1], a, z, P);
    if (e != cudaSuccess) return e;
    return launch_pdl(join_kernel<T, DC>, dim3(ctas, join_blocks(a, P)), dim3(256), 0, st, a, P);
}

// Queries in bf16 as halves, rows side by side, and the factor that a row's scores get for it.  Half a warp has a row, eight channels
// a lane; four rows of it are on their way.
__global__ void __launch_bounds__(256) halve_kernel(const AttnArgs a, __half* out, float* row_scale) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int kAtOnce = 4;
    const int64_t rows = a.n_tok * a.n_heads, step = (int64_t)gridDim.x * 16;
    const int at = 8 * (threadIdx.x & 15), D = a.c.head_dim;
    for (int64_t i0 = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); i0 < (rows + 1) / 2 * 2; i0 += kAtOnce * step) {  // (both halves of a warp)
        uint4 x[kAtOnce];
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) {
            const int64_t i = i0 + e * step, tok = i / a.n_heads;
            x[e] = make_uint4(0, 0, 0, 0);
            if (i < rows && at < D)
                x[e] = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q.p) + tok * a.q.tok + (i - tok * a.n_heads) * a.q.head + at));
        }
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) {
            const int64_t i = i0 + e * step;
            const uint32_t w[4] = {x[e].x, x[e].y, x[e].z, x[e].w};
            uint32_t top = 0, h[4];  // the largest finite magnitude
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t lo = w[c] & 0x7fffu, hi = w[c] >> 16 & 0x7fffu;
                top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
            }
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
            const int k = halving(top);
            const float f = power_of_two(k);
#pragma unroll
            for (int c = 0; c < 4; ++c) h[c] = Half<__half>::pack(__uint_as_float(w[c] << 16) * f, __uint_as_float(w[c] & 0xffff0000u) * f);
            if (i < rows && at < D) *reinterpret_cast<uint4*>(out + i * D + at) = make_uint4(h[0], h[1], h[2], h[3]);
            if (i < rows && at == 0) row_scale[i] = power_of_two(-k);
        }
    }
}

size_t parts4_bytes(int64_t n_tok, int group, int head_dim) {
    const size_t x = std::max(part_bytes(kMaxCtas4, 16, head_dim), part_bytes(kMaxCtas, Rows(n_tok, group).cap, head_dim));
    return (x + 255) / 256 * 256;
}
size_t halves_bytes(int64_t n_tok, int n_heads, int head_dim) { return ((size_t)n_tok * n_heads * head_dim * 2 + 255) / 256 * 256; }

template <typename T, int DC>
cudaError_t launch_tiles(const AttnArgs& given, const Q4View& z, cudaStream_t st) {
    AttnArgs a = given;
    AttnPlan P;
    std::memset(&P, 0, sizeof(P));
    P.group = a.n_heads / a.c.n_kv_heads;
    const Rows rows(a.n_tok, P.group);
    P.nsub = rows.nsub;
    P.gs = rows.gs;
    P.tt = rows.tt;
    P.bt = 2 * rows.tt;
    P.fix = kFixTiles4;
    P.cap_rows = rows.cap;
    P.shift = Half<__half>::kShift;
    plan_common(P, a);
    carve(P, a.ws, kMaxCtas);
    const int ctas = std::min(device_sm_count(), kMaxCtas);
    Q4Rows r4 = {z, nullptr, is_by_head(a, z, DC)};
    if constexpr (std::is_same_v<T, __nv_bfloat16>) {
        char* w = static_cast<char*>(a.ws) + parts4_bytes(a.n_tok, P.group, a.c.head_dim);
        __half* halves = reinterpret_cast<__half*>(w);
        float* factors = reinterpret_cast<float*>(w + halves_bytes(a.n_tok, a.n_heads, a.c.head_dim));
        const int64_t blocks = std::min<int64_t>((a.n_tok * a.n_heads + 15) / 16, (int64_t)ctas * 8);
        const cudaError_t e = launch_pdl(halve_kernel, dim3((unsigned)blocks), dim3(256), 0, st, a, halves, factors);
        if (e != cudaSuccess) return e;
        a.q = {halves, (int64_t)a.n_heads * a.c.head_dim, a.c.head_dim};
        r4.row_scale = factors;
    }
    CUtensorMap tmQ;
    if (!query_map(&tmQ, a, P, PPS_F16)) return cudaErrorInvalidValue;
    constexpr int kSmem = Cfg<DC, true>::kSmem;
    static std::atomic<uint64_t> ready{0};
    cudaError_t e = allow_smem(ready, (const void*)attention_kernel<T, DC, true>, kSmem);
    if (e != cudaSuccess) return e;
    e = launch_pdl(attention_kernel<T, DC, true>, dim3(ctas), dim3(Cfg<DC, true>::kThreads), kSmem, st, tmQ, tmQ, tmQ, a, P, r4);
    if (e != cudaSuccess) return e;
    return launch_pdl(join_kernel<T, DC>, dim3(ctas, join_blocks(a, P)), dim3(256), 0, st, a, P);
}

template <typename T, int DC>
cudaError_t by_rows(const AttnArgs& a, const Q4View& z, cudaStream_t st) {
    const int group = a.n_heads / a.c.n_kv_heads;
    if ((a.n_tok + a.n_seq - 1) / a.n_seq * group > kFewRows) return launch_tiles<T, DC>(a, z, st);
    const Rows4 rows(a.n_tok, a.n_seq, group);
    return rows.nt == 1 ? launch_few<T, DC, 1>(a, z, rows, st) : launch_few<T, DC, 2>(a, z, rows, st);
}

template <typename T>
cudaError_t by_channels4(const AttnArgs& a, const Q4View& z, cudaStream_t st) {
    return channel_class(a.c.head_dim) == 64 ? by_rows<T, 64>(a, z, st) : by_rows<T, 128>(a, z, st);
}

}  // namespace

size_t attention_q4_workspace_bytes(int64_t n_tok, int n_heads, int n_kv_heads, int head_dim) {
    return parts4_bytes(n_tok, (n_heads + n_kv_heads - 1) / n_kv_heads, head_dim) + halves_bytes(n_tok, n_heads, head_dim) +
           sizeof(float) * (size_t)n_tok * n_heads;
}

cudaError_t launch_attention_q4(const AttnArgs& a, const Q4View& z, int dtype, cudaStream_t stream) {
    return dtype == PPS_BF16 ? by_channels4<__nv_bfloat16>(a, z, stream) : by_channels4<__half>(a, z, stream);
}

}  // namespace pps
