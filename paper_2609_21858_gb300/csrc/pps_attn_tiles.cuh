// pps_attn_tiles.cuh -- the attention kernel of 128-row tiles on the tensor cores (tcgen05), over a cache of 16 bits
// (pps_attention.cu, where its plan is explained) or of 4 (pps_attention_q4.cu).
#pragma once
#include <atomic>
#include <cstring>
#include <type_traits>

#include "pps_attn.cuh"
#include "pps_q4.cuh"

namespace pps {
namespace {

using namespace tc;

constexpr int kLoadWarp = 8;       // the first after two softmax warpgroups
constexpr int kMaxCtas = 160;      // shares of the work (one per SM)
// Key tiles that an item's start and end cost.  (2, 3, 4: decoding batches and ragged chunks 1 to 3 percent faster, trees 3 to 11
// and one long sequence 4 to 6 percent slower.)
constexpr int kFix = 6;
constexpr int kLeast = 3;          // of a cut item's key tiles, at most, for a cut to move to the item's end
constexpr float kLazy = 8.0f;      // log2 of the rise of a maximum that O is not rescaled for
constexpr uint32_t kColO = 256;    // tensor memory columns: S/P of streams 0, 1; O of streams 0, 1

// what depends on the channels' class DC: 64 (head_dim <= 64) or 128
template <int DC, bool Q4>
struct Cfg {
    static constexpr int kBlock = 128 * 128;                 // 128 rows of 64 channels, 128-byte swizzle
    static constexpr int kTile = kBlock * (DC / 64);         // 16 or 32 KB: a tile of Q, K or V
    // Warps that load, one that issues products, one that loads queries: the same number of warps on each quarter of the SM.  Of 16
    // bits one loads keys, one values; of 4 bits six take the halves of the tiles of keys and of values in turn.
    static constexpr int kLoaders = Q4 ? 6 : 2;
    static constexpr int kMmaWarp = kLoadWarp + kLoaders, kQueryWarp = kMmaWarp + 1, kThreads = 32 * (kQueryWarp + 1);
    static constexpr int kHalves = Q4 ? 2 : 1;               // loads that fill a tile
    // of 4 bits: codes, then scales of half a tile, as they come; how many such a warp has, on their way or in use
    static constexpr int kHalf = 64, kRow = DC / 2, kScales = DC / 16, kPack = kHalf * (kRow + kScales), kPacks = 2;
    // tiles of K and V in flight: 5 (or 12); of 4 bits 3 (or 6)
    static constexpr int kStages = Q4 ? 3 * 128 / DC : (224 * 1024 - 2 * kTile) / kTile;
    static constexpr int kBars = (2 + kStages) * kTile + (Q4 ? kLoaders * kPacks * kPack : 0);
    static constexpr int kSmem = kBars + 320 /* barriers */ + 224 /* plan */ + 2048 /* maxima and sums */;
    static_assert(8 * (2 * kStages + 13) <= 320 && kThreads % 128 == 0 && kSmem <= 227 * 1024, "barriers and shared memory fit");
};

// beside the cache, for 4 bits: scales and units; a factor per row (token, head) on its scores, null: ones
struct Q4Rows {
    Q4View z;
    const float* row_scale;
    bool dense;  // as CopyKeys has it
};

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}

// A warp copies 32 or 64 keys, codes and scales of one half of the cache, from a head's rows (`codes`, `scales`: of page 0) into shared
// memory, row after row.  Keys of a missing page, and those from `last` on in blocks without any key, get scales of zero, whatever
// their codes.  Sixteen bytes a lane and instruction throughout: bulk copies of a page's rows take a warp longer, as each of its
// lanes' is issued by itself (16 rows at a time: 64 keys of one half 1500 clocks, 64 trees of 41 nodes 246 us where copies of 16 bytes a lane took 239).
// DENSE: all DC channels are there, 16 keys in a row share their page, and a page's rows of a head follow one another, from
// 16-byte boundaries on (a page laid out head by head).
template <int DC, bool DENSE, int KEYS>
struct CopyKeys {
    static constexpr int kRow = DC / 2, kScales = DC / 16, kBytes = KEYS * (kRow + kScales);
    static constexpr int kKeys = DENSE ? 16 : 8;  // with a page to themselves
    int page, k0;                                 // of keys k0 + kKeys (lane modulo KEYS / kKeys) on
    // of the keys from key k0_ on
    __device__ __forceinline__ void find(const int32_t* table, int page_log2, int k0_, int last) {
        const int k = k0_ + kKeys * (threadIdx.x & (KEYS / kKeys - 1));
        k0 = k0_;
        page = k < last ? __ldg(table + (k >> page_log2)) : 0;
    }
    __device__ __forceinline__ void go(uint8_t* to, const uint8_t* codes, const uint8_t* scales, const CacheView& c, const Q4View& z, int last, int D,
                                       bool wide, uint32_t* status) const {
        const int lane = threadIdx.x & 31;
        const bool key = k0 + kKeys * (lane & (KEYS / kKeys - 1)) < last, good = key && (uint32_t)page < (uint32_t)c.n_pages;
        if (key && !good && status) atomicOr(status, PPS_FLAG_INDEX);
        const uint32_t who = __ballot_sync(0xffffffffu, good), dst = tc::smem_u32(to);
        if constexpr (DENSE) {
            constexpr int kTurns = 16 * kRow / 512;  // of 16 keys' codes
#pragma unroll
            for (int G = 0; G < KEYS / 16; ++G) {
                const int p = __shfl_sync(0xffffffffu, page, G);
                if (!(who >> G & 1u)) continue;  // (warp-uniform)
                const uint8_t* src = codes + p * c.page + ((k0 + 16 * G) & (c.page_size - 1)) * kRow + 16 * lane;
#pragma unroll
                for (int i = 0; i < kTurns; ++i) copy_async<16>(dst + 16 * G * kRow + 512 * i + 16 * lane, src + 512 * i);
            }
            constexpr int kLanes = 16 * kScales / 16;  // of 16 keys' scales
            const int G = lane / kLanes & (KEYS / 16 - 1), p = __shfl_sync(0xffffffffu, page, G);
            if (lane < KEYS / 16 * kLanes) {
                const uint32_t at = dst + KEYS * kRow + 16 * lane;
                if (who >> G & 1u)
                    copy_async<16>(at, scales + p * z.page + ((k0 + 16 * G) & (c.page_size - 1)) * kScales + 16 * (lane % kLanes));
                else
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0) : "memory");
            }
        } else {
            const int part = lane & 3;  // four lanes copy a row of codes
            const int64_t mine = (lane >> 2) * c.tok + part * (DC / 8);
#pragma unroll
            for (int i = 0; i < KEYS / 8; ++i) {
                const int p = __shfl_sync(0xffffffffu, page, i), k = k0 + 8 * i;
                if (!(who >> i & 1u) || k + (lane >> 2) >= last || part * (DC / 4) >= D) continue;
                const uint8_t* src = codes + p * c.page + (k & (c.page_size - 1)) * c.tok + mine;
                const uint32_t at = dst + (8 * i + (lane >> 2)) * kRow + part * (DC / 8);
                if (DC == 128 && wide)
                    copy_async<16>(at, src);
                else {
                    copy_async<8>(at, src);
                    if (DC == 128 && part * (DC / 4) + 16 < D) copy_async<8>(at + 8, src + 8);
                }
            }
#pragma unroll
            for (int i = 0; i < KEYS / 32; ++i) {
                const int r = lane + 32 * i, p = __shfl_sync(0xffffffffu, page, r >> 3);
                const uint32_t at = dst + KEYS * kRow + r * kScales;
                const bool there = (who >> (r >> 3) & 1u) && k0 + r < last;
                const uint8_t* src = scales + p * z.page + ((k0 + r) & (c.page_size - 1)) * z.tok;
#pragma unroll
                for (int w = 0; w < DC / 64; ++w) {
                    if (there && 64 * w < D)
                        copy_async<4>(at + 4 * w, src + 4 * w);
                    else
                        asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + 4 * w), "r"(0) : "memory");
                }
            }
        }
    }
};

__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int* abort) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort));
}

// T: of the result, and but for Q4 of all operands.  Q4: queries are halves (with a factor per row), the cache has 4 bits: the loading
// warps copy a tile's codes ahead, widen them and write the tile as TMA would have.
template <typename T, int DC, bool Q4>
__global__ void __launch_bounds__(Cfg<DC, Q4>::kThreads, 1)
    attention_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                     const __grid_constant__ CUtensorMap tmV, const AttnArgs a, const AttnPlan P, const Q4Rows R4) {
    using C = Cfg<DC, Q4>;
    using H = Half<std::conditional_t<Q4, __half, T>>;
    constexpr int kMmaWarp = C::kMmaWarp;
    extern __shared__ __align__(1024) uint8_t attn_smem[];
    const uint32_t base = smem_u32(attn_smem);
    const uint32_t ring = base + 2 * C::kTile;
    const uint32_t bars = base + C::kBars;
    auto bar = [&](uint32_t i) { return bars + 8u * i; };
    auto full = [&](uint32_t s) { return bar(s); };
    auto empty = [&](uint32_t s) { return bar(C::kStages + s); };
    auto sfull = [&](uint32_t w) { return bar(2 * C::kStages + w); };
    auto pready = [&](uint32_t w, uint32_t half) { return bar(2 * C::kStages + (half ? 11 : 2) + w); };  // a barrier per half: no warp may count twice
    auto odone = [&](uint32_t w) { return bar(2 * C::kStages + 4 + w); };
    auto qfull = [&](uint32_t t) { return bar(2 * C::kStages + 6 + t); };
    auto qfree = [&](uint32_t t) { return bar(2 * C::kStages + 8 + t); };
    const uint32_t segbar = bar(2 * C::kStages + 10);
    uint8_t* tail = attn_smem + C::kBars + 320;
    volatile int* abort = reinterpret_cast<volatile int*>(tail);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tail + 4);
    int64_t* s_sum = reinterpret_cast<int64_t*>(tail + 16);          // a sum per warp
    Start* s_start = reinterpret_cast<Start*>(tail + 16 + 16 * 8);
    float2* s_ml = reinterpret_cast<float2*>(tail + 224);            // [2][128]
    static_assert(C::kThreads <= 16 * 32 && 16 + 16 * 8 + sizeof(Start) <= 224, "plan fits");

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    if (tid == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(full(s), C::kHalves);
            mbar_init(empty(s), 1);
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(sfull(w), 1);
            mbar_init(pready(w, 0), 4);  // the weights of a tile's first 64 keys
            mbar_init(pready(w, 1), 4);  // of the others
            mbar_init(odone(w), 1);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(qfull(t), 1);
            mbar_init(qfree(t), 1);
        }
        mbar_init(segbar, 8);
        *abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kLoadWarp && lane == 0) {
        tma_prefetch_map(&tmQ);
        if constexpr (!Q4) {
            tma_prefetch_map(&tmK);
            tma_prefetch_map(&tmV);
        }
    }
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    pdl_wait();  // what comes before this runs while the stream's last kernel ends
    pdl_launch_dependents();
    // the share of the line of costs, and where on it the share starts
    int64_t c0, c1;
    const int64_t share = find_share<C::kThreads>(a, P, s_sum, s_start, c0, c1);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    if (c0 >= c1 || (base & 1023u) != 0) {  // no work (or a base that the swizzled tiles cannot have)
        if (c0 < c1 && tid == 0 && a.status) atomicOr(a.status, PPS_FLAG_TIMEOUT);
        if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
        return;
    }
    const int least = (int)min(max(share / 8, (int64_t)1), (int64_t)kLeast);
    Walk W(P, *s_start, c0, c1, least);
    const int D = a.c.head_dim;

    // registers: 384 x 168 at launch = 256 x 216 + 128 x 72; of 4 bits 512 x 128 = 256 x 192 + 256 x 64
    if (warp >= kLoadWarp) {
        if constexpr (Q4)
            asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        else
            asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (Q4 && warp < kMmaWarp) {
            // ---- as below, of 4 bits: half a tile of keys or of values at a time
            auto load = [&](auto is_dense) {
                using Copy = CopyKeys<DC, decltype(is_dense)::value, C::kHalf>;
                const int me = warp - kLoadWarp;
                uint8_t* const packs = attn_smem + (2 + C::kStages) * C::kTile + me * C::kPacks * C::kPack;
                const bool wide = ((reinterpret_cast<uintptr_t>(a.c.k) | reinterpret_cast<uintptr_t>(a.c.v) | (uintptr_t)a.c.page | (uintptr_t)a.c.tok |
                                    (uintptr_t)a.c.head | (uintptr_t)(D / 2)) & 15) == 0;
                uint32_t ring0 = 0;
                bool ok = true;
                while (ok && W.next(a, P)) {
                    const int n = W.t1 - W.t0, ahead = min(W.ntok <= P.tt ? 2 : 1, n), len = W.q.len, kvh = W.heads / P.nsub;
                    const int32_t* table = a.pages + (int64_t)W.s * a.pages_stride;
                    const int last = min(len, W.t1 * kTileKeys);
                    Copy copy;
                    uint32_t to_fill = 0, to_use = 0;
                    // load u: the half u % 2 of the tile at place u / 2 of the segment's in the ring (below); twice the tile's number, + 1: values.
                    // A warp takes every sixth load of all segments, so that its places in the ring are 3 apart: a wait for a
                    // place's last use, told by its parity, would not tell it from the use before that if they were over kStages apart.
                    auto tile_of = [&](int u) {
                        const int x = u / 2, y = x - ahead;
                        return x < ahead ? 2 * x : y < 2 * (n - ahead) ? (y & 1 ? 2 * (ahead + y / 2) : 2 * (y / 2) + 1) : 2 * (y - (n - ahead)) + 1;
                    };
                    auto key_of = [&](int u) { return (W.t0 + tile_of(u) / 2) * kTileKeys + C::kHalf * (u & 1); };
                    const int first = (int)((me + 2 * C::kLoaders - 2 * ring0 % C::kLoaders) % C::kLoaders);
                    auto issue = [&](int u) {
                        if (u < 4 * n) {
                            const bool is_v = tile_of(u) & 1;
                            copy.go(packs + to_fill * C::kPack, static_cast<const uint8_t*>(is_v ? a.c.v : a.c.k) + kvh * a.c.head,
                                    (is_v ? R4.z.vs : R4.z.ks) + kvh * R4.z.head, a.c, R4.z, last, D, wide, a.status);
                        }
                        to_fill ^= 1u;
                        asm volatile("cp.async.commit_group;" ::: "memory");
                        copy.find(table, P.page_log2, key_of(u + C::kLoaders), last);
                    };
                    static_assert(C::kPacks == 2, "one on its way, one in use");
                    copy.find(table, P.page_log2, key_of(first), last);
                    issue(first);
#pragma unroll 1
                    for (int u = first; u < 4 * n; u += C::kLoaders) {
                        __syncwarp();  // what is filled now has been read
                        issue(u + C::kLoaders);
                        asm volatile("cp.async.wait_group 1;" ::: "memory");
                        __syncwarp();
                        const uint8_t* const src = packs + to_use * C::kPack;
                        to_use ^= 1u;
                        const int half0 = C::kHalf * (u & 1);
                        const uint32_t it = ring0 + u / 2;
                        const uint32_t s = it % C::kStages;
                        if (!(ok = wait_warp(empty(s), ((it / C::kStages) & 1u) ^ 1u, abort))) break;
                        // a lane widens 16 bytes of codes, 32 channels, of a key at a time; lanes of a key are neighbours
                        constexpr int kU = DC / 32, kAt = 32 / kU;  // lanes of a key, keys of a turn
                        const int c = lane % kU, r0 = lane / kU, there = len - key_of(u);
                        uint8_t* dst = attn_smem + (2 + s) * C::kTile + (c >> 1) * C::kBlock + (half0 + r0) * 128;
                        const bool lo_there = 32 * c < D, hi_there = 32 * c + 16 < D;  // (the bytes behind the last block's may be anything)
#pragma unroll 2
                        for (int i = 0; i < C::kHalf / kAt; ++i) {
                            const int r = i * kAt + r0;
                            const uint4 w = *reinterpret_cast<const uint4*>(src + r * C::kRow + 16 * c);
                            const uint32_t s2 = q4::scales2(*reinterpret_cast<const uint16_t*>(src + C::kHalf * C::kRow + r * C::kScales + 2 * c));
                            const bool key = r < there;
                            const uint32_t lo = key && lo_there ? __byte_perm(s2, 0, 0x1010) : 0u, hi = key && hi_there ? __byte_perm(s2, 0, 0x3232) : 0u;
                            // lanes of the second 64 channels begin with the other block of 16, so that eight lanes' stores touch all banks
                            const bool swap = (c & 2) != 0;
                            const uint32_t x[4] = {swap ? w.z : w.x, swap ? w.w : w.y, swap ? w.x : w.z, swap ? w.y : w.w};
                            const uint32_t y[2] = {swap ? hi : lo, swap ? lo : hi};
                            const uint32_t turn = (uint32_t)((c & 1) * 4 + (swap ? 2 : 0)) ^ (uint32_t)(r & 7);
                            uint8_t* to = dst + i * kAt * 128;
#pragma unroll
                            for (int b = 0; b < 4; ++b) {
                                uint32_t h[4];
                                q4::widen8(x[b], h);
#pragma unroll
                                for (int e = 0; e < 4; ++e) h[e] = q4::mul_halves(h[e], y[b >> 1]);
                                *reinterpret_cast<uint4*>(to + ((turn ^ b) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
                            }
                        }
                        fence_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(full(s));
                    }
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    __syncwarp();
                    ring0 += 2 * n;
                }
            };
            if (R4.dense)
                load(std::true_type());
            else
                load(std::false_type());
        } else if (warp < kMmaWarp) {
            // ---- one warp loads the keys' tiles, one the values'.  The ring holds them in the order of their use: K of
            // the first tile (or two, one per stream), then V_j and the next K in turn.
            const bool is_v = warp != kLoadWarp;
            const int box = min(kTileKeys, a.c.page_size), boxes = kTileKeys / box, box_log2 = 31 - __clz(boxes);
            // the segment's first place in the ring; one past the last place this warp filled, and which it filled before it
            uint32_t ring0 = 0, last = 0, filled = 0;
            bool ok = true;
            while (ok && W.next(a, P)) {
                const int n = W.t1 - W.t0, ahead = W.ntok <= P.tt ? 2 : 1, len = W.q.len, kvh = W.heads / P.nsub;
                const int32_t* table = a.pages + (int64_t)W.s * a.pages_stride;
                // pages of 32 boxes at a time, one per lane; the next 32 are on their way
                const int per = 32 >> box_log2;  // tiles of 32 boxes
                auto pages_from = [&](int j) {
                    const int64_t k = (int64_t)(W.t0 + j) * kTileKeys + lane * box;
                    return k < len && j < n ? __ldg(table + (k >> P.page_log2)) : 0;
                };
                int cur = pages_from(0), nxt = pages_from(per);
                for (int j = 0; j < n; ++j) {
                    if (j > 0 && (j & (per - 1)) == 0) {
                        cur = nxt;
                        nxt = pages_from(j + per);
                    }
                    const uint32_t it = ring0 + (is_v ? (j + ahead < n ? ahead + 2 * j : n + j) : j < ahead ? j : 2 * j - ahead + 1);
                    const uint32_t s = it % C::kStages;
                    if (!(ok = wait_warp(empty(s), ((it / C::kStages) & 1u) ^ 1u, abort))) break;
                    filled = (filled << (it + 1 - last)) | 1u;
                    last = it + 1;
                    const int k0 = (W.t0 + j) * kTileKeys, need = (min(kTileKeys, len - k0) + box - 1) / box;
                    const uint32_t dst = ring + s * C::kTile;
                    int page = __shfl_sync(0xffffffffu, cur, ((j & (per - 1)) << box_log2) + (lane & (boxes - 1)));
                    if (lane == 0) mbar_expect_tx(full(s), (uint32_t)(need * box * 128 * (DC / 64)));
                    __syncwarp();
                    if (lane < need) {
                        if (page < 0 || page >= a.c.n_pages) {  // reads as zeros past the last page
                            if (a.status) atomicOr(a.status, PPS_FLAG_INDEX);
                            page = (int)a.c.n_pages;
                        }
                        const int in_page = (k0 + lane * box) & (a.c.page_size - 1);
#pragma unroll
                        for (int b = 0; b < DC / 64; ++b)
                            if (is_v)
                                tma_load_4d(dst + b * C::kBlock + lane * box * 128, &tmV, full(s), b * 64, in_page, kvh, page);
                            else
                                tma_load_4d(dst + b * C::kBlock + lane * box * 128, &tmK, full(s), b * 64, in_page, kvh, page);
                    }
                }
                ring0 += 2 * n;
            }
            // copies in flight when the CTA gives up: wait (bounded) for each
            for (uint32_t j = 0; j < (uint32_t)C::kStages && *abort; ++j)
                if (filled >> j & 1u)
                    for (uint32_t n = 0, i = last - 1 - j; n < kDrainLimit && !mbar_try_wait(full(i % C::kStages), (i / C::kStages) & 1u); ++n) {
                    }
        } else if (warp == kMmaWarp) {
            // ---- products (one thread): per stream S = Q K^T, then O += P V as its weights arrive
            // Straight-line products of the class's full width (channels past head_dim are zeros): in a loop they issue at
            // 100 cycles each, so at the tensor core's 64.  No product stands under a condition of its own.
            if (elect_one()) {
                constexpr uint32_t id_qk = (1u << 4) | (H::kType << 7) | (H::kType << 10) | ((kTileKeys / 8u) << 17) | ((kTileRows / 16u) << 24);
                constexpr uint32_t id_pv = (1u << 4) | (H::kType << 7) | (H::kType << 10) | (1u << 16) | ((DC / 8u) << 17) | ((kTileRows / 16u) << 24);
                uint32_t it = 0, np0 = 0, np1 = 0, nq0 = 0, nq1 = 0, turn = 0;
                auto stage = [&](uint32_t i) { return ring + (i % C::kStages) * C::kTile; };
                auto landed = [&](uint32_t i) {
                    const bool ok = mbar_wait(full(i % C::kStages), (i / C::kStages) & 1u, abort);
                    tc_fence_after();
                    return ok;
                };
                auto scores = [&](uint32_t w, uint32_t tile, uint32_t k, bool last) {  // last: the segment needs the queries no more
                    const uint64_t qd = sw128_desc(base + tile * C::kTile), kd = sw128_desc(stage(k));
#pragma unroll
                    for (uint32_t c = 0; c < DC / 16; ++c) {
                        const uint64_t o = ((c >> 2) * C::kBlock + (c & 3u) * 32u) >> 4;
                        tc_mma(tmem + w * 128u, qd + o, kd + o, id_qk, c != 0);
                    }
                    tc_commit(sfull(w));
                    if (last) tc_commit(qfree(tile));
                };
                // O += P V in two halves, each as soon as its weights are there
                auto values = [&](uint32_t w, uint32_t v, bool first) {
                    const uint64_t vd = sw128_desc_mn(stage(v), C::kBlock);
                    const uint32_t o = tmem + kColO + w * 128u, p = tmem + w * 128u, at = w ? np1 : np0;
                    ++(w ? np1 : np0);
                    if (!mbar_wait(pready(w, 0), at & 1u, abort)) return false;
                    tc_fence_after();
#pragma unroll
                    for (uint32_t c = 0; c < kTileKeys / 32; ++c) tc_mma_ts(o, p + c * 8u, vd + c * (2048u >> 4), id_pv, !first || c != 0);
                    if (!mbar_wait(pready(w, 1), at & 1u, abort)) return false;
                    tc_fence_after();
#pragma unroll
                    for (uint32_t c = kTileKeys / 32; c < kTileKeys / 16; ++c) tc_mma_ts(o, p + c * 8u, vd + c * (2048u >> 4), id_pv, 1u);
                    tc_commit(odone(w));
                    return true;
                };
                bool ok = true;
                while (ok && W.next(a, P)) {
                    const int n = W.t1 - W.t0;
                    if (n == 0) continue;
                    if (W.ntok > P.tt) {  // a tile per stream, the same keys
                        ok = mbar_wait(qfull(0), nq0++ & 1u, abort) && mbar_wait(qfull(1), nq1++ & 1u, abort) && landed(it);
                        if (!ok) break;
                        scores(0, 0, it, n == 1);
                        scores(1, 1, it, n == 1);
                        tc_commit(empty(it % C::kStages));
                        ++it;
                        for (int j = 0; j < n && ok; ++j) {
                            const uint32_t v = it, k = it + 1;
                            const bool more_keys = j + 1 < n;
                            ok = landed(v);
                            for (uint32_t w = 0; w < 2 && ok; ++w) {
                                ok = values(w, v, j == 0);
                                if (!ok) break;
                                if (w == 1) tc_commit(empty(v % C::kStages));
                                if (more_keys) {
                                    if (w == 0) ok = landed(k);
                                    if (!ok) break;
                                    scores(w, w, k, j + 2 == n);
                                    if (w == 1) tc_commit(empty(k % C::kStages));
                                }
                            }
                            it += more_keys ? 2 : 1;
                        }
                    } else {  // one tile, every other key tile per stream: S of tile j + 2 follows O += P V of tile j
                        const uint32_t tile = turn;
                        turn ^= 1u;
                        ok = mbar_wait(qfull(tile), (tile ? nq1++ : nq0++) & 1u, abort);
#pragma unroll 1
                        for (int j = -2; j < n && ok; ++j) {
                            const uint32_t w = (uint32_t)j & 1u;
                            if (j >= 0) {
                                if (!(ok = landed(it) && values(w, it, j < 2))) break;
                                tc_commit(empty(it % C::kStages));
                                ++it;
                            }
                            if (j + 2 < n) {
                                if (!(ok = landed(it))) break;
                                scores(w, tile, it, j + 3 == n);
                                tc_commit(empty(it % C::kStages));
                                ++it;
                            }
                        }
                    }
                }
            }
            __syncwarp();
        } else if (warp == C::kQueryWarp) {
            // ---- queries: both tiles of a block of two, or the tile that the last block of one did not use
            uint32_t n0 = 0, n1 = 0, turn = 0;
            bool ok = true;
            while (ok && W.next(a, P)) {
                if (W.t0 == W.t1) continue;
                const bool two = W.ntok > P.tt;
                const int kvh = W.heads / P.nsub, sub = W.heads - kvh * P.nsub;
                for (uint32_t i = 0; i < (two ? 2u : 1u) && ok; ++i) {
                    const uint32_t tile = two ? i : turn;
                    ok = wait_warp(qfree(tile), ((tile ? n1 : n0) & 1u) ^ 1u, abort);
                    if (!ok) break;
                    if (tile) ++n1; else ++n0;
                    if (lane == 0) {
                        mbar_expect_tx(qfull(tile), (uint32_t)(P.gs * P.tt * 128 * (DC / 64)));
#pragma unroll
                        for (int b = 0; b < DC / 64; ++b)
                            tma_load_4d(base + tile * C::kTile + b * C::kBlock, &tmQ, qfull(tile), b * 64, sub * P.gs,
                                        W.q.off + W.i0 + (int)i * P.tt, kvh);
                    }
                    __syncwarp();
                }
                if (!two) turn ^= 1u;
            }
            // copies in flight when the CTA gives up: wait (bounded) for each
            for (uint32_t tile = 0; tile < 2 && *abort; ++tile) {
                const uint32_t u = tile ? n1 : n0;
                for (uint32_t n = 0; u > 0 && n < kDrainLimit && !mbar_try_wait(qfull(tile), (u - 1) & 1u); ++n) {
                }
            }
        }
    } else {
        if constexpr (Q4)
            asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        else
            asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // ---- softmax: warpgroup w drives stream w, thread = row r of its tile
        const uint32_t w = warp >> 2, q4 = warp & 3;
        const int r = (int)(q4 * 32) + lane;
        const int row_tok = r / P.gs, row_head = r - row_tok * P.gs;  // the row's token in its tile, its head of the turn
        const uint32_t lanes = (q4 * 32u) << 16;
        const uint32_t tS = tmem + lanes + w * 128u, tO = tmem + lanes + kColO;
        uint32_t done = 0, done_other = 0;  // tiles of this stream and of the other one so far
        uint32_t it = 0, syncs = 0;
        auto seg_sync = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(segbar);
            return wait_warp(segbar, syncs++ & 1u, abort);
        };
        bool ok = true;
        const bool odd_scale = P.s_xor != 0 || P.s_and == 0;
        while (ok && W.next(a, P)) {
            const bool two = W.ntok > P.tt;  // a tile per stream
            const int n = W.t1 - W.t0;
            const int kvh = W.heads / P.nsub, in_group = (W.heads - kvh * P.nsub) * P.gs + row_head;
            const int in_tok = (two ? (int)w * P.tt : 0) + row_tok;  // in the block
            const bool valid = row_tok < P.tt && in_tok < W.ntok && in_group < P.group;
            const bool busy = __any_sync(0xffffffffu, valid);
            const int tok = W.i0 + min(in_tok, W.ntok - 1), head = kvh * P.group + in_group;
            const int in_block = (two ? (int)w * kTileRows : 0) + r;
            const int prefix = W.q.len - W.q.n;
            const uint32_t* mask = a.mask ? a.mask + (int64_t)(W.q.off + tok) * a.mask_words : nullptr;
            const int vis = mask ? W.q.len : prefix + tok + 1;
            const int plain = mask ? prefix : vis;  // keys below it are seen by the row
            float sc = P.sc, vu = 1.0f;
            if constexpr (Q4) {
                if (R4.z.k_unit) sc *= __ldg(R4.z.k_unit + kvh);
                if (R4.z.v_unit) vu = __ldg(R4.z.v_unit + kvh);
                if (R4.row_scale && valid) sc = fminf(sc * __ldg(R4.row_scale + (int64_t)(W.q.off + tok) * a.n_heads + head), FLT_MAX);
                sc = fmaxf(sc, FLT_MIN);  // (a factor of zero would make scores that are not seen NaN)
            }
            float m = -INFINITY, l = 0.0f;
            int i = 0;  // tiles of the stream in this segment
            for (int j = two ? 0 : (int)w; j < n; j += two ? 1 : 2, ++i) {
                const int k0 = (W.t0 + j) * kTileKeys;
                const bool partly = __any_sync(0xffffffffu, k0 + kTileKeys > plain) || odd_scale;  // not all as it stands
                if (!(ok = wait_warp(sfull(w), (done + i) & 1u, abort))) break;
                // values past the sequence's end (in its last tile): whatever the pages hold there becomes zero before any
                // weight is handed over
                if (!Q4 && k0 + kTileKeys > W.q.len && (w == 0 || !two)) {
                    const uint32_t v = it + 2 * n - 1;  // the segment's last value tile
                    if (!(ok = wait_warp(full(v % C::kStages), (v / C::kStages) & 1u, abort))) break;
                    const uint32_t from = ring + (v % C::kStages) * C::kTile + (W.q.len - k0) * 128;
                    const uint32_t bytes = (k0 + kTileKeys - W.q.len) * 128;
#pragma unroll
                    for (int b = 0; b < DC / 64; ++b)
                        for (uint32_t o = r * 16; o < bytes; o += 128 * 16)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(from + b * C::kBlock + o), "r"(0) : "memory");
                    fence_async_smem();
                }
                tc_fence_after();
                if (busy) {
                    uint32_t v[4][32];
                    tmem_ld32(tS, v[0]);
                    tmem_ld32(tS + 32, v[1]);
                    tmem_wait_ld();
                    tmem_landed(v[0]);
                    tmem_landed(v[1]);
                    tmem_ld32(tS + 64, v[2]);
                    tmem_ld32(tS + 96, v[3]);
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    auto highest = [&](int c) {  // of 32 scores, in four chains
#pragma unroll
                        for (int e = 0; e < 32; e += 2)
                            mx[(e >> 1) & 3] = max3(mx[(e >> 1) & 3], __uint_as_float(v[c][e]), __uint_as_float(v[c][e + 1]));
                    };
                    highest(0);
                    highest(1);
                    tmem_wait_ld();
                    tmem_landed(v[2]);
                    tmem_landed(v[3]);
                    highest(2);
                    highest(3);
                    if (partly) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) mx[c] = -INFINITY;
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t bits = seen_bits(k0 + 32 * c, vis, prefix, mask, a.mask_words);
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                v[c][e] = (v[c][e] & P.s_and) ^ P.s_xor;
                                if (!(bits & (1u << e))) v[c][e] = 0xff800000u;  // -inf
                            }
                            highest(c);
                        }
                    }
                    const float top = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]);
                    if (__any_sync(0xffffffffu, valid && (top - m) * sc > kLazy)) {
                        const float M = fmaxf(m, top), f = m == M ? 1.0f : ex2((m - M) * sc);
                        m = M;
                        l *= f;
                        if (i > 0) {
                            if (!(ok = wait_warp(odone(w), (done + i - 1) & 1u, abort))) break;
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < D; c += 16) {  // few columns: the scores stay in registers
                                uint32_t o[16];
                                tmem_ld16(tO + w * 128u + c, o);
                                tmem_wait_ld();
                                tmem_landed(o);
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_st16(tO + w * 128u + c, o);
                            }
                        }
                    }
                    const float neg = (m == -INFINITY ? 0.0f : -m * sc) + H::kShift;
                    const uint64_t sc2 = pack2(sc, sc), neg2 = pack2(neg, neg);
                    uint64_t sum[2] = {0, 0};
                    auto weights = [&](int c) {  // of 32 keys, into tensor memory
                        uint32_t pk[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float x0, x1;
                            unpack2(fma2(pack2(__uint_as_float(v[c][2 * e]), __uint_as_float(v[c][2 * e + 1])), sc2, neg2), x0, x1);
                            x0 = ex2(x0);
                            x1 = ex2(x1);
                            sum[e & 1] = add2(sum[e & 1], pack2(x0, x1));
                            pk[e] = H::pack(x0, x1);
                        }
                        tmem_st16(tS + c * 16, pk);
                    };
                    weights(0);
                    weights(1);
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(pready(w, 0));
                    weights(2);
                    weights(3);
                    float s0, s1;
                    unpack2(add2(sum[0], sum[1]), s0, s1);
                    l += s0 + s1;
                    tmem_wait_st();
                } else {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(pready(w, 0));
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pready(w, 1));
            }
            if (!ok) break;
            // ---- the segment's result
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
            const uint32_t tiles = i, tiles_other = n + (two ? n : 0) - i;
            if (tiles > 0) ok = wait_warp(odone(w), (done + tiles - 1) & 1u, abort);
            if (!ok) break;
            m = fmaxf(m * sc, -INFINITY);  // log2 of the largest weight (-inf stays, whatever the scale)
            if (l != l) m = INFINITY;  // a score that is not a number, or infinite: so is the row, whatever it is joined with
            float f = 1.0f, f1 = 0.0f;  // factors of the first accumulator (the stream's own) and, of one tile, the second
            if (!two) {
                s_ml[w * 128 + r] = make_float2(m, l);
                if (!(ok = seg_sync())) break;
                if (tiles_other > 0 && !(ok = wait_warp(odone(w ^ 1u), (done_other + tiles_other - 1) & 1u, abort))) break;
                const float2 x = s_ml[r], y = s_ml[128 + r];
                m = fmaxf(x.x, y.x);
                f = x.x == -INFINITY ? 0.0f : ex2(x.x - m);
                f1 = y.x == -INFINITY ? 0.0f : ex2(y.x - m);
                l = x.y * f + y.y * f1;
            }
            if constexpr (Q4) {
                f *= vu;
                f1 *= vu;
            }
            tc_fence_after();
            if (busy) {
                if (whole) {
                    const float inv = l > 0.0f ? 1.0f / l : l;  // (l: zero, or not a number)
                    f *= inv;
                    f1 *= inv;
                }
                const uint32_t first = two ? w : 0u;
                const int from = two ? 0 : (int)w * (DC / 2), to = two ? DC : from + DC / 2;
                // the quad's rows: where they go, which of them are there
                const unsigned long long out = reinterpret_cast<unsigned long long>(
                    static_cast<T*>(a.out.p) + (int64_t)(W.q.off + tok) * a.out.tok + head * a.out.head);
                unsigned long long out4[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) out4[k] = __shfl_sync(0xffffffffu, out, (lane & ~3) + k);
                const uint32_t rows4 = __ballot_sync(0xffffffffu, valid) >> (lane & ~3) & 15u;
                float* part = P.part_o + ((int64_t)slot * P.cap_rows + in_block) * DC;
                if (valid && (two || w == 0)) {
                    if (!whole)
                        P.part_ml[(int64_t)slot * P.cap_rows + in_block] = make_float2(m, l);
                    else if (a.lse)
                        a.lse[(int64_t)(W.q.off + tok) * a.n_heads + head] =
                            l == 0.0f ? -INFINITY : (m + log2f(l) - H::kShift) * 0.69314718055994531f;
                }
                int kind = (whole ? 1 : 0) | (!two && n > 1 ? 2 : 0);
#pragma unroll 1
                for (int c = from; c < to && c < D; c += 32) {
                    asm volatile("" : "+r"(kind));  // one body for all kinds: the compiler would make a loop of each
                    uint32_t o[32];
                    if (n > 0) {
                        tmem_ld32(tO + first * 128u + c, o);
                        tmem_wait_ld();
                        tmem_landed(o);
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        o[e] = n > 0 && f != 0.0f ? __float_as_uint(__uint_as_float(o[e]) * f) : 0u;
                    if (kind & 2) {
                        uint32_t o1[32];
                        tmem_ld32(tO + 128u + c, o1);
                        tmem_wait_ld();
                        tmem_landed(o1);
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (f1 != 0.0f) o[e] = __float_as_uint(fmaf(__uint_as_float(o1[e]), f1, __uint_as_float(o[e])));
                    }
                    const int q = lane & 3;
                    if (kind & 1) {
                        uint4 u[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t* x = o + 8 * e;
                            u[e] = make_uint4(Half<T>::pack(__uint_as_float(x[0]), __uint_as_float(x[1])), Half<T>::pack(__uint_as_float(x[2]), __uint_as_float(x[3])),
                                              Half<T>::pack(__uint_as_float(x[4]), __uint_as_float(x[5])), Half<T>::pack(__uint_as_float(x[6]), __uint_as_float(x[7])));
                        }
                        quad_transpose(u, q);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if ((rows4 >> k & 1u) && c + 8 * q < D)
                                *reinterpret_cast<uint4*>(reinterpret_cast<T*>(out4[k]) + c + 8 * q) = u[k];
                    } else {
#pragma unroll
                        for (int b = 0; b < 32; b += 16) {
                            uint4 u[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) u[e] = make_uint4(o[b + 4 * e], o[b + 4 * e + 1], o[b + 4 * e + 2], o[b + 4 * e + 3]);
                            quad_transpose(u, q);
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (rows4 >> k & 1u) *reinterpret_cast<uint4*>(part + (k - q) * DC + c + b + 4 * q) = u[k];
                        }
                    }
                    __syncwarp();
                }
            }
            done += tiles;
            done_other += tiles_other;
            it += 2 * n;
            tc_fence_before();
            ok = seg_sync();  // the accumulators, queries and s_ml are free
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (tid == 0 && *abort && a.status) atomicOr(a.status, PPS_FLAG_TIMEOUT);
}

// the heads of a key head taken at a time, the tokens of a tile, the rows of a block
struct Rows {
    int nsub, gs, tt, cap;
    Rows(int64_t n_tok, int group) {
        nsub = (group + kTileRows - 1) / kTileRows;
        gs = (group + nsub - 1) / nsub;
        tt = kTileRows / gs;
        cap = n_tok > tt ? 2 * kTileRows : (int)((n_tok * gs + 31) / 32 * 32);
    }
};

// the queries as [key head, token, head of the group, channel], loaded in boxes of tt tokens x gs heads x 64 channels
bool query_map(CUtensorMap* m, const AttnArgs& a, const AttnPlan& P, int dtype) {
    EncodeTiledFn f = encode_fn();
    if (f == nullptr) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)a.c.head_dim, (cuuint64_t)P.group, (cuuint64_t)a.n_tok, (cuuint64_t)a.c.n_kv_heads};
    const cuuint64_t strides[3] = {P.group > 1 ? (cuuint64_t)a.q.head * 2 : 256, a.n_tok > 1 ? (cuuint64_t)a.q.tok * 2 : 256,
                                   a.c.n_kv_heads > 1 ? (cuuint64_t)a.q.head * P.group * 2 : 256};
    const cuuint32_t box[4] = {64, (cuuint32_t)P.gs, (cuuint32_t)P.tt, 1}, es[4] = {1, 1, 1, 1};
    return f(m, dtype == PPS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, a.q.p, dims, strides,
             box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace pps
