// pps_pages.cu -- page tables and slot maps from request lengths, on the GPU.
//
// reserve: sequence s is to hold kv_len + n_new tokens; what its page table lacks is taken from the top of the pool's stack, by
//          sequence and column; every new token gets its slot, position and sequence.
// trim:    pages behind the kept tokens go back, in the order in which reserve takes them again.
//
// Both are prefix sums over the sequences (tokens, pages), then independent writes.  Integer work on a few hundred kilobytes at
// most: a launch's latency bounds it, so one launch of one cluster does it all: every CTA forms all sums for itself in shared
// memory, the cluster waits until all have read the state, and the writes are dealt out (a token or a page finds its sequence by
// bisection, so that long and short ones cost the same).
#include <algorithm>
#include <atomic>
#include <cstdint>

#include "pps.h"
#include "pps_internal.h"

namespace pps {
namespace {

// At most (512 trees of 41 nodes, launched after the end of what is before: 8.4 us; with 1024 9.0, with 256 11.4; on its drain 7.6).
constexpr int kPageThreads = 512;
constexpr int kPageCluster = 8;

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

// exclusive sums over the CTA of two numbers per thread; their totals
__device__ __forceinline__ void scan2(int64_t& x, int64_t& y, int64_t& all_x, int64_t& all_y, longlong2* s) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t a = x, b = y;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t u = __shfl_up_sync(0xffffffffu, a, o), v = __shfl_up_sync(0xffffffffu, b, o);
        if (lane >= o) {
            a += u;
            b += v;
        }
    }
    __syncthreads();  // s is free
    if (lane == 31) s[warp] = make_longlong2(a, b);
    __syncthreads();
    x = a - x;
    y = b - y;
    all_x = all_y = 0;
    for (int w = 0; w < (int)blockDim.x / 32; ++w) {
        const longlong2 v = s[w];
        if (w < warp) {
            x += v.x;
            y += v.y;
        }
        all_x += v.x;
        all_y += v.y;
    }
}

// the last i of [0, n) with start[i] <= x (start[0] <= x, non-decreasing)
__device__ __forceinline__ int find(const int* start, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= x)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// (two lengths' sum is below 2^32; a division of 64 bits takes several times as long)
__device__ __forceinline__ uint32_t pages_of(uint32_t tokens, int page_size) { return tokens / (uint32_t)page_size + (tokens % (uint32_t)page_size != 0); }

__global__ void __launch_bounds__(kPageThreads) reserve_kernel(const ReserveArgs a) {
    extern __shared__ int s_seq[];  // [n_seq] each: tokens before it, pages before it, its length, its pages (~: not served)
    __shared__ longlong2 s_sum[kPageThreads / 32];
    const int n = a.n_seq, tid = threadIdx.x;
    int *s_tok = s_seq, *s_page = s_tok + n, *s_len = s_page + n, *s_held = s_len + n;
    const int rank = blockIdx.x, ranks = gridDim.x;  // one cluster
    pdl_wait();
    pdl_launch_dependents();
    const int avail = max(min(a.free_count[0], a.free_cap), 0);
    const int64_t most = INT32_MAX;
    __shared__ int s_granted;  // pages: the demands before the first one that the pool cannot meet
    if (tid == 0) s_granted = 0;
    int64_t tok0 = 0, page0 = 0;
    bool bad = false, out_of = false;
    for (int s0 = 0; s0 < n; s0 += blockDim.x) {
        const int s = s0 + tid;
        int64_t n_new = 0, need = 0;
        int len = 0, held = 0;
        bool fits = true;
        if (s < n) {
            const int nn = __ldg(a.n_new + s), ll = a.kv_len[s], hh = a.held[s];
            n_new = max(nn, 0);
            len = max(ll, 0);
            held = min(max(hh, 0), a.columns);
            bad |= nn < 0 || ll < 0 || hh != held;
            const int64_t want = pages_of((uint32_t)len + (uint32_t)n_new, a.page_size);
            // (one that holds fewer pages than its tokens take is not served: pages from the pool would stand for tokens that nothing wrote)
            fits = want <= a.columns && len <= (int64_t)held * a.page_size;
            if (fits) need = max(want - held, (int64_t)0);
        }
        int64_t x = n_new, y = need, all_x, all_y;
        scan2(x, y, all_x, all_y, s_sum);
        x += tok0;
        y += page0;
        if (s < n) {
            const bool served = fits && (need == 0 || y + need <= avail);
            if (!fits) bad = true;
            if (fits && !served) out_of = true;
            if (served && need > 0) atomicMax(&s_granted, (int)(y + need));
            s_tok[s] = (int)min(x, most);
            s_page[s] = (int)min(y, most);
            s_len[s] = len;
            s_held[s] = served ? held : ~held;
        }
        tok0 += all_x;
        page0 += all_y;
    }
    __syncthreads();
    const int granted = s_granted;
    cluster_sync();  // every CTA has read the state
    const int stride = blockDim.x * ranks, me = rank * blockDim.x + tid;
    // sequences
    for (int s = me; s < n; s += stride) {
        const int next_t = s + 1 < n ? s_tok[s + 1] : (int)min(tok0, most), next_p = s + 1 < n ? s_page[s + 1] : (int)min(page0, most);
        const bool served = s_held[s] >= 0;
        a.out_q_off[s] = s_tok[s];
        a.out_len[s] = served ? (int)min((int64_t)s_len[s] + (next_t - s_tok[s]), most) : 0;
        if (served && next_p > s_page[s]) a.held[s] = s_held[s] + (next_p - s_page[s]);
    }
    if (me == 0) {
        a.out_q_off[n] = (int)min(tok0, most);
        a.free_count[0] = avail - granted;
    }
    // pages
    for (int p = me; p < granted; p += stride) {
        const int s = find(s_page, n, p);
        a.pages[s * a.pages_stride + s_held[s] + (p - s_page[s])] = __ldg(a.free_list + (avail - 1 - p));
    }
    // tokens
    const int64_t tokens = min(tok0, a.n_tok);
    constexpr int kAtOnce = 4;
    for (int64_t i0 = me; i0 < a.n_tok; i0 += (int64_t)kAtOnce * stride) {
        int seq[kAtOnce], off[kAtOnce], page[kAtOnce];
        uint32_t in_page[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {  // what has to be loaded, on its way together
            const int64_t i = i0 + (int64_t)k * stride;
            seq[k] = -1;
            if (i >= tokens) continue;
            seq[k] = find(s_tok, n, (int)i);
            const int at = (int)i - s_tok[seq[k]], held = s_held[seq[k]];
            const uint32_t place = (uint32_t)s_len[seq[k]] + (uint32_t)at, col_ = place / (uint32_t)a.page_size;
            in_page[k] = place - col_ * (uint32_t)a.page_size;
            const int col = (int)col_;
            off[k] = a.pos_off ? __ldg(a.pos_off + i) : at;
            page[k] = held < 0 ? INT32_MIN : col < held ? a.pages[seq[k] * a.pages_stride + col] : __ldg(a.free_list + (avail - 1 - (s_page[seq[k]] + col - held)));
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int64_t i = i0 + (int64_t)k * stride;
            if (i >= a.n_tok) break;
            int64_t slot = -1;
            int pos = 0;
            if (seq[k] >= 0) {
                pos = s_len[seq[k]] + off[k];
                if (page[k] >= 0) slot = (int64_t)page[k] * a.page_size + in_page[k];
                bad |= page[k] < 0 && s_held[seq[k]] >= 0;
            }
            a.out_slot[i] = slot;
            a.out_pos[i] = pos;
            if (a.out_seq) a.out_seq[i] = seq[k];
        }
    }
    if (a.status && (bad || (tok0 > a.n_tok && me == 0))) atomicOr(a.status, PPS_FLAG_INDEX);
    if (a.status && out_of) atomicOr(a.status, PPS_FLAG_POOL);
}

__global__ void __launch_bounds__(kPageThreads) trim_kernel(const ReserveArgs a) {
    extern __shared__ int s_seq[];  // [n_seq] each: pages that sequences before it give back, the pages it keeps
    __shared__ longlong2 s_sum[kPageThreads / 32];
    const int n = a.n_seq, tid = threadIdx.x;
    int *s_back = s_seq, *s_keep = s_back + n;
    const int rank = blockIdx.x, ranks = gridDim.x;
    pdl_wait();
    pdl_launch_dependents();
    const int have = max(min(a.free_count[0], a.free_cap), 0);
    int64_t back0 = 0;
    bool bad = false;
    for (int s0 = 0; s0 < n; s0 += blockDim.x) {
        const int s = s0 + tid;
        int64_t back = 0;
        int keep = 0;
        if (s < n) {
            const int ll = __ldg(a.kv_len + s), hh = a.held[s], held = min(max(hh, 0), a.columns);
            const uint32_t want = pages_of(max(ll, 0), a.page_size);
            keep = (int)min(want, (uint32_t)held);
            bad |= ll < 0 || hh != held || want > (uint32_t)held;
            back = held - keep;
        }
        int64_t x = back, y = 0, all, none;
        scan2(x, y, all, none, s_sum);
        if (s < n) {
            s_back[s] = (int)min(back0 + x, (int64_t)INT32_MAX);
            s_keep[s] = keep;
        }
        back0 += all;
    }
    __syncthreads();
    cluster_sync();  // every CTA has read the state
    const int64_t total = min(back0, (int64_t)INT32_MAX);
    const int stride = blockDim.x * ranks, me = rank * blockDim.x + tid;
    for (int s = me; s < n; s += stride) a.held[s] = s_keep[s];
    const bool over = have + total > a.free_cap;  // more pages than there are: what passes the list's end is lost
    if (me == 0) a.free_count[0] = (int)min(have + total, (int64_t)a.free_cap);
    for (int64_t p = me; p < total; p += stride) {
        const int s = find(s_back, n, (int)p);
        int32_t* from = a.pages + s * a.pages_stride + s_keep[s] + (p - s_back[s]);
        const int64_t to = have + total - 1 - p;
        if (to < a.free_cap) a.free_list[to] = *from;
        *from = -1;
    }
    if (a.status && (bad || over)) atomicOr(a.status, PPS_FLAG_INDEX);
}

cudaError_t launch_cluster(void (*kernel)(const ReserveArgs), const ReserveArgs& a, int64_t items, int smem, std::atomic<uint64_t>& ready, cudaStream_t st) {
    cudaError_t e = allow_smem(ready, (const void*)kernel, 4 * (int)sizeof(int) * kMaxPageSeqs);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    // one CTA where its threads have a turn or two (2053 tokens: one 6.9 us; 5125: a cluster 5.2), else a cluster
    const int ctas = items <= 2 * kPageThreads ? 1 : kPageCluster;
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(ctas > 1 ? kPageThreads : (int)std::min<int64_t>(std::max<int64_t>((items + 31) / 32 * 32, 128), kPageThreads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // as launch_pdl
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

}  // namespace

cudaError_t launch_kv_reserve(const ReserveArgs& a, cudaStream_t stream) {
    static std::atomic<uint64_t> ready{0};
    return launch_cluster(reserve_kernel, a, std::max<int64_t>(a.n_tok, a.n_seq), 4 * (int)sizeof(int) * a.n_seq, ready, stream);
}

cudaError_t launch_kv_trim(const ReserveArgs& a, cudaStream_t stream) {
    static std::atomic<uint64_t> ready{0};
    return launch_cluster(trim_kernel, a, a.n_seq, 2 * (int)sizeof(int) * a.n_seq, ready, stream);
}

}  // namespace pps
