// pps_attention.cu -- attention of the newest tokens of each sequence over a paged cache (tcgen05, sm_103a).
//
//   out[i] = sum_j w_j v_j / sum_j w_j,   w_j = exp(scale q_i . k_j)   over the keys j that row i sees,
//
// with the running maximum and sum of an online softmax, so that every key and value is read once per row block.
//
// Rows.  The tokens of a sequence and the heads that share a key head (group; taken gs <= 128 at a time) are packed
// into rows, token after token, so that a decoding step's few rows read their keys once.  A tile is 128 rows (tensor
// memory's lanes) of which tt gs are used, tt = 128 / gs whole tokens: one TMA box of queries.  A row block is two
// tiles, or one where its tokens fit into one.  Keys are taken 128 at a time.
//
// Two streams.  Each of two softmax warpgroups drives one stream: scores S = Q K^T into its own 128 columns of
// tensor memory, weights P written over them in 16 bits, O += P V into its own accumulator (P is read from tensor
// memory).  A block of two tiles gives each stream a tile and both the same keys; a block of one tile gives
// both streams the same rows and every other key tile, and their results are merged at the end.  Either way the tensor
// cores work for one stream while the other is in its softmax.
//
// Softmax.  A thread owns a row.  O is rescaled only when a row's maximum has risen by more than 2^kLazy since the
// maximum in use (then by its own warpgroup, in place): the weights may pass 1 by that factor, which neither
// the fp32 sums nor the 16-bit types' ranges feel.  Weights are rounded to the cache's type for the second product
// (up to 2^-8 of each in bf16, 2^-11 in fp16, as the result's own rounding); their sum is formed before rounding.  The largest
// weight of a row is 2^kShift and loses nothing as long as its score is the maximum in use; below a later, larger one (by less than
// kLazy) it is any number, so a row with one key that matters may be off by one such rounding more.  Against 64 bits the error is 1.4 times
// that of a result formed in fp32 and rounded once (bf16 2.3e-3 to 1.7e-3, fp16 2.8e-4 to 2.1e-4): weights of 32 bits would double the products.
//
// Work split.  The line of pps_attn.cuh: equal shares, one per SM, joined by a second launch.
//
// Every wait gives up after tc::kWaitLimit polls and raises PPS_FLAG_TIMEOUT.
//
// Measured (bf16, 32 heads over 8 key heads of 128 channels unless said; a copy moves 6.78 TB/s, library products run
// at 1936 TFLOP/s):
//   64 sequences, a token each, up to 8000 keys      216 us = 6.1 TB/s, 0.91 of the copy's: bound by HBM
//   one sequence of 130001 keys, 28 over 4 heads      55 us = 4.8 TB/s: one segment per CTA, of which 8 us of start, end, join
//   64 trees of 41 nodes, up to 4100 keys            180 to 183 us = 4.0 TB/s: a key tile takes 3200 clocks (164 rows padded to 256), and
//                                                    CTAs go through 3.8 segments, 10000 clocks of start and end each
//   8192 tokens after 8192                          1030 to 1050 us = 1600 TFLOP/s, 0.82 of the library's rate: a key tile of two row tiles
//                                                    takes 2880 clocks, 2048 of them tensor work; the rest is the softmax's latency.
//                                                    Over seconds 1120 us = 1480 TFLOP/s, 0.86 of the library's sustained rate: the power
//                                                    limit (1.38 kW) takes the clock from 2070 to 1935 MHz
//   7 chunks of up to 777 tokens, 14 over 2 x 64      51 us = 380 TFLOP/s: 64 channels halve the products, not the softmax (2650 clocks)
//   one sequence of 900 keys                          13 us: some 6 us from the launch to the first scores, of which most is
//                                                    fetching each role's instructions; 4 us for the join
// Code size is speed here: with the wait loops unrolled by the compiler (198 KB of code, now 110) the long sequence took 66 us.
//
// Built and measured slower: P apart from S at 64 channels, so that the next scores need not wait for O += P V (3 to 5 percent: the
// softmax, not the products' latency, is what a tile takes); the next segment's page table read ahead by the loaders (1 percent);
// the plan made by every warp for itself (3 to 8 percent: more code at the start); four softmax warpgroups, half of a row's keys each
// (28 percent: a vote per tile on the common maximum, 96 registers, so that some scores are read twice); shares of at least 2, 4 or 8 key tiles (short
// contexts up to 45 percent).
#include <atomic>
#include <cstring>

#include "pps_attn_tiles.cuh"

namespace pps {
namespace {

// ---------------------------------------------------------------- host side

// one half of the cache as [page, head, token, channel], loaded in boxes of up to 128 tokens x 64 channels
bool cache_map(CUtensorMap* m, const void* ptr, const CacheView& c, int dtype) {
    EncodeTiledFn f = encode_fn();
    if (f == nullptr) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_size, (cuuint64_t)c.n_kv_heads,
                                (cuuint64_t)std::max<int64_t>(c.n_pages, 1)};
    // the stride of a dimension of one is never used, but has to be a multiple of 16 bytes
    const cuuint64_t strides[3] = {(cuuint64_t)c.tok * 2, c.n_kv_heads > 1 ? (cuuint64_t)c.head * 2 : 256,
                                   c.n_pages > 1 ? (cuuint64_t)c.page * 2 : 256};
    const cuuint32_t box[4] = {64, (cuuint32_t)std::min(kTileKeys, c.page_size), 1, 1}, es[4] = {1, 1, 1, 1};
    // What a miss brings into L2: no more than the rows fill, since their neighbours are other heads' and are read much later.
    // 35 sequences decoding over 20 / 4 heads, pages token by token, with 256 -> 64 bytes: 64 channels 133 -> 104 us, 80 203 -> 145,
    // 96 208 -> 153 (128 bytes: 177); rows that follow one another (pages head by head), of 72 channels: 256 180, 128 145, 64 150;
    // 128 channels: no difference.
    const auto fetch = c.head_dim % 128 == 0 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B
                       : c.tok == c.head_dim    ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B
                                                : CU_TENSOR_MAP_L2_PROMOTION_L2_64B;
    return f(m, dtype == PPS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
             const_cast<void*>(ptr), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, fetch,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int DC>
cudaError_t launch(const AttnArgs& a, int dtype, cudaStream_t st) {
    AttnPlan P;
    P.group = a.n_heads / a.c.n_kv_heads;
    const Rows rows(a.n_tok, P.group);
    P.nsub = rows.nsub;
    P.gs = rows.gs;
    P.tt = rows.tt;
    P.bt = 2 * rows.tt;
    P.fix = kFix;
    P.cap_rows = rows.cap;
    P.shift = Half<T>::kShift;
    plan_common(P, a);
    carve(P, a.ws, kMaxCtas);
    CUtensorMap tmQ, tmK, tmV;
    // an empty cache has nothing to read: any mapped memory will do for its maps
    if (!query_map(&tmQ, a, P, dtype) || !cache_map(&tmK, a.c.n_pages > 0 ? a.c.k : a.ws, a.c, dtype) || !cache_map(&tmV, a.c.n_pages > 0 ? a.c.v : a.ws, a.c, dtype))
        return cudaErrorInvalidValue;
    static std::atomic<uint64_t> ready{0};
    cudaError_t e = allow_smem(ready, (const void*)attention_kernel<T, DC, false>, Cfg<DC, false>::kSmem);
    if (e != cudaSuccess) return e;
    const int ctas = std::min(device_sm_count(), kMaxCtas);
    e = launch_pdl(attention_kernel<T, DC, false>, dim3(ctas), dim3(Cfg<DC, false>::kThreads), Cfg<DC, false>::kSmem, st, tmQ, tmK, tmV, a, P, Q4Rows());
    if (e != cudaSuccess) return e;
    return launch_pdl(join_kernel<T, DC>, dim3(ctas, join_blocks(a, P)), dim3(256), 0, st, a, P);
}

template <typename T>
cudaError_t by_channels(const AttnArgs& a, int dtype, cudaStream_t st) {
    return channel_class(a.c.head_dim) == 64 ? launch<T, 64>(a, dtype, st) : launch<T, 128>(a, dtype, st);
}

}  // namespace

size_t attention_workspace_bytes(int64_t n_tok, int n_heads, int n_kv_heads, int head_dim) {
    const int rows = Rows(n_tok, (n_heads + n_kv_heads - 1) / n_kv_heads).cap;
    return part_bytes(kMaxCtas, rows, head_dim);
}

cudaError_t launch_attention(const AttnArgs& a, int dtype, cudaStream_t stream) {
    return dtype == PPS_BF16 ? by_channels<__nv_bfloat16>(a, dtype, stream) : by_channels<__half>(a, dtype, stream);
}

}  // namespace pps
