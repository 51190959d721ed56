// Attention of drafted tokens that see the cache and, of each other, what their masks say (fluxbin_kv_attend_tree).
#include "fluxbin_kv_tree.cuh"

namespace {

// Rows that share a key head in an average request up to which the kernel for few rows is taken.  That kernel / the other, us, int8 and
// bf16 (with e4m3 and fp16 from 20 % less to 6 % more for that kernel, from 6 % less to 10 % more for the other):
//                                        16 requests of 8190      2000 tokens   500          100          one of 16000
//   64 query heads on 8 of 128, 16 rows  92 / 114                 43 / 45       26 / 28      20 / 17      35 / 43
//                               24       161 / 114                60 / 45       36 / 28      20 / 17      41 / 44
//   24 on 6 of 64, 32 rows               75 / 81                  35 / 33       19 / 21      13 / 15      25 / 31
//                  48                    101 / 81                 42 / 34       26 / 22      13 / 15      26 / 32
//   16 on 2 of 256, 32 rows              90 / 91                  40 / 49       23 / 33      14 / 24      36 / 235
//                   48                   124 / 92                 50 / 51       24 / 34      14 / 25      37 / 244
// Where the rule is wrong: 64 heads on 8 of 256 (32 rows 310 / 214), a request alone on two key heads of 256 (its 74 parts are joined one
// after the other, 256 elements of a row by one thread), and batches that mix wide trees with single tokens, since it goes by the average.
int few_rows(int head_dim) { return head_dim == 128 ? 16 : 32; }

// (what fluxbin_debug_tree_waits set)
std::atomic<unsigned> g_wait_limit{kWaitLimit};
std::atomic<int> g_withheld{-1};

template <typename T> cudaError_t run_type(Args a, char *workspace, cudaStream_t s)
{
    const long long rows = (long long)(a.q_heads / a.c.kv_heads) * ((a.tokens + a.batch - 1) / a.batch);
    if (rows <= few_rows(a.c.head_dim)) return run_dim<T, true>(a, s);
    a.arrived = (unsigned *)(workspace + kManyCountersAt);
    a.partial_lse = (float *)(workspace + kCounterBytes);
    a.partial = (float *)(workspace + kCounterBytes + kTreeLseBytes);
    a.wait_limit = g_wait_limit.load(std::memory_order_relaxed);
    a.withheld = g_withheld.load(std::memory_order_relaxed);
    const bool bf16 = !std::is_same<T, __half>::value;
    return a.c.head_dim == 64 ? launch_tree_64(a, bf16, s) : a.c.head_dim == 128 ? launch_tree_128(a, bf16, s) : launch_tree_256(a, bf16, s);
}

} // namespace

extern "C" size_t fluxbin_kv_attend_tree_workspace_size(int32_t batch, int32_t tokens, int32_t q_heads, int32_t kv_heads, int32_t head_dim)
{
    if (fluxbin_kv_attend_workspace_size(batch, tokens, q_heads, kv_heads, head_dim) == 0) return 0;
    return kCounterBytes + (kLseBytes > kTreeLseBytes ? kLseBytes : kTreeLseBytes) * (1 + (size_t)head_dim);
}

extern "C" fluxbin_status_t fluxbin_kv_attend_tree(const fluxbin_kv_cache_t *cache, int32_t dtype, int32_t batch, int32_t tokens,
                                                   const void *d_q, int32_t q_heads, int64_t q_token, int64_t q_head,
                                                   const int32_t *d_query_start, const int32_t *d_lengths,
                                                   const int32_t *d_tree, int64_t tree_stride, int32_t tree_words,
                                                   const int32_t *d_block_table, int64_t block_table_stride, int32_t block_table_width,
                                                   float scale, void *d_out, int64_t out_token, int64_t out_head, float *d_lse,
                                                   void *d_workspace, size_t ws_bytes, void *cuda_stream)
{
    const fluxbin_status_t st = check_cache(cache);
    if (st != FLUXBIN_OK) return st;
    if (dtype != FLUXBIN_TYPE_FP16 && dtype != FLUXBIN_TYPE_BF16) return FLUXBIN_ERR_UNSUPPORTED;
    if (batch < 1 || tokens < 0 || q_heads < 1 || q_heads > 65535 || q_heads % cache->kv_heads != 0 || block_table_width < 1 ||
        (block_table_stride != 0 && block_table_stride < block_table_width) || (!d_query_start && tokens != batch) || tree_words < 1 ||
        tree_words > INT32_MAX / 32 || tree_stride < 0 || (int64_t)tokens * (q_heads / cache->kv_heads) > INT32_MAX) return FLUXBIN_ERR_RANGE;
    if (tokens == 0) return FLUXBIN_OK;
    if (!d_q || !d_out || !d_lengths || !d_block_table || !d_tree || !d_workspace) return FLUXBIN_ERR_NULL;
    if (!aligned_to(d_q, 16) || !aligned_to(d_out, 16) || (tokens > 1 && (q_token % 8 || out_token % 8)) || (q_heads > 1 && (q_head % 8 || out_head % 8)) ||
        !aligned_to(d_query_start, 4) || !aligned_to(d_lengths, 4) || !aligned_to(d_block_table, 4) || !aligned_to(d_tree, 4) || !aligned_to(d_lse, 4) ||
        !aligned_to(d_workspace, 16)) return FLUXBIN_ERR_ALIGNMENT;
    if (!heads_apart(tokens, q_heads, out_token, out_head, cache->head_dim)) return FLUXBIN_ERR_RANGE;
    if (ws_bytes < fluxbin_kv_attend_tree_workspace_size(batch, tokens, q_heads, cache->kv_heads, cache->head_dim)) return FLUXBIN_ERR_BUFFER_TOO_SMALL;
    const Args a = {*cache, batch, tokens, q_heads, block_table_width, d_q, q_token, q_head, d_query_start, d_lengths, d_block_table,
                    block_table_stride, scale, d_out, out_token, out_head, d_lse,
                    (unsigned *)d_workspace, (unsigned *)d_workspace + 1, (float *)((char *)d_workspace + kCounterBytes),
                    (float *)((char *)d_workspace + kCounterBytes + kLseBytes), (const uint32_t *)d_tree, tree_stride, tree_words};
    cudaStream_t s = (cudaStream_t)cuda_stream;
    FBD_CUDA((dtype == FLUXBIN_TYPE_FP16 ? run_type<__half>(a, (char *)d_workspace, s) : run_type<__nv_bfloat16>(a, (char *)d_workspace, s)));
    return FLUXBIN_OK;
}

extern "C" fluxbin_status_t fluxbin_debug_tree_waits(int64_t limit_ns, int32_t withheld)
{
    if (limit_ns < 0 || limit_ns > (int64_t)kWaitLimit || withheld < -1) return FLUXBIN_ERR_RANGE;
    g_wait_limit.store(limit_ns ? (unsigned)limit_ns : kWaitLimit, std::memory_order_relaxed);
    g_withheld.store(withheld, std::memory_order_relaxed);
    return FLUXBIN_OK;
}
