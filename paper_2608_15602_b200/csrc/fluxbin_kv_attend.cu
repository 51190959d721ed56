// Attention of new tokens over the 8-bit block-paged cache (fluxbin_kv_attend).
#include "fluxbin_cache.cuh"

using namespace fbd;

namespace {

constexpr int kThreads = 128;

struct Args {
    fluxbin_kv_cache_t c;
    int batch, tokens, q_heads, width;
    const void *q;
    long long q_token, q_head;
    const int *query_start, *lengths, *table;
    long long table_stride;
    float scale;
    void *out;
    long long out_token, out_head;
    float *lse;
};

__device__ __forceinline__ float block_max(float v, float *scratch)
{
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    return fmaxf(fmaxf(scratch[0], scratch[1]), fmaxf(scratch[2], scratch[3]));
}
__device__ __forceinline__ float block_sum(float v, float *scratch)
{
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    return (scratch[0] + scratch[1]) + (scratch[2] + scratch[3]);
}

// One CTA per (new token, query head).  128 cached tokens at a time: a thread forms the score of one token, then
// accumulates up to two elements of the output over all of them.
template <typename T, int FMT>
__global__ void __launch_bounds__(kThreads) attend_kernel(Args a)
{
    __shared__ float qs[256], ps[kThreads], scratch[4];
    __shared__ long long at[kThreads];
    wait_for_predecessor();
    const int t = blockIdx.x, h = blockIdx.y, D = a.c.head_dim, bs = a.c.block_tokens, kh = h / (a.q_heads / a.c.kv_heads);
    int r = t, first = t, last = t + 1;
    if (a.query_start) {
        // the request of the token: the last one that starts at or before it
        int lo = 0, hi = a.batch;
        while (hi - lo > 1) { const int m = (lo + hi) / 2; if (a.query_start[m] <= t) lo = m; else hi = m; }
        r = lo;
        first = min(max(a.query_start[r], 0), a.tokens);
        last = min(max(a.query_start[r + 1], 0), a.tokens);
        if (t < first || t >= last) return;
    }
    const long long length = min((long long)a.lengths[r], (long long)a.width * bs);
    const long long seen = length - (last - 1 - t);
    const T *q = (const T *)a.q + t * a.q_token + h * a.q_head;
    for (int e = threadIdx.x; e < D; e += kThreads) qs[e] = to_float(q[e]);
    __syncthreads();
    float m = -INFINITY, l = 0.f, acc[2] = {0.f, 0.f};
    for (long long j0 = 0; j0 < seen; j0 += kThreads) {
        const long long j = j0 + threadIdx.x;
        float x = -INFINITY, vs = 0.f;
        long long base = -1;
        if (j < seen) {
            const int b = a.table[r * a.table_stride + j / bs];
            if (b >= 0 && b < a.c.num_blocks) {
                base = b * a.c.block_stride + kh * a.c.head_stride + j % bs * a.c.token_stride;
                const unsigned char *kp = (const unsigned char *)a.c.d_k + base;
                x = 0.f;
                for (int e = 0; e < D; ++e) x = fmaf(qs[e], Entry<FMT>::load(kp[e]), x);
                x *= a.scale * a.c.d_k_scale[(long long)b * a.c.kv_heads + kh];
                vs = a.c.d_v_scale[(long long)b * a.c.kv_heads + kh];
            }
        }
        const float m_now = fmaxf(m, block_max(x, scratch));
        const float p = x == -INFINITY ? 0.f : expf(x - m_now), f = m == -INFINITY ? 0.f : expf(m - m_now);
        l = l * f + block_sum(p, scratch);
        ps[threadIdx.x] = p * vs;
        at[threadIdx.x] = base;
        m = m_now;
        __syncthreads();
        for (int i = 0; i < 2; ++i) {
            const int e = threadIdx.x + i * kThreads;
            acc[i] *= f;
            if (e < D)
                for (int k = 0; k < kThreads; ++k)
                    if (at[k] >= 0) acc[i] = fmaf(ps[k], Entry<FMT>::load(((const unsigned char *)a.c.d_v)[at[k] + e]), acc[i]);
        }
        __syncthreads();
    }
    T *out = (T *)a.out + t * a.out_token + h * a.out_head;
    for (int i = 0; i < 2; ++i)
        if (threadIdx.x + i * kThreads < D) out[threadIdx.x + i * kThreads] = from_float<T>(l == 0.f ? 0.f : acc[i] / l);
    if (a.lse && threadIdx.x == 0) a.lse[(long long)t * a.q_heads + h] = l == 0.f ? -INFINITY : m + logf(l);
}

template <typename T>
cudaError_t run(const Args &a, cudaStream_t s)
{
    const dim3 grid((unsigned)a.tokens, (unsigned)a.q_heads);
    if (a.c.format == FLUXBIN_CACHE_INT8) return launch(attend_kernel<T, FLUXBIN_CACHE_INT8>, grid, kThreads, 0, s, a);
    return launch(attend_kernel<T, FLUXBIN_CACHE_E4M3>, grid, kThreads, 0, s, a);
}

} // namespace

extern "C" size_t fluxbin_kv_attend_workspace_size(int32_t batch, int32_t tokens, int32_t q_heads, int32_t kv_heads, int32_t head_dim)
{
    if (batch < 1 || tokens < 0 || q_heads < 1 || kv_heads < 1 || q_heads % kv_heads != 0 || head_dim < 1) return 0;
    return 256;
}

extern "C" fluxbin_status_t fluxbin_kv_attend(const fluxbin_kv_cache_t *cache, int32_t dtype, int32_t batch, int32_t tokens,
                                              const void *d_q, int32_t q_heads, int64_t q_token, int64_t q_head,
                                              const int32_t *d_query_start, const int32_t *d_lengths,
                                              const int32_t *d_block_table, int64_t block_table_stride, int32_t block_table_width,
                                              float scale, void *d_out, int64_t out_token, int64_t out_head, float *d_lse,
                                              void *d_workspace, size_t ws_bytes, void *cuda_stream)
{
    const fluxbin_status_t st = check_cache(cache);
    if (st != FLUXBIN_OK) return st;
    if (dtype != FLUXBIN_TYPE_FP16 && dtype != FLUXBIN_TYPE_BF16) return FLUXBIN_ERR_UNSUPPORTED;
    if (batch < 1 || tokens < 0 || q_heads < 1 || q_heads > 65535 || q_heads % cache->kv_heads != 0 || block_table_width < 1 ||
        block_table_stride < block_table_width || (!d_query_start && tokens != batch)) return FLUXBIN_ERR_RANGE;
    if (tokens == 0) return FLUXBIN_OK;
    if (!d_q || !d_out || !d_lengths || !d_block_table || !d_workspace) return FLUXBIN_ERR_NULL;
    if (!aligned_to(d_q, 16) || !aligned_to(d_out, 16) || q_token % 8 || q_head % 8 || out_token % 8 || out_head % 8 ||
        !aligned_to(d_query_start, 4) || !aligned_to(d_lengths, 4) || !aligned_to(d_block_table, 4) || !aligned_to(d_lse, 4) ||
        !aligned_to(d_workspace, 16)) return FLUXBIN_ERR_ALIGNMENT;
    if (ws_bytes < fluxbin_kv_attend_workspace_size(batch, tokens, q_heads, cache->kv_heads, cache->head_dim)) return FLUXBIN_ERR_BUFFER_TOO_SMALL;
    const Args a = {*cache, batch, tokens, q_heads, block_table_width, d_q, q_token, q_head, d_query_start, d_lengths, d_block_table,
                    block_table_stride, scale, d_out, out_token, out_head, d_lse};
    cudaStream_t s = (cudaStream_t)cuda_stream;
    FBD_CUDA(dtype == FLUXBIN_TYPE_FP16 ? run<__half>(a, s) : run<__nv_bfloat16>(a, s));
    return FLUXBIN_OK;
}
