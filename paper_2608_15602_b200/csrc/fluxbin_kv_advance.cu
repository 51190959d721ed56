// Block tables and slot maps of a step, from request lengths (fluxbin_kv_advance).
#include "fluxbin_device.cuh"

using namespace fbd;

namespace {

constexpr int kThreads = 1024;

struct Args {
    int batch, tokens, bs, width, capacity;
    const int *lengths, *fresh, *num_free;
    int *table, *free;
    long long table_stride;
    int *num_free_out, *lengths_out, *granted, *query_start, *positions, *slots, *requests;
};

// inclusive sum over the CTA
__device__ __forceinline__ long long block_scan(long long v, long long *scratch)
{
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += up;
    }
    __syncthreads();
    if (lane == 31) scratch[w] = v;
    __syncthreads();
    for (int i = 0; i < w; ++i) v += scratch[i];
    return v;
}

// One CTA; a thread per request, in passes of 1024 requests.  Pass 1 returns blocks, pass 2 takes them.
__global__ void __launch_bounds__(kThreads) advance_kernel(Args a)
{
    __shared__ long long scratch[kThreads / 32];
    __shared__ long long carry[3];
    wait_for_predecessor();
    const int bs = a.bs;
    const long long nf = min(max(a.num_free[0], 0), a.capacity);
    if (threadIdx.x < 3) carry[threadIdx.x] = 0;
    for (int r0 = 0; r0 < a.batch; r0 += kThreads) {
        const int r = r0 + threadIdx.x;
        long long gone = 0, had = 0, want = 0;
        if (r < a.batch) {
            const long long len = max(a.lengths[r], 0), n = a.fresh[r];
            had = (len + bs - 1) / bs;
            want = (max(len + n, 0ll) + bs - 1) / bs;
            gone = max(had - want, 0ll);
            if (had > a.width) gone = 0;
        }
        __syncthreads();
        const long long base = carry[0], upto = block_scan(gone, scratch) + base;
        for (long long i = 0; i < gone; ++i) {
            const long long at = nf + upto - gone + i;
            if (at < a.capacity) a.free[at] = a.table[r * a.table_stride + want + i];
        }
        __syncthreads();
        if (threadIdx.x == kThreads - 1) carry[0] = upto;
    }
    __syncthreads();
    const long long end = min(nf + carry[0], (long long)a.capacity);
    long long taken = 0;
    for (int r0 = 0; r0 < a.batch; r0 += kThreads) {
        const int r = r0 + threadIdx.x;
        long long len = 0, n = 0, had = 0, want = 0, need = 0;
        bool fits = true;
        if (r < a.batch) {
            len = max(a.lengths[r], 0);
            n = a.fresh[r];
            had = (len + bs - 1) / bs;
            want = (max(len + n, 0ll) + bs - 1) / bs;
            fits = want <= a.width && len + n <= INT32_MAX;
            need = fits ? max(want - had, 0ll) : 0;
        }
        __syncthreads();
        const long long b1 = carry[1], b2 = carry[2];
        const long long asked = block_scan(need, scratch) + b1, upto = block_scan(max(n, 0ll), scratch) + b2;
        const bool ok = n <= 0 || (fits && (need == 0 || asked <= end));
        if (r < a.batch) {
            for (long long i = 0; ok && i < need; ++i) a.table[r * a.table_stride + had + i] = a.free[end - 1 - (asked - need) - i];
            a.lengths_out[r] = (int)(ok ? max(len + n, 0ll) : len);
            a.granted[r] = ok;
            const long long first = upto - max(n, 0ll);
            a.query_start[r] = (int)min(first, (long long)INT32_MAX);
            for (long long i = 0; i < n && first + i < a.tokens; ++i) {
                const long long p = len + i;
                a.positions[first + i] = (int)p;
                const long long b = ok ? a.table[r * a.table_stride + p / bs] : -1, s = b * bs + p % bs;
                a.slots[first + i] = b >= 0 && s <= INT32_MAX ? (int)s : -1;
                a.requests[first + i] = r;
            }
            if (ok && need > 0) taken = asked;
        }
        __syncthreads();
        if (threadIdx.x == kThreads - 1) { carry[1] = asked; carry[2] = upto; }
    }
    // what the last granted request had asked for in all
    for (int o = 16; o; o >>= 1) taken = max(taken, __shfl_xor_sync(0xffffffffu, taken, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = taken;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 0; i < kThreads / 32; ++i) taken = max(taken, scratch[i]);
        a.num_free_out[0] = (int)(end - taken);
        a.query_start[a.batch] = (int)min(carry[2], (long long)INT32_MAX);
    }
    for (long long t = carry[2] + threadIdx.x; t < a.tokens; t += kThreads) {
        a.positions[t] = 0;
        a.slots[t] = -1;
        a.requests[t] = -1;
    }
}

} // namespace

extern "C" fluxbin_status_t fluxbin_kv_advance(int32_t batch, int32_t tokens, int32_t block_tokens, const int32_t *d_lengths,
                                               const int32_t *d_new, int32_t *d_table, int64_t table_stride, int32_t table_width,
                                               int32_t *d_free, int32_t free_capacity, const int32_t *d_num_free,
                                               int32_t *d_num_free_out, int32_t *d_lengths_out, int32_t *d_granted,
                                               int32_t *d_query_start, int32_t *d_positions, int32_t *d_slots, int32_t *d_requests,
                                               void *cuda_stream)
{
    if (batch < 1 || batch > 8192 || tokens < 0 || block_tokens < 1 || block_tokens > 1024 || table_width < 1 || table_stride < table_width ||
        free_capacity < 1) return FLUXBIN_ERR_RANGE;
    if (!d_lengths || !d_new || !d_table || !d_free || !d_num_free || !d_num_free_out || !d_lengths_out || !d_granted || !d_query_start ||
        (tokens > 0 && (!d_positions || !d_slots || !d_requests))) return FLUXBIN_ERR_NULL;
    if (d_lengths == d_lengths_out || d_num_free == d_num_free_out) return FLUXBIN_ERR_RANGE;
    const void *all[] = {d_lengths, d_new, d_table, d_free, d_num_free, d_num_free_out, d_lengths_out, d_granted, d_query_start, d_positions, d_slots, d_requests};
    for (const void *p : all)
        if (!aligned_to(p, 4)) return FLUXBIN_ERR_ALIGNMENT;
    const Args a = {batch, tokens, block_tokens, table_width, free_capacity, d_lengths, d_new, d_num_free, d_table, d_free, table_stride,
                    d_num_free_out, d_lengths_out, d_granted, d_query_start, d_positions, d_slots, d_requests};
    FBD_CUDA(launch(advance_kernel, dim3(1), kThreads, 0, (cudaStream_t)cuda_stream, a));
    return FLUXBIN_OK;
}
