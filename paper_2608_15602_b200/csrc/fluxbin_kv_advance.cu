// Block tables and slot maps of a step, from request lengths (fluxbin_kv_advance).
#include "fluxbin_device.cuh"

#include <atomic>

using namespace fbd;

namespace {

constexpr int kMaxBatch = 8192, kWarpSums = 3 * 32;
constexpr unsigned kMany = 0xffffffffu;         // sums stay there once they get there: past every size

struct Args {
    int batch, tokens, bs, width, capacity;
    const int *lengths, *fresh, *num_free;
    int *table, *free;
    long long table_stride;
    int *num_free_out, *lengths_out, *granted, *query_start, *positions, *slots, *requests;
};

// what a step does to one request
struct Change {
    long long len, n;            // its length and its new tokens (< 0: dropped ones)
    int had, want;               // blocks before and after
    unsigned gone, need, count;  // blocks given back, blocks asked for, tokens added
    bool fits;
};
__device__ __forceinline__ Change change_of(const Args &a, int r)
{
    Change c;
    c.len = max(a.lengths[r], 0);
    c.n = a.fresh[r];
    const long long after = max(c.len + c.n, 0ll);
    const long long had = (c.len + a.bs - 1) / a.bs, want = (after + a.bs - 1) / a.bs;
    c.fits = want <= a.width && after <= INT32_MAX;
    c.had = (int)had;
    c.want = (int)want;
    c.gone = had > want && had <= a.width ? (unsigned)(had - want) : 0;
    c.need = c.fits && want > had ? (unsigned)(want - had) : 0;
    c.count = c.n > 0 ? (unsigned)c.n : 0;
    return c;
}
__device__ __forceinline__ unsigned add(unsigned x, unsigned y) { return x + y < x ? kMany : x + y; }

// the first entry of an ascending array that is above x
__device__ __forceinline__ int first_above(const unsigned *sums, int n, unsigned x)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int m = (lo + hi) / 2;
        if (sums[m] > x) hi = m; else lo = m + 1;
    }
    return lo;
}

// Three running sums over the requests -- blocks given back, blocks asked for, new tokens -- say where everything goes, so
// that no block, slot or token waits for another: each is a thread that looks its request up in the sums.  Every CTA
// forms the sums for itself (a few thousand integers); a block that is given back and taken again in one step is read
// where its last owner's table has it, not from the free list that another CTA is writing.
__global__ void __launch_bounds__(1024) advance_kernel(const __grid_constant__ Args a)
{
    extern __shared__ unsigned sums[];           // [3][32] of the warps, then [3][batch], including the request itself
    unsigned (&warp_sum)[3][32] = *reinterpret_cast<unsigned (*)[3][32]>(sums);
    unsigned *gone = sums + kWarpSums, *need = gone + a.batch, *count = need + a.batch;
    const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 31, warp = tid >> 5;
    let_successor_start();
    wait_for_predecessor();
    const int per = (a.batch + threads - 1) / threads, lo = min(tid * per, a.batch), hi = min(lo + per, a.batch);
    const int nf = min(max(a.num_free[0], 0), a.capacity);
    unsigned mine[3] = {0, 0, 0};
    for (int r = lo; r < hi; ++r) {
        const Change c = change_of(a, r);
        gone[r] = mine[0] = add(mine[0], c.gone);
        need[r] = mine[1] = add(mine[1], c.need);
        count[r] = mine[2] = add(mine[2], c.count);
    }
    unsigned upto[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        upto[k] = mine[k];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned x = __shfl_up_sync(0xffffffffu, upto[k], o);
            if (lane >= o) upto[k] = add(upto[k], x);
        }
        if (lane == 31) warp_sum[k][warp] = upto[k];
        upto[k] = __shfl_up_sync(0xffffffffu, upto[k], 1);       // of the threads before
        if (lane == 0) upto[k] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        unsigned x = lane < warp ? warp_sum[k][lane] : 0;
#pragma unroll
        for (int o = 16; o; o >>= 1) x = add(x, __shfl_xor_sync(0xffffffffu, x, o));
        upto[k] = add(upto[k], x);
    }
    for (int r = lo; r < hi; ++r) {
        gone[r] = add(gone[r], upto[0]);
        need[r] = add(need[r], upto[1]);
        count[r] = add(count[r], upto[2]);
    }
    __syncthreads();

    const unsigned back = min(gone[a.batch - 1], (unsigned)(a.capacity - nf)), end = (unsigned)nf + back;
    const int over = first_above(need, a.batch, end);            // the first request whose blocks are not there
    const unsigned taken = over > 0 ? need[over - 1] : 0;
    const unsigned added = min(count[a.batch - 1], (unsigned)a.tokens);
    auto given_back = [&](unsigned i) {
        const int r = first_above(gone, a.batch, i);
        return a.table[r * a.table_stride + change_of(a, r).want + (i - (r > 0 ? gone[r - 1] : 0))];
    };
    auto taken_block = [&](unsigned i) {         // the i-th block asked for, off the end of the list
        const unsigned at = end - 1 - i;
        return at >= (unsigned)nf ? given_back(at - nf) : a.free[at];
    };
    auto is_granted = [&](const Change &c, int r) { return c.n <= 0 || (c.fits && (c.need == 0 || need[r] <= end)); };

    const unsigned step = gridDim.x * threads, first = blockIdx.x * threads + tid;
    for (unsigned i = first; i < (unsigned)a.batch; i += step) {
        const Change c = change_of(a, i);
        const bool ok = is_granted(c, i);
        a.lengths_out[i] = (int)(ok ? max(c.len + c.n, 0ll) : c.len);
        a.granted[i] = ok;
        a.query_start[i + 1] = (int)min(count[i], (unsigned)INT32_MAX);
    }
    for (unsigned i = first; i < (unsigned)a.tokens; i += step) {
        int p = 0, slot = -1, r = -1;
        if (i < added) {
            r = first_above(count, a.batch, i);
            const Change c = change_of(a, r);
            const long long at = c.len + (i - (r > 0 ? count[r - 1] : 0));
            p = (int)min(at, (long long)INT32_MAX);
            if (is_granted(c, r)) {
                const int b = (int)(at / a.bs);
                const long long id = b < c.had ? a.table[r * a.table_stride + b] : taken_block((r > 0 ? need[r - 1] : 0) + (b - c.had));
                const long long s = id * a.bs + at % a.bs;
                slot = id >= 0 && s <= INT32_MAX ? (int)s : -1;
            }
        }
        a.positions[i] = p;
        a.slots[i] = slot;
        a.requests[i] = r;
    }
    for (unsigned i = first; i < taken; i += step) {
        const int r = first_above(need, a.batch, i);
        a.table[r * a.table_stride + change_of(a, r).had + (i - (r > 0 ? need[r - 1] : 0))] = taken_block(i);
    }
    for (unsigned i = first; i < back; i += step) a.free[nf + i] = given_back(i);
    if (first == 0) {
        a.num_free_out[0] = (int)(end - taken);
        a.query_start[0] = 0;
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
    if (batch < 1 || batch > kMaxBatch || tokens < 0 || block_tokens < 1 || block_tokens > 1024 || table_width < 1 || table_stride < table_width ||
        free_capacity < 1) return FLUXBIN_ERR_RANGE;
    if (!d_lengths || !d_new || !d_table || !d_free || !d_num_free || !d_num_free_out || !d_lengths_out || !d_granted || !d_query_start ||
        (tokens > 0 && (!d_positions || !d_slots || !d_requests))) return FLUXBIN_ERR_NULL;
    if (d_lengths == d_lengths_out || d_num_free == d_num_free_out) return FLUXBIN_ERR_RANGE;
    const void *all[] = {d_lengths, d_new, d_table, d_free, d_num_free, d_num_free_out, d_lengths_out, d_granted, d_query_start, d_positions, d_slots, d_requests};
    for (const void *p : all)
        if (!aligned_to(p, 4)) return FLUXBIN_ERR_ALIGNMENT;
    const Args a = {batch, tokens, block_tokens, table_width, free_capacity, d_lengths, d_new, d_num_free, d_table, d_free, table_stride,
                    d_num_free_out, d_lengths_out, d_granted, d_query_start, d_positions, d_slots, d_requests};
    // CTAs for the tokens (at most one on each of 148 SMs); narrow ones while a thread has few requests to sum up (256 against
    // 1024 threads: 200 requests 6.2 us against 7.7, 1024 with 33 K tokens 11.0 against 12.4, 2000 16.4 both, 4000 24.9 against
    // 19.1, 8000 63 against 29)
    const int threads = batch <= 2048 ? 256 : 1024;
    const int64_t ctas = ((int64_t)tokens + threads - 1) / threads;
    const size_t smem = ((size_t)batch * 3 + kWarpSums) * sizeof(unsigned);
    if (smem > 48 * 1024) {
        static std::atomic<bool> opted[fb::kMaxDevices];
        int dev = 0;
        FBD_CUDA(cudaGetDevice(&dev));
        if (dev < 0 || dev >= fb::kMaxDevices) return FLUXBIN_ERR_UNSUPPORTED;
        if (!opted[dev].load(std::memory_order_relaxed)) {
            FBD_CUDA(cudaFuncSetAttribute(advance_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (kMaxBatch * 3 + kWarpSums) * (int)sizeof(unsigned)));
            opted[dev].store(true, std::memory_order_relaxed);
        }
    }
    FBD_CUDA(launch(advance_kernel, dim3((unsigned)(ctas < 1 ? 1 : ctas < 148 ? ctas : 148)), threads, smem, (cudaStream_t)cuda_stream, a));
    return FLUXBIN_OK;
}
