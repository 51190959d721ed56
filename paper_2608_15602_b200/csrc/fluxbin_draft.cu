// Trees of drafted tokens: from their parents to masks and positions (fluxbin_draft_tree), and from the model's answers to the
// path that it would have taken (fluxbin_draft_accept).  A CTA or a warp for each request, the request's tokens in shared memory.
// Bound by the launch and two dependent reads.
#include "fluxbin_device.cuh"

using namespace fbd;

namespace {

constexpr int kMaxNodes = 1024;

struct Span { int first, count; };
__device__ __forceinline__ Span span_of(const int *query_start, int r, int tokens)
{
    const int a = min(max(query_start[r], 0), tokens), b = min(max(query_start[r + 1], 0), tokens);
    return {a, max(b - a, 0)};
}
// what = f(token) for tokens that are no request's, by one CTA
template <typename F> __device__ __forceinline__ void others(const int *query_start, int batch, int tokens, F f)
{
    const int from = min(max(query_start[0], 0), tokens), to = min(max(query_start[batch], from), tokens);
    for (int i = threadIdx.x; i < tokens - (to - from); i += blockDim.x) f(i < from ? i : i + (to - from));
}

struct TreeArgs {
    int batch, tokens, nodes, words;
    const int *query_start, *lengths, *parents;
    int *mask, *positions;
};
// A thread for each token walks up its ancestors.  They come in descending order, so a word of the mask is complete once a
// lower one is met.
__global__ void __launch_bounds__(256) tree_kernel(const __grid_constant__ TreeArgs a)
{
    extern __shared__ int parent[];
    const int r = blockIdx.x, tid = threadIdx.x;
    let_successor_start();
    wait_for_predecessor();
    if (r == 0)
        others(a.query_start, a.batch, a.tokens, [&](int t) {
            for (int w = 0; w < a.words; ++w) a.mask[(long long)t * a.words + w] = 0;
            a.positions[t] = 0;
        });
    const Span s = span_of(a.query_start, r, a.tokens);
    const int base = (int)max((long long)max(a.lengths[r], 0) - s.count, 0ll), n = min(s.count, a.nodes);
    for (int i = tid; i < n; i += blockDim.x) {
        const int p = a.parents[s.first + i];
        parent[i] = p >= 0 && p < i ? p : -1;
    }
    __syncthreads();
    for (int i = tid; i < s.count; i += blockDim.x) {
        int *row = a.mask + (long long)(s.first + i) * a.words;
        int depth = 0, word = a.words - 1;
        if (i < n) {
            unsigned bits = 0;
            depth = -1;
            for (int j = i; j >= 0; j = parent[j]) {
                for (; word > j / 32; --word) {
                    row[word] = (int)bits;
                    bits = 0;
                }
                bits |= 1u << (j % 32);
                ++depth;
            }
            row[word--] = (int)bits;
        }
        for (; word >= 0; --word) row[word] = 0;
        a.positions[s.first + i] = base + depth;
    }
}

struct AcceptArgs {
    int batch, tokens, nodes;
    const int *query_start, *parents, *drafted, *answers;
    int *path, *count, *answer, *surplus;
};
// A warp for each request: 32 tokens at a time are asked whether they are the next of the path.  The next one lies behind the
// last, so the tokens are gone through once.
__global__ void __launch_bounds__(32) accept_kernel(const __grid_constant__ AcceptArgs a)
{
    extern __shared__ int node[];                // parents, drafted tokens, answers
    const int r = blockIdx.x, lane = threadIdx.x;
    let_successor_start();
    wait_for_predecessor();
    if (r == 0) others(a.query_start, a.batch, a.tokens, [&](int t) { a.path[t] = -1; });
    const Span s = span_of(a.query_start, r, a.tokens);
    const int n = min(s.count, a.nodes);
    int *parent = node, *drafted = node + a.nodes, *answers = node + 2 * a.nodes;
    for (int i = lane; i < n; i += 32) {
        parent[i] = a.parents[s.first + i];
        drafted[i] = a.drafted[s.first + i];
        answers[i] = a.answers[s.first + i];
    }
    __syncwarp();
    int count = 0, said = -1;
    if (n > 0) {
        int last = 0;
        said = answers[0];
        if (lane == 0) a.path[s.first] = 0;
        count = 1;
        for (int i = 0; i < n;) {                // from a whole 32 on
            const int at = i + lane;
            const unsigned next = __ballot_sync(0xffffffffu, at < n && at > last && parent[at] == last && drafted[at] == said);
            if (next == 0) {
                i += 32;
                continue;
            }
            last = i + __ffs(next) - 1;
            said = answers[last];
            if (lane == 0) a.path[s.first + count] = last;
            ++count;
        }
    }
    for (int i = count + lane; i < s.count; i += 32) a.path[s.first + i] = -1;
    if (lane == 0) {
        a.count[r] = count;
        a.answer[r] = said;
        a.surplus[r] = count - s.count;
    }
}

fluxbin_status_t check(int batch, int tokens, int nodes)
{
    return batch < 1 || tokens < 0 || nodes < 1 || nodes > kMaxNodes ? FLUXBIN_ERR_RANGE : FLUXBIN_OK;
}

} // namespace

extern "C" fluxbin_status_t fluxbin_draft_tree(int32_t batch, int32_t tokens, int32_t nodes, const int32_t *d_query_start, const int32_t *d_lengths,
                                               const int32_t *d_parents, int32_t *d_mask, int32_t *d_positions, void *cuda_stream)
{
    const fluxbin_status_t st = check(batch, tokens, nodes);
    if (st != FLUXBIN_OK) return st;
    if (tokens == 0) return FLUXBIN_OK;
    if (!d_query_start || !d_lengths || !d_parents || !d_mask || !d_positions) return FLUXBIN_ERR_NULL;
    for (const void *p : {(const void *)d_query_start, (const void *)d_lengths, (const void *)d_parents, (const void *)d_mask, (const void *)d_positions})
        if (!aligned_to(p, 4)) return FLUXBIN_ERR_ALIGNMENT;
    const TreeArgs a = {batch, tokens, nodes, (nodes + 31) / 32, d_query_start, d_lengths, d_parents, d_mask, d_positions};
    const int threads = nodes >= 256 ? 256 : (nodes + 31) / 32 * 32;
    FBD_CUDA(launch(tree_kernel, dim3((unsigned)batch), threads, sizeof(int) * nodes, (cudaStream_t)cuda_stream, a));
    return FLUXBIN_OK;
}

extern "C" fluxbin_status_t fluxbin_draft_accept(int32_t batch, int32_t tokens, int32_t nodes, const int32_t *d_query_start, const int32_t *d_parents,
                                                 const int32_t *d_drafted, const int32_t *d_answers, int32_t *d_path, int32_t *d_count,
                                                 int32_t *d_answer, int32_t *d_surplus, void *cuda_stream)
{
    const fluxbin_status_t st = check(batch, tokens, nodes);
    if (st != FLUXBIN_OK) return st;
    if (!d_query_start || !d_count || !d_answer || !d_surplus || (tokens > 0 && (!d_parents || !d_drafted || !d_answers || !d_path))) return FLUXBIN_ERR_NULL;
    for (const void *p : {(const void *)d_query_start, (const void *)d_parents, (const void *)d_drafted, (const void *)d_answers, (const void *)d_path,
                          (const void *)d_count, (const void *)d_answer, (const void *)d_surplus})
        if (!aligned_to(p, 4)) return FLUXBIN_ERR_ALIGNMENT;
    const AcceptArgs a = {batch, tokens, nodes, d_query_start, d_parents, d_drafted, d_answers, d_path, d_count, d_answer, d_surplus};
    FBD_CUDA(launch(accept_kernel, dim3((unsigned)batch), 32, sizeof(int) * 3 * nodes, (cudaStream_t)cuda_stream, a));
    return FLUXBIN_OK;
}
