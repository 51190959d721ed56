// Moving the entries of accepted paths to the first slots of their step's tokens (fluxbin_kv_keep).
//
// A warp for each request, key head and side.  The path ascends and no entry of it moves up, so going along it in order never
// writes an entry that is still to be read, and what is read for a block lies in that block or behind it.  A block's tokens are one
// run, or several where slots outside the cache or offsets that are left out lie between them: what a later run reads of the block
// is still under the scale that the block had when its first run began.  Entries are read for the largest magnitude, several tokens
// of each lane at once, and stored from registers, those of long runs read again.  Bound by a chain of dependent accesses
// (start, path, slots, entries).  256 requests with 40 heads of 128: 30 us (read twice, one token of a lane after the other, 31).
#include "fluxbin_cache.cuh"

using namespace fbd;

namespace {

constexpr int kWarps = 4;

struct Args {
    fluxbin_kv_cache_t c;
    int batch, tokens;
    const int *query_start, *slots, *path;
};

template <int FMT> __device__ __forceinline__ void values16(const uint4 &x, float scale, float (&v)[16])
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __fmul_rn(Entry<FMT>::load((unsigned char)(w[i / 4] >> (i % 4 * 8))), scale);
}
template <int FMT> __device__ __forceinline__ uint4 entries16(const float (&v)[16], float factor)
{
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i / 4] |= (uint32_t)Entry<FMT>::store(__fmul_rn(v[i], factor)) << (i % 4 * 8);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int FMT, int D>
__global__ void __launch_bounds__(kWarps * 32) keep_kernel(const __grid_constant__ Args a)
{
    constexpr int LANES = D / 16, AT_ONCE = 32 / LANES, DEEP = 32 / AT_ONCE < 4 ? 32 / AT_ONCE : 4;      // of a token, tokens side by side, those one after the other
    const int lane = threadIdx.x & 31, bs = a.c.block_tokens, limit = a.c.num_blocks * bs, H = a.c.kv_heads;
    const long long task = (long long)blockIdx.x * kWarps + threadIdx.x / 32;
    let_successor_start();
    wait_for_predecessor();
    if (task >= (long long)a.batch * H * 2) return;
    const int r = (int)(task / (2 * H)), h = (int)(task / 2 % H), side = (int)(task & 1);
    const int first = min(max(a.query_start[r], 0), a.tokens), n = max(min(max(a.query_start[r + 1], 0), a.tokens) - first, 0);
    const int *path = a.path + first, *slots = a.slots + first;
    unsigned char *cells = (unsigned char *)(side ? a.c.d_v : a.c.d_k) + h * a.c.head_stride;
    float *scales = (side ? a.c.d_v_scale : a.c.d_k_scale) + h;

    // ---- the tokens that move: from the first that is not where it belongs to the end of the path
    int begin = n, end = n;
    for (int i = 0; i < n; i += 32) {
        const int j = i + lane, p = j < n ? path[j] : -1, before = j > 0 && j < n ? path[j - 1] : -1;
        const unsigned over = __ballot_sync(0xffffffffu, p < j || p >= n || (j > 0 && p <= before)), moved = __ballot_sync(0xffffffffu, p != j);
        if (begin == n && moved) begin = min(i + __ffs(moved) - 1, n);
        if (over) {
            end = min(i + __ffs(over) - 1, n);
            break;
        }
    }
    const int sub = lane / LANES, e0 = lane % LANES * 16;
    const float top_inverse = 1.f / Entry<FMT>::kTop;
    int held = -1;                               // the block of the last run, and its scale before the first one there
    float held_scale = 0.f;
    for (int j = begin; j < end;) {
        const int s0 = slots[j];
        if (s0 < 0 || s0 >= limit) {
            ++j;
            continue;
        }
        // ---- a run: tokens that go to consecutive slots of one block
        const int block = s0 / bs, offset = s0 % bs;
        int run = 1;
        for (const int most = min(bs - offset, end - j); run < most;) {
            const int i = run + lane;
            const unsigned on = __ballot_sync(0xffffffffu, i < most && slots[j + min(i, most - 1)] == s0 + i);
            const int more = on == 0xffffffffu ? 32 : __ffs(~on) - 1;
            run += more;
            if (more < 32) break;
        }
        unsigned char *to = cells + block * a.c.block_stride;
        float *scale = scales + (long long)block * H;
        const float now = *scale, before = offset ? now : 0.f;
        if (block != held) {
            held = block;
            held_scale = now;
        }
        // entries of `count` tokens of the run from `first` on, a lane's 16 of every AT_ONCE-th; -1 for a source outside the cache: zeros
        uint4 x[DEEP];
        float scale_of_x[DEEP];
        auto sources = [&](int first) { return first + lane < run ? slots[path[j + first + lane]] : -1; };         // of 32 tokens, one a lane
        auto read = [&](int from, int first, int upto) {
#pragma unroll
            for (int k = 0; k < DEEP; ++k) {
                if (first + k * AT_ONCE >= upto) break;          // (the same for every lane)
                const int i = first + k * AT_ONCE + sub, f = __shfl_sync(0xffffffffu, from, i & 31);
                const bool live = i < upto && f >= 0 && f < limit;
                x[k] = live ? *reinterpret_cast<const uint4 *>(cells + f / bs * a.c.block_stride + f % bs * a.c.token_stride + e0) : make_uint4(0, 0, 0, 0);
                scale_of_x[k] = !live ? 0.f : f / bs == held ? held_scale : scales[(long long)(f / bs) * H];
            }
        };
        unsigned most = 0;
        for (int base = 0; base < run; base += 32) {
            const int from = sources(base), upto = min(run - base, 32);
            for (int i = 0; i < upto; i += DEEP * AT_ONCE) {
                read(from, i, upto);
#pragma unroll
                for (int k = 0; k < DEEP; ++k) {
                    if (i + k * AT_ONCE >= upto) break;
                    float v[16];
                    values16<FMT>(x[k], scale_of_x[k], v);
#pragma unroll
                    for (int e = 0; e < 16; ++e) most = max(most, __float_as_uint(v[e]) & 0x7fffffffu);
                }
            }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
        const Scale s = scale_of(before, __uint_as_float(most), top_inverse);
        if (offset && !(s.now == before)) {
            const float ratio = __fmul_rn(before, s.inverse);
            for (int i = sub; i < offset; i += AT_ONCE) {
                uint4 *p = reinterpret_cast<uint4 *>(to + i * a.c.token_stride + e0);
                float v[16];
                values16<FMT>(*p, 1.f, v);
                *p = entries16<FMT>(v, ratio);
            }
        }
        for (int base = 0; base < run; base += 32) {
            const int from = run > DEEP * AT_ONCE ? sources(base) : 0, upto = min(run - base, 32);
            for (int i = 0; i < upto; i += DEEP * AT_ONCE) {
                if (run > DEEP * AT_ONCE) read(from, i, upto);   // (a short run's are still held)
                __syncwarp();                    // read before anything is written there
#pragma unroll
                for (int k = 0; k < DEEP; ++k) {
                    if (i + k * AT_ONCE >= upto) break;
                    const int n = i + k * AT_ONCE + sub;
                    float v[16];
                    values16<FMT>(x[k], scale_of_x[k], v);
                    if (n < upto) *reinterpret_cast<uint4 *>(to + (offset + base + n) * a.c.token_stride + e0) = entries16<FMT>(v, s.inverse);
                }
                __syncwarp();
            }
        }
        if (lane == 0) *scale = s.now;
        __syncwarp();
        j += run;
    }
}

template <int FMT> cudaError_t run(const Args &a, cudaStream_t s)
{
    const long long tasks = (long long)a.batch * a.c.kv_heads * 2;
    const dim3 grid((unsigned)((tasks + kWarps - 1) / kWarps));
    if (a.c.head_dim == 64) return launch(keep_kernel<FMT, 64>, grid, kWarps * 32, 0, s, a);
    if (a.c.head_dim == 128) return launch(keep_kernel<FMT, 128>, grid, kWarps * 32, 0, s, a);
    return launch(keep_kernel<FMT, 256>, grid, kWarps * 32, 0, s, a);
}

} // namespace

extern "C" fluxbin_status_t fluxbin_kv_keep(const fluxbin_kv_cache_t *cache, int32_t batch, int32_t tokens, const int32_t *d_query_start,
                                            const int32_t *d_slots, const int32_t *d_path, void *cuda_stream)
{
    const fluxbin_status_t st = check_cache(cache);
    if (st != FLUXBIN_OK) return st;
    if (batch < 1 || tokens < 0 || (int64_t)batch * cache->kv_heads * 2 / kWarps >= INT32_MAX) return FLUXBIN_ERR_RANGE;
    if (tokens == 0) return FLUXBIN_OK;
    if (!d_query_start || !d_slots || !d_path) return FLUXBIN_ERR_NULL;
    if (!aligned_to(d_query_start, 4) || !aligned_to(d_slots, 4) || !aligned_to(d_path, 4)) return FLUXBIN_ERR_ALIGNMENT;
    const Args a = {*cache, batch, tokens, d_query_start, d_slots, d_path};
    FBD_CUDA(cache->format == FLUXBIN_CACHE_INT8 ? run<FLUXBIN_CACHE_INT8>(a, (cudaStream_t)cuda_stream) : run<FLUXBIN_CACHE_E4M3>(a, (cudaStream_t)cuda_stream));
    return FLUXBIN_OK;
}
