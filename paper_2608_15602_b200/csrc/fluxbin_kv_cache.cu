// Writing the 8-bit block-paged cache (fluxbin_kv_append) and reading its values back (fluxbin_kv_read).
#include "fluxbin_cache.cuh"
#include "fluxbin_rotary.cuh"

using namespace fbd;

extern "C" fluxbin_status_t fluxbin_kv_validate(const fluxbin_kv_cache_t *cache) { return check_cache(cache); }

namespace {

struct Heads { const void *p; long long token, head; int heads; };
struct HeadsOut { void *p; long long token, head; };

constexpr int kThreads = 128;

__device__ __forceinline__ float block_max(float v, float *scratch)
{
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    return fmaxf(fmaxf(scratch[0], scratch[1]), fmaxf(scratch[2], scratch[3]));
}

// element e of a head after its turn
template <typename T>
__device__ __forceinline__ float turned(const T *x, int e, const fluxbin_rotary_t &rot, int position)
{
    if (e >= rot.rotary_dim) return to_float(x[e]);
    const int half = rot.rotary_dim / 2;
    const int i = rot.interleaved ? e >> 1 : e % half;
    const bool second = rot.interleaved ? (e & 1) : e >= half;
    float c, s, u, v;
    pair_angle(position, rot.d_turns[i], rot.magnitude, 1.f, c, s);
    turn_pair(to_float(x[rot.interleaved ? 2 * i : i]), to_float(x[rot.interleaved ? 2 * i + 1 : i + half]), c, s, u, v);
    return second ? v : u;
}

// One CTA per (token, head).  The first token of a run -- new tokens at consecutive slots of one block -- does the run.
template <typename T, int FMT, bool ROT>
__global__ void append_kernel(fluxbin_kv_cache_t c, int tokens, const int *slots, Heads k, Heads v, fluxbin_rotary_t rot,
                              const int *positions, Heads q, HeadsOut qo)
{
    __shared__ float scratch[4];
    wait_for_predecessor();
    const int t0 = blockIdx.x, h = blockIdx.y;
    if (ROT && h >= c.kv_heads) {
        // a q head: both elements of a pair are read before either is written (the output may be the input)
        const T *x = (const T *)q.p + t0 * q.token + (h - c.kv_heads) * q.head;
        T *y = (T *)qo.p + t0 * qo.token + (h - c.kv_heads) * qo.head;
        const int half = rot.rotary_dim / 2;
        for (int u = threadIdx.x; u < c.head_dim - half; u += kThreads) {
            if (u >= half) { y[u + half] = x[u + half]; continue; }
            const int e0 = rot.interleaved ? 2 * u : u, e1 = rot.interleaved ? 2 * u + 1 : u + half;
            float cs, sn, a, b;
            pair_angle(positions[t0], rot.d_turns[u], rot.magnitude, 1.f, cs, sn);
            turn_pair(to_float(x[e0]), to_float(x[e1]), cs, sn, a, b);
            y[e0] = from_float<T>(a);
            y[e1] = from_float<T>(b);
        }
        return;
    }
    const int bs = c.block_tokens, s0 = slots[t0];
    if (s0 < 0 || s0 >= c.num_blocks * bs) return;
    const int b = s0 / bs, off = s0 % bs;
    if (off > 0 && t0 > 0 && slots[t0 - 1] == s0 - 1) return;
    int run = 1;
    while (off + run < bs && t0 + run < tokens && slots[t0 + run] == s0 + run) ++run;
    const int D = c.head_dim;
    for (int side = 0; side < 2; ++side) {
        const Heads &src = side ? v : k;
        unsigned char *cells = (unsigned char *)(side ? c.d_v : c.d_k) + b * c.block_stride + h * c.head_stride;
        float *scale = (side ? c.d_v_scale : c.d_k_scale) + (long long)b * c.kv_heads + h;
        float most = 0.f;
        bool bad = false;
        for (int i = threadIdx.x; i < run * D; i += kThreads) {
            const int t = t0 + i / D, e = i % D;
            const T *x = (const T *)src.p + t * src.token + h * src.head;
            const float a = fabsf(ROT && side == 0 ? turned(x, e, rot, positions[t]) : to_float(x[e]));
            bad |= !(a < INFINITY);
            most = fmaxf(most, a);
        }
        most = block_max(bad ? INFINITY : most, scratch);
        const float before = off ? *scale : 0.f;
        const Scale s = scale_of(before, most, 1.f / Entry<FMT>::kTop);
        if (off && !(s.now == before)) {
            const float ratio = __fmul_rn(before, s.inverse);
            for (int i = threadIdx.x; i < off * D; i += kThreads) {
                unsigned char *p = cells + i / D * c.token_stride + i % D;
                *p = Entry<FMT>::store(__fmul_rn(Entry<FMT>::load(*p), ratio));
            }
        }
        for (int i = threadIdx.x; i < run * D; i += kThreads) {
            const int t = t0 + i / D, e = i % D;
            const T *x = (const T *)src.p + t * src.token + h * src.head;
            const float a = ROT && side == 0 ? turned(x, e, rot, positions[t]) : to_float(x[e]);
            cells[(off + i / D) * c.token_stride + e] = Entry<FMT>::store(__fmul_rn(a, s.inverse));
        }
        __syncthreads();                         // `before` has been read by every thread
        if (threadIdx.x == 0) *scale = s.now;
    }
}

template <typename T, int FMT>
__global__ void read_kernel(fluxbin_kv_cache_t c, const int *slots, T *k_out, T *v_out)
{
    wait_for_predecessor();
    const int t = blockIdx.x, s = slots[t], n = c.kv_heads * c.head_dim;
    const bool live = s >= 0 && s < c.num_blocks * c.block_tokens;
    const int b = live ? s / c.block_tokens : 0, off = live ? s % c.block_tokens : 0;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int h = i / c.head_dim, e = i % c.head_dim;
        const long long at = b * c.block_stride + h * c.head_stride + off * c.token_stride + e;
        const long long sc = (long long)b * c.kv_heads + h;
        if (k_out) k_out[(long long)t * n + i] = from_float<T>(live ? Entry<FMT>::load(((const unsigned char *)c.d_k)[at]) * c.d_k_scale[sc] : 0.f);
        if (v_out) v_out[(long long)t * n + i] = from_float<T>(live ? Entry<FMT>::load(((const unsigned char *)c.d_v)[at]) * c.d_v_scale[sc] : 0.f);
    }
}

template <typename T, int FMT>
cudaError_t run_append(const fluxbin_kv_cache_t &c, int tokens, const int *slots, const Heads &k, const Heads &v, const fluxbin_rotary_t *rot,
                       const int *positions, const Heads &q, const HeadsOut &qo, cudaStream_t s)
{
    if (rot)
        return launch(append_kernel<T, FMT, true>, dim3((unsigned)tokens, (unsigned)(c.kv_heads + (q.p ? q.heads : 0))), kThreads, 0, s, c, tokens,
                      slots, k, v, *rot, positions, q, qo);
    return launch(append_kernel<T, FMT, false>, dim3((unsigned)tokens, (unsigned)c.kv_heads), kThreads, 0, s, c, tokens, slots, k, v,
                  fluxbin_rotary_t{}, positions, q, qo);
}

template <typename T>
cudaError_t run_read(const fluxbin_kv_cache_t &c, int tokens, const int *slots, void *k_out, void *v_out, cudaStream_t s)
{
    if (c.format == FLUXBIN_CACHE_INT8)
        return launch(read_kernel<T, FLUXBIN_CACHE_INT8>, dim3((unsigned)tokens), kThreads, 0, s, c, slots, (T *)k_out, (T *)v_out);
    return launch(read_kernel<T, FLUXBIN_CACHE_E4M3>, dim3((unsigned)tokens), kThreads, 0, s, c, slots, (T *)k_out, (T *)v_out);
}

} // namespace

extern "C" fluxbin_status_t fluxbin_kv_append(const fluxbin_kv_cache_t *cache, int32_t dtype, int32_t tokens, const int32_t *d_slots,
                                              const void *d_k, int64_t k_token, int64_t k_head, const void *d_v, int64_t v_token, int64_t v_head,
                                              const fluxbin_rotary_t *rotary, const int32_t *d_positions,
                                              const void *d_q, int32_t q_heads, int64_t q_token, int64_t q_head,
                                              void *d_q_out, int64_t qo_token, int64_t qo_head, void *cuda_stream)
{
    fluxbin_status_t st = check_cache(cache);
    if (st != FLUXBIN_OK) return st;
    if (!type_known(dtype)) return FLUXBIN_ERR_UNSUPPORTED;
    if (tokens < 0) return FLUXBIN_ERR_RANGE;
    if (rotary) {
        st = check_rotary(rotary);
        if (st != FLUXBIN_OK) return st;
        if (rotary->head_dim != cache->head_dim) return FLUXBIN_ERR_UNSUPPORTED;
        if (d_q && q_heads < 1) return FLUXBIN_ERR_RANGE;
    } else {
        d_q = nullptr;
        d_q_out = nullptr;
    }
    if (cache->kv_heads + (d_q ? (int64_t)q_heads : 0) > 65535) return FLUXBIN_ERR_RANGE;
    if (tokens == 0) return FLUXBIN_OK;
    if (!d_slots || !d_k || !d_v || (rotary && !d_positions) || (d_q && !d_q_out)) return FLUXBIN_ERR_NULL;
    const size_t size = (size_t)type_size(dtype);
    if (!aligned_to(d_k, size) || !aligned_to(d_v, size) || !aligned_to(d_q, size) || !aligned_to(d_q ? d_q_out : nullptr, size) ||
        !aligned_to(d_slots, 4) || (rotary && !aligned_to(d_positions, 4))) return FLUXBIN_ERR_ALIGNMENT;
    const Heads k = {d_k, k_token, k_head, cache->kv_heads}, v = {d_v, v_token, v_head, cache->kv_heads}, q = {d_q, q_token, q_head, q_heads};
    const HeadsOut qo = {d_q_out, qo_token, qo_head};
    cudaStream_t s = (cudaStream_t)cuda_stream;
#define FB_APPEND(T) (cache->format == FLUXBIN_CACHE_INT8 ? run_append<T, FLUXBIN_CACHE_INT8>(*cache, tokens, d_slots, k, v, rotary, d_positions, q, qo, s) \
                                                          : run_append<T, FLUXBIN_CACHE_E4M3>(*cache, tokens, d_slots, k, v, rotary, d_positions, q, qo, s))
    if (dtype == FLUXBIN_TYPE_FP16) FBD_CUDA(FB_APPEND(__half));
    else if (dtype == FLUXBIN_TYPE_BF16) FBD_CUDA(FB_APPEND(__nv_bfloat16));
    else FBD_CUDA(FB_APPEND(float));
#undef FB_APPEND
    return FLUXBIN_OK;
}

extern "C" fluxbin_status_t fluxbin_kv_read(const fluxbin_kv_cache_t *cache, int32_t dtype, int32_t tokens, const int32_t *d_slots,
                                            void *d_k_out, void *d_v_out, void *cuda_stream)
{
    const fluxbin_status_t st = check_cache(cache);
    if (st != FLUXBIN_OK) return st;
    if (!type_known(dtype)) return FLUXBIN_ERR_UNSUPPORTED;
    if (tokens < 0) return FLUXBIN_ERR_RANGE;
    if (tokens == 0 || (!d_k_out && !d_v_out)) return FLUXBIN_OK;
    if (!d_slots) return FLUXBIN_ERR_NULL;
    if (!aligned_to(d_k_out, 16) || !aligned_to(d_v_out, 16) || !aligned_to(d_slots, 4)) return FLUXBIN_ERR_ALIGNMENT;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (dtype == FLUXBIN_TYPE_FP16) FBD_CUDA(run_read<__half>(*cache, tokens, d_slots, d_k_out, d_v_out, s));
    else if (dtype == FLUXBIN_TYPE_BF16) FBD_CUDA(run_read<__nv_bfloat16>(*cache, tokens, d_slots, d_k_out, d_v_out, s));
    else FBD_CUDA(run_read<float>(*cache, tokens, d_slots, d_k_out, d_v_out, s));
    return FLUXBIN_OK;
}
