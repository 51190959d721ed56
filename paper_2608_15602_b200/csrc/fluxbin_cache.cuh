// The 8-bit cache as the kernels see it, shared by append, read and attention.
#ifndef FLUXBIN_CACHE_CUH
#define FLUXBIN_CACHE_CUH

#include "fluxbin_device.cuh"

#include <cuda_fp8.h>

namespace fbd {

inline fluxbin_status_t check_cache(const fluxbin_kv_cache_t *c)
{
    if (!c || !c->d_k || !c->d_v || !c->d_k_scale || !c->d_v_scale) return FLUXBIN_ERR_NULL;
    if (c->num_blocks < 1 || c->kv_heads < 1 || c->block_tokens < 1 || c->head_dim < 1) return FLUXBIN_ERR_RANGE;
    if (c->format != FLUXBIN_CACHE_INT8 && c->format != FLUXBIN_CACHE_E4M3) return FLUXBIN_ERR_UNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return FLUXBIN_ERR_UNSUPPORTED;
    if (c->block_tokens % 16 != 0 || c->block_tokens > 1024) return FLUXBIN_ERR_UNSUPPORTED;
    if ((int64_t)c->num_blocks * c->block_tokens > INT32_MAX) return FLUXBIN_ERR_RANGE;
    if (!aligned_to(c->d_k, 16) || !aligned_to(c->d_v, 16) || !aligned_to(c->d_k_scale, 4) || !aligned_to(c->d_v_scale, 4)) return FLUXBIN_ERR_ALIGNMENT;
    // (the stride of an axis of one is never used)
    if ((c->num_blocks > 1 && c->block_stride % 16) || (c->kv_heads > 1 && c->head_stride % 16) || c->token_stride % 16) return FLUXBIN_ERR_ALIGNMENT;
    // entries do not overlap: sorted by size, each stride covers what the smaller ones span
    int64_t s[3] = {c->block_stride, c->head_stride, c->token_stride}, n[3] = {c->num_blocks, c->kv_heads, c->block_tokens};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (s[j] > s[j + 1]) { int64_t t = s[j]; s[j] = s[j + 1]; s[j + 1] = t; t = n[j]; n[j] = n[j + 1]; n[j + 1] = t; }
    int64_t span = c->head_dim;
    for (int i = 0; i < 3; ++i) {
        if (n[i] == 1) continue;
        if (s[i] < span || s[i] > (int64_t)1 << 44) return FLUXBIN_ERR_RANGE;
        span = s[i] * (n[i] - 1) + span;
    }
    return FLUXBIN_OK;
}

template <int FMT> struct Entry;
template <> struct Entry<FLUXBIN_CACHE_INT8> {
    static constexpr float kTop = 127.f;
    static __device__ __forceinline__ unsigned char store(float v) { return (unsigned char)(signed char)__float2int_rn(fminf(fmaxf(v, -127.f), 127.f)); }
    static __device__ __forceinline__ float load(unsigned char b) { return (float)(signed char)b; }
};
template <> struct Entry<FLUXBIN_CACHE_E4M3> {
    static constexpr float kTop = 448.f;
    static __device__ __forceinline__ unsigned char store(float v) { return __nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }
    static __device__ __forceinline__ float load(unsigned char b) { return __half2float(__half(__nv_cvt_fp8_to_halfraw(b, __NV_E4M3))); }
};

// The scale of a block after new entries of largest magnitude `most` came in (a NaN or infinity among them: NaN), and
// the factor that turns values into entries.  `top_inverse` is 1 / kTop rounded to fp32.
struct Scale { float now, inverse; };
__device__ __forceinline__ Scale scale_of(float before, float most, float top_inverse)
{
    float need = __fmul_rn(most, top_inverse);
    if (!(need < INFINITY)) need = NAN;
    Scale s;
    s.now = (need > before || need != need) ? need : before;       // a NaN already there stays
    if (s.now < 7.888609052210118e-31f) s.now = 0.f;               // 2^-100: the reciprocal stays finite
    s.inverse = s.now > 0.f ? __frcp_rn(s.now) : 0.f;
    return s;
}

} // namespace fbd

#endif
