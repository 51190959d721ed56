// Rotary positions: fluxbin_rotary_frequencies (host) and fluxbin_rotary.
#include "fluxbin_rotary.cuh"

#include <cmath>

using namespace fbd;

extern "C" fluxbin_status_t fluxbin_rotary_frequencies(int32_t rotary_dim, double base, int32_t kind, double factor, double original,
                                                       double a, double b, uint64_t *h_turns, float *h_magnitude)
{
    if (!h_turns || !h_magnitude) return FLUXBIN_ERR_NULL;
    if (rotary_dim < 2 || rotary_dim > 512 || (rotary_dim & 1) || !(base > 1.0) || !std::isfinite(base)) return FLUXBIN_ERR_RANGE;
    if (kind < FLUXBIN_ROPE_NONE || kind > FLUXBIN_ROPE_BANDS) return FLUXBIN_ERR_UNSUPPORTED;
    if (kind != FLUXBIN_ROPE_NONE && !(factor >= 1.0 && std::isfinite(factor))) return FLUXBIN_ERR_RANGE;
    if (kind == FLUXBIN_ROPE_BASE && rotary_dim == 2) return FLUXBIN_ERR_RANGE;
    if (kind == FLUXBIN_ROPE_RAMP || kind == FLUXBIN_ROPE_BANDS) {
        if (!(original >= 1.0 && std::isfinite(original) && std::isfinite(a) && std::isfinite(b))) return FLUXBIN_ERR_RANGE;
        if (kind == FLUXBIN_ROPE_RAMP ? !(b > 0.0 && a > b) : !(a > 0.0 && b > a)) return FLUXBIN_ERR_RANGE;
    }
    const double two_pi = 6.283185307179586476925286766559;
    const int d = rotary_dim, half = d / 2;
    if (kind == FLUXBIN_ROPE_BASE) base *= std::pow(factor, (double)d / (d - 2));
    double lo = 0.0, hi = 0.0;
    if (kind == FLUXBIN_ROPE_RAMP) {
        // the (fractional) pair that turns t times in `original` positions: base^(-2 i / d) * original = 2 pi t
        const double ia = d * std::log(original / (a * two_pi)) / (2.0 * std::log(base));
        const double ib = d * std::log(original / (b * two_pi)) / (2.0 * std::log(base));
        lo = std::fmax(0.0, std::floor(ia));
        hi = std::fmin(d - 1.0, std::ceil(ib));
    }
    for (int i = 0; i < half; ++i) {
        double f = std::pow(base, -2.0 * i / d);
        if (kind == FLUXBIN_ROPE_LINEAR) f /= factor;
        if (kind == FLUXBIN_ROPE_RAMP) {
            const double slow = std::fmin(1.0, std::fmax(0.0, (i - lo) / std::fmax(hi - lo, 1e-3)));
            f = f / factor * slow + f * (1.0 - slow);
        }
        if (kind == FLUXBIN_ROPE_BANDS) {
            const double turns = original * f / two_pi;
            const double keep = std::fmin(1.0, std::fmax(0.0, (turns - a) / (b - a)));
            f = f * keep + f / factor * (1.0 - keep);
        }
        h_turns[i] = (uint64_t)std::llround(f / two_pi * 9223372036854775808.0) << 1;     // f <= 1: below 2^62
    }
    *h_magnitude = kind == FLUXBIN_ROPE_RAMP ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
    return FLUXBIN_OK;
}

namespace {

struct Side {
    const void *in;
    void *out;
    int heads;
    long long in_token, in_head, out_token, out_head;
};

// one thread per element pair (or per element past the turned part)
template <typename T>
__global__ void rotary_kernel(fluxbin_rotary_t rot, int inverse, int tokens, const int *positions, Side q, Side k)
{
    wait_for_predecessor();
    const int half = rot.rotary_dim / 2, units = rot.head_dim - half;
    const long long n = (long long)tokens * (q.heads + k.heads) * units;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
        const int u = (int)(i % units);
        int h = (int)(i / units % (q.heads + k.heads));
        const long long t = i / units / (q.heads + k.heads);
        const Side &S = h < q.heads ? q : k;
        if (h >= q.heads) h -= q.heads;
        const T *x = (const T *)S.in + t * S.in_token + h * S.in_head;
        T *y = (T *)S.out + t * S.out_token + h * S.out_head;
        if (u >= half) { y[u + half] = x[u + half]; continue; }
        float c, s, a, b;
        pair_angle(positions[t], rot.d_turns[u], rot.magnitude, inverse ? -1.f : 1.f, c, s);
        const int e0 = rot.interleaved ? 2 * u : u, e1 = rot.interleaved ? 2 * u + 1 : u + half;
        turn_pair(to_float(x[e0]), to_float(x[e1]), c, s, a, b);
        y[e0] = from_float<T>(a);
        y[e1] = from_float<T>(b);
    }
}

template <typename T>
cudaError_t run(const fluxbin_rotary_t &rot, int inverse, int tokens, const int *positions, const Side &q, const Side &k, cudaStream_t s)
{
    const long long n = (long long)tokens * (q.heads + k.heads) * (rot.head_dim - rot.rotary_dim / 2);
    const long long grid = (n + 255) / 256;
    return launch(rotary_kernel<T>, dim3((unsigned)(grid < 65536 ? grid : 65536)), 256, 0, s, rot, inverse, tokens, positions, q, k);
}

} // namespace

extern "C" fluxbin_status_t fluxbin_rotary(const fluxbin_rotary_t *rotary, int32_t dtype, int32_t inverse, int32_t tokens,
                                           const int32_t *d_positions, const void *d_q, int32_t q_heads, int64_t q_token, int64_t q_head,
                                           void *d_q_out, int64_t qo_token, int64_t qo_head, const void *d_k, int32_t k_heads,
                                           int64_t k_token, int64_t k_head, void *d_k_out, int64_t ko_token, int64_t ko_head,
                                           void *cuda_stream)
{
    const fluxbin_status_t st = check_rotary(rotary);
    if (st != FLUXBIN_OK) return st;
    if (!type_known(dtype)) return FLUXBIN_ERR_UNSUPPORTED;
    if (tokens < 0 || q_heads < 1 || (d_k && k_heads < 1)) return FLUXBIN_ERR_RANGE;
    if (tokens == 0) return FLUXBIN_OK;
    if (!d_positions || !d_q || !d_q_out || (d_k && !d_k_out)) return FLUXBIN_ERR_NULL;
    const size_t size = (size_t)type_size(dtype);
    if (!aligned_to(d_q, size) || !aligned_to(d_q_out, size) || !aligned_to(d_k, size) || !aligned_to(d_k ? d_k_out : nullptr, size) ||
        !aligned_to(d_positions, 4)) return FLUXBIN_ERR_ALIGNMENT;
    const Side q = {d_q, d_q_out, q_heads, q_token, q_head, qo_token, qo_head};
    const Side k = {d_k, d_k_out, d_k ? k_heads : 0, k_token, k_head, ko_token, ko_head};
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (dtype == FLUXBIN_TYPE_FP16) FBD_CUDA(run<__half>(*rotary, inverse, tokens, d_positions, q, k, s));
    else if (dtype == FLUXBIN_TYPE_BF16) FBD_CUDA(run<__nv_bfloat16>(*rotary, inverse, tokens, d_positions, q, k, s));
    else FBD_CUDA(run<float>(*rotary, inverse, tokens, d_positions, q, k, s));
    return FLUXBIN_OK;
}
