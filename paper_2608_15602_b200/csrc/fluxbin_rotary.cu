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

constexpr int kThreads = 256;
constexpr int kPrompt = 148;                     // tokens that go to the prompt kernel: one for each SM
constexpr int kCtas = 148 * 4;                   // of a prompt: those that are resident at once

// Few tokens, or accesses of single elements: a CTA takes a token, or a group of its heads.  Bound by its launch and two
// dependent accesses.
template <typename T, int VE, bool INTER>
__global__ void __launch_bounds__(kThreads, 3) rotary_kernel(const __grid_constant__ fluxbin_rotary_t rot, float sign, const int *positions,
                                                             const __grid_constant__ Side q, const __grid_constant__ Side k, int heads_each)
{
    __shared__ float2 angles[kMaxPairs];
    let_successor_start();
    wait_for_predecessor();
    const int t = blockIdx.x, h0 = blockIdx.y * heads_each, h1 = min(h0 + heads_each, q.heads + k.heads);
    turn_heads<T, VE, INTER>(rot, angles, q, k, t, h0, h1, threadIdx.x, kThreads, [&]() {
        token_angles(rot, positions[t], sign, angles, threadIdx.x, kThreads);
        __syncthreads();
    });
}

// Prompts, 16-byte accesses: the CTAs that are resident go over the tokens, all heads of a token at a time, so that what a
// thread works out about its place is worked out once.  The angles of a token are formed while its first heads are on
// their way.  Bound by memory and, nearly as much, by instructions (two conversions, two products and two sums a pair).
// 8191 tokens of 80 heads, half of each turned: 57 us (5.9 TB/s); three CTAs on an SM 62, a CTA a token that works its place
// out again 71 to 78.  Whole heads in halves (two accesses each): one head under way at a time 65 us for 9216 tokens of 72
// heads, two 67.
template <typename T, int VE, bool INTER>
__global__ void __launch_bounds__(kThreads, 4) rotary_prompt_kernel(const __grid_constant__ fluxbin_rotary_t rot, float sign, int tokens, const int *positions,
                                                                    const __grid_constant__ Side q, const __grid_constant__ Side k)
{
    constexpr int NA = INTER ? VE / 2 : VE, BATCH = INTER ? 4 : 1;
    __shared__ float2 angles[2][kMaxPairs];
    let_successor_start();
    wait_for_predecessor();
    const int half = rot.rotary_dim / 2, turning = half / NA, units = turning + (rot.head_dim - rot.rotary_dim) / VE, rows = kThreads / units;
    const int u = threadIdx.x % units, row = threadIdx.x / units, e0 = u < turning ? u * (INTER ? VE : NA) : rot.rotary_dim + (u - turning) * VE;
    const bool turns = u < turning;
    Elements<T, VE> a[BATCH], b[BATCH];
    float c[NA], s[NA];
    // `left` heads, one in every `rows`, from x to y; the first of them may be loaded already
    auto heads = [&](const T *x, T *y, long long xs, long long ys, int left, bool copies, bool loaded) {
        for (; left > 0; left -= BATCH) {
            if (!loaded) {
#pragma unroll
                for (int j = 0; j < BATCH; ++j)
                    if (j < left) {
                        a[j].load(x + j * xs, VE);
                        if (!INTER && turns) b[j].load(x + j * xs + half, VE);
                    }
            }
            loaded = false;
            x += BATCH * xs;
#pragma unroll
            for (int j = 0; j < BATCH; ++j, y += ys) {
                if (j >= left) break;
                if (!turns) {
                    if (copies) a[j].store(y, VE);
                    continue;
                }
                float f[NA], g[NA];
#pragma unroll
                for (int i = 0; i < NA; ++i)
                    turn_pair(to_float(a[j].e[INTER ? 2 * i : i]), to_float(INTER ? a[j].e[INTER ? 2 * i + 1 : 0] : b[j].e[i]), c[i], s[i], f[i], g[i]);
                if constexpr (INTER) {
#pragma unroll
                    for (int i = 0; i < NA; ++i) a[j].set(2 * i, f[i], g[i]);
                } else {
#pragma unroll
                    for (int i = 0; i < NA; i += 2) {
                        a[j].set(i, f[i], f[i + 1]);
                        b[j].set(i, g[i], g[i + 1]);
                    }
                    b[j].store(y + half, VE);
                }
                a[j].store(y, VE);
            }
        }
    };
    const int nq = row < rows && row < q.heads ? (q.heads - row + rows - 1) / rows : 0, nk = row < rows && row < k.heads ? (k.heads - row + rows - 1) / rows : 0;
    const bool q_copies = q.in != q.out, k_copies = k.in != k.out;
    const long long qs = rows * q.in_head, qos = rows * q.out_head, ks = rows * k.in_head, kos = rows * k.out_head;
    const T *xq = (const T *)q.in + blockIdx.x * q.in_token + row * q.in_head + e0, *xk = (const T *)k.in + blockIdx.x * k.in_token + row * k.in_head + e0;
    T *yq = (T *)q.out + blockIdx.x * q.out_token + row * q.out_head + e0, *yk = (T *)k.out + blockIdx.x * k.out_token + row * k.out_head + e0;
    int position = positions[blockIdx.x], buffer = 0;
    // two sets of angles: a thread may form those of the next token while another still reads these, but not those of the
    // one after that, which it does behind the next token's barrier
    for (int t = blockIdx.x; t < tokens; t += gridDim.x, buffer ^= 1) {
        const int next = t + (int)gridDim.x < tokens ? positions[t + gridDim.x] : 0;
#pragma unroll
        for (int j = 0; j < BATCH; ++j)
            if (j < nq) {
                a[j].load(xq + j * qs, VE);
                if (!INTER && turns) b[j].load(xq + j * qs + half, VE);
            }
        token_angles(rot, position, sign, angles[buffer], threadIdx.x, kThreads);
        __syncthreads();
        position = next;
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const float2 x = turns ? angles[buffer][u * NA + i] : make_float2(1.f, 0.f);
            c[i] = x.x;
            s[i] = x.y;
        }
        heads(xq, yq, qs, qos, nq, q_copies, true);
        heads(xk, yk, ks, kos, nk, k_copies, false);
        xq += gridDim.x * q.in_token;
        yq += gridDim.x * q.out_token;
        xk += gridDim.x * k.in_token;
        yk += gridDim.x * k.out_token;
    }
}

template <typename T, int VE, bool INTER>
cudaError_t run_as(const fluxbin_rotary_t &rot, int inverse, int tokens, const int *positions, const Side &q, const Side &k, cudaStream_t s)
{
    const int heads = q.heads + k.heads;
    const float sign = inverse ? -1.f : 1.f;
    if constexpr (VE * sizeof(T) == 16) {
        // (64 + 8 heads of 128: 300 tokens 6.2 us against 7.2 with split heads, 600 8.3 both, 1500 16.4 against 19.6)
        if (tokens >= kPrompt) return launch(rotary_prompt_kernel<T, VE, INTER>, dim3((unsigned)(tokens < kCtas ? tokens : kCtas)), kThreads, 0, s, rot, sign, tokens, positions, q, k);
    }
    int each = heads;
    if (tokens < kFewTokens) {
        const int units = rot.rotary_dim / 2 / (INTER ? VE / 2 : VE) + (rot.head_dim - rot.rotary_dim + VE - 1) / VE;
        const int at_once = kThreads / units > 0 ? kThreads / units : 1, groups = (kFewTokens + tokens - 1) / tokens;
        each = (heads + groups - 1) / groups;
        if (each < at_once) each = at_once;
        if (each > heads) each = heads;
    }
    return launch(rotary_kernel<T, VE, INTER>, dim3((unsigned)tokens, (unsigned)((heads + each - 1) / each)), kThreads, 0, s, rot, sign, positions, q, k, each);
}
template <typename T>
cudaError_t run(const fluxbin_rotary_t &rot, int dtype, int inverse, int tokens, const int *positions, const Side &q, const Side &k, cudaStream_t s)
{
    constexpr int WIDE = 16 / sizeof(T);
    if (wide_heads(rot, dtype, q) && wide_heads(rot, dtype, k))
        return rot.interleaved ? run_as<T, WIDE, true>(rot, inverse, tokens, positions, q, k, s) : run_as<T, WIDE, false>(rot, inverse, tokens, positions, q, k, s);
    return rot.interleaved ? run_as<T, 2, true>(rot, inverse, tokens, positions, q, k, s) : run_as<T, 1, false>(rot, inverse, tokens, positions, q, k, s);
}

} // namespace

cudaError_t fbd::launch_rotary(const fluxbin_rotary_t &rot, int dtype, int inverse, int tokens, const int *positions, const Side &q, const Side &k,
                               cudaStream_t s)
{
    if (dtype == FLUXBIN_TYPE_FP16) return run<__half>(rot, dtype, inverse, tokens, positions, q, k, s);
    if (dtype == FLUXBIN_TYPE_BF16) return run<__nv_bfloat16>(rot, dtype, inverse, tokens, positions, q, k, s);
    return run<float>(rot, dtype, inverse, tokens, positions, q, k, s);
}

extern "C" fluxbin_status_t fluxbin_rotary(const fluxbin_rotary_t *rotary, int32_t dtype, int32_t inverse, int32_t tokens,
                                           const int32_t *d_positions, const void *d_q, int32_t q_heads, int64_t q_token, int64_t q_head,
                                           void *d_q_out, int64_t qo_token, int64_t qo_head, const void *d_k, int32_t k_heads,
                                           int64_t k_token, int64_t k_head, void *d_k_out, int64_t ko_token, int64_t ko_head,
                                           void *cuda_stream)
{
    const fluxbin_status_t st = check_rotary(rotary);
    if (st != FLUXBIN_OK) return st;
    if (!type_known(dtype)) return FLUXBIN_ERR_UNSUPPORTED;
    if (tokens < 0 || q_heads < 1 || q_heads > 65535 || (d_k && (k_heads < 1 || k_heads > 65535))) return FLUXBIN_ERR_RANGE;
    if (tokens == 0) return FLUXBIN_OK;
    if (!d_positions || !d_q || !d_q_out || (d_k && !d_k_out)) return FLUXBIN_ERR_NULL;
    const size_t size = (size_t)type_size(dtype);
    if (!aligned_to(d_q, size) || !aligned_to(d_q_out, size) || !aligned_to(d_k, size) || !aligned_to(d_k ? d_k_out : nullptr, size) ||
        !aligned_to(d_positions, 4)) return FLUXBIN_ERR_ALIGNMENT;
    if (!heads_apart(tokens, q_heads, qo_token, qo_head, rotary->head_dim) || (d_k && !heads_apart(tokens, k_heads, ko_token, ko_head, rotary->head_dim)))
        return FLUXBIN_ERR_RANGE;
    const Side q = {d_q, d_q_out, q_heads, q_token, q_head, qo_token, qo_head};
    const Side k = {d_k, d_k_out, d_k ? k_heads : 0, k_token, k_head, ko_token, ko_head};
    FBD_CUDA(launch_rotary(*rotary, dtype, inverse, tokens, d_positions, q, k, (cudaStream_t)cuda_stream));
    return FLUXBIN_OK;
}
