// Writing the 8-bit block-paged cache (fluxbin_kv_append) and reading its values back (fluxbin_kv_read).
#include "fluxbin_cache.cuh"
#include "fluxbin_rotary.cuh"

using namespace fbd;

extern "C" fluxbin_status_t fluxbin_kv_validate(const fluxbin_kv_cache_t *cache) { return check_cache(cache); }

namespace {

struct Heads { const void *p; long long token, head; int heads; };
struct HeadsOut { void *p; long long token, head; };

constexpr int kThreads = 128;
constexpr int kMaxTokens = 1 << 24;              // of a call: the grids stay within 31 bits

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

// Any strides, alignment and rotary dimension: one CTA per (token, head), element by element.  The first token of a run --
// new tokens at consecutive slots of one block -- does the run.
template <typename T, int FMT, bool ROT>
__global__ void append_any_kernel(fluxbin_kv_cache_t c, int tokens, const int *slots, Heads k, Heads v, fluxbin_rotary_t rot,
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

// ---- 16-byte accesses ------------------------------------------------------------------------------------
//
// A run of new tokens in a block and a head share one scale, so their largest magnitude has to be known before the first
// is stored; both halves of the work read the values once, into registers.
//   short runs (a decode step: one token a run): a warp per head, half its lanes the keys, half the values;
//   long runs (a prompt: whole blocks): the CTA on one head at a time, four pieces of eight elements a thread and pass.
//   Bound by latency, not by bytes: three CTAs on an SM (80 registers) 43 us for 9 K tokens of 8 heads, two 53, one that has
//   the next head's loads under way (204 registers) 72.
// Keys are turned in fp32 on the way; the angles of a run's tokens are formed once for all heads of the CTA.  The q heads of
// the same tokens are turned by CTAs of the same launch.

constexpr int kWide = 256, kWarpsWide = kWide / 32;
constexpr int kShortRun = 4;

template <typename T> struct Eight {
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        __align__(16) T e[8];
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(e)[i] = w[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_float(e[i]);
    }
};

// elements e0 .. e0 + 7 of a head after its turn; `angles` are those of its token
template <typename T>
__device__ __forceinline__ void turned8(const T *x, int e0, const fluxbin_rotary_t &rot, const float2 *angles, float (&v)[8])
{
    Eight<T> own;
    own.load(x + e0);
    own.get(v);
    if (e0 >= rot.rotary_dim) return;
    if (rot.interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 a = angles[e0 / 2 + i];
            float f, g;
            turn_pair(v[2 * i], v[2 * i + 1], a.x, a.y, f, g);
            v[2 * i] = f;
            v[2 * i + 1] = g;
        }
        return;
    }
    const int half = rot.rotary_dim / 2;
    const bool second = e0 >= half;
    float w[8];
    Eight<T> other;
    other.load(x + (second ? e0 - half : e0 + half));
    other.get(w);
    const float4 *pair = reinterpret_cast<const float4 *>(angles + (second ? e0 - half : e0));
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const float4 a = pair[i / 2];
        // (turn_second(other, own) and turn_first(own, other) differ in the sign of the other's product alone)
        v[i] = fmaf(v[i], a.x, __fmul_rn(w[i], second ? a.y : -a.y));
        v[i + 1] = fmaf(v[i + 1], a.z, __fmul_rn(w[i + 1], second ? a.w : -a.w));
    }
}

// the largest |v| as its bits, which order like the magnitudes; infinities and NaN lie above all others
__device__ __forceinline__ unsigned largest8(unsigned most, const float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(v[i]) & 0x7fffffffu);
    return most;
}
// eight entries; |v * inverse| exceeds the format's largest value by rounding at most
template <int FMT> __device__ __forceinline__ uint2 entries8(const float (&v)[8], float inverse)
{
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (FMT == FLUXBIN_CACHE_INT8) {
            // added to 1.5 * 2^23 a value is rounded to a whole number, to nearest even, in the low bits
            uint32_t e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = __float_as_uint(__fadd_rn(__fmul_rn(v[4 * i + j], inverse), 12582912.f));
            w[i] = __byte_perm(__byte_perm(e[0], e[1], 0x0040), __byte_perm(e[2], e[3], 0x0040), 0x5410);
        } else {
            const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(__fmul_rn(v[4 * i], inverse), __fmul_rn(v[4 * i + 1], inverse)), __NV_SATFINITE, __NV_E4M3);
            const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(__fmul_rn(v[4 * i + 2], inverse), __fmul_rn(v[4 * i + 3], inverse)), __NV_SATFINITE, __NV_E4M3);
            w[i] = lo | hi << 16;
        }
    }
    return make_uint2(w[0], w[1]);
}
template <int FMT> __device__ __forceinline__ void requantise8(unsigned char *p, float ratio)
{
    const uint2 w = *reinterpret_cast<const uint2 *>(p);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = Entry<FMT>::load((unsigned char)((i < 4 ? w.x : w.y) >> (i % 4 * 8)));
    *reinterpret_cast<uint2 *>(p) = entries8<FMT>(v, ratio);
}

struct Run { int first, count, block, offset; };

struct AppendArgs {
    fluxbin_kv_cache_t c;
    int tokens;
    const int *slots;
    Heads k, v;
    fluxbin_rotary_t rot;
    const int *positions;
    Side q;
    int tokens_each, heads_each, groups;         // tokens a CTA looks for runs in, heads it does, groups of heads
    int append_ctas, q_heads_each, q_groups;
};

template <typename T, int FMT, int D, bool ROT>
__global__ void __launch_bounds__(kWide, D == 256 ? 2 : 3) append_kernel(const __grid_constant__ AppendArgs a)
{
    constexpr int PIECES = D / 8;                // of eight elements
    constexpr int AT_ONCE = kWide / PIECES;      // tokens a pass has side by side
    constexpr int DEEP = 4, PASS = AT_ONCE * DEEP;
    extern __shared__ __align__(16) float2 angles[];           // [PASS][pairs], or [kMaxPairs] for the q heads
    __shared__ unsigned part[2][kWarpsWide];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    let_successor_start();
    wait_for_predecessor();

    if (ROT && (int)blockIdx.x >= a.append_ctas) {
        const int i = blockIdx.x - a.append_ctas, t = i / a.q_groups, h0 = i % a.q_groups * a.q_heads_each;
        const Side none = {};
        const int h1 = min(h0 + a.q_heads_each, a.q.heads);
        auto form = [&]() {
            token_angles(a.rot, a.positions[t], 1.f, angles, tid, kWide);
            __syncthreads();
        };
        if (a.rot.interleaved) turn_heads<T, 16 / sizeof(T), true>(a.rot, angles, a.q, none, t, h0, h1, tid, kWide, form);
        else turn_heads<T, 16 / sizeof(T), false>(a.rot, angles, a.q, none, t, h0, h1, tid, kWide, form);
        return;
    }

    const int bs = a.c.block_tokens, limit = a.c.num_blocks * bs, H = a.c.kv_heads;
    const int h0 = blockIdx.x % a.groups * a.heads_each, h1 = min(h0 + a.heads_each, H);
    const int t_begin = blockIdx.x / a.groups * a.tokens_each, t_end = min(t_begin + a.tokens_each, a.tokens);
    const int pairs = ROT ? a.rot.rotary_dim / 2 : 0;
    const float top_inverse = 1.f / Entry<FMT>::kTop;

    // ---- the runs that begin in this CTA's tokens: lane i looks at token i
    unsigned short_runs, long_runs;
    int my_count = 0, my_slot = -1;
    {
        const int t = t_begin + lane;
        if (t < t_end) {
            const int s = a.slots[t];
            const bool first = s >= 0 && s < limit && !(s % bs > 0 && t > 0 && a.slots[t - 1] == s - 1);
            if (first) {
                const int most = min(bs - s % bs, a.tokens - t);
                my_slot = s;
                my_count = 1;
                while (my_count < most && my_count <= kShortRun && a.slots[t + my_count] == s + my_count) ++my_count;
            }
        }
        short_runs = __ballot_sync(0xffffffffu, my_count > 0 && my_count <= kShortRun);
        long_runs = __ballot_sync(0xffffffffu, my_count > kShortRun);
    }
    if ((short_runs | long_runs) == 0) return;

    if (short_runs) {
        // ---- a warp per run and head: lanes of the lower half the keys, of the upper half the values
        if constexpr (ROT) {
            // (the angles of every token up to the last one of the last short run)
            const int n = min(t_end - t_begin + kShortRun - 1, a.tokens - t_begin);
            for (int i = tid; i < n * pairs; i += kWide) {
                float2 x;
                pair_angle(a.positions[t_begin + i / pairs], a.rot.d_turns[i % pairs], a.rot.magnitude, 1.f, x.x, x.y);
                angles[i] = x;
            }
            __syncthreads();
        }
        constexpr int LANES = PIECES < 16 ? PIECES : 16;                             // lanes of a side
        constexpr int EACH = PIECES / LANES;                                         // pieces of a lane
        const int side = lane >> 4, sl = lane & 15, tasks = __popc(short_runs) * (h1 - h0);
        for (int task = warp; task < tasks; task += kWarpsWide) {
            const int h = h0 + task % (h1 - h0), at_lane = __fns(short_runs, 0, task / (h1 - h0) + 1);
            const int t0 = t_begin + at_lane, count = __shfl_sync(0xffffffffu, my_count, at_lane), s0 = __shfl_sync(0xffffffffu, my_slot, at_lane);
            const int block = s0 / bs, offset = s0 % bs;
            const Heads &src = side ? a.v : a.k;
            float *scale = (side ? a.c.d_v_scale : a.c.d_k_scale) + (long long)block * H + h;
            const float before = offset ? *scale : 0.f;
            float v[kShortRun][EACH][8];
            unsigned most = 0;
#pragma unroll
            for (int i = 0; i < kShortRun; ++i)
#pragma unroll
                for (int j = 0; j < EACH; ++j) {
                    if (i >= count || sl >= LANES) continue;
                    const T *x = (const T *)src.p + (long long)(t0 + i) * src.token + h * src.head;
                    const int e0 = (j * LANES + sl) * 8;
                    if (ROT && side == 0) turned8<T>(x, e0, a.rot, angles + (at_lane + i) * pairs, v[i][j]);
                    else {
                        Eight<T> w;
                        w.load(x + e0);
                        w.get(v[i][j]);
                    }
                    most = largest8(most, v[i][j]);
                }
#pragma unroll
            for (int o = 8; o; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));        // of this half
            const Scale s = scale_of(before, __uint_as_float(most), top_inverse);
            unsigned char *cells = (unsigned char *)(side ? a.c.d_v : a.c.d_k) + block * a.c.block_stride + h * a.c.head_stride;
            if (offset && !(s.now == before) && sl < LANES) {
                const float ratio = __fmul_rn(before, s.inverse);
                for (int i = 0; i < offset; ++i)
#pragma unroll
                    for (int j = 0; j < EACH; ++j) requantise8<FMT>(cells + i * a.c.token_stride + (j * LANES + sl) * 8, ratio);
            }
#pragma unroll
            for (int i = 0; i < kShortRun; ++i)
#pragma unroll
                for (int j = 0; j < EACH; ++j)
                    if (i < count && sl < LANES)
                        *reinterpret_cast<uint2 *>(cells + (offset + i) * a.c.token_stride + (j * LANES + sl) * 8) = entries8<FMT>(v[i][j], s.inverse);
            __syncwarp();
            if (sl == 0) *scale = s.now;
        }
        if (ROT) __syncthreads();                                                    // the angles are free again
    }

    for (; long_runs; long_runs &= long_runs - 1) {
        const int at_lane = __ffs(long_runs) - 1, t0 = t_begin + at_lane, s0 = __shfl_sync(0xffffffffu, my_slot, at_lane);
        Run r = {t0, kShortRun + 1, s0 / bs, s0 % bs};
        // its length: all lanes look at once, 32 tokens at a time
        for (int most = min(bs - r.offset, a.tokens - t0); r.count < most;) {
            const int i = r.count + lane;
            const unsigned on = __ballot_sync(0xffffffffu, i < most && a.slots[min(t0 + i, a.tokens - 1)] == s0 + i);
            const int n = on == 0xffffffffu ? 32 : __ffs(~on) - 1;
            r.count += n;
            if (n < 32) break;
        }

        // ---- the CTA on one head at a time
        const int e0 = tid % PIECES * 8, sub = tid / PIECES;
        const bool one_pass = r.count <= PASS;
        auto pass_angles = [&](int base) {
            if constexpr (ROT) {
                const int n = min(PASS, r.count - base) * pairs;
                __syncthreads();
                for (int i = tid; i < n; i += kWide) {
                    float2 x;
                    pair_angle(a.positions[t0 + base + i / pairs], a.rot.d_turns[i % pairs], a.rot.magnitude, 1.f, x.x, x.y);
                    angles[i] = x;
                }
                __syncthreads();
            }
        };
        if (one_pass) pass_angles(0);
        for (int h = h0; h < h1; ++h) {
            float kv[DEEP][8];
            unsigned most[2] = {0, 0};
            Eight<T> vv[DEEP];
            auto load = [&](int base) {
#pragma unroll
                for (int j = 0; j < DEEP; ++j) {
                    const int i = base + sub + j * AT_ONCE;
                    if (i < r.count) vv[j].load((const T *)a.v.p + (long long)(t0 + i) * a.v.token + h * a.v.head + e0);
                }
#pragma unroll
                for (int j = 0; j < DEEP; ++j) {
                    const int i = base + sub + j * AT_ONCE;
                    if (i >= r.count) continue;
                    const T *x = (const T *)a.k.p + (long long)(t0 + i) * a.k.token + h * a.k.head;
                    if (ROT) turned8<T>(x, e0, a.rot, angles + (i - base) * pairs, kv[j]);
                    else {
                        Eight<T> w;
                        w.load(x + e0);
                        w.get(kv[j]);
                    }
                }
            };
            for (int base = 0; base < r.count; base += PASS) {
                if (!one_pass) pass_angles(base);
                load(base);
#pragma unroll
                for (int j = 0; j < DEEP; ++j) {
                    if (base + sub + j * AT_ONCE >= r.count) continue;
                    float w[8];
                    vv[j].get(w);
                    most[0] = largest8(most[0], kv[j]);
                    most[1] = largest8(most[1], w);
                }
            }
#pragma unroll
            for (int o = 16; o; o >>= 1)
#pragma unroll
                for (int x = 0; x < 2; ++x) most[x] = max(most[x], __shfl_xor_sync(0xffffffffu, most[x], o));
            __syncthreads();                                                         // `part` of the head before has been read
            if (lane == 0) { part[0][warp] = most[0]; part[1][warp] = most[1]; }
            __syncthreads();
            Scale sc[2];
            unsigned char *cells[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                unsigned m = 0;
#pragma unroll
                for (int w = 0; w < kWarpsWide; ++w) m = max(m, part[x][w]);
                float *scale = (x ? a.c.d_v_scale : a.c.d_k_scale) + (long long)r.block * H + h;
                const float before = r.offset ? *scale : 0.f;
                sc[x] = scale_of(before, __uint_as_float(m), top_inverse);
                cells[x] = (unsigned char *)(x ? a.c.d_v : a.c.d_k) + r.block * a.c.block_stride + h * a.c.head_stride;
                if (r.offset && !(sc[x].now == before)) {
                    const float ratio = __fmul_rn(before, sc[x].inverse);
                    for (int i = sub; i < r.offset; i += AT_ONCE) requantise8<FMT>(cells[x] + i * a.c.token_stride + e0, ratio);
                }
            }
            for (int base = 0; base < r.count; base += PASS) {
                if (!one_pass) {
                    pass_angles(base);
                    load(base);
                }
#pragma unroll
                for (int j = 0; j < DEEP; ++j) {
                    const int i = base + sub + j * AT_ONCE;
                    if (i >= r.count) continue;
                    const long long at = (r.offset + i) * a.c.token_stride + e0;
                    float w[8];
                    vv[j].get(w);
                    *reinterpret_cast<uint2 *>(cells[0] + at) = entries8<FMT>(kv[j], sc[0].inverse);
                    *reinterpret_cast<uint2 *>(cells[1] + at) = entries8<FMT>(w, sc[1].inverse);
                }
            }
            __syncthreads();                                                         // every thread has read the old scales
            if (tid < 2) (tid ? a.c.d_v_scale : a.c.d_k_scale)[(long long)r.block * H + h] = tid ? sc[1].now : sc[0].now;
        }
    }
}

// Eight entries a thread and side; the entries of a token and head are PIECES neighbouring threads.
template <typename T, int FMT>
__global__ void __launch_bounds__(kWide) read_kernel(fluxbin_kv_cache_t c, int tokens, const int *slots, T *k_out, T *v_out)
{
    let_successor_start();
    wait_for_predecessor();
    const int pieces = c.head_dim / 8, each = c.kv_heads * pieces;
    const long long n = (long long)tokens * each, i = (long long)blockIdx.x * kWide + threadIdx.x;
    if (i >= n) return;
    const int t = (int)(i / each), h = (int)(i % each) / pieces, e0 = (int)(i % pieces) * 8;
    const int s = slots[t];
    const bool live = s >= 0 && s < c.num_blocks * c.block_tokens;
    const int b = live ? s / c.block_tokens : 0, off = live ? s % c.block_tokens : 0;
    const long long at = b * c.block_stride + h * c.head_stride + off * c.token_stride + e0, sc = (long long)b * c.kv_heads + h;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        T *out = side ? v_out : k_out;
        if (!out) continue;
        const uint2 w = *reinterpret_cast<const uint2 *>((const unsigned char *)(side ? c.d_v : c.d_k) + at);
        const float scale = (side ? c.d_v_scale : c.d_k_scale)[sc];
        __align__(16) T e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = from_float<T>(live ? Entry<FMT>::load((unsigned char)((j < 4 ? w.x : w.y) >> (j % 4 * 8))) * scale : 0.f);
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j) reinterpret_cast<uint4 *>(out + i * 8)[j] = reinterpret_cast<const uint4 *>(e)[j];
    }
}

template <typename T, int FMT, int D>
cudaError_t run_wide(AppendArgs a, bool rotary, cudaStream_t s)
{
    // A CTA looks through a few tokens for the first ones of runs, for a few heads: eight tokens and one head are a task
    // for each warp in a decode step (16 requests: 8.3 us, with 16 tokens 10.0).  In a prompt a CTA is busy only if a run begins in its tokens; its heads share the
    // run's angles, so they are no more cut than it takes to give every SM two CTAs that are busy.
    // Twice the tokens where even so there are CTAs enough (3000 tokens: 47 us with 8, 56 with 16; 9000: 116 and 107).
    const int H = a.c.kv_heads;
    a.tokens_each = a.tokens >= 4096 ? 16 : 8;
    const long long chunks = (a.tokens + a.tokens_each - 1) / a.tokens_each;
    const long long each = (long long)a.tokens / a.c.block_tokens * H / (148 * 2);
    a.heads_each = each < 1 ? 1 : each < H ? (int)each : H;
    a.groups = (H + a.heads_each - 1) / a.heads_each;
    a.append_ctas = (int)chunks * a.groups;
    a.q_groups = 0;
    if (rotary && a.q.heads > 0 && a.tokens >= kFewTokens) {
        // a prompt's queries fill the device by themselves, in a kernel that goes over tokens (9000 tokens: 107 us; as CTAs of
        // this launch 166)
        const cudaError_t e = launch_rotary(a.rot, std::is_same<T, float>::value ? FLUXBIN_TYPE_FP32 : std::is_same<T, __half>::value ? FLUXBIN_TYPE_FP16 : FLUXBIN_TYPE_BF16,
                                            0, a.tokens, a.positions, a.q, Side{}, s);
        if (e != cudaSuccess) return e;
        a.q.heads = 0;
    }
    if (rotary && a.q.heads > 0) {
        int g = (kFewTokens + a.tokens - 1) / a.tokens;
        const int at_least = kWide / (D * (int)sizeof(T) / 32);                      // heads that a CTA has in flight
        a.q_heads_each = (a.q.heads + g - 1) / g;
        if (a.q_heads_each < at_least) a.q_heads_each = at_least < a.q.heads ? at_least : a.q.heads;
        a.q_groups = (a.q.heads + a.q_heads_each - 1) / a.q_heads_each;
    }
    const dim3 grid((unsigned)(a.append_ctas + a.tokens * a.q_groups));
    constexpr int kPass = kWide / (D / 8) * 4;
    if (rotary) {
        const size_t smem = sizeof(float2) * (a.rot.rotary_dim / 2) * kPass;         // at most 64 pairs of 64 tokens: 32 KB
        return launch(append_kernel<T, FMT, D, true>, grid, kWide, smem, s, a);
    }
    return launch(append_kernel<T, FMT, D, false>, grid, kWide, 0, s, a);
}

template <typename T, int FMT>
cudaError_t run_append(const fluxbin_kv_cache_t &c, int tokens, const int *slots, const Heads &k, const Heads &v, const fluxbin_rotary_t *rot,
                       const int *positions, const Heads &q, const HeadsOut &qo, cudaStream_t s)
{
    const int n = 16 / (int)sizeof(T);
    bool wide = aligned_to(k.p, 16) && aligned_to(v.p, 16) && k.token % n == 0 && k.head % n == 0 && v.token % n == 0 && v.head % n == 0;
    AppendArgs a = {};
    if (rot) {
        a.rot = *rot;
        a.q = {q.p, qo.p, q.p ? q.heads : 0, q.token, q.head, qo.token, qo.head};
        wide = wide && rot->rotary_dim % (rot->interleaved ? 8 : 16) == 0 && wide_heads(*rot, sizeof(T) == 4 ? FLUXBIN_TYPE_FP32 : FLUXBIN_TYPE_FP16, a.q);
    }
    if (wide) {
        a.c = c;
        a.tokens = tokens;
        a.slots = slots;
        a.k = k;
        a.v = v;
        a.positions = positions;
        return c.head_dim == 64 ? run_wide<T, FMT, 64>(a, rot, s) : c.head_dim == 128 ? run_wide<T, FMT, 128>(a, rot, s) : run_wide<T, FMT, 256>(a, rot, s);
    }
    if (rot)
        return launch(append_any_kernel<T, FMT, true>, dim3((unsigned)tokens, (unsigned)(c.kv_heads + (q.p ? q.heads : 0))), kThreads, 0, s, c, tokens,
                      slots, k, v, *rot, positions, q, qo);
    return launch(append_any_kernel<T, FMT, false>, dim3((unsigned)tokens, (unsigned)c.kv_heads), kThreads, 0, s, c, tokens, slots, k, v,
                  fluxbin_rotary_t{}, positions, q, qo);
}

template <typename T>
cudaError_t run_read(const fluxbin_kv_cache_t &c, int tokens, const int *slots, void *k_out, void *v_out, cudaStream_t s)
{
    const long long n = (long long)tokens * c.kv_heads * (c.head_dim / 8);
    const dim3 grid((unsigned)((n + kWide - 1) / kWide));
    if (c.format == FLUXBIN_CACHE_INT8) return launch(read_kernel<T, FLUXBIN_CACHE_INT8>, grid, kWide, 0, s, c, tokens, slots, (T *)k_out, (T *)v_out);
    return launch(read_kernel<T, FLUXBIN_CACHE_E4M3>, grid, kWide, 0, s, c, tokens, slots, (T *)k_out, (T *)v_out);
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
    if (tokens < 0 || tokens > kMaxTokens) return FLUXBIN_ERR_RANGE;
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
    if (d_q && !heads_apart(tokens, q_heads, qo_token, qo_head, cache->head_dim)) return FLUXBIN_ERR_RANGE;
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
    if (tokens < 0 || tokens > kMaxTokens || (int64_t)tokens * cache->kv_heads * (cache->head_dim / 8) / kWide >= INT32_MAX) return FLUXBIN_ERR_RANGE;
    if (tokens == 0 || (!d_k_out && !d_v_out)) return FLUXBIN_OK;
    if (!d_slots) return FLUXBIN_ERR_NULL;
    if (!aligned_to(d_k_out, 16) || !aligned_to(d_v_out, 16) || !aligned_to(d_slots, 4)) return FLUXBIN_ERR_ALIGNMENT;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (dtype == FLUXBIN_TYPE_FP16) FBD_CUDA(run_read<__half>(*cache, tokens, d_slots, d_k_out, d_v_out, s));
    else if (dtype == FLUXBIN_TYPE_BF16) FBD_CUDA(run_read<__nv_bfloat16>(*cache, tokens, d_slots, d_k_out, d_v_out, s));
    else FBD_CUDA(run_read<float>(*cache, tokens, d_slots, d_k_out, d_v_out, s));
    return FLUXBIN_OK;
}
