// Norms of query and key heads with the rotary's turn in the same pass, and its gradients.
//
//     y = turn_p(w * n),  n = x * r,  r = (mean(x^2) + eps)^(-1/2)        forward: reads x, writes y
//     e = turn_p^-1(dy),  dx = r (w e - n mean(w e n)),  dw = sum e n     backward: reads x and dy, writes dx
//
// A head is held by head_dim / 16 neighbouring lanes, two pieces of eight elements each -- the two halves of eight pairs, or
// 16 neighbours where pairs are neighbours -- so a turn is a lane's own business and a mean is a few shuffles.  Warps go on their own,
// without a barrier (with one for each token 8191 tokens of 72 heads took 92 us), over equal parts of all tokens' heads; a warp forms a
// token's angles for itself and holds them and the gains in registers.
// The backward pass forms r again (one more sum beside mean(w e n), on the same shuffles) instead of reading it: nothing is
// kept from the forward pass but its inputs.  Gradients of the gains are summed in registers over a token's heads, then in
// shared memory over all that a thread sees, then over the CTA, then by a second launch over the CTAs: no atomics, the same sums each time.
// Bound by memory, with instructions close behind (a value at a time instead of two 109 us for the backward pass of 8190 tokens of 80
// heads of 128 in bf16, two 85: 503 MB, 5.9 TB/s).  8191 tokens of 72 heads forward: 53 us, 302 MB, 5.7 TB/s.  In fp32 the same 80 heads take
// 167 us forward and 271 backward (4.0 and 3.7 TB/s): as many bytes on their way, but a lane's 16-byte copies lie 32 bytes apart, so every sector
// is asked for twice.
#include "fluxbin_rotary.cuh"

#include <atomic>

using namespace fbd;

namespace {

constexpr int kThreads = 256, kMaxDim = 512;
constexpr int kMaxParts = 148 * 2;               // CTAs of a backward pass at most, each with its sums for the gradients of the gains

struct NormSide {
    const void *x, *weight;
    void *y;                                     // the result, or the gradient of x (may be NULL then)
    const void *grad;
    float *part;                                 // [parts][head_dim]: sums for the gradient of the gain, or NULL
    int heads;
    long long x_token, x_head, y_token, y_head, g_token, g_head;
};
struct NormArgs {
    fluxbin_rotary_t rot;
    float eps;
    int tokens, weight_dtype;
    long long share, over;                       // rounds of a warp; so many of the first warps have one more
    int rounds, q_rounds;                        // of a token, of its query heads
    const int *positions;
    NormSide q, k;
};

__device__ __forceinline__ float gain(const void *w, int dtype, int e)
{
    if (!w) return 1.f;
    if (dtype == FLUXBIN_TYPE_FP32) return static_cast<const float *>(w)[e];
    return dtype == FLUXBIN_TYPE_FP16 ? __half2float(static_cast<const __half *>(w)[e]) : __bfloat162float(static_cast<const __nv_bfloat16 *>(w)[e]);
}

// eight neighbouring elements
template <typename T> struct Piece {
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
    __device__ __forceinline__ void get(float *v) const
    {
        __align__(16) T e[8];
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(e)[i] = w[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_float(e[i]);
    }
    static __device__ __forceinline__ void put(T *p, const float *v)
    {
        Elements<T, 8> e;
#pragma unroll
        for (int i = 0; i < 8; i += 2) e.set(i, v[i], v[i + 1]);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(p)[i] = reinterpret_cast<const uint4 *>(e.e)[i];
    }
};

// a lane's share of a head: where its two pieces begin, and which pairs they are
struct Place {
    int e0, e1;
    bool there, turns;
};
template <bool INTER> __device__ __forceinline__ Place place_of(const fluxbin_rotary_t &rot, int u)
{
    Place p;
    p.there = u < rot.head_dim / 16;
    if (INTER) {
        p.turns = u < rot.rotary_dim / 16;
        p.e0 = 16 * u;
        p.e1 = 16 * u + 8;
    } else {
        const int turning = rot.rotary_dim / 16;
        p.turns = u < turning;
        p.e0 = p.turns ? 8 * u : rot.rotary_dim + 16 * (u - turning);
        p.e1 = p.turns ? 8 * u + rot.rotary_dim / 2 : p.e0 + 8;
    }
    return p;
}
// A lane's 16 elements are held two at a time (the unit for two fp32 values makes both in one instruction): the first elements
// of its eight pairs, then the second ones
typedef unsigned long long Two;
template <bool INTER> __device__ __forceinline__ int element(const Place &p, int k)
{
    return INTER ? p.e0 + (k < 8 ? 2 * k : 2 * k - 15) : k < 8 ? p.e0 + k : p.e1 + k - 8;
}
template <typename T, bool INTER> __device__ __forceinline__ void get_all(const Piece<T> (&p)[2], Two (&v)[8])
{
    float f[16];
    p[0].get(f);
    p[1].get(f + 8);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = !INTER ? two(f[2 * i], f[2 * i + 1]) : i < 4 ? two(f[4 * i], f[4 * i + 2]) : two(f[4 * i - 15], f[4 * i - 13]);
}
template <typename T, bool INTER> __device__ __forceinline__ void put_all(T *to, const Place &at, const Two (&v)[8])
{
    float f[16], x, y;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        apart(v[i], x, y);
        f[!INTER ? 2 * i : i < 4 ? 4 * i : 4 * i - 15] = x;
        f[!INTER ? 2 * i + 1 : i < 4 ? 4 * i + 2 : 4 * i - 13] = y;
    }
    Piece<T>::put(to + at.e0, f);
    Piece<T>::put(to + at.e1, f + 8);
}
// (as turn_pair; BACK: the other way round)
template <bool BACK> __device__ __forceinline__ void turn_all(Two (&v)[8], const Two (&c)[4], const Two (&s)[4])
{
    constexpr Two SIGNS = 0x8000000080000000ull;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Two x = v[i], y = v[i + 4];
        v[i] = fma_two(x, c[i], mul_two(y, BACK ? s[i] : s[i] ^ SIGNS));
        v[i + 4] = fma_two(y, c[i], mul_two(x, BACK ? s[i] ^ SIGNS : s[i]));
    }
}
__device__ __forceinline__ float sum_of_two(Two v)
{
    float x, y;
    apart(v, x, y);
    return x + y;
}
template <int LANES> __device__ __forceinline__ float sum_of(float v)
{
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// A round is ROWS heads of q or of k of a token, those that a warp's lanes hold side by side.  The rounds of all tokens are a line
// that is cut into equal parts for all warps, so that they end together wherever tokens do (with tokens whole, 8190 over 2368 warps
// are three or four for each, and some wait while others have a fourth of the work to do).
// A warp goes over its part of the line by runs: rounds of one token and side.
struct Runs {
    long long left;                              // rounds
    int t, first, n;                             // the run's token, its first round and how many
    bool k;
    __device__ __forceinline__ void begin(const NormArgs &a, long long w)
    {
        const long long at = w * a.share + min(w, a.over);
        left = a.share + (w < a.over);
        t = at >> 32 ? (int)(at / a.rounds) : (int)((unsigned)at / (unsigned)a.rounds);
        first = (int)(at - (long long)t * a.rounds);
        k = first >= a.q_rounds;
        if (k) first -= a.q_rounds;
        measure(a);
    }
    __device__ __forceinline__ void measure(const NormArgs &a)
    {
        const int whole = (k ? a.rounds - a.q_rounds : a.q_rounds) - first;
        n = left < whole ? (int)left : whole;
        left -= n;
    }
    // the next one (n == 0: there is none); whether a token begins
    __device__ __forceinline__ bool next(const NormArgs &a)
    {
        const bool both = !k && a.rounds > a.q_rounds;
        k = both || a.q_rounds == 0;
        t += !both;
        first = 0;
        measure(a);
        return !both;
    }
};
// What a round reads is brought by asynchronous copies, each thread's to places that only it reads again, rounds ahead
template <typename T, int TENSORS> struct Ahead {
    static constexpr int kPieces = TENSORS * (int)sizeof(T);     // of 16 bytes
    static constexpr int kStages = sizeof(T) == 2 ? 7 - 2 * TENSORS : 4 - TENSORS;
    static constexpr int kBytes = kStages * kPieces * kThreads * 16 + (TENSORS == 2 ? 2 * 8 * kThreads * (int)sizeof(Two) : 0);
};
template <typename T, int TENSORS, int ROWS> struct Bringer {
    using A = Ahead<T, TENSORS>;
    Runs runs;
    const unsigned char *from[TENSORS];
    long long step[TENSORS];
    int heads;                                   // from this row on
    uint32_t base, to;
    __device__ __forceinline__ void begin(const NormArgs &a, const Runs &r, const uint4 *places, int row)
    {
        runs = r;
        base = to = (uint32_t)__cvta_generic_to_shared(places);
        aim(a, row);
    }
    __device__ __forceinline__ void aim(const NormArgs &a, int row)
    {
        const NormSide &S = runs.k ? a.k : a.q;
        const int h = runs.first * ROWS + row;
        heads = S.heads - h;
        from[0] = (const unsigned char *)((const T *)S.x + runs.t * S.x_token + h * S.x_head);
        step[0] = S.x_head * (ROWS * (int)sizeof(T));
        if constexpr (TENSORS == 2) {
            from[1] = (const unsigned char *)((const T *)S.grad + runs.t * S.g_token + h * S.g_head);
            step[1] = S.g_head * (ROWS * (int)sizeof(T));
        }
    }
    // a round's pieces at e0 and e1
    __device__ __forceinline__ void bring(const NormArgs &a, const Place &at, int row)
    {
        constexpr int N = sizeof(T) / 2;
        if (runs.n > 0) {
            if (at.there && heads > 0) {
#pragma unroll
                for (int i = 0; i < TENSORS; ++i)
#pragma unroll
                    for (int k = 0; k < 2 * N; ++k)
                        copy_ahead<16>(to + (i * 2 * N + k) * kThreads * 16, from[i] + (k < N ? at.e0 : at.e1) * (int)sizeof(T) + k % N * 16);
            }
#pragma unroll
            for (int i = 0; i < TENSORS; ++i) from[i] += step[i];
            heads -= ROWS;
            if (--runs.n == 0 && runs.left > 0) {
                runs.next(a);
                aim(a, row);
            }
        }
        copies_commit();
        to = to == base + (A::kStages - 1) * A::kPieces * kThreads * 16 ? base : to + A::kPieces * kThreads * 16;
    }
};
template <typename T> __device__ __forceinline__ void take_pieces(const uint4 *from, Piece<T> (&p)[2])
{
    constexpr int N = sizeof(T) / 2;
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) p[i / N].w[i % N] = from[i * kThreads];
}
// Gains and a token's angles (cosines, then sines) as the lanes want them: 16 values of each lane, four at a time, side by side
template <int LANES> struct Lanes {
    float4 weight[2][4][LANES];
    float4 angles[kThreads / 32][4][LANES];
};
template <bool INTER, int LANES> __device__ __forceinline__ void keep_weights(const NormArgs &a, Lanes<LANES> &sm)
{
    for (int i = threadIdx.x; i < 2 * LANES * 16; i += kThreads) {
        const int side = i / (LANES * 16), u = i / 16 % LANES, k = i % 16;
        const Place p = place_of<INTER>(a.rot, u);
        reinterpret_cast<float *>(&sm.weight[side][k / 4][u])[k % 4] = p.there ? gain(side ? a.k.weight : a.q.weight, a.weight_dtype, element<INTER>(p, k)) : 0.f;
    }
    __syncthreads();
}
template <int LANES> __device__ __forceinline__ void take_weights(const Lanes<LANES> &sm, int side, int u, Two (&w)[8])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float4 x = sm.weight[side][k][u];
        w[2 * k] = two(x.x, x.y);
        w[2 * k + 1] = two(x.z, x.w);
    }
}
template <int LANES> __device__ __forceinline__ void lane_angles(const NormArgs &a, Lanes<LANES> &sm, int position, int warp, int lane, Two (&c)[4], Two (&s)[4])
{
    __syncwarp();                                // the last token's have been read
    float *to = reinterpret_cast<float *>(sm.angles[warp]);
    for (int p = lane; p < a.rot.rotary_dim / 2; p += 32) {
        const int at = (p % 8 / 4 * LANES + p / 8) * 4 + p % 4;
        pair_angle(position, a.rot.d_turns[p], a.rot.magnitude, 1.f, to[at], to[at + 2 * LANES * 4]);
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float4 x = sm.angles[warp][k][lane % LANES], y = sm.angles[warp][k + 2][lane % LANES];
        c[2 * k] = two(x.x, x.y);
        c[2 * k + 1] = two(x.z, x.w);
        s[2 * k] = two(y.x, y.y);
        s[2 * k + 1] = two(y.z, y.w);
    }
}

template <typename T, bool INTER, int LANES>
__global__ void __launch_bounds__(kThreads, 2) norm_kernel(const __grid_constant__ NormArgs a)
{
    using A = Ahead<T, 1>;
    constexpr int ROWS = 32 / LANES;
    __shared__ Lanes<LANES> sm;
    extern __shared__ uint4 brought[];           // [stage][piece][thread]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32, row = lane / LANES, u = lane % LANES;
    const Place at = place_of<INTER>(a.rot, u);
    const float inverse_dim = 1.f / a.rot.head_dim;
    let_successor_start();
    wait_for_predecessor();
    Runs now;
    now.begin(a, (long long)blockIdx.x * (kThreads / 32) + warp);
    Bringer<T, 1, ROWS> ahead;
    ahead.begin(a, now, brought + tid, row);
#pragma unroll 1
    for (int i = 0; i < A::kStages - 1; ++i) ahead.bring(a, at, row);
    int position = now.n > 0 ? a.positions[now.t] : 0;
    keep_weights<INTER, LANES>(a, sm);
    Two c[4], s[4];
    int stage = 0;
    for (bool begins = true; now.n > 0; begins = now.next(a)) {
        if (begins) {
            lane_angles<LANES>(a, sm, position, warp, lane, c, s);
            if (now.t + 1 < a.tokens) position = a.positions[now.t + 1];
        }
        const NormSide &S = now.k ? a.k : a.q;
        int h = now.first * ROWS + row;
        T *y = (T *)S.y + now.t * S.y_token + h * S.y_head;
        const long long y_step = S.y_head * ROWS;
        const int heads = S.heads;
        Two w[8];
        take_weights<LANES>(sm, now.k, u, w);
#pragma unroll 1
        for (int i = now.n; i > 0; --i, h += ROWS, y += y_step) {
            Two v[8], squares = 0;
            copies_wait<A::kStages - 2>();
            {
                Piece<T> p[2];
                take_pieces(brought + stage * A::kPieces * kThreads + tid, p);
                get_all<T, INTER>(p, v);
            }
            stage = stage == A::kStages - 1 ? 0 : stage + 1;
            ahead.bring(a, at, row);
            const bool mine = at.there && h < heads;
            if (mine) {
#pragma unroll
                for (int k = 0; k < 8; ++k) squares = fma_two(v[k], v[k], squares);
            }
            const float r = __frsqrt_rn(fmaf(sum_of<LANES>(sum_of_two(squares)), inverse_dim, a.eps));
            if (mine) {
                const Two r2 = two(r, r);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = mul_two(mul_two(v[k], r2), w[k]);
                if (at.turns) turn_all<false>(v, c, s);
                put_all<T, INTER>(y, at, v);
            }
        }
    }
    copies_wait<0>();
}

template <typename T, bool INTER, int LANES>
__global__ void __launch_bounds__(kThreads, 2) norm_backward_kernel(const __grid_constant__ NormArgs a)
{
    using A = Ahead<T, 2>;
    constexpr int ROWS = 32 / LANES;
    __shared__ Lanes<LANES> sm;
    extern __shared__ uint4 brought[];           // [stage][piece][thread], then the sums
    const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32, row = lane / LANES, u = lane % LANES, D = a.rot.head_dim;
    const Place at = place_of<INTER>(a.rot, u);
    const float inverse_dim = 1.f / D;
    let_successor_start();
    wait_for_predecessor();
    Runs now;
    now.begin(a, (long long)blockIdx.x * (kThreads / 32) + warp);
    Bringer<T, 2, ROWS> ahead;
    ahead.begin(a, now, brought + tid, row);
#pragma unroll 1
    for (int i = 0; i < A::kStages - 1; ++i) ahead.bring(a, at, row);
    int position = now.n > 0 ? a.positions[now.t] : 0;
    keep_weights<INTER, LANES>(a, sm);
    // sums for the gradients of the gains: a run's in registers, all runs' in places of this thread
    Two *sums = reinterpret_cast<Two *>(brought + A::kStages * A::kPieces * kThreads) + tid;           // [side][pair][thread]
#pragma unroll
    for (int i = 0; i < 16; ++i) sums[i * kThreads] = 0;
    Two c[4], s[4];
    int stage = 0;
    for (bool begins = true; now.n > 0; begins = now.next(a)) {
        if (begins) {
            lane_angles<LANES>(a, sm, position, warp, lane, c, s);
            if (now.t + 1 < a.tokens) position = a.positions[now.t + 1];
        }
        const NormSide &S = now.k ? a.k : a.q;
        int h = now.first * ROWS + row;
        T *dx = (T *)S.y + now.t * S.y_token + h * S.y_head;
        const long long dx_step = S.y_head * ROWS;
        const int heads = S.heads;
        const bool write = S.y != nullptr;
        Two w[8], dw[8];
        take_weights<LANES>(sm, now.k, u, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) dw[k] = 0;
#pragma unroll 1
        for (int i = now.n; i > 0; --i, h += ROWS, dx += dx_step) {
            const bool mine = at.there && h < heads;
            Two v[8], e[8], squares = 0, both = 0;
            copies_wait<A::kStages - 2>();
            {
                Piece<T> p[2];
                take_pieces(brought + stage * A::kPieces * kThreads + tid, p);
                get_all<T, INTER>(p, v);
                take_pieces(brought + (stage * A::kPieces + A::kPieces / 2) * kThreads + tid, p);
                get_all<T, INTER>(p, e);
            }
            stage = stage == A::kStages - 1 ? 0 : stage + 1;
            ahead.bring(a, at, row);
            if (mine) {
                if (at.turns) turn_all<true>(e, c, s);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    squares = fma_two(v[k], v[k], squares);
                    both = fma_two(mul_two(w[k], e[k]), v[k], both);
                }
            }
            const float r = __frsqrt_rn(fmaf(sum_of<LANES>(sum_of_two(squares)), inverse_dim, a.eps)), mean = sum_of<LANES>(sum_of_two(both)) * r * inverse_dim;
            if (mine) {
                const Two r2 = two(r, r), minus_mean = two(-mean, -mean);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    v[k] = mul_two(v[k], r2);
                    dw[k] = fma_two(e[k], v[k], dw[k]);
                    v[k] = mul_two(r2, fma_two(v[k], minus_mean, mul_two(w[k], e[k])));
                }
                if (write) put_all<T, INTER>(dx, at, v);
            }
        }
        Two *to = sums + now.k * 8 * kThreads;
#pragma unroll
        for (int k = 0; k < 8; ++k) to[k * kThreads] = add_two(to[k * kThreads], dw[k]);
    }
    copies_wait<0>();
    __syncthreads();
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
        float *to = side ? a.k.part : a.q.part;
        if (!to) continue;
        for (int j = tid; j < LANES * 16; j += kThreads) {
            const int lane_of = j / 16, i = j % 16;
            const Place p = place_of<INTER>(a.rot, lane_of);
            if (!p.there) continue;
            const float *from = reinterpret_cast<const float *>(sums - tid + (side * 8 + i / 2) * kThreads + lane_of) + i % 2;
            float s = 0.f;
            for (int k = 0; k < kThreads / LANES; ++k) s += from[2 * k * LANES];
            to[(long long)blockIdx.x * D + element<INTER>(p, i)] = s;
        }
    }
}

// Any strides, alignment and dimensions: a warp for each head, element by element.  Both elements of a pair are read before
// either is written, after all of the head has been read once.  8190 tokens of 80 heads of 128 in bf16, off 16-byte boundaries: 350 us
// forward, 1271 backward, which forms each head's angles twice (the kernels above 61 and 87).
struct Pair { int x, y; bool turns, two; };
__device__ __forceinline__ Pair pair_of(const fluxbin_rotary_t &rot, int u)
{
    const int half = rot.rotary_dim / 2;
    if (u >= half) return {u + half, u + half, false, false};
    return rot.interleaved ? Pair{2 * u, 2 * u + 1, true, true} : Pair{u, u + half, true, true};
}
template <typename T>
__global__ void __launch_bounds__(kThreads) norm_any_kernel(const __grid_constant__ NormArgs a)
{
    const int lane = threadIdx.x & 31, heads = a.q.heads + a.k.heads, D = a.rot.head_dim, units = D - a.rot.rotary_dim / 2;
    const long long rows = (long long)a.tokens * heads, step = (long long)gridDim.x * (kThreads / 32);
    let_successor_start();
    wait_for_predecessor();
    for (long long i = (long long)blockIdx.x * (kThreads / 32) + threadIdx.x / 32; i < rows; i += step) {
        const long long t = i / heads;
        const int j = (int)(i % heads), h = j < a.q.heads ? j : j - a.q.heads;
        const NormSide &S = j < a.q.heads ? a.q : a.k;
        const T *x = (const T *)S.x + t * S.x_token + h * S.x_head;
        T *y = (T *)S.y + t * S.y_token + h * S.y_head;
        float squares = 0.f;
        for (int e = lane; e < D; e += 32) {
            const float v = to_float(x[e]);
            squares = fmaf(v, v, squares);
        }
        const float r = __frsqrt_rn(sum_of<32>(squares) / D + a.eps);
        for (int u = lane; u < units; u += 32) {
            const Pair p = pair_of(a.rot, u);
            const float v = to_float(x[p.x]) * r * gain(S.weight, a.weight_dtype, p.x);
            if (!p.two) {
                y[p.x] = from_float<T>(v);
                continue;
            }
            const float w = to_float(x[p.y]) * r * gain(S.weight, a.weight_dtype, p.y);
            float c, s, f, g;
            pair_angle(a.positions[t], a.rot.d_turns[u], a.rot.magnitude, 1.f, c, s);
            turn_pair(v, w, c, s, f, g);
            y[p.x] = from_float<T>(f);
            y[p.y] = from_float<T>(g);
        }
    }
}
template <typename T>
__global__ void __launch_bounds__(kThreads) norm_any_backward_kernel(const __grid_constant__ NormArgs a)
{
    extern __shared__ float any_sums[];          // [warps][2][D]: each element is one lane's
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, heads = a.q.heads + a.k.heads, D = a.rot.head_dim, units = D - a.rot.rotary_dim / 2;
    const long long rows = (long long)a.tokens * heads, step = (long long)gridDim.x * (kThreads / 32);
    let_successor_start();
    wait_for_predecessor();
    for (int e = threadIdx.x; e < kThreads / 32 * 2 * D; e += kThreads) any_sums[e] = 0.f;
    __syncthreads();
    for (long long i = (long long)blockIdx.x * (kThreads / 32) + warp; i < rows; i += step) {
        const long long t = i / heads;
        const int j = (int)(i % heads), side = j >= a.q.heads, h = side ? j - a.q.heads : j;
        const NormSide &S = side ? a.k : a.q;
        const T *x = (const T *)S.x + t * S.x_token + h * S.x_head, *g = (const T *)S.grad + t * S.g_token + h * S.g_head;
        T *dx = (T *)S.y + t * S.y_token + h * S.y_head;
        float *dw = any_sums + (warp * 2 + side) * D;
        float squares = 0.f, both = 0.f;
        // e of a pair, formed twice: for the sums, then for the results
        auto turned_back = [&](int u, const Pair &p, float &ex, float &ey) {
            ex = to_float(g[p.x]);
            ey = 0.f;
            if (!p.two) return;
            const float second = to_float(g[p.y]);
            float c, s, f;
            pair_angle(a.positions[t], a.rot.d_turns[u], a.rot.magnitude, -1.f, c, s);
            turn_pair(ex, second, c, s, f, ey);
            ex = f;
        };
        for (int u = lane; u < units; u += 32) {
            const Pair p = pair_of(a.rot, u);
            float ex, ey;
            turned_back(u, p, ex, ey);
            const float v = to_float(x[p.x]), w = p.two ? to_float(x[p.y]) : 0.f;
            squares = fmaf(v, v, fmaf(w, w, squares));
            both = fmaf(ex * gain(S.weight, a.weight_dtype, p.x), v, both);
            if (p.two) both = fmaf(ey * gain(S.weight, a.weight_dtype, p.y), w, both);
        }
        const float r = __frsqrt_rn(sum_of<32>(squares) / D + a.eps), mean = sum_of<32>(both) * r / D;
        for (int u = lane; u < units; u += 32) {
            const Pair p = pair_of(a.rot, u);
            float e[2];
            turned_back(u, p, e[0], e[1]);
            for (int k = 0; k < (p.two ? 2 : 1); ++k) {
                const int at = k ? p.y : p.x;
                const float n = to_float(x[at]) * r;
                dw[at] = fmaf(e[k], n, dw[at]);
                if (S.y) dx[at] = from_float<T>(r * fmaf(-n, mean, gain(S.weight, a.weight_dtype, at) * e[k]));
            }
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
        float *to = i < D ? a.q.part : a.k.part;
        if (!to) continue;
        float s = 0.f;
        for (int w = 0; w < kThreads / 32; ++w) s += any_sums[w * 2 * D + i];
        to[(long long)blockIdx.x * D + i % D] = s;
    }
}

// the sums of all CTAs: 32 elements a CTA, 32 parts at a time
constexpr int kJoin = 1024;
__global__ void __launch_bounds__(kJoin) norm_join_kernel(int D, int parts, const float *q_part, const float *k_part, void *q_dw, void *k_dw, int weight_dtype)
{
    __shared__ float s[32][33];
    const int lane = threadIdx.x & 31, row = threadIdx.x / 32, e = blockIdx.x * 32 + lane;
    const float *part = blockIdx.y ? k_part : q_part;
    void *dw = blockIdx.y ? k_dw : q_dw;
    let_successor_start();
    wait_for_predecessor();
    if (!dw) return;
    float v = 0.f;
    if (e < D)
        for (int p = row; p < parts; p += 32) v += part[(long long)p * D + e];
    s[row][lane] = v;
    __syncthreads();
    v = sum_of<32>(s[lane][row]);
    const int to = blockIdx.x * 32 + row;
    if (lane == 0 && to < D) {
        if (weight_dtype == FLUXBIN_TYPE_FP32) static_cast<float *>(dw)[to] = v;
        else if (weight_dtype == FLUXBIN_TYPE_FP16) static_cast<__half *>(dw)[to] = __float2half_rn(v);
        else static_cast<__nv_bfloat16 *>(dw)[to] = __float2bfloat16_rn(v);
    }
}

// ---- launches ------------------------------------------------------------------------------------------

template <typename T> bool wide(const NormArgs &a, bool backward)
{
    const int64_t n = 16 / sizeof(T);
    if (a.rot.head_dim % 16 || a.rot.rotary_dim % 16) return false;
    for (const NormSide *s : {&a.q, &a.k}) {
        if (s->heads == 0) continue;
        if (!aligned_to(s->x, 16) || !aligned_to(s->y, 16) || s->x_token % n || s->x_head % n || s->y_token % n || s->y_head % n) return false;
        if (backward && (!aligned_to(s->grad, 16) || s->g_token % n || s->g_head % n)) return false;
    }
    return true;
}

template <typename K> cudaError_t run_ahead(K kernel, std::atomic<bool> *opted, int ctas, int bytes, cudaStream_t s, const NormArgs &a)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= fb::kMaxDevices) return cudaErrorInvalidDevice;
    if (!opted[dev].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != cudaSuccess) return e;
        opted[dev].store(true, std::memory_order_relaxed);
    }
    return launch(kernel, dim3((unsigned)ctas), kThreads, (size_t)bytes, s, a);
}
template <typename T, bool INTER, int LANES> cudaError_t run_wide(NormArgs a, bool backward, int &parts, cudaStream_t s)
{
    constexpr int ROWS = 32 / LANES, WARPS = kThreads / 32;
    a.q_rounds = (a.q.heads + ROWS - 1) / ROWS;
    a.rounds = a.q_rounds + (a.k.heads + ROWS - 1) / ROWS;
    // Two CTAs an SM are resident; the forward pass cuts the line finer, so that SMs that get more of the memory's rate do more of it (resident
    // CTAs once, twice, three, four times: 8191 tokens of 72 heads 54.5, 53.1, 54.0, 56.4 us; the backward pass, whose
    // sums cost each CTA something, 8190 tokens of 80 heads with the forward one: 149, 153, 160, 160)
    const long long total = (long long)a.tokens * a.rounds, ctas = backward ? kMaxParts : 148 * 4, need = (total + WARPS - 1) / WARPS;
    parts = (int)(need < ctas ? need : ctas);
    a.share = total / (parts * WARPS);
    a.over = total - a.share * parts * WARPS;
    static std::atomic<bool> opted[2][fb::kMaxDevices];
    if (backward) return run_ahead(norm_backward_kernel<T, INTER, LANES>, opted[1], parts, Ahead<T, 2>::kBytes, s, a);
    return run_ahead(norm_kernel<T, INTER, LANES>, opted[0], parts, Ahead<T, 1>::kBytes, s, a);
}
template <typename T, bool INTER> cudaError_t run_lanes(const NormArgs &a, bool backward, int &parts, cudaStream_t s)
{
    const int lanes = a.rot.head_dim / 16;
    if (lanes <= 4) return run_wide<T, INTER, 4>(a, backward, parts, s);
    if (lanes <= 8) return run_wide<T, INTER, 8>(a, backward, parts, s);
    if (lanes <= 16) return run_wide<T, INTER, 16>(a, backward, parts, s);
    return run_wide<T, INTER, 32>(a, backward, parts, s);
}
template <typename T> cudaError_t run(const NormArgs &a, bool backward, int &parts, cudaStream_t s)
{
    if (wide<T>(a, backward)) return a.rot.interleaved ? run_lanes<T, true>(a, backward, parts, s) : run_lanes<T, false>(a, backward, parts, s);
    const long long rows = (long long)a.tokens * (a.q.heads + a.k.heads), ctas = (rows + kThreads / 32 - 1) / (kThreads / 32);
    const long long most = backward ? kMaxParts : 148 * 8;
    parts = (int)(ctas < most ? ctas : most);
    if (backward) return launch(norm_any_backward_kernel<T>, dim3((unsigned)parts), kThreads, sizeof(float) * (kThreads / 32) * 2 * a.rot.head_dim, s, a);
    return launch(norm_any_kernel<T>, dim3((unsigned)parts), kThreads, 0, s, a);
}
cudaError_t run_type(const NormArgs &a, int dtype, bool backward, int &parts, cudaStream_t s)
{
    if (dtype == FLUXBIN_TYPE_FP16) return run<__half>(a, backward, parts, s);
    if (dtype == FLUXBIN_TYPE_BF16) return run<__nv_bfloat16>(a, backward, parts, s);
    return run<float>(a, backward, parts, s);
}

fluxbin_status_t check(const fluxbin_rotary_t *rotary, float eps, int dtype, int weight_dtype, int tokens)
{
    const fluxbin_status_t st = check_rotary(rotary);
    if (st != FLUXBIN_OK) return st;
    if (!type_known(dtype) || !type_known(weight_dtype)) return FLUXBIN_ERR_UNSUPPORTED;
    if (tokens < 0 || !(eps > 0.f && eps < 3e38f)) return FLUXBIN_ERR_RANGE;
    return FLUXBIN_OK;
}

} // namespace

extern "C" fluxbin_status_t fluxbin_norm_rotary(const fluxbin_rotary_t *rotary, float eps, int32_t dtype, int32_t weight_dtype, int32_t tokens,
                                                const int32_t *d_positions,
                                                const void *d_q, int32_t q_heads, int64_t q_token, int64_t q_head, const void *d_q_weight,
                                                void *d_q_out, int64_t qo_token, int64_t qo_head,
                                                const void *d_k, int32_t k_heads, int64_t k_token, int64_t k_head, const void *d_k_weight,
                                                void *d_k_out, int64_t ko_token, int64_t ko_head, void *cuda_stream)
{
    const fluxbin_status_t st = check(rotary, eps, dtype, weight_dtype, tokens);
    if (st != FLUXBIN_OK) return st;
    if (q_heads < 1 || q_heads > 65535 || (d_k && (k_heads < 1 || k_heads > 65535))) return FLUXBIN_ERR_RANGE;
    if (tokens == 0) return FLUXBIN_OK;
    if (!d_positions || !d_q || !d_q_out || (d_k && !d_k_out)) return FLUXBIN_ERR_NULL;
    const size_t size = (size_t)type_size(dtype), wsize = (size_t)type_size(weight_dtype);
    if (!d_k) d_k_weight = d_k_out = nullptr;
    for (const void *p : {d_q, (const void *)d_q_out, d_k, (const void *)d_k_out})
        if (!aligned_to(p, size)) return FLUXBIN_ERR_ALIGNMENT;
    if (!aligned_to(d_q_weight, wsize) || !aligned_to(d_k_weight, wsize) || !aligned_to(d_positions, 4)) return FLUXBIN_ERR_ALIGNMENT;
    if (!heads_apart(tokens, q_heads, qo_token, qo_head, rotary->head_dim) || (d_k && !heads_apart(tokens, k_heads, ko_token, ko_head, rotary->head_dim)))
        return FLUXBIN_ERR_RANGE;
    NormArgs a = {};
    a.rot = *rotary;
    a.eps = eps;
    a.tokens = tokens;
    a.weight_dtype = weight_dtype;
    a.positions = d_positions;
    a.q = {d_q, d_q_weight, d_q_out, nullptr, nullptr, q_heads, q_token, q_head, qo_token, qo_head, 0, 0};
    if (d_k) a.k = {d_k, d_k_weight, d_k_out, nullptr, nullptr, k_heads, k_token, k_head, ko_token, ko_head, 0, 0};
    int parts;
    FBD_CUDA(run_type(a, dtype, false, parts, (cudaStream_t)cuda_stream));
    return FLUXBIN_OK;
}

extern "C" size_t fluxbin_norm_rotary_backward_workspace_size(int32_t head_dim)
{
    return head_dim < 2 || head_dim > kMaxDim ? 0 : sizeof(float) * 2 * kMaxParts * (size_t)head_dim;
}

extern "C" fluxbin_status_t fluxbin_norm_rotary_backward(const fluxbin_rotary_t *rotary, float eps, int32_t dtype, int32_t weight_dtype, int32_t tokens,
                                                         const int32_t *d_positions,
                                                         const void *d_q, int32_t q_heads, int64_t q_token, int64_t q_head, const void *d_q_weight,
                                                         const void *d_q_grad, int64_t qg_token, int64_t qg_head,
                                                         void *d_q_dx, int64_t qd_token, int64_t qd_head, void *d_q_dweight,
                                                         const void *d_k, int32_t k_heads, int64_t k_token, int64_t k_head, const void *d_k_weight,
                                                         const void *d_k_grad, int64_t kg_token, int64_t kg_head,
                                                         void *d_k_dx, int64_t kd_token, int64_t kd_head, void *d_k_dweight,
                                                         void *d_workspace, size_t ws_bytes, void *cuda_stream)
{
    const fluxbin_status_t st = check(rotary, eps, dtype, weight_dtype, tokens);
    if (st != FLUXBIN_OK) return st;
    const int D = rotary->head_dim;
    const size_t size = (size_t)type_size(dtype), wsize = (size_t)type_size(weight_dtype);
    NormArgs a = {};
    a.rot = *rotary;
    a.eps = eps;
    a.tokens = tokens;
    a.weight_dtype = weight_dtype;
    a.positions = d_positions;
    if (d_q) a.q = {d_q, d_q_weight, d_q_dx, d_q_grad, (float *)d_q_dweight, q_heads, q_token, q_head, qd_token, qd_head, qg_token, qg_head};
    if (d_k) a.k = {d_k, d_k_weight, d_k_dx, d_k_grad, (float *)d_k_dweight, k_heads, k_token, k_head, kd_token, kd_head, kg_token, kg_head};
    bool any = false;
    for (const NormSide *s : {&a.q, &a.k}) {
        if (!s->x) continue;
        any = any || s->y || s->part;
        if (s->heads < 1 || s->heads > 65535) return FLUXBIN_ERR_RANGE;
        if (!s->grad) return FLUXBIN_ERR_NULL;
        if (!aligned_to(s->x, size) || !aligned_to(s->y, size) || !aligned_to(s->grad, size) || !aligned_to(s->weight, wsize) || !aligned_to(s->part, wsize))
            return FLUXBIN_ERR_ALIGNMENT;
        if (s->y && !heads_apart(tokens, s->heads, s->y_token, s->y_head, D)) return FLUXBIN_ERR_RANGE;
    }
    if (!any) return FLUXBIN_OK;
    if (!d_positions && tokens > 0) return FLUXBIN_ERR_NULL;
    if (!aligned_to(d_positions, 4)) return FLUXBIN_ERR_ALIGNMENT;
    void *q_dw = a.q.part, *k_dw = a.k.part;
    if (q_dw || k_dw) {
        if (!d_workspace) return FLUXBIN_ERR_NULL;
        if (!aligned_to(d_workspace, 16)) return FLUXBIN_ERR_ALIGNMENT;
        if (ws_bytes < fluxbin_norm_rotary_backward_workspace_size(D)) return FLUXBIN_ERR_BUFFER_TOO_SMALL;
        if (q_dw) a.q.part = (float *)d_workspace;
        if (k_dw) a.k.part = (float *)d_workspace + (size_t)kMaxParts * D;
    }
    // (strides that are not used must not keep a call from the wide kernel)
    for (NormSide *s : {&a.q, &a.k})
        if (!s->y) s->y_token = s->y_head = 0;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    int parts = 0;
    if (tokens > 0) FBD_CUDA(run_type(a, dtype, true, parts, s));
    if (q_dw || k_dw)
        FBD_CUDA(launch(norm_join_kernel, dim3((unsigned)((D + 31) / 32), 2), kJoin, 0, s, D, parts, (const float *)a.q.part, (const float *)a.k.part, q_dw, k_dw,
                        weight_dtype));
    return FLUXBIN_OK;
}
