// Norms of query and key heads with the rotary's turn in the same pass, and its gradients.
//
//     y = turn_p(w * n),  n = x * r,  r = (mean(x^2) + eps)^(-1/2)        forward: reads x, writes y
//     e = turn_p^-1(dy),  dx = r (w e - n mean(w e n)),  dw = sum e n     backward: reads x and dy, writes dx
//
// A head is held by head_dim / 16 neighbouring lanes, two pieces of eight elements each -- the two halves of eight pairs, or
// 16 neighbours where pairs are neighbours -- so a turn is a lane's own business and a mean is a few shuffles.  A warp takes a token,
// or a part of its heads: it forms the token's angles for itself, keeps them and the gains in registers, and has two heads of
// each lane under way.  No barrier of a CTA: with one for each token 8191 tokens of 72 heads took 92 us.
// The backward pass forms r again (one more sum beside mean(w e n), on the same shuffles) instead of reading it: nothing is
// kept from the forward pass but its inputs.  Gradients of the gains are summed in registers over all that a thread sees,
// then over the CTA, then by a second launch over the CTAs: no atomics, the same sums each time.
// Bound by memory.
#include "fluxbin_rotary.cuh"

using namespace fbd;

namespace {

constexpr int kThreads = 256, kMaxDim = 512;
constexpr int kMaxParts = 148 * 4;               // CTAs of a backward pass

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
    unsigned splits;
    int heads_each;
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
// the eight pairs of a lane's 16 elements
template <bool INTER> __device__ __forceinline__ void turn_all(float (&v)[16], const float2 (&a)[8], float sign)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int x = INTER ? 2 * i : i, y = INTER ? 2 * i + 1 : i + 8;
        float f, g;
        turn_pair(v[x], v[y], a[i].x, sign * a[i].y, f, g);
        v[x] = f;
        v[y] = g;
    }
}
template <int LANES> __device__ __forceinline__ float sum_of(float v)
{
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// What a warp's item is: a token and a range of its heads
struct Item { int t, h0, h1; };
__device__ __forceinline__ Item item_of(const NormArgs &a, unsigned i)
{
    Item x;
    x.t = (int)(i / a.splits);
    x.h0 = (int)(i % a.splits) * a.heads_each;
    x.h1 = min(x.h0 + a.heads_each, a.q.heads + a.k.heads);
    return x;
}
// Gains and a token's angles as the lanes want them: 16 values of each lane, four at a time, side by side
template <int LANES> struct Lanes {
    float4 weight[2][4][LANES];
    float4 angles[kThreads / 32][4][LANES];
};
template <bool INTER, int LANES> __device__ __forceinline__ void keep_weights(const NormArgs &a, Lanes<LANES> &sm)
{
    for (int i = threadIdx.x; i < 2 * LANES * 16; i += kThreads) {
        const int side = i / (LANES * 16), u = i / 16 % LANES, k = i % 16;
        const Place p = place_of<INTER>(a.rot, u);
        reinterpret_cast<float *>(&sm.weight[side][k / 4][u])[k % 4] = p.there ? gain(side ? a.k.weight : a.q.weight, a.weight_dtype, k < 8 ? p.e0 + k : p.e1 + k - 8) : 0.f;
    }
    __syncthreads();
}
// f(element, gain) for a lane's 16 elements, gains from shared memory each time: registers are what limits the bytes under way
template <int LANES, typename F> __device__ __forceinline__ void with_weights(const Lanes<LANES> &sm, int side, int u, F f)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float4 w = sm.weight[side][k][u];
        f(4 * k, w.x);
        f(4 * k + 1, w.y);
        f(4 * k + 2, w.z);
        f(4 * k + 3, w.w);
    }
}
template <int LANES> __device__ __forceinline__ void lane_angles(const NormArgs &a, Lanes<LANES> &sm, int position, int warp, int lane, float2 (&cs)[8])
{
    __syncwarp();                                // the last token's have been read
    for (int p = lane; p < a.rot.rotary_dim / 2; p += 32) {
        float2 x;
        pair_angle(position, a.rot.d_turns[p], a.rot.magnitude, 1.f, x.x, x.y);
        reinterpret_cast<float2 *>(&sm.angles[warp][p % 8 / 2][p / 8])[p & 1] = x;
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 4; ++k) *reinterpret_cast<float4 *>(cs + 2 * k) = sm.angles[warp][k][lane % LANES];
}

template <typename T, bool INTER, int LANES>
__global__ void __launch_bounds__(kThreads, 3) norm_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int ROWS = 32 / LANES, AHEAD = sizeof(T) == 4 ? 1 : 2;
    __shared__ Lanes<LANES> sm;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, row = lane / LANES, u = lane % LANES;
    const Place at = place_of<INTER>(a.rot, u);
    const float inverse_dim = 1.f / a.rot.head_dim;
    let_successor_start();
    wait_for_predecessor();
    keep_weights<INTER, LANES>(a, sm);
    const unsigned items = (unsigned)a.tokens * a.splits, step = gridDim.x * (kThreads / 32);          // (more than 2^31 tokens are not split)
    for (unsigned i = blockIdx.x * (kThreads / 32) + warp; i < items; i += step) {
        const Item item = item_of(a, i);
        float2 cs[8];
        bool formed = false;
#pragma unroll 1
        for (int side = 0; side < 2; ++side) {
            const NormSide &S = side ? a.k : a.q;
            const int lo = max(item.h0 - (side ? a.q.heads : 0), 0), hi = min(item.h1 - (side ? a.q.heads : 0), S.heads);
            if (lo >= hi) continue;
            const T *x = (const T *)S.x + item.t * S.x_token + (long long)(lo + row) * S.x_head;
            T *y = (T *)S.y + item.t * S.y_token + (long long)(lo + row) * S.y_head;
            Piece<T> p[AHEAD][2];
            auto load = [&](int h, Piece<T> (&to)[2]) {
                if (at.there && h + row < hi) {
                    to[0].load(x + at.e0);
                    to[1].load(x + at.e1);
                }
                x += ROWS * S.x_head;
            };
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) load(lo + j * ROWS, p[j]);
            if (!formed) lane_angles<LANES>(a, sm, a.positions[item.t], warp, lane, cs);         // (while the first heads are on their way)
            formed = true;
            // (every lane goes as many rounds: they meet in the shuffles)
            for (int h0 = lo; h0 < hi; h0 += AHEAD * ROWS)
#pragma unroll
                for (int j = 0; j < AHEAD; ++j, y += ROWS * S.y_head) {
                    const int h = h0 + j * ROWS;
                    if (h >= hi) break;
                    const bool mine = at.there && h + row < hi;
                    float v[16], squares = 0.f;
                    p[j][0].get(v);
                    p[j][1].get(v + 8);
                    load(h + AHEAD * ROWS, p[j]);
                    if (mine) {
#pragma unroll
                        for (int k = 0; k < 16; ++k) squares = fmaf(v[k], v[k], squares);
                    }
                    const float r = __frsqrt_rn(fmaf(sum_of<LANES>(squares), inverse_dim, a.eps));
                    if (!mine) continue;
                    with_weights<LANES>(sm, side, u, [&](int k, float w) { v[k] = v[k] * r * w; });
                    if (at.turns) turn_all<INTER>(v, cs, 1.f);
                    Piece<T>::put(y + at.e0, v);
                    Piece<T>::put(y + at.e1, v + 8);
                }
        }
    }
}

template <typename T, bool INTER, int LANES>
__global__ void __launch_bounds__(kThreads, 2) norm_backward_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int ROWS = 32 / LANES;
    __shared__ union { Lanes<LANES> lanes; float sums[16][kThreads]; } sm;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32, row = lane / LANES, u = lane % LANES, D = a.rot.head_dim;
    const Place at = place_of<INTER>(a.rot, u);
    const float inverse_dim = 1.f / D;
    let_successor_start();
    wait_for_predecessor();
    keep_weights<INTER, LANES>(a, sm.lanes);
    float dw[2][16];
#pragma unroll
    for (int i = 0; i < 16; ++i) dw[0][i] = dw[1][i] = 0.f;
    const unsigned items = (unsigned)a.tokens * a.splits, step = gridDim.x * (kThreads / 32);          // (more than 2^31 tokens are not split)
    for (unsigned i = blockIdx.x * (kThreads / 32) + warp; i < items; i += step) {
        const Item item = item_of(a, i);
        float2 cs[8];
        bool formed = false;
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const NormSide &S = side ? a.k : a.q;
            const int lo = max(item.h0 - (side ? a.q.heads : 0), 0), hi = min(item.h1 - (side ? a.q.heads : 0), S.heads);
            if (lo >= hi) continue;
            const T *x = (const T *)S.x + item.t * S.x_token + (long long)(lo + row) * S.x_head;
            const T *g = (const T *)S.grad + item.t * S.g_token + (long long)(lo + row) * S.g_head;
            T *dx = S.y ? (T *)S.y + item.t * S.y_token + (long long)(lo + row) * S.y_head : nullptr;
            Piece<T> p[4];
            auto load = [&](int h) {
                if (at.there && h + row < hi) {
                    p[0].load(x + at.e0);
                    p[1].load(x + at.e1);
                    p[2].load(g + at.e0);
                    p[3].load(g + at.e1);
                }
            };
            load(lo);
            if (!formed) lane_angles<LANES>(a, sm.lanes, a.positions[item.t], warp, lane, cs);
            formed = true;
            for (int h = lo; h < hi; h += ROWS) {
                const bool mine = at.there && h + row < hi;
                float v[16], e[16], squares = 0.f, both = 0.f;
                p[0].get(v);
                p[1].get(v + 8);
                p[2].get(e);
                p[3].get(e + 8);
                x += ROWS * S.x_head;
                g += ROWS * S.g_head;
                if (sizeof(T) == 2) load(h + ROWS);              // (registers for the next ones)
                if (mine) {
                    if (at.turns) turn_all<INTER>(e, cs, -1.f);
                    with_weights<LANES>(sm.lanes, side, u, [&](int k, float w) {
                        squares = fmaf(v[k], v[k], squares);
                        both = fmaf(w * e[k], v[k], both);
                    });
                }
                squares = sum_of<LANES>(squares);
                both = sum_of<LANES>(both);
                if (mine) {
                    const float r = __frsqrt_rn(fmaf(squares, inverse_dim, a.eps)), mean = both * r * inverse_dim;
                    with_weights<LANES>(sm.lanes, side, u, [&](int k, float w) {
                        const float n = v[k] * r;
                        dw[side][k] = fmaf(e[k], n, dw[side][k]);
                        v[k] = r * fmaf(-n, mean, w * e[k]);
                    });
                    if (dx) {
                        Piece<T>::put(dx + at.e0, v);
                        Piece<T>::put(dx + at.e1, v + 8);
                    }
                }
                if (dx) dx += ROWS * S.y_head;
                if (sizeof(T) != 2) load(h + ROWS);
            }
        }
    }
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        float *to = side ? a.k.part : a.q.part;
        if (!to) continue;                       // (the same for every thread)
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) sm.sums[i][tid] = dw[side][i];
        __syncthreads();
        for (int j = tid; j < LANES * 16; j += kThreads) {
            const int lane_of = j / 16, i = j % 16;
            const Place p = place_of<INTER>(a.rot, lane_of);
            if (!p.there) continue;
            float s = 0.f;
            for (int k = 0; k < kThreads / LANES; ++k) s += sm.sums[i][k * LANES + lane_of];
            to[(long long)blockIdx.x * D + (i < 8 ? p.e0 + i : p.e1 + i - 8)] = s;
        }
    }
}

// Any strides, alignment and dimensions: a warp for each head, element by element.  Both elements of a pair are read before
// either is written, after all of the head has been read once.
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

template <typename T, bool INTER, int LANES> cudaError_t run_wide(NormArgs a, bool backward, int &parts, cudaStream_t s)
{
    // Resident warps go over tokens.  Tokens are split into parts of their heads until there are three for every warp, but no part is
    // less than four rounds of heads, since the angles are formed for each; fewer tokens than warps are split until every warp has one.
    constexpr int ROWS = 32 / LANES, WARPS = kThreads / 32;
    const long long heads = a.q.heads + a.k.heads, rounds = (heads + ROWS - 1) / ROWS, ctas = 148 * (backward ? 2 : 3), warps = ctas * WARPS;
    long long splits = (3 * warps + a.tokens - 1) / a.tokens, most = rounds / 4 > 1 ? rounds / 4 : 1;
    if (splits > most) splits = most;
    if (a.tokens * splits < warps) splits = (warps + a.tokens - 1) / a.tokens < rounds ? (warps + a.tokens - 1) / a.tokens : rounds;
    a.heads_each = (int)((rounds + splits - 1) / splits) * ROWS;
    a.splits = (unsigned)((heads + a.heads_each - 1) / a.heads_each);
    const long long items = (long long)a.tokens * a.splits, need = (items + WARPS - 1) / WARPS;
    parts = (int)(need < ctas ? need : ctas);
    const dim3 grid((unsigned)parts);
    return backward ? launch(norm_backward_kernel<T, INTER, LANES>, grid, kThreads, 0, s, a) : launch(norm_kernel<T, INTER, LANES>, grid, kThreads, 0, s, a);
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
    const long long most = backward ? 148 * 2 : 148 * 8;
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
