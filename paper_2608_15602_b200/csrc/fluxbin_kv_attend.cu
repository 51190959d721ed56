// Attention of new tokens over the 8-bit block-paged cache (fluxbin_kv_attend).
//
// For one key head and a group of query rows (the query heads that share it, over the request's new tokens) the kernel
// forms, 16 cached tokens at a time,
//     S^T = K Q^T  [16 tokens x rows],   P = exp2(S c - m),   O^T += V^T P^T  [dim x rows],   l += sum P
// with the tokens (then the elements of a head) as the 16-row side of the matrix instruction and the query rows as its
// 8-column side: a decode step has as few rows as query heads share a key head, and 8 columns waste the least.
//
// What bounds it is the cache's bytes.  Every byte goes from memory straight into the register of the lane that holds it
// as a matrix operand -- no shared memory, no shuffles: which element a lane's operand slot stands for is free as long as
// both operands agree, so a lane takes 16 consecutive bytes wherever the instruction would want scattered pairs.
//   keys:    lane (r, q) = (lane / 4, lane % 4) reads elements 16 q .. + 15 of each 64-byte piece of tokens r and r + 8
//   values:  the same lane reads elements 16 r .. + 15 (of 128) of tokens 2q, 2q + 1, 2q + 8, 2q + 9 and interleaves the
//            bytes of two tokens, which the conversion to fp16 does on the way
// P leaves the first product with a lane per token and enters the second with a lane per row: movmatrix turns it.
// 8-bit entries are exact in fp16.  The block's key scale multiplies the score in fp32; the value scale, relative to the
// largest one met so far (vref), multiplies P before P is rounded to fp16.  That rounding (2^-11 of each probability,
// against 2^-9 of bf16) is the only one below 32 bits; probabilities are held between 2^15 and fp16's smallest steps by
// letting the reference m lag: it is raised to (row maximum - 7) only when a P would pass 2^15, so that most steps need no
// reduction over lanes and what is flushed to zero is below 2^-31 of the largest probability.
//
// Work is cut evenly whatever the lengths are: all (request, rows, head) jobs in units of 128 tokens form a line, CTA i of
// n takes the i-th n-th of it (the lengths are read on the device: a captured graph serves every step).  A job cut between
// CTAs leaves normalised partial results and their lse in the workspace; the CTA that arrives last joins them in order.
#include "fluxbin_cache.cuh"

#include <atomic>

using namespace fbd;

namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kUnit = kWarps * 16;              // cached tokens of a unit: 16 for each warp
constexpr int kMaxGrid = 320;                   // two CTAs on each SM
constexpr int kMaxRows = 16;

struct Args {
    fluxbin_kv_cache_t c;
    int batch, tokens, q_heads, width;
    const void *q;
    long long q_token, q_head;
    const int *query_start, *lengths, *table;
    long long table_stride;
    float scale;
    void *out;
    long long out_token, out_head;
    float *lse;
    unsigned *arrived;                          // [kMaxGrid], by the CTA in which a cut job begins
    float *partial;                             // [kMaxGrid][2][rows][D], then [kMaxGrid][2][rows] lse (base 2)
    int min_share;                              // units a CTA has at least
};

// ---- conversions of four 8-bit entries to two pairs of fp16 ---------------------------------------------

template <int FMT> __device__ __forceinline__ void to_half4(uint32_t x, uint32_t &lo, uint32_t &hi);
// int8: the byte with its sign bit flipped, under the exponent of 1024, is 1024 + 128 + value; fp16 holds that exactly
template <> __device__ __forceinline__ void to_half4<FLUXBIN_CACHE_INT8>(uint32_t x, uint32_t &lo, uint32_t &hi)
{
    x ^= 0x80808080u;
    const uint32_t a = __byte_perm(x, 0x64646464u, 0x4140), b = __byte_perm(x, 0x64646464u, 0x4342);
    const __half2 off = __half2half2(__ushort_as_half(0x6480));           // 1152
    const __half2 ra = __hsub2(*reinterpret_cast<const __half2 *>(&a), off), rb = __hsub2(*reinterpret_cast<const __half2 *>(&b), off);
    lo = *reinterpret_cast<const uint32_t *>(&ra);
    hi = *reinterpret_cast<const uint32_t *>(&rb);
}
template <> __device__ __forceinline__ void to_half4<FLUXBIN_CACHE_E4M3>(uint32_t x, uint32_t &lo, uint32_t &hi)
{
    asm("{ .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n }" : "=r"(lo), "=r"(hi) : "r"(x));
}

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t v)
{
    uint32_t t;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(t) : "r"(v));
    return t;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float exp2_fast(float x)         // relative error 2^-22, exp2(-inf) = 0
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// the cache is read once: past L1
template <int N> struct Words { uint32_t w[N]; };
template <int N> __device__ __forceinline__ Words<N> load_stream(const unsigned char *p)
{
    Words<N> v;
    if constexpr (N == 4)
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]) : "l"(p));
    else
        asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.w[0]), "=r"(v.w[1]) : "l"(p));
    return v;
}

// ---- the line of work -----------------------------------------------------------------------------------

struct Request {
    int first, count;            // its new tokens
    int length;                  // its cached tokens
    int row_tiles, pieces;       // tiles of query rows a head has, units of cached tokens
};
template <int ROWS> __device__ __forceinline__ Request request_of(const Args &a, int r)
{
    Request q;
    if (a.query_start) {
        q.first = min(max(a.query_start[r], 0), a.tokens);
        q.count = max(min(max(a.query_start[r + 1], 0), a.tokens) - q.first, 0);
    } else {
        q.first = r;
        q.count = 1;
    }
    q.length = (int)min((long long)max(a.lengths[r], 0), (long long)a.width * a.c.block_tokens);
    q.row_tiles = (int)(((long long)q.count * (a.q_heads / a.c.kv_heads) + ROWS - 1) / ROWS);
    q.pieces = max((q.length + kUnit - 1) / kUnit, 1);          // an empty request still has rows to write
    return q;
}
__device__ __forceinline__ long long units_of(const Args &a, const Request &q) { return (long long)q.row_tiles * a.c.kv_heads * q.pieces; }

template <int D, int ROWS> struct Shared {
    float o[kWarps][ROWS][D + 4];
    float m[kWarps][ROWS], l[kWarps][ROWS], v[kWarps];
    long long scan[kWarps], before;
    int request, last;
};

// one CTA: its part of the line, job after job
template <int D, int FMT, int NT, typename T>
__global__ void __launch_bounds__(kThreads, D == 256 || NT == 2 ? 1 : 2) attend_kernel(const __grid_constant__ Args a)
{
    constexpr int ROWS = 8 * NT;
    constexpr int KC = D / 64;                   // 64-byte pieces of a key
    constexpr int VW = D >= 128 ? 4 : 2;         // words of a load of values
    constexpr int VC = D / (VW * 32);            // pieces of a value row (eight lanes of VW words each)
    constexpr int MT = D / 16;                   // 16-element tiles of the output
    extern __shared__ __align__(16) unsigned char smem_raw[];
    Shared<D, ROWS> &sm = *reinterpret_cast<Shared<D, ROWS> *>(smem_raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, lr = lane >> 2, lq = lane & 3;
    const int H = a.c.kv_heads, G = a.q_heads / H, bs = a.c.block_tokens;

    let_successor_start();
    wait_for_predecessor();

    // ---- where this CTA's part begins: a sum over the requests, each thread over a run of them
    const int per = (a.batch + kThreads - 1) / kThreads, r_lo = min(tid * per, a.batch), r_hi = min(r_lo + per, a.batch);
    long long mine = 0;
    for (int r = r_lo; r < r_hi; ++r) mine += units_of(a, request_of<ROWS>(a, r));
    long long upto = mine;
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    if (lane == 31) sm.scan[warp] = upto;
    __syncthreads();
    long long total = 0;
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) upto += sm.scan[w];
        total += sm.scan[w];
    }
    const long long shares = min((long long)gridDim.x, (total + a.min_share - 1) / a.min_share);
    if (blockIdx.x >= shares) return;
    auto cut = [&](long long i) { return i * total / shares; };
    long long u = cut(blockIdx.x);
    const long long u_end = cut(blockIdx.x + 1);
    if (u >= upto - mine && u < upto) {
        long long before = upto - mine;
        for (int r = r_lo; r < r_hi; ++r) {
            const long long n = units_of(a, request_of<ROWS>(a, r));
            if (u < before + n) { sm.request = r; sm.before = before; break; }
            before += n;
        }
    }
    __syncthreads();
    int r = sm.request;
    long long r_before = sm.before;
    Request rq = request_of<ROWS>(a, r);

    while (u < u_end) {
        while (u >= r_before + units_of(a, rq)) {
            r_before += units_of(a, rq);
            rq = request_of<ROWS>(a, ++r);
        }
        const long long in_request = u - r_before;
        const int job = (int)(in_request / rq.pieces), p0 = (int)(in_request % rq.pieces);
        const int p1 = (int)min((long long)rq.pieces, p0 + (u_end - u));
        const int h = job / rq.row_tiles, row0 = job % rq.row_tiles * ROWS;
        const int rows = (int)min((long long)ROWS, (long long)rq.count * G - row0);
        // tokens that the last and the first row of the tile see
        const int seen = rq.length - (rq.count - 1 - (row0 + rows - 1) / G);
        const int seen_first = rq.length - (rq.count - 1 - row0 / G);
        int limit[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) limit[t][e] = rq.length - (rq.count - 1 - min(row0 + t * 8 + 2 * lq + e, row0 + rows - 1) / G);

        // ---- the block ids and scales of this warp's tiles: lane i holds those of tile i of a batch of 32
        const int tok0 = p0 * kUnit + warp * 16;
        const int tiles = max((min(seen, p1 * kUnit) - tok0 + kUnit - 1) / kUnit, 0);
        const int *row_table = a.table + r * a.table_stride;
        auto id_of = [&](int tile) {
            if (tile >= tiles) return -1;
            const int id = row_table[(tok0 + tile * kUnit) / bs];
            return id >= 0 && id < a.c.num_blocks ? id : -1;
        };
        int id_now = id_of(lane), id_next = -1;
        float ks_now = 0.f, vs_now = 0.f, ks_next = 0.f, vs_next = 0.f;
        if (id_now >= 0) {
            ks_now = a.c.d_k_scale[(long long)id_now * H + h];
            vs_now = a.c.d_v_scale[(long long)id_now * H + h];
        }

        // ---- the query rows as the 8-column operand: lane (r, q) holds row r, 16 elements of each 64-element piece
        uint32_t qf[NT][KC * 4][2];
        float factor[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int row = row0 + t * 8 + lr;
            const bool live = t * 8 + lr < rows;
            const T *qp = (const T *)a.q + (rq.first + (live ? row / G : 0)) * a.q_token + (h * G + (live ? row % G : 0)) * a.q_head;
            float largest = 0.f;
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                uint4 w[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    w[i] = live ? *reinterpret_cast<const uint4 *>(qp + c * 64 + lq * 16 + i * 8) : make_uint4(0, 0, 0, 0);
                    const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        qf[t][c * 4 + i * 2 + k / 2][k % 2] = v[k];
                        if constexpr (sizeof(T) == 2 && !std::is_same<T, __half>::value) {
                            largest = fmaxf(largest, fabsf(__uint_as_float(v[k] << 16)));
                            largest = fmaxf(largest, fabsf(__uint_as_float(v[k] & 0xffff0000u)));
                        }
                    }
                }
            }
            float f = 1.f;
            if constexpr (!std::is_same<T, __half>::value) {
                // bf16 rows become fp16 exactly, multiplied by the power of two that takes their largest element to
                // 2^14 .. 2^15; elements below 2^-39 of it lose bits that fp32 sums would not keep
                largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, 1));
                largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, 2));
                const int e = largest > 0.f ? min(max((int)(__float_as_uint(largest) >> 23), 1), 254) - 127 - 14 : 0;
#pragma unroll
                for (int i = 0; i < KC * 4; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        qf[t][i][k] = pack_half2(ldexpf(__uint_as_float(qf[t][i][k] << 16), -e), ldexpf(__uint_as_float(qf[t][i][k] & 0xffff0000u), -e));
                f = ldexpf(a.scale * 1.4426950408889634f, e);
            } else {
                f = a.scale * 1.4426950408889634f;
            }
            // the factor of a row is wanted by the lanes that hold its column
#pragma unroll
            for (int e = 0; e < 2; ++e) factor[t][e] = __shfl_sync(0xffffffffu, f, (2 * lq + e) * 4);
        }

        float o[NT][MT][4], ref[NT][2], sum[NT][2], vref = 0.f, vref_inverse = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < MT; ++i) o[t][i][0] = o[t][i][1] = o[t][i][2] = o[t][i][3] = 0.f;
            ref[t][0] = ref[t][1] = -INFINITY;
            sum[t][0] = sum[t][1] = 0.f;
        }

        Words<4> kw[2][KC];
        Words<VW> vw[4][VC];
        auto load_k = [&](int id, int tok) {
            const unsigned char *p = (const unsigned char *)a.c.d_k + id * a.c.block_stride + h * a.c.head_stride + (tok % bs + lr) * a.c.token_stride + lq * 16;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int c = 0; c < KC; ++c) {
                    if (id >= 0) kw[i][c] = load_stream<4>(p + i * 8 * a.c.token_stride + c * 64);
                    else kw[i][c] = Words<4>{{0, 0, 0, 0}};
                }
        };
        auto load_v = [&](int id, int tok) {
            const unsigned char *p = (const unsigned char *)a.c.d_v + id * a.c.block_stride + h * a.c.head_stride + (tok % bs + 2 * lq) * a.c.token_stride + lr * (VW * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < VC; ++c) {
                    if (id >= 0) vw[i][c] = load_stream<VW>(p + ((i & 1) + (i >> 1) * 8) * a.c.token_stride + c * (VW * 32));
                    else vw[i][c] = Words<VW>{};
                }
        };

        int id = __shfl_sync(0xffffffffu, id_now, 0);
        float ks = __shfl_sync(0xffffffffu, ks_now, 0), vs = __shfl_sync(0xffffffffu, vs_now, 0);
        if (tiles > 0) {
            load_k(id, tok0);
            load_v(id, tok0);
        }
        if (tiles > 32) id_next = id_of(32 + lane);

        for (int tile = 0; tile < tiles; ++tile) {
            const int tok = tok0 + tile * kUnit;
            // ---- scores
            float s[NT][4];
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.f;
#pragma unroll
            for (int c = 0; c < KC; ++c)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t a0, a1, a2, a3;
                    to_half4<FMT>(kw[0][c].w[w], a0, a2);
                    to_half4<FMT>(kw[1][c].w[w], a1, a3);
#pragma unroll
                    for (int t = 0; t < NT; ++t) mma(s[t], a0, a1, a2, a3, qf[t][c * 4 + w][0], qf[t][c * 4 + w][1]);
                }
            // ---- the next tile's block and scales, its keys on their way
            const int nt = tile + 1, slot = nt & 31;
            if (slot == 0) { id_now = id_next; ks_now = ks_next; vs_now = vs_next; if (nt + 32 < tiles) id_next = id_of(nt + 32 + lane); }
            if (slot == 16 && id_next >= 0) {
                ks_next = a.c.d_k_scale[(long long)id_next * H + h];
                vs_next = a.c.d_v_scale[(long long)id_next * H + h];
            }
            const int id_then = __shfl_sync(0xffffffffu, id_now, slot);
            const float ks_then = __shfl_sync(0xffffffffu, ks_now, slot), vs_then = __shfl_sync(0xffffffffu, vs_now, slot);
            if (nt < tiles) load_k(id_then, tok + kUnit);

            // ---- softmax against a lagging reference
            bool above = false;
            const bool edge = tok + 16 > seen_first || id < 0;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[t][e] *= factor[t][e & 1] * ks;
                    if (edge && (id < 0 || tok + lr + (e >> 1) * 8 >= limit[t][e & 1])) s[t][e] = -INFINITY;
                    above |= s[t][e] > ref[t][e & 1] + 15.f;
                }
            if (__any_sync(0xffffffffu, above)) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float m = fmaxf(s[t][e], s[t][e + 2]);
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16)) - 7.f;
                        if (m > ref[t][e]) {
                            const float f = exp2_fast(ref[t][e] - m);
                            ref[t][e] = m;
                            sum[t][e] *= f;
#pragma unroll
                            for (int i = 0; i < MT; ++i) { o[t][i][e] *= f; o[t][i][e + 2] *= f; }
                        }
                    }
            }
            if (vs > vref && vs >= 7.888609052210118e-31f) {
                const float f = vref / vs;
                vref = vs;
                vref_inverse = 1.f / vs;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[t][i][e] *= f;
            }
            const float vf = vs * vref_inverse;
            uint32_t pf[NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = exp2_fast(s[t][e] - (ref[t][e & 1] == -INFINITY ? 0.f : ref[t][e & 1]));
                    sum[t][e & 1] += p[e];
                }
                pf[t][0] = transposed(pack_half2(p[0] * vf, p[1] * vf));
                pf[t][1] = transposed(pack_half2(p[2] * vf, p[3] * vf));
            }
            // ---- values: what lies past the request's length may be a NaN pattern
            if (FMT == FLUXBIN_CACHE_E4M3 && tok + 16 > rq.length) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (tok + 2 * lq + (i & 1) + (i >> 1) * 8 >= rq.length)
#pragma unroll
                        for (int c = 0; c < VC; ++c) vw[i][c] = Words<VW>{};
            }
#pragma unroll
            for (int c = 0; c < VC; ++c)
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    uint32_t f[2][4];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {            // tokens 2q, 2q + 1, then 2q + 8, 2q + 9
                        const uint32_t x = vw[2 * i][c].w[w], y = vw[2 * i + 1][c].w[w];
                        to_half4<FMT>(__byte_perm(x, y, 0x5140), f[i][0], f[i][1]);
                        to_half4<FMT>(__byte_perm(x, y, 0x7362), f[i][2], f[i][3]);
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        mma(o[t][(c * VW + w) * 2], f[0][0], f[0][1], f[1][0], f[1][1], pf[t][0], pf[t][1]);
                        mma(o[t][(c * VW + w) * 2 + 1], f[0][2], f[0][3], f[1][2], f[1][3], pf[t][0], pf[t][1]);
                    }
                }
            if (nt < tiles) load_v(id_then, tok + kUnit);
            id = id_then;
            ks = ks_then;
            vs = vs_then;
        }

        // ---- the warps' results, then one for the CTA
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float l = sum[t][e];
                l += __shfl_xor_sync(0xffffffffu, l, 4);
                l += __shfl_xor_sync(0xffffffffu, l, 8);
                l += __shfl_xor_sync(0xffffffffu, l, 16);
                const int row = t * 8 + 2 * lq + e;
                if (lr == 0) { sm.m[warp][row] = ref[t][e]; sm.l[warp][row] = l; }
#pragma unroll
                for (int c = 0; c < VC; ++c)
#pragma unroll
                    for (int i = 0; i < VW * 2; i += 2)
                        *reinterpret_cast<float4 *>(&sm.o[warp][row][c * VW * 32 + lr * VW * 4 + i * 2]) =
                            make_float4(o[t][c * VW * 2 + i][e], o[t][c * VW * 2 + i][e + 2], o[t][c * VW * 2 + i + 1][e], o[t][c * VW * 2 + i + 1][e + 2]);
            }
        if (lane == 0) sm.v[warp] = vref;
        __syncthreads();
        const bool whole = p0 == 0 && p1 == rq.pieces;
        const int first_cta_slot = p0 == 0;                  // this job begins here, or goes on from the CTA before
        float *part = a.partial + ((long long)blockIdx.x * 2 + first_cta_slot) * ROWS * D;
        float *part_lse = a.partial + (long long)kMaxGrid * 2 * kMaxRows * D + ((long long)blockIdx.x * 2 + first_cta_slot) * kMaxRows;
        auto write_out = [&](int row, int d, float4 v, float lse2) {
            const int g = row0 + row;
            const long long tok = rq.first + g / G;
            const int head = h * G + g % G;
            T *op = (T *)a.out + tok * a.out_token + head * a.out_head + d;
            T e[4] = {from_float<T>(v.x), from_float<T>(v.y), from_float<T>(v.z), from_float<T>(v.w)};
            *reinterpret_cast<uint2 *>(op) = *reinterpret_cast<const uint2 *>(e);
            if (d == 0 && a.lse) a.lse[tok * a.q_heads + head] = lse2 * 0.6931471805599453f;
        };
        for (int i = tid; i < ROWS * (D / 4); i += kThreads) {
            const int row = i / (D / 4), d = i % (D / 4) * 4;
            float m = -INFINITY, l = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) m = fmaxf(m, sm.m[w][row]);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            const float m_safe = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {           // a warp without tokens has l = 0; a NaN in l stays
                const float f = sm.l[w][row] == 0.f ? 0.f : exp2_fast(sm.m[w][row] - m_safe), fv = f * sm.v[w];
                const float4 x = *reinterpret_cast<const float4 *>(&sm.o[w][row][d]);
                l += f * sm.l[w][row];
                if (f != 0.f) { v.x += fv * x.x; v.y += fv * x.y; v.z += fv * x.z; v.w += fv * x.w; }
            }
            const float inv = l == 0.f ? 0.f : 1.f / l, lse2 = l == 0.f ? -INFINITY : m + log2f(l);
            v.x *= inv; v.y *= inv; v.z *= inv; v.w *= inv;
            if (whole) {
                if (row < rows) write_out(row, d, v, lse2);
            } else {
                *reinterpret_cast<float4 *>(part + row * D + d) = v;
                if (d == 0) part_lse[row] = lse2;
            }
        }
        if (!whole) {
            // the CTAs that hold parts of this job, by the cut of the line
            const long long job_begin = u - p0, job_end = job_begin + rq.pieces;
            auto owner = [&](long long x) {
                long long i = x * shares / total;
                while (cut(i + 1) <= x) ++i;
                while (cut(i) > x) --i;
                return (int)i;
            };
            const int c0 = owner(job_begin), c1 = owner(job_end - 1);
            __threadfence();
            __syncthreads();
            if (tid == 0) sm.last = atomicAdd(&a.arrived[c0], 1u) == (unsigned)(c1 - c0);
            __syncthreads();
            if (sm.last) {
                __threadfence();
                const float *lses = a.partial + (long long)kMaxGrid * 2 * kMaxRows * D;
                auto slot_of = [&](int c) { return (long long)c * 2 + (c == c0); };
                for (int i = tid; i < ROWS * (D / 4); i += kThreads) {
                    const int row = i / (D / 4), d = i % (D / 4) * 4;
                    if (row >= rows) continue;
                    float m = -INFINITY, l = 0.f;
                    for (int c = c0; c <= c1; ++c) m = fmaxf(m, __ldcg(lses + slot_of(c) * kMaxRows + row));
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
                    for (int c = c0; c <= c1; ++c) {
                        const float x = __ldcg(lses + slot_of(c) * kMaxRows + row), f = x == -INFINITY ? 0.f : exp2_fast(x - m);
                        const float4 y = __ldcg(reinterpret_cast<const float4 *>(a.partial + slot_of(c) * ROWS * D + row * D + d));
                        l += f;
                        v.x += f * y.x; v.y += f * y.y; v.z += f * y.z; v.w += f * y.w;
                    }
                    const float inv = l == 0.f ? 0.f : 1.f / l;
                    write_out(row, d, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv), l == 0.f ? -INFINITY : m + log2f(l));
                }
                if (tid == 0) a.arrived[c0] = 0;
            }
        }
        __syncthreads();                          // the shared arrays are free again
        u += p1 - p0;
    }
}

int num_sms()
{
    static std::atomic<int> of[fb::kMaxDevices];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= fb::kMaxDevices) return 0;
    int n = of[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
        of[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

template <int D, int FMT, int NT, typename T>
cudaError_t run(const Args &a, cudaStream_t s)
{
    const size_t smem = sizeof(Shared<D, 8 * NT>);
    static std::atomic<bool> opted[fb::kMaxDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= fb::kMaxDevices) return cudaErrorInvalidDevice;
    if (!opted[dev].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(attend_kernel<D, FMT, NT, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        opted[dev].store(true, std::memory_order_relaxed);
    }
    const int sms = num_sms();
    if (sms == 0) return cudaErrorInvalidDevice;
    const int grid = sms * (D == 256 || NT == 2 ? 1 : 2);
    return launch(attend_kernel<D, FMT, NT, T>, dim3((unsigned)(grid < kMaxGrid ? grid : kMaxGrid)), kThreads, smem, s, a);
}
template <int D, int FMT, typename T> cudaError_t run_rows(const Args &a, cudaStream_t s)
{
    // rows that share a key head in an average request
    const long long rows = (long long)(a.q_heads / a.c.kv_heads) * ((a.tokens + a.batch - 1) / a.batch);
    if constexpr (D != 256) {
        if (rows > 8) return run<D, FMT, 2, T>(a, s);
    }
    return run<D, FMT, 1, T>(a, s);
}
template <int D, typename T> cudaError_t run_format(const Args &a, cudaStream_t s)
{
    return a.c.format == FLUXBIN_CACHE_INT8 ? run_rows<D, FLUXBIN_CACHE_INT8, T>(a, s) : run_rows<D, FLUXBIN_CACHE_E4M3, T>(a, s);
}
template <typename T> cudaError_t run_dim(const Args &a, cudaStream_t s)
{
    return a.c.head_dim == 64 ? run_format<64, T>(a, s) : a.c.head_dim == 128 ? run_format<128, T>(a, s) : run_format<256, T>(a, s);
}

constexpr size_t kCounterBytes = (kMaxGrid * sizeof(unsigned) + 255) / 256 * 256;

} // namespace

extern "C" size_t fluxbin_kv_attend_workspace_size(int32_t batch, int32_t tokens, int32_t q_heads, int32_t kv_heads, int32_t head_dim)
{
    if (batch < 1 || tokens < 0 || q_heads < 1 || kv_heads < 1 || q_heads % kv_heads != 0 || head_dim < 1) return 0;
    return kCounterBytes + (size_t)kMaxGrid * 2 * kMaxRows * (head_dim + 1) * sizeof(float);
}

extern "C" fluxbin_status_t fluxbin_kv_attend(const fluxbin_kv_cache_t *cache, int32_t dtype, int32_t batch, int32_t tokens,
                                              const void *d_q, int32_t q_heads, int64_t q_token, int64_t q_head,
                                              const int32_t *d_query_start, const int32_t *d_lengths,
                                              const int32_t *d_block_table, int64_t block_table_stride, int32_t block_table_width,
                                              float scale, void *d_out, int64_t out_token, int64_t out_head, float *d_lse,
                                              void *d_workspace, size_t ws_bytes, void *cuda_stream)
{
    const fluxbin_status_t st = check_cache(cache);
    if (st != FLUXBIN_OK) return st;
    if (dtype != FLUXBIN_TYPE_FP16 && dtype != FLUXBIN_TYPE_BF16) return FLUXBIN_ERR_UNSUPPORTED;
    if (batch < 1 || tokens < 0 || q_heads < 1 || q_heads > 65535 || q_heads % cache->kv_heads != 0 || block_table_width < 1 ||
        block_table_stride < block_table_width || (!d_query_start && tokens != batch)) return FLUXBIN_ERR_RANGE;
    if (tokens == 0) return FLUXBIN_OK;
    if (!d_q || !d_out || !d_lengths || !d_block_table || !d_workspace) return FLUXBIN_ERR_NULL;
    if (!aligned_to(d_q, 16) || !aligned_to(d_out, 16) || q_token % 8 || q_head % 8 || out_token % 8 || out_head % 8 ||
        !aligned_to(d_query_start, 4) || !aligned_to(d_lengths, 4) || !aligned_to(d_block_table, 4) || !aligned_to(d_lse, 4) ||
        !aligned_to(d_workspace, 16)) return FLUXBIN_ERR_ALIGNMENT;
    if (ws_bytes < fluxbin_kv_attend_workspace_size(batch, tokens, q_heads, cache->kv_heads, cache->head_dim)) return FLUXBIN_ERR_BUFFER_TOO_SMALL;
    const Args a = {*cache, batch, tokens, q_heads, block_table_width, d_q, q_token, q_head, d_query_start, d_lengths, d_block_table,
                    block_table_stride, scale, d_out, out_token, out_head, d_lse,
                    (unsigned *)d_workspace, (float *)((char *)d_workspace + kCounterBytes), 1};
    cudaStream_t s = (cudaStream_t)cuda_stream;
    FBD_CUDA(dtype == FLUXBIN_TYPE_FP16 ? run_dim<__half>(a, s) : run_dim<__nv_bfloat16>(a, s));
    return FLUXBIN_OK;
}
