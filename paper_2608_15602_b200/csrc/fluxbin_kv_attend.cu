// Attention of new tokens over the 8-bit block-paged cache (fluxbin_kv_attend).
//
// For one key head and a group of query rows (the query heads that share it, over the request's new tokens) the kernel
// forms, 16 cached tokens at a time,
//     S^T = K Q^T  [16 tokens x rows],   P = exp2(S c - m),   O^T += V^T P^T  [dim x rows],   l += sum P
// with the tokens (then the elements of a head) as the 16-row side of the matrix instruction and the query rows as its
// 8-column side: a decode step has as few rows as query heads share a key head, and 8 columns waste the least.  (The
// instructions that accumulate outside the registers take 64 tokens or more a step, from operands of 16 bits in shared
// memory: the 8-bit cache would have to be converted there and back again for 8 columns.)
//
// What bounds it is the cache's bytes.  Each lane copies (cp.async) the 16-byte pieces that it will hold as matrix operands
// into its own places of a ring in shared memory, a few tiles ahead, and takes them from there itself: no barrier, no bank
// conflict, no shuffle.  Which element a lane's operand slot stands for is free as long as both operands agree, so a lane
// takes 16 consecutive bytes wherever the instruction would want scattered pairs.
//   keys:    lane (r, q) = (lane / 4, lane % 4) reads elements 16 q .. + 15 of each 64-byte piece of tokens r and r + 8
//   values:  the same lane reads elements 16 r .. + 15 (of 128) of tokens 2q, 2q + 1, 2q + 8, 2q + 9 and interleaves the
//            bytes of two tokens, which the conversion to bf16 does on the way
// P leaves the first product with a lane per token and enters the second with a lane per row: movmatrix turns it.
// 8-bit entries are exact in fp16 and in bf16.  The block's key scale multiplies the score in fp32.  A probability times its
// block's value scale (over the largest one met so far, vref) is the sum of two bf16 operands, the second of which rounds what
// the first left: 2^-16 of it is lost, and nothing is flushed to zero short of fp32's own range, so a result does not suffer
// where small probabilities or blocks of small values decide it.  (One fp16 operand: 2^-11 lost, and all of it 2^-31 below the
// largest.  With two products in the place of one 8 rows of 128 take 1 to 2 % more time, 16 rows 2 to 11 %, 40 rows 11 %.)
// The reference m lags: it is raised to (row maximum - 7) only when a P would pass 2^15, so that most steps need no reduction
// over lanes.
//
// Work is cut evenly whatever the lengths are: all (request, head, rows) jobs in units of cached tokens form a line, which is
// cut into a range for each CTA (the lengths are read on the device: a captured graph serves every step).  A job cut between
// CTAs leaves normalised partial results and their lse in the workspace; the CTA that arrives last joins them in order.
#include "fluxbin_cache.cuh"

#include <atomic>

using namespace fbd;

namespace {

// Warps of a CTA, CTAs on an SM, tiles of 16 tokens that a warp has under way, whether the queries stay in shared memory (the
// output takes the registers), by head dimension and tiles of 8 query rows.  Measured, as the figures below up to kTailMin, while
// the probabilities were one operand of the second product: at 128 with 8 rows on 64 requests of up
// to 16384 tokens: 4 x 3 with 4 tiles 242 us, 8 x 2 with 3 249, 6 x 2 with 4 257, 4 x 4 with 3 (128 registers, spills) 277, 12 x
// 1 with 4 288: small CTAs, so that the others go on while one ends a job, and tiles on their way rather than warps.  With 16
// rows on 16 requests of up to 8190: 4 x 2 64 us, 8 x 1 74.  40 rows are as many as the registers take.
template <int D, int NT> struct Shape;
template <> struct Shape<64, 1> { static constexpr int warps = 8, ctas = 2, stages = 6; static constexpr bool shared_queries = false; };
template <> struct Shape<64, 2> { static constexpr int warps = 8, ctas = 2, stages = 6; static constexpr bool shared_queries = false; };
template <> struct Shape<128, 1> { static constexpr int warps = 4, ctas = 3, stages = 4; static constexpr bool shared_queries = false; };
template <> struct Shape<128, 2> { static constexpr int warps = 4, ctas = 2, stages = 6; static constexpr bool shared_queries = false; };
template <> struct Shape<128, 5> { static constexpr int warps = 8, ctas = 1, stages = 5; static constexpr bool shared_queries = true; };
template <> struct Shape<256, 1> { static constexpr int warps = 8, ctas = 1, stages = 3; static constexpr bool shared_queries = false; };
template <> struct Shape<256, 2> { static constexpr int warps = 8, ctas = 1, stages = 3; static constexpr bool shared_queries = true; };

// Units that it costs to begin a job (the chain from the block table to the first tile, the ring that runs dry, the warps'
// results put together): CTAs that cross from job to job get fewer tokens.  Units are 64 tokens with 4 warps.  Measured 0 / 2 /
// 4 / 6 / 9: 36.7 / 35.2 / 33.9 / 33.0 / 33.4 us on 16 requests, 64.8 / 58.0 / 56.8 / 56.8 / 59.1 on 8 with 40 key heads.
constexpr int kJobCost = 6;

// The part of a range that is drawn, and the units that it has to have: below that the further partial results cost more
// than the evener end gives.  10 % of 156 units: 240 -> 226 us; of 37 units (one request of 131071 tokens): 74 -> 86 us.
constexpr int kTailPercent = 10, kTailMin = 8;
constexpr int kMaxLength = INT32_MAX - 4095;    // rounded up to units it is still an int
constexpr float kNoRef = -3e38f;                // the reference before the first score: below every one, and finite
constexpr int kMaxSms = 160, kMaxShares = kMaxSms * 3 * 2;

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
    unsigned *drawn;                            // shares drawn so far
    unsigned *arrived;                          // [kMaxShares], by the share in which a cut job begins
    float *partial_lse;                         // [shares][2][rows], base 2
    float *partial;                             // [shares][2][rows][D]
};

// ---- conversions of 8-bit entries ------------------------------------------------------------------------

// bf16 rows of queries become fp16, multiplied by the power of two that takes their largest element to 2^14 .. 2^15: exactly
// down to 2^-31 of that element, what is smaller to 2^-39 of it (fp16's smallest steps)
__device__ __forceinline__ int exponent_of(float largest) { return largest > 0.f ? min(max((int)(__float_as_uint(largest) >> 23), 1), 254) - 127 - 14 : 0; }
__device__ __forceinline__ uint32_t half2_of_bf16(uint32_t w, int e)
{
    const __half2 h = __floats2half2_rn(ldexpf(__uint_as_float(w << 16), -e), ldexpf(__uint_as_float(w & 0xffff0000u), -e));
    return *reinterpret_cast<const uint32_t *>(&h);
}

// four entries of a key to two pairs of fp16
template <int FMT> __device__ __forceinline__ void to_half4(uint32_t x, uint32_t &lo, uint32_t &hi);
// int8: the byte with its sign bit flipped, under the exponent of 1024, is 1024 + 128 + value; fp16 holds that exactly (the
// conversion of Kim, Henry, Fahim and Awadalla, "Who Says Elephants Can't Run", 2022)
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

// four entries of two tokens' values to four pairs (x, y) of bf16, as parts 1 / kPart of them
template <int FMT> constexpr float kPart = FMT == FLUXBIN_CACHE_INT8 ? 64.f : 1.f;
template <int FMT> __device__ __forceinline__ void to_bfloat2x4(uint32_t x, uint32_t y, uint32_t (&pair)[4]);
__device__ __forceinline__ uint32_t bfloat2_of_half2(__half2 h)      // exact for 8-bit entries
{
    const float2 f = __half22float2(h);
    const __nv_bfloat162 r = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t *>(&r);
}
// int8: the byte with its sign bit flipped, u = 128 + value, is as a bf16 pattern u * 2^-133 (the smallest numbers and the
// first normal ones have one step); times 2^127, less 128 * 2^-6, that is value * 2^-6 exactly
template <> __device__ __forceinline__ void to_bfloat2x4<FLUXBIN_CACHE_INT8>(uint32_t x, uint32_t y, uint32_t (&pair)[4])
{
    x ^= 0x80808080u;
    y ^= 0x80808080u;
    const __nv_bfloat162 up = __bfloat162bfloat162(__ushort_as_bfloat16(0x7f00)), down = __bfloat162bfloat162(__ushort_as_bfloat16(0xc000));     // 2^127, -2
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const uint32_t z = __byte_perm(x, y, i ? 0x7362 : 0x5140);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t u = __byte_perm(z, 0, k ? 0x4342 : 0x4140);
            const __nv_bfloat162 r = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&u), up, down);
            pair[i + k] = *reinterpret_cast<const uint32_t *>(&r);
        }
    }
}
// e4m3: by way of fp16 and fp32, both exact (a NaN stays one)
template <> __device__ __forceinline__ void to_bfloat2x4<FLUXBIN_CACHE_E4M3>(uint32_t x, uint32_t y, uint32_t (&pair)[4])
{
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        uint32_t h[2];
        to_half4<FLUXBIN_CACHE_E4M3>(__byte_perm(x, y, i ? 0x7362 : 0x5140), h[0], h[1]);
#pragma unroll
        for (int k = 0; k < 2; ++k) pair[i + k] = bfloat2_of_half2(*reinterpret_cast<const __half2 *>(&h[k]));
    }
}

// the top bits of the bytes that are e4m3 NaN
__device__ __forceinline__ uint32_t nan_bytes(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&x)[4], const uint32_t (&y)[4], int i, const uint32_t (&b)[2])
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(x[i]), "r"(x[i + 1]), "r"(y[i]), "r"(y[i + 1]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ uint32_t transposed(uint32_t v)
{
    uint32_t t;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(t) : "r"(v));
    return t;
}
// two values as bf16, and what that rounding left of them as another two
__device__ __forceinline__ void split_bfloat2(float x, float y, uint32_t &upper, uint32_t &rest)
{
    const __nv_bfloat162 u = __floats2bfloat162_rn(x, y);
    upper = *reinterpret_cast<const uint32_t *>(&u);
    const __nv_bfloat162 r = __floats2bfloat162_rn(x - __uint_as_float(upper << 16), y - __uint_as_float(upper & 0xffff0000u));
    rest = *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ float exp2_fast(float x)         // relative error 2^-22, exp2(-inf) = 0
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Copies from the cache into a lane's own places of the ring, past L1 (the cache is read once).  A lane reads back only
// what it copied itself, so its own wait is all the order that is needed.
template <int N> __device__ __forceinline__ void copy_ahead(uint32_t to, const unsigned char *from)
{
    if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }
template <int N> struct Words { uint32_t w[N]; };
template <int N> __device__ __forceinline__ Words<N> take(uint32_t from)
{
    Words<N> v;
    if constexpr (N == 4)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]) : "r"(from) : "memory");
    else
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.w[0]), "=r"(v.w[1]) : "r"(from) : "memory");
    return v;
}

// ---- the line of work -----------------------------------------------------------------------------------

struct Request {
    int first, count;            // its new tokens
    int length;                  // its cached tokens
    int row_tiles, pieces;       // tiles of query rows a head has, units of cached tokens
};
template <int ROWS, int kUnit> __device__ __forceinline__ Request request_of(const Args &a, int r)
{
    Request q;
    if (a.query_start) {
        q.first = min(max(a.query_start[r], 0), a.tokens);
        q.count = max(min(max(a.query_start[r + 1], 0), a.tokens) - q.first, 0);
    } else {
        q.first = r;
        q.count = 1;
    }
    q.length = (int)min((long long)min(max(a.lengths[r], 0), kMaxLength), (long long)a.width * a.c.block_tokens);
    q.row_tiles = (int)(((long long)q.count * (a.q_heads / a.c.kv_heads) + ROWS - 1) / ROWS);
    q.pieces = max((q.length + kUnit - 1) / kUnit, 1);          // an empty request still has rows to write
    return q;
}
__device__ __forceinline__ long long units_of(const Args &a, const Request &q) { return (long long)q.row_tiles * a.c.kv_heads * (q.pieces + kJobCost); }

template <int D, int ROWS, int WARPS, int STAGES, bool QSHARED> struct Shared {
    static constexpr int kTile = 32 * D;            // 16 tokens of keys and of values
    union {
        unsigned char ring[WARPS][STAGES][kTile];
        struct {                                    // after a job: the warps' results
            float o[WARPS][ROWS][D + 4];
            float m[WARPS][ROWS], l[WARPS][ROWS], v[WARPS];
        };
        struct { float join_max[ROWS], join_inv[ROWS], join_lse[ROWS]; };       // after the last part of a cut job
    };
    uint2 q[QSHARED ? ROWS / 8 : 1][D / 16][32];         // the queries as operands, by lane
    float factor[ROWS];
    long long scan[WARPS], before;
    int request, last, share, any_nan;
    uint32_t nan[ROWS][D / 32];                          // elements of this job's rows that see a NaN (see hide_nan)
};

// the rows of tokens that are no request's
template <int D, typename T> __device__ __noinline__ void empty_rows(const Args &a, int tid, int threads)
{
    const int from = min(max(a.query_start[0], 0), a.tokens), to = min(max(a.query_start[a.batch], from), a.tokens), n = a.tokens - (to - from);
    if (n == 0) return;
    for (long long i = (long long)blockIdx.x * threads + tid; i < (long long)n * a.q_heads * (D / 4); i += (long long)gridDim.x * threads) {
        const int row = (int)(i / (D / 4)), nth = row / a.q_heads, h = row % a.q_heads, d = (int)(i % (D / 4)) * 4;
        const long long t = nth < from ? nth : nth + (to - from);
        *reinterpret_cast<uint2 *>((T *)a.out + t * a.out_token + h * a.out_head + d) = make_uint2(0, 0);
        if (d == 0 && a.lse) a.lse[t * a.q_heads + h] = -INFINITY;
    }
}

// one CTA: its part of the line, job after job
template <int D, int FMT, int NT, typename T>
__global__ void __launch_bounds__(Shape<D, NT>::warps * 32, Shape<D, NT>::ctas) attend_kernel(const __grid_constant__ Args a)
{
    constexpr int ROWS = 8 * NT;
    constexpr int kWarps = Shape<D, NT>::warps, kThreads = kWarps * 32;
    constexpr int STAGES = Shape<D, NT>::stages;
    constexpr int kUnit = kWarps * 16;           // cached tokens of a unit: 16 for each warp
    constexpr bool QSHARED = Shape<D, NT>::shared_queries;
    constexpr int KC = D / 64;                   // 64-byte pieces of a key
    constexpr int VW = D >= 128 ? 4 : 2;         // words of a load of values
    constexpr int VC = D / (VW * 32);            // pieces of a value row (eight lanes of VW words each)
    constexpr int MT = D / 16;                   // 16-element tiles of the output
    extern __shared__ __align__(16) unsigned char smem_raw[];
    Shared<D, ROWS, kWarps, STAGES, QSHARED> &sm = *reinterpret_cast<Shared<D, ROWS, kWarps, STAGES, QSHARED> *>(smem_raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, lr = lane >> 2, lq = lane & 3;
    const int H = a.c.kv_heads, G = a.q_heads / H, bs = a.c.block_tokens;

    let_successor_start();
    wait_for_predecessor();

    if (a.query_start) empty_rows<D, T>(a, tid, kThreads);

    // ---- where this CTA's part begins: a sum over the requests, each thread over a run of them
    const int per = (a.batch + kThreads - 1) / kThreads, r_lo = min(tid * per, a.batch), r_hi = min(r_lo + per, a.batch);
    long long mine = 0;
    for (int r = r_lo; r < r_hi; ++r) mine += units_of(a, request_of<ROWS, kUnit>(a, r));
    long long upto = mine;
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    if (lane == 31) sm.scan[warp] = upto;
    for (int i = tid; i < ROWS * (D / 32); i += kThreads) sm.nan[i / (D / 32)][i % (D / 32)] = 0;
    if (tid == 0) sm.any_nan = 0;
    __syncthreads();
    long long total = 0;
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) upto += sm.scan[w];
        total += sm.scan[w];
    }
    const long long active = min((long long)gridDim.x, total);
    if (blockIdx.x >= active) return;
    // A range of the line for each CTA.  Of long ranges the last part is a share of its own, drawn by whoever is through
    // with the first part of its own range, since SMs do not all get the same part of the memory's rate.  The cuts depend
    // on the line alone, so results do not depend on who drew what.  Shares are numbered along the line.
    const long long tail = total / active * kTailPercent / 100, extra = tail >= kTailMin ? active : 0;
    const long long size = total / active, over = total - size * active;
    auto cut = [&](long long i) {
        if (extra == 0) return i * size + min(i, over);
        const long long at = (i + 1) / 2 * size + min((i + 1) / 2, over);
        return i & 1 ? at - tail : at;
    };
    auto owner = [&](long long x) {
        const int i = (int)(x < over * (size + 1) ? x / (size + 1) : over + (x - over * (size + 1)) / size);
        return extra == 0 ? i : 2 * i + (x >= cut(2 * i + 1));
    };

    for (long long share = extra ? 2 * blockIdx.x : blockIdx.x;;) {
    long long u = cut(share);
    const long long u_end = cut(share + 1);
    if (u >= upto - mine && u < upto) {
        long long before = upto - mine;
        for (int r = r_lo; r < r_hi; ++r) {
            const long long n = units_of(a, request_of<ROWS, kUnit>(a, r));
            if (u < before + n) { sm.request = r; sm.before = before; break; }
            before += n;
        }
    }
    __syncthreads();
    int r = sm.request;
    long long r_before = sm.before;
    Request rq = request_of<ROWS, kUnit>(a, r);

    while (u < u_end) {
        while (u >= r_before + units_of(a, rq)) {
            r_before += units_of(a, rq);
            rq = request_of<ROWS, kUnit>(a, ++r);
        }
        // a job is kJobCost places for what it costs to begin it, then its pieces
        const int span = rq.pieces + kJobCost, job = (int)((u - r_before) / span);
        const long long job_begin = r_before + (long long)job * span;
        const int p0 = max((int)(u - job_begin) - kJobCost, 0);
        const int p1 = (int)min(u_end - job_begin, (long long)span) - kJobCost;
        u = min(u_end, job_begin + span);
        if (p1 <= p0) continue;
        const int h = job / rq.row_tiles, row0 = job % rq.row_tiles * ROWS;
        const int rows = (int)min((long long)ROWS, (long long)rq.count * G - row0);
        // tokens that the last and the first row of the tile see
        const int seen = rq.length - (rq.count - 1 - (row0 + rows - 1) / G);
        const int seen_first = rq.length - (rq.count - 1 - row0 / G);
        auto limit = [&](int t, int e) { return rq.length - (rq.count - 1 - min(row0 + t * 8 + 2 * lq + e, row0 + rows - 1) / G); };

        // ---- the places and scales of this warp's tiles: lane i holds those of tile i of a batch of 32
        const int tok0 = p0 * kUnit + warp * 16;
        const int tiles = max((min(seen, p1 * kUnit) - tok0 + kUnit - 1) / kUnit, 0);
        const int *row_table = a.table + r * a.table_stride;
        // (a tile of 16 tokens lies in one block): where they begin in the cache, -1 for a block that is none
        struct Place { long long at; float ks, vs; };
        auto block_of = [&](int tile) {
            if (tile >= tiles) return -1;
            const int id = row_table[(tok0 + tile * kUnit) / bs];
            return id >= 0 && id < a.c.num_blocks ? id : -1;
        };
        auto place_of = [&](int id, int tile) {
            Place x = {-1, 0.f, 0.f};
            if (id >= 0) {
                x.at = id * a.c.block_stride + (tok0 + tile * kUnit) % bs * a.c.token_stride;
                x.ks = a.c.d_k_scale[(long long)id * H + h];
                x.vs = a.c.d_v_scale[(long long)id * H + h];
            }
            return x;
        };
        Place now = place_of(block_of(lane), lane), next = {-1, 0.f, 0.f};
        int id_next = tiles > 32 ? block_of(32 + lane) : -1;

        // ---- the ring: where a lane's pieces of a tile lie, and their way there
        const long long ts = a.c.token_stride;
        const unsigned char *k_lane = (const unsigned char *)a.c.d_k + h * a.c.head_stride + lr * ts + lq * 16;
        const unsigned char *v_lane = (const unsigned char *)a.c.d_v + h * a.c.head_stride + 2 * lq * ts + lr * (VW * 4);
        const uint32_t k_ring = (uint32_t)__cvta_generic_to_shared(&sm.ring[warp][0][lane * 16]);
        const uint32_t v_ring = (uint32_t)__cvta_generic_to_shared(&sm.ring[warp][0][16 * D + lane * (VW * 4)]);
        // a block that is none reads the cache's first one instead (and is masked out)
        auto fetch = [&](long long at, int stage) {
            const unsigned char *kp = k_lane + max(at, 0ll), *vp = v_lane + max(at, 0ll);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int c = 0; c < KC; ++c) copy_ahead<16>(k_ring + stage * (32 * D) + (i * KC + c) * 512, kp + i * 8 * ts + c * 64);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < VC; ++c)
                    copy_ahead<VW * 4>(v_ring + stage * (32 * D) + (i * VC + c) * (VW * 128), vp + ((i & 1) + (i >> 1) * 8) * ts + c * (VW * 32));
        };
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i) {
            const long long at = __shfl_sync(0xffffffffu, now.at, i);
            if (i < tiles) fetch(at, i);
            copies_commit();
        }

        // ---- the query rows as the 8-column operand: lane (r, q) holds row r, 16 elements of each 64-element piece
        uint32_t qf[QSHARED ? 1 : NT][KC * 4][2];
        float factor[QSHARED ? 1 : NT][2];
        if constexpr (QSHARED) {
            // a warp takes every kWarps-th row, a lane four elements at a time
            for (int row = warp; row < ROWS; row += kWarps) {
                const bool live = row < rows;
                const int g = row0 + (live ? row : 0);
                const T *qp = (const T *)a.q + (rq.first + g / G) * a.q_token + (h * G + g % G) * a.q_head;
                uint2 w[(D + 127) / 128];
                float largest = 0.f;
#pragma unroll
                for (int i = 0; i < (D + 127) / 128; ++i) {
                    w[i] = live && i * 128 + lane * 4 < D ? *reinterpret_cast<const uint2 *>(qp + i * 128 + lane * 4) : make_uint2(0, 0);
                    if constexpr (!std::is_same<T, __half>::value)
                        largest = fmaxf(largest, fmaxf(fmaxf(fabsf(__uint_as_float(w[i].x << 16)), fabsf(__uint_as_float(w[i].x & 0xffff0000u))),
                                                       fmaxf(fabsf(__uint_as_float(w[i].y << 16)), fabsf(__uint_as_float(w[i].y & 0xffff0000u)))));
                }
                float f = a.scale * 1.4426950408889634f;
                if constexpr (!std::is_same<T, __half>::value) {
#pragma unroll
                    for (int x = 16; x; x >>= 1) largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, x));
                    const int e = exponent_of(largest);
#pragma unroll
                    for (int i = 0; i < (D + 127) / 128; ++i) w[i] = make_uint2(half2_of_bf16(w[i].x, e), half2_of_bf16(w[i].y, e));
                    f = ldexpf(f, e);
                }
#pragma unroll
                for (int i = 0; i < (D + 127) / 128; ++i) {
                    const int d = i * 128 + lane * 4;
                    if (d < D) sm.q[row / 8][d / 64 * 4 + d % 16 / 4][row % 8 * 4 + d % 64 / 16] = w[i];
                }
                if (lane == 0) sm.factor[row] = f;
            }
            __syncthreads();
        } else {
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
                largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, 1));
                largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, 2));
                const int e = exponent_of(largest);
#pragma unroll
                for (int i = 0; i < KC * 4; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k) qf[t][i][k] = half2_of_bf16(qf[t][i][k], e);
                f = ldexpf(a.scale * 1.4426950408889634f, e);
            } else {
                f = a.scale * 1.4426950408889634f;
            }
            // the factor of a row is wanted by the lanes that hold its column
#pragma unroll
            for (int e = 0; e < 2; ++e) factor[t][e] = __shfl_sync(0xffffffffu, f, (2 * lq + e) * 4);
        }
        }

        float o[NT][MT][4], ref[NT][2], sum[NT][2], vref = 0.f, vref_inverse = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < MT; ++i) o[t][i][0] = o[t][i][1] = o[t][i][2] = o[t][i][3] = 0.f;
            ref[t][0] = ref[t][1] = kNoRef;
            sum[t][0] = sum[t][1] = 0.f;
        }

        // On tiles that not all rows see to their end: what must not meet the probability 0 of a row that does not see its token
        // is taken out of the values, and noted for the rows that do.  Each lane looks through its own places of the ring.
        //   values past the request's length, or in no block of its own (e4m3: may be NaN patterns): become 0
        //   a NaN entry of a new token: becomes 0; its element is NaN in every row that sees the token
        //   a scale that is no number: the caller takes 0 for it; all elements are NaN in every row that sees a token of the tile
        auto hide_nan = [&](int tok, int stage, bool none, float vs) {
            auto sees = [&](int row) { return rq.length - (rq.count - 1 - (row0 + row) / G); };
            if (!(vs < INFINITY)) {
                for (int row = lane; row < rows; row += 32)
                    if (tok < sees(row)) {
                        for (int d = 0; d < D / 32; ++d) atomicOr(&sm.nan[row][d], 0xffffffffu);
                        sm.any_nan = 1;
                    }
            }
            if constexpr (FMT == FLUXBIN_CACHE_E4M3) {
#pragma unroll 1
                for (int part = 0; part < 4 * VC; ++part) {
                    const int token = tok + 2 * lq + (part / VC & 1) + (part / VC >> 1) * 8;
                    const uint32_t at = v_ring + stage * (32 * D) + part * (VW * 128);
                    Words<VW> x = take<VW>(at);
                    uint32_t any = 0;
#pragma unroll
                    for (int w = 0; w < VW; ++w) any |= nan_bytes(x.w[w]);
                    if (none || token >= rq.length) x = Words<VW>{};
                    else if (any == 0) continue;
#pragma unroll
                    for (int w = 0; w < VW; ++w) {
                        uint32_t nan = nan_bytes(x.w[w]);
                        x.w[w] &= ~(nan | (nan - (nan >> 7)));
                        asm volatile("st.shared.u32 [%0], %1;" ::"r"(at + w * 4), "r"(x.w[w]) : "memory");
                        for (; nan; nan &= nan - 1) {
                            const int d = part % VC * (VW * 32) + lr * (VW * 4) + w * 4 + (__ffs(nan) - 1) / 8;
                            for (int row = 0; row < rows; ++row)
                                if (token < sees(row)) atomicOr(&sm.nan[row][d / 32], 1u << (d % 32));
                            sm.any_nan = 1;
                        }
                    }
                }
            }
        };

        int stage = 0, stage_ahead = STAGES - 1;
        for (int tile = 0; tile < tiles; ++tile) {
            const int tok = tok0 + tile * kUnit, slot = tile & 31;
            // ---- the place of this tile and of the one to fetch; a new batch of 32 is looked up well ahead
            if (slot == 0 && tile > 0) {
                now = next;
                if (tile + 32 < tiles) id_next = block_of(tile + 32 + lane);
            }
            if (slot == 8 && tile + 24 < tiles) next = place_of(id_next, tile + 24 + lane);
            const bool none = __shfl_sync(0xffffffffu, (int)(now.at >> 32), slot) < 0;
            const float ks = __shfl_sync(0xffffffffu, now.ks, slot), vs = __shfl_sync(0xffffffffu, now.vs, slot);
            const long long ahead = __shfl_sync(0xffffffffu, slot + STAGES - 1 < 32 ? now.at : next.at, (slot + STAGES - 1) & 31);
            copies_wait<STAGES - 2>();
            Words<4> kw[2][KC];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int c = 0; c < KC; ++c) kw[i][c] = take<4>(k_ring + stage * (32 * D) + (i * KC + c) * 512);
            // ---- scores
            // (two chains of products, so that one is issued while the other's last is under way)
            float s[NT][4], s2[QSHARED ? 1 : NT][4];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[t][e] = s2[QSHARED ? 0 : t][e] = 0.f;
#pragma unroll
            for (int c = 0; c < KC; ++c)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t a0, a1, a2, a3;
                    to_half4<FMT>(kw[0][c].w[w], a0, a2);
                    to_half4<FMT>(kw[1][c].w[w], a1, a3);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        uint2 b;
                        if constexpr (QSHARED) b = sm.q[t][c * 4 + w][lane];
                        else b = make_uint2(qf[t][c * 4 + w][0], qf[t][c * 4 + w][1]);
                        mma(!QSHARED && (w & 1) ? s2[QSHARED ? 0 : t] : s[t], a0, a1, a2, a3, b.x, b.y);
                    }
                }
            // (here and not before the scores: 4 % less time with 40 rows)
            if (tile + STAGES - 1 < tiles) fetch(ahead, stage_ahead);
            copies_commit();

            // ---- softmax against a lagging reference
            bool above = false;
            const bool edge = tok + 16 > seen_first || none;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (QSHARED) s[t][e] *= sm.factor[t * 8 + 2 * lq + (e & 1)] * ks;
                    else s[t][e] = (s[t][e] + s2[t][e]) * (factor[t][e & 1] * ks);
                }
            if (edge) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (none || tok + lr + (e >> 1) * 8 >= limit(t, e & 1)) s[t][e] = -INFINITY;
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) above |= s[t][e] > ref[t][e & 1] + 15.f;
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
            if (vs > vref && vs >= 7.888609052210118e-31f && vs < INFINITY) {
                const float f = vref / vs;
                vref = vs;
                vref_inverse = kPart<FMT> / vs;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[t][i][e] *= f;
            }
            const float vf = edge && !(vs < INFINITY) ? 0.f : vs * vref_inverse;
            uint32_t pf[NT][2], pr[NT][2];       // probabilities times scales as the second operand, and what bf16 left of them
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = exp2_fast(s[t][e] - ref[t][e & 1]);
                    sum[t][e & 1] += p[e];
                }
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    uint32_t upper, rest;
                    split_bfloat2(p[e] * vf, p[e + 1] * vf, upper, rest);
                    pf[t][e / 2] = transposed(upper);
                    pr[t][e / 2] = transposed(rest);
                }
            }
            // ---- values
            if (edge && (FMT == FLUXBIN_CACHE_E4M3 || !(vs < INFINITY))) hide_nan(tok, stage, none, vs);
            Words<VW> vw[4][VC];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < VC; ++c) vw[i][c] = take<VW>(v_ring + stage * (32 * D) + (i * VC + c) * (VW * 128));
#pragma unroll
            for (int c = 0; c < VC; ++c)
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    uint32_t f[2][4];            // tokens 2q, 2q + 1, then 2q + 8, 2q + 9
#pragma unroll
                    for (int i = 0; i < 2; ++i) to_bfloat2x4<FMT>(vw[2 * i][c].w[w], vw[2 * i + 1][c].w[w], f[i]);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) mma_bf16(o[t][(c * VW + w) * 2 + i], f[0], f[1], 2 * i, pf[t]);
#pragma unroll
                        for (int i = 0; i < 2; ++i) mma_bf16(o[t][(c * VW + w) * 2 + i], f[0], f[1], 2 * i, pr[t]);
                    }
                }
            stage = stage + 1 == STAGES ? 0 : stage + 1;
            stage_ahead = stage_ahead + 1 == STAGES ? 0 : stage_ahead + 1;
        }
        copies_wait<0>();
        __syncthreads();                          // the ring is done with: its place holds the results now

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
        const bool whole = p0 == 0 && p1 == rq.pieces, any_nan = sm.any_nan;
        const int first_cta_slot = p0 == 0;                  // this job begins here, or goes on from the CTA before
        float *part = a.partial + (share * 2 + first_cta_slot) * ROWS * D, *part_lse = a.partial_lse + (share * 2 + first_cta_slot) * ROWS;
        auto write_out = [&](int row, int d, float4 v, float lse2) {
            const int g = row0 + row;
            const long long tok = rq.first + g / G;
            const int head = h * G + g % G;
            T *op = (T *)a.out + tok * a.out_token + head * a.out_head + d;
            __align__(8) T e[4] = {from_float<T>(v.x), from_float<T>(v.y), from_float<T>(v.z), from_float<T>(v.w)};
            *reinterpret_cast<uint2 *>(op) = *reinterpret_cast<const uint2 *>(e);
            if (d == 0 && a.lse) a.lse[tok * a.q_heads + head] = lse2 * 0.6931471805599453f;
        };
        for (int i = tid; i < ROWS * (D / 4); i += kThreads) {
            const int row = i / (D / 4), d = i % (D / 4) * 4;
            float m = -INFINITY, l = 0.f, f[kWarps];
#pragma unroll
            for (int w = 0; w < kWarps; ++w) m = fmaxf(m, sm.m[w][row]);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {           // a warp without tokens has l = 0; a NaN in l stays
                f[w] = sm.l[w][row] == 0.f ? 0.f : exp2_fast(sm.m[w][row] - m);
                l += f[w] * sm.l[w][row];
            }
            const float inv = l == 0.f ? 0.f : 1.f / l, lse2 = l == 0.f ? -INFINITY : m + log2f(l);
            // (divided before the value scale comes in: the mean is no larger than the values, the sums are)
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float fv = f[w] * sm.v[w];
                const float4 x = *reinterpret_cast<const float4 *>(&sm.o[w][row][d]);
                v.x += fv * (x.x * inv); v.y += fv * (x.y * inv); v.z += fv * (x.z * inv); v.w += fv * (x.w * inv);
            }
            if (any_nan) {
                const uint32_t nan = sm.nan[row][d / 32] >> (d % 32);
                if (nan & 1) v.x = NAN;
                if (nan & 2) v.y = NAN;
                if (nan & 4) v.z = NAN;
                if (nan & 8) v.w = NAN;
            }
            if (whole) {
                if (row < rows) write_out(row, d, v, lse2);
            } else {
                *reinterpret_cast<float4 *>(part + row * D + d) = v;
                if (d == 0) part_lse[row] = lse2;
            }
        }
        if (!whole) {
            // the CTAs that hold parts of this job, by the cut of the line
            const int c0 = owner(job_begin + kJobCost), c1 = owner(job_begin + span - 1);
            __threadfence();
            __syncthreads();
            if (tid == 0) sm.last = atomicAdd(&a.arrived[c0], 1u) == (unsigned)(c1 - c0);
            __syncthreads();
            if (sm.last) {
                __threadfence();
                const int parts = c1 - c0 + 1;
                auto slot_of = [&](int c) { return (long long)(c0 + c) * 2 + (c == 0); };
                for (int row = warp; row < rows; row += kWarps) {
                    float m = -INFINITY, l = 0.f;
                    for (int c = lane; c < parts; c += 32) {
                        const float x = __ldcg(a.partial_lse + slot_of(c) * ROWS + row), m_now = fmaxf(m, x);
                        l = l * (m == -INFINITY ? 0.f : exp2_fast(m - m_now)) + (x == -INFINITY ? 0.f : exp2_fast(x - m_now));
                        m = m_now;
                    }
                    float top = m;
                    for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                    l *= m == -INFINITY ? (l == l ? 0.f : 1.f) : exp2_fast(m - top);
                    for (int x = 16; x; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
                    if (lane == 0) {
                        sm.join_max[row] = top == -INFINITY ? 0.f : top;
                        sm.join_inv[row] = l == 0.f ? 0.f : 1.f / l;
                        sm.join_lse[row] = l == 0.f ? -INFINITY : top + log2f(l);
                    }
                }
                __syncthreads();
                constexpr int kItems = ROWS * (D / 4), kEach = (kItems + kThreads - 1) / kThreads;
                float4 v[kEach];
#pragma unroll
                for (int k = 0; k < kEach; ++k) v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll(16 / kEach > 1 ? 16 / kEach : 1)
                for (int c = 0; c < parts; ++c)
#pragma unroll
                    for (int k = 0; k < kEach; ++k) {
                        const int i = min(tid + k * kThreads, kItems - 1), row = i / (D / 4);
                        const float f = exp2_fast(__ldcg(a.partial_lse + slot_of(c) * ROWS + row) - sm.join_max[row]) * sm.join_inv[row];
                        const float4 y = __ldcg(reinterpret_cast<const float4 *>(a.partial + slot_of(c) * (ROWS * D)) + i);
                        v[k].x += f * y.x; v[k].y += f * y.y; v[k].z += f * y.z; v[k].w += f * y.w;
                    }
#pragma unroll
                for (int k = 0; k < kEach; ++k) {
                    const int i = tid + k * kThreads, row = i / (D / 4);
                    if (i >= kItems || row >= rows) continue;
                    write_out(row, i % (D / 4) * 4, v[k], sm.join_lse[row]);
                }
                if (tid == 0) a.arrived[c0] = 0;
            }
        }
        __syncthreads();                          // the shared arrays are free again
        if (any_nan) {
            for (int i = tid; i < ROWS * (D / 32); i += kThreads) sm.nan[i / (D / 32)][i % (D / 32)] = 0;
            if (tid == 0) sm.any_nan = 0;
            __syncthreads();
        }
    }
    if (extra == 0) return;
    // every CTA draws until one draw is past the end: after as many draws as there are, the counter is 0 again
    if (tid == 0) sm.share = (int)atomicInc(a.drawn, (unsigned)(extra + active - 1));
    __syncthreads();
    if (sm.share >= extra) return;
    share = 2 * sm.share + 1;
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
    const size_t smem = sizeof(Shared<D, 8 * NT, Shape<D, NT>::warps, Shape<D, NT>::stages, Shape<D, NT>::shared_queries>);
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
    const int grid = (sms < kMaxSms ? sms : kMaxSms) * Shape<D, NT>::ctas;
    return launch(attend_kernel<D, FMT, NT, T>, dim3((unsigned)grid), Shape<D, NT>::warps * 32, smem, s, a);
}
template <int D, int FMT, typename T> cudaError_t run_rows(const Args &a, cudaStream_t s)
{
    // rows that share a key head in an average request; a tile of 40 rows takes 2.2 times one of 16 (at 128, 16 requests of up to
    // 8190 tokens: 24 rows 109 us against 117 in one tile, 32 112 against 119, 40 169 against 122, 64 213 in both, 72 256 against
    // 215 in two, 112 337 against 324 in three; at 64 tiles of 40 never won)
    const long long rows = (long long)(a.q_heads / a.c.kv_heads) * ((a.tokens + a.batch - 1) / a.batch);
    if constexpr (D == 128) {
        if ((rows + 39) / 40 * 11 < (rows + 15) / 16 * 5) return run<D, FMT, 5, T>(a, s);
    }
    // (9 to 16 rows in one tile of 16 instead of two of 8: 68 against 80 us at 128, 92 against 138 at 256, 41 against 48 at 64)
    if (rows > 8) return run<D, FMT, 2, T>(a, s);
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

constexpr size_t kCounterBytes = ((1 + kMaxShares) * sizeof(unsigned) + 255) / 256 * 256;
// the most rows that partial results of a launch take: those of the CTAs on an SM, two shares each, two parts a share
constexpr size_t kPartRows = (size_t)kMaxSms * 40 * 2 * 2, kLseBytes = kPartRows * sizeof(float);

} // namespace

extern "C" size_t fluxbin_kv_attend_workspace_size(int32_t batch, int32_t tokens, int32_t q_heads, int32_t kv_heads, int32_t head_dim)
{
    if (batch < 1 || tokens < 0 || q_heads < 1 || kv_heads < 1 || q_heads % kv_heads != 0 || head_dim < 1) return 0;
    return kCounterBytes + kLseBytes * (1 + (size_t)head_dim);
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
        (block_table_stride != 0 && block_table_stride < block_table_width) || (!d_query_start && tokens != batch) ||
        (int64_t)tokens * (q_heads / cache->kv_heads) > INT32_MAX) return FLUXBIN_ERR_RANGE;
    if (tokens == 0) return FLUXBIN_OK;
    if (!d_q || !d_out || !d_lengths || !d_block_table || !d_workspace) return FLUXBIN_ERR_NULL;
    if (!aligned_to(d_q, 16) || !aligned_to(d_out, 16) || (tokens > 1 && (q_token % 8 || out_token % 8)) || (q_heads > 1 && (q_head % 8 || out_head % 8)) ||
        !aligned_to(d_query_start, 4) || !aligned_to(d_lengths, 4) || !aligned_to(d_block_table, 4) || !aligned_to(d_lse, 4) ||
        !aligned_to(d_workspace, 16)) return FLUXBIN_ERR_ALIGNMENT;
    if (!heads_apart(tokens, q_heads, out_token, out_head, cache->head_dim)) return FLUXBIN_ERR_RANGE;
    if (ws_bytes < fluxbin_kv_attend_workspace_size(batch, tokens, q_heads, cache->kv_heads, cache->head_dim)) return FLUXBIN_ERR_BUFFER_TOO_SMALL;
    const Args a = {*cache, batch, tokens, q_heads, block_table_width, d_q, q_token, q_head, d_query_start, d_lengths, d_block_table,
                    block_table_stride, scale, d_out, out_token, out_head, d_lse,
                    (unsigned *)d_workspace, (unsigned *)d_workspace + 1, (float *)((char *)d_workspace + kCounterBytes),
                    (float *)((char *)d_workspace + kCounterBytes + kLseBytes)};
    cudaStream_t s = (cudaStream_t)cuda_stream;
    FBD_CUDA(dtype == FLUXBIN_TYPE_FP16 ? run_dim<__half>(a, s) : run_dim<__nv_bfloat16>(a, s));
    return FLUXBIN_OK;
}
