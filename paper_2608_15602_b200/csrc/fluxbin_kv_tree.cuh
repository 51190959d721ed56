// Attention over the 8-bit cache for many query rows of a key head: trees of drafted tokens (fluxbin_kv_attend_tree).
//
// A tile of 128 query rows (the query heads that share a key head, over a request's new tokens) goes over the cached tokens,
// kTokens at a time:
//     S = Q K^T  [rows x tokens],   P = exp2(S c - m),   O += P V  [rows x dim],   l += sum P
// on the matrix unit that accumulates in its own memory: a row of Q, S, P and O is a lane of it, so a softmax thread has a row to
// itself and needs no shuffle.  The unit takes operands of 16 bits:
//   K      8-bit entries are exact in fp16; Q is fp16, or bf16 as fp16 times a power of two, and stays in the unit's memory
//   V      exact in bf16 (int8 as parts 1 / 64)
//   P      times its token's value scale: two bf16 numbers, written where S was, which lose 2^-16 of it and flush nothing
//          short of fp32's range (see the kernel for few rows); so the second product is made twice
// The cache's bytes come in by asynchronous copies, 16 a thread, into places of shared memory that only this thread reads again, a few
// tiles ahead; the same thread converts them into swizzled tiles.  (In registers instead a warp that waits for the older tile's bytes
// waits for the younger one's too.)
//
// Warps: four or eight for the softmax, eight that load and convert, two that issue the products.  At head dimension 64 and 128
// the softmax is two groups of four warps that take the tiles in turn, each with accumulators of its own; what they have at the end
// of a job is put together as parts of the line are (at 256 the accumulators of one group fill half of the unit's memory: one
// group).  Scores and probabilities go through three places in turn, so that the scores of the next two tiles are under way
// while a tile's probabilities are formed.
//
// Every wait has a limit; one that runs out (a fault of the machine) ends the waiting of the whole CTA, and its jobs' rows become NaN.
// Products that are under way then end before the unit's memory is given back, and the counters of cut jobs are as after any other call.
#ifndef FLUXBIN_KV_TREE_CUH
#define FLUXBIN_KV_TREE_CUH

#include "fluxbin_kv_attend.cuh"

namespace {

constexpr int kRows = 128;                   // of a tile: the lanes of the matrix unit's memory
// Units that it costs to begin a job.  Measured 2, 4, 8, 14: 132, 132, 131, 130 us with 128 rows on 16 requests of 8190 tokens, 55, 47, 48, 55 on 64
// requests of 100, 241, 240, 237, 232 with 256 rows on one of 131071.
constexpr int kTreeJobCost = 8;
constexpr int kMetaRing = 32;                // tiles whose scales are kept
constexpr float kValueLag = 1048576.f;       // 2^20: value scales may pass the largest one met so far by this much before O is rescaled
// A wait's limit, in ns of a CTA that runs: between two looks at the clock no more counts than kWaitStep (the rest is time in which the
// device was another context's)
constexpr unsigned kWaitLimit = 2000000000u, kWaitStep = 10000000u;

template <int D> struct Tree {
    static constexpr int kTokens = D == 256 ? 32 : 64;           // of a tile
    static constexpr int kGroups = D == 256 ? 1 : 2;             // of four softmax warps
    static constexpr int kStages = D == 64 ? 6 : 4;              // tiles in shared memory
    static constexpr int kRing = D == 64 ? 6 : 4;                // tiles on their way there
    static constexpr int kConverters = 8;                        // warps
    static constexpr int kSoft = 128 * kGroups, kThreads = kSoft + kConverters * 32 + 64;
    static constexpr int kSlab = kTokens * 128;                  // 64 elements of every token
    static constexpr int kSide = D / 64 * kSlab, kStageBytes = 2 * kSide, kRingBytes = 2 * kTokens * D;
    // columns of the unit's memory: the sums, the queries, three places for scores and then probabilities
    static constexpr int kO = 0, kQ = kGroups * D, kS = kQ + D / 2, kPlaces = 3, kColumns = 512;
    static_assert(kS + kPlaces * kTokens <= kColumns, "the unit's memory");
    // With 18 warps 96 registers a thread are there, 55296 in all: 120 for the softmax, 72 for the converters
    static constexpr bool kSplit = kGroups == 2;
};

// What the softmax wants to know about a tile: key scales of its groups of 16 tokens, value scales as factors of the probabilities
// (over `vref`, the reference that the sums are in), which groups are in no block and whether rows may differ in what they see
struct __align__(16) Meta { float ks[4], f[4], vref; int none, edge; };

// ---- barriers, fences, the matrix unit -------------------------------------------------------------------

__device__ __forceinline__ uint32_t shared_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void barrier_init(unsigned long long &b, unsigned count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(shared_address(&b)), "r"(count) : "memory"); }
__device__ __forceinline__ void arrive(unsigned long long &b) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(shared_address(&b)) : "memory"); }
__device__ __forceinline__ bool try_wait(uint32_t b, unsigned parity)
{
    unsigned ok;
    asm volatile("{ .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n }" : "=r"(ok) : "r"(b), "r"(parity) : "memory");
    return ok;
}
__device__ __forceinline__ unsigned now_ns()         // modulo 2^32
{
    unsigned t;
    asm volatile("mov.u32 %0, %globaltimer_lo;" : "=r"(t));
    return t;
}
// Whether a wait of this CTA has run out, and what each may take
struct Waits { int failed; unsigned limit; };
// false once one has run out
__device__ __forceinline__ bool wait_for(unsigned long long &barrier, unsigned parity, Waits &waits)
{
    const uint32_t b = shared_address(&barrier);
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
        if (try_wait(b, parity)) return true;
    for (unsigned spent = 0, last = now_ns();;) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i)
            if (try_wait(b, parity)) return true;
        if (*(volatile int *)&waits.failed) return false;
        const unsigned now = now_ns();
        spent += min(now - last, kWaitStep);
        last = now;
        if (spent > waits.limit) {
            *(volatile int *)&waits.failed = 1;
            return false;
        }
    }
}
// the same for a whole warp, which goes on together
__device__ __forceinline__ bool wait_together(unsigned long long &barrier, unsigned parity, Waits &waits) { return __all_sync(0xffffffffu, wait_for(barrier, parity, waits)); }
template <int ID, int THREADS> __device__ __forceinline__ void sync_some() { asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(THREADS) : "memory"); }

__device__ __forceinline__ void unit_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void unit_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void unit_commit(unsigned long long &b)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(shared_address(&b)) : "memory");
}
// C [128 x N] (+)= A B^T, A in the unit's memory, B in shared memory
__device__ __forceinline__ void unit_mma(uint32_t c, uint32_t a, uint64_t b, uint32_t kind, bool add)
{
    asm volatile("{ .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n }" ::"r"(c), "r"(a), "l"(b), "r"(kind), "r"((int)add) : "memory");
}
// one lane of a warp, always the same
__device__ __forceinline__ bool elected()
{
    unsigned one;
    asm volatile("{ .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n }" : "=r"(one));
    return one;
}
template <int REGISTERS> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGISTERS)); }
template <int REGISTERS> __device__ __forceinline__ void leave_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGISTERS)); }
// What a product is told about its operands: fp32 sums; A and B of fp16 (0) or bf16 (1); whether B's rows lie along its columns; sizes
__host__ __device__ constexpr uint32_t unit_kind(int type, bool b_turned, int n) { return 1u << 4 | (uint32_t)type << 7 | (uint32_t)type << 10 | (uint32_t)b_turned << 16 | (uint32_t)(n / 8) << 17 | (uint32_t)(kRows / 16) << 24; }
// An operand in shared memory: rows of 128 bytes whose 16-byte pieces are swizzled by the row's number, eight rows every 1024 bytes; `slab`
// is the stride between pieces of 64 elements along the rows (used where rows lie along the operand's columns)
__device__ __forceinline__ uint64_t operand(uint32_t address, uint32_t slab)
{
    return (uint64_t)(address >> 4) | (uint64_t)(slab >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

template <int N> struct Columns { uint32_t w[N]; };
__device__ __forceinline__ void load_columns(uint32_t from, uint32_t (&r)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, "
                 "%26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
                   "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
                   "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(from) : "memory");
}
__device__ __forceinline__ void load_columns(uint32_t from, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
                   "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(from) : "memory");
}
__device__ __forceinline__ void store_columns(uint32_t to, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(to), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                 "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void store_columns(uint32_t to, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(to), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]),
                 "r"(r[7]) : "memory");
}
__device__ __forceinline__ void loads_done() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void stores_done() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---- the line of work ------------------------------------------------------------------------------------
// As in the kernel for few rows: jobs (request, head, tile of rows) of kTreeJobCost units and their pieces, a range for each CTA.
// Every role walks its CTA's range by itself.

struct Job {
    int r, h, row0, rows, p0, p1, tiles;
    long long begin;                             // of its units on the line
    int span;
};
template <int D> struct Walk {
    long long u, u_end, before;
    int r;
    Request rq;
    Job j;
    __device__ __forceinline__ long long units(const Args &a) const { return (long long)rq.row_tiles * a.c.kv_heads * (rq.pieces + kTreeJobCost); }
    // the next job of a warp whose lanes all ask
    __device__ __forceinline__ bool next(const Args &a, int lane)
    {
        Walk w = *this;
        const bool any = w.step(a);
        __syncwarp();
        if (lane == 0) *this = w;
        __syncwarp();
        return any;
    }
    __device__ __forceinline__ bool step(const Args &a)
    {
        const int G = a.q_heads / a.c.kv_heads;
        while (u < u_end) {
            while (u >= before + units(a)) {
                before += units(a);
                rq = request_of<kRows, Tree<D>::kTokens>(a, ++r);
            }
            j.span = rq.pieces + kTreeJobCost;
            const int job = (int)((u - before) / j.span);
            j.begin = before + (long long)job * j.span;
            j.p0 = max((int)(u - j.begin) - kTreeJobCost, 0);
            j.p1 = (int)min(u_end - j.begin, (long long)j.span) - kTreeJobCost;
            u = min(u_end, j.begin + j.span);
            if (j.p1 <= j.p0) continue;
            j.r = r;
            j.h = job / rq.row_tiles;
            j.row0 = job % rq.row_tiles * kRows;
            j.rows = (int)min((long long)kRows, (long long)rq.count * G - j.row0);
            j.tiles = max(min(j.p1, (rq.length + Tree<D>::kTokens - 1) / Tree<D>::kTokens) - j.p0, 0);
            return true;
        }
        return false;
    }
};

template <int D> struct TreeShared {
    uint32_t nan[2][kRows][D / 32];              // by the parity of the job
    int any_nan[2];
    float m[2][kRows], l[2][kRows], vref[2];     // of the two softmax groups
    float largest[2][kRows];                     // of the parts of the query rows
    Meta meta[kMetaRing];
    unsigned long long full[Tree<D>::kStages], free[Tree<D>::kStages];
    unsigned long long q_full, s_full[3], p_full[3], pv_done[3], ended[2], drained[2];
    long long place[Tree<D>::kConverters][2][32];                // of each converting warp: where 16 tokens lie
    uint32_t none[Tree<D>::kConverters][2];                      // which of them are in no block (and read the cache's first one instead)
    long long scan[32], before;
    int request, last;
    Waits waits;
    uint32_t columns;
    Walk<D> walk[Tree<D>::kThreads / 32];        // of each warp: in registers only while it is looked at
};

// bf16 elements times 2^-e as fp16 (half2_of_bf16), by two products, since 2^-e may pass fp32's range
struct Power { float first, second; };
__device__ __forceinline__ Power power_of(int e) { return {__int_as_float((127 - (e >> 1)) << 23), __int_as_float((127 - (e - (e >> 1))) << 23)}; }
__device__ __forceinline__ uint32_t half2_scaled(uint32_t w, const Power &p)
{
    const __half2 h = __floats2half2_rn(__uint_as_float(w << 16) * p.first * p.second, __uint_as_float(w & 0xffff0000u) * p.first * p.second);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// which of the tokens tok .. tok + 63 a row sees: those before the new ones, of those what its mask says, none past the length
__device__ __forceinline__ unsigned long long seen_bits(const Args &a, const Request &rq, int row, int tok)
{
    const int base = rq.length - rq.count, lead = min(max(base - tok, 0), 64), valid = rq.length - tok;
    unsigned long long bits = ~0ull;
    if (lead < 64) {
        const int j = max(tok - base, 0), w = j / 32, sh = j % 32;
        const uint32_t *words = a.tree + (long long)(rq.first + row / (a.q_heads / a.c.kv_heads)) * a.tree_stride;
        const unsigned long long w0 = w < a.tree_words ? words[w] : 0u, w1 = w + 1 < a.tree_words ? words[w + 1] : 0u, w2 = w + 2 < a.tree_words ? words[w + 2] : 0u;
        unsigned long long window = (w0 | w1 << 32) >> sh;
        if (sh) window |= w2 << (64 - sh);
        bits = window << lead | ((1ull << lead) - 1);
    }
    return valid >= 64 ? bits : valid <= 0 ? 0 : bits & ((1ull << valid) - 1);
}

// ---- the converters --------------------------------------------------------------------------------------

template <int FMT> __device__ __forceinline__ uint4 key_chunk(uint32_t x, uint32_t y)
{
    uint4 v;
    to_half4<FMT>(x, v.x, v.y);
    to_half4<FMT>(y, v.z, v.w);
    return v;
}
template <int FMT> __device__ __forceinline__ void to_bfloat4(uint32_t x, uint32_t &lo, uint32_t &hi);
// (as to_bfloat2x4, of four elements of one token)
template <> __device__ __forceinline__ void to_bfloat4<FLUXBIN_CACHE_INT8>(uint32_t x, uint32_t &lo, uint32_t &hi)
{
    x ^= 0x80808080u;
    const __nv_bfloat162 up = __bfloat162bfloat162(__ushort_as_bfloat16(0x7f00)), down = __bfloat162bfloat162(__ushort_as_bfloat16(0xc000));     // 2^127, -2
    const uint32_t a = __byte_perm(x, 0, 0x4140), b = __byte_perm(x, 0, 0x4342);
    const __nv_bfloat162 ra = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&a), up, down), rb = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&b), up, down);
    lo = *reinterpret_cast<const uint32_t *>(&ra);
    hi = *reinterpret_cast<const uint32_t *>(&rb);
}
template <> __device__ __forceinline__ void to_bfloat4<FLUXBIN_CACHE_E4M3>(uint32_t x, uint32_t &lo, uint32_t &hi)
{
    uint32_t h[2];
    to_half4<FLUXBIN_CACHE_E4M3>(x, h[0], h[1]);
    lo = bfloat2_of_half2(*reinterpret_cast<const __half2 *>(&h[0]));
    hi = bfloat2_of_half2(*reinterpret_cast<const __half2 *>(&h[1]));
}
template <int FMT> __device__ __forceinline__ uint4 value_chunk(uint32_t x, uint32_t y)
{
    uint4 v;
    to_bfloat4<FMT>(x, v.x, v.y);
    to_bfloat4<FMT>(y, v.z, v.w);
    return v;
}
__device__ __forceinline__ void put16(uint32_t to, const uint4 &v) { asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory"); }

template <int D, int FMT, typename T>
__device__ __forceinline__ void convert_role(const Args &a, TreeShared<D> &sm, uint32_t stages, Walk<D> &walk, int tid)
{
    using C = Tree<D>;
    constexpr int PIECES = D / 16, THREADS = C::kConverters * 32, PASS = THREADS / PIECES, N = C::kTokens / PASS, GROUPS = C::kTokens / 16, BATCH = 32 / GROUPS, RING = C::kRing;
    static_assert(PASS % 16 == 0 && C::kStages + RING + BATCH + 1 <= kMetaRing && RING <= BATCH, "places and scales ahead");
    const int lane = tid & 31, warp = tid >> 5, bs = a.c.block_tokens, H = a.c.kv_heads;
    // a thread's 16 elements of tokens sub, sub + PASS ...; eight neighbouring lanes hold four pieces of two neighbouring tokens: their
    // chunks go to all banks
    const int piece = lane % 4 + lane / (128 / PIECES) * 4, sub = warp * (32 / PIECES) + lane / 4 % (32 / PIECES);
    const uint32_t to0 = piece / 4 * C::kSlab + sub * 128 + (((uint32_t)(piece % 4 * 2) ^ (sub & 7)) << 4);
    const int shift = bs & (bs - 1) ? -1 : 31 - __clz(bs);       // (blocks are mostly of a power of two tokens)
    const uint32_t ring = stages + C::kStages * C::kStageBytes + tid * 16;
    unsigned stage = 0, stage_phase = 1;         // (the first time round a stage is free)
    bool ok = true;
    unsigned it = 0, jobs = 0;
    const Job &j = walk.j;
    const Request &rq = walk.rq;
    while (walk.next(a, lane)) {
        const int tiles = j.tiles;
        if (tiles == 0) continue;
        const unsigned parity = jobs & 1;
        // ---- what the job before the last left is done with
        if (jobs >= 2) ok = ok && wait_together(sm.ended[parity], (jobs / 2 - 1) & 1, sm.waits);
        for (int i = tid; i < kRows * (D / 32); i += C::kConverters * 32) sm.nan[parity][i / (D / 32)][i % (D / 32)] = 0;
        if (tid == 0) sm.any_nan[parity] = 0;
        sync_some<1, C::kConverters * 32>();

        // ---- places of the tokens, 16 at a time: 32 of them (a batch) are looked up together, well ahead, and kept in shared memory
        const int tok0 = j.p0 * C::kTokens, base = rq.length - rq.count;
        auto block_of = [&](int group) {
            const int tok = tok0 + group * 16;
            if (group >= tiles * GROUPS || tok >= rq.length) return -1;
            const int id = a.table[j.r * a.table_stride + (shift >= 0 ? tok >> shift : tok / bs)];
            return id >= 0 && id < a.c.num_blocks ? id : -1;
        };
        struct Place { long long at; float ks, vs; };
        auto place_of = [&](int id, int group) {
            Place x = {-1, 0.f, 0.f};
            if (id >= 0) {
                const int tok = tok0 + group * 16;
                x.at = id * a.c.block_stride + (shift >= 0 ? tok & (bs - 1) : tok % bs) * a.c.token_stride;
                if (warp == 0) {
                    x.ks = a.c.d_k_scale[(long long)id * H + j.h];
                    x.vs = a.c.d_v_scale[(long long)id * H + j.h];
                }
            }
            return x;
        };
        float vref = 0.f;                        // (warp 0)
        auto keep_places = [&](const Place &x, int batch) {
            const unsigned none = __ballot_sync(0xffffffffu, x.at < 0);
            sm.place[warp][batch & 1][lane] = max(x.at, 0ll);
            if (lane == 0) sm.none[warp][batch & 1] = none;
            if (warp == 0) {
                const int tok = tok0 + (batch * 32 + lane) * 16, mine = lane / GROUPS;
                const int none_here = (int)(none >> (mine * GROUPS) & ((1u << GROUPS) - 1)), edge = tok0 + (batch * BATCH + mine + 1) * C::kTokens > base || none_here;
                float vs = x.vs;
                if (x.at >= 0 && !(vs < INFINITY) && edge) {
                    // a scale that is no number, of tokens that not all rows see: 0, and noted for those that do
                    for (int row = 0; row < j.rows; ++row)
                        if (seen_bits(a, rq, j.row0 + row, tok) & 0xffff) {
                            for (int d = 0; d < D / 32; ++d) atomicOr(&sm.nan[parity][row][d], 0xffffffffu);
                            sm.any_nan[parity] = 1;
                        }
                    vs = 0.f;
                }
                // the reference is raised where the largest scale of a tile passes it by more than the sums' range is good for
                float most = vs < INFINITY ? vs : 0.f, own = 0.f;
#pragma unroll
                for (int o = GROUPS / 2; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
                if (__any_sync(0xffffffffu, vref == 0.f || most > vref * kValueLag)) {
                    for (int t = 0; t < BATCH; ++t) {
                        const float m = __shfl_sync(0xffffffffu, most, t * GROUPS);
                        if (m >= 7.888609052210118e-31f && (vref == 0.f || m > vref * kValueLag)) vref = m;
                        if (t == mine) own = vref;
                    }
                } else own = vref;
                Meta &m = sm.meta[(it + batch * BATCH + mine) % kMetaRing];
                m.ks[lane % GROUPS] = x.ks;
                m.f[lane % GROUPS] = vs * (own == 0.f ? 0.f : kPart<FMT> / own);
                if (lane % GROUPS == 0) {
                    m.vref = own;
                    m.none = none_here;
                    m.edge = edge;
                }
            }
            __syncwarp();
        };
        keep_places(place_of(block_of(lane), lane), 0);
        int id = -1;
        Place ahead = {-1, 0.f, 0.f};
        const long long mine = (long long)j.h * a.c.head_stride + sub % 16 * a.c.token_stride + piece * 16;
        const unsigned char *k_mine = (const unsigned char *)a.c.d_k + mine, *v_mine = (const unsigned char *)a.c.d_v + mine;
        uint32_t ring_in = ring, ring_out = ring;
        auto load = [&](int t) {                 // in order
            if (t < tiles) {
                const int slot = t % BATCH, batch = t / BATCH;
                if (slot % (BATCH / 2) == 0) {
                    if (slot == 0) id = block_of((batch + 1) * 32 + lane);
                    else ahead = place_of(id, (batch + 1) * 32 + lane);
                }
                const long long *place = &sm.place[warp][batch & 1][slot * GROUPS + sub / 16];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const long long at = place[i * PASS / 16];
                    copy_ahead<16>(ring_in + i * (THREADS * 16), k_mine + at);
                    copy_ahead<16>(ring_in + (N + i) * (THREADS * 16), v_mine + at);
                }
                if (slot == BATCH - 1) keep_places(ahead, batch + 1);
            }
            copies_commit();
            ring_in = ring_in + C::kRingBytes == ring + RING * C::kRingBytes ? ring : ring_in + C::kRingBytes;
        };
#pragma unroll 1
        for (int t = 0; t < RING - 1; ++t) load(t);

        // ---- tile after tile
#pragma unroll 1
        for (int t = 0; t < tiles; ++t) {
            copies_wait<RING - 2>();
            Words<4> k[N], v[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                k[i] = take<4>(ring_out + i * (THREADS * 16));
                v[i] = take<4>(ring_out + (N + i) * (THREADS * 16));
            }
            ring_out = ring_out + C::kRingBytes == ring + RING * C::kRingBytes ? ring : ring_out + C::kRingBytes;
            load(t + RING - 1);
            if constexpr (FMT == FLUXBIN_CACHE_E4M3) {
                // values that must not meet the probability 0 of a row that does not see them (see the kernel for few rows)
                const int tok = tok0 + t * C::kTokens;
                const uint32_t none = sm.none[warp][t / BATCH & 1] >> (t % BATCH * GROUPS) & ((1u << GROUPS) - 1);
                if (tok + C::kTokens > base || none) {
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const int token = tok + sub + i * PASS;
                        const bool out = (none >> ((sub + i * PASS) / 16) & 1) || token >= rq.length;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t nan = nan_bytes(v[i].w[e]);
                            if (out) v[i].w[e] = 0;
                            else if (nan) {
                                v[i].w[e] &= ~(nan | (nan - (nan >> 7)));
                                for (; nan; nan &= nan - 1) {
                                    const int d = piece * 16 + e * 4 + (__ffs(nan) - 1) / 8;
                                    for (int row = 0; row < j.rows; ++row)
                                        if (seen_bits(a, rq, j.row0 + row, token) & 1) atomicOr(&sm.nan[parity][row][d / 32], 1u << (d % 32));
                                    sm.any_nan[parity] = 1;
                                }
                            }
                        }
                    }
                }
            }
            ok = ok && wait_together(sm.free[stage], stage_phase, sm.waits);
            const uint32_t to = stages + stage * C::kStageBytes + to0;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                put16(to + i * (PASS * 128), key_chunk<FMT>(k[i].w[0], k[i].w[1]));
                put16((to ^ 16) + i * (PASS * 128), key_chunk<FMT>(k[i].w[2], k[i].w[3]));
                put16(to + C::kSide + i * (PASS * 128), value_chunk<FMT>(v[i].w[0], v[i].w[1]));
                put16((to ^ 16) + C::kSide + i * (PASS * 128), value_chunk<FMT>(v[i].w[2], v[i].w[3]));
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) arrive(sm.full[stage]);
            if (++stage == C::kStages) { stage = 0; stage_phase ^= 1; }
        }
        copies_wait<0>();
        it += tiles;
        ++jobs;
    }
}

// ---- the products ----------------------------------------------------------------------------------------

// The stage, the place and the group of a tile, and how often stage and place have been gone through
template <int D> struct Turn {
    int stage = 0, place = 0, group = 0;
    unsigned stage_phase = 0, place_phase = 0;
    __device__ __forceinline__ void next()
    {
        if (++stage == Tree<D>::kStages) { stage = 0; stage_phase ^= 1; }
        if (++place == Tree<D>::kPlaces) { place = 0; place_phase ^= 1; }
        if (Tree<D>::kGroups == 2) group ^= 1;
    }
};

// Two warps issue the products, one the scores', one the values', so that neither waits for what the other waits for.  The whole
// warp goes along, so that what it works out is the same for all lanes and stays in the registers that the unit's instructions
// take; one lane issues them.  (128 rows of fp16 on 16 requests of 8190 tokens: one warp that looked for either's turn 133 us, two 133,
// one in a fixed order 180; a single thread spent twice the products' time on issuing them.)
template <int D, bool VALUES>
__device__ __forceinline__ void product_role(const Args &a, TreeShared<D> &sm, uint32_t stages, Walk<D> &walk, int lane)
{
    using C = Tree<D>;
    constexpr uint32_t kind = VALUES ? unit_kind(1, true, D) : unit_kind(0, false, C::kTokens);
    const uint32_t unit = __shfl_sync(0xffffffffu, sm.columns, 0);
    const uint64_t operands = VALUES ? operand(stages + C::kSide, C::kSlab) : operand(stages, 16);
    bool ok = true;
    Turn<D> turn;
    unsigned jobs = 0, asked = 0;
    while (ok && walk.next(a, lane)) {
        const int tiles = __shfl_sync(0xffffffffu, walk.j.tiles, 0);
        if (tiles == 0) continue;
        if (!VALUES) ok = wait_together(sm.q_full, jobs & 1, sm.waits);
        for (int t = 0; ok && t < tiles; ++t, turn.next()) {
            const uint32_t place = unit + C::kS + turn.place * C::kTokens;
            const uint64_t b = operands + (turn.stage * C::kStageBytes >> 4);
            if constexpr (!VALUES) {
                ok = (asked < C::kPlaces || wait_together(sm.pv_done[turn.place], turn.place_phase ^ 1, sm.waits)) && wait_together(sm.full[turn.stage], turn.stage_phase, sm.waits);
                if (!ok) break;
                unit_after_sync();
                if (elected()) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) unit_mma(place, unit + C::kQ + k * 8, b + ((k / 4 * C::kSlab + k % 4 * 32) >> 4), kind, k > 0);
                    unit_commit(sm.s_full[turn.place]);
                }
                asked += asked < C::kPlaces;
            } else {
                ok = wait_together(sm.p_full[turn.place], turn.place_phase, sm.waits);
                if (!ok) break;
                unit_after_sync();
                const uint32_t o = unit + C::kO + turn.group * D;
                if (elected()) {
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int k = 0; k < C::kTokens / 16; ++k)
                            unit_mma(o, place + half * (C::kTokens / 2) + k * 8, b + (k * 2048 >> 4), kind, t >= C::kGroups || half > 0 || k > 0);
                    unit_commit(sm.pv_done[turn.place]);
                    unit_commit(sm.free[turn.stage]);
                }
            }
            __syncwarp();
        }
        ++jobs;
    }
    // what was issued ends before the unit's memory is given back, whoever's wait may have run out
    if (elected()) unit_commit(sm.drained[VALUES]);
    Waits own = {0, kWaitLimit};
    wait_together(sm.drained[VALUES], 0, own);
}

__device__ __forceinline__ float max_of(float x, float y, float z)
{
    float v;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(v) : "f"(x), "f"(y), "f"(z));
    return v;
}
// ---- the softmax -----------------------------------------------------------------------------------------

template <int D, int FMT, typename T>
__device__ __forceinline__ void softmax_role(const Args &a, TreeShared<D> &sm, Walk<D> &walk, long long size, long long over, int tid)
{
    using C = Tree<D>;
    constexpr int N = C::kTokens, GROUPS = C::kGroups;
    const int lane = tid & 31, warp = tid >> 5, group = warp / 4, row = tid % 128, H = a.c.kv_heads, G = a.q_heads / H;
    const uint32_t unit = sm.columns + ((uint32_t)(warp % 4 * 32) << 16);
    const long long share = blockIdx.x;
    bool ok = true;
    Turn<D> turn;
    unsigned it = 0, jobs = 0;
    const Job &j = walk.j;
    const Request &rq = walk.rq;
    while (walk.next(a, lane)) {
        const int tiles = j.tiles;
        const unsigned parity = jobs & 1;
        const bool live = warp % 4 * 32 < j.rows;                // (the rows of a warp are all past the end, or not)
        const int my_row = min(row, j.rows - 1);
        float ref = kNoRef, sum = 0.f, vref = 0.f, factor = a.scale * 1.4426950408889634f;
        if (tiles > 0) {
            // ---- the query row to the unit's memory, a part of it by each group (the last job's products are through)
            constexpr int PARTS = D / 8 / GROUPS, HELD = PARTS < 8 ? PARTS : 8;
            const int g = j.row0 + my_row;
            const uint4 *q = reinterpret_cast<const uint4 *>((const T *)a.q + (long long)(rq.first + g / G) * a.q_token + (long long)(j.h * G + g % G) * a.q_head) + group * PARTS;
            uint4 v[HELD];
            auto load = [&](int first) {
#pragma unroll
                for (int i = 0; i < HELD; ++i) v[i] = row < j.rows ? q[first + i] : make_uint4(0, 0, 0, 0);
            };
            Power power = {1.f, 1.f};
            if constexpr (!std::is_same<T, __half>::value) {
                float largest = 0.f;
#pragma unroll 1
                for (int first = PARTS - HELD; first >= 0; first -= HELD) {
                    load(first);
#pragma unroll
                    for (int i = 0; i < HELD; ++i) {
                        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) largest = fmaxf(largest, fmaxf(fabsf(__uint_as_float(w[k] << 16)), fabsf(__uint_as_float(w[k] & 0xffff0000u))));
                    }
                }
                if (GROUPS == 2) {
                    sm.largest[group][row] = largest;
                    sync_some<2, C::kSoft>();
                    largest = fmaxf(largest, sm.largest[group ^ 1][row]);
                }
                const int e = exponent_of(largest);
                power = power_of(e);
                factor = ldexpf(factor, e);
            } else load(0);
#pragma unroll 1
            for (int first = 0; first < PARTS; first += HELD) {
                if (first > 0) load(first);      // (the first are still held)
#pragma unroll
                for (int i = 0; i < HELD; i += 2) {
                    uint32_t w[8] = {v[i].x, v[i].y, v[i].z, v[i].w, v[i + 1].x, v[i + 1].y, v[i + 1].z, v[i + 1].w};
                    if constexpr (!std::is_same<T, __half>::value) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) w[k] = half2_scaled(w[k], power);
                    }
                    store_columns(unit + C::kQ + (group * PARTS + first + i) * 4, w);
                }
            }
            stores_done();
            unit_before_sync();
            __syncwarp();
            if (lane == 0) arrive(sm.q_full);
        }
        const int t_first = (group - (int)it) & (GROUPS - 1);    // tiles go to the groups in turn, from job to job
        for (int t = 0; t < tiles; ++t, turn.next()) {
            if (GROUPS == 2 && t % 2 != t_first) continue;
            ok = ok && wait_together(sm.s_full[turn.place], turn.place_phase, sm.waits);
            if (!ok) break;
            if (live) {
                unit_after_sync();
                const uint32_t at = unit + C::kS + turn.place * N;
                uint32_t s[N];
                const float *x = reinterpret_cast<const float *>(s);
#pragma unroll
                for (int i = 0; i < N; i += 32) load_columns(at + i, reinterpret_cast<uint32_t (&)[32]>(s[i]));
                const Meta &m = sm.meta[(it + t) % kMetaRing];
                const float4 ks = *reinterpret_cast<const float4 *>(m.ks), fs = *reinterpret_cast<const float4 *>(m.f), other = *reinterpret_cast<const float4 *>(&m.vref);
                const float c[4] = {factor * ks.x, factor * ks.y, factor * ks.z, factor * ks.w}, f[4] = {fs.x, fs.y, fs.z, fs.w};
                const bool edge = __float_as_int(other.z), plain = !edge && fminf(fminf(c[0], c[1]), fminf(c[2], c[3])) >= 0.f;
                float rescale = 1.f;
                if (vref != other.x) {           // (the same for every row)
                    rescale = vref / other.x;
                    vref = other.x;
                }
                unsigned long long bits = ~0ull;
                if (edge) {
                    bits = seen_bits(a, rq, j.row0 + my_row, (j.p0 + t) * N);
#pragma unroll
                    for (int i = 0; i < N / 16; ++i)
                        if (__float_as_int(other.y) >> i & 1) bits &= ~(0xffffull << (i * 16));
                }
                loads_done();
                // ---- the largest score against the lagging reference (scores times c, which is formed with the exponents)
                float most = -INFINITY;
                if (plain) {
#pragma unroll
                    for (int i = 0; i < N / 16; ++i) {
                        const float *y = x + i * 16;
                        const float t0 = max_of(y[0], y[1], y[2]), t1 = max_of(y[3], y[4], y[5]), t2 = max_of(y[6], y[7], y[8]), t3 = max_of(y[9], y[10], y[11]), t4 = max_of(y[12], y[13], y[14]);
                        most = fmaxf(most, max_of(max_of(t0, t1, y[15]), t2, max_of(t3, t4, t4)) * c[i]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (bits >> i & 1) most = fmaxf(most, x[i] * c[i / 16]);
                }
                if (most > ref + 15.f) {
                    const float now = most - 7.f, less = exp2_fast(ref - now);
                    ref = now;
                    sum *= less;
                    rescale *= less;
                }
                // ---- probabilities, 16 tokens at a time
                const unsigned long long minus_ref = two(-ref, -ref), minus_one = two(-1.f, -1.f);
                unsigned long long sums = two(sum, 0.f);
#pragma unroll
                for (int i = 0; i < N / 16; ++i) {
                    const unsigned long long c2 = two(c[i], c[i]);
                    float q[16];
#pragma unroll
                    for (int k = 0; k < 16; k += 2) {
                        apart(fma_two(two(x[i * 16 + k], x[i * 16 + k + 1]), c2, minus_ref), q[k], q[k + 1]);
                        q[k] = exp2_fast(q[k]);
                        q[k + 1] = exp2_fast(q[k + 1]);
                    }
                    if (edge) {
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (!(bits >> (i * 16 + k) & 1)) q[k] = 0.f;
                    }
                    const unsigned long long f2 = two(f[i], f[i]);
                    uint32_t upper[8], rest[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const unsigned long long pair = two(q[2 * k], q[2 * k + 1]);
                        sums = add_two(sums, pair);
                        const unsigned long long w = mul_two(pair, f2);
                        float w0, w1, r0, r1;
                        apart(w, w0, w1);
                        // (cut off, not rounded: what is left is exact in fp32 and rounded to eight bits more)
                        upper[k] = __byte_perm(__float_as_uint(w0), __float_as_uint(w1), 0x7632);
                        apart(fma_two(two(__uint_as_float(__float_as_uint(w0) & 0xffff0000u), __uint_as_float(__float_as_uint(w1) & 0xffff0000u)), minus_one, w), r0, r1);
                        const __nv_bfloat162 r = __floats2bfloat162_rn(r0, r1);
                        rest[k] = *reinterpret_cast<const uint32_t *>(&r);
                    }
                    store_columns(at + i * 8, upper);
                    store_columns(at + N / 2 + i * 8, rest);
                }
                {
                    float s0, s1;
                    apart(sums, s0, s1);
                    sum = s0 + s1;
                }
                if (t >= GROUPS && __any_sync(0xffffffffu, rescale != 1.f)) {
                    const unsigned before = it + t - GROUPS;     // the last tile that went to the same sums
                    ok = wait_together(sm.pv_done[before % C::kPlaces], before / C::kPlaces & 1, sm.waits);
                    unit_after_sync();
                    const uint32_t o = unit + C::kO + group * D;
#pragma unroll 1
                    for (int i = 0; i < D; i += 16) {
                        uint32_t v[16];
                        load_columns(o + i, v);
                        loads_done();
#pragma unroll
                        for (int k = 0; k < 16; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * rescale);
                        store_columns(o + i, v);
                    }
                }
                stores_done();
                unit_before_sync();
            }
            __syncwarp();
            if (lane == 0) arrive(sm.p_full[turn.place]);
        }
        // ---- the end of the job: sums of both groups
        sm.m[group][row] = ref;
        sm.l[group][row] = sum;
        if (row == 0) sm.vref[group] = vref;
        if (tiles > 0) {                       // (the products end in order)
            const unsigned n = it + tiles - 1;
            ok = ok && wait_together(sm.pv_done[n % C::kPlaces], n / C::kPlaces & 1, sm.waits);
        }
        sync_some<2, C::kSoft>();
        unit_after_sync();
        ok = ok && !*(volatile int *)&sm.waits.failed;                 // (the other group's waits count too)
        const bool whole = j.p0 == 0 && j.p1 == rq.pieces;
        const long long slot = share * 2 + (j.p0 == 0);
        // partial results lie element by element with the rows side by side, four elements together
        auto part_of = [&](long long slot) { return reinterpret_cast<float4 *>(a.partial + slot * kRows * D) + row; };
        auto put_eight = [&](int d, const float *v) {
            const int g = j.row0 + my_row, head = j.h * G + g % G;
            const long long tok = rq.first + g / G;
            __align__(16) T e[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) e[k] = from_float<T>(v[k]);
            *reinterpret_cast<uint4 *>((T *)a.out + tok * a.out_token + (long long)head * a.out_head + d) = *reinterpret_cast<const uint4 *>(e);
        };
        auto put_lse = [&](float lse2) {
            const int g = j.row0 + my_row;
            if (group == 0 && a.lse) a.lse[(long long)(rq.first + g / G) * a.q_heads + j.h * G + g % G] = lse2 * 0.6931471805599453f;
        };
        constexpr int OWN = D / GROUPS;          // elements of a thread
        if (live) {
            float m = -INFINITY, l = 0.f, f[GROUPS];
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) m = fmaxf(m, sm.m[g][row]);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const float lg = sm.l[g][row];
                f[g] = lg == 0.f ? 0.f : exp2_fast(sm.m[g][row] - m);
                l += f[g] * lg;
            }
            if (!ok) l = NAN;
            const float inv = l == 0.f ? 0.f : 1.f / l, lse2 = l == 0.f ? -INFINITY : m + log2f(l);
            const bool any_nan = tiles > 0 && sm.any_nan[parity];
#pragma unroll 1
            for (int d0 = group * (D / GROUPS); d0 < (group + 1) * (D / GROUPS); d0 += 16) {
                float v[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] = ok ? 0.f : NAN;
                uint32_t o[GROUPS][16];
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) load_columns(unit + C::kO + g * D + d0, o[g]);
                loads_done();
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    if (tiles <= ((g - (int)it) & (GROUPS - 1)) || !ok) continue;           // no tile was this group's
                    const float fv = f[g] * sm.vref[g];
#pragma unroll
                    for (int k = 0; k < 16; ++k) v[k] += fv * (__uint_as_float(o[g][k]) * inv);
                }
                if (any_nan) {
                    const uint32_t nan = sm.nan[parity][row][d0 / 32] >> (d0 % 32);
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (nan >> k & 1) v[k] = NAN;
                }
                if (row < j.rows) {
                    if (whole) {
                        put_eight(d0, v);
                        put_eight(d0 + 8, v + 8);
                    } else {
#pragma unroll
                        for (int k = 0; k < 16; k += 4) part_of(slot)[(d0 + k) / 4 * kRows] = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
                    }
                }
            }
            if (row < j.rows) {
                if (whole) put_lse(lse2);
                else if (group == 0) a.partial_lse[slot * kRows + row] = lse2;
            }
            unit_before_sync();
        }
        if (!whole) {
            // the CTAs that hold parts of this job, by the cut of the line
            auto owner = [&](long long x) { return x < over * (size + 1) ? x / (size + 1) : over + (x - over * (size + 1)) / size; };
            const int c0 = (int)owner(j.begin + kTreeJobCost), c1 = (int)owner(j.begin + j.span - 1);
            __threadfence();
            sync_some<2, C::kSoft>();
            if (tid == 0) sm.last = atomicAdd(&a.arrived[c0], 1u) == (unsigned)(c1 - c0);
            sync_some<2, C::kSoft>();
            if (sm.last) {
                __threadfence();
                const int parts = c1 - c0 + 1;
                auto slot_of = [&](int c) { return (long long)(c0 + c) * 2 + (c == 0); };
                if (row < j.rows) {
                    float top = -INFINITY, l = 0.f;
#pragma unroll 8
                    for (int c = 0; c < parts; ++c) {
                        const float x = __ldcg(a.partial_lse + slot_of(c) * kRows + row), now = fmaxf(top, x);
                        l = l * (top == -INFINITY ? 0.f : exp2_fast(top - now)) + (x == -INFINITY ? 0.f : exp2_fast(x - now));
                        top = now;
                    }
                    put_lse(l == 0.f ? -INFINITY : top + log2f(l));
                    if (top == -INFINITY) top = 0.f;
                    l = l == 0.f ? 0.f : 1.f / l;
                    constexpr int AT_ONCE = 32;
#pragma unroll 1
                    for (int d0 = group * OWN; d0 < (group + 1) * OWN; d0 += AT_ONCE) {
                        float v[AT_ONCE];
#pragma unroll
                        for (int k = 0; k < AT_ONCE; ++k) v[k] = 0.f;
#pragma unroll 1
                        for (int c = 0; c < parts; ++c) {
                            float4 y[AT_ONCE / 4];
#pragma unroll
                            for (int k = 0; k < AT_ONCE / 4; ++k) y[k] = __ldcg(part_of(slot_of(c)) + (d0 / 4 + k) * kRows);
                            const float w = exp2_fast(__ldcg(a.partial_lse + slot_of(c) * kRows + row) - top) * l;
#pragma unroll
                            for (int k = 0; k < AT_ONCE / 4; ++k) {
                                v[4 * k] += w * y[k].x; v[4 * k + 1] += w * y[k].y; v[4 * k + 2] += w * y[k].z; v[4 * k + 3] += w * y[k].w;
                            }
                        }
#pragma unroll
                        for (int k = 0; k < AT_ONCE; k += 8) put_eight(d0 + k, v + k);
                    }
                }
                if (tid == 0) a.arrived[c0] = 0;
            }
        }
        sync_some<2, C::kSoft>();                // both groups have read the sums, which the next job's products write
        if (tiles > 0) {
            if (tid == 0) arrive(sm.ended[parity]);
            ++jobs;
        }
        it += tiles;
    }
}

template <int D, int FMT, typename T>
__global__ void __launch_bounds__(Tree<D>::kThreads, 1) tree_attend_kernel(const __grid_constant__ Args a)
{
    using C = Tree<D>;
    extern __shared__ unsigned char smem_tree[];
    const uint32_t tiles = (shared_address(smem_tree) + 1023) & ~1023u;
    TreeShared<D> &sm = *reinterpret_cast<TreeShared<D> *>(smem_tree + (tiles - shared_address(smem_tree)) + C::kStages * C::kStageBytes + C::kRing * C::kRingBytes);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    wait_for_predecessor();
    // ---- where this CTA's part begins: a sum over the requests, each thread over a run of them
    const int per = (a.batch + C::kThreads - 1) / C::kThreads, r_lo = min(tid * per, a.batch), r_hi = min(r_lo + per, a.batch);
    auto units = [&](int r) {
        const Request q = request_of<kRows, C::kTokens>(a, r);
        return (long long)q.row_tiles * a.c.kv_heads * (q.pieces + kTreeJobCost);
    };
    long long mine = 0;
    for (int r = r_lo; r < r_hi; ++r) mine += units(r);
    long long upto = mine;
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    if (lane == 31) sm.scan[warp] = upto;
    __syncthreads();
    long long total = 0;
    for (int w = 0; w < C::kThreads / 32; ++w) {
        if (w < warp) upto += sm.scan[w];
        total += sm.scan[w];
    }
    const long long active = min((long long)gridDim.x, total);
    if (a.query_start) empty_rows<D, T>(a, tid, C::kThreads);
    if (blockIdx.x >= active) return;            // (the whole CTA)
    const long long size = total / active, over = total - size * active;
    auto cut = [&](long long i) { return i * size + min(i, over); };
    const long long u = cut(blockIdx.x), u_end = cut(blockIdx.x + 1);
    if (u >= upto - mine && u < upto) {
        long long before = upto - mine;
        for (int r = r_lo; r < r_hi; ++r) {
            const long long n = units(r);
            if (u < before + n) { sm.request = r; sm.before = before; break; }
            before += n;
        }
    }
    if (tid == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            barrier_init(sm.full[i], C::kConverters + (i == a.withheld));
            barrier_init(sm.free[i], 1);
        }
        barrier_init(sm.q_full, C::kSoft / 32);
        for (int i = 0; i < C::kPlaces; ++i) {
            barrier_init(sm.s_full[i], 1);
            barrier_init(sm.p_full[i], 4);
            barrier_init(sm.pv_done[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            barrier_init(sm.ended[i], 1);
            barrier_init(sm.drained[i], 1);
        }
        sm.waits.failed = 0;
        sm.waits.limit = a.wait_limit;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    constexpr int kIssuer = C::kThreads / 32 - 2;
    if (warp == kIssuer) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_address(&sm.columns)), "n"(C::kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    unit_before_sync();
    __syncthreads();
    unit_after_sync();
    let_successor_start();                       // (not before: it might take some of the unit's memory and wait for this kernel with it)
    Walk<D> walk;
    walk.u = u;
    walk.u_end = u_end;
    walk.before = sm.before;
    walk.r = sm.request;
    walk.rq = request_of<kRows, C::kTokens>(a, walk.r);
    if (lane == 0) sm.walk[warp] = walk;
    __syncwarp();
    if (warp < C::kSoft / 32) {
        if constexpr (C::kSplit) take_registers<120>();
        softmax_role<D, FMT, T>(a, sm, sm.walk[warp], size, over, tid);
    } else if (warp < kIssuer) {
        if constexpr (C::kSplit) leave_registers<72>();
        convert_role<D, FMT, T>(a, sm, tiles, sm.walk[warp], tid - C::kSoft);
    } else if (warp == kIssuer) product_role<D, false>(a, sm, tiles, sm.walk[warp], lane);
    else product_role<D, true>(a, sm, tiles, sm.walk[warp], lane);
    unit_before_sync();
    __syncthreads();
    unit_after_sync();
    if (warp == kIssuer) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sm.columns), "n"(C::kColumns) : "memory");
}

// CTAs of a launch, and what their partial results take: two parts each
constexpr size_t kTreePartRows = (size_t)kMaxSms * 2 * kRows, kTreeLseBytes = kTreePartRows * sizeof(float);

template <int D, int FMT, typename T> cudaError_t run_tree(const Args &a, cudaStream_t s)
{
    const size_t smem = 1024 + Tree<D>::kStages * Tree<D>::kStageBytes + Tree<D>::kRing * Tree<D>::kRingBytes + sizeof(TreeShared<D>);
    static std::atomic<bool> opted[fb::kMaxDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= fb::kMaxDevices) return cudaErrorInvalidDevice;
    if (!opted[dev].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(tree_attend_kernel<D, FMT, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        opted[dev].store(true, std::memory_order_relaxed);
    }
    const int sms = num_sms();
    if (sms == 0) return cudaErrorInvalidDevice;
    return launch(tree_attend_kernel<D, FMT, T>, dim3((unsigned)(sms < kMaxSms ? sms : kMaxSms)), Tree<D>::kThreads, smem, s, a);
}

template <int D> cudaError_t run_tree_of(const Args &a, bool bf16, cudaStream_t s)
{
    if (bf16) return a.c.format == FLUXBIN_CACHE_INT8 ? run_tree<D, FLUXBIN_CACHE_INT8, __nv_bfloat16>(a, s) : run_tree<D, FLUXBIN_CACHE_E4M3, __nv_bfloat16>(a, s);
    return a.c.format == FLUXBIN_CACHE_INT8 ? run_tree<D, FLUXBIN_CACHE_INT8, __half>(a, s) : run_tree<D, FLUXBIN_CACHE_E4M3, __half>(a, s);
}

} // namespace

// by head dimension, in files of their own
namespace fbd {
cudaError_t launch_tree_64(const AttendArgs &a, bool bf16, cudaStream_t s);
cudaError_t launch_tree_128(const AttendArgs &a, bool bf16, cudaStream_t s);
cudaError_t launch_tree_256(const AttendArgs &a, bool bf16, cudaStream_t s);
} // namespace fbd

#endif
