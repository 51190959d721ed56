// The turn of a pair of elements by a token's position, shared by the rotary and the cache kernels.
//
// A pair's frequency is a 64-bit binary fraction of a turn.  position * frequency mod 2^64 is the angle mod one turn,
// exact up to position * 2^-65 turns; its upper 32 bits, read as a signed number, are the angle in units of 2^-31 half
// turns, rounded once to fp32 (error 2^-25 half turns) for sincospif.  A product in fp32 would be off by 2^-25 of the
// whole angle, which is 4e-3 radians at position 131,072.
#ifndef FLUXBIN_ROTARY_CUH
#define FLUXBIN_ROTARY_CUH

#include "fluxbin_device.cuh"

#include <type_traits>

namespace fbd {

__device__ __forceinline__ void pair_angle(int position, unsigned long long turns, float magnitude, float sign, float &c, float &s)
{
    const unsigned long long phase = (unsigned long long)(long long)position * turns;
    const float half_turns = (float)(int)(phase >> 32) * 4.656612873077393e-10f;     // 2^-31
    sincospif(half_turns, &s, &c);
    c *= magnitude;
    s *= magnitude * sign;
}

// y = (a c - b s, b c + a s), one rounding of each product that is added: the append turns keys by the same expressions, so
// turning first (in fp32) and appending gives the same entries
__device__ __forceinline__ float turn_first(float a, float b, float c, float s) { return fmaf(a, c, -__fmul_rn(b, s)); }
__device__ __forceinline__ float turn_second(float a, float b, float c, float s) { return fmaf(b, c, __fmul_rn(a, s)); }
__device__ __forceinline__ void turn_pair(float a, float b, float c, float s, float &u, float &v)
{
    u = turn_first(a, b, c, s);
    v = turn_second(a, b, c, s);
}

// ---- the heads of one token ------------------------------------------------------------------------------
// A unit is VE neighbouring elements (interleaved) or VE elements of the first half with those of the second: one or two
// 16-byte accesses, or single elements where strides or addresses allow no wider ones.  A thread keeps its unit, with
// the unit's sines and cosines in registers, and goes over the heads; both elements of a pair are read before either is
// written, so the output may be the input.

struct Side {
    const void *in;
    void *out;
    int heads;
    long long in_token, in_head, out_token, out_head;
};

template <typename T, int VE> struct Elements {
    __align__(VE * sizeof(T) < 16 ? VE * sizeof(T) : 16) T e[VE];
    __device__ __forceinline__ void load(const T *p, int n)
    {
        if constexpr (VE * sizeof(T) == 16) *reinterpret_cast<uint4 *>(e) = *reinterpret_cast<const uint4 *>(p);
        else
#pragma unroll
            for (int i = 0; i < VE; ++i) if (i < n) e[i] = p[i];
    }
    __device__ __forceinline__ void store(T *p, int n) const
    {
        if constexpr (VE * sizeof(T) == 16) *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(e);
        else
#pragma unroll
            for (int i = 0; i < VE; ++i) if (i < n) p[i] = e[i];
    }
    // two neighbours at a time where there are two
    __device__ __forceinline__ void set(int i, float v0, float v1)
    {
        if constexpr (std::is_same<T, __half>::value) *reinterpret_cast<__half2 *>(e + i) = __floats2half2_rn(v0, v1);
        else if constexpr (std::is_same<T, __nv_bfloat16>::value) *reinterpret_cast<__nv_bfloat162 *>(e + i) = __floats2bfloat162_rn(v0, v1);
        else { e[i] = v0; e[i + 1] = v1; }
    }
};

constexpr int kMaxPairs = 256;

// (cosine, sine) of every pair of a token's position into shared memory, by `threads` threads
__device__ __forceinline__ void token_angles(const fluxbin_rotary_t &rot, int position, float sign, float2 *angles, int tid, int threads)
{
    for (int i = tid; i < rot.rotary_dim / 2; i += threads) pair_angle(position, rot.d_turns[i], rot.magnitude, sign, angles[i].x, angles[i].y);
}

// Heads h0, h0 + 1 ... h1 - 1 of token t (those of q, then those of k).  form_angles() fills `angles` and ends with a
// barrier; every thread of the CTA calls it at the same place, after its first loads are under way.
template <typename T, int VE, bool INTER, typename Form>
__device__ __forceinline__ void turn_heads(const fluxbin_rotary_t &rot, const float2 *angles, const Side &q, const Side &k, long long t, int h0, int h1,
                                           int tid, int threads, Form form_angles)
{
    constexpr int NA = INTER ? VE / 2 : VE;      // pairs of a unit
    constexpr int BATCH = INTER ? 4 : 2;         // heads whose loads are under way at once (one or two accesses each)
    const int D = rot.head_dim, half = rot.rotary_dim / 2;
    const int turning = half / NA, units = turning + (D - rot.rotary_dim + VE - 1) / VE;
    const int rows = threads / units;            // heads side by side
    const int step = rows ? rows : 1, row = rows ? tid / units : 0;
    // more units than threads (single elements of wide heads): a thread takes several, one after the other
    const int u_step = rows ? units : threads;
    const int u0 = rows ? (row < rows ? tid % units : units) : tid;
    Elements<T, VE> a[BATCH], b[BATCH];
    auto element_of = [&](int u) { return u < turning ? u * (INTER ? VE : NA) : rot.rotary_dim + (u - turning) * VE; };
    auto load = [&](const T *x, long long stride, int left, int u, int n) {
#pragma unroll
        for (int j = 0; j < BATCH; ++j)
            if (j * step < left) {
                a[j].load(x + j * stride, n);
                if (!INTER && u < turning) b[j].load(x + j * stride + half, n);
            }
    };
    // the heads of q in the range, then those of k
    bool loaded = false, formed = false;
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
        const Side &S = side ? k : q;
        const int lo = max(h0 - (side ? q.heads : 0), 0), hi = min(h1 - (side ? q.heads : 0), S.heads);
        if (lo >= hi) continue;                  // the same for every thread
        const T *in = (const T *)S.in + t * S.in_token + (long long)(lo + row) * S.in_head;
        T *out = (T *)S.out + t * S.out_token + (long long)(lo + row) * S.out_head;
        if (!formed) {
            if (u0 < units && lo + row < hi) {
                load(in + element_of(u0), step * S.in_head, hi - lo - row, u0, min(D - element_of(u0), VE));
                loaded = true;
            }
            form_angles();
            formed = true;
        }
        for (int u = u0; u < units; u += u_step) {
            const bool turns = u < turning;
            const int e0 = element_of(u), n = min(D - e0, VE);
            float c[NA], s[NA];
#pragma unroll
            for (int i = 0; i < NA; ++i) {
                const float2 x = turns ? angles[u * NA + i] : make_float2(1.f, 0.f);
                c[i] = x.x;
                s[i] = x.y;
            }
            const T *x = in + e0;
            T *y = out + e0;
            for (int h = lo + row; h < hi; h += BATCH * step, x += BATCH * step * S.in_head, y += BATCH * step * S.out_head) {
                if (!loaded) load(x, step * S.in_head, hi - h, u, n);
                loaded = false;
#pragma unroll
                for (int j = 0; j < BATCH; ++j) {
                    if (j * step >= hi - h) break;
                    T *to = y + j * step * S.out_head;
                    if (!turns) {
                        if (to != x + j * step * S.in_head) a[j].store(to, n);
                        continue;
                    }
                    float f[NA], g[NA];
#pragma unroll
                    for (int i = 0; i < NA; ++i)
                        turn_pair(to_float(a[j].e[INTER ? 2 * i : i]), to_float(INTER ? a[j].e[INTER ? 2 * i + 1 : 0] : b[j].e[i]), c[i], s[i], f[i], g[i]);
                    if constexpr (INTER) {
#pragma unroll
                        for (int i = 0; i < NA; ++i) a[j].set(2 * i, f[i], g[i]);
                    } else if constexpr (NA > 1) {
#pragma unroll
                        for (int i = 0; i < NA; i += 2) {
                            a[j].set(i, f[i], f[i + 1]);
                            b[j].set(i, g[i], g[i + 1]);
                        }
                    } else {
                        a[j].e[0] = from_float<T>(f[0]);
                        b[j].e[0] = from_float<T>(g[0]);
                    }
                    a[j].store(to, n);
                    if (!INTER) b[j].store(to + half, n);
                }
            }
        }
    }
}

// fluxbin_rotary's launch, for the append of a prompt
cudaError_t launch_rotary(const fluxbin_rotary_t &rot, int dtype, int inverse, int tokens, const int *positions, const Side &q, const Side &k,
                          cudaStream_t s);
constexpr int kFewTokens = 148 * 4;              // CTAs that fill the device: fewer tokens split their heads

// whether every access of turn_heads may be 16 bytes wide
inline bool wide_heads(const fluxbin_rotary_t &r, int dtype, const Side &s)
{
    const int64_t n = 16 / type_size(dtype);
    if (s.heads == 0) return true;
    return aligned_to(s.in, 16) && aligned_to(s.out, 16) && s.in_token % n == 0 && s.in_head % n == 0 && s.out_token % n == 0 && s.out_head % n == 0 &&
           r.head_dim % n == 0 && r.rotary_dim % (r.interleaved ? n : 2 * n) == 0;
}

inline fluxbin_status_t check_rotary(const fluxbin_rotary_t *r)
{
    if (!r || !r->d_turns) return FLUXBIN_ERR_NULL;
    if (r->head_dim < 2 || r->head_dim > 512 || r->rotary_dim < 2 || r->rotary_dim > r->head_dim || (r->rotary_dim & 1)) return FLUXBIN_ERR_RANGE;
    if (!aligned_to(r->d_turns, 8)) return FLUXBIN_ERR_ALIGNMENT;
    return FLUXBIN_OK;
}

} // namespace fbd

#endif
