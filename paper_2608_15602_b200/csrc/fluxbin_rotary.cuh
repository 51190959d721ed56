// The turn of a pair of elements by a token's position, shared by the rotary and the cache kernels.
//
// A pair's frequency is a 64-bit binary fraction of a turn.  position * frequency mod 2^64 is the angle mod one turn,
// exact up to position * 2^-65 turns; its upper 32 bits, read as a signed number, are the angle in units of 2^-31 half
// turns, rounded once to fp32 (error 2^-25 half turns) for sincospif.  A product in fp32 would be off by 2^-25 of the
// whole angle, which is 4e-3 radians at position 131,072.
#ifndef FLUXBIN_ROTARY_CUH
#define FLUXBIN_ROTARY_CUH

#include "fluxbin_device.cuh"

namespace fbd {

__device__ __forceinline__ void pair_angle(int position, unsigned long long turns, float magnitude, float sign, float &c, float &s)
{
    const unsigned long long phase = (unsigned long long)(long long)position * turns;
    const float half_turns = (float)(int)(phase >> 32) * 4.656612873077393e-10f;     // 2^-31
    sincospif(half_turns, &s, &c);
    c *= magnitude;
    s *= magnitude * sign;
}

// y = (a c - b s, b c + a s), every product and the difference rounded on their own: a user who turns keys before
// appending them gets the same values as one who lets the append turn them
__device__ __forceinline__ void turn_pair(float a, float b, float c, float s, float &u, float &v)
{
    u = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
    v = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
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
    T e[VE];
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
};

constexpr int kMaxPairs = 256;

// (cosine, sine) of every pair of a token's position into shared memory, by `threads` threads
__device__ __forceinline__ void token_angles(const fluxbin_rotary_t &rot, int position, float sign, float2 *angles, int tid, int threads)
{
    for (int i = tid; i < rot.rotary_dim / 2; i += threads) pair_angle(position, rot.d_turns[i], rot.magnitude, sign, angles[i].x, angles[i].y);
}

// heads h0, h0 + 1 ... h1 - 1 of token t (those of q, then those of k), angles in shared memory
template <typename T, int VE, bool INTER>
__device__ __forceinline__ void turn_heads(const fluxbin_rotary_t &rot, const float2 *angles, const Side &q, const Side &k, long long t, int h0, int h1,
                                           int tid, int threads)
{
    constexpr int NA = INTER ? VE / 2 : VE;      // pairs of a unit
    const int D = rot.head_dim, half = rot.rotary_dim / 2;
    const int turning = half / NA, units = turning + (D - rot.rotary_dim + VE - 1) / VE;
    const int rows = threads / units;            // heads in flight
    // more units than threads (single elements of wide heads): a thread takes several, one after the other
    for (int u = rows ? tid % units : tid; u < units; u += rows ? units : threads) {
        const bool turns = u < turning;
        float c[NA], s[NA];
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const float2 a = turns ? angles[u * NA + i] : make_float2(1.f, 0.f);
            c[i] = a.x;
            s[i] = a.y;
        }
        const int e0 = turns ? u * (INTER ? VE : NA) : rot.rotary_dim + (u - turning) * VE, n = min(D - e0, VE);
        const int step = rows ? rows : 1, first = h0 + (rows ? tid / units : 0);
        if (rows && tid / units >= rows) break;
        // a few heads' loads under way before the first is turned (a store would hold back the loads behind it)
        constexpr int BATCH = 4;
        for (int hb = first; hb < h1; hb += BATCH * step) {
            Elements<T, VE> a[BATCH], b[BATCH];
            T *y[BATCH];
            bool copy[BATCH];
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int h = hb + j * step;
                if (h >= h1) break;
                const bool of_q = h < q.heads;
                const int hs = of_q ? h : h - q.heads;
                const T *x = (const T *)(of_q ? q.in : k.in) + t * (of_q ? q.in_token : k.in_token) + hs * (of_q ? q.in_head : k.in_head) + e0;
                y[j] = (T *)(of_q ? q.out : k.out) + t * (of_q ? q.out_token : k.out_token) + hs * (of_q ? q.out_head : k.out_head) + e0;
                copy[j] = x != y[j];
                a[j].load(x, n);
                if (!INTER && turns) b[j].load(x + half, n);
            }
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                if (hb + j * step >= h1) break;
                if (!turns) {
                    if (copy[j]) a[j].store(y[j], n);
                    continue;
                }
#pragma unroll
                for (int i = 0; i < NA; ++i) {
                    T &lo = a[j].e[INTER ? 2 * i : i], &hi = INTER ? a[j].e[INTER ? 2 * i + 1 : 0] : b[j].e[i];
                    float f, g;
                    turn_pair(to_float(lo), to_float(hi), c[i], s[i], f, g);
                    lo = from_float<T>(f);
                    hi = from_float<T>(g);
                }
                a[j].store(y[j], n);
                if (!INTER) b[j].store(y[j] + half, n);
            }
        }
    }
}

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
