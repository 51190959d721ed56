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

inline fluxbin_status_t check_rotary(const fluxbin_rotary_t *r)
{
    if (!r || !r->d_turns) return FLUXBIN_ERR_NULL;
    if (r->head_dim < 2 || r->head_dim > 512 || r->rotary_dim < 2 || r->rotary_dim > r->head_dim || (r->rotary_dim & 1)) return FLUXBIN_ERR_RANGE;
    if (!aligned_to(r->d_turns, 8)) return FLUXBIN_ERR_ALIGNMENT;
    return FLUXBIN_OK;
}

} // namespace fbd

#endif
