// Rotary positions on the device: which channels and pairs a lane has, its angles, the turn itself.
//
// Pair j of a head's n pairs turns by the angle of position p = positions[axis(j)][token] and of its own frequency; the table
// holds (cos, sin) of both for every position, so a row of it is 8 n bytes and all heads of a token read the same one (or, with
// several axes, pieces of one row for each).
//   first' = first * cos - second * sin,  second' = second * cos + first * sin     IEEE fp32, every step rounded once
// A lane has eight channels and, where they turn, pairs 4i .. 4i + 3: neighbouring pairs are eight channels in a row, pairs of
// the halves are four channels of each half, so that no lane needs another's.
#ifndef ATOM_ROTARY_H
#define ATOM_ROTARY_H

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include "atom_internal.h"

namespace atom_rotary_device {

using atom_internal::Turn;

struct Angles { float c[4], s[4]; };

// Where a lane's two times four channels begin.
struct Channels { int lo, hi; bool turned; };

__device__ __forceinline__ Channels channels(const Turn &t, int i)
{
    const bool turned = 4 * i < t.n_pairs, apart = turned && !t.interleaved;
    return {apart ? 4 * i : 8 * i, apart ? t.n_pairs + 4 * i : 8 * i + 4, turned};
}

// The axes of the lane's four pairs, two bits each.
__device__ __forceinline__ uint32_t lane_axes(const Turn &t, int i)
{
    uint32_t word = t.axis[0];
#pragma unroll
    for (int w = 1; w < 8; ++w) word = (i >> 2) == w ? t.axis[w] : word;
    return (word >> (8 * (i & 3))) & 0xffu;
}

// A token's positions (those of the axes that there are).
struct Positions { int32_t p[4]; };

template <bool ONE>
__device__ __forceinline__ Positions positions(const Turn &t, int64_t token)
{
    Positions at;
    at.p[0] = t.positions[token];
    if constexpr (!ONE) {
#pragma unroll
        for (int a = 1; a < 4; ++a) at.p[a] = t.positions[(a < t.axes ? a : 0) * t.ldp + token];
    }
    return at;
}

// cos and sin of pairs 4i .. 4i + 3 (of pairs 0 .. 3 in a lane whose channels do not turn: loads without a branch around them); of a position outside the
// table NaN, by bits, as a choice between the loaded and NaN becomes a branch with single loads in it.  axes: lane_axes()
template <bool ONE>
__device__ __forceinline__ Angles angles(const Turn &t, const Positions &at, int i, uint32_t axes)
{
    Angles r;
    if (4 * i >= t.n_pairs) i = 0;
    auto marked = [](float c, bool inside) __attribute__((always_inline)) {
        return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, c) | (inside ? 0u : 0x7fc00000u));
    };
    if constexpr (ONE) {
        const bool inside = (uint32_t)at.p[0] < t.n_pos;
        const float4 *row = reinterpret_cast<const float4 *>(t.table + (int64_t)(inside ? at.p[0] : 0) * (2 * t.n_pairs) + 8 * i);
        const float4 u = row[0], v = row[1];
        r = {{u.x, u.z, v.x, v.z}, {u.y, u.w, v.y, v.w}};
#pragma unroll
        for (int k = 0; k < 4; ++k) r.c[k] = marked(r.c[k], inside);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int a = (axes >> (2 * k)) & 3;
            const int32_t p = a == 0 ? at.p[0] : a == 1 ? at.p[1] : a == 2 ? at.p[2] : at.p[3];
            const bool inside = (uint32_t)p < t.n_pos;
            const float2 u = *reinterpret_cast<const float2 *>(t.table + (int64_t)(inside ? p : 0) * (2 * t.n_pairs) + 8 * i + 2 * k);
            r.c[k] = marked(u.x, inside);
            r.s[k] = u.y;
        }
    }
    return r;
}

// The lane's eight values (x[0..3] from channels().lo on, x[4..7] from hi on) turned; sign -1: the other way.
template <bool NEIGHBOURS>
__device__ __forceinline__ void turn(float x[8], const Angles &r, float sign)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float &first = x[NEIGHBOURS ? 2 * k : k], &second = x[NEIGHBOURS ? 2 * k + 1 : 4 + k];
        const float s = sign * r.s[k];
        const float a = first * r.c[k] - second * s, b = second * r.c[k] + first * s;
        first = a;
        second = b;
    }
}

__device__ __forceinline__ void widen(const uint2 &v, float *x)
{
    const __half2 a = __builtin_bit_cast(__half2, v.x), b = __builtin_bit_cast(__half2, v.y);
    x[0] = __low2float(a);
    x[1] = __high2float(a);
    x[2] = __low2float(b);
    x[3] = __high2float(b);
}
__device__ __forceinline__ uint2 narrow(const float *x)
{
    return make_uint2(__builtin_bit_cast(uint32_t, __floats2half2_rn(x[0], x[1])), __builtin_bit_cast(uint32_t, __floats2half2_rn(x[2], x[3])));
}

}  // namespace atom_rotary_device
#endif
