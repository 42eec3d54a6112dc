// Rotary positions for gfx950: the table of cosines and sines, and the operator that turns the heads of a step's queries and
// keys (what atom_kv8_append and atom_attention_kv8 take; atom_rotary_kv8.hip turns and appends in one launch).

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include "atom_internal.h"
#include "atom_launch.h"
#include "atom_rotary.h"

namespace {

using namespace atom_rotary_device;

// Angles in 64 bits: at position 2^20 a 32-bit product of position and frequency is off by up to 2^-5.  Once per model, not tuned.
__global__ __launch_bounds__(256)
void rotary_table_kernel(const double *__restrict__ freq, int n_pairs, int64_t entries, float *__restrict__ table)
{
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= entries) return;
    const int64_t p = e / n_pairs;
    double s, c;
    sincos((double)p * freq[e - p * n_pairs], &s, &c);
    reinterpret_cast<float2 *>(table)[e] = make_float2((float)c, (float)s);
}

template <bool ONCE>
__device__ __forceinline__ uint2 load4(const __half *p)
{
    typedef unsigned u2 __attribute__((ext_vector_type(2)));
    if constexpr (ONCE) return __builtin_bit_cast(uint2, __builtin_nontemporal_load(reinterpret_cast<const u2 *>(p)));
    else return *reinterpret_cast<const uint2 *>(p);
}

// A lane has eight channels of HEADS heads of a token, all on their way at once.  ONCE: what is read is not kept in the caches.
template <bool ONE, bool NEIGHBOURS, int HEADS, bool ONCE>
__global__ __launch_bounds__(256)
void rotary_kernel(const __half *x, int64_t ldx, uint32_t heads, uint32_t D, Turn t, float sign, __half *out, int64_t ldo,
                   uint32_t chunks, uint32_t lanes)
{
    const uint32_t e = blockIdx.x * 256 + threadIdx.x;
    if (e >= lanes) return;
    const uint32_t per = D / 8, row = e / per, i = e - row * per;
    const uint32_t token = row / chunks, h0 = (row - token * chunks) * HEADS;
    const Channels at = channels(t, (int)i);
    const Positions where = positions<ONE>(t, token);        // (first, so that the table's row is asked for while the heads come)
    x += (int64_t)token * ldx;
    out += (int64_t)token * ldo;
    uint2 lo[HEADS], hi[HEADS];
#pragma unroll
    for (int u = 0; u < HEADS; ++u) {
        const uint32_t h = min(h0 + u, heads - 1);
        lo[u] = load4<ONCE>(x + h * D + at.lo);
        hi[u] = load4<ONCE>(x + h * D + at.hi);
    }
    const Angles r = angles<ONE>(t, where, (int)i, lane_axes(t, (int)i));
#pragma unroll
    for (int u = 0; u < HEADS; ++u) {
        if (h0 + u >= heads) break;
        float v[8];
        widen(lo[u], v);
        widen(hi[u], v + 4);
        if (at.turned) turn<NEIGHBOURS>(v, r, sign);
        *reinterpret_cast<uint2 *>(out + (h0 + u) * D + at.lo) = narrow(v);
        *reinterpret_cast<uint2 *>(out + (h0 + u) * D + at.hi) = narrow(v + 4);
    }
}

}  // namespace

namespace atom_internal {

hipError_t launch_rotary_table(const double *freq, int n_pairs, int64_t n_pos, float *table, hipStream_t stream)
{
    const int64_t entries = n_pos * n_pairs;
    hipLaunchKernelGGL(rotary_table_kernel, dim3((unsigned)((entries + 255) / 256)), dim3(256), 0, stream, freq, n_pairs, entries, table);
    return hipGetLastError();
}

// Values from which a lane takes four heads and their angles once (a step of 64 tokens of 40 heads of 128: 3.2 us with one, 3.55 with four; 200 tokens 4.2
// and 3.75; 1600 20.8 and 9.3), and from which the heads come past the caches (3200 such tokens: 14.8 us through them, 16.8 past them; 6400 29.3 and
// 27.4; 4999 tokens of 72 heads with three axes 37.4 and 33.3, and 31.4 with the positions asked for first: 5.9 TB/s, what is read and written bounds it).
// Of two heads a lane takes both, and one where there is no other: a place without a head reads the last one once more (300000 tokens of one head 32.9 us, with four places
// 44.6; 120000 of two 22.9 and 28.0; of three 25.1 with four places and 25.7 with two).
constexpr int64_t kFourHeads = 1 << 19, kReadOnce = (int64_t)24 << 20;

hipError_t launch_rotary(const void *x, int64_t T, int64_t ldx, int heads, int D, const Turn &t, bool transposed, void *out, int64_t ldo,
                         hipStream_t stream)
{
#define ATOM_ROTARY(ONE, NEIGHBOURS, HEADS, ONCE)                                                                                                       \
    do {                                                                                                                              \
        const uint32_t chunks = (uint32_t)((heads + HEADS - 1) / HEADS);                                                              \
        const uint64_t lanes = (uint64_t)T * chunks * (D / 8);                                                                        \
        hipLaunchKernelGGL((rotary_kernel<ONE, NEIGHBOURS, HEADS, ONCE>), dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, stream, (const __half *)x, ldx, \
                           (uint32_t)heads, (uint32_t)D, t, transposed ? -1.0f : 1.0f, (__half *)out, ldo, chunks, (uint32_t)lanes);           \
    } while (0)
#define ATOM_ROTARY_SIZE(ONE, NEIGHBOURS)                                                  \
    do {                                                                                   \
        if (work < kFourHeads || heads == 1)     ATOM_ROTARY(ONE, NEIGHBOURS, 1, false);   \
        else if (heads == 2 && work < kReadOnce) ATOM_ROTARY(ONE, NEIGHBOURS, 2, false);   \
        else if (heads == 2)                     ATOM_ROTARY(ONE, NEIGHBOURS, 2, true);    \
        else if (work < kReadOnce)               ATOM_ROTARY(ONE, NEIGHBOURS, 4, false);   \
        else                                     ATOM_ROTARY(ONE, NEIGHBOURS, 4, true);    \
    } while (0)
    const int64_t work = T * heads * D;
    if (t.axes == 1) {
        if (t.interleaved) ATOM_ROTARY_SIZE(true, true);
        else               ATOM_ROTARY_SIZE(true, false);
    } else {
        if (t.interleaved) ATOM_ROTARY_SIZE(false, true);
        else               ATOM_ROTARY_SIZE(false, false);
    }
#undef ATOM_ROTARY_SIZE
#undef ATOM_ROTARY
    return hipGetLastError();
}

}  // namespace atom_internal
