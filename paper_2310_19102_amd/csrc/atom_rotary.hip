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

// A lane has eight channels of HEADS heads of a token.
template <bool ONE, bool NEIGHBOURS, int HEADS>
__global__ __launch_bounds__(256)
void rotary_kernel(const __half *x, int64_t ldx, uint32_t heads, uint32_t D, Turn t, float sign, __half *out, int64_t ldo,
                   uint32_t chunks, uint64_t lanes)
{
    const uint64_t e = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= lanes) return;
    const uint32_t per = D / 8, row = (uint32_t)(e / per), i = (uint32_t)(e - (uint64_t)row * per);
    const uint32_t token = row / chunks, h0 = (row - token * chunks) * HEADS;
    const Channels at = channels(t, (int)i);
    Angles r;
    if (at.turned) r = angles<ONE>(t, positions<ONE>(t, token), (int)i, lane_axes(t, (int)i));
    x += (int64_t)token * ldx;
    out += (int64_t)token * ldo;
    uint2 lo[HEADS], hi[HEADS];
#pragma unroll
    for (int u = 0; u < HEADS; ++u) {
        const uint32_t h = min(h0 + u, heads - 1);
        lo[u] = *reinterpret_cast<const uint2 *>(x + h * D + at.lo);
        hi[u] = *reinterpret_cast<const uint2 *>(x + h * D + at.hi);
    }
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

hipError_t launch_rotary(const void *x, int64_t T, int64_t ldx, int heads, int D, const Turn &t, bool transposed, void *out, int64_t ldo,
                         hipStream_t stream)
{
#define ATOM_ROTARY(ONE, NEIGHBOURS, HEADS)                                                                                                       \
    do {                                                                                                                              \
        const uint32_t chunks = (uint32_t)((heads + HEADS - 1) / HEADS);                                                              \
        const uint64_t lanes = (uint64_t)T * chunks * (D / 8);                                                                        \
        hipLaunchKernelGGL((rotary_kernel<ONE, NEIGHBOURS, HEADS>), dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, stream, (const __half *)x, ldx, \
                           (uint32_t)heads, (uint32_t)D, t, transposed ? -1.0f : 1.0f, (__half *)out, ldo, chunks, lanes);           \
    } while (0)
    if (t.axes == 1) {
        if (t.interleaved) ATOM_ROTARY(true, true, 1);
        else               ATOM_ROTARY(true, false, 1);
    } else {
        if (t.interleaved) ATOM_ROTARY(false, true, 1);
        else               ATOM_ROTARY(false, false, 1);
    }
#undef ATOM_ROTARY
    return hipGetLastError();
}

}  // namespace atom_internal
