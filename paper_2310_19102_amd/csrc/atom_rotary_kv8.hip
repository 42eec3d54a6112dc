// Queries turned, keys turned, quantised and appended to the paged 8-bit cache, values quantised and appended: the whole step
// between the fused projection and atom_attention_kv8 in one launch.
//
// A turned key is never stored, nor rounded to fp16: it goes from fp32 registers into the block's maximum and codes, by the
// definition of atom_kv8_append with |turned value| in the place of |x|.

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include "atom_internal.h"
#include "atom_kv8_append.h"
#include "atom_launch.h"
#include "atom_rotary.h"

namespace {

using namespace atom_kv8;
using namespace atom_rotary_device;

__device__ __forceinline__ uint32_t codes4(const float *x, float r)
{
    return pack4(code_of(x[0] * r), code_of(x[1] * r), code_of(x[2] * r), code_of(x[3] * r));
}

// Run (atom_kv8_append.h) of turned rows: the same members and steps on fp32 values, the maximum as the bits of a float.
template <int D, int ROWS, bool ONE, bool NEIGHBOURS>
struct TurnedRun {
    static constexpr int LPR = D / 8, RPL = 64 / LPR, kLoads = ROWS / RPL;
    float x[kLoads][8];
    const __half *rows; int64_t ld, token;
    int8_t *block; float *scale;
    int o, at, len, g, i;
    Channels ch;
    uint32_t axes;
    float s_old;

    __device__ __forceinline__ void load(const Turn &t, int row, float *v) const
    {
        const int r = min(row, len - 1);
        const __half *p = rows + (int64_t)r * ld;
        const uint2 lo = *reinterpret_cast<const uint2 *>(p + ch.lo), hi = *reinterpret_cast<const uint2 *>(p + ch.hi);
        widen(lo, v);
        widen(hi, v + 4);
        if (ch.turned) turn<NEIGHBOURS>(v, angles<ONE>(t, positions<ONE>(t, token + r), i, axes), 1.0f);
    }
    static __device__ __forceinline__ uint32_t magnitude(const float *v)
    {
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = max(top, __builtin_bit_cast(uint32_t, v[k]) & 0x7fffffffu);
        return top;
    }

    __device__ __forceinline__ uint32_t begin(const Turn &t, const Side &side, int h, int Hkv, int32_t first, int len_, int64_t tok, int shift,
                                              int row0 = 0)
    {
        const int lane = threadIdx.x & 63;
        g = lane / LPR;
        i = lane % LPR;
        ch = channels(t, i);
        axes = lane_axes(t, i);
        len = len_;
        ld = side.ld;
        token = tok + row0;
        o = first & ((1 << shift) - 1);
        at = o + row0;
        const int64_t head = (int64_t)(first >> shift) * Hkv + h;
        block = side.codes + (head << shift) * D;
        scale = side.scale + head;
        rows = side.x + (int64_t)h * D + token * ld;
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (u * RPL < len) load(t, u * RPL + g, x[u]);
        s_old = o > 0 ? *scale : 0.0f;
        uint32_t top = 0;
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (u * RPL < len) top = max(top, magnitude(x[u]));
        for (int row = ROWS; row < len; row += RPL) {
            float v[8];
            load(t, row + g, v);
            top = max(top, magnitude(v));
        }
        return wave_max(top);
    }

    __device__ __forceinline__ void store(int row, const float *v, float r)
    {
        if (row >= len) return;
        // (a NaN that came with the table may have anything in its low byte)
        const uint32_t a = r > 0.0f ? codes4(v, r) : 0, b = r > 0.0f ? codes4(v + 4, r) : 0;
        *reinterpret_cast<uint32_t *>(block + (at + row) * D + ch.lo) = a;
        *reinterpret_cast<uint32_t *>(block + (at + row) * D + ch.hi) = b;
    }

    __device__ __forceinline__ void end(const Turn &t, uint32_t top, int thread, int threads)
    {
        const float s_new = __builtin_bit_cast(float, top) / 127.0f, s = s_new > s_old || s_new != s_new ? s_new : s_old;
        // (a scale below the normal numbers has no reciprocal)
        const float r = s >= 1.17549435e-38f ? 1.0f / s : 0.0f;
        if (s > s_old && s_old > 0.0f) {
            const float ratio = s_old / s;
            for (int b = 16 * thread; b < o * D; b += 16 * threads) {
                uint4 w = *reinterpret_cast<const uint4 *>(block + b);
                w = make_uint4(recode4(w.x, ratio), recode4(w.y, ratio), recode4(w.z, ratio), recode4(w.w, ratio));
                *reinterpret_cast<uint4 *>(block + b) = w;
            }
        }
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (u * RPL < len) store(u * RPL + g, x[u], r);
        for (int row = ROWS; row < len; row += RPL) {
            float v[8];
            load(t, row + g, v);
            store(row + g, v, r);
        }
        if (thread == 0) *scale = s;
    }
};

struct Queries { const __half *x; int64_t ld; __half *out; int64_t ldo; int heads; };

// Eight channels of a query head to a lane.
template <int D, bool ONE, bool NEIGHBOURS>
__device__ __forceinline__ void turn_queries(const Queries &q, const Turn &t, int64_t T, int64_t group)
{
    const int64_t e = group * 256 + threadIdx.x, row = e / (D / 8);
    const int i = (int)(e % (D / 8));
    const int64_t token = row / q.heads;
    if (token >= T) return;
    const int h = (int)(row - token * q.heads);
    const Channels ch = channels(t, i);
    const __half *x = q.x + token * q.ld + (int64_t)h * D;
    __half *out = q.out + token * q.ldo + (int64_t)h * D;
    const uint2 lo = *reinterpret_cast<const uint2 *>(x + ch.lo), hi = *reinterpret_cast<const uint2 *>(x + ch.hi);
    float v[8];
    widen(lo, v);
    widen(hi, v + 4);
    if (ch.turned) turn<NEIGHBOURS>(v, angles<ONE>(t, positions<ONE>(t, token), i, lane_axes(t, i)), 1.0f);
    *reinterpret_cast<uint2 *>(out + ch.lo) = narrow(v);
    *reinterpret_cast<uint2 *>(out + ch.hi) = narrow(v + 4);
}

// One wavefront for a head (of K or of V) and a token; where a run begins with that token it writes the run, whole.  The first
// `appends` workgroups do this, four wavefronts each, the others turn queries.
template <int D, bool ONE, bool NEIGHBOURS>
__global__ __launch_bounds__(256)
void rotary_kv8_kernel(Queries q, Side k, Side v, int T, int Hkv, Turn turn, const int32_t *__restrict__ slot, int32_t slots, int shift, uint32_t appends)
{
    if (blockIdx.x >= appends) return turn_queries<D, ONE, NEIGHBOURS>(q, turn, T, blockIdx.x - appends);
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = item / (2 * Hkv);
    const int which = (int)(item - t * (2 * Hkv)), h = which % Hkv;
    if (t >= T) return;
    const Window w = window(slot, slots, T, t, 1, 1 << shift);
    if (!w.leaders) return;
    const int32_t first = __builtin_amdgcn_readlane(w.got, 0);
    const int len = run_length(slot, T, w, t, 0, 1 << shift), lane = threadIdx.x & 63;
    if (which < Hkv) {
        TurnedRun<D, 16, ONE, NEIGHBOURS> run;
        run.end(turn, run.begin(turn, k, h, Hkv, first, len, t, shift), lane, 64);
    } else {
        Run<D, 16> run;
        run.end(run.begin(v, h, Hkv, first, len, t, shift), lane, 64);
    }
}

}  // namespace

namespace atom_internal {

static int64_t append_groups(int64_t T, int Hkv) { return (T * 2 * Hkv + 3) / 4; }
static int64_t query_groups(int64_t T, int H, int D) { return (T * H * (D / 8) + 255) / 256; }

bool rotary_kv8_fits(int64_t T, int H, int Hkv, int D, int block_tokens)
{
    (void)block_tokens;
    return append_groups(T, Hkv) + query_groups(T, H, D) <= atom_launch::kMostThreads / 256;
}

hipError_t launch_rotary_kv8_append(const RotaryKv8 &a, hipStream_t stream)
{
    const Queries q = {(const __half *)a.q, a.ldq, (__half *)a.q_out, a.ldqo, a.H};
    const Side k = {(const __half *)a.k, a.ldk, (int8_t *)a.k_codes, a.k_scale}, v = {(const __half *)a.v, a.ldv, (int8_t *)a.v_codes, a.v_scale};
    const int32_t slots = (int32_t)(a.n_blocks * a.block_tokens);
    const int     shift = __builtin_ctz((unsigned)a.block_tokens);
    const int64_t appends = append_groups(a.T, a.Hkv), groups = appends + query_groups(a.T, a.H, a.D);
#define ATOM_TURN(D, ONE, NEIGHBOURS)                                                                                                          \
    hipLaunchKernelGGL((rotary_kv8_kernel<D, ONE, NEIGHBOURS>), dim3((unsigned)groups), dim3(256), 0, stream, q, k, v, (int)a.T, a.Hkv, a.turn, \
                       a.slot, slots, shift, (uint32_t)appends)
#define ATOM_TURN_D(D)                                                \
    do {                                                              \
        if (a.turn.axes == 1) {                                       \
            if (a.turn.interleaved) ATOM_TURN(D, true, true);         \
            else                    ATOM_TURN(D, true, false);        \
        } else {                                                      \
            if (a.turn.interleaved) ATOM_TURN(D, false, true);        \
            else                    ATOM_TURN(D, false, false);       \
        }                                                             \
    } while (0)
    if (a.D == 128) ATOM_TURN_D(128);
    else            ATOM_TURN_D(64);
#undef ATOM_TURN_D
#undef ATOM_TURN
    return hipGetLastError();
}

}  // namespace atom_internal
