// Linear layers on this library's 4-bit weights with activations in fp16 (the W4A16 setting that the paper compares with), and
// the gated half of a feed-forward block made of two of them:
//   y[m, n] = fp16( residual[m, n] + sum_g scale[n, g] * sum_{k in g} code[n, k] * xr[m, k] )
//   h[m, n] = fp16( silu(gate) * up ),  gate and up two such sums of one xr
// xr: the activations in reordered order, behind RMSNorm where gamma is given (then rounded to fp16, which the matrix cores take).
//
// MFMA 16x16x32 f16: lane l supplies row (l & 15) of its operand and the 8 values of k-chunk (l >> 4); the result has column
// (l & 15) in lane l and rows 4 (l >> 4) + e in register e.  Activations are the row operand, weights the columns.

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include "atom_internal.h"
#include "atom_launch.h"

namespace {

using atom_internal::W4;

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float    f4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8, kThreads = 64 * kWaves;

__device__ __forceinline__ h2 as_h2(uint32_t v) { return __builtin_bit_cast(h2, v); }
__device__ __forceinline__ uint32_t bits(h2 v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ h8 as_h8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return __builtin_bit_cast(h8, make_uint4(a, b, c, d)); }

// Eight 4-bit codes, exact in fp16, as pairs (0, 4), (1, 5), (2, 6), (3, 7): a nibble with its sign bit turned over is code + 8; under the
// exponent of 1024 it is 1024 + that, or 16 times it where it lies four bits higher.
__device__ __forceinline__ h8 widen4(uint32_t w)
{
    w ^= 0x88888888u;
    const uint32_t v = w >> 8;
    const h2 low = {(_Float16)-1032.0f, (_Float16)-1032.0f}, high = {(_Float16)-72.0f, (_Float16)-72.0f}, sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
    const h2 a = as_h2((w & 0x000f000fu) | 0x64006400u) + low;
    const h2 b = __builtin_elementwise_fma(as_h2((w & 0x00f000f0u) | 0x64006400u), sixteenth, high);
    const h2 c = as_h2((v & 0x000f000fu) | 0x64006400u) + low;
    const h2 d = __builtin_elementwise_fma(as_h2((v & 0x00f000f0u) | 0x64006400u), sixteenth, high);
    return as_h8(bits(a), bits(b), bits(c), bits(d));
}
// The activations that meet them, from eight in a row.
__device__ __forceinline__ h8 paired(const uint4 &x)
{
    return as_h8(__builtin_amdgcn_perm(x.z, x.x, 0x05040100u), __builtin_amdgcn_perm(x.z, x.x, 0x07060302u),
                 __builtin_amdgcn_perm(x.w, x.y, 0x05040100u), __builtin_amdgcn_perm(x.w, x.y, 0x07060302u));
}
// Eight 8-bit codes in a row, likewise: 1024 + (code + 128).
__device__ __forceinline__ h8 widen8(uint32_t lo, uint32_t hi)
{
    const h2 off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
    lo ^= 0x80808080u;
    hi ^= 0x80808080u;
    auto two = [&](uint32_t w, uint32_t sel) { return bits(as_h2(__builtin_amdgcn_perm(0x64646464u, w, sel)) + off); };
    return as_h8(two(lo, 0x04010400u), two(lo, 0x04030402u), two(hi, 0x04010400u), two(hi, 0x04030402u));
}

struct Args {
    const __half *x; int64_t ldx, M;
    int K, O;
    W4 w[2]; int64_t N;
    const __half *residual; int64_t ldr;
    __half *y; int64_t ldy;
    uint32_t row_tiles;
};

// A workgroup has 16 output channels (of gate and of up) and 16 MT rows; its eight wavefronts have a run of groups each, and
// their sums meet in LDS, added in order.
template <int MT, bool GATED>
__global__ __launch_bounds__(kThreads)
void w4a16_kernel(Args p)
{
    constexpr int WM = GATED ? 2 : 1;
    __shared__ float red[kWaves][WM * MT][4][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, kc = lane >> 4;
    const int K4 = p.K - p.O, G = p.K >> 7, G4 = K4 >> 7;
    const uint32_t tile = blockIdx.x / p.row_tiles;
    const int64_t n0 = (int64_t)tile * 16, m0 = (int64_t)(blockIdx.x - tile * p.row_tiles) * (16 * MT);
    const int g_begin = (int)((int64_t)wave * G / kWaves), g_end = (int)((int64_t)(wave + 1) * G / kWaves);

    const int64_t row = min(n0 + col, p.N - 1);               // (columns >= N are computed and never stored, rows >= M likewise)
    const __half *x[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) x[mt] = p.x + min(m0 + 16 * mt + col, p.M - 1) * p.ldx + kc * 32;
    f4 acc[WM][MT] = {};
    for (int g = g_begin; g < g_end; ++g) {
        f4 part[WM][MT] = {};
        h8 w[WM][4];
        float scale[WM];
        const bool is4 = g < G4;
#pragma unroll
        for (int i = 0; i < WM; ++i) {
            scale[i] = __half2float(__ushort_as_half(p.w[i].scale[row * G + g]));
            if (is4) {
                const uint4 q = *reinterpret_cast<const uint4 *>(p.w[i].q4 + row * (K4 >> 1) + g * 64 + kc * 16);
                w[i][0] = widen4(q.x);
                w[i][1] = widen4(q.y);
                w[i][2] = widen4(q.z);
                w[i][3] = widen4(q.w);
            } else {
                const uint4 *q = reinterpret_cast<const uint4 *>(p.w[i].q8 + row * p.O + (g - G4) * 128 + kc * 32);
                const uint4 a = q[0], b = q[1];
                w[i][0] = widen8(a.x, a.y);
                w[i][1] = widen8(a.z, a.w);
                w[i][2] = widen8(b.x, b.y);
                w[i][3] = widen8(b.z, b.w);
            }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint4 v = *reinterpret_cast<const uint4 *>(x[mt] + g * 128 + c * 8);
                const h8 a = is4 ? paired(v) : as_h8(v.x, v.y, v.z, v.w);
#pragma unroll
                for (int i = 0; i < WM; ++i) part[i][mt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, w[i][c], part[i][mt], 0, 0, 0);
            }
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][mt][e] = fmaf(part[i][mt][e], scale[i], acc[i][mt][e]);
    }
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int e = 0; e < 4; ++e) red[wave][i * MT + mt][e][lane] = acc[i][mt][e];
    __syncthreads();
    for (int at = tid; at < MT * 256; at += kThreads) {
        const int l = at & 63, e = (at >> 6) & 3, mt = at >> 8;
        float sum[WM];
#pragma unroll
        for (int i = 0; i < WM; ++i) {
            sum[i] = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) sum[i] += red[w][i * MT + mt][e][l];
        }
        const int64_t m = m0 + 16 * mt + 4 * (l >> 4) + e, n = n0 + (l & 15);
        if (m >= p.M || n >= p.N) continue;
        float y = sum[0];
        if constexpr (GATED) y = y / (1.0f + expf(-y)) * sum[WM - 1];
        else if (p.residual) y += __half2float(p.residual[m * p.ldr + n]);
        p.y[m * p.ldy + n] = __float2half_rn(y);
    }
}

// The activations as the product takes them: a row to a workgroup.
__global__ __launch_bounds__(256)
void w4a16_rows_kernel(const __half *__restrict__ x, int64_t ldx, const __half *__restrict__ gamma, float eps, const int32_t *__restrict__ idx, int K,
                       __half *__restrict__ out)
{
    __shared__ float s_sum[4];
    const int tid = threadIdx.x;
    x += (int64_t)blockIdx.x * ldx;
    out += (int64_t)blockIdx.x * K;
    float r = 1.0f;
    if (gamma) {
        float sum = 0.0f;
        for (int k = tid; k < K; k += 256) {
            const float v = __half2float(x[k]);
            sum += v * v;
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d, 64);
        if ((tid & 63) == 0) s_sum[tid >> 6] = sum;
        __syncthreads();
        sum = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
        r = 1.0f / sqrtf(sum / (float)K + eps);
    }
    for (int k = tid; k < K; k += 256) {
        const uint32_t at = idx ? min((uint32_t)idx[k], (uint32_t)(K - 1)) : (uint32_t)k;
        const float v = __half2float(x[at]);
        out[k] = __float2half_rn(gamma ? v * r * __half2float(gamma[at]) : v);
    }
}

}  // namespace

namespace atom_internal {

size_t w4a16_workspace_bytes(int64_t M, int64_t N, int K, int O, bool gated, bool norm, bool index)
{
    (void)N, (void)O, (void)gated;
    return norm || index ? (size_t)M * K * 2 : 0;
}

static int row_tiles_of(int64_t M) { return M <= 16 ? 1 : M <= 32 ? 2 : 4; }

bool w4a16_fits(int64_t M, int64_t N, int K, int O, bool gated)
{
    (void)K, (void)O, (void)gated;
    if (M == 0 || N == 0) return true;
    const int64_t rows = (M + 63) / 64, tiles = (N + 15) / 16, most = atom_launch::kMostThreads / kThreads;
    return rows <= most && tiles <= most / rows && M <= most;
}

hipError_t launch_w4a16(const W4A16 &a, hipStream_t stream)
{
    Args p = {(const __half *)a.x, a.ldx, a.M, a.K, a.O, {a.w[0], a.w[1]}, a.N, (const __half *)a.residual, a.ldr, (__half *)a.y, a.ldy, 1};
    if (a.gamma || a.idx) {
        hipLaunchKernelGGL(w4a16_rows_kernel, dim3((unsigned)a.M), dim3(256), 0, stream, p.x, a.ldx, (const __half *)a.gamma, a.eps, a.idx, a.K,
                           (__half *)a.workspace);
        p.x = (const __half *)a.workspace;
        p.ldx = a.K;
    }
    const int     MT = row_tiles_of(a.M);
    p.row_tiles = (uint32_t)((a.M + 16 * MT - 1) / (16 * MT));
    const int64_t groups = (a.N + 15) / 16 * p.row_tiles;
    const bool    gated = a.w[1].q4 != nullptr;
#define ATOM_W4A16(MT, GATED) hipLaunchKernelGGL((w4a16_kernel<MT, GATED>), dim3((unsigned)groups), dim3(kThreads), 0, stream, p)
    if (gated) {
        if (MT == 1)      ATOM_W4A16(1, true);
        else if (MT == 2) ATOM_W4A16(2, true);
        else              ATOM_W4A16(4, true);
    } else {
        if (MT == 1)      ATOM_W4A16(1, false);
        else if (MT == 2) ATOM_W4A16(2, false);
        else              ATOM_W4A16(4, false);
    }
#undef ATOM_W4A16
    return hipGetLastError();
}

}  // namespace atom_internal
