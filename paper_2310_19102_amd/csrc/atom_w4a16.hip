// Linear layers on this library's 4-bit weights with activations in fp16 (the W4A16 setting that the paper compares with), and
// the gated half of a feed-forward block made of two of them:
//   y[m, n] = fp16( residual[m, n] + sum_g scale[n, g] * sum_{k in g} code[n, k] * xr[m, k] )
//   h[m, n] = fp16( silu(gate) * up ),  gate and up two such sums of one xr
// xr: the activations in reordered order, behind RMSNorm where gamma is given.  The matrix cores take fp16; what the norm gives has more bits,
// and rounding it would be the largest error of the whole layer (1.4 to 1.8 times that of the output's own rounding), so it goes in as
// two halves, hi + lo, 22 bits.
//
// MFMA 16x16x32 f16: lane l supplies row (l & 15) of its operand and the 8 values of k-chunk (l >> 4); the result has column
// (l & 15) in lane l and rows 4 (l >> 4) + e in register e.  Activations are the row operand, weights the columns.  Which channels a
// chunk has is free as long as both operands agree: a lane reads 16 bytes of a weight row, channels 32 c .. 32 c + 31 of a
// group in its chunk c, and the i-th instruction takes eight of them; activations are laid out so that its four chunks are
// 64 bytes in a row, with the eight in the order in which the codes come out of their word.

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
    const __half *gamma; float eps; const int32_t *idx;
    int K, O;
    W4 w[2]; int64_t N;
    const __half *residual; int64_t ldr;
    __half *y; int64_t ldy;
    const __half *staged; int rows;                          // laid out, `rows` rows of hi and behind them those of lo
    bool combine;                                            // lo in rows 8 .. 15 of the one tile
    uint32_t tiles, row_tiles;
};

// ---- the activations as the product takes them

// Row x in reordered order, behind the norm where there is gamma, laid out for the product (lo: null where there is no
// norm).  nat: K words of LDS (halves without norm, none without an index either); all threads of the workgroup call.
template <int THREADS>
__device__ __forceinline__ void lay_out(const Args &p, const __half *__restrict__ x, uint32_t *nat, float *s_sum, __half *hi, __half *lo)
{
    const int tid = threadIdx.x, blocks = p.K / 8, K4 = p.K - p.O;
    const uint4 *row = reinterpret_cast<const uint4 *>(x);
    auto half_of = [](const uint4 &v, int i) -> uint32_t { return ((i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w) >> (16 * (i & 1))) & 0xffffu; };
    auto value = [](uint32_t h) { return __half2float(__ushort_as_half((unsigned short)h)); };
    if (p.gamma) {
        float sum = 0.0f;
        for (int b = tid; b < blocks; b += THREADS) {
            const uint4 v = row[b];
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(value(half_of(v, i)), value(half_of(v, i)), sum);
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d, 64);
        if ((tid & 63) == 0) s_sum[tid >> 6] = sum;
        __syncthreads();
        sum = 0.0f;
        for (int w = 0; w < THREADS / 64; ++w) sum += s_sum[w];
        const float r = 1.0f / sqrtf(sum / (float)p.K + p.eps);
        for (int b = tid; b < blocks; b += THREADS) {
            const uint4 v = row[b], g = reinterpret_cast<const uint4 *>(p.gamma)[b];
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = value(half_of(v, i)) * r * value(half_of(g, i));
                const __half h = __float2half_rn(y);
                // (of what is not finite hi says it all: infinity minus infinity would be NaN)
                const __half l = __hisinf(h) || __hisnan(h) ? __ushort_as_half(0) : __float2half_rn(y - __half2float(h));
                w[i] = (uint32_t)__half_as_ushort(h) | (uint32_t)__half_as_ushort(l) << 16;
            }
            reinterpret_cast<uint4 *>(nat)[2 * b] = make_uint4(w[0], w[1], w[2], w[3]);
            reinterpret_cast<uint4 *>(nat)[2 * b + 1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
        __syncthreads();
    } else if (p.idx) {
        for (int b = tid; b < blocks; b += THREADS) reinterpret_cast<uint4 *>(nat)[b] = row[b];
        __syncthreads();
    }
    for (int b = tid; b < blocks; b += THREADS) {
        const int g = b >> 4, k = g * 128 + (b & 3) * 32 + ((b >> 2) & 3) * 8;        // the eight channels of place b
        uint32_t w[8];
        if (p.idx) {
            const int4 i0 = *reinterpret_cast<const int4 *>(p.idx + k), i1 = *reinterpret_cast<const int4 *>(p.idx + k + 4);
            const int32_t at[8] = {i0.x, i0.y, i0.z, i0.w, i1.x, i1.y, i1.z, i1.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t c = min((uint32_t)at[i], (uint32_t)(p.K - 1));
                w[i] = p.gamma ? nat[c] : reinterpret_cast<const uint16_t *>(nat)[c];
            }
        } else if (p.gamma) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = nat[k + i];
        } else {
            const uint4 v = row[k / 8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = half_of(v, i);
        }
        if (k < K4) {
            const uint32_t t1 = w[1], t2 = w[2], t3 = w[3];                           // 0 4 1 5 2 6 3 7
            w[1] = w[4];
            w[2] = t1;
            w[3] = w[5];
            w[4] = t2;
            w[5] = w[6];
            w[6] = t3;
        }
        auto pack = [&](uint32_t sel) {
            return make_uint4(__builtin_amdgcn_perm(w[1], w[0], sel), __builtin_amdgcn_perm(w[3], w[2], sel), __builtin_amdgcn_perm(w[5], w[4], sel),
                              __builtin_amdgcn_perm(w[7], w[6], sel));
        };
        *reinterpret_cast<uint4 *>(hi + 8 * b) = pack(0x05040100u);
        if (lo) *reinterpret_cast<uint4 *>(lo + 8 * b) = pack(0x07060302u);
    }
}

__host__ __device__ constexpr size_t natural_bytes(int K, bool norm, bool index) { return norm ? 4 * (size_t)K : index ? 2 * (size_t)K : 0; }

// A row to a workgroup, into the workspace.
__global__ __launch_bounds__(512)
void w4a16_rows_kernel(Args p, __half *out)
{
    extern __shared__ uint32_t s_nat[];
    __shared__ float s_sum[8];
    lay_out<512>(p, p.x + (int64_t)blockIdx.x * p.ldx, s_nat, s_sum, out + (int64_t)blockIdx.x * p.K,
                 p.gamma ? out + ((int64_t)p.M + blockIdx.x) * p.K : nullptr);
}

// ---- the product

// A workgroup has 16 NT output channels (of gate and of up) and 16 RT rows; its eight wavefronts share the groups, and their sums
// meet in LDS, added in order.  A wavefront has a run of INT4 groups and every eighth INT8 group; CH of them are on their way while it
// works, across the tiles that the workgroup has in turn.
//   HL: halves of the activations that go in one after the other (2: hi and lo)
//   KEPT: the activations are laid out in LDS by the workgroup itself (RT = HL = 1), under way with the first weights
template <int NT, bool GATED, int RT, int HL, int CH, bool KEPT>
__global__ __launch_bounds__(kThreads, KEPT ? 4 : 2)
void w4a16_kernel(Args p)
{
    constexpr int WM = GATED ? 2 : 1, CT = WM * NT, AT = KEPT ? 1 : RT * HL;
    static_assert(CT <= 4, "a lane's chunk loads the scales of one tile");
    extern __shared__ __align__(16) unsigned char s_all[];   // KEPT: the rows, then the sums or what is laid out; else the sums
    __shared__ float s_part[8];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, kc = lane >> 4;
    const int K4 = p.K - p.O, G = p.K >> 7, G4 = K4 >> 7, G8 = G - G4;
    const int begin = (int)((int64_t)wave * G4 / kWaves), n4 = (int)((int64_t)(wave + 1) * G4 / kWaves) - begin;
    const int n = n4 + (G8 > wave ? (G8 - wave + kWaves - 1) / kWaves : 0);           // elements of this wavefront

    // (rows >= M are computed and never stored, columns >= N likewise)
    const uint32_t row_tile = blockIdx.x % p.row_tiles, first = blockIdx.x / p.row_tiles, stride = gridDim.x / p.row_tiles;
    const int64_t m0 = (int64_t)row_tile * (16 * RT);
    const int rows = p.rows, lds_row = p.K + 8;
    const __half *act[AT];
    const __half *s_act = nullptr;
    if constexpr (KEPT) {
        const int r = p.combine && col >= 8 ? rows + min(col - 8, rows - 1) : min(col, rows - 1);
        s_act = reinterpret_cast<const __half *>(s_all) + (size_t)r * lds_row + kc * 8;
    } else {
#pragma unroll
        for (int t = 0; t < AT; ++t) {
            const int64_t m = p.combine ? (col >= 8 ? rows + min(col - 8, rows - 1) : min(col, rows - 1))
                                        : min(m0 + 16 * (t % RT) + col, (int64_t)rows - 1) + (t / RT) * (int64_t)rows;
            act[t] = p.staged + m * p.K + kc * 8;
        }
    }
    float *red = reinterpret_cast<float *>(s_all + (KEPT ? (size_t)rows * (p.gamma ? 2 : 1) * lds_row * 2 : 0));

    struct Element { uint4 q[CT], q1[CT]; uint16_t scale; uint4 a[AT][4]; };
    Element ring[CH];
    // the element that is loaded next
    uint32_t load_tile = first;
    int load_i = 0;
    int64_t row4[CT], row8[CT], row_s;
    auto rows_of = [&](uint32_t tile) {
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const int64_t r = min((int64_t)tile * (16 * NT) + 16 * (t % NT) + col, p.N - 1);
            row4[t] = r * (K4 >> 1) + kc * 16;
            row8[t] = r * p.O + kc * 32;
        }
        row_s = min((int64_t)tile * (16 * NT) + 16 * ((kc % CT) % NT) + col, p.N - 1) * G;
    };
    auto load = [&](Element &e) {
        if (load_tile >= p.tiles) return;
        const bool is4 = load_i < n4;
        const int  g = is4 ? begin + load_i : wave + kWaves * (load_i - n4);          // of the INT4 or of the INT8 groups
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const W4 &w = p.w[t / NT];
            const uint8_t *at = is4 ? w.q4 + row4[t] + g * 64 : reinterpret_cast<const uint8_t *>(w.q8) + row8[t] + g * 128;
            e.q[t] = *reinterpret_cast<const uint4 *>(at);
            if (!is4) e.q1[t] = *reinterpret_cast<const uint4 *>(at + 16);
        }
        const int k = is4 ? g : G4 + g;
        e.scale = (CT > 1 && (kc % CT) / NT ? p.w[WM - 1] : p.w[0]).scale[row_s + k];
        if constexpr (!KEPT) {
#pragma unroll
            for (int t = 0; t < AT; ++t)
#pragma unroll
                for (int c = 0; c < 4; ++c) e.a[t][c] = *reinterpret_cast<const uint4 *>(act[t] + k * 128 + c * 32);
        }
        if (++load_i == n) {
            load_i = 0;
            load_tile += stride;
            rows_of(load_tile);
        }
    };
    f4 acc[CT][RT] = {};
    auto compute = [&](const Element &e, int i) {
        const bool is4 = i < n4;
        const int  k = is4 ? begin + i : G4 + wave + kWaves * (i - n4);
        f4 part[CT][RT] = {};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            h8 w[CT];
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                if (is4) w[t] = widen4(c == 0 ? e.q[t].x : c == 1 ? e.q[t].y : c == 2 ? e.q[t].z : e.q[t].w);
                else     w[t] = c == 0 ? widen8(e.q[t].x, e.q[t].y) : c == 1 ? widen8(e.q[t].z, e.q[t].w) : c == 2 ? widen8(e.q1[t].x, e.q1[t].y) : widen8(e.q1[t].z, e.q1[t].w);
            }
#pragma unroll
            for (int a = 0; a < AT; ++a) {
                h8 x;
                if constexpr (KEPT) x = *reinterpret_cast<const h8 *>(s_act + k * 128 + c * 32);
                else x = __builtin_bit_cast(h8, e.a[a][c]);
#pragma unroll
                for (int t = 0; t < CT; ++t) part[t][a % RT] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, w[t], part[t][a % RT], 0, 0, 0);
            }
        }
        const float mine = __half2float(__ushort_as_half(e.scale));
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const float s = CT == 1 ? mine : __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(4 * (16 * t + col), __builtin_bit_cast(int, mine)));
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[t][r][j] = fmaf(part[t][r][j], s, acc[t][r][j]);
        }
    };
    int buffer = 0;
    auto finish = [&](uint32_t tile) {
        float *mine = red + (size_t)buffer * (kWaves * CT * RT * 256);
        buffer ^= 1;                                         // (nobody writes a buffer before all have read what it held two tiles ago)
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    mine[((wave * CT + t) * RT + r) * 256 + j * 64 + lane] = acc[t][r][j];
                    acc[t][r][j] = 0.0f;
                }
        __syncthreads();
        for (int at = tid; at < NT * RT * 256; at += kThreads) {
            const int l = at & 63, j = (at >> 6) & 3, r = (at >> 8) % RT, t = (at >> 8) / RT;
            const int64_t m = m0 + 16 * r + 4 * (l >> 4) + j, out = (int64_t)tile * (16 * NT) + 16 * t + (l & 15);
            if (m >= p.M || out >= p.N) continue;
            float sum[WM];
#pragma unroll
            for (int i = 0; i < WM; ++i) {
                float lo = 0.0f;
                sum[i] = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float *s = mine + ((w * CT + i * NT + t) * RT + r) * 256 + j * 64 + l;
                    sum[i] += s[0];
                    if (p.combine) lo += s[32];
                }
                sum[i] += lo;
            }
            float y = sum[0];
            if constexpr (GATED) y = y / (1.0f + expf(-y)) * sum[WM - 1];
            else if (p.residual) y += __half2float(p.residual[m * p.ldr + out]);
            p.y[m * p.ldy + out] = __float2half_rn(y);
        }
    };

    rows_of(first);
    if (n > 0) {
#pragma unroll
        for (int s = 0; s < CH; ++s) load(ring[s]);
    }
    if constexpr (KEPT) {
        uint32_t *nat = reinterpret_cast<uint32_t *>(red);
        __half *out = reinterpret_cast<__half *>(s_all);
        for (int m = 0; m < rows; ++m) {
            if (m) __syncthreads();
            lay_out<kThreads>(p, p.x + m * p.ldx, nat, s_part, out + (size_t)m * lds_row, p.gamma ? out + (size_t)(rows + m) * lds_row : nullptr);
        }
        __syncthreads();
    }
    if (n == 0) {
        for (uint32_t tile = first; tile < p.tiles; tile += stride) finish(tile);
        return;
    }
    uint32_t tile = first;
    for (int i = 0;;) {
#pragma unroll
        for (int s = 0; s < CH; ++s) {
            compute(ring[s], i);
            load(ring[s]);
            if (++i == n) {
                i = 0;
                finish(tile);
                tile += stride;
                if (tile >= p.tiles) return;
            }
        }
    }
}

}  // namespace

namespace atom_internal {

// How a call runs: whether the workgroups lay the activations out themselves, column and row tiles, LDS.
struct ProductShape { bool kept, combine; int NT, RT; size_t lds; };

static ProductShape product_shape(int64_t M, int64_t N, int K, bool gated, bool norm, bool index)
{
    const int WM = gated ? 2 : 1;
    ProductShape s = {};
    s.NT = 1;
    s.RT = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    s.combine = norm && M <= 8;
    const size_t sums = (size_t)2 * kWaves * WM * 1024, nat = natural_bytes(K, norm, index), rest = nat > sums ? nat : sums;
    if (M <= (norm ? 8 : 16)) {
        s.lds = (size_t)M * (norm ? 2 : 1) * (K + 8) * 2 + rest;
        s.kept = s.lds <= 80 * 1024;
    }
    if (!s.kept) {
        while (M <= 16 && s.NT * WM < 4 && (N + 32 * s.NT - 1) / (32 * s.NT) >= 192) s.NT *= 2;
        s.lds = (size_t)2 * kWaves * WM * s.NT * s.RT * 1024;
    }
    return s;
}

size_t w4a16_workspace_bytes(int64_t M, int64_t N, int K, int O, bool gated, bool norm, bool index)
{
    (void)O;
    return product_shape(M, N, K, gated, norm, index).kept ? 0 : (size_t)M * K * (norm ? 4 : 2);
}

bool w4a16_fits(int64_t M, int64_t N, int K, int O, bool gated)
{
    (void)K, (void)O, (void)gated;
    if (M == 0 || N == 0) return true;
    const int64_t rows = (M + 63) / 64, tiles = (N + 15) / 16, most = atom_launch::kMostThreads / kThreads;
    return rows <= most && tiles <= most / rows && M <= most;
}

hipError_t launch_w4a16(const W4A16 &a, hipStream_t stream)
{
    const bool gated = a.w[1].q4 != nullptr, norm = a.gamma != nullptr;
    const ProductShape s = product_shape(a.M, a.N, a.K, gated, norm, a.idx != nullptr);
    Args p = {(const __half *)a.x, a.ldx, a.M, (const __half *)a.gamma, a.eps, a.idx, a.K, a.O, {a.w[0], a.w[1]}, a.N, (const __half *)a.residual, a.ldr,
              (__half *)a.y, a.ldy, (const __half *)a.workspace, (int)a.M, s.combine, 0, 1};
    p.tiles = (uint32_t)((a.N + 16 * s.NT - 1) / (16 * s.NT));
    p.row_tiles = (uint32_t)((a.M + 16 * s.RT - 1) / (16 * s.RT));
    const uint32_t room = (uint32_t)(2 * atom_launch::compute_units());
    const uint32_t grid = (p.tiles < room ? p.tiles : room) * p.row_tiles;
    if (!s.kept) {
        static atom_launch::LdsOptIn opt;
        const size_t nat = natural_bytes(a.K, norm, a.idx != nullptr);
        if (nat > 60 * 1024) {
            const hipError_t err = atom_launch::ensure_dynamic_lds(opt, reinterpret_cast<const void *>(&w4a16_rows_kernel), nat);
            if (err != hipSuccess) return err;
        }
        hipLaunchKernelGGL(w4a16_rows_kernel, dim3((unsigned)a.M), dim3(512), nat, stream, p, (__half *)a.workspace);
    }
#define ATOM_W4A16(...)                                                                        \
    do {                                                                                       \
        static atom_launch::LdsOptIn opt;                                                      \
        auto kern = &w4a16_kernel<__VA_ARGS__>;                                                \
        if (s.lds > 60 * 1024) {                                                               \
            const hipError_t err = atom_launch::ensure_dynamic_lds(opt, reinterpret_cast<const void *>(kern), s.lds); \
            if (err != hipSuccess) return err;                                                 \
        }                                                                                      \
        hipLaunchKernelGGL(kern, dim3(grid), dim3(kThreads), s.lds, stream, p);                \
        return hipGetLastError();                                                              \
    } while (0)
    const bool twice = norm && !s.combine;
    if (s.kept) {
        if (gated) ATOM_W4A16(1, true, 1, 1, 3, true);
        else       ATOM_W4A16(1, false, 1, 1, 4, true);
    }
#define ATOM_ROWS(NT, GATED, RT, CH)                                 \
    do {                                                             \
        if (twice) ATOM_W4A16(NT, GATED, RT, 2, CH, false);          \
        else       ATOM_W4A16(NT, GATED, RT, 1, CH, false);          \
    } while (0)
    if (gated) {
        if (s.RT == 4) ATOM_ROWS(1, true, 4, 1);
        if (s.RT == 2) ATOM_ROWS(1, true, 2, 1);
        if (s.NT == 2) ATOM_ROWS(2, true, 1, 2);
        ATOM_ROWS(1, true, 1, 2);
    }
    if (s.RT == 4) ATOM_ROWS(1, false, 4, 1);
    if (s.RT == 2) ATOM_ROWS(1, false, 2, 1);
    if (s.NT == 4) ATOM_ROWS(4, false, 1, 2);
    if (s.NT == 2) ATOM_ROWS(2, false, 1, 2);
    ATOM_ROWS(1, false, 1, 2);
#undef ATOM_ROWS
#undef ATOM_W4A16
}

}  // namespace atom_internal
