// Linear layers on this library's 4-bit weights with activations in fp16 (the W4A16 setting that the paper compares with), and
// the gated half of a feed-forward block made of two of them:
//   y[m, n] = fp16( residual[m, n] + sum_g scale[n, g] * sum_{k in g} code[n, k] * xr[m, k] )
//   h[m, n] = fp16( silu(gate) * up ),  gate and up two such sums of one xr
// xr: the activations in reordered order, behind RMSNorm where gamma is given.  The matrix cores take fp16; what the norm gives has more bits,
// and rounding it would be the largest error of the whole layer (1.4 to 1.8 times that of the output's own rounding), so it goes in as
// two halves, hi + lo, 22 bits.  A half's last step is 2^-24, so a row of small values (a small gamma, a row below eps) is brought to 2^14 by a power of two
// first, which is taken back from its fp32 sums: what lo loses is 2^-22 of the value, or 2^-38 of the row's largest where that is more.  (Without it 2^-25 was lost
// whatever the value: with a gamma of 2e-5 up to nine times all other errors.  It costs 0.1 to 0.4 us of the launch that lays out the rows.)
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
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kScales = 64;                                   // of a weight row, in LDS at once

__device__ __forceinline__ h2 as_h2(uint32_t v) { return __builtin_bit_cast(h2, v); }
__device__ __forceinline__ uint32_t bits(h2 v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ h8 as_h8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return __builtin_bit_cast(h8, make_uint4(a, b, c, d)); }

// Eight 4-bit codes, exact in fp16, as pairs (0, 4), (1, 5), (2, 6), (3, 7): a nibble with its sign bit turned over is code + 8; under the
// exponent of 1024 it is 1024 + that, or 16 times it where it lies four bits higher.
__device__ __forceinline__ h8 widen4(uint32_t w)
{
    const uint32_t v = w >> 8;
    const h2 low = {(_Float16)-1032.0f, (_Float16)-1032.0f}, high = {(_Float16)-72.0f, (_Float16)-72.0f}, sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
    const h2 a = as_h2((w & 0x000f000fu) ^ 0x64086408u) + low;
    const h2 b = __builtin_elementwise_fma(as_h2((w & 0x00f000f0u) ^ 0x64806480u), sixteenth, high);
    const h2 c = as_h2((v & 0x000f000fu) ^ 0x64086408u) + low;
    const h2 d = __builtin_elementwise_fma(as_h2((v & 0x00f000f0u) ^ 0x64806480u), sixteenth, high);
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
    float *back;                                             // behind a norm: what takes a row's power of two back
    bool combine;                                            // lo in rows 8 .. 15 of the one tile
    uint32_t tiles;
    int parts, span; float *sums;                            // parts of K, INT4 groups of one (few rows), their sums
    // the kernel of many rows: tiles of 32 rows in a block, halves of the activations
    int wide, halves; uint32_t row_blocks;
};

// ---- the activations as the product takes them

// Where the eight channels from k on lie in a row that is laid out for the kernel of few rows, in blocks of eight.  Of an INT4 group chunk c of
// the instructions has channels 32 c .. 32 c + 31, eight an instruction; of 64 INT8 channels 16 c .. 16 c + 15.
__device__ __forceinline__ int row_place(int k, int K4)
{
    const int g = k >> 7, j = (k >> 3) & 15;
    return 16 * g + (k < K4 ? 4 * (j & 3) + (j >> 2) : (j & 8) + 4 * (j & 1) + ((j >> 1) & 3));
}

__device__ __forceinline__ uint32_t half_of(const uint4 &v, int i) { return ((i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w) >> (16 * (i & 1))) & 0xffffu; }
__device__ __forceinline__ float value_of(uint32_t h) { return __half2float(__ushort_as_half((unsigned short)h)); }

// A normed value as hi (the low half) and lo.  (Of what is not finite hi says it all: infinity minus infinity would be NaN.)
__device__ __forceinline__ uint32_t halves_of(float y)
{
    const __half h = __float2half_rn(y), l = __hisinf(h) || __hisnan(h) ? __ushort_as_half(0) : __float2half_rn(y - __half2float(h));
    return (uint32_t)__half_as_ushort(h) | (uint32_t)__half_as_ushort(l) << 16;
}

// The eight halves in the low or the high parts of w, in the order in which the codes come out of their word (INT4), or as they are.
__device__ __forceinline__ void in_order(uint32_t (&w)[8], bool is4)
{
    if (!is4) return;
    const uint32_t t1 = w[1], t2 = w[2], t3 = w[3];          // 0 4 1 5 2 6 3 7
    w[1] = w[4], w[2] = t1, w[3] = w[5], w[4] = t2, w[5] = w[6], w[6] = t3;
}
template <bool HIGH>
__device__ __forceinline__ uint4 packed(const uint32_t (&w)[8])
{
    constexpr uint32_t sel = HIGH ? 0x07060302u : 0x05040100u;
    return make_uint4(__builtin_amdgcn_perm(w[1], w[0], sel), __builtin_amdgcn_perm(w[3], w[2], sel), __builtin_amdgcn_perm(w[5], w[4], sel),
                      __builtin_amdgcn_perm(w[7], w[6], sel));
}

// A row behind the norm: the sum of its squares, the largest magnitude of x times gamma; what a thread found of them.
struct Norm {
    float sum = 0.0f, top = 0.0f;
    __device__ __forceinline__ void add(const uint4 &x, const float (&xg)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sum = fmaf(value_of(half_of(x, i)), value_of(half_of(x, i)), sum);
            top = fmaxf(top, fabsf(xg[i]));
        }
    }
};

// x times gamma, exact.
__device__ __forceinline__ void products(float (&xg)[8], const uint4 &x, const uint4 &gamma)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) xg[i] = value_of(half_of(x, i)) * value_of(half_of(gamma, i));
}

// The reciprocal root of the mean square, times the power of two that the row goes in with (1, or what brings its largest value to 2^14 or just below 2^15);
// what takes that back.
struct Factors { float r, back; };

template <int THREADS>
__device__ __forceinline__ Factors factors_of(Norm n, int K, float eps, float2 *s_norm)
{
    uint32_t top = __builtin_bit_cast(uint32_t, n.top);       // (in the order of the values, as none is below zero)
    // to lane 15 of each row of 16, then to lane 63 (lanes that have nobody to take from take 0)
#define ATOM_FROM(v, ctrl, rows) __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), ctrl, rows, 0xF, false)
#define ATOM_STEP(ctrl, rows)                                              \
    n.sum += __builtin_bit_cast(float, ATOM_FROM(n.sum, ctrl, rows));      \
    top = max(top, (uint32_t)ATOM_FROM(top, ctrl, rows))
    ATOM_STEP(0x111, 0xF);
    ATOM_STEP(0x112, 0xF);
    ATOM_STEP(0x114, 0xF);
    ATOM_STEP(0x118, 0xF);
    ATOM_STEP(0x142, 0xA);
    ATOM_STEP(0x143, 0xC);
#undef ATOM_STEP
#undef ATOM_FROM
    if ((threadIdx.x & 63) == 63) s_norm[threadIdx.x >> 6] = make_float2(n.sum, __builtin_bit_cast(float, top));
    __syncthreads();
    n.sum = 0.0f;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        n.sum += s_norm[w].x;
        top = max(top, __builtin_bit_cast(uint32_t, s_norm[w].y));
    }
    const float r = 1.0f / sqrtf(n.sum / (float)K + eps);
    // (What is not finite has the largest exponent, a row of zeros the smallest: both go in as they are.  A product of two halves is 2^-48 at least, so top * r is a normal
    // number whatever eps.)
    const int exponent = (int)(__builtin_bit_cast(uint32_t, __builtin_bit_cast(float, top) * r) >> 23 & 0xffu);
    const int e = exponent ? min(max(127 + 14 - exponent, 0), 126) : 0;
    return {r * __builtin_bit_cast(float, (127 + e) << 23), __builtin_bit_cast(float, (127 - e) << 23)};
}

// What a thread reads of a row first, so that it is on its way before anything waits.
struct Front { uint4 x, gamma; int4 i0, i1; };

template <int THREADS>
__device__ __forceinline__ Front front_of(const Args &p, const __half *__restrict__ x)
{
    Front f = {};
    const int b = min((int)threadIdx.x, p.K / 8 - 1);
    f.x = reinterpret_cast<const uint4 *>(x)[b];
    if (p.gamma) f.gamma = reinterpret_cast<const uint4 *>(p.gamma)[b];
    if (p.idx) {
        f.i0 = reinterpret_cast<const int4 *>(p.idx)[2 * b];
        f.i1 = reinterpret_cast<const int4 *>(p.idx)[2 * b + 1];
    }
    return f;
}

// Row x in reordered order, behind the norm where there is gamma, laid out for the product: eight channels from k on go to
// place(k), hi and lo apart (lo only behind a norm).  nat: LDS of natural_bytes(); all threads of the workgroup call.  Gives what takes the row's power of two back.
template <int THREADS, class Place>
__device__ __forceinline__ float lay_out(const Args &p, const __half *__restrict__ x, const Front &f, uint32_t *nat, float2 *s_norm, Place place)
{
    const int tid = threadIdx.x, blocks = p.K / 8, K4 = p.K - p.O;
    const uint4 *row = reinterpret_cast<const uint4 *>(x);
    float back = 1.0f;
    if (p.gamma) {
        const uint4 *gamma = reinterpret_cast<const uint4 *>(p.gamma);
        Norm norm;
        float xg[8], more[8];
        products(xg, f.x, f.gamma);
        if (tid < blocks) norm.add(f.x, xg);
        for (int b = tid + THREADS; b < blocks; b += THREADS) {
            const uint4 v = row[b];
            products(more, v, gamma[b]);
            norm.add(v, more);
        }
        const Factors by = factors_of<THREADS>(norm, p.K, p.eps, s_norm);
        back = by.back;
        for (int b = tid; b < blocks; b += THREADS) {
            if (b != tid) products(xg, row[b], gamma[b]);
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = halves_of(xg[i] * by.r);
            reinterpret_cast<uint4 *>(nat)[2 * b] = make_uint4(w[0], w[1], w[2], w[3]);
            reinterpret_cast<uint4 *>(nat)[2 * b + 1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
        __syncthreads();
    } else if (p.idx) {
        for (int b = tid; b < blocks; b += THREADS) reinterpret_cast<uint4 *>(nat)[b] = b == tid ? f.x : row[b];
        __syncthreads();
    }
    for (int b = tid; b < blocks; b += THREADS) {
        uint32_t w[8];
        if (p.idx) {
            const int4 i0 = b == tid ? f.i0 : reinterpret_cast<const int4 *>(p.idx)[2 * b], i1 = b == tid ? f.i1 : reinterpret_cast<const int4 *>(p.idx)[2 * b + 1];
            const int32_t at[8] = {i0.x, i0.y, i0.z, i0.w, i1.x, i1.y, i1.z, i1.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t c = min((uint32_t)at[i], (uint32_t)(p.K - 1));
                w[i] = p.gamma ? nat[c] : reinterpret_cast<const uint16_t *>(nat)[c];
            }
        } else if (p.gamma) {
            const uint4 u = reinterpret_cast<const uint4 *>(nat)[2 * b], v = reinterpret_cast<const uint4 *>(nat)[2 * b + 1];
            w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w, w[4] = v.x, w[5] = v.y, w[6] = v.z, w[7] = v.w;
        } else {
            const uint4 v = b == tid ? f.x : row[b];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = half_of(v, i);
        }
        in_order(w, 8 * b < K4);
        place(8 * b, 0, packed<false>(w));
        if (p.gamma) place(8 * b, 1, packed<true>(w));
    }
    return back;
}

__host__ __device__ constexpr size_t natural_bytes(int K, bool norm, bool index) { return norm ? 4 * (size_t)K : index ? 2 * (size_t)K : 0; }

// Rows into the workspace, in the order in which the product's loads take them (64 lanes of 16 bytes in a row): for every unit and half the operands
// of its instructions, of a tile of 16 rows, or (WIDE) of tiles of 32.
template <bool WIDE>
__device__ __forceinline__ void put(const Args &p, uint4 *out, int64_t m, int k, int half, const uint4 &v)
{
    const int  K4 = p.K - p.O, G4 = K4 >> 7, U = (p.K + p.O) >> 7, j = k - K4;
    const bool is4 = k < K4;
    const int  u = is4 ? k >> 7 : G4 + (j >> 6);
    if constexpr (!WIDE) {
        const int place = row_place(k, K4) & (is4 ? 15 : 7);                              // (instruction, chunk)
        const int tile = p.combine ? 0 : half, row = (int)m + (p.combine && half ? p.rows : 0);
        out[(((int64_t)u * p.halves + tile) * 16 + place) * (p.combine ? 2 * p.rows : p.rows) + row] = v;
    } else {
        const int i = is4 ? (k >> 3) & 7 : (j >> 3) & 3, c = is4 ? (k >> 6) & 1 : (j >> 5) & 1;
        const int s = p.wide - 1;                             // (wide is 1 or 2)
        const int64_t block = m >> (5 + s), t = m >> 5 & s;
        out[((((block * U + u) * p.halves + half) * p.wide + t) * 8 + i) * 64 + c * 32 + (m & 31)] = v;
    }
}

// With an index: a row to a workgroup, gathered in LDS (from memory 2 bytes at a time it takes longer: eight rows of 4096 channels behind the norm 5.6 us
// against 4.1).  Bound by its chain of reads, barriers and launch; a thread for eight channels up to 8192 of them.
template <bool WIDE, int THREADS>
__global__ __launch_bounds__(THREADS)
void w4a16_gather_kernel(Args p, uint4 *out)
{
    extern __shared__ uint32_t s_nat[];
    __shared__ float2 s_norm[THREADS / 64];
    const int64_t m = blockIdx.x;
    const __half *x = p.x + m * p.ldx;
    const float back = lay_out<THREADS>(p, x, front_of<THREADS>(p, x), s_nat, s_norm, [&](int k, int half, const uint4 &v) { put<WIDE>(p, out, m, k, half, v); });
    if (p.gamma && threadIdx.x == 0) p.back[m] = back;
}

constexpr int kRowChannels = 4096;                            // of a row, of a workgroup

// Without: 4096 channels of a row to a workgroup, each of which adds up the whole row.
template <bool WIDE>
__global__ __launch_bounds__(512)
void w4a16_rows_kernel(Args p, uint4 *out)
{
    __shared__ float2 s_norm[8];
    const int tid = threadIdx.x, blocks = p.K / 8, b = (int)blockIdx.y * (kRowChannels / 8) + tid, k = 8 * min(b, blocks - 1);
    const int64_t m = blockIdx.x;
    const __half *x = p.x + m * p.ldx;
    const uint4 v = *reinterpret_cast<const uint4 *>(x + k), g = p.gamma ? *reinterpret_cast<const uint4 *>(p.gamma + k) : v;
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = half_of(v, i);
    if (p.gamma) {
        Norm norm;
        float xg[8];
        for (int j = tid; j < blocks; j += 512) {
            const uint4 y = reinterpret_cast<const uint4 *>(x)[j];
            products(xg, y, reinterpret_cast<const uint4 *>(p.gamma)[j]);
            norm.add(y, xg);
        }
        const Factors by = factors_of<512>(norm, p.K, p.eps, s_norm);
        products(xg, v, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = halves_of(xg[i] * by.r);
        if (blockIdx.y == 0 && tid == 0) p.back[m] = by.back;
    }
    if (b >= blocks) return;
    in_order(w, k < p.K - p.O);
    put<WIDE>(p, out, m, k, 0, packed<false>(w));
    if (p.gamma) put<WIDE>(p, out, m, k, 1, packed<true>(w));
}

// ---- the product

#define ATOM_INLINE __attribute__((always_inline))      // of lambdas that registers go through: one that is called in many places is not inlined by itself

// Between the loads before a loop and the loop, which goes on loading: without it the compiler, which orders the first ones as it likes, has the
// loop wait for all loads under way in every turn, not in the first alone.
__device__ __forceinline__ void all_loads_done() { __builtin_amdgcn_s_waitcnt(0x0f70); }

// Between LDS writes of a wavefront's lanes and reads of other lanes of it: the LDS takes a wavefront's operations in their order, so no instruction is needed, but the
// compiler must not change that order.
__device__ __forceinline__ void lanes_see_lds()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

__device__ __forceinline__ float gated(float gate, float up) { return gate / (1.0f + expf(-gate)) * up; }

template <bool GATED>
__device__ __forceinline__ void store(const Args &p, int64_t m, int64_t n, float y, float up)
{
    if constexpr (GATED) y = gated(y, up);
    else if (p.residual) y += __half2float(p.residual[m * p.ldr + n]);
    p.y[m * p.ldy + n] = __float2half_rn(y);
}

// Up to 16 rows.  A workgroup has 16 NT output channels (of gate and of up); its eight wavefronts share the K channels in runs of INT4 groups and
// every eighth half of an INT8 group each (64 bytes of every weight row either way: a unit), and their sums meet in LDS, added in order.  A wavefront's
// next unit is on its way while it works, across the tiles that the workgroup has in turn (behind the last, one address for all lanes).  With a tile or
// two for a workgroup the time is latencies, among them the code's own way to the wavefronts: two to five units under way in unrolled code were slower.
// One row: 4096 x 4096 5.0 us, gated 11008 of 4096 12.4 (3.9 TB/s of weights from the last-level cache), 8192 x 24576 33 (3.0, from memory); eight rows
// behind the norm, 12288 of 4096, 13.9.
//   HL: halves of the activations that go in one after the other (2: hi and lo)
//   COMBINE: up to eight rows, hi in rows 0 .. 7 and lo in rows 8 .. 15 of the one tile (HL = 1)
//   KEPT: the activations are laid out in LDS by the workgroup itself (HL = 1), under way with the first weights
template <int NT, bool GATED, int HL, bool COMBINE, bool KEPT>
__global__ __launch_bounds__(kThreads, KEPT ? 4 : 2)
void w4a16_kernel(Args p)
{
    constexpr int WM = GATED ? 2 : 1, CT = WM * NT, AT = HL;
    static_assert(CT <= 4, "a lane's chunk loads the scales of one tile");
    extern __shared__ __align__(16) unsigned char s_all[];   // KEPT: the rows; the weights' way to the operands; the sums (before: what is laid out)
    __shared__ float2 s_norm[8];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, kc = lane >> 4;
    const int K4 = p.K - p.O, G = p.K >> 7, G4 = K4 >> 7, V = 2 * (G - G4);
    const int part = (int)blockIdx.y, from = part * p.span, share = min(G4 - from, p.span);
    const int begin = from + wave, n = (share - wave + kWaves - 1) / kWaves;       // INT4 units of this wavefront
    const int first_half = wave + part * kWaves;
    const int rows = p.rows, lds_row = p.K + 8;

    Front front;
    if constexpr (KEPT) front = front_of<kThreads>(p, p.x);

    // (rows >= M are computed and never stored, columns >= N likewise)
    const int r = COMBINE && col >= 8 ? rows + min(col - 8, rows - 1) : min(col, rows - 1);
    const __half *s_act = reinterpret_cast<const __half *>(s_all) + (size_t)r * lds_row + kc * 8;
    const int laid_rows = COMBINE ? 2 * rows : rows;          // rows that are laid out; lanes of others read the last
    const u4 *acts = reinterpret_cast<const u4 *>(p.staged) + kc * laid_rows + r;
    unsigned char *s_mine = s_all + (KEPT ? (size_t)rows * (p.gamma ? 2 : 1) * lds_row * 2 : 0);
    u4 *s_turn = reinterpret_cast<u4 *>(s_mine) + wave * (CT * 64);     // this wavefront's own
    float *red = reinterpret_cast<float *>(s_mine + kWaves * CT * 1024);

    // A load brings 64 bytes of 16 rows, four lanes a row: lanes that go to one line apart, or one load after the other, hold up the cache until the line
    // is there.  The operands want a row in one lane of each 16, so the pieces go through LDS.
    struct { u4 q[CT], a[KEPT ? 1 : 4 * AT]; uint16_t scale; } e;    // (lane 16 t + c: the scale of row c of tile t)
    struct { u4 q[CT], a[KEPT ? 1 : 2 * AT]; uint16_t scale; } half;                // of an INT8 group
    uint32_t load_tile = blockIdx.x;                         // of the unit that is loaded next
    int load_i = 0;
    uint32_t at4[CT], at_scale;                              // (bytes from the arrays' beginnings are below 4 GiB: host)
    const uint16_t *scale_of = kc < CT && kc >= NT ? p.w[WM - 1].scale : p.w[0].scale;
    auto rows_of = [&](uint32_t tile) ATOM_INLINE {
        const bool live = tile < p.tiles;
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const uint32_t r = (uint32_t)min((int64_t)tile * (16 * NT) + 16 * (t % NT) + (lane >> 2), p.N - 1);
            at4[t] = live ? r * (uint32_t)(K4 >> 1) + (lane & 3) * 16 : 0;
        }
        const uint32_t r = (uint32_t)min((int64_t)tile * (16 * NT) + (kc < CT ? 16 * (kc % NT) + col : 0), p.N - 1);
        at_scale = live ? r * (uint32_t)G : 0;
    };
    auto load = [&]() ATOM_INLINE {
        const bool live = load_i < n;
        const int  u = live ? begin + load_i * kWaves : 0;
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const uint32_t at = live ? at4[t] : 0;
            e.q[t] = *reinterpret_cast<const u4 *>(p.w[t / NT].q4 + u * 64 + at);
        }
        e.scale = scale_of[u + (live ? at_scale : 0)];
        if constexpr (!KEPT) {
#pragma unroll
            for (int a = 0; a < AT; ++a)
#pragma unroll
                for (int c = 0; c < 4; ++c) e.a[4 * a + c] = acts[((u * AT + a) * 16 + c * 4) * laid_rows];
        }
        if (++load_i >= n) {
            load_i = 0;
            load_tile += gridDim.x;
            rows_of(load_tile);
        }
    };
    auto load_half = [&](uint32_t tile, int v) ATOM_INLINE {
        const bool live = tile < p.tiles && v < V;
        const int  i = live ? v : 0;
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const uint32_t r = (uint32_t)min((int64_t)tile * (16 * NT) + 16 * (t % NT) + (lane >> 2), p.N - 1), at = live ? r * (uint32_t)p.O + (lane & 3) * 16 : 0;
            half.q[t] = *reinterpret_cast<const u4 *>(reinterpret_cast<const uint8_t *>(p.w[t / NT].q8) + i * 64 + at);
        }
        const uint32_t r = (uint32_t)min((int64_t)tile * (16 * NT) + (kc < CT ? 16 * (kc % NT) + col : 0), p.N - 1), at = live ? r * (uint32_t)G : 0;
        half.scale = scale_of[at + G4 + (i >> 1)];
        if constexpr (!KEPT) {
#pragma unroll
            for (int a = 0; a < AT; ++a)
#pragma unroll
                for (int c = 0; c < 2; ++c) half.a[2 * a + c] = acts[(((G4 + i) * AT + a) * 16 + c * 4) * laid_rows];
        }
    };
    f4 acc[CT] = {};
    // piece p of row r lies at 4 r + (p ^ (r / 4 & 3)): the 16 lanes of a chunk read all banks
    u4 *turn_to = s_turn + (lane & ~3) + ((lane ^ (lane >> 4)) & 3), *turn_from = s_turn + 4 * col + ((kc ^ (col >> 2)) & 3);
    auto operands = [&](const u4 (&from)[CT], u4 (&q)[CT]) ATOM_INLINE {
        lanes_see_lds();                                     // (what was read there is read)
#pragma unroll
        for (int t = 0; t < CT; ++t) turn_to[t * 64] = from[t];
        lanes_see_lds();
#pragma unroll
        for (int t = 0; t < CT; ++t) q[t] = turn_from[t * 64];
    };
    auto add = [&](int t, const f4 &part, uint32_t scale) ATOM_INLINE {
        const float s = __half2float(__ushort_as_half((unsigned short)scale));
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[t][j] = fmaf(part[j], s, acc[t][j]);
    };
    auto compute = [&](int u) ATOM_INLINE {
        f4 part[CT] = {};
        u4 q[CT];
        operands(e.q, q);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                const h8 w = widen4(q[t][c]);
#pragma unroll
                for (int a = 0; a < AT; ++a) {
                    h8 x;
                    if constexpr (KEPT) x = *reinterpret_cast<const h8 *>(s_act + u * 128 + c * 32);
                    else x = __builtin_bit_cast(h8, e.a[4 * a + c]);
                    part[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, w, part[t], 0, 0, 0);
                }
            }
#pragma unroll
        for (int t = 0; t < CT; ++t) add(t, part[t], (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (16 * t + col), (int)e.scale));
    };
    auto compute_half = [&](int v) ATOM_INLINE {
        f4 part[CT] = {};
        u4 q[CT];
        operands(half.q, q);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                const h8 w = widen8(q[t][2 * c], q[t][2 * c + 1]);
#pragma unroll
                for (int a = 0; a < AT; ++a) {
                    h8 x;
                    if constexpr (KEPT) x = *reinterpret_cast<const h8 *>(s_act + K4 + v * 64 + c * 32);
                    else x = __builtin_bit_cast(h8, half.a[2 * a + c]);
                    part[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, w, part[t], 0, 0, 0);
                }
            }
#pragma unroll
        for (int t = 0; t < CT; ++t) add(t, part[t], (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (16 * t + col), (int)half.scale));
    };
    constexpr int kLanes = COMBINE ? 32 : 64;                // that have rows: half of them where lo is added to hi
    constexpr int kTile = 4 * kLanes, kOut = (NT * kTile + kThreads - 1) / kThreads;       // outputs of a tile, of a thread
    auto output = [&](uint32_t tile, int i, int64_t &m, int64_t &out) ATOM_INLINE {
        const int at = tid + i * kThreads, l = at % kLanes;
        m = 4 * (l >> 4) + (at / kLanes & 3);
        out = (int64_t)tile * (16 * NT) + 16 * (at / kTile) + (l & 15);
        return at < NT * kTile && m < p.M && out < p.N;
    };
    const int my_row = min(4 * (tid % kLanes >> 4) + (tid / kLanes & 3), rows - 1);       // of all outputs of this thread
    float back = 1.0f;
    if constexpr (!KEPT && (COMBINE || HL == 2)) back = p.back[my_row];
    uint16_t residual[kOut];
    auto fetch_residual = [&](uint32_t tile) ATOM_INLINE {               // (at a tile's beginning: at its end all loads under way would be waited for)
        if constexpr (!GATED) {
            int64_t m, out;
            if (p.residual && p.parts == 1)
#pragma unroll
                for (int i = 0; i < kOut; ++i)
                    if (output(tile, i, m, out)) residual[i] = reinterpret_cast<const uint16_t *>(p.residual)[m * p.ldr + out];
        }
    };
    int buffer = 0;
    auto finish = [&](uint32_t tile) ATOM_INLINE {
        float *mine = red + buffer * (kWaves * CT * kTile);
        buffer ^= 1;                                         // (nobody writes a buffer before all have read what it held two tiles ago)
        if constexpr (COMBINE)                               // rows 8 .. 15 to rows 0 .. 7
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[t][j] += __shfl_xor(acc[t][j], 32, 64);
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (lane < kLanes) mine[(wave * CT + t) * kTile + j * kLanes + lane] = acc[t][j];
                acc[t][j] = 0.0f;
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kOut; ++i) {
            int64_t m, out;
            if (!output(tile, i, m, out)) continue;
            const int at = tid + i * kThreads;
            float sum[WM];
#pragma unroll
            for (int x = 0; x < WM; ++x) {
                sum[x] = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) sum[x] += mine[(w * CT + x * NT) * kTile + at];
                if constexpr (COMBINE || HL == 2) sum[x] *= back;
            }
            float y = sum[0];
            if (p.parts > 1) {
#pragma unroll
                for (int x = 0; x < WM; ++x) p.sums[((int64_t)(part * WM + x) * p.M + m) * p.N + out] = sum[x];
                continue;
            }
            if constexpr (GATED) y = gated(y, sum[WM - 1]);
            else if (p.residual) y += __half2float(__ushort_as_half(residual[i]));
            p.y[m * p.ldy + out] = __float2half_rn(y);
        }
    };

    uint32_t tile = blockIdx.x;
    rows_of(tile);
    fetch_residual(tile);
    load();
    load_half(tile, first_half);
    if constexpr (KEPT) {
        uint32_t *nat = reinterpret_cast<uint32_t *>(s_mine);
        __half *out = reinterpret_cast<__half *>(s_all);
        for (int m = 0; m < rows; ++m) {
            if (m) {
                __syncthreads();
                front.x = front_of<kThreads>(p, p.x + m * p.ldx).x;
            }
            const float by = lay_out<kThreads>(p, p.x + m * p.ldx, front, nat, s_norm,
                                               [&](int k, int half, const uint4 &v) { *reinterpret_cast<uint4 *>(out + (size_t)(m + half * rows) * lds_row + 8 * row_place(k, K4)) = v; });
            if (COMBINE && m == my_row) back = by;
        }
        __syncthreads();
    }
    all_loads_done();
    for (; tile < p.tiles; tile += gridDim.x) {
        for (int i = 0; i < n; ++i) {
            compute(begin + i * kWaves);
            load();
        }
        if (first_half < V) compute_half(first_half);
        for (int v = first_half + kWaves * p.parts; v < V; v += kWaves * p.parts) {       // (more than 512 outlier channels)
            load_half(tile, v);
            compute_half(v);
        }
        load_half(tile + gridDim.x, first_half);
        finish(tile);
        fetch_residual(min(tile + gridDim.x, p.tiles - 1));
    }
}

typedef float f16 __attribute__((ext_vector_type(16)));

// More than 16 rows: MFMA 32x32x16, whose operands bring twice the products for their bytes (lane l: row or column l & 31, the eight values
// of k-chunk l >> 5; register r of the result: row 8 (r / 4) + 4 (l >> 5) + r % 4).  A workgroup has 32 RT rows and eight tiles of 32 weight
// rows (of a gated call four of the gate and the same four of the up projection in turn).  Each wavefront has one of them for all rows.  Activations
// and weights come a unit at a time through LDS, a tile by each wavefront.  `parts` workgroups share a tile's units where the tiles alone do not
// fill the card; their sums meet in the workspace.  What the L2 delivers to all compute units together (about 8 TB/s) is the tightest bound beside
// memory, so scales come 64 of a row at a time (by themselves, 2 bytes bring a line each: as much as the weights), and rows behind M are not fetched.
// 33 rows, 8192 outputs of 28672 channels: 42.5 us of the call's 51 (2.9 TB/s of weights; a second tile of 32 rows for one); 64 rows, gated 28672 of 8192
// behind the norm: 130 of 138, at 920 TFLOP/s with both halves of the activations.  One or two units under way and short code: with three or four, and scales
// eight rows at a time, 20 rows and 4000 outputs of 8192 channels took 25.2 us, now 20.7.
template <bool GATED, int RT, int HL>
__global__ __launch_bounds__(kThreads, 2)
void w4a16_wide_kernel(Args p)
{
    constexpr int CH = HL == 1 ? 2 : 1;                      // units under way
    constexpr int kOps = RT * HL;                            // 16-byte pieces of a unit's activations that a thread brings
    extern __shared__ __align__(16) unsigned char s_all[];
    u4 (*s_act)[kOps * 512] = reinterpret_cast<u4 (*)[kOps * 512]>(s_all);                     // [2], and behind them
    u4 (*s_turn)[kWaves][128] = reinterpret_cast<u4 (*)[kWaves][128]>(s_act + 2);              // [2]: the weights' way to the operands
    uint16_t (*s_scale)[kScales + 2] = reinterpret_cast<uint16_t (*)[kScales + 2]>(s_turn + 2);    // [256]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, kc = lane >> 5;
    const int K4 = p.K - p.O, G = p.K >> 7, G4 = K4 >> 7, U = 2 * G - G4;
    const uint32_t block = blockIdx.x % p.row_blocks, rest = blockIdx.x / p.row_blocks, part = rest % (uint32_t)p.parts, tile = rest / (uint32_t)p.parts;
    const int begin = (int)(part * (uint32_t)U / (uint32_t)p.parts), end = (int)((part + 1) * (uint32_t)U / (uint32_t)p.parts);

    // The first weight row of a tile; its matrix.  (Columns >= N are computed and never stored.)
    auto rows_of = [&](int t) ATOM_INLINE { return GATED ? ((int64_t)tile * (kWaves / 2) + t / 2) * 32 : ((int64_t)tile * kWaves + t) * 32; };
    auto matrix_of = [&](int t) ATOM_INLINE { return GATED ? t & 1 : 0; };
    // This wavefront brings tile `wave`, 64 bytes of 16 rows at a time, four lanes a row (lanes that go to one line apart, or one load after the
    // other, hold up the cache until the line is there).
    const W4 w = p.w[matrix_of(wave)];
    const uint32_t row0 = (uint32_t)min(rows_of(wave) + (lane >> 2), p.N - 1), row1 = (uint32_t)min(rows_of(wave) + 16 + (lane >> 2), p.N - 1);
    const uint32_t at4_0 = row0 * (uint32_t)(K4 >> 1) + (lane & 3) * 16, at4_1 = row1 * (uint32_t)(K4 >> 1) + (lane & 3) * 16;
    const uint32_t at8_0 = row0 * (uint32_t)p.O + (lane & 3) * 16, at8_1 = row1 * (uint32_t)p.O + (lane & 3) * 16;
    // (a load is waited for with all before it, so a unit's weights and activations come the same way ahead)
    struct Unit { u4 q[2], a[kOps]; };
    Unit ring[CH];
    const u4 *acts = reinterpret_cast<const u4 *>(p.staged) + (int64_t)block * U * (kOps * 512);
    int piece[RT];                                           // (lanes of rows >= M take the last row's)
#pragma unroll
    for (int r = 0; r < RT; ++r) piece[r] = (tid & ~31) + min(tid & 31, max((int)(p.M - ((int64_t)block * RT + r) * 32) - 1, 0));
    int load_u = begin;
    auto load = [&](Unit &e) ATOM_INLINE {
        const int  u = min(load_u, end - 1), v = u - G4;
        const bool is4 = u < G4;
        const u4 *from = acts + (int64_t)u * (kOps * 512);
#pragma unroll
        for (int c = 0; c < kOps; ++c) e.a[c] = from[c * 512 + piece[c % RT]];
        const uint8_t *base = is4 ? w.q4 + u * 64 : reinterpret_cast<const uint8_t *>(w.q8) + v * 64;
        e.q[0] = *reinterpret_cast<const u4 *>(base + (is4 ? at4_0 : at8_0));
        e.q[1] = *reinterpret_cast<const u4 *>(base + (is4 ? at4_1 : at8_1));
        ++load_u;
    };
    auto keep = [&](const Unit &e, int u) ATOM_INLINE {
#pragma unroll
        for (int c = 0; c < kOps; ++c) s_act[(u - begin) & 1][c * 512 + tid] = e.a[c];
        // piece p of row r lies at 4 r + (p ^ (r / 4 & 3)): the lanes of a chunk read all banks
#pragma unroll
        for (int i = 0; i < 2; ++i) s_turn[(u - begin) & 1][wave][64 * i + (lane & ~3) + ((lane ^ (lane >> 4)) & 3)] = e.q[i];
    };

    // the scales of kScales groups from that of unit u on, each wavefront those of its own rows
    uint16_t *my_scales = s_scale[32 * wave];
    int scale0 = 0, scale_end = begin;
    auto fetch_scales = [&](int u) ATOM_INLINE {
        scale0 = u < G4 ? u : G4 + ((u - G4) >> 1);
        const int count = min(kScales, G - scale0);
        scale_end = scale0 + count <= G4 ? scale0 + count : G4 + 2 * (scale0 + count - G4);
        const uint16_t *from = w.scale + scale0 + min(lane, count - 1);
        lanes_see_lds();                                     // (what was read there is read)
#pragma unroll 16
        for (int r = 0; r < 32; ++r) my_scales[r * (kScales + 2) + lane] = from[min(rows_of(wave) + r, p.N - 1) * G];
        lanes_see_lds();
    };
    f16 acc[RT] = {};
    auto compute = [&](int u) ATOM_INLINE {
        const u4 *a = s_act[(u - begin) & 1] + lane;
        u4 q[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) q[i] = s_turn[(u - begin) & 1][wave][4 * col + (((2 * kc + i) ^ (col >> 2)) & 3)];
        f16 sum[RT] = {};
        h8 x[2][kOps];                                       // the next k-chunk's operands come while this one's are in use
        auto operands = [&](int i) ATOM_INLINE {
#pragma unroll
            for (int o = 0; o < kOps; ++o) x[i & 1][o] = __builtin_bit_cast(h8, a[o * 512 + i * 64]);
        };
        auto chunks = [&](int count, bool is4) ATOM_INLINE {
            operands(0);
#pragma unroll
            for (int i = 0; i < count; ++i) {
                if (i + 1 < count) operands(i + 1);
                __builtin_amdgcn_sched_barrier(0);           // (or the reads move to where they are used)
                const h8 y = is4 ? widen4(q[i >> 2][i & 3]) : widen8(q[i >> 1 & 1][2 * (i & 1)], q[i >> 1 & 1][2 * (i & 1) + 1]);
#pragma unroll
                for (int o = 0; o < kOps; ++o) sum[o % RT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i & 1][o], y, sum[o % RT], 0, 0, 0);
            }
        };
        if (u < G4) chunks(8, true);
        else        chunks(4, false);
        const float s = __half2float(__ushort_as_half(my_scales[col * (kScales + 2) + (u < G4 ? u : G4 + ((u - G4) >> 1)) - scale0]));
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[r][j] = fmaf(sum[r][j], s, acc[r][j]);
    };

    Unit first;
    load(first);
#pragma unroll
    for (int s = 0; s < CH; ++s) load(ring[s]);
    all_loads_done();
    fetch_scales(begin);
    keep(first, begin);
    __syncthreads();
    for (int u = begin; u < end; u += CH) {
        if (u + CH > scale_end && scale_end < end) fetch_scales(u);
#pragma unroll
        for (int s = 0; s < CH; ++s) {                       // (no way out of the loop here: the compiler would wait at its head for what had been asked for by then)
            keep(ring[s], u + s + 1);
            load(ring[s]);
            if (u + s < end) compute(u + s);
            __syncthreads();                                 // (all have read this unit, the next one is there)
        }
    }

    const int64_t n = rows_of(wave) + col, m0 = (int64_t)block * (32 * RT) + 4 * kc;
    auto row_of = [&](int r, int j) ATOM_INLINE { return m0 + 32 * r + 8 * (j >> 2) + (j & 3); };
    if constexpr (HL == 2)                                   // behind a norm (of rows >= M there is room for it)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f4 back = *reinterpret_cast<const f4 *>(p.back + row_of(r, 4 * q));
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[r][4 * q + j] *= back[j];
            }
    if (p.parts > 1) {
        if (n < p.N)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (row_of(r, j) < p.M) p.sums[(((int64_t)part * (GATED ? 2 : 1) + matrix_of(wave)) * p.M + row_of(r, j)) * p.N + n] = acc[r][j];
        return;
    }
    if constexpr (GATED) {                                   // the wavefront after a gate's has the up projection
        float *s_up = reinterpret_cast<float *>(s_all) + (wave >> 1) * (RT * 1024) + lane;
        if (wave & 1)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int j = 0; j < 16; ++j) s_up[(16 * r + j) * 64] = acc[r][j];
        __syncthreads();
        if (wave & 1) return;
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (row_of(r, j) < p.M && n < p.N) p.y[row_of(r, j) * p.ldy + n] = __float2half_rn(gated(acc[r][j], s_up[(16 * r + j) * 64]));
    } else {
        if (p.residual)                                      // (all of them on their way at once)
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                uint16_t res[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) res[j] = reinterpret_cast<const uint16_t *>(p.residual)[min(row_of(r, j), p.M - 1) * p.ldr + min(n, p.N - 1)];
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[r][j] += __half2float(__ushort_as_half(res[j]));
            }
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (row_of(r, j) < p.M && n < p.N) p.y[row_of(r, j) * p.ldy + n] = __float2half_rn(acc[r][j]);
    }
}

// The parts' sums, in their order.
template <bool GATED>
__global__ __launch_bounds__(256)
void w4a16_join_kernel(Args p)
{
    const uint32_t e = blockIdx.x * 256 + threadIdx.x, m = e / (uint32_t)p.N;              // (fewer than 2^30: host)
    const int64_t outputs = p.M * p.N;
    if (e >= outputs) return;
    float y = 0.0f, up = 0.0f;
    for (int s = 0; s < p.parts; ++s) {
        y += p.sums[s * (GATED ? 2 : 1) * outputs + e];
        if constexpr (GATED) up += p.sums[(2 * s + 1) * outputs + e];
    }
    store<GATED>(p, m, e - m * (uint32_t)p.N, y, up);
}

}  // namespace

namespace atom_internal {

// How a call runs.  Up to 16 rows: whether the workgroups lay the activations out themselves, tiles of 16 channels, LDS.  More: tiles of
// 32 rows in a block, parts of K.
struct ProductShape { bool kept, combine; int NT; size_t lds; int wide, parts, span; };

// Up to 16 rows, few outputs of many channels: INT4 groups of a part of K at least, and as many parts as leave a workgroup a CU.  A wavefront takes 0.3 to
// 0.5 us for a unit and a join 2.5: one row, 64 outputs of 24576 channels 17.0 us whole and 12.0 in parts, 2048 of them 19.8 and 17.0; of 8192 channels
// 6.5 and (parts of 16) 7.2; 4096 outputs of 24576 in two parts (two workgroups a CU) 26.9 instead of 24.2.
constexpr int kPartGroups = 32, kPartWorkgroups = 256;

// LDS of a workgroup where two of them share a CU, and where one has it (less what the kernel has beside).  Rows that the workgroups lay out themselves
// cost no launch: gated 11008 of 4096 channels, one row, 12.4 us and 20.8 with a launch for it; two rows 13.2 and 9.4 to 8.3 for 64 outputs; where one
// workgroup has a CU only a single row pays, and only without a second round (64 outputs of 24576 channels 10.8 and 12.0, 8192 of them 42.9 and 33.2).
constexpr size_t kTwoGroupsLds = 80 * 1024 - 64, kOneGroupLds = 150 * 1024;

// The weights' way to the operands and the wavefronts' sums, twice.
static size_t sums_bytes(const ProductShape &s, int WM) { return (size_t)kWaves * WM * s.NT * 1024 * (s.combine ? 2 : 3); }

static ProductShape product_shape(int64_t M, int64_t N, int K, int O, bool gated, bool norm, bool index)
{
    const int WM = gated ? 2 : 1;
    ProductShape s = {};
    if (M > 16) {
        s.wide = M <= 32 ? 1 : 2;
        const int U = (K + O) / 128;
        const int64_t tiles = (N + (gated ? 127 : 255)) / (gated ? 128 : 256) * ((M + 32 * s.wide - 1) / (32 * s.wide)), cus = 256;
        // Rounds of workgroups, each as long as its units; a join costs about two units and what it moves.  More than 16 parts only of six units and more (64
        // outputs, 50 rows: of 24576 channels 30.7 us in 16 parts and 28.1 in 32, of 8192 18.8 in 16 and 19.0 in 32; of 2048 15.0 in 4 and 14.3 in 8).
        double best = 1e30;
        for (int parts = 1; parts <= 32 && parts * (parts > 16 ? 6 : 2) <= U; ++parts) {
            const double cost = (double)((tiles * parts + cus - 1) / cus) * ((U + parts - 1) / parts + 3) + (parts > 1 ? 4 + (double)parts * M * N * WM * 8 / 5e6 : 0);
            if (cost < best) {
                best = cost;
                s.parts = parts;
            }
        }
        if (!s.parts) s.parts = 1;
        return s;
    }
    s.NT = 1;
    s.combine = norm && M <= 8;
    const size_t sums = sums_bytes(s, WM), nat = natural_bytes(K, norm, index), rest = nat > sums ? nat : sums;
    if (M <= (norm ? 8 : 16)) {
        s.lds = (size_t)M * (norm ? 2 : 1) * (K + 8) * 2 + rest;
        s.kept = s.lds <= kTwoGroupsLds || (M == 1 && s.lds <= kOneGroupLds && (N + 15) / 16 <= kPartWorkgroups);
    }
    if (!s.kept) {
        // Rounds of workgroups, a CU each, times what they read for a unit: 1 KB of weights for 16 rows of them, and the activations, which the L2 gives four
        // times as fast.  (16 rows, 20000 outputs of 24576 channels: NT = 1 111 us, 2 101, 4 117; 6000 of them 34, 25, 28; 28672 152, 133, 123; four rows
        // and 12288 outputs 50, 56, 56.)
        const double rows = norm ? 2 * M : M;
        double best = 1e30;
        for (int NT = 1; NT * WM <= 4; NT *= 2) {
            const double cost = (double)(((N + 16 * NT - 1) / (16 * NT) + kPartWorkgroups - 1) / kPartWorkgroups) * (NT * WM + rows / 16);
            if (cost < best) {
                best = cost;
                s.NT = NT;
            }
        }
        s.lds = sums_bytes(s, WM);
    }
    const int64_t tiles = (N + 16 * s.NT - 1) / (16 * s.NT);
    const int     G4 = (K - O) / 128;
    s.parts = 1;
    s.span = G4;
    const int64_t most = kPartWorkgroups / tiles;
    int wanted = G4 / kPartGroups;
    if (wanted > most) wanted = (int)most;
    if (wanted > 1) {
        s.span = (G4 + wanted - 1) / wanted;
        s.parts = (G4 + s.span - 1) / s.span;
    }
    return s;
}

static size_t laid_out_bytes(const ProductShape &s, int64_t M, int K, int O, bool norm)
{
    if (s.kept) return 0;
    if (!s.wide) return (size_t)((K + O) / 128) * (norm ? 2 : 1) * M * 256;
    return (size_t)((M + 32 * s.wide - 1) / (32 * s.wide)) * ((K + O) / 128) * s.wide * (norm ? 2 : 1) * 8192;
}

// What takes the rows' powers of two back, of whole blocks of 64 rows.
static size_t back_bytes(const ProductShape &s, int64_t M, bool norm) { return norm && !s.kept ? (size_t)((M + 63) / 64) * 256 : 0; }

// The rows, what takes their powers of two back, the parts' sums.
size_t w4a16_workspace_bytes(int64_t M, int64_t N, int K, int O, bool gated, bool norm, bool index)
{
    const ProductShape s = product_shape(M, N, K, O, gated, norm, index);
    return laid_out_bytes(s, M, K, O, norm) + back_bytes(s, M, norm) + (s.parts > 1 ? (size_t)s.parts * M * N * (gated ? 8 : 4) : 0);
}

bool w4a16_fits(int64_t M, int64_t N, int K, int O, bool gated)
{
    (void)gated;
    if (M == 0 || N == 0) return true;
    const int64_t G = K / 128, widest = (K - O) / 2 > O ? (K - O) / 2 : O;
    if (N > 0xffffffffLL / (widest > 2 * G ? widest : 2 * G)) return false;           // 32-bit offsets
    // threads: 1024 for a row, 512 for each of up to 32 parts (as 16 times 1024) of a tile of 128 outputs at least and 32 rows, 256 for as many outputs of a join
    const int64_t most = atom_launch::kMostThreads / 1024;
    return M <= most && (N + 15) / 16 <= most && (N + 127) / 128 * 16 <= most / ((M + 31) / 32) && M <= most * 256 / N;
}

hipError_t launch_w4a16(const W4A16 &a, hipStream_t stream)
{
    const bool gated = a.w[1].q4 != nullptr, norm = a.gamma != nullptr;
    const ProductShape s = product_shape(a.M, a.N, a.K, a.O, gated, norm, a.idx != nullptr);
    const int  halves = norm && !s.combine ? 2 : 1;           // that go in one after the other
    char *back = (char *)a.workspace + laid_out_bytes(s, a.M, a.K, a.O, norm);
    Args p = {(const __half *)a.x, a.ldx, a.M, (const __half *)a.gamma, a.eps, a.idx, a.K, a.O, {a.w[0], a.w[1]}, a.N, (const __half *)a.residual, a.ldr,
              (__half *)a.y, a.ldy, (const __half *)a.workspace, (int)a.M, (float *)back, s.combine, 0, s.parts, s.span,
              (float *)(back + back_bytes(s, a.M, norm)), s.wide, halves, 1};
#define ATOM_LAUNCH(grid, threads, lds, kernel, ...)                                                                  \
    do {                                                                                                              \
        static atom_launch::LdsOptIn opt;                                                                             \
        auto kern = &kernel;                                                                                          \
        if ((lds) > 60 * 1024) {                                                                                      \
            const hipError_t err = atom_launch::ensure_dynamic_lds(opt, reinterpret_cast<const void *>(kern), lds);   \
            if (err != hipSuccess) return err;                                                                        \
        }                                                                                                             \
        hipLaunchKernelGGL(kern, dim3(grid), dim3(threads), lds, stream, __VA_ARGS__);                                \
        const hipError_t err = hipGetLastError();                                                                     \
        if (err != hipSuccess) return err;                                                                            \
    } while (0)
    uint4 *laid_out = (uint4 *)a.workspace;
#define ATOM_ROWS(WIDE)                                                                                                               \
    do {                                                                                                                              \
        const size_t nat = natural_bytes(a.K, norm, true);                                                                            \
        const dim3 split((unsigned)a.M, (unsigned)((a.K + kRowChannels - 1) / kRowChannels));                                         \
        if (!a.idx)             ATOM_LAUNCH(split, 512, 0, w4a16_rows_kernel<WIDE>, p, laid_out);                                     \
        else if (a.K <= 4096)   ATOM_LAUNCH((unsigned)a.M, 512, nat, (w4a16_gather_kernel<WIDE, 512>), p, laid_out);                  \
        else                    ATOM_LAUNCH((unsigned)a.M, 1024, nat, (w4a16_gather_kernel<WIDE, 1024>), p, laid_out);                \
    } while (0)
    if (s.wide)       ATOM_ROWS(true);
    else if (!s.kept) ATOM_ROWS(false);
#undef ATOM_ROWS

    if (s.wide) {
        const int64_t per = gated ? 128 : 256;
        p.row_blocks = (uint32_t)((a.M + 32 * s.wide - 1) / (32 * s.wide));
        const unsigned grid = (unsigned)((a.N + per - 1) / per * s.parts * p.row_blocks);
#define ATOM_WIDE(GATED, RT, HL) ATOM_LAUNCH(grid, kThreads, (size_t)2 * ((RT) * (HL) * 8192 + kWaves * 2048) + 256 * (kScales + 2) * 2, (w4a16_wide_kernel<GATED, RT, HL>), p)
#define ATOM_WIDE_ROWS(GATED)                                  \
    do {                                                       \
        if (s.wide == 1) {                                     \
            if (norm) ATOM_WIDE(GATED, 1, 2);                  \
            else      ATOM_WIDE(GATED, 1, 1);                  \
        } else {                                               \
            if (norm) ATOM_WIDE(GATED, 2, 2);                  \
            else      ATOM_WIDE(GATED, 2, 1);                  \
        }                                                      \
    } while (0)
        if (gated) ATOM_WIDE_ROWS(true);
        else       ATOM_WIDE_ROWS(false);
#undef ATOM_WIDE_ROWS
#undef ATOM_WIDE
    } else {
        p.tiles = (uint32_t)((a.N + 16 * s.NT - 1) / (16 * s.NT));
        const uint32_t room = (uint32_t)(2 * atom_launch::compute_units()), groups = p.tiles < room ? p.tiles : room;
        const dim3 grid(groups, s.parts);
#define ATOM_FEW(...) ATOM_LAUNCH(grid, kThreads, s.lds, (w4a16_kernel<__VA_ARGS__>), p)
#define ATOM_FEW_ROWS(NT, GATED)                                          \
        do {                                                              \
            if (!norm)          ATOM_FEW(NT, GATED, 1, false, false);     \
            else if (s.combine) ATOM_FEW(NT, GATED, 1, true, false);      \
            else                ATOM_FEW(NT, GATED, 2, false, false);     \
        } while (0)
        if (s.kept) {
            if (gated && norm) ATOM_FEW(1, true, 1, true, true);
            else if (gated)    ATOM_FEW(1, true, 1, false, true);
            else if (norm)     ATOM_FEW(1, false, 1, true, true);
            else               ATOM_FEW(1, false, 1, false, true);
        } else if (gated) {
            if (s.NT == 2) ATOM_FEW_ROWS(2, true);
            else           ATOM_FEW_ROWS(1, true);
        } else {
            if (s.NT == 4)      ATOM_FEW_ROWS(4, false);
            else if (s.NT == 2) ATOM_FEW_ROWS(2, false);
            else                ATOM_FEW_ROWS(1, false);
        }
#undef ATOM_FEW_ROWS
#undef ATOM_FEW
    }
    if (s.parts > 1) {
        const unsigned groups = (unsigned)((a.M * a.N + 255) / 256);
        if (gated) ATOM_LAUNCH(groups, 256, 0, w4a16_join_kernel<true>, p);
        else       ATOM_LAUNCH(groups, 256, 0, w4a16_join_kernel<false>, p);
    }
#undef ATOM_LAUNCH
    return hipSuccess;
}

}  // namespace atom_internal
