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

template <bool ONCE>
__device__ __forceinline__ uint2 load4(const __half *p)
{
    typedef unsigned u2 __attribute__((ext_vector_type(2)));
    if constexpr (ONCE) return __builtin_bit_cast(uint2, __builtin_nontemporal_load(reinterpret_cast<const u2 *>(p)));
    else return *reinterpret_cast<const uint2 *>(p);
}

// A run's scale from its maximum (the bits of a float) and that of the block's older rows (0: none), its reciprocal, and what older codes are brought to it with.
struct Scale { float s, r, ratio; bool grown; };

__device__ __forceinline__ Scale scale_of(uint32_t top, float s_old)
{
    const float s_new = __builtin_bit_cast(float, top) / 127.0f, s = s_new > s_old || s_new != s_new ? s_new : s_old;
    // (a scale below the normal numbers has no reciprocal)
    return {s, s >= 1.17549435e-38f ? 1.0f / s : 0.0f, s_old / s, s > s_old && s_old > 0.0f};
}

__device__ __forceinline__ uint4 recode16(const uint4 &w, float ratio)
{
    return make_uint4(recode4(w.x, ratio), recode4(w.y, ratio), recode4(w.z, ratio), recode4(w.w, ratio));
}

// A run of rows of K, turned, or of V, for one head after another: Run (atom_kv8_append.h) on fp32 values, the maximum as the bits of a
// float.  Row r is token `token` + r; a wavefront has ROWS of them in registers (those of a longer run are read twice), with
// their angles, which all heads share.  ONCE: what is read is not kept in the caches.  LONGER: there may be runs of more than ROWS.
template <int D, int ROWS, bool ONE, bool NEIGHBOURS, bool ONCE, bool LONGER>
struct TurnedRun {
    static constexpr int LPR = D / 8, RPL = 64 / LPR, kLoads = ROWS / RPL;
    Angles ang[kLoads];
    uint2 raw[kLoads][2];
    float x[kLoads][8];
    int64_t token; int last;                                // (the last row that there is, of this run or not)
    int g, i, len, at, o;
    Channels ch;
    uint32_t axes;
    bool keys, turns;                                       // rows of K; channels of this lane that turn

    __device__ __forceinline__ void place(const Turn &t, int64_t tok, int T, bool turns_)
    {
        const int lane = threadIdx.x & 63;
        g = lane / LPR;
        i = lane % LPR;
        ch = channels(t, i);
        keys = turns_;
        turns = turns_ && ch.turned;
        axes = lane_axes(t, i);
        token = tok;
        last = (int)((int64_t)T - 1 - tok);
    }
    __device__ __forceinline__ int64_t token_of(int row) const { return token + min(row, last); }
    // near: the positions of 64 tokens, of which this run's first is `first`, a lane each
    __device__ __forceinline__ void fetch_angles(const Turn &t, const Positions &near, int first, int u)
    {
        if (!keys) return;
        const int row = u * RPL + g;
        Positions at;
        if (first + (u + 1) * RPL <= 64) {
            at.p[0] = __shfl(near.p[0], first + row, 64);
            if constexpr (!ONE)
#pragma unroll
                for (int a = 1; a < 4; ++a) at.p[a] = __shfl(near.p[a], first + row, 64);
        } else at = positions<ONE>(t, token_of(row));
        ang[u] = angles<ONE>(t, at, i, axes);
    }
    __device__ __forceinline__ void fetch(const Side &side, int h, int u)
    {
        const __half *p = side.x + token_of(u * RPL + g) * side.ld + (int64_t)h * D;
        raw[u][0] = load4<ONCE>(p + ch.lo);
        raw[u][1] = load4<ONCE>(p + ch.hi);
    }
    // a row beyond those in registers
    __device__ __forceinline__ void again(const Turn &t, const Side &side, int h, int row, float *v) const
    {
        const int64_t tok = token_of(row);
        const __half *p = side.x + tok * side.ld + (int64_t)h * D;
        widen(*reinterpret_cast<const uint2 *>(p + ch.lo), v);
        widen(*reinterpret_cast<const uint2 *>(p + ch.hi), v + 4);
        if (turns) turn<NEIGHBOURS>(v, angles<ONE>(t, positions<ONE>(t, tok), i, axes), 1.0f);
    }
    __device__ __forceinline__ uint32_t magnitude(int row, const float *v) const
    {
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = max(top, __builtin_bit_cast(uint32_t, v[k]) & 0x7fffffffu);
        return row < len ? top : 0;
    }

    // the rows that were fetched as fp32 values
    __device__ __forceinline__ void take()
    {
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (u * RPL < len) {
                widen(raw[u][0], x[u]);
                widen(raw[u][1], x[u] + 4);
                if (turns) turn<NEIGHBOURS>(x[u], ang[u], 1.0f);
            }
    }
    __device__ __forceinline__ uint32_t largest(const Turn &t, const Side &side, int h)
    {
        uint32_t top = 0;
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (u * RPL < len) top = max(top, magnitude(u * RPL + g, x[u]));
        for (int row = ROWS; LONGER && row < len; row += RPL) {
            float v[8];
            again(t, side, h, row + g, v);
            top = max(top, magnitude(row + g, v));
        }
        return wave_max(top);
    }

    __device__ __forceinline__ void store(int8_t *block, int row, const float *v, float r)
    {
        if (row >= len) return;
        // (a NaN that came with the table may have anything in its low byte)
        const uint32_t a = r > 0.0f ? codes4(v, r) : 0, b = r > 0.0f ? codes4(v + 4, r) : 0;
        *reinterpret_cast<uint32_t *>(block + (at + row) * D + ch.lo) = a;
        *reinterpret_cast<uint32_t *>(block + (at + row) * D + ch.hi) = b;
    }

    // `top` of the whole run, s_old of its block (0 where it begins the block); `thread` of `threads` that have one: the older rows are theirs in turn
    __device__ __forceinline__ void end(const Turn &t, const Side &side, int h, int64_t head, int shift, float s_old, uint32_t top, int thread, int threads)
    {
        int8_t *block = side.codes + (head << shift) * D;
        const Scale scale = scale_of(top, s_old);
        const float r = scale.r;
        if (scale.grown)
            for (int b = 16 * thread; b < o * D; b += 16 * threads)
                *reinterpret_cast<uint4 *>(block + b) = recode16(*reinterpret_cast<const uint4 *>(block + b), scale.ratio);
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (u * RPL < len) store(block, u * RPL + g, x[u], r);
        for (int row = ROWS; LONGER && row < len; row += RPL) {
            float v[8];
            again(t, side, h, row + g, v);
            store(block, row + g, v, r);
        }
        if (thread == 0) side.scale[head] = scale.s;
    }
};

// The first `bytes` of a block's codes on a grown scale, by a wavefront: eight pieces of a lane are on their way before the first is written (behind the last piece: that
// one again; loads under a condition each are slower).
__device__ __forceinline__ void recode_block(int8_t *block, int bytes, float ratio)
{
    constexpr int DEEP = 8;
    for (int b = 16 * (int)(threadIdx.x & 63); b < bytes; b += 1024 * DEEP) {
        uint4 w[DEEP];
#pragma unroll
        for (int u = 0; u < DEEP; ++u) w[u] = *reinterpret_cast<const uint4 *>(block + min(b + 1024 * u, bytes - 16));
#pragma unroll
        for (int u = 0; u < DEEP; ++u)
            if (b + 1024 * u < bytes) *reinterpret_cast<uint4 *>(block + b + 1024 * u) = recode16(w[u], ratio);
    }
}

// Runs of one row each, a row to D / 8 lanes: those of tokens t_first + l that begin one, l from `group` on in steps of `groups`, for heads h0 .. h1 - 1 of K (keys) or
// of V.  (Taken by a wavefront each, 300 tokens of 32 heads were 21.0 us, now 7.0, 1000 60 and 14.8.)
template <int D, bool ONE, bool NEIGHBOURS>
__device__ __forceinline__ void append_singles(const Turn &t, const Side &side, bool keys, const Window &w, const Positions &near, int64_t t_first, int slab,
                                               int Hkv, int shift, int h0, int h1, int group, int groups)
{
    constexpr int LPR = D / 8;
    const int i = threadIdx.x % LPR;
    const Channels ch = channels(t, i);
    const uint32_t axes = lane_axes(t, i);
    for (int l0 = 0; l0 < slab; l0 += groups) {
        const int l = min(l0 + group, 63);
        const int32_t slot = __shfl(w.got, l, 64);
        Positions at;
        at.p[0] = __shfl(near.p[0], l, 64);
        if constexpr (!ONE)
#pragma unroll
            for (int a = 1; a < 4; ++a) at.p[a] = __shfl(near.p[a], l, 64);
        const bool mine = l0 + group < slab && (w.leaders >> l & 1);
        if (!__ballot(mine)) continue;
        const __half *row = side.x + (t_first + l) * side.ld;
        uint2 lo, hi;
        Angles r;
        if (mine) {
            lo = load4<false>(row + h0 * D + ch.lo);
            hi = load4<false>(row + h0 * D + ch.hi);
            if (keys) r = angles<ONE>(t, at, i, axes);
        }
        const int o = slot & ((1 << shift) - 1);
        for (int h = h0; h < h1; ++h) {
            const uint32_t head = (uint32_t)(slot >> shift) * Hkv + h;         // (fewer than 2^31: host)
            Scale s = {};
            if (mine) {
                const float s_old = o > 0 ? side.scale[head] : 0.0f;
                float x[8];
                widen(lo, x);
                widen(hi, x + 4);
                if (h + 1 < h1) {
                    lo = load4<false>(row + (h + 1) * D + ch.lo);
                    hi = load4<false>(row + (h + 1) * D + ch.hi);
                }
                if (keys && ch.turned) turn<NEIGHBOURS>(x, r, 1.0f);
                uint32_t top = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) top = max(top, __builtin_bit_cast(uint32_t, x[k]) & 0x7fffffffu);
#pragma unroll
                for (int step = 1; step < LPR; step *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, step, 64));
                s = scale_of(top, s_old);
                int8_t *block = side.codes + ((int64_t)head << shift) * D;
                const uint32_t a = s.r > 0.0f ? codes4(x, s.r) : 0, b = s.r > 0.0f ? codes4(x + 4, s.r) : 0;
                *reinterpret_cast<uint32_t *>(block + o * D + ch.lo) = a;
                *reinterpret_cast<uint32_t *>(block + o * D + ch.hi) = b;
                if (i == 0) side.scale[head] = s.s;
            }
            // Older rows by the whole wavefront, as their arithmetic takes as long for a row's own lanes as for all.  (Steps of 64 tokens of 32 heads behind one another, where
            // some scales grow with every step, at rows 24 to 63 of blocks of 64: 6.6 us, by a row's own lanes 14.7; 4.4 where none grows.)
            for (uint64_t grown = __ballot(mine && s.grown && i == 0); grown; grown &= grown - 1) {
                const int from = __builtin_ctzll(grown);
                recode_block(side.codes + ((int64_t)(uint32_t)__builtin_amdgcn_readlane((int)head, from) << shift) * D, __builtin_amdgcn_readlane(o, from) * D,
                             __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, s.ratio), from)));
            }
        }
    }
}

struct Queries { const __half *x; int64_t ld; __half *out; int64_t ldo; int heads; };

constexpr int kQueryHeads = 4;                               // of a lane, in flight together; through the caches (where the step comes from the projection before it:
                                                             // 1116 tokens, 64 heads on 8, 13.9 us; past the caches 15.6, and up to 5 % less where nothing is cached)

// Eight channels of a lane, for `count` heads of a token from h0 on.
template <int D, bool ONE, bool NEIGHBOURS>
__device__ __forceinline__ void turn_queries(const Queries &q, const Turn &t, int64_t token, int i, int h0, int count)
{
    const Channels ch = channels(t, i);
    const Positions where = positions<ONE>(t, token);        // (first, so that the table's row is asked for while the heads come)
    const __half *x = q.x + token * q.ld + (int64_t)h0 * D;
    __half *out = q.out + token * q.ldo + (int64_t)h0 * D;
    uint2 raw[kQueryHeads][2];
    auto fetch = [&](int h) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kQueryHeads; ++u) {
            const int at = min(h + u, count - 1) * D;
            raw[u][0] = load4<false>(x + at + ch.lo);
            raw[u][1] = load4<false>(x + at + ch.hi);
        }
    };
    fetch(0);
    const Angles r = angles<ONE>(t, where, i, lane_axes(t, i));
    for (int h = 0; h < count; h += kQueryHeads) {
        if (h) fetch(h);
#pragma unroll
        for (int u = 0; u < kQueryHeads; ++u) {
            if (h + u >= count) break;
            float v[8];
            widen(raw[u][0], v);
            widen(raw[u][1], v + 4);
            if (ch.turned) turn<NEIGHBOURS>(v, r, 1.0f);
            *reinterpret_cast<uint2 *>(out + (h + u) * D + ch.lo) = narrow(v);
            *reinterpret_cast<uint2 *>(out + (h + u) * D + ch.hi) = narrow(v + 4);
        }
    }
}

struct Step {
    Queries q; Side k, v;
    Turn turn;
    const int32_t *slot; int32_t slots;
    int T, Hkv, shift;
    int slab, heads;                                         // of a workgroup: tokens, cache heads
    uint32_t appends;                                        // workgroups that append; the others turn queries
    int q_heads;                                             // heads of a lane there
};

template <int D, int THREADS, bool ONE, bool NEIGHBOURS>
__device__ __forceinline__ void query_group(const Step &p, uint32_t group)
{
    constexpr int LPR = D / 8;
    const int chunks = (p.q.heads + p.q_heads - 1) / p.q_heads;
    const uint32_t row = group * (THREADS / LPR) + threadIdx.x / LPR, token = row / (uint32_t)chunks;      // (2^24 workgroups at most)
    if (token >= (uint32_t)p.T) return;
    const int h0 = (int)(row - token * chunks) * p.q_heads;
    turn_queries<D, ONE, NEIGHBOURS>(p.q, p.turn, token, threadIdx.x % LPR, h0, min(p.q_heads, p.q.heads - h0));
}

// Few tokens: one wavefront for a head (of K or of V) and a token; where a run begins with that token it writes the run, whole.  Bound by its
// chain of reads, so the token's position, angles and row are on their way before its slot is known.
template <int D, bool ONE, bool NEIGHBOURS>
__global__ __launch_bounds__(256)
void rotary_kv8_kernel(Step p)
{
    if (blockIdx.x >= p.appends) return query_group<D, 256, ONE, NEIGHBOURS>(p, blockIdx.x - p.appends);
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t item = blockIdx.x * 4 + wave, token = item / (uint32_t)(2 * p.Hkv);
    const int which = (int)(item - token * (2 * p.Hkv));
    const int64_t t = token;
    if (t >= p.T) return;
    const bool is_k = which < p.Hkv;
    const int h = is_k ? which : which - p.Hkv;
    const Side side = is_k ? p.k : p.v;
    TurnedRun<D, 16, ONE, NEIGHBOURS, false, false> run;
    // (what the rest waits for in turn comes first: slots, positions, then the row, then the angles)
    const Slots slots = slots_from(p.slot, p.T, t);
    const Positions near = positions<ONE>(p.turn, min(t + (threadIdx.x & 63), (int64_t)p.T - 1));
    run.place(p.turn, t, p.T, is_k);
    run.fetch(side, h, 0);
    run.fetch_angles(p.turn, near, 0, 0);
    const Window w = window(slots, p.slots, p.T, t, 1, 1 << p.shift);
    if (!w.leaders) return;
    const int32_t first = __builtin_amdgcn_readlane(w.got, 0);
    run.o = run.at = first & ((1 << p.shift) - 1);
    const int64_t head = (int64_t)(first >> p.shift) * p.Hkv + h;
    const float s_old = run.o > 0 ? side.scale[head] : 0.0f;
    run.len = run_length(p.slot, p.T, w, t, 0, 1 << p.shift);
#pragma unroll
    for (int u = 1; u < run.kLoads; ++u)
        if (u * run.RPL < run.len) {
            run.fetch(side, h, u);
            run.fetch_angles(p.turn, near, 0, u);
        }
    run.take();
    run.end(p.turn, side, h, head, p.shift, s_old, run.largest(p.turn, side, h), threadIdx.x & 63, 64);
}

// Many tokens: a workgroup of four wavefronts (eight for blocks of 128) for `slab` tokens and some heads of K or of V writes the runs that begin among them, each whole, also past
// the slab's end.  Up to three runs are written by all of them, ROWS rows each; more of them, and runs of blocks of ROWS at most (LONG: of more), one by each in turn.
// ROWS is 16: 32 rows of 128 channels with their angles are all registers of a SIMD's lane, and one workgroup a CU (15000 tokens of 32 heads, blocks of
// 32, 396 us for 153; blocks of 128, four wavefronts of 32 rows, 231 for 175).  Past the caches where blocks are longer and heads of 128 (2381 tokens of 32
// heads, blocks of 64, 56.5 us and 60.8 through them; heads of 64 33.3 and 30.4).  10240 tokens of 32 heads and as many query heads, blocks of 64: 86.4 us.
template <int D, int ROWS, int WAVES, bool ONE, bool NEIGHBOURS, bool LONG>
__global__ __launch_bounds__(64 * WAVES)
void rotary_kv8_many_kernel(Step p)
{
    __shared__ uint32_t s_top[2][WAVES];
    if (blockIdx.x >= p.appends) return query_group<D, 64 * WAVES, ONE, NEIGHBOURS>(p, blockIdx.x - p.appends);
    const int chunks = (p.Hkv + p.heads - 1) / p.heads;
    const int64_t group = blockIdx.x / (2 * chunks), t_first = group * p.slab;
    const int which = (int)(blockIdx.x - group * (2 * chunks));
    const bool is_k = which < chunks;
    const int h0 = (is_k ? which : which - chunks) * p.heads, h1 = min(h0 + p.heads, p.Hkv);
    const Side side = is_k ? p.k : p.v;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), bs = 1 << p.shift;
    const Slots slots = slots_from(p.slot, p.T, t_first);
    const Positions near = positions<ONE>(p.turn, min(t_first + (threadIdx.x & 63), (int64_t)p.T - 1));
    const Window w = window(slots, p.slots, p.T, t_first, p.slab, bs);         // (the same in all of them)
    if (p.slab < 64 && !(w.followers & (((uint64_t)2 << p.slab) - 2))) {       // single tokens (or none)
        constexpr int RPL = 512 / D;
        append_singles<D, ONE, NEIGHBOURS>(p.turn, side, is_k, w, near, t_first, p.slab, p.Hkv, p.shift, h0, h1,
                                           wave * RPL + (int)(threadIdx.x & 63) / (D / 8), WAVES * RPL);
        return;
    }
    const bool alone = !LONG || __builtin_popcountll(w.leaders) > 3;
    int turn = 0, sync = 0;                                                  // of the runs; nobody writes maxima before all have read the last but one's
    for (uint64_t leaders = w.leaders; leaders; leaders &= leaders - 1, ++turn) {
        if (alone && (turn & (WAVES - 1)) != wave) continue;
        const int l0 = __builtin_ctzll(leaders), len = run_length(p.slot, p.T, w, t_first, l0, bs);
        const int row0 = alone ? 0 : wave * ROWS;
        const int32_t first = __builtin_amdgcn_readlane(w.got, l0);
        TurnedRun<D, ROWS, ONE, NEIGHBOURS, LONG && D == 128, LONG> run;
        run.place(p.turn, t_first + l0 + row0, p.T, is_k);
        run.o = first & (bs - 1);
        run.at = run.o + row0;
        run.len = alone ? len : min(max(len - row0, 0), ROWS);
#pragma unroll
        for (int u = 0; u < run.kLoads; ++u)
            if (u * run.RPL < run.len) run.fetch(side, h0, u);
#pragma unroll
        for (int u = 0; u < run.kLoads; ++u)
            if (u * run.RPL < run.len) run.fetch_angles(p.turn, near, l0 + row0, u);
        for (int h = h0; h < h1; ++h) {
            const int64_t head = (int64_t)(first >> p.shift) * p.Hkv + h;
            const float s_old = run.o > 0 ? side.scale[head] : 0.0f;
            run.take();
#pragma unroll
            for (int u = 0; u < run.kLoads; ++u)
                if (u * run.RPL < run.len && h + 1 < h1) run.fetch(side, h + 1, u);
            uint32_t top = run.largest(p.turn, side, h);
            if (!alone) {
                uint32_t *tops = s_top[sync++ & 1];
                if ((threadIdx.x & 63) == 0) tops[wave] = top;
                __syncthreads();
                top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
#pragma unroll
                for (int v = 4; v < WAVES; ++v) top = max(top, tops[v]);
            }
            run.end(p.turn, side, h, head, p.shift, s_old, top, alone ? threadIdx.x & 63 : threadIdx.x, alone ? 64 : 64 * WAVES);
        }
    }
}

}  // namespace

namespace atom_internal {

// How a call runs: tokens to a workgroup (0: a wavefront for each token and head), cache heads to a workgroup, workgroups that append;
// query heads to a lane, workgroups that turn them.
struct TurnShape { int slab, heads; int64_t appends; int q_heads; int64_t queries; int threads; };

//
// A wavefront for each token and head is the shorter chain for a few single tokens (20 of 32 heads 3.6 us and 3.7 by workgroups, 100 5.5 and 5.0), and slow
// where one has a long run to itself (a prompt of 60 tokens, blocks of 64, 15.0 and 5.2).  Tokens to a workgroup: eight while there are few, then 32
// (300 tokens of 32 heads in runs of one, each by a wavefront, blocks of 64: 64 of them 34.0 us, 32 21.1; a step with chunks of 200 26.1 and 23.2), 64 with many.
// Heads are shared out while there are fewer than 1024 workgroups.
constexpr int kFewTokens = 16;                               // (so no run is longer than the rows that a wavefront keeps)

static TurnShape turn_shape(int64_t T, int H, int Hkv, int D, int block_tokens)
{
    TurnShape s = {};
    s.threads = 256;
    const int64_t items = T * 2 * Hkv;
    if (T < kFewTokens) {
        s.heads = 1;
        s.appends = (items + 3) / 4;
    } else {
        if (block_tokens == 128) s.threads = 512;
        s.slab = items <= 16384 ? 8 : block_tokens >= 64 && items > 131072 ? 64 : 32;
        const int64_t slabs = (T + s.slab - 1) / s.slab;
        s.heads = 8;
        while (s.heads > 1 && slabs * 2 * ((Hkv + s.heads - 1) / s.heads) < 1024) s.heads /= 2;
        s.appends = slabs * 2 * ((Hkv + s.heads - 1) / s.heads);
    }
    s.q_heads = 8;
    const int64_t rows = s.threads / (D / 8);
    while (s.q_heads > 1 && T * ((H + s.q_heads - 1) / s.q_heads) / rows < 512) s.q_heads /= 2;
    s.queries = (T * ((H + s.q_heads - 1) / s.q_heads) + rows - 1) / rows;
    return s;
}

bool rotary_kv8_fits(int64_t T, int H, int Hkv, int D, int block_tokens)
{
    const TurnShape s = turn_shape(T, H, Hkv, D, block_tokens);
    return s.appends + s.queries <= atom_launch::kMostThreads / s.threads;
}

hipError_t launch_rotary_kv8_append(const RotaryKv8 &a, hipStream_t stream)
{
    const TurnShape s = turn_shape(a.T, a.H, a.Hkv, a.D, a.block_tokens);
    const Step p = {{(const __half *)a.q, a.ldq, (__half *)a.q_out, a.ldqo, a.H},
                    {(const __half *)a.k, a.ldk, (int8_t *)a.k_codes, a.k_scale},
                    {(const __half *)a.v, a.ldv, (int8_t *)a.v_codes, a.v_scale},
                    a.turn, a.slot, (int32_t)(a.n_blocks * a.block_tokens), (int)a.T, a.Hkv, __builtin_ctz((unsigned)a.block_tokens),
                    s.slab, s.heads, (uint32_t)s.appends, s.q_heads};
    const dim3 grid((unsigned)(s.appends + s.queries));
#define ATOM_TURN(D, ONE, NEIGHBOURS)                                                                                      \
    do {                                                                                                                   \
        auto kern = !s.slab ? &rotary_kv8_kernel<D, ONE, NEIGHBOURS>                                                       \
                    : a.block_tokens == 16  ? &rotary_kv8_many_kernel<D, 16, 4, ONE, NEIGHBOURS, false>                    \
                    : a.block_tokens == 128 ? &rotary_kv8_many_kernel<D, 16, 8, ONE, NEIGHBOURS, true>                     \
                                            : &rotary_kv8_many_kernel<D, 16, 4, ONE, NEIGHBOURS, true>;                    \
        hipLaunchKernelGGL(kern, grid, dim3(s.threads), 0, stream, p);                                                          \
    } while (0)
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
