// Quantising a run of rows into a block of the paged 8-bit cache: what the append (atom_kv8.hip) and the append of turned
// keys (atom_rotary_kv8.hip) share.
#ifndef ATOM_KV8_APPEND_H
#define ATOM_KV8_APPEND_H

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

namespace atom_kv8 {

typedef unsigned short us2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pair_max_u16(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b)));
}

// The larger magnitude of each half: their bits without the sign are in order, infinity above all numbers and NaN above that.
__device__ __forceinline__ uint32_t magnitudes(const uint4 &v)
{
    constexpr uint32_t m = 0x7fff7fffu;
    return pair_max_u16(pair_max_u16(v.x & m, v.y & m), pair_max_u16(v.z & m, v.w & m));
}

// The largest of the wavefront's values (none is below zero), in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
#define ATOM_STEP(ctrl, rows) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xF, false))
    ATOM_STEP(0x111, 0xF);
    ATOM_STEP(0x112, 0xF);
    ATOM_STEP(0x114, 0xF);
    ATOM_STEP(0x118, 0xF);
    ATOM_STEP(0x142, 0xA);
    ATOM_STEP(0x143, 0xC);
#undef ATOM_STEP
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// rne(v) in the low byte, for |v| <= 127.5: adding 1.5 * 2^23 rounds to the nearest even integer and leaves it there.  The clamp to 127 is implied: a value is at
// most max|x|, the scale at least max|x| / 127, each of the three roundings on the way below 2^-23 of 127.  Under a scale that is not finite the factor is 0, and
// so are the codes: also of NaN, whose low byte is 0 when it comes from a half (the low 13 bits of its significand are).
__device__ __forceinline__ uint32_t code_of(float v) { return __builtin_bit_cast(uint32_t, v + 12582912.0f); }
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
// (x * r + 0 is x * r, as one instruction that takes half of a register)
__device__ __forceinline__ uint32_t codes4(uint32_t h01, uint32_t h23, float r)
{
    const __half2 a = __builtin_bit_cast(__half2, h01), b = __builtin_bit_cast(__half2, h23);
    return pack4(code_of(fmaf(__low2float(a), r, 0.0f)), code_of(fmaf(__high2float(a), r, 0.0f)), code_of(fmaf(__low2float(b), r, 0.0f)),
                 code_of(fmaf(__high2float(b), r, 0.0f)));
}
__device__ __forceinline__ uint32_t recode4(uint32_t w, float ratio)
{
    auto c = [&](int i) { return code_of((float)(int8_t)(w >> (8 * i)) * ratio); };
    return pack4(c(0), c(1), c(2), c(3));
}

// What a call writes to and from, of K or of V.
struct Side { const __half *x; int64_t ld; int8_t *codes; float *scale; };

// A wavefront's window of 64 slots: which of the first `slab` tokens begin a run (a run: tokens whose slots follow one another inside one block), which of all go on with one.
struct Window { int32_t got; bool valid; uint64_t leaders, followers; };

// What it reads: a lane's slot and the one before the first.
struct Slots { int32_t got, before; };

__device__ __forceinline__ Slots slots_from(const int32_t *__restrict__ slot, int T, int64_t t_first)
{
    return {slot[min(t_first + (threadIdx.x & 63), (int64_t)T - 1)], slot[max(t_first - 1, (int64_t)0)]};
}

__device__ __forceinline__ Window window(const Slots &s, int32_t slots, int T, int64_t t_first, int slab, int bs)
{
    const int lane = threadIdx.x & 63;
    Window w;
    w.got = s.got;
    w.valid = t_first + lane < T && w.got >= 0 && w.got < slots;
    int32_t prev = __shfl_up(w.got, 1, 64);
    if (lane == 0) prev = t_first > 0 ? s.before : -2;
    const bool follows = prev >= 0 && prev < slots && w.got == prev + 1 && (w.got & (bs - 1)) != 0;
    w.leaders = __ballot(w.valid && !follows && lane < slab);
    w.followers = __ballot(w.valid && follows);
    return w;
}

__device__ __forceinline__ Window window(const int32_t *__restrict__ slot, int32_t slots, int T, int64_t t_first, int slab, int bs)
{
    return window(slots_from(slot, T, t_first), slots, T, t_first, slab, bs);
}

// The run that token t_first + l0 begins: from its slots at hand, and from those beyond them if it goes on there.
__device__ __forceinline__ int run_length(const int32_t *__restrict__ slot, int T, const Window &w, int64_t t_first, int l0, int bs)
{
    const int lane = threadIdx.x & 63;
    const int32_t first = __builtin_amdgcn_readlane(w.got, l0);
    const int o = first & (bs - 1);
    const uint64_t same = __ballot(w.valid && lane >= l0 && w.got == first + (lane - l0) && o + (lane - l0) < bs) >> l0;
    int len = ~same ? __builtin_ctzll(~same) : 64;
    if (len == 64 - l0)
        while (o + len < bs) {
            const int64_t t = t_first + l0 + len + lane;
            const bool ok = t < T && o + len + lane < bs && slot[min(t, (int64_t)T - 1)] == first + len + lane;
            const uint64_t m = __ballot(ok);
            const int more = ~m ? __builtin_ctzll(~m) : 64;
            len += more;
            if (more < 64) break;
        }
    return len;
}

// A run of one head's rows, by one wavefront.  A run's scale is the larger of the block's
// (where the block holds older rows, those before the run's first) and max|x| / 127:
//   s = max(s_old, max|x| / 127), r = 1 / s, code = clamp(rne(x * r), -127, 127)   IEEE fp32, every step rounded once
// and where s grows, the older rows become rne(code * (s_old / s)).  The maximum of a NaN and anything is NaN, so what is not finite stays in
// the scale, where readers find it.
// Rows stay in registers between the maximum and the codes (ROWS of them; those of a longer run are read twice, the second time
// from the cache).  16-byte loads, 8 values a lane: D / 8 lanes a row.
template <int D, int ROWS>
struct Run {
    static constexpr int LPR = D / 8, RPL = 64 / LPR, kLoads = ROWS / RPL;  // lanes a row, rows a load, loads of ROWS
    uint4 raw[kLoads];
    const __half *rows; int64_t ld;
    int8_t *block; float *scale;
    int o, at, len, g, j;                                                   // o: older rows; at: of the block, this wavefront's first row
    float s_old;

    // ONCE: with the hint that nothing reads the row again
    template <bool ONCE>
    __device__ __forceinline__ uint4 load(int row) const
    {
        typedef unsigned u4 __attribute__((ext_vector_type(4)));
        const u4 *p = reinterpret_cast<const u4 *>(rows + (int64_t)min(row, len - 1) * ld);
        const u4  v = ONCE ? __builtin_nontemporal_load(p) : *p;
        return make_uint4(v[0], v[1], v[2], v[3]);
    }

    // the run's rows (or ROWS of them from `row0` on) on their way to the registers, and their largest magnitude (the bits of a half)
    __device__ __forceinline__ uint32_t begin(const Side &side, int h, int Hkv, int32_t first, int len_, int64_t t, int shift, int row0 = 0)
    {
        const int lane = threadIdx.x & 63;
        g = lane / LPR;
        j = lane % LPR;
        len = len_;
        ld = side.ld;
        o = first & ((1 << shift) - 1);
        at = o + row0;
        const int64_t head = (int64_t)(first >> shift) * Hkv + h;           // block and head
        block = side.codes + (head << shift) * D;
        scale = side.scale + head;
        rows = side.x + (int64_t)h * D + (t + row0) * ld + 8 * j;
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (u * RPL < len) raw[u] = load<true>(u * RPL + g);
        s_old = o > 0 ? *scale : 0.0f;
        uint32_t top = 0;
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (u * RPL < len) top = pair_max_u16(top, magnitudes(raw[u]));
        for (int row = ROWS; row < len; row += RPL) top = pair_max_u16(top, magnitudes(load<false>(row + g)));
        return wave_max(max(top & 0xffffu, top >> 16));
    }

    __device__ __forceinline__ void store(int row, const uint4 &v, float r)
    {
        if (row < len)
            *reinterpret_cast<uint2 *>(block + (at + row) * D + 8 * j) = make_uint2(codes4(v.x, v.y, r), codes4(v.z, v.w, r));
    }

    // `top` of the whole run; `thread` of `threads` that have one: the older rows are theirs in turn
    __device__ __forceinline__ void end(uint32_t top, int thread, int threads)
    {
        const float amax = __half2float(__ushort_as_half((unsigned short)top));
        const float s_new = amax / 127.0f, s = s_new > s_old || s_new != s_new ? s_new : s_old;      // (NaN if either is)
        const float r = s > 0.0f ? 1.0f / s : 0.0f;
        if (s > s_old && s_old > 0.0f) {                                    // the older rows on the new scale
            const float ratio = s_old / s;
            for (int i = 16 * thread; i < o * D; i += 16 * threads) {
                uint4 w = *reinterpret_cast<const uint4 *>(block + i);
                w = make_uint4(recode4(w.x, ratio), recode4(w.y, ratio), recode4(w.z, ratio), recode4(w.w, ratio));
                *reinterpret_cast<uint4 *>(block + i) = w;
            }
        }
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (u * RPL < len) store(u * RPL + g, raw[u], r);
        for (int row = ROWS; row < len; row += RPL) store(row + g, load<false>(row + g), r);
        if (thread == 0) *scale = s;
    }
};

}  // namespace atom_kv8
#endif
