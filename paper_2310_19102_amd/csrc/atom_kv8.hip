// Paged 8-bit KV cache for gfx950: block tables and slot maps from the requests' lengths, and the
// operator that quantises a step's keys and values into the blocks (Section 4.5 of the paper serves
// from a paged cache; atom_kv8_attention.hip reads it).
//
// Cache layout (one K cache and one V cache, same shape):
//   codes [n_blocks, Hkv, block_tokens, D] int8,  scale [n_blocks, Hkv] fp32
// i.e. one scale for each block of tokens and head: 8 + 32 / (block_tokens * D) bits per element.

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include "atom_internal.h"
#include "atom_launch.h"

namespace {

// ---------------------------------------------------------------- block tables and slot maps

constexpr int kMapThreads = 1024;

__device__ __forceinline__ int32_t saturate(int64_t v) { return v > 0x7fffffffLL ? 0x7fffffff : (int32_t)v; }

// One launch; every workgroup scans all B requests by itself (two int32 per request in its LDS: first token, first taken
// block) and then writes its share of the table and of the slots, so nothing waits for another workgroup.  A slot whose
// page is a new one reads the free list, not the table, which another workgroup may be writing.
// Bound by its own latency: two dependent reads and the scan, 1024 requests a round.
__global__ __launch_bounds__(kMapThreads)
void kv_block_map_kernel(const int32_t *__restrict__ past, const int32_t *__restrict__ fresh, int B, int shift,
                         const int32_t *__restrict__ free_blocks, int64_t n_free, const int32_t *__restrict__ cursor,
                         int32_t *table, int W, int T, int32_t *__restrict__ token_start, int32_t *__restrict__ seq_len,
                         int32_t *__restrict__ slot, int32_t *__restrict__ cursor_out)
{
    extern __shared__ int32_t s_first[];                     // [B + 1] first token, [B] first taken block
    __shared__ int64_t s_wave[2][kMapThreads / 64];
    int32_t *s_token = s_first, *s_taken = s_first + B + 1;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int bs = 1 << shift;
    const int64_t start = cursor ? *cursor : 0;
    const bool first_group = blockIdx.x == 0;

    auto pages = [&](int64_t tokens) -> int { const int64_t n = (tokens + bs - 1) >> shift; return n < W ? (int)n : W; };
    int64_t tokens = 0, taken = 0;                           // of the requests before this round
    for (int base = 0; base < B; base += kMapThreads) {
        const int b = base + tid;
        const int64_t p = b < B ? max(past[b], 0) : 0, n = b < B ? max(fresh[b], 0) : 0;
        const int64_t mine[2] = {n, pages(p + n) - pages(p)};
        int64_t sum[2] = {mine[0], mine[1]};                 // inclusive over the wavefront, then exclusive over all
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int64_t v = __shfl_up(sum[k], d, 64);
                if (lane >= d) sum[k] += v;
            }
        __syncthreads();                                     // (the last round's sums are read)
        if (lane == 63) {
            s_wave[0][wave] = sum[0];
            s_wave[1][wave] = sum[1];
        }
        __syncthreads();
        int64_t before[2] = {tokens, taken};
#pragma unroll 2
        for (int w = 0; w < kMapThreads / 64; ++w) {
            const int64_t v0 = s_wave[0][w], v1 = s_wave[1][w];
            if (w < wave) { before[0] += v0; before[1] += v1; }
            tokens += v0;
            taken += v1;
        }
        if (b < B) {
            const int32_t at = saturate(before[0] + sum[0] - mine[0]);
            s_token[b] = at;
            s_taken[b] = saturate(before[1] + sum[1] - mine[1]);
            if (first_group) {
                token_start[b] = at;
                seq_len[b] = saturate(p + n);
            }
        }
    }
    const int32_t total = saturate(tokens);
    if (tid == 0) {
        s_token[B] = total;
        if (first_group) {
            token_start[B] = total;
            if (cursor_out) *cursor_out = saturate(start + taken);
        }
    }
    __syncthreads();

    auto taken_block = [&](int b, int nth) -> int32_t {      // the nth block that request b takes
        const int64_t f = start + s_taken[b] + nth;
        return f >= 0 && f < n_free ? free_blocks[f] : -1;
    };
    const int64_t step = (int64_t)gridDim.x * kMapThreads, me = (int64_t)blockIdx.x * kMapThreads + tid;
    for (int64_t e = me; e < (int64_t)B * W; e += step) {
        const int b = (int)((uint32_t)e / (uint32_t)W), j = (int)((uint32_t)e - (uint32_t)b * (uint32_t)W);
        const int64_t p = max(past[b], 0), n = max(fresh[b], 0);
        const int have = pages(p);
        if (j >= have) table[e] = j < pages(p + n) ? taken_block(b, j - have) : -1;
    }
    for (int64_t t = me; t < T; t += step) {
        int32_t where = -1;
        if (t < total) {
            int lo = 0, hi = B;                              // the last request that starts at or before t
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_token[mid] <= t) lo = mid;
                else hi = mid;
            }
            const int64_t p0 = max(past[lo], 0), p = p0 + (t - s_token[lo]);
            const int64_t j = p >> shift;
            if (j < W) {
                const int have = pages(p0);
                const int32_t page = j < have ? table[(int64_t)lo * W + j] : taken_block(lo, (int)j - have);
                const int64_t at = ((int64_t)page << shift) + (p & (bs - 1));
                if (page >= 0 && at <= 0x7fffffffLL) where = (int32_t)at;
            }
        }
        slot[t] = where;
    }
}

// ---------------------------------------------------------------- quantise and append

typedef unsigned short us2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pair_max_u16(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b)));
}

// The larger magnitude of each half (of finite numbers: their bits without the sign are in order).
__device__ __forceinline__ uint32_t magnitudes(const uint4 &v)
{
    constexpr uint32_t m = 0x7fff7fffu;
    return pair_max_u16(pair_max_u16(v.x & m, v.y & m), pair_max_u16(v.z & m, v.w & m));
}

// clamp(rne(v), -127, 127) in the low byte: adding 1.5 * 2^23 rounds to the nearest even integer and leaves it there.
__device__ __forceinline__ uint32_t code_of(float v)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(v, -127.0f, 127.0f) + 12582912.0f);
}
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), hi = __builtin_amdgcn_perm(d, c, 0x04000c0cu);
    return lo | hi;
}
__device__ __forceinline__ uint32_t codes4(uint32_t h01, uint32_t h23, float r)
{
    const __half2 a = __builtin_bit_cast(__half2, h01), b = __builtin_bit_cast(__half2, h23);
    return pack4(code_of(__low2float(a) * r), code_of(__high2float(a) * r), code_of(__low2float(b) * r),
                 code_of(__high2float(b) * r));
}
__device__ __forceinline__ uint32_t recode4(uint32_t w, float ratio)
{
    auto c = [&](int i) { return code_of((float)(int8_t)(w >> (8 * i)) * ratio); };
    return pack4(c(0), c(1), c(2), c(3));
}

// One wavefront for a head (of K or of V) and `slab` tokens: it finds the runs that begin among them (a run: tokens whose
// slots follow one another inside one block) and writes each whole, also past the slab's end.  A run's scale is the larger of the block's
// (where the block holds older rows, those before the run's first) and max|x| / 127:
//   s = max(s_old, max|x| / 127), r = 1 / s, code = clamp(rne(x * r), -127, 127)   IEEE fp32, every step rounded once
// and where s grows, the older rows become rne(code * (s_old / s)).
// Rows stay in registers between the maximum and the codes (64 rows; a longer run is read twice, the second time
// from the cache).  16-byte loads, 8 values a lane: D / 8 lanes a row.
template <int D>
__global__ __launch_bounds__(256)
void kv8_append_kernel(const __half *__restrict__ xk, const __half *__restrict__ xv, int T, int64_t ldk, int64_t ldv, int Hkv,
                       const int32_t *__restrict__ slot, int32_t slots, int shift, int slab, int8_t *__restrict__ kq,
                       float *__restrict__ ks, int8_t *__restrict__ vq, float *__restrict__ vs)
{
    constexpr int LPR = D / 8, RPL = 64 / LPR, kLoads = 64 / RPL;   // lanes a row, rows a load, loads of 64 rows
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t group = item / (2 * Hkv);
    const int which = (int)(item - group * (2 * Hkv)), h = which % Hkv;
    const bool is_v = which >= Hkv;
    const int64_t t_first = group * slab;
    if (t_first >= T) return;
    const int bs = 1 << shift;

    const int32_t got = slot[min(t_first + lane, (int64_t)T - 1)];
    const bool    valid = t_first + lane < T && got >= 0 && got < slots;
    int32_t prev = __shfl_up(got, 1, 64);
    if (lane == 0) prev = t_first > 0 ? slot[t_first - 1] : -2;
    const bool follows = prev >= 0 && prev < slots && got == prev + 1 && (got & (bs - 1)) != 0;
    uint64_t leaders = __ballot(valid && !follows && lane < slab);

    const __half *x = (is_v ? xv : xk) + (int64_t)h * D;
    const int64_t ld = is_v ? ldv : ldk;
    int8_t *cq = is_v ? vq : kq;
    float  *cs = is_v ? vs : ks;
    const int j = lane % LPR, g = lane / LPR;

    while (leaders) {
        const int l0 = __builtin_ctzll(leaders);
        leaders &= leaders - 1;
        const int32_t first = __builtin_amdgcn_readlane(got, l0);
        const int     o = first & (bs - 1);
        // length of the run: in the slots at hand, and beyond them if it goes on there
        const uint64_t same = __ballot(valid && lane >= l0 && got == first + (lane - l0) && o + (lane - l0) < bs) >> l0;
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
        const int64_t at = (int64_t)(first >> shift) * Hkv + h;             // block and head
        const float   s_old = o > 0 ? cs[at] : 0.0f;
        const __half *rows = x + (t_first + l0) * ld + 8 * j;
        auto load = [&](int row) { return *reinterpret_cast<const uint4 *>(rows + (int64_t)min(row, len - 1) * ld); };

        uint4 raw[kLoads];
        uint32_t top = 0;
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (u * RPL < len) raw[u] = load(u * RPL + g);
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (u * RPL < len) top = pair_max_u16(top, magnitudes(raw[u]));
        for (int row = 64; row < len; row += RPL) top = pair_max_u16(top, magnitudes(load(row + g)));
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) top = pair_max_u16(top, (uint32_t)__shfl_xor((int)top, d, 64));
        top = max(top & 0xffffu, top >> 16);
        const float amax = __half2float(__ushort_as_half((unsigned short)top));
        const float s_new = amax / 127.0f, s = s_new > s_old ? s_new : s_old;
        const float r = s > 0.0f ? 1.0f / s : 0.0f;

        int8_t *block = cq + (at << shift) * D;
        auto store = [&](int row, const uint4 &v) {
            if (row < len)
                *reinterpret_cast<uint2 *>(block + (o + row) * D + 8 * j) = make_uint2(codes4(v.x, v.y, r), codes4(v.z, v.w, r));
        };
        if (s > s_old && s_old > 0.0f) {                                    // the older rows on the new scale
            const float ratio = s_old / s;
            for (int i = 16 * lane; i < o * D; i += 1024) {
                uint4 w = *reinterpret_cast<const uint4 *>(block + i);
                w = make_uint4(recode4(w.x, ratio), recode4(w.y, ratio), recode4(w.z, ratio), recode4(w.w, ratio));
                *reinterpret_cast<uint4 *>(block + i) = w;
            }
        }
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (u * RPL < len) store(u * RPL + g, raw[u]);
        for (int row = 64; row < len; row += RPL) store(row + g, load(row + g));
        if (lane == 0) cs[at] = s;
    }
}

}  // namespace

namespace atom_internal {

hipError_t launch_kv_block_map(const int32_t *past, const int32_t *fresh, int B, int block_tokens, const int32_t *free_blocks,
                               int64_t n_free, const int32_t *cursor, int32_t *table, int64_t W, int64_t T,
                               int32_t *token_start, int32_t *seq_len, int32_t *slot, int32_t *cursor_out, hipStream_t stream)
{
    const size_t lds = (size_t)(2 * B + 1) * sizeof(int32_t);
    static atom_launch::LdsOptIn opt;
    if (lds > 60 * 1024) {
        hipError_t err = atom_launch::ensure_dynamic_lds(opt, reinterpret_cast<const void *>(&kv_block_map_kernel), lds);
        if (err != hipSuccess) return err;
    }
    const int64_t work = (int64_t)B * W + T;
    int64_t grid = (work + 4 * kMapThreads - 1) / (4 * kMapThreads);
    if (grid > 256) grid = 256;
    if (grid < 1) grid = 1;
    hipLaunchKernelGGL(kv_block_map_kernel, dim3((unsigned)grid), dim3(kMapThreads), lds, stream, past, fresh, B,
                       __builtin_ctz((unsigned)block_tokens), free_blocks, n_free, cursor, table, (int)W, (int)T, token_start,
                       seq_len, slot, cursor_out);
    return hipGetLastError();
}

hipError_t launch_kv8_append(const void *k, const void *v, int64_t T, int64_t ldk, int64_t ldv, int Hkv, int D,
                             const int32_t *slot, int64_t n_blocks, int block_tokens, void *k_codes, float *k_scale,
                             void *v_codes, float *v_scale, hipStream_t stream)
{
    const int64_t heads = 2 * (int64_t)Hkv;
    const int     slab = T * heads <= 16384 ? 1 : T * heads <= 131072 ? 4 : 16;
    const int64_t waves = (T + slab - 1) / slab * heads, grid = (waves + 3) / 4;
    if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
    auto kern = D == 128 ? &kv8_append_kernel<128> : &kv8_append_kernel<64>;
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(256), 0, stream, (const __half *)k, (const __half *)v, (int)T, ldk, ldv,
                       Hkv, slot, (int32_t)(n_blocks * block_tokens), __builtin_ctz((unsigned)block_tokens), slab,
                       (int8_t *)k_codes, k_scale, (int8_t *)v_codes, v_scale);
    return hipGetLastError();
}

}  // namespace atom_internal
