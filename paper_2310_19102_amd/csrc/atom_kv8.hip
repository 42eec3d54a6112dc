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

constexpr int kMapKept = 8192;                               // requests whose lengths a workgroup keeps

__device__ __forceinline__ int32_t saturate(int64_t v) { return v > 0x7fffffffLL ? 0x7fffffff : (int32_t)v; }

// Sum over the lanes up to this one, on the vector unit.
__device__ __forceinline__ int64_t running(int64_t v)
{
#define ATOM_STEP(ctrl, rows)                                                                                        \
    {                                                                                                                \
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, ctrl, rows, 0xF, false);      \
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(v >> 32), ctrl, rows, 0xF, false);        \
        v += (int64_t)(((uint64_t)hi << 32) | lo);                                                                   \
    }
    ATOM_STEP(0x111, 0xF)                                    // one, two, four, eight lanes below in the row of 16
    ATOM_STEP(0x112, 0xF)
    ATOM_STEP(0x114, 0xF)
    ATOM_STEP(0x118, 0xF)
    ATOM_STEP(0x142, 0xA)                                    // the row below's last lane, into rows 1 and 3
    ATOM_STEP(0x143, 0xC)                                    // the lower half's, into the upper
#undef ATOM_STEP
    return v;
}
__device__ __forceinline__ int64_t of_lane(int64_t v, int lane)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane);
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

// One launch; every workgroup scans all B requests by itself (per request its first token, its first taken block and, of up to 8192, both
// lengths in its LDS) and then writes its share of the table and of the slots, so nothing waits for another workgroup.  A slot whose
// page is a new one reads the free list, not the table, which another workgroup may be writing.
// Bound by its latency: the lengths, one barrier (three in a round of many requests), the search in LDS, the free list.  200 requests with a table of 300 columns: with a
// scan by lane exchanges through LDS, lengths read again for each entry and four entries a thread in turn 7.7 us, 4.5 so; one request 2.4, 1024 with a table of 1024 columns 7.4.
template <int THREADS, bool KEPT>
__global__ __launch_bounds__(THREADS)
void kv_block_map_kernel(const int32_t *__restrict__ past, const int32_t *__restrict__ fresh, int B, int shift,
                         const int32_t *__restrict__ free_blocks, int64_t n_free, const int32_t *__restrict__ cursor,
                         int32_t *table, int W, uint32_t w_mul, int w_shift, int T, int32_t *__restrict__ token_start, int32_t *__restrict__ seq_len,
                         int32_t *__restrict__ slot, int32_t *__restrict__ cursor_out)
{
    constexpr int kWaves = THREADS / 64;
    extern __shared__ int32_t s_first[];                     // [B + 1] first token, [B] first taken block, and of KEPT [B] past, [B] new
    __shared__ int64_t s_wave[2][kWaves];
    int32_t *s_token = s_first, *s_taken = s_first + B + 1, *s_past = s_taken + B, *s_new = s_past + B;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int bs = 1 << shift;
    const int64_t start = cursor ? *cursor : 0;
    const bool first_group = blockIdx.x == 0;

    auto pages = [&](int64_t tokens) -> int { const int64_t n = (tokens + bs - 1) >> shift; return n < W ? (int)n : W; };
    int64_t tokens = 0, taken = 0;                           // of the requests before this round
    for (int base = 0; base < B; base += THREADS) {
        const int b = base + tid;
        const int64_t p = b < B ? max(past[b], 0) : 0, n = b < B ? max(fresh[b], 0) : 0;
        const int64_t blocks = pages(p + n) - pages(p);
        const int64_t sum0 = running(n), sum1 = running(blocks);         // inclusive over the wavefront
        int64_t before0 = tokens, before1 = taken;
        if constexpr (kWaves > 1) {
            if (base) __syncthreads();                       // (the last round's sums are read)
            if (lane == 63) {
                s_wave[0][wave] = sum0;
                s_wave[1][wave] = sum1;
            }
            __syncthreads();
            const int64_t all0 = running(lane < kWaves ? s_wave[0][lane] : 0), all1 = running(lane < kWaves ? s_wave[1][lane] : 0);
            const int w = __builtin_amdgcn_readfirstlane(wave);
            if (w) {
                before0 += of_lane(all0, w - 1);
                before1 += of_lane(all1, w - 1);
            }
            tokens += of_lane(all0, kWaves - 1);
            taken += of_lane(all1, kWaves - 1);
        } else {
            tokens += of_lane(sum0, 63);
            taken += of_lane(sum1, 63);
        }
        if (b < B) {
            const int32_t at = saturate(before0 + sum0 - n);
            s_token[b] = at;
            s_taken[b] = saturate(before1 + sum1 - blocks);
            if constexpr (KEPT) {
                s_past[b] = (int32_t)p;
                s_new[b] = (int32_t)n;
            }
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

    auto past_of = [&](int b) -> int64_t { if constexpr (KEPT) return s_past[b]; else return max(past[b], 0); };
    auto new_of = [&](int b) -> int64_t { if constexpr (KEPT) return s_new[b]; else return max(fresh[b], 0); };
    auto taken_block = [&](int b, int nth) -> int32_t {      // the nth block that request b takes
        const int64_t f = start + s_taken[b] + nth;
        return f >= 0 && f < n_free ? free_blocks[f] : -1;
    };
    const int64_t step = (int64_t)gridDim.x * THREADS, me = (int64_t)blockIdx.x * THREADS + tid, entries = (int64_t)B * W;
    // slots first: their chain of reads is the longer one
    for (int64_t t = me; t < T; t += step) {
        int32_t where = -1;
        if (t < total) {
            int lo = 0, hi = B;                              // the last request that starts at or before t
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_token[mid] <= t) lo = mid;
                else hi = mid;
            }
            const int64_t p0 = past_of(lo), p = p0 + (t - s_token[lo]);
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
    for (int64_t e = me; e < entries; e += step) {
        const int b = (int)(((uint64_t)(uint32_t)e * w_mul) >> w_shift), j = (int)e - b * W;
        const int64_t p = past_of(b);
        const int have = pages(p);
        if (j >= have) table[e] = j < pages(p + new_of(b)) ? taken_block(b, j - have) : -1;
    }
}

// ---------------------------------------------------------------- quantise and append

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

// A wavefront's window of 64 slots: which of the first `slab` tokens begin a run (a run: tokens whose slots follow one another inside one block).
struct Window { int32_t got; bool valid; uint64_t leaders; };

__device__ __forceinline__ Window window(const int32_t *__restrict__ slot, int32_t slots, int T, int64_t t_first, int slab, int bs)
{
    const int lane = threadIdx.x & 63;
    Window w;
    w.got = slot[min(t_first + lane, (int64_t)T - 1)];
    const int32_t before = slot[max(t_first - 1, (int64_t)0)];
    w.valid = t_first + lane < T && w.got >= 0 && w.got < slots;
    int32_t prev = __shfl_up(w.got, 1, 64);
    if (lane == 0) prev = t_first > 0 ? before : -2;
    const bool follows = prev >= 0 && prev < slots && w.got == prev + 1 && (w.got & (bs - 1)) != 0;
    w.leaders = __ballot(w.valid && !follows && lane < slab);
    return w;
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

// Few tokens: one wavefront for a head (of K or of V) and a token; where a run begins with that token it writes the run, whole.
template <int D>
__global__ __launch_bounds__(256)
void kv8_append_kernel(Side k, Side v, int T, int Hkv, const int32_t *__restrict__ slot, int32_t slots, int shift)
{
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = item / (2 * Hkv);
    const int which = (int)(item - t * (2 * Hkv)), h = which % Hkv;
    if (t >= T) return;
    const Window w = window(slot, slots, T, t, 1, 1 << shift);
    if (!w.leaders) return;
    Run<D, 64> run;
    run.end(run.begin(which < Hkv ? k : v, h, Hkv, __builtin_amdgcn_readlane(w.got, 0), run_length(slot, T, w, t, 0, 1 << shift), t, shift),
            threadIdx.x & 63, 64);
}

// Many tokens: a workgroup of four wavefronts for a head and `slab` tokens writes the runs that begin among them, each whole, also past the slab's end.  Up to three
// runs are written by all four, ROWS rows each; more of them, and runs of ROWS at most, one by each in turn.  A lone wavefront's code for 64 rows is 9 KB that it goes through once, at the
// pace of the instructions' way from the L2: 9 us for a chunk of 512 tokens of 8 heads where four together take 4.1, and 30 for 5120 tokens in blocks of 128 where they take
// 9.6.  Bound by memory where there is much to write: 10240 tokens of 32 heads of 128 (252 MB) 43.4 us, 5.8 TB/s; without the hint on the loads 52.
template <int D, int ROWS>
__global__ __launch_bounds__(256)
void kv8_append_many_kernel(Side k, Side v, int T, int Hkv, const int32_t *__restrict__ slot, int32_t slots, int shift, int slab)
{
    __shared__ uint32_t s_top[2][4];
    const int64_t group = blockIdx.x / (2 * Hkv), t_first = group * slab;
    const int which = (int)(blockIdx.x - group * (2 * Hkv)), h = which % Hkv, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Side side = which < Hkv ? k : v;
    const Window w = window(slot, slots, T, t_first, slab, 1 << shift);        // (the same in all four)
    const bool alone = __builtin_popcountll(w.leaders) > 3 || 1 << shift <= ROWS;
    int turn = 0;                                                            // of the runs; nobody writes maxima before all have read the last but one's
    for (uint64_t leaders = w.leaders; leaders; leaders &= leaders - 1, ++turn) {
        if (alone && (turn & 3) != wave) continue;
        const int l0 = __builtin_ctzll(leaders), len = run_length(slot, T, w, t_first, l0, 1 << shift);
        const int row0 = alone ? 0 : wave * ROWS, rows = alone ? len : min(max(len - row0, 0), ROWS);
        Run<D, ROWS> run;
        uint32_t top = run.begin(side, h, Hkv, __builtin_amdgcn_readlane(w.got, l0), rows, t_first + l0, shift, row0);
        if (!alone) {
            uint32_t *tops = s_top[turn & 1];
            if ((threadIdx.x & 63) == 0) tops[wave] = top;
            __syncthreads();
            top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
        }
        run.end(top, alone ? threadIdx.x & 63 : threadIdx.x, alone ? 64 : 256);
    }
}

}  // namespace

namespace atom_internal {

hipError_t launch_kv_block_map(const int32_t *past, const int32_t *fresh, int B, int block_tokens, const int32_t *free_blocks,
                               int64_t n_free, const int32_t *cursor, int32_t *table, int64_t W, int64_t T,
                               int32_t *token_start, int32_t *seq_len, int32_t *slot, int32_t *cursor_out, hipStream_t stream)
{
    const bool   kept = B <= kMapKept;
    const size_t lds = (size_t)((kept ? 4 : 2) * B + 1) * sizeof(int32_t);
    const int    log = W > 1 ? 64 - __builtin_clzll((uint64_t)(W - 1)) : 0;
    const uint32_t w_mul = W > 0 ? (uint32_t)(((uint64_t)1 << (31 + log)) / (uint64_t)W + 1) : 0;       // n / W = n * w_mul >> 31 + log below 2^31
    // Entries and tokens one to a thread as long as the card has room for the workgroups at once.  A lone wavefront needs no barrier for
    // the scan: up to 64 requests and little to write.
    const int64_t work = (int64_t)B * W + T;
#define ATOM_MAP(THREADS, KEPT)                                                                                                      \
    do {                                                                                                                             \
        auto kern = &kv_block_map_kernel<THREADS, KEPT>;                                                                             \
        static atom_launch::LdsOptIn opt;                                                                                            \
        if (lds > 60 * 1024) {                                                                                                       \
            hipError_t err = atom_launch::ensure_dynamic_lds(opt, reinterpret_cast<const void *>(kern), lds);                        \
            if (err != hipSuccess) return err;                                                                                       \
        }                                                                                                                            \
        int64_t grid = (work + THREADS - 1) / THREADS;                                                                               \
        if (grid > 512) grid = 512;                                                                                                  \
        if (grid < 1) grid = 1;                                                                                                      \
        hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(THREADS), lds, stream, past, fresh, B, __builtin_ctz((unsigned)block_tokens), \
                           free_blocks, n_free, cursor, table, (int)W, w_mul, 31 + log, (int)T, token_start, seq_len, slot, cursor_out); \
    } while (0)
    if (!kept)                             ATOM_MAP(1024, false);
    else if (B > 256 || work > 64 * 1024)  ATOM_MAP(1024, true);
    else if (B > 64 || work > 1024)        ATOM_MAP(256, true);
    else                                   ATOM_MAP(64, true);
#undef ATOM_MAP
    return hipGetLastError();
}

constexpr int64_t kManyTokens = 256;

// How a call runs: tokens to a workgroup and head (0: a wavefront for each of them), and workgroups.
struct AppendShape { int slab; int64_t groups; };

static AppendShape append_shape(int64_t T, int Hkv, int block_tokens)
{
    const int64_t heads = 2 * (int64_t)Hkv;
    // Blocks of 64 tokens and more have long runs, which want four wavefronts; short ones a lone wavefront writes as fast, so the many of a workgroup start later there
    // (16 cache heads of 64, blocks of 16, 331 tokens 4.4 us, 5.5 the other way; 8 of 128, blocks of 64, a chunk of 512 9.0 and 4.3).
    const bool long_runs = block_tokens >= 64;
    if (long_runs ? T < kManyTokens : T * heads <= 16384) return {0, (T * heads + 3) / 4};
    // 8 tokens to a workgroup, and 64 from as many on as fill the card so (a workgroup that finds no run's beginning costs more than several runs in one).  Single tokens
    // pay for it, 16 to a wavefront: 32 cache heads of 128, blocks of 64, 256 of them 8.3 us, 257 18.3; 8 heads, blocks of 16, 1024 10.8, 1025 18.0.
    const int slab = T * heads <= 16384 ? 8 : 64;
    return {slab, (T + slab - 1) / slab * heads};
}

bool kv8_append_fits(int64_t T, int Hkv, int block_tokens) { return append_shape(T, Hkv, block_tokens).groups <= atom_launch::kMostThreads / 256; }

hipError_t launch_kv8_append(const void *k, const void *v, int64_t T, int64_t ldk, int64_t ldv, int Hkv, int D,
                             const int32_t *slot, int64_t n_blocks, int block_tokens, void *k_codes, float *k_scale,
                             void *v_codes, float *v_scale, hipStream_t stream)
{
    const Side ks = {(const __half *)k, ldk, (int8_t *)k_codes, k_scale}, vs = {(const __half *)v, ldv, (int8_t *)v_codes, v_scale};
    const int32_t slots = (int32_t)(n_blocks * block_tokens);
    const int     shift = __builtin_ctz((unsigned)block_tokens);
    const AppendShape s = append_shape(T, Hkv, block_tokens);
    if (!s.slab) {
        hipLaunchKernelGGL((D == 128 ? &kv8_append_kernel<128> : &kv8_append_kernel<64>), dim3((unsigned)s.groups), dim3(256), 0, stream, ks, vs, (int)T, Hkv, slot, slots, shift);
        return hipGetLastError();
    }
    auto kern = block_tokens == 128 || block_tokens == 32 ? (D == 128 ? &kv8_append_many_kernel<128, 32> : &kv8_append_many_kernel<64, 32>)
                                     : (D == 128 ? &kv8_append_many_kernel<128, 16> : &kv8_append_many_kernel<64, 16>);
    hipLaunchKernelGGL(kern, dim3((unsigned)s.groups), dim3(256), 0, stream, ks, vs, (int)T, Hkv, slot, slots, shift, s.slab);
    return hipGetLastError();
}

}  // namespace atom_internal
