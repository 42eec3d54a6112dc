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
#include "atom_kv8_append.h"
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

using namespace atom_kv8;

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
