// Attention over the paged 8-bit KV cache for gfx950 (Section 4.4 of the paper: the cache is loaded in its low
// precision and dequantised inside the attention operator, whose arithmetic stays in floating point; Section 4.5);
// atom_kv8.hip fills the cache and has its layout.

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include "atom_internal.h"
#include "atom_launch.h"

namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef unsigned u2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e   = 1.4426950408889634f;
constexpr float kNoScore = -1e30f;                // the running bound M before the first key: below every score, and finite
// Weights are 2^(e - M) up to 2^kLargest, inside fp16's range (M: so far below the largest e when it is set).  A row's M moves when its e have grown by 2^8 (few
// rows) or a sum of eight weights by 2^10 (many rows) since.
constexpr float kLargest = 15.0f, kMostSum = 32768.0f, kRaisedFew = 7.0f, kRaisedMany = 5.0f;
constexpr int   kAllKeys = 0x40000000;            // as many as a request has at most, and a multiple of 128
// A block's factor and value scale as the kernels take them lie between these: never zero and never infinite, so that a masked score of minus infinity
// stays one whatever the block holds, and a block of zeros has a weight to be divided out again.
constexpr float kLeastFactor = 1e-37f, kLeastValue = 2.3283064365386963e-10f, kMost = 1e35f;
// A block whose scale is not finite gives NaN to the rows that see it: their sum is made NaN at the end, by the first key of such a block (0x7fffffff: none), so
// that masked rows of the same tile keep finite numbers all the way and the loops carry nothing for it.
constexpr int kNoKey = 0x7fffffff;

// The first lane's `key` (they ascend) whose block exists (unit) and has a scale that is not finite.
__device__ __forceinline__ int first_spoiled(int key, int unit, float k_scale, float v_scale)
{
    const uint64_t bad = __ballot(unit >= 0 && !(__builtin_isfinite(k_scale) && __builtin_isfinite(v_scale)));
    return bad ? __builtin_amdgcn_readlane(key, __builtin_ctzll(bad)) : kNoKey;
}
// What a row's accumulators are multiplied by (values were 2^-9 of the codes): 0 for a row that sees no key, NaN for a NaN sum.
__device__ __forceinline__ float quotient(float sum) { return sum == 0.0f ? 0.0f : 512.0f / sum; }

// What all kernels of a call are told.
struct Args {
    const __half *q; int T; int64_t ldq;
    int B, Hkv, group;                            // group = H / Hkv query heads to a cache head
    uint32_t div_mul; int div_shift;              // n / group = n * div_mul >> div_shift for n below 2^31
    int max_new;
    const int32_t *token_start, *seq_len, *table;
    int W, shift;                                 // table columns; block_tokens = 1 << shift
    int64_t capacity;                             // W * block_tokens
    int32_t n_blocks;
    const int8_t *kq; const float *ks; const int8_t *vq; const float *vs;
    float sm_scale;
    __half *out; int64_t ldo;
};

// One of the two kinds of work of a call, by the rows (tokens times heads of a group) of a request.
struct Job {
    int rows_min, rows_max;
    int log;                                      // a tile has 1 << log query rows
    int budget;                                   // workgroups for each cache head that tiles may be cut into (0: none is cut)
    float *part; int part_rows;                   // records of the pieces, and rows of a record
    int groups, merges;                           // workgroups for each cache head of the kernel, of the merge
};

__device__ __forceinline__ int by_group(const Args &a, int n) { return (int)(((uint64_t)(uint32_t)n * a.div_mul) >> a.div_shift); }

// A request's share of the call.
struct Request {
    int start, n;                                 // its first token, its tokens that are computed
    int before;                                   // position of its first token (may be negative: such a row sees nothing)
    int keys;                                     // keys that exist for it
};

__device__ __forceinline__ Request request(const Args &a, int b)
{
    Request r;
    const int first = a.token_start[b], end = a.token_start[b + 1], len = a.seq_len[b];
    r.start = min(max(first, 0), a.T);
    const int e = min(max(end, r.start), a.T);
    r.n = min(e - r.start, a.max_new);
    const int64_t before = (int64_t)len - max((int64_t)end - first, (int64_t)0);
    r.before = (int)min(max(before, (int64_t)-0x40000000), (int64_t)0x3fffffff);        // (there are at most 2^30 keys)
    r.keys = (int)min((int64_t)max(len, 0), a.capacity);
    return r;
}

// ---- which part of the work a workgroup has
//
// The query rows of a request and cache head (token after token, the group's heads of each) come in tiles of 1 << job.log rows.  Where the tiles are
// fewer than the workgroups that a call is to have for each cache head (budget), their keys are cut into pieces of about one size in the whole call:
// sequences of any lengths keep the card evenly busy, and the pieces of a tile meet in the merge kernel.  Every wavefront
// finds its place from the lengths by itself, 64 requests at a time: for as many it is one read, which it needs anyway.
struct Place { int b, tile, split, splits, keys_per, first_slot; Request r; bool found; };

// Sum over the lanes up to this one, on the vector unit (lane exchanges through LDS cost a microsecond in front of the first load).
template <class V>
__device__ __forceinline__ V running(V v)
{
#define ATOM_STEP(ctrl, rows) \
    v += __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), ctrl, rows, 0xF, false))
    ATOM_STEP(0x111, 0xF);                        // one, two, four, eight lanes below in the row of 16
    ATOM_STEP(0x112, 0xF);
    ATOM_STEP(0x114, 0xF);
    ATOM_STEP(0x118, 0xF);
    ATOM_STEP(0x142, 0xA);                        // the row below's last lane, into rows 1 and 3
    ATOM_STEP(0x143, 0xC);                        // the lower half's, into the upper
#undef ATOM_STEP
    return v;
}
__device__ __forceinline__ int total(int v) { return __builtin_amdgcn_readlane(running(v), 63); }
__device__ __forceinline__ float total(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, running(v)), 63));
}

// FROM_TILE: `index` counts tiles (all of a tile's pieces are meant), else pieces.
template <bool FROM_TILE>
__device__ __forceinline__ Place place(const Args &a, const Job &job, int index)
{
    const int budget = job.budget;
    const int lane = threadIdx.x & 63;
    Request r = {0, 0, 0, 0};
    auto tiles_keys = [&](int base, int &tiles, int &keys) {
        tiles = 0;
        keys = 0;
        if (base + lane < a.B) {
            r = request(a, base + lane);
            const int64_t rows = (int64_t)r.n * a.group;
            if (rows >= job.rows_min && rows <= job.rows_max) {
                tiles = (int)((rows + (1 << job.log) - 1) >> job.log);
                keys = r.keys;
            }
        }
    };
    Place p;
    p.found = false;
    int tiles, keys;
    tiles_keys(0, tiles, keys);
    int per = kAllKeys;                           // keys of a piece at most, a multiple of 128: one step of 32 for each of four wavefronts
    if (budget) {                                 // (with more than 64 requests r is read again below)
        // sum over tiles of ceil(keys / per) is below tiles + all / per
        int64_t mine = (int64_t)tiles * keys;
        int     count = tiles;
        for (int base = 64; base < a.B; base += 64) {
            int t2, k2;
            tiles_keys(base, t2, k2);
            mine += (int64_t)t2 * k2;
            count += t2;
        }
        count = total(count);
        if (count < budget) {
            const float all = total((float)mine) * 1.00001f;          // (64 values: rounded by less than that)
            auto share = [&](float pieces) {
                const float want = ceilf(all / (128.0f * pieces));
                return want < 1.0f ? 128 : want < 8388607.0f ? 128 * (int)want : kAllKeys;
            };
            per = share((float)(budget - count));
            if (a.B <= 64) {                      // mostly it is half a piece a tile less
                const int tight = share((float)budget - 0.5f * (float)count);
                if (total(tiles * (keys > tight ? (keys + tight - 1) / tight : 1)) <= budget) per = tight;
            }
        }
    }
    int count = 0, slots = 0;                     // tiles and pieces of the requests before
    for (int base = 0; base < a.B; base += 64) {
        if (base || (budget && a.B > 64)) tiles_keys(base, tiles, keys);
        const int splits = keys > per ? (keys + per - 1) / per : 1;
        const int ct = running(tiles), cs = running(tiles * splits);
        const int mine = FROM_TILE ? count + ct : slots + cs;
        const uint64_t past = __ballot(index < mine);
        if (past) {
            const int l = __builtin_ctzll(past);
            p.found = true;
            p.b = base + l;
            p.r = Request{__builtin_amdgcn_readlane(r.start, l), __builtin_amdgcn_readlane(r.n, l), __builtin_amdgcn_readlane(r.before, l),
                          __builtin_amdgcn_readlane(r.keys, l)};
            p.splits = __builtin_amdgcn_readlane(splits, l);
            const int t0 = count + __builtin_amdgcn_readlane(ct - tiles, l);
            const int s0 = slots + __builtin_amdgcn_readlane(cs - tiles * splits, l);
            if (FROM_TILE) {
                p.tile = index - t0;
                p.split = 0;
            } else {
                p.tile = (index - s0) / p.splits;
                p.split = (index - s0) - p.tile * p.splits;
            }
            const int all = __builtin_amdgcn_readlane(keys, l);
            p.keys_per = p.splits == 1 ? kAllKeys : ((all + p.splits - 1) / p.splits + 127) & ~127;      // even pieces
            p.first_slot = s0 + p.tile * p.splits;
            return p;
        }
        count += __builtin_amdgcn_readlane(ct, 63);
        slots += __builtin_amdgcn_readlane(cs, 63);
    }
    return p;
}

// ---- codes to fp16
//
// A code with its sign bit flipped is u = code + 128.  As the low byte of a half it is the subnormal number u * 2^-24 exactly, which the
// matrix instructions take: a byte selection makes two of them.
__device__ __forceinline__ uint32_t flip(uint32_t w) { return w ^ 0x80808080u; }

// bytes i of lo and of hi as one pair of subnormal halves
template <int i>
__device__ __forceinline__ uint32_t pair_of(uint32_t lo, uint32_t hi)
{
    return __builtin_amdgcn_perm(hi, lo, 0x0c000c00u | ((4u + i) << 16) | i);
}

// u * 2^-24 to (u - 128) * 2^-9, exactly: the values' side keeps no offset that a long sum would have to carry.
__device__ __forceinline__ uint32_t centred(uint32_t pair)
{
    const h2 v = __builtin_elementwise_fma(__builtin_bit_cast(h2, pair), h2{(_Float16)32768.0f, (_Float16)32768.0f},
                                           h2{(_Float16)-0.25f, (_Float16)-0.25f});
    return __builtin_bit_cast(uint32_t, v);
}

// v + the sum of eight halves
__device__ __forceinline__ float add8(const h8 &x, float v)
{
    const u4 w = __builtin_bit_cast(u4, x);
    const h2 one = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) v = __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, (uint32_t)w[i]), one, v, false);
    return v;
}

__device__ __forceinline__ h8 halves(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_bit_cast(h8, u4{a, b, c, d});
}

// Part of a row of codes.  ONCE: with the hint that nothing reads it again.
template <bool ONCE, class V>
__device__ __forceinline__ V load(const int8_t *p)
{
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const V *>(p));
    else return *reinterpret_cast<const V *>(p);
}

// Two loads of eight rows of 128 codes, 16 a lane: lanes 0 .. 7 of each 16 have the first half of the dimensions of row l (of a) and of row 8 + l (of b), lanes
// 8 .. 15 the second half of rows l - 8 and l.  Afterwards a is the first half and b the second half of row l in every lane.
__device__ __forceinline__ void ordered(u4 &a, u4 &b)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int x = a[i], y = b[i];
        a[i] = __builtin_amdgcn_update_dpp(x, y, 0x128, 0xF, 0xC, false);      // lanes 8 .. 15: b of the lane eight below
        b[i] = __builtin_amdgcn_update_dpp(y, x, 0x128, 0xF, 0x3, false);      // lanes 0 .. 7: a of the lane eight above
    }
}

// max over the lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float max_of_chunks(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float sum_of_chunks(float v)
{
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

// ---------------------------------------------------------------- few query rows
//
// One workgroup of four wavefronts (8 or 16 where a lone one has a whole context) for a tile of 16 or 32 query rows of a (request, cache head) and a piece of its keys;
// the wavefronts take steps of 32 keys in turn, each with a softmax of its own, and meet in LDS.  Bound by memory where there is enough of it: 64 single tokens over
// up to 2048 keys of 32 heads of 128 (673 MB) 113 us, 5.95 TB/s; 16 over up to 16000 keys of 8 cache heads, 8 heads to each (329 MB), 57.6 us, 5.7 TB/s, and the merge 4.8.
// With little to read by the chain of lengths, block numbers, scales and codes: one token over 1000 keys of 32 heads 6.9 us.
//
//   scores: S^T = K Q^T on 16x16x32 fp16 matrix instructions.  Keys are the rows, so that a lane holds four keys of ONE query row.  Lane (l & 15, c =
//           l >> 4) has the 16 dimensions from 16 c on of every 64 of key l & 15; the order of the dimensions within a product is free as long as Q has the
//           same.  A load of 1 KB takes eight whole rows of 128 dimensions (half rows of 16 keys: 6.1 TB/s became 5.6), and lanes eight apart then trade halves.  The offset of u = code + 128 leaves through the accumulator's start, -128 sum(q) 2^-24.
//   softmax: e = score * log2(e) * sm_scale * k_scale + log2(v_scale), p = 2^(e - M) with M seven below the largest e so far: the block's value scale sits in the
//           weight, so the matrix instruction adds codes of blocks of different scales, and the weights are in one range where
//           they count, whatever the scales are.  The sum of the softmax takes p / v_scale.  M moves only where some e passes it by 15 (p <= 2^15 then).
//   values: O^T = V^T P^T.  The weights lie in the registers of the scores as the second operand wants them when its order of keys is
//           that of the scores' rows; V's rows are loaded in that order, D / 16 bytes a lane, and the byte selection that makes halves also
//           transposes.  No LDS in the loop, and no lane exchange but ordered()'s.  The weights travel as fp16 (fp32 products run at a sixteenth of the rate): rounded to nearest
//           even, by 2^-11 of themselves, or by 2^-25 below 2^-14.  The largest one is 2^7 at least, so that is 2^-32 of it (2^-30 with
//           many rows): with the largest at one, a context of small weights beside it (a first key that all attend to, 65536 others of 2^-22.7) was 20 % off.
//   loads: the next step's rows of K are asked for once the scores have used this step's, those of V after the values: half the registers of two
//           buffers.  Block numbers and scales of 64 blocks of 16 keys are read at once, a lane each.
//   rows:  SETS = 2: tiles of 32 rows, the codes turned into halves once for two sets of 16.
constexpr int kStep = 32, kRowsLog = 4, kSetRows = 1 << kRowsLog;

template <int D, int kWaves, int SETS>
struct RowsLds { float acc[kWaves][SETS * kSetRows][D + 4], m[kWaves][SETS * kSetRows], l[kWaves][SETS * kSetRows]; };

template <int D, bool ONCE, int kWaves, int SETS>
__device__ __forceinline__ void rows_tile(const Args &a, const Job &job, int index, RowsLds<D, kWaves, SETS> &lds)
{
    constexpr int KB = D / 4, VB = D / 16;            // bytes of a K row and of a V row in a lane
    constexpr int KS = D / 32;                        // matrix instructions for 16 keys' scores
    constexpr int kTileRows = SETS * kSetRows;
    auto &s_acc = lds.acc;
    auto &s_m = lds.m, &s_l = lds.l;

    const int h = index % a.Hkv;
    const Place w = place<false>(a, job, index / a.Hkv);
    if (!w.found) return;
    const Request r = w.r;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m = lane & 15, c = lane >> 4;           // query row (or key) of the set, chunk
    const int rows = min(kTileRows, r.n * a.group - w.tile * kTileRows);
    // keys that this lane's rows see, and the fewest and the most of the tile
    int token[SETS], head[SETS], sees[SETS];
#pragma unroll
    for (int t = 0; t < SETS; ++t) {
        const int row = w.tile * kTileRows + min(t * kSetRows + m, rows - 1);
        token[t] = by_group(a, row);
        head[t] = h * a.group + row - token[t] * a.group;
        sees[t] = min(max(r.before + token[t] + 1, 0), r.keys);
    }
    const int sees_least = min(max(r.before + by_group(a, w.tile * kTileRows) + 1, 0), r.keys);
    const int sees_most = min(max(r.before + by_group(a, w.tile * kTileRows + rows - 1) + 1, 0), r.keys);
    const int key0 = w.split * w.keys_per, key1 = min(sees_most, key0 + w.keys_per);     // (a split below 2^31: keys_per is at most keys)

    h8 q[SETS][KS];
    const float to_e = a.sm_scale * kLog2e * 16777216.0f;

    f4 acc[SETS][VB];
    float M[SETS], l[SETS], start[SETS];              // start: what u = code + 128 adds to a score, negated
#pragma unroll
    for (int t = 0; t < SETS; ++t) {
        M[t] = kNoScore;
        l[t] = start[t] = 0.0f;
#pragma unroll
        for (int e = 0; e < VB; ++e) acc[t][e] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    u4 kr[2][KB / 16];
    uint32_t vr[8][VB / 4];
    // lane i: block of 16 keys number i of this wavefront's (two to a step)
    int   unit = -1, spoiled = kNoKey;
    float b_scale = 0.0f, b_log = 0.0f, b_inv = 0.0f;
    const int32_t *table = a.table + (int64_t)w.b * a.W;
    auto key_of = [&](int step) { return key0 + (step * kWaves + wave) * kStep; };
    auto block_key = [&](int step) { return key_of(step + (lane >> 1)) + 16 * (lane & 1); };
    auto page_of = [&](int step) { const int key = block_key(step); return key < key1 ? table[key >> a.shift] : -1; };
    auto look_up = [&](int step, int page) {          // the blocks of 32 steps from `step` on; their scales are on the way
        const int  key = block_key(step);
        const bool there = page >= 0 && page < a.n_blocks;
        const int64_t at = there ? (int64_t)page * a.Hkv + h : 0;
        unit = there ? (int)(at << (a.shift - 4)) + ((key & ((1 << a.shift) - 1)) >> 4) : -1;
        b_scale = a.ks[at];
        b_log = a.vs[at];
    };
    auto take_scales = [&](int step) {                // (no such keys: e is minus infinity)
        spoiled = min(spoiled, first_spoiled(block_key(step), unit, b_scale, b_log));
        const float v = fminf(fmaxf(b_log, kLeastValue), kMost);
        b_scale = unit < 0 ? 1.0f : fminf(fmaxf(b_scale * to_e, kLeastFactor), kMost);
        b_log = unit < 0 ? -INFINITY : __builtin_amdgcn_logf(v);
        b_inv = unit < 0 ? 0.0f : __builtin_amdgcn_rcpf(v);
    };
    // (blocks past the end or without a page: the cache's first rows, masked)
    auto block_at = [&](int step, int u) { return (int64_t)max(__builtin_amdgcn_readlane(unit, 2 * (step & 31) + u), 0) * (16 * D); };
    auto fetch_k = [&](int step) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int8_t *kp = a.kq + block_at(step, u) + (uint32_t)(D == 128 ? (m & 7) * D + 16 * (c + 4 * (m >> 3)) : m * D + 16 * c);
#pragma unroll
            for (int i = 0; i < KB / 16; ++i) kr[u][i] = load<ONCE, u4>(kp + 1024 * i);
        }
    };
    auto fetch_v = [&](int step) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int8_t *vp = a.vq + block_at(step, u) + (uint32_t)(4 * c * D + m * VB);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (VB == 8) {
                    const u2 v = load<ONCE, u2>(vp + i * D);
                    vr[4 * u + i][0] = v[0];
                    vr[4 * u + i][1] = v[1];
                } else {
                    vr[4 * u + i][0] = load<ONCE, uint32_t>(vp + i * D);
                }
            }
        }
    };
    // the blocks of the next step: of this look-up, or (`turn`) still to be looked up
    auto compute = [&](int step, bool more) __attribute__((always_inline)) {
        const int at = 2 * (step & 31), key = key_of(step);
        const bool turn = ((step + 1) & 31) == 0;
        float e[SETS][8], top[SETS], inv_v[2];
#pragma unroll
        for (int t = 0; t < SETS; ++t) top[t] = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if constexpr (D == 128) ordered(kr[u][0], kr[u][1]);
            f4 s[SETS];
#pragma unroll
            for (int t = 0; t < SETS; ++t) s[t] = f4{start[t], start[t], start[t], start[t]};
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const uint32_t w0 = flip(kr[u][i >> 1][(2 * i) & 3]), w1 = flip(kr[u][i >> 1][(2 * i + 1) & 3]);
                const h8 k = halves(__builtin_amdgcn_perm(0, w0, 0x0c010c00u), __builtin_amdgcn_perm(0, w0, 0x0c030c02u),
                                    __builtin_amdgcn_perm(0, w1, 0x0c010c00u), __builtin_amdgcn_perm(0, w1, 0x0c030c02u));
#pragma unroll
                for (int t = 0; t < SETS; ++t) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[t][i], s[t], 0, 0, 0);
            }
            if (key + 16 * u + 16 > min(sees_least, key1)) {
#pragma unroll
                for (int t = 0; t < SETS; ++t) {
                    const int room = min(sees[t], key1) - (key + 16 * u + 4 * c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[t][i] = i < room ? s[t][i] : -INFINITY;
                }
            }
            const float f = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, b_scale), at + u));
            const float log_v = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, b_log), at + u));
            inv_v[u] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, b_inv), at + u));
#pragma unroll
            for (int t = 0; t < SETS; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e[t][4 * u + i] = fmaf(s[t][i], f, log_v);
                    top[t] = fmaxf(top[t], e[t][4 * u + i]);
                }
        }
        if (more && !turn) fetch_k(step + 1);
        h8 p[SETS];
#pragma unroll
        for (int t = 0; t < SETS; ++t) {
            if (__ballot(top[t] > M[t] + kLargest)) { // rare after the first steps
                const float to = fmaxf(M[t], max_of_chunks(top[t]) - kRaisedFew);
                const float down = __builtin_amdgcn_exp2f(M[t] - to);
                M[t] = to;
                l[t] *= down;
#pragma unroll
                for (int i = 0; i < VB; ++i) acc[t][i] *= down;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e[t][4 * u + i] = __builtin_amdgcn_exp2f(e[t][4 * u + i] - M[t]);
                    sum += e[t][4 * u + i];
                }
                l[t] = fmaf(sum, inv_v[u], l[t]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) p[t][i] = (_Float16)e[t][i];
        }
        __builtin_amdgcn_sched_barrier(0);            // (or registers for all of it at once)
#define ATOM_VALUES(j, n)                                                                                                    \
        {                                                                                                                    \
            const h8 v = halves(centred(pair_of<n>(vr[0][j], vr[1][j])), centred(pair_of<n>(vr[2][j], vr[3][j])),            \
                                centred(pair_of<n>(vr[4][j], vr[5][j])), centred(pair_of<n>(vr[6][j], vr[7][j])));           \
            _Pragma("unroll") for (int t = 0; t < SETS; ++t)                                                                 \
                acc[t][4 * (j) + (n)] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[t], acc[t][4 * (j) + (n)], 0, 0, 0);     \
        }
#pragma unroll
        for (int j = 0; j < VB / 4; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) vr[i][j] = flip(vr[i][j]);
            ATOM_VALUES(j, 0)
            ATOM_VALUES(j, 1)
            ATOM_VALUES(j, 2)
            ATOM_VALUES(j, 3)
        }
#undef ATOM_VALUES
    };

    if (key_of(0) < key1) {                           // (the same in all lanes)
        const int steps = (key1 - key_of(0) + kWaves * kStep - 1) / (kWaves * kStep);
        const int page = page_of(0);
#pragma unroll
        for (int t = 0; t < SETS; ++t) {
            const __half *qp = a.q + (int64_t)(r.start + token[t]) * a.ldq + (int64_t)head[t] * D + 16 * c;
#pragma unroll
            for (int s = 0; s < KS; ++s) q[t][s] = __builtin_bit_cast(h8, *reinterpret_cast<const u4 *>(qp + 64 * (s >> 1) + 8 * (s & 1)));
        }
        look_up(0, page);
        fetch_k(0);
        fetch_v(0);
        take_scales(0);
#pragma unroll
        for (int t = 0; t < SETS; ++t) {
#pragma unroll
            for (int s = 0; s < KS; ++s) start[t] = add8(q[t][s], start[t]);
            start[t] = sum_of_chunks(start[t]) * (-128.0f * 5.9604644775390625e-08f);
        }
        for (int step = 0; step < steps; ++step) {
            const bool more = step + 1 < steps;
            compute(step, more);
            if (more) {
                if (((step + 1) & 31) == 0) {
                    look_up(step + 1, page_of(step + 1));
                    fetch_k(step + 1);
                }
                fetch_v(step + 1);
                if (((step + 1) & 31) == 0) take_scales(step + 1);
            }
        }
    }

    // ---- the wavefronts meet
#pragma unroll
    for (int t = 0; t < SETS; ++t) {
        l[t] = sees[t] > spoiled ? NAN : sum_of_chunks(l[t]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < VB; ++e) s_acc[wave][t * kSetRows + m][VB * (4 * c + i) + e] = acc[t][e][i];
        if (c == 0) {
            s_m[wave][t * kSetRows + m] = M[t];
            s_l[wave][t * kSetRows + m] = l[t];
        }
    }
    __syncthreads();
    const bool whole = w.splits == 1;
    const int64_t record = whole ? 0 : ((int64_t)(w.first_slot + w.split) * a.Hkv + h) * job.part_rows;
    for (int i = tid; i < rows * (D / 4); i += kWaves * 64) {
        const int rr = i / (D / 4), d = 4 * (i % (D / 4));
        float top = s_m[0][rr];
#pragma unroll
        for (int k = 1; k < kWaves; ++k) top = fmaxf(top, s_m[k][rr]);
        float sum = 0.0f;
        f4 o = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            const float f = __builtin_amdgcn_exp2f(s_m[k][rr] - top);
            sum = fmaf(s_l[k][rr], f, sum);
            const f4 v = *reinterpret_cast<const f4 *>(&s_acc[k][rr][d]);
            o += v * f;
        }
        if (whole) {
            const float f = quotient(sum);
            const int rw = w.tile * kTileRows + rr, t = by_group(a, rw);
            __half *to = a.out + (int64_t)(r.start + t) * a.ldo + (int64_t)(h * a.group + rw - t * a.group) * D + d;
            const __half2 lo = __floats2half2_rn(o[0] * f, o[1] * f), hi = __floats2half2_rn(o[2] * f, o[3] * f);
            *reinterpret_cast<u2 *>(to) = u2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
        } else {
            float *to = job.part + (record + rr) * (D + 4);
            *reinterpret_cast<f4 *>(to + 4 + d) = o;
            if (d == 0) {
                to[0] = top;
                to[1] = sum;
            }
        }
    }
}

// (two sets: two wavefronts a SIMD, by their registers)
template <int D, bool ONCE, int kWaves, int SETS>
__global__ __launch_bounds__(kWaves * 64, SETS == 2 ? 2 : 4)
void attention_kv8_rows_kernel(const Args a, const Job few)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    rows_tile<D, ONCE, kWaves, SETS>(a, few, blockIdx.x, *reinterpret_cast<RowsLds<D, kWaves, SETS> *>(lds));
}

// ---------------------------------------------------------------- many query rows
//
// One workgroup of four wavefronts for a tile of 128 query rows of a (request, cache head) and a piece of its keys; a wavefront has
// 32 rows, and all four read the same 64 keys from LDS.  The arithmetic is that of the kernel above on 32x32x16 matrix instructions: S^T = K Q^T, so that
// a lane has one query row and 16 of 32 keys, and O^T = V^T P^T with the weights where the scores were.
//
//   LDS:   the four wavefronts turn 64 rows of codes into halves once for all 128 query rows (each for itself it would be
//          four times the work: 256 vector instructions a tile).  K as [key][D]; V as [D][key], its keys in the order of the scores' rows, so that
//          an operand is one 16-byte read: byte selection makes the halves and transposes.  Rows are padded by 16 bytes, which spreads the reads (16 lanes,
//          16 rows) and V's writes (16 groups of keys of two dimensions) over all banks.
//   order of work: 32 keys at a time; the scores of the next 32 are multiplied while the vector unit makes weights of the last ones and halves of the next
//          tile's codes, so that the matrix unit and the vector unit of a lone wavefront work at the same time.  The tiles of K lie 32 keys behind those of V for that:
//          the scores of keys 32 .. 95 of a tile of V are multiplied with it.
//   loads: codes of the next tile but one are on their way, and their block numbers a tile earlier, while one is computed; two buffers, a barrier a tile.
//   order: the last tiles of a request, which see the most keys, first.
//
// Bound by the issue of both units: two prompts of up to 4096 tokens, 64 heads on 8 cache heads of 128 (292 GFLOP), 311 to 342 us by card, 854 to 940 TFLOP/s; of a SIMD's cycles the matrix
// unit has 46 % and the vector unit 61 %, which hold each other up (a matrix instruction keeps the vector unit from starting one for 13 to 16 cycles of its 32).

__device__ __forceinline__ float larger(float a, float b, float c)
{
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

constexpr int kTileLog = 7, kTile = 1 << kTileLog, kKeys = 64;

template <int D>
struct TileLds {
    static constexpr int kPitch = 2 * D + 16, vPitch = 2 * kKeys + 16;          // bytes
    static constexpr int k = 0, v = kKeys * kPitch, bytes = v + D * vPitch;     // of one buffer
};

template <int D>
__device__ __forceinline__ void many_rows_tile(const Args &a, const Job &job, int index, unsigned char *lds)
{
    typedef TileLds<D> L;
    constexpr int KS = D / 16, DB = D / 32;           // matrix instructions for 32 keys' scores; blocks of 32 output dimensions
    constexpr int KL = D / 64, VB = D / 16;           // 16-byte loads of K, bytes of a V row in a lane

    const int h = index % a.Hkv;
    const Place w = place<false>(a, job, index / a.Hkv);
    if (!w.found) return;
    const Request r = w.r;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int all = r.n * a.group;
    const int tile = ((all - 1) >> kTileLog) - w.tile;
    const int row0 = tile * kTile + wave * 32, rows = min(32, all - row0);      // of this wavefront; none: rows <= 0
    const int row = min(row0 + n, all - 1);
    const int token = by_group(a, row), head = h * a.group + row - token * a.group;
    auto keys_of = [&](int row_) { return min(max(r.before + by_group(a, min(row_, all - 1)) + 1, 0), r.keys); };
    const int sees = keys_of(row), key0 = w.split * w.keys_per;
    const int key1 = min(keys_of(tile * kTile + kTile - 1), key0 + w.keys_per);           // of the workgroup
    const int wave1 = rows > 0 ? min(keys_of(row0 + rows - 1), key1) : 0, least = min(keys_of(row0), key1);

    h8 q[KS];
    float start = 0.0f;                               // what u = code + 128 adds to a score, negated
    auto read_q = [&]() {
        const __half *qp = a.q + (int64_t)(r.start + token) * a.ldq + (int64_t)head * D + 8 * hh;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = __builtin_bit_cast(h8, *reinterpret_cast<const u4 *>(qp + 16 * s));
    };
    const float to_e = a.sm_scale * kLog2e * 16777216.0f;
    f16v o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;
    float M = kNoScore, l = 0.0f;

    // ---- blocks: lane i has the block of 16 keys number i of 16 tiles, its place and its scales; another register the blocks of K's tiles
    const int32_t *table = a.table + (int64_t)w.b * a.W;
    int   spoiled = kNoKey;
    int   page = -1, page_k = -1, unit = -1, unit_k = -1;      // block numbers of the table; rows / 16 in the whole cache, -1: no such keys
    float ks = 0.0f, vs = 0.0f, b_scale, b_log, b_inv;
    auto key_of = [&](int tile) { return key0 + tile * kKeys + 16 * lane; };
    auto exists = [&](int p) { return p >= 0 && p < a.n_blocks; };
    auto place_of = [&](int p, int key) {
        return exists(p) ? (int)(((int64_t)p * a.Hkv + h) << (a.shift - 4)) + ((key & ((1 << a.shift) - 1)) >> 4) : -1;
    };
    auto read_pages = [&](int tile) {
        const int key = key_of(tile);
        page = key < key1 ? table[key >> a.shift] : -1;
        page_k = key + 32 < key1 ? table[(key + 32) >> a.shift] : -1;
    };
    auto take_units = [&](int tile) {                 // a tile later: the scales are on their way
        const int key = key_of(tile);
        unit = place_of(page, key);
        unit_k = place_of(page_k, key + 32);
        const int64_t at = exists(page) ? (int64_t)page * a.Hkv + h : 0;
        ks = a.ks[at];
        vs = a.vs[at];
    };
    auto take_scales = [&](int tile) {
        spoiled = min(spoiled, first_spoiled(key_of(tile), unit, ks, vs));
        const float v = fminf(fmaxf(vs, kLeastValue), kMost);
        b_scale = unit < 0 ? 1.0f : fminf(fmaxf(ks * to_e, kLeastFactor), kMost);
        b_log = unit < 0 ? -INFINITY : __builtin_amdgcn_logf(v);
        b_inv = unit < 0 ? 0.0f : __builtin_amdgcn_rcpf(v);
    };
    // ---- loading: a thread has 16 (or 32) codes of one key of K, and D / 16 of four keys of V
    const int kt = tid >> 2, tq = lane & 15, vd = VB * (4 * wave + (lane >> 4));
    u4 kr[KL];
    uint32_t vr[4][VB / 4];
    auto fetch_k = [&](int unit_, int at, u4 (&to)[KL]) {       // (no such keys: the cache's first rows, masked)
        const int8_t *kp = a.kq + (int64_t)max(__builtin_amdgcn_readlane(unit_, at + wave), 0) * (16 * D) + (uint32_t)((kt & 15) * D + 16 * (tid & 3));
#pragma unroll
        for (int i = 0; i < KL; ++i) to[i] = *reinterpret_cast<const u4 *>(kp + 64 * i);
    };
    auto fetch_v = [&](int at) {
        const int8_t *vp = a.vq + (int64_t)max(__shfl(unit, at + (tq >> 2), 64), 0) * (16 * D) + (uint32_t)((4 * tq & 15) * D + vd);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (VB == 8) {
                const u2 v = *reinterpret_cast<const u2 *>(vp + i * D);
                vr[i][0] = v[0];
                vr[i][1] = v[1];
            } else {
                vr[i][0] = *reinterpret_cast<const uint32_t *>(vp + i * D);
            }
        }
    };
    constexpr int kPieces = 2 * KL, vPieces = VB;      // of a thread's staging
    auto stage_k = [&](unsigned char *buf, const u4 (&kr)[KL], int piece) __attribute__((always_inline)) {
        const uint32_t w0 = flip(kr[piece >> 1][2 * (piece & 1)]), w1 = flip(kr[piece >> 1][2 * (piece & 1) + 1]);
        *reinterpret_cast<u4 *>(buf + L::k + kt * L::kPitch + 32 * (tid & 3) + 128 * (piece >> 1) + 16 * (piece & 1)) =
            u4{__builtin_amdgcn_perm(0, w0, 0x0c010c00u), __builtin_amdgcn_perm(0, w0, 0x0c030c02u),
               __builtin_amdgcn_perm(0, w1, 0x0c010c00u), __builtin_amdgcn_perm(0, w1, 0x0c030c02u)};
    };
    auto stage_v = [&](unsigned char *buf, int piece) __attribute__((always_inline)) {
        // one dimension of keys 4 tq .. 4 tq + 3: step u = tq / 4 of 16 keys, half-wave tq & 1, its first or second four
        const int j = piece >> 2;
        const uint32_t sel = 0x0c040c00u + (piece & 3) * 0x00010001u;
        if ((piece & 3) == 0)
#pragma unroll
            for (int i = 0; i < 4; ++i) vr[i][j] = flip(vr[i][j]);
        *reinterpret_cast<u2 *>(buf + L::v + (vd + piece) * L::vPitch + 16 * (2 * (tq >> 2) + (tq & 1)) + 8 * ((tq >> 1) & 1)) =
            u2{centred(__builtin_amdgcn_perm(vr[1][j], vr[0][j], sel)), centred(__builtin_amdgcn_perm(vr[3][j], vr[2][j], sel))};
    };
    // ---- computing, 32 keys: e = score * factor + shift (the offset of the codes in the shift), the weights to be divided by 1 / inv
    float factor[2], shift[2], inv[2];
    auto scales_of = [&](int at) __attribute__((always_inline)) {              // block `at` of the lanes' and the one behind it
        auto of_block = [&](float v, int b) {
            return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), at + b));
        };
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            factor[b] = of_block(b_scale, b);
            shift[b] = fmaf(start, factor[b], of_block(b_log, b));
            inv[b] = of_block(b_inv, b);
        }
    };
    auto largest = [&](const f16v &s, int b) __attribute__((always_inline)) {
        const int i = 8 * b;
        const float m = larger(larger(larger(s[i], s[i + 1], s[i + 2]), s[i + 3], s[i + 4]), s[i + 5], larger(s[i + 6], s[i + 7], s[i + 7]));
        return fmaf(m, factor[b], shift[b]);
    };
    // Half a tile: the scores of the next 32 keys (K's rows 32 half ..) and between their products the weights of the last ones, `now`; then the weights'
    // products with V, and between them `pieces` of staging.  Operands are read from LDS four products ahead, and a weight's argument, power of two and sum lie a product
    // apart, so that none waits for the one before (one after the other 321 us for 316, two prompts of up to 4096 tokens).  The order is the one written.
    auto half_tile = [&](const unsigned char *buf, int half, const f16v &now, f16v &then, int at, auto stage, int pieces) __attribute__((always_inline)) {
        constexpr int kAhead = 4, per = 16 / KS;
        const unsigned char *kp = buf + L::k + (32 * half + n) * L::kPitch + 16 * hh;
        const unsigned char *vp = buf + L::v + n * L::vPitch + 16 * hh + 64 * half;
        h8 f[KS + 2 * DB];
        auto read = [&](int i) __attribute__((always_inline)) {
            f[i] = i < KS ? *reinterpret_cast<const h8 *>(kp + 32 * i)
                          : *reinterpret_cast<const h8 *>(vp + 32 * ((i - KS) % DB) * L::vPitch + 32 * ((i - KS) / DB));
        };
        h8 p[2];
        float sum[2] = {0.0f, 0.0f};
        const float to_p[2] = {shift[0] - M, shift[1] - M};
#pragma unroll
        for (int i = 0; i < 16; ++i) then[i] = 0.0f;
        __builtin_amdgcn_sched_barrier(0);
        float e[16];
        auto arguments = [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int k = per * i; k < per * (i + 1); ++k) e[k] = fmaf(now[k], factor[k >> 3], to_p[k >> 3]);
        };
        auto weights = [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int k = per * i; k < per * (i + 1); ++k) {
                sum[k >> 3] += e[k];
                p[k >> 3][k & 7] = (_Float16)e[k];
            }
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read(i);
        arguments(0);
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            read(i + kAhead);
            then = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[i], q[i], then, 0, 0, 0);
#pragma unroll
            for (int k = per * i; k < per * (i + 1); ++k) e[k] = __builtin_amdgcn_exp2f(e[k]);
            if (i + 1 < KS) arguments(i + 1);
            if (i) weights(i - 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        weights(KS - 1);
        // M is five below the largest e, or up to ten lower: what passes it by more shows in the sums (the first keys of a row: M is none yet).  No
        // maxima where it does not, a sixth of the vector unit's work.
        if (__ballot(sum[0] > kMostSum || sum[1] > kMostSum)) {
            const float top = fmaxf(largest(now, 0), largest(now, 1));
            const float to = fmaxf(M, fmaxf(top, __shfl_xor(top, 32, 64)) - kRaisedMany);
            const float down = __builtin_amdgcn_exp2f(M - to);
            M = to;
            l *= down;
#pragma unroll
            for (int i = 0; i < DB; ++i) o[i] *= down;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                sum[b] = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(now[8 * b + i], factor[b], shift[b] - M));
                    sum[b] += e;
                    p[b][i] = (_Float16)e;
                }
            }
        }
        l = fmaf(sum[0], inv[0], l);
        l = fmaf(sum[1], inv[1], l);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 2 * DB; ++i) {
            if (i + kAhead < 2 * DB) read(KS + i + kAhead);
            o[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[KS + i], p[i / DB], o[i % DB], 0, 0, 0);
#pragma unroll
            for (int k = pieces * i / (2 * DB); k < pieces * (i + 1) / (2 * DB); ++k) stage(k);
            if (i == 0) scales_of(at);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto first_scores = [&](const unsigned char *buf, f16v &s) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
        for (int i = 0; i < KS; ++i)
            s = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const h8 *>(buf + L::k + (32 + n) * L::kPitch + 16 * hh + 32 * i), q[i], s, 0, 0, 0);
    };
    // Scores of the 32 keys from `key` on: minus infinity where a row does not see them.
    auto mask = [&](int key, f16v &s) __attribute__((always_inline)) {
        if (key + 32 > least) {                       // (the same in all lanes)
            const int room = min(sees, key1) - (key + 4 * hh);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (8 * (i >> 2) + (i & 3) >= room) s[i] = -INFINITY;
        }
    };

    if (key0 < key1) {                                // (the same in all threads)
        const int tiles = (key1 - key0 + kKeys - 1) / kKeys;
        u4 kr0[KL];
        read_pages(0);
        const int key_first = key0 - 32 + 16 * lane;  // the first 32 keys: as the last ones of a tile of K
        const int page_first = key_first >= key0 && key_first < key1 ? table[key_first >> a.shift] : -1;
        read_q();                                     // (behind the block numbers, which the codes wait for)
        take_units(0);
        fetch_k(place_of(page_first, key_first), 0, kr0);
        fetch_k(unit_k, 0, kr);
        fetch_v(0);
#pragma unroll
        for (int k = 0; k < kPieces; ++k) stage_k(lds + L::bytes, kr0, k);
#pragma unroll
        for (int k = 0; k < kPieces; ++k) stage_k(lds, kr, k);
#pragma unroll
        for (int k = 0; k < vPieces; ++k) stage_v(lds, k);
        fetch_k(unit_k, 4, kr);
        fetch_v(4);
#pragma unroll
        for (int s = 0; s < KS; ++s) start = add8(q[s], start);
        start += __shfl_xor(start, 32, 64);
        start *= -128.0f * 5.9604644775390625e-08f;
        take_scales(0);
        __syncthreads();
        f16v x, y;
        first_scores(lds + L::bytes, x);
        scales_of(0);
        mask(key0, x);
        __syncthreads();
        int at = 0;
        for (int t = 0; t < tiles; ++t, at ^= L::bytes) {
            unsigned char *here = lds + at, *next = lds + (at ^ L::bytes);
            const int key = key0 + t * kKeys, block = 4 * (t & 15), ahead = 4 * ((t + 2) & 15);
            auto next_k = [&](int k) __attribute__((always_inline)) { stage_k(next, kr, k); };
            auto next_v = [&](int k) __attribute__((always_inline)) { stage_v(next, k); };
            if (key < wave1) {                        // (the same in all lanes)
                half_tile(here, 0, x, y, block + 2, next_k, kPieces);
                mask(key + 32, y);
            } else {
#pragma unroll
                for (int k = 0; k < kPieces; ++k) next_k(k);
            }
            if (ahead == 0) take_units(t + 2);
            if (block == 60) take_scales(t + 1);
            fetch_k(unit_k, ahead, kr);
            if (key + 32 < wave1) {
                half_tile(here, 1, y, x, (block + 4) & 63, next_v, vPieces);
                mask(key + 64, x);
            } else {
#pragma unroll
                for (int k = 0; k < vPieces; ++k) next_v(k);
            }
            fetch_v(ahead);
            if (ahead == 60) read_pages(t + 3);
            __syncthreads();
        }
    }

    l += __shfl_xor(l, 32, 64);
    if (sees > spoiled) l = NAN;
    if (w.splits == 1) {
        // by way of this wavefront's own part of LDS, so that a store has whole rows (nobody reads codes there any more)
        constexpr int pitch = 2 * D + 16, lanes = D / 8;      // lanes of a row
        unsigned char *mine = lds + wave * 32 * pitch;
        const float f = quotient(l);
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const __half2 lo = __floats2half2_rn(o[i][4 * j] * f, o[i][4 * j + 1] * f), hi = __floats2half2_rn(o[i][4 * j + 2] * f, o[i][4 * j + 3] * f);
                *reinterpret_cast<u2 *>(mine + n * pitch + 64 * i + 16 * j + 8 * hh) = u2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
            }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 32 * lanes / 64; ++i) {
            const int rr = i * (64 / lanes) + lane / lanes;
            if (rr < rows) {
                const int t = by_group(a, row0 + rr);
                __half *to = a.out + (int64_t)(r.start + t) * a.ldo + (int64_t)(h * a.group + row0 + rr - t * a.group) * D + 8 * (lane % lanes);
                *reinterpret_cast<u4 *>(to) = *reinterpret_cast<const u4 *>(mine + rr * pitch + 16 * (lane % lanes));
            }
        }
    } else if (n < rows) {
        float *part = job.part + (((int64_t)(w.first_slot + w.split) * a.Hkv + h) * job.part_rows + wave * 32 + n) * (D + 4);
        if (hh == 0) *reinterpret_cast<f2 *>(part) = f2{M, l};
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<f4 *>(part + 4 + 32 * i + 8 * j + 4 * hh) = f4{o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]};
    }
}

// A step with requests of many rows: its few-row requests, which wait for memory, run beside the tiles of the others, which keep the matrix units
// busy (one launch after the other, 32 single tokens and two chunks of 125 and 318 tokens took 27 + 45 us).  Tiles come first: they take longest, and start on compute
// units of their own (the same step 48.6 -> 40.3 us; 40 requests of 32 heads, four of them chunks of up to 400 tokens, 104 -> 79; 100 requests, 12 chunks, 248 -> 232).
template <int D>
__global__ __launch_bounds__(256, 2)
void attention_kv8_step_kernel(const Args a, const Job few, const Job many)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    static_assert(sizeof(RowsLds<D, 4, 1>) <= 2 * TileLds<D>::bytes, "one workgroup's LDS");
    const int first = many.groups * a.Hkv;
    if ((int)blockIdx.x >= first) rows_tile<D, false, 4, 1>(a, few, blockIdx.x - first, *reinterpret_cast<RowsLds<D, 4, 1> *>(lds));
    else                         many_rows_tile<D>(a, many, blockIdx.x, lds);
}

// The pieces of tiles, in their order: 16 rows of a tile and cache head for a workgroup, first those of few rows, then those of
// many.  What bounds it is its chain of reads (lengths, then the pieces), so eight pieces are read at once.
template <int D>
__global__ __launch_bounds__(256)
void attention_kv8_merge_kernel(const Args a, const Job few, const Job many)
{
    const bool is_few = (int)blockIdx.x < few.merges * a.Hkv;
    const Job job = is_few ? few : many;
    const int index = is_few ? blockIdx.x : blockIdx.x - few.merges * a.Hkv, h = index % a.Hkv;
    const int subs = 1 << (job.log - kRowsLog), sub = index / a.Hkv & (subs - 1);
    const Place w = place<true>(a, job, index / a.Hkv >> (job.log - kRowsLog));
    if (!w.found || w.splits == 1) return;
    const Request r = w.r;
    const int all = r.n * a.group, part_rows = job.part_rows;
    const float *part = job.part;
    // (the kernel of many rows takes a request's tiles from the last one on)
    const int tile = is_few ? w.tile : ((all - 1) >> job.log) - w.tile;
    const int first = (tile << job.log) + sub * kSetRows, rows = min(kSetRows, all - first);
    const int64_t stride = (int64_t)a.Hkv * part_rows * (D + 4);
    for (int i = threadIdx.x; i < rows * (D / 4); i += 256) {
        const int rr = i / (D / 4), d = 4 * (i % (D / 4));
        const float *from = part + (((int64_t)w.first_slot * a.Hkv + h) * part_rows + sub * kSetRows + rr) * (D + 4);
        float top = kNoScore, sum = 0.0f;
        f4 o = f4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < w.splits; s += 8) {
            float m[8], l[8];
            f4 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float *piece = from + min(s + k, w.splits - 1) * stride;
                const f2 ml = *reinterpret_cast<const f2 *>(piece);
                m[k] = s + k < w.splits ? ml[0] : kNoScore;
                l[k] = s + k < w.splits ? ml[1] : 0.0f;
                v[k] = *reinterpret_cast<const f4 *>(piece + 4 + d);
            }
            float to = top;
#pragma unroll
            for (int k = 0; k < 8; ++k) to = fmaxf(to, m[k]);
            const float down = __builtin_amdgcn_exp2f(top - to);
            top = to;
            sum *= down;
            o *= down;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float f = s + k < w.splits ? __builtin_amdgcn_exp2f(m[k] - top) : 0.0f;
                sum = fmaf(l[k], f, sum);
                o += v[k] * f;
            }
        }
        const float f = quotient(sum);
        const int row = first + rr, t = by_group(a, row);
        __half *to = a.out + (int64_t)(r.start + t) * a.ldo + (int64_t)(h * a.group + row - t * a.group) * D + d;
        const __half2 lo = __floats2half2_rn(o[0] * f, o[1] * f), hi = __floats2half2_rn(o[2] * f, o[3] * f);
        *reinterpret_cast<u2 *>(to) = u2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
    }
}

// ---------------------------------------------------------------- shape of a call

// Requests of up to kFew query rows (tokens times the heads of a group) are work of the first kind, larger ones of the second if the call has enough of that.
constexpr int kFew = 64;
// Workgroups that the card has room for at once: of the kernel of few rows; of few rows beside many; of many rows one a compute unit, and two.
constexpr int kFewWorkgroups = 1024, kFewBeside = 512, kManyWorkgroups = 256;
// Tiles of many rows are cut to one workgroup a compute unit, and to two where they fill half of those at most and sequences are long: then a tile is
// halved at least, which pays for the pieces' starts and the merge (tokens, earlier keys: heads 64 on 8, 200 (6000) 80.2 -> 69.3 us, 2 x 300 (2000) 56.1 -> 47.0; 32 on 32,
// 400 (4000) 63.1 -> 54.9; but 32 single tokens and two chunks of 125 and 318 (2000), which share the card, 48.1 -> 57.5).
int many_workgroups(int64_t tiles, int Hkv, int64_t capacity) { return tiles * Hkv <= kManyWorkgroups && capacity >= 1536 ? 2 * kManyWorkgroups : kManyWorkgroups; }
// Beside many rows, sequences of up to so many keys are not cut (a merge is a launch of 4 us).
constexpr int kUncutBeside = 4096;
// Few rows alone, uncut: workgroups of 4, 8 or 16 wavefronts (the most that run at once and have a step each), where the longest sequence costs less than a
// merge.  Its compute unit reads 50 bytes a ns; of a full card the shorter sequences of a batch leave it a part of what they would read.
// Uncut / cut, us, the longest sequence 500, 1000, 2000 (lengths from a quarter of it): 32 cache heads of 128, one sequence 8.1 / 10.0, 10.6 / 10.0, 16.7 / 10.3;
// 8 sequences 9.2 / 12.2, 13.1 / 15.5, 19.3 / 21.4; 8 cache heads, 64 sequences 12.6 / 17.2, 18.7 / 23.9, -; 4 of 64, one of 1000 6.8 / 8.2.
constexpr double kUncutBytes = 205e3;
int wavefronts(int64_t tiles, int Hkv, int D, int64_t capacity)              // 0: cut
{
    const int64_t groups = tiles * Hkv;
    if (groups > kFewWorkgroups || capacity <= 128) return 4;
    const int    room = groups <= kFewWorkgroups / 4 ? 16 : groups <= kFewWorkgroups / 2 ? 8 : 4;
    const double full = (double)groups * room / (4 * kFewWorkgroups);
    if ((double)capacity * 2 * D * (16 / room) * (1.0 - 0.75 * full) >= kUncutBytes) return 0;
    return capacity <= 256 && room > 8 ? 8 : room;
}

// Few rows alone, but more than 16 to a request (drafts): tiles of 32 from so many tiles times keys on, below that the tiles of 16 run at once anyway. Of 16 / of 32, us
// (tokens, keys): heads 64 on 8 of 128, 64 sequences of 4 (3000) 72.5 / 52.4, 16 of 4 (4000) 29.7 / 26.1; 32 on 8, 32 of 6 (3000) 36.6 / 33.1, 8 of 8 (1500) 17.2 / 17.6;
// 16 on 4 of 64, 23 of 5 (5000) 17.4 / 16.0, one of 8 (9000) 16.6 / 17.4.
constexpr double kTwoSets = 2e5;

struct Shape { Job few, many; size_t floats; int waves, sets; };    // of a workgroup of few rows: its wavefronts, its sets of 16 rows

// `want` workgroups together, for each cache head: where there are fewer tiles (and 128 keys to a piece) they are cut.
void size_job(Job &job, int64_t tiles, int log, int part_rows, int64_t want, int Hkv, int64_t capacity)
{
    job.log = log;
    const int64_t most = tiles * ((capacity + 127) / 128);
    int64_t budget = (want + Hkv - 1) / Hkv;
    if (budget > most) budget = most;
    job.budget = budget > tiles ? (int)budget : 0;
    job.groups = (int)(job.budget ? budget : tiles);
    job.merges = job.budget ? (int)(tiles << (log - kRowsLog)) : 0;
    job.part_rows = part_rows;
}

size_t records(const Job &job, int Hkv, int D) { return job.budget ? (size_t)job.groups * Hkv * job.part_rows * (D + 4) : 0; }

int64_t many_tiles(int64_t T, int B, int group, int64_t rows, int few_most)
{
    const int64_t each = (int64_t)B * ((rows + kTile - 1) / kTile), requests = T * group / (few_most + 1) < B ? T * group / (few_most + 1) : B;
    return each < T * group / kTile + requests ? each : T * group / kTile + requests;
}

// Whether a call's requests of more than kFew rows are better tiles of 128 rows, in us, by what the host knows (tables may be wider than they are full).
// 16 or 32 rows at a time the work spreads over the card, but turns each code into halves more often: 1.4 us for a million pairs of rows and keys (D = 64:
// 0.6).  128 at a time a tile takes 1.5 us for 64 keys, 1.85 where two share a compute unit, and where tiles are cut
// their pieces' starts and the merge take 18.  Tiles / few rows, measured (tokens, earlier keys): heads 64 on 8: 1000 31.9 / 51.7 us, 2000 87.3 / 143, 299 (229) 21.2 / 19.8, 100 (3000) 33.3 / 33.5,
// 65 (679) 18.2 / 17.3; 32 on 32: 1000 27.4 / 29.3, 400 (4000) 55.3 / 63.1; 16 on 4: 1046 (398) 37.9 / 29.6, 2 x 470 20.2 / 13.0; 20 on 1: 3 x 353 20.2 / 10.6, 3000 74 / 99;
// 12 on 12: 2 x 196 15.7 / 6.0; of 64: 16 on 4: 3000 55.8 / 46.5, 12 on 12: 2000 (1000) 49.8 / 33.0, 64 on 8: 4 x 706 25.4 / 34.9, 40 on 8: 900 (3000) 76.9 / 68.3.
bool worth_tiles(int64_t T, int64_t tiles, int Hkv, int group, int D, int max_new, int64_t capacity)
{
    const double keys = max_new < capacity ? (double)capacity - 0.5 * max_new : 0.5 * (double)capacity, steps = (double)capacity / 64, n = (double)tiles * Hkv;
    const double few = 8 + (double)T * group * Hkv * keys * 1e-6 * (D == 128 ? 1.4 : 0.6);
    const double shared = n * keys / 64 * 0.0048, alone = steps * (n > 256 ? 1.85 : 1.5);
    const int    want = many_workgroups(tiles, Hkv, capacity);
    const double many = (want + Hkv - 1) / Hkv > tiles ? 18 + n * steps / 256 * (want > kManyWorkgroups ? 1.2 : 1.95) : 7 + (shared > alone ? shared : alone);
    return many * (D == 128 ? 1.0 : 0.8) < few;
}

Shape shape(int64_t T, int B, int Hkv, int group, int D, int max_new, int64_t capacity)
{
    Shape s = {};
    if (T == 0 || B == 0 || max_new == 0) return s;
    const int64_t rows = (int64_t)max_new * group;   // of one request, at most
    const bool many = rows > kFew && worth_tiles(T, many_tiles(T, B, group, rows, B > 1 ? kFew : 0), Hkv, group, D, max_new, capacity);
    const int  few_most = many ? (B > 1 ? kFew : 0) : (int)rows;         // (one request is work of the second kind whatever its size)
    s.few.rows_min = 1;
    s.few.rows_max = few_most;
    s.many.rows_min = few_most + 1;
    s.many.rows_max = 0x7fffffff;
    if (few_most) {
        auto tiles = [&](int rows) {
            const int64_t each = (int64_t)B * ((few_most + rows - 1) / rows), by_token = T * group / rows + B;
            return each < by_token ? each : by_token;
        };
        const int waves = many ? 4 : wavefronts(tiles(kSetRows), Hkv, D, capacity);
        s.sets = !many && few_most > kSetRows && (waves == 0 || waves == 4) && (double)tiles(2 * kSetRows) * Hkv * capacity >= kTwoSets ? 2 : 1;
        s.waves = waves ? waves : 4;
        const int rows = s.sets * kSetRows;
        size_job(s.few, tiles(rows), kRowsLog + s.sets - 1, few_most < rows ? few_most : rows,
                 !many ? (waves ? 0 : s.sets == 2 ? kFewWorkgroups / 2 : kFewWorkgroups) : capacity > kUncutBeside ? kFewBeside : 0, Hkv, capacity);
    }
    if (many) {
        const int64_t tiles = many_tiles(T, B, group, rows, few_most);
        size_job(s.many, tiles, kTileLog, kTile, many_workgroups(tiles, Hkv, capacity), Hkv, capacity);
    }
    s.floats = records(s.few, Hkv, D) + records(s.many, Hkv, D);
    return s;
}

// A cache that the last-level cache (256 MB) does not keep until the next step is read with the hint that nothing reads it again, where a row is read
// by one workgroup only.
bool reads_once(const Args &a, const Job &few)
{
    return few.rows_max <= 1 << few.log && (int64_t)a.B * a.Hkv * a.capacity * 128 >= (int64_t)1 << 27;
}

template <int D, int kWaves, int SETS = 1>
hipError_t launch_rows(const Args &a, const Job &few, dim3 grid, hipStream_t stream)
{
    constexpr int bytes = sizeof(RowsLds<D, kWaves, SETS>);
    const bool once = reads_once(a, few);
    auto kern = once ? &attention_kv8_rows_kernel<D, true, kWaves, SETS> : &attention_kv8_rows_kernel<D, false, kWaves, SETS>;
    if (bytes > 60 * 1024) {
        static atom_launch::LdsOptIn opt[2];
        hipError_t err = atom_launch::ensure_dynamic_lds(opt[once], reinterpret_cast<const void *>(kern), bytes);
        if (err != hipSuccess) return err;
    }
    hipLaunchKernelGGL(kern, grid, dim3(kWaves * 64), bytes, stream, a, few);
    return hipGetLastError();
}

template <int D>
hipError_t launch(const Args &a, Shape s, float *workspace, hipStream_t stream)
{
    s.few.part = workspace;
    s.many.part = workspace + records(s.few, a.Hkv, D);
    if (!s.many.groups) {
        if (!s.few.groups) return hipSuccess;
        const dim3 grid((unsigned)(s.few.groups * a.Hkv));
        hipError_t err = s.sets == 2 ? launch_rows<D, 4, 2>(a, s.few, grid, stream)
                         : s.waves == 16 ? launch_rows<D, 16>(a, s.few, grid, stream)
                         : s.waves == 8 ? launch_rows<D, 8>(a, s.few, grid, stream) : launch_rows<D, 4>(a, s.few, grid, stream);
        if (err != hipSuccess) return err;
    } else {
        static atom_launch::LdsOptIn opt;
        constexpr int bytes = 2 * TileLds<D>::bytes;
        hipError_t err = atom_launch::ensure_dynamic_lds(opt, reinterpret_cast<const void *>(&attention_kv8_step_kernel<D>), bytes);
        if (err != hipSuccess) return err;
        hipLaunchKernelGGL((attention_kv8_step_kernel<D>), dim3((unsigned)((s.few.groups + s.many.groups) * a.Hkv)), dim3(256), bytes, stream, a,
                           s.few, s.many);
    }
    hipError_t err = hipGetLastError();
    const int merges = (s.few.merges + s.many.merges) * a.Hkv;
    if (err != hipSuccess || !merges) return err;
    hipLaunchKernelGGL((attention_kv8_merge_kernel<D>), dim3((unsigned)merges), dim3(256), 0, stream, a, s.few, s.many);
    return hipGetLastError();
}

}  // namespace

namespace atom_internal {

size_t attention_kv8_workspace_bytes(int64_t T, int B, int H, int Hkv, int D, int max_new, int64_t W, int block_tokens)
{
    return shape(T, B, Hkv, H / Hkv, D, max_new, W * block_tokens).floats * sizeof(float);
}

bool attention_kv8_fits(int64_t T, int B, int H, int Hkv, int D, int max_new, int64_t W, int block_tokens)
{
    // first, that shape() can count in 32 bits: every count is below (rows / 16 + B) * blocks of 128 rows and the workgroups wanted, as doubles here
    const double group = H / Hkv, rows = (double)max_new * group, tiles = (double)T * group / kSetRows + B, each = (double)B * (rows / kSetRows + 1);
    const double most = (tiles < each ? tiles : each) + kFewWorkgroups;
    if (2.0 * most * Hkv >= 2147483647.0) return false;
    const Shape   s = shape(T, B, Hkv, H / Hkv, D, max_new, W * block_tokens);
    const int64_t threads = ((int64_t)s.few.groups + s.many.groups) * Hkv * 64 * (s.many.groups ? 4 : s.waves);
    return threads <= atom_launch::kMostThreads && ((int64_t)s.few.merges + s.many.merges) * Hkv * 256 <= atom_launch::kMostThreads;
}

// How a call of these sizes runs, as its tests ask it: wavefronts of a workgroup of few rows, 32 where those requests' keys may be cut, 64 where
// requests of many rows are tiles of 128, 128 where those may be cut, 256 where few rows
// are tiles of 32.
extern "C" int atom_internal_attention_kv8_route(int64_t T, int32_t B, int32_t H, int32_t Hkv, int32_t D, int32_t max_new, int64_t W, int32_t block_tokens)
{
    const Shape s = shape(T, B, Hkv, H / Hkv, D, max_new, W * block_tokens);
    return (s.few.groups ? (s.many.groups ? 4 : s.waves) : 0) + (s.sets == 2 ? 256 : 0) + (s.few.budget ? 32 : 0) + (s.many.groups ? 64 : 0) + (s.many.budget ? 128 : 0);
}

hipError_t launch_attention_kv8(const AttentionKv8 &c, hipStream_t stream)
{
    Args a;
    a.q = (const __half *)c.q; a.T = (int)c.T; a.ldq = c.ldq;
    a.B = c.B; a.Hkv = c.Hkv; a.group = c.H / c.Hkv;
    const int log = a.group > 1 ? 32 - __builtin_clz((unsigned)(a.group - 1)) : 0;
    a.div_shift = 31 + log;
    a.div_mul = (uint32_t)(((uint64_t)1 << a.div_shift) / (unsigned)a.group + 1);
    a.max_new = c.max_new;
    a.token_start = c.token_start; a.seq_len = c.seq_len; a.table = c.block_table;
    a.W = (int)c.W; a.shift = __builtin_ctz((unsigned)c.block_tokens);
    a.capacity = c.W * c.block_tokens;
    a.n_blocks = (int32_t)c.n_blocks;
    a.kq = (const int8_t *)c.k_codes; a.ks = c.k_scale; a.vq = (const int8_t *)c.v_codes; a.vs = c.v_scale;
    a.sm_scale = c.sm_scale;
    a.out = (__half *)c.out; a.ldo = c.ldo;
    const Shape s = shape(c.T, c.B, c.Hkv, a.group, c.D, c.max_new, a.capacity);
    return c.D == 128 ? launch<128>(a, s, (float *)c.workspace, stream) : launch<64>(a, s, (float *)c.workspace, stream);
}

}  // namespace atom_internal
