// The lookup at a model's start: rows of an MX4 table by their ids, and the gradient of the whole
// table, for which the ids are sorted first, so that every row of it is one sum in the order of
// the tokens.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "launch.h"
#include "mx_dev.h"
#include "mx_model.h"
#include "mx_small.h"

namespace fastrack {
namespace mx {

// ---- lookup ---------------------------------------------------------------------------------
//
// A lane loads a block, 16 bytes of codes: with 4 bytes to a lane there is too little on its way to
// cover the way to memory. (16384 rows of 4096 out of 143 MB, 170 MB in all: 32 us, 5.3 TB/s; with 4 bytes 44.) Four
// neighbouring lanes hold blocks 16 apart and exchange their words, so that a wave writes 1 KB that
// lies together at a time, 8 values to a lane.
constexpr int kThreads = 256;

struct Lookup {
    MxIds ids;
    MxMatrix table;
    uint32_t rows, cols, nb, recip, blocks;   // blocks of a row; of this launch
    uint64_t t0;                              // first token of this launch
    float scale;
    MxRows y;
};

// The value of lane I of each four.
template <int I>
__device__ __forceinline__ uint32_t from_lane(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, I * 0x55, 0xF, 0xF, true);
}

template <uint32_t T>
__global__ __launch_bounds__(kThreads) void lookup_kernel(Lookup g)
{
    const uint32_t lane = threadIdx.x & 63, j = lane & 3, first = blockIdx.x * kThreads + threadIdx.x - lane;
    if (first >= g.blocks)   // a whole wave
        return;
    // (Past the last block it is read again.)
    const uint32_t at = min(first + j * 16 + lane / 4, g.blocks - 1), r = div_recip(at, g.nb, g.recip);
    const int64_t id = id_of(g.ids, g.t0 + r);
    u32x4 codes = {0, 0, 0, 0};
    uint32_t e = id < 0 ? 127 : 255;   // padding: zeros; no row of the table: NaN
    if (id >= 0 && id < (int64_t)g.rows) {
        const uint64_t block = (uint64_t)id * g.nb + (at - r * g.nb);
        codes = reinterpret_cast<const u32x4 *>(g.table.codes)[block];
        e = g.table.scales[block];
    }
    auto put_unit = [&](auto i_) {
        constexpr int I = decltype(i_)::value;
        const uint32_t w0 = from_lane<I>(codes[0]), w1 = from_lane<I>(codes[1]), w2 = from_lane<I>(codes[2]), w3 = from_lane<I>(codes[3]);
        const uint32_t to = first + I * 16 + lane / 4, row = div_recip(to, g.nb, g.recip), c = (to - row * g.nb) * 32 + j * 8;
        float v[8];
        decode4_f32(j & 2 ? (j & 1 ? w3 : w2) : (j & 1 ? w1 : w0), scale4_f32(from_lane<I>(e)), v);
#pragma unroll
        for (int x = 0; x < 8; ++x)
            v[x] *= g.scale;
        if (to < g.blocks && c < g.cols)
            store8<T>(g.y.p, (g.t0 + row) * g.y.ld, c, g.cols, v);
    };
    put_unit(Const<0>());
    put_unit(Const<1>());
    put_unit(Const<2>());
    put_unit(Const<3>());
}

// ---- sorting ids -------------------------------------------------------------------------------
//
// Keys below 2^bits (the number of rows itself for ids that count for none), each with its place,
// sorted by key and then by place: passes over a digit each, the lowest first. In a pass a
// wave ranks its 64 keys among equal digits by one vote per bit, and adds what came before
// them: in its own earlier keys, in the waves before it, and in the blocks before.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr uint32_t kDigitBits = 9, kDigits = 1u << kDigitBits;

struct Sort {
    MxIds ids;                    // of the first pass; later ones read keys and places
    const uint32_t *keys, *places;
    uint32_t *keys_out, *places_out;
    uint32_t n, rows, shift, bits, blocks;
    uint32_t *counts;             // [1 << bits][blocks], then the sums before each
    bool first;
};

constexpr int kMostItems = 16;    // keys of a thread
constexpr uint32_t kSortBlock = kSortThreads * kMostItems;

__device__ __forceinline__ uint32_t key_of(const MxIds &ids, uint32_t i, uint32_t rows)
{
    const int64_t id = id_of(ids, i);
    return id >= 0 && id < (int64_t)rows ? (uint32_t)id : rows;
}

// A wave's keys are 64 K that follow one another, 64 at a time. `counts[digit]` of the wave grows;
// rank[] is a key's number among the wave's equal digits.
template <int K>
__device__ __forceinline__ void rank_keys(const uint32_t (&key)[K], uint32_t (&rank)[K], uint32_t valid, uint32_t shift,
                                          uint32_t bits, uint32_t *counts)
{
    const uint32_t lane = threadIdx.x & 63, mask = (1u << bits) - 1;
#pragma unroll
    for (int i = 0; i < K; ++i) {
        if (i * 64u >= valid)   // the whole wave
            break;
        const bool in = i * 64u + lane < valid;
        const uint32_t d = key[i] >> shift & mask, so_far = counts[d];
        const uint64_t all = __ballot(in);
        uint32_t lo = (uint32_t)all, hi = (uint32_t)(all >> 32);   // lanes with the same digit
        for (uint32_t b = 0; b < bits; ++b) {
            const int32_t s = (int32_t)(d << (31 - b)) >> 31;
            const uint64_t v = __ballot(s != 0);
            lo &= ~((uint32_t)v ^ (uint32_t)s);
            hi &= ~((uint32_t)(v >> 32) ^ (uint32_t)s);
        }
        rank[i] = so_far + __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
        if (in && lane == (hi ? 63u - (uint32_t)__builtin_clz(hi) : 31u - (uint32_t)__builtin_clz(lo | 1)))   // the last of them
            counts[d] = rank[i] + 1;
        wave_fence();
    }
}

// counts[wave][digit] of a workgroup to where each wave's first key of a digit goes among the
// workgroup's; total[digit] of thread `digit` is returned. Threads past the digits bring 0.
__device__ __forceinline__ uint32_t digits_before(uint32_t (*counts)[kDigits], uint32_t *sums, uint32_t mask, uint32_t &before)
{
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6;
    uint32_t total = 0;
    if (t <= mask) {
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = counts[w][t];
            counts[w][t] = total;
            total += c;
        }
    }
    uint32_t sum = total;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_up(sum, d, 64);
        sum += lane >= (uint32_t)d ? o : 0;
    }
    if (lane == 63 && wave < kDigits / 64)
        sums[wave] = sum;
    __syncthreads();
    before = sum - total;
    for (uint32_t w = 0; w < wave && w < kDigits / 64; ++w)
        before += sums[w];
    return total;
}

// Zeros into rows of `width` bytes, by `parts` workgroups: 16 KB each of all bytes as they follow one
// another (16 bytes to a thread and no loop: 1 GiB in 171 us, 156 in workgroups of 256, 190-250 in
// loops of as many workgroups as run at once), or a row to a wave, where gaps stay as they are.
struct Zero {
    uint8_t *p;
    uint64_t stride, width, rows;
    uint32_t parts;
};

// The 16-byte pieces first, first + step, ... of p[0, n), and the 16-bit values before and behind the
// aligned ones.
__device__ __forceinline__ void zero_bytes(uint8_t *p, uint64_t n, uint64_t first, uint64_t step)
{
    const u32x4 zero = {0, 0, 0, 0};
    const uint64_t align = (16 - reinterpret_cast<uintptr_t>(p) % 16) % 16, head = align < n ? align : n;
    const uint64_t whole = (n - head) / 16, tail = head + whole * 16, ends = head + (n - tail);
    for (uint64_t i = first; i < whole; i += step)
        reinterpret_cast<u32x4 *>(p + head)[i] = zero;
    for (uint64_t b = first * 2; b < ends; b += step * 2)
        *reinterpret_cast<uint16_t *>(p + (b < head ? b : tail + (b - head))) = 0;
}

template <uint32_t THREADS>
__device__ __forceinline__ void zero_part(const Zero &z, uint32_t part)
{
    if (z.rows == 1) {
        zero_bytes(z.p, z.width, (uint64_t)part * THREADS + threadIdx.x, (uint64_t)z.parts * THREADS);
        return;
    }
    for (uint64_t r = (uint64_t)part * (THREADS / 64) + threadIdx.x / 64; r < z.rows; r += (uint64_t)z.parts * (THREADS / 64))
        zero_bytes(z.p + r * z.stride, z.width, threadIdx.x % 64, 64);
}

__global__ __launch_bounds__(256) void zero_kernel(Zero z) { zero_part<256>(z, blockIdx.x); }

// All passes by one workgroup, up to kSortBlock ids. Keys and places go from pass to pass through
// LDS.
struct SortSmall {
    MxIds ids;
    uint32_t *keys_out, *places_out;
    uint32_t n, rows, bits, passes;   // bits of a digit
};

// (64 KB at most: two workgroups to a CU, so that those that write zeros fill the GPU.)
template <int K>
union SortLds {
    uint32_t swap[kSortThreads * K];
    struct {
        uint32_t counts[kSortWaves][kDigits];
        uint32_t base[kDigits];
        uint32_t sums[kDigits / 64];
    };
};

template <int K>
__device__ __forceinline__ void sort_small(const SortSmall &g, SortLds<K> &l)
{
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const uint32_t per = (g.n + kSortThreads - 1) / kSortThreads * 64, w0 = wave * per;   // keys of a wave
    const uint32_t valid = w0 < g.n ? min(per, g.n - w0) : 0;
    uint32_t key[K], place[K], to[K];
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const uint32_t at = i * 64 + lane;
        place[i] = w0 + at;
        key[i] = at < valid ? key_of(g.ids, w0 + at, g.rows) : 0;
    }
    auto swap = [&](uint32_t (&v)[K]) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i * 64 + lane < valid)
                l.swap[to[i]] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i * 64 + lane < valid)
                v[i] = l.swap[w0 + i * 64 + lane];
    };
    for (uint32_t p = 0; p < g.passes; ++p) {
        const uint32_t shift = p * g.bits, mask = (1u << g.bits) - 1;
        __syncthreads();
        for (uint32_t i = t; i < kSortWaves << g.bits; i += kSortThreads)
            l.counts[i >> g.bits][i & mask] = 0;
        __syncthreads();
        rank_keys(key, to, valid, shift, g.bits, l.counts[wave]);
        __syncthreads();
        uint32_t before;
        digits_before(l.counts, l.sums, mask, before);
        if (t < kDigits)
            l.base[t] = before;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const uint32_t d = key[i] >> shift & mask;
            to[i] += l.base[d] + l.counts[wave][d];
        }
        if (p + 1 < g.passes) {
            swap(key);
            swap(place);
        }
    }
#pragma unroll
    for (int i = 0; i < K; ++i)
        if (i * 64 + lane < valid) {
            g.keys_out[to[i]] = key[i];
            g.places_out[to[i]] = place[i];
        }
}

// Workgroup 0 sorts; the others write zeros meanwhile.
template <int K>
__global__ __launch_bounds__(kSortThreads) void sort_small_kernel(SortSmall g, Zero z)
{
    __shared__ SortLds<K> l;
    if (blockIdx.x)
        zero_part<kSortThreads>(z, blockIdx.x - 1);
    else
        sort_small(g, l);
}

// A pass of many workgroups: the digits of each block counted, the counts added up (digit by
// digit, block by block), the keys put where they go.
__device__ __forceinline__ void load_keys(const Sort &g, uint32_t w0, uint32_t valid, uint32_t (&key)[kMostItems])
{
    const uint32_t lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < kMostItems; ++i) {
        const uint32_t at = i * 64 + lane;
        key[i] = at >= valid ? 0 : g.first ? key_of(g.ids, w0 + at, g.rows) : g.keys[w0 + at];
    }
}

template <bool PUT>
__global__ __launch_bounds__(kSortThreads) void sort_pass_kernel(Sort g)
{
    __shared__ uint32_t counts[kSortWaves][kDigits];
    __shared__ uint32_t sums[kDigits / 64];
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6, mask = (1u << g.bits) - 1;
    const uint64_t first = (uint64_t)blockIdx.x * kSortBlock + wave * (64 * kMostItems);
    const uint32_t w0 = (uint32_t)first, valid = first < g.n ? min(64u * kMostItems, g.n - w0) : 0;
    uint32_t key[kMostItems], rank[kMostItems];
    load_keys(g, w0, valid, key);
    for (uint32_t i = t; i < kSortWaves * kDigits; i += kSortThreads)
        (&counts[0][0])[i] = 0;
    __syncthreads();
    rank_keys(key, rank, valid, g.shift, g.bits, counts[wave]);
    __syncthreads();
    uint32_t before;
    const uint32_t total = digits_before(counts, sums, mask, before);
    if (!PUT) {
        if (t <= mask)
            g.counts[(uint64_t)t * g.blocks + blockIdx.x] = total;
        return;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMostItems; ++i)
        if (i * 64 + lane < valid) {
            const uint32_t d = key[i] >> g.shift & mask;
            const uint32_t to = g.counts[(uint64_t)d * g.blocks + blockIdx.x] + counts[wave][d] + rank[i];
            g.keys_out[to] = key[i];
            g.places_out[to] = g.first ? w0 + i * 64 + lane : g.places[w0 + i * 64 + lane];
        }
}

// Each count becomes the sum of those before it; one workgroup. The others write zeros meanwhile.
__global__ __launch_bounds__(1024) void sums_before_kernel(uint32_t *counts, uint32_t n, Zero z)
{
    __shared__ uint32_t sums[16];
    if (blockIdx.x) {
        zero_part<kSortThreads>(z, blockIdx.x - 1);
        return;
    }
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6;
    uint32_t carry = 0;
    for (uint32_t i0 = 0; i0 < n; i0 += 4096) {
        uint32_t v[4], own = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t i = i0 + t * 4 + j;
            v[j] = i < n ? counts[i] : 0;
            own += v[j];
        }
        uint32_t sum = own;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t o = __shfl_up(sum, d, 64);
            sum += lane >= (uint32_t)d ? o : 0;
        }
        if (lane == 63)
            sums[wave] = sum;
        __syncthreads();
        uint32_t before = carry + sum - own;
#pragma unroll
        for (uint32_t w = 0; w < 16; ++w) {
            before += w < wave ? sums[w] : 0;
            carry += sums[w];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t i = i0 + t * 4 + j;
            if (i < n)
                counts[i] = before;
            before += v[j];
        }
        __syncthreads();
    }
}

// ---- the gradient --------------------------------------------------------------------------------

struct Sums {
    const uint32_t *keys, *places;   // sorted
    uint32_t n, rows, cols;
    uint32_t chunks, tiles;          // of kChunk sorted tokens; of kTileCols columns
    MxRows dy;
    float scale;
    Out out;
    float *parts;                    // [chunks][2][part_ld], whole units
    uint32_t part_ld;
};

constexpr uint32_t kChunk = 16, kTileCols = 64 * 8;

template <uint32_t OT>
__device__ __forceinline__ void put_row(const Out &o, uint64_t row, uint32_t c, uint32_t cols, float (&v)[8], float scale)
{
    const uint64_t at = row * o.ld;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] *= scale;
    if (OT == kFp32 && o.accumulate) {
        float w[8];
        load8<kFp32>(o.p, at, c, cols, w);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] += w[e];
    }
    store8<OT>(o.p, at, c, cols, v);
}

// Few tokens: no sorting. A workgroup has 16 rows of the table, one to a wave, and 512 columns, looks
// through all ids for them, and writes its rows once, sums and zeros. Its waves look through a part
// of the ids each; what they find, one list after the other, is in the order of the tokens.
constexpr uint32_t kOwnWaves = 16, kOwnMost = 2048;
constexpr uint32_t kTokensMost = 1024;
constexpr uint32_t kOwnAlone = 8;   // tokens of a row that its wave adds up alone

struct Owned {
    MxIds ids;
    uint32_t n, rows, cols, tiles;
    MxRows dy;
    float scale;
    Out out;
};

template <uint32_t T, uint32_t OT>
__global__ __launch_bounds__(64 * kOwnWaves, 8) void owned_kernel(Owned g)
{
    constexpr int B = T == kFp32 ? 4 : 8;   // rows on their way at once
    __shared__ uint16_t found[kOwnMost];     // a row of this workgroup's << 11 | the token
    __shared__ uint16_t some[kOwnWaves][kOwnAlone], many[kOwnMost];   // tokens of a wave's row; of one of more
    __shared__ uint32_t count[kOwnWaves], total[kOwnWaves];
    __shared__ float part[kOwnWaves - 1][512];
    const uint32_t t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t own = blockIdx.x / g.tiles, c = (blockIdx.x - own * g.tiles) * 512 + lane * 8, r0 = own * kOwnWaves;
    const uint32_t rows = min(kOwnWaves, g.rows - r0);
    auto before = [&](uint64_t lanes) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0)); };
    // 64 or 128 ids to a wave.
    const uint32_t halves = g.n > 64 * kOwnWaves ? 2 : 1;
    uint32_t entry[2];
    uint64_t in[2];
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h) {
        const uint32_t at = (wave * halves + h) * 64 + lane;
        const int64_t r = h < halves && at < g.n ? id_of(g.ids, at) - (int64_t)r0 : -1;
        in[h] = __ballot(r >= 0 && r < (int64_t)rows);
        entry[h] = (uint32_t)r << 11 | at;
    }
    const uint32_t n0 = (uint32_t)__popcll(in[0]);
    if (lane == 0)
        count[wave] = n0 + (uint32_t)__popcll(in[1]);
    __syncthreads();
    uint32_t at = 0, all = 0;   // what the waves before found, and all of them
#pragma unroll
    for (uint32_t w = 0; w < kOwnWaves; ++w) {
        at += w < wave ? count[w] : 0;
        all += count[w];
    }
    if (in[0] >> lane & 1)
        found[at + before(in[0])] = (uint16_t)entry[0];
    if (in[1] >> lane & 1)
        found[at + n0 + before(in[1])] = (uint16_t)entry[1];
    __syncthreads();
    // The first `most` tokens of row r into a list; how many there are.
    auto gather = [&](uint32_t r, uint16_t *list, uint32_t most) {
        uint32_t m = 0;
        for (uint32_t i = 0; i < all; i += 64) {
            const uint32_t f = i + lane < all ? found[i + lane] : 0;
            const uint64_t lanes = __ballot(i + lane < all && f >> 11 == r);
            const uint32_t to = m + before(lanes);
            if ((lanes >> lane & 1) && to < most)
                list[to] = (uint16_t)(f & 2047);
            m += (uint32_t)__popcll(lanes);
        }
        wave_fence();
        return m;
    };
    auto add = [&](const uint16_t *list, uint32_t from, uint32_t to, float (&sum)[8]) {
        for (uint32_t i = from; i < to; i += B) {
            Raw8<T> raw[B];
#pragma unroll
            for (int j = 0; j < B; ++j)
                if (i + j < to)
                    raw[j].load(g.dy.p, list[i + j] * g.dy.ld, c, g.cols);
#pragma unroll
            for (int j = 0; j < B; ++j)
                if (i + j < to) {
                    raw[j].settle(c, g.cols);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        sum[e] += (float)raw[j].v[e];
                }
        }
    };
    uint32_t m = 0;
    if (wave < rows) {
        m = gather(wave, some[wave], kOwnAlone);
        if (lane == 0)
            total[wave] = m;
        if (c < g.cols && m <= kOwnAlone && (m || !g.out.accumulate)) {
            float sum[8] = {};
            add(some[wave], 0, m, sum);
            put_row<OT>(g.out, r0 + wave, c, g.cols, sum, g.scale);
        }
    }
    if (all <= kOwnAlone)   // (the whole workgroup)
        return;
    __syncthreads();
    for (uint32_t r = 0; r < rows; ++r) {   // rows of many tokens: a part of them to each wave
        const uint32_t m = total[r], per = (m + kOwnWaves - 1) / kOwnWaves;
        if (m <= kOwnAlone)
            continue;
        if (wave == 0)
            gather(r, many, kOwnMost);
        __syncthreads();
        float sum[8] = {};
        if (c < g.cols)
            add(many, min(m, wave * per), min(m, (wave + 1) * per), sum);
        if (wave)
            store8<kFp32>(part[wave - 1], 0, lane * 8, 512, sum);
        __syncthreads();
        if (wave == 0 && c < g.cols) {
#pragma unroll
            for (uint32_t w = 0; w < kOwnWaves - 1; ++w)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    sum[e] += part[w][lane * 8 + e];
            put_row<OT>(g.out, r0 + r, c, g.cols, sum, g.scale);
        }
        __syncthreads();
    }
}

// Few tokens of a large table: no sorting either. A workgroup has one token and 512 columns, and looks for
// the token's id in all of them, a quarter to each wave. The first token of an id adds up all of
// them, each wave those that it found, and their sums are added in the order of the waves: in that
// of the tokens.
template <uint32_t T, uint32_t OT>
__global__ __launch_bounds__(256) void tokens_kernel(Owned g)
{
    constexpr int B = T == kFp32 ? 8 : 16;   // rows on their way at once
    constexpr uint32_t K = kTokensMost / 256;
    __shared__ uint16_t list[4][64 * K];
    __shared__ uint32_t count[4], before[4];
    __shared__ float part[3][512];
    const uint32_t t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t token = blockIdx.x / g.tiles, c = (blockIdx.x - token * g.tiles) * 512 + lane * 8;
    const int64_t id = id_of(g.ids, token);
    if (id < 0 || id >= (int64_t)g.rows)   // the whole workgroup
        return;
    const uint32_t per = (g.n + 255) / 256 * 64;
    int64_t ids[K];
#pragma unroll
    for (uint32_t k = 0; k < K; ++k) {
        const uint32_t at = wave * per + k * 64 + lane;
        ids[k] = k * 64 < per && at < g.n ? id_of(g.ids, at) : -1;
    }
    uint32_t m = 0;
    bool early = false;
#pragma unroll
    for (uint32_t k = 0; k < K; ++k) {
        const uint32_t at = wave * per + k * 64 + lane;
        const bool same = ids[k] == id;
        const uint64_t lanes = __ballot(same);
        if (same)
            list[wave][m + __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0))] = (uint16_t)at;
        early |= same && at < token;
        m += (uint32_t)__popcll(lanes);
    }
    if (lane == 0)
        count[wave] = m;
    early = __ballot(early) != 0;
    if (lane == 0)
        before[wave] = early;
    __syncthreads();
    if (before[0] | before[1] | before[2] | before[3])   // another one's
        return;
    float sum[8] = {};
    if (c < g.cols)
        for (uint32_t i = 0; i < m; i += B) {
            Raw8<T> raw[B];
#pragma unroll
            for (int j = 0; j < B; ++j)
                if (i + j < m)
                    raw[j].load(g.dy.p, list[wave][i + j] * g.dy.ld, c, g.cols, true);
#pragma unroll
            for (int j = 0; j < B; ++j)
                if (i + j < m) {
                    raw[j].settle(c, g.cols);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        sum[e] += (float)raw[j].v[e];
                }
        }
    if (wave && m)
        store8<kFp32>(part[wave - 1], 0, lane * 8, 512, sum);
    __syncthreads();
    if (wave || c >= g.cols)
        return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
        if (count[w + 1])
#pragma unroll
            for (int e = 0; e < 8; ++e)
                sum[e] += part[w][lane * 8 + e];
    put_row<OT>(g.out, (uint64_t)id, c, g.cols, sum, g.scale);
}

// The sums of kChunk sorted tokens, 8 columns to a lane, a wave to a workgroup. All of the tokens' rows
// are on their way before the first is added, past the caches, which hold zeros that are still to be
// written (16384 tokens of 4096 after 1 GiB of zeros: 53 us, kept in them 80, of which the zeros then
// take 17 less). A sum that lies in the chunk whole is put out; one
// that goes on from the chunk before is left in part 0, one that begins here and goes on in part 1.
template <uint32_t T, uint32_t OT>
__global__ __launch_bounds__(64) void sums_kernel(Sums g)
{
    const uint32_t chunk = blockIdx.x / g.tiles, lane = threadIdx.x, c = (blockIdx.x - chunk * g.tiles) * kTileCols + lane * 8;
    const uint32_t begin = chunk * kChunk, count = min(kChunk, g.n - begin);
    // Lane i + 1 holds the key of the chunk's token i: the one before it and the one after it too.
    const uint32_t at = begin + lane - 1;
    const uint32_t key = lane <= kChunk + 1 && begin + lane > 0 && at < g.n ? g.keys[at] : ~0u;
    const uint32_t place = lane < count ? g.places[begin + lane] : 0;
    uint32_t keys[kChunk + 2], places[kChunk];   // (read from all lanes, before any of them leaves)
#pragma unroll
    for (int i = 0; i < (int)kChunk + 2; ++i)
        keys[i] = (uint32_t)__builtin_amdgcn_readlane((int)key, i);
#pragma unroll
    for (int i = 0; i < (int)kChunk; ++i)
        places[i] = (uint32_t)__builtin_amdgcn_readlane((int)place, i);
    auto key_at = [&](int i) { return keys[i + 1]; };
    Raw8<T> raw[kChunk];
    if (c < g.cols)
#pragma unroll
        for (int i = 0; i < (int)kChunk; ++i)
            if (i < (int)count && key_at(i) < g.rows)
                raw[i].load(g.dy.p, places[i] * g.dy.ld, c, g.cols, true);
    if (c >= g.cols)
        return;
    float sum[8] = {};
    bool here = key_at(-1) != key_at(0);   // whether the running sum began in this chunk
#pragma unroll
    for (int i = 0; i < (int)kChunk; ++i) {
        if (i < (int)count && key_at(i) < g.rows) {   // (ids that name no row are sorted last)
            raw[i].settle(c, g.cols);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                sum[e] += (float)raw[i].v[e];
            const bool last = key_at(i + 1) != key_at(i);
            if (last && here)
                put_row<OT>(g.out, key_at(i), c, g.cols, sum, g.scale);
            else if (last || i + 1 == (int)kChunk)
                store8<kFp32>(g.parts, ((uint64_t)chunk * 2 + here) * g.part_ld, c, g.part_ld, sum);
            if (last) {
                here = true;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    sum[e] = 0.0f;
            }
        }
    }
}

// The sums that go on from the chunk in which they began: its part 1, and part 0 of those after.
template <uint32_t OT>
__global__ __launch_bounds__(64) void join_sums_kernel(Sums g)
{
    const uint32_t chunk = blockIdx.x / g.tiles, c = (blockIdx.x - chunk * g.tiles) * kTileCols + threadIdx.x * 8;
    const uint32_t begin = chunk * kChunk, end = begin + kChunk;
    if (end >= g.n)
        return;
    const uint32_t key = g.keys[end - 1];
    if (key >= g.rows || g.keys[end] != key)
        return;
    if (begin != 0 && g.keys[begin - 1] == key)
        return;   // it began before
    // The chunks that it reaches into: 64 looked at at once.
    uint32_t last = chunk;
    for (;;) {
        const uint64_t k = (uint64_t)last + 1 + threadIdx.x;
        const uint32_t more = (uint32_t)__builtin_ctzll(~__ballot(k < g.chunks && g.keys[k * kChunk] == key) | 1ull << 63);
        const bool all = more == 63 && last + 64 < g.chunks && g.keys[(uint64_t)(last + 64) * kChunk] == key;
        last += all ? 64 : more;
        if (!all)
            break;
    }
    if (c >= g.cols)
        return;
    float sum[8];
    load8<kFp32>(g.parts, ((uint64_t)chunk * 2 + 1) * g.part_ld, c, g.part_ld, sum);
    uint32_t k = chunk + 1;
    for (; k + 8 <= last + 1; k += 8) {   // 8 on their way at once, added in their order
        float v[8][8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            load8<kFp32>(g.parts, (uint64_t)(k + i) * 2 * g.part_ld, c, g.part_ld, v[i]);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                sum[e] += v[i][e];
    }
    for (; k <= last; ++k) {
        float v[8];
        load8<kFp32>(g.parts, (uint64_t)k * 2 * g.part_ld, c, g.part_ld, v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sum[e] += v[e];
    }
    put_row<OT>(g.out, key, c, g.cols, sum, g.scale);
}

}  // namespace mx

using namespace mx;

hipError_t launch_mx_embedding(const Embedding &e, hipStream_t s)
{
    if (e.m == 0 || e.cols == 0)
        return hipSuccess;
    Lookup g = {};
    g.ids = e.ids;
    g.table = e.table;
    g.rows = (uint32_t)e.rows;
    g.cols = (uint32_t)e.cols;
    g.nb = (uint32_t)mx_blocks(e.cols);
    g.recip = div_recip_of(g.nb);
    g.scale = e.scale;
    g.y = e.y;
    const uint64_t most = 0xFFFFFF00u / g.nb;
    for (g.t0 = 0; g.t0 < e.m; g.t0 += most) {
        g.blocks = (uint32_t)((e.m - g.t0 < most ? e.m - g.t0 : most) * g.nb);
        MX_TYPE(e.type, hipLaunchKernelGGL((lookup_kernel<T>), dim3((g.blocks + kThreads - 1) / kThreads), dim3(kThreads), 0, s, g));
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess)
            return err;
    }
    return hipSuccess;
}

namespace {

uint64_t round16(uint64_t v) { return (v + 15) / 16 * 16; }

struct GradPlan {
    bool small;            // one workgroup sorts
    uint32_t bits, passes, blocks, chunks;
    uint64_t keys, counts, parts;   // bytes of one array of keys, of the counts, of the parts
    uint64_t bytes() const { return (small ? 2 : 4) * keys + counts + parts; }
};

GradPlan plan_of(uint64_t m, uint64_t rows, uint64_t cols)
{
    GradPlan p = {};
    uint32_t bits = 1;
    while (rows >> bits)
        ++bits;
    p.passes = (bits + kDigitBits - 1) / kDigitBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.small = m <= kSortBlock;
    p.blocks = (uint32_t)((m + kSortBlock - 1) / kSortBlock);
    p.chunks = (uint32_t)((m + kChunk - 1) / kChunk);
    p.keys = round16(m * 4);
    p.counts = p.small ? 0 : round16(((uint64_t)p.blocks << p.bits) * 4);
    p.parts = p.chunks > 1 ? (uint64_t)p.chunks * 2 * ((cols + 7) / 8 * 8) * 4 : 0;
    return p;
}

enum Unsorted : int { kSorted, kOwned, kTokens };

// How few tokens' gradient goes without sorting. By the table's rows, where no row has many tokens on average
// and few workgroups have to look through the ids. (us sorted, owned, bf16: 1001 tokens, 5003 x 1111: 22.6, 13.7; 2048
// tokens, 5003 x 1111: 28.9, 18.4; 1 token, 32768 x 512, 2048 workgroups: 13.6, 17.4; 1001 tokens, 20000 x 1024, 2500
// workgroups: 23.0, 23.6; 500 and 2048 tokens, 100 x 4096: 14.1, 11.2 and 17.4, 31.7.) By the tokens, where the table is
// large and no launch of theirs is. (us sorted, by tokens: 87 tokens, 25917 x 615: 27.4, 16.9; 204 tokens, 11520 x 8192:
// 75.9, 64.6; 1001 tokens, 20000 x 1024 23.7, 19.4, 32768 x 4096, 8008 workgroups, 102.3, 102.2; 2048 tokens, 32768 x 1024:
// 30.6, 33.9.)
Unsorted unsorted(uint64_t m, uint64_t rows, uint64_t cols)
{
    const uint64_t tiles = (cols + 511) / 512;
    if (m == 0 || m > kOwnMost || m > 8 * rows)
        return kSorted;
    if ((rows + kOwnWaves - 1) / kOwnWaves * tiles <= 1536)
        return kOwned;
    return m <= kTokensMost && m * tiles <= 8192 ? kTokens : kSorted;
}

}  // namespace

uint64_t mx_embedding_grad_work(uint64_t m, uint64_t rows, uint64_t cols)
{
    return m && rows && cols && unsorted(m, rows, cols) == kSorted ? plan_of(m, rows, cols).bytes() : 0;
}

hipError_t launch_mx_embedding_grad(const EmbeddingGrad &e, hipStream_t s)
{
    if (e.rows == 0 || e.cols == 0)
        return hipSuccess;
    hipError_t err;
    const uint64_t size = mx_type_size(e.otype);
    const bool whole = e.dw.ld == e.cols || e.rows == 1;
    const Unsorted way = unsorted(e.m, e.rows, e.cols);
    // Zeros by workgroups of so many threads, 16 bytes to each.
    auto zeros = [&](uint32_t threads) {
        Zero z = {reinterpret_cast<uint8_t *>(e.dw.p), e.dw.ld * size, (whole ? e.rows : 1) * e.cols * size, whole ? 1 : e.rows, 0};
        const uint64_t parts = whole ? (z.width + threads * 16 - 1) / (threads * 16) : (z.rows + threads / 64 - 1) / (threads / 64);
        const uint64_t most = 0xFFFFFF00u / threads - 1;   // (a launch has fewer than 2^32 threads)
        z.parts = (uint32_t)(parts < most ? parts : most);
        return z;
    };
    if (way != kSorted) {
        if (way == kTokens && !e.accumulate) {
            const Zero z = zeros(256);
            hipLaunchKernelGGL(zero_kernel, dim3(z.parts), dim3(256), 0, s, z);
            if ((err = hipGetLastError()) != hipSuccess)
                return err;
        }
        Owned g = {};
        g.ids = e.ids;
        g.n = (uint32_t)e.m;
        g.rows = (uint32_t)e.rows;
        g.cols = (uint32_t)e.cols;
        g.tiles = (uint32_t)((e.cols + 511) / 512);
        g.dy = e.dy;
        g.scale = e.scale;
        g.out = {e.dw.p, e.dw.ld, e.otype, e.accumulate, nullptr};
        const dim3 grid((way == kOwned ? (uint32_t)((e.rows + kOwnWaves - 1) / kOwnWaves) : g.n) * g.tiles);
        MX_TYPE(e.type, {
            constexpr uint32_t D = T;
            MX_TYPE(e.otype, {
                if (way == kOwned)
                    hipLaunchKernelGGL((owned_kernel<D, T>), grid, dim3(64 * kOwnWaves), 0, s, g);
                else
                    hipLaunchKernelGGL((tokens_kernel<D, T>), grid, dim3(256), 0, s, g);
            });
        });
        return hipGetLastError();
    }
    Zero z = {};
    if (!e.accumulate)
        z = zeros(kSortThreads);
    if (e.m == 0) {
        if (!z.parts)
            return hipSuccess;
        hipLaunchKernelGGL(sums_before_kernel, dim3(1 + z.parts), dim3(1024), 0, s, nullptr, 0, z);
        return hipGetLastError();
    }
    const GradPlan p = plan_of(e.m, e.rows, e.cols);
    uint8_t *at = reinterpret_cast<uint8_t *>(e.work);
    uint32_t *keys[2], *places[2];
    for (int i = 0; i < (p.small ? 1 : 2); ++i) {
        keys[i] = reinterpret_cast<uint32_t *>(at);
        places[i] = reinterpret_cast<uint32_t *>(at + p.keys);
        at += 2 * p.keys;
    }
    int in = 0;
    if (p.small) {
        const SortSmall g = {e.ids, keys[0], places[0], (uint32_t)e.m, (uint32_t)e.rows, p.bits, p.passes};
        const dim3 grid(1 + z.parts);
        if (e.m <= kSortThreads)
            hipLaunchKernelGGL((sort_small_kernel<1>), grid, dim3(kSortThreads), 0, s, g, z);
        else if (e.m <= 4 * kSortThreads)
            hipLaunchKernelGGL((sort_small_kernel<4>), grid, dim3(kSortThreads), 0, s, g, z);
        else
            hipLaunchKernelGGL((sort_small_kernel<kMostItems>), grid, dim3(kSortThreads), 0, s, g, z);
        if ((err = hipGetLastError()) != hipSuccess)
            return err;
    } else {
        Sort g = {};
        g.ids = e.ids;
        g.n = (uint32_t)e.m;
        g.rows = (uint32_t)e.rows;
        g.bits = p.bits;
        g.blocks = p.blocks;
        g.counts = reinterpret_cast<uint32_t *>(at);
        for (uint32_t pass = 0; pass < p.passes; ++pass, in ^= 1) {
            g.first = pass == 0;
            g.shift = pass * p.bits;
            g.keys = keys[in];
            g.places = places[in];
            g.keys_out = keys[in ^ 1];
            g.places_out = places[in ^ 1];
            hipLaunchKernelGGL((sort_pass_kernel<false>), dim3(p.blocks), dim3(kSortThreads), 0, s, g);
            if ((err = hipGetLastError()) != hipSuccess)
                return err;
            const uint32_t zeros = pass == 0 ? z.parts : 0;
            hipLaunchKernelGGL(sums_before_kernel, dim3(1 + zeros), dim3(1024), 0, s, g.counts, p.blocks << p.bits, z);
            if ((err = hipGetLastError()) != hipSuccess)
                return err;
            hipLaunchKernelGGL((sort_pass_kernel<true>), dim3(p.blocks), dim3(kSortThreads), 0, s, g);
            if ((err = hipGetLastError()) != hipSuccess)
                return err;
        }
    }
    at += p.counts;
    Sums g = {};
    g.keys = keys[in];
    g.places = places[in];
    g.n = (uint32_t)e.m;
    g.rows = (uint32_t)e.rows;
    g.cols = (uint32_t)e.cols;
    g.chunks = p.chunks;
    g.tiles = (uint32_t)((e.cols + kTileCols - 1) / kTileCols);
    g.dy = e.dy;
    g.scale = e.scale;
    g.out = {e.dw.p, e.dw.ld, e.otype, e.accumulate, nullptr};
    g.parts = reinterpret_cast<float *>(at);
    g.part_ld = (uint32_t)((e.cols + 7) / 8 * 8);
    const dim3 grid(g.chunks * g.tiles);
    MX_TYPE(e.type, {
        constexpr uint32_t D = T;
        MX_TYPE(e.otype, hipLaunchKernelGGL((sums_kernel<D, T>), grid, dim3(64), 0, s, g));
    });
    if ((err = hipGetLastError()) != hipSuccess || g.chunks == 1)
        return err;
    MX_TYPE(e.otype, hipLaunchKernelGGL((join_sums_kernel<T>), grid, dim3(64), 0, s, g));
    return hipGetLastError();
}

}  // namespace fastrack
