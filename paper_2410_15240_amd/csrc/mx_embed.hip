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

__device__ __forceinline__ int64_t id_of(const MxIds &ids, uint64_t i)
{
    return ids.wide ? reinterpret_cast<const int64_t *>(ids.p)[i] : reinterpret_cast<const int32_t *>(ids.p)[i];
}

// ---- lookup ---------------------------------------------------------------------------------
//
// A unit of 8 values to a thread, as in mx.hip. What bounds it is the writing of y.
constexpr int kThreads = 256;

struct Lookup {
    MxIds ids;
    MxMatrix table;
    uint32_t rows, cols, per_row, recip, units;
    uint64_t t0;   // first token of this launch
    float scale;
    MxRows y;
};

template <uint32_t T>
__global__ __launch_bounds__(kThreads) void lookup_kernel(Lookup g)
{
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= g.units)
        return;
    const uint32_t r = div_recip(i, g.per_row, g.recip), j = i - r * g.per_row;
    const uint64_t t = g.t0 + r;
    const int64_t id = id_of(g.ids, t);
    float v[8];
    if (id >= 0 && id < (int64_t)g.rows) {
        const uint64_t block = (uint64_t)id * ((g.per_row + 3) / 4) + j / 4;
        decode4_f32(reinterpret_cast<const uint32_t *>(g.table.codes)[block * 4 + j % 4], scale4_f32(g.table.scales[block]), v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] *= g.scale;
    } else {   // padding; no row of the table
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = id < 0 ? 0.0f : __builtin_nanf("");
    }
    store8<T>(g.y.p, t * g.y.ld, j * 8, g.cols, v);
}

// ---- sorting ids -------------------------------------------------------------------------------
//
// Keys below 2^bits (the number of rows itself for ids that count for none), each with its place,
// sorted by key and then by place: passes over a digit each, the lowest first. In a pass a
// wave ranks its 64 keys among equal digits by one vote per bit, and adds what came before
// them: in its own earlier keys, in the waves before it, and in the blocks before.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr uint32_t kDigits = 256;

struct Sort {
    MxIds ids;                    // of the first pass; later ones read keys and places
    const uint32_t *keys, *places;
    uint32_t *keys_out, *places_out;
    uint32_t n, rows, shift, bits, blocks;
    uint32_t *counts;             // [1 << bits][blocks], then the sums before each
    bool first;
};

constexpr int kItems = 16;        // keys of a thread
constexpr uint32_t kSortBlock = kSortThreads * kItems;

__device__ __forceinline__ uint32_t key_of(const MxIds &ids, uint32_t i, uint32_t rows)
{
    const int64_t id = id_of(ids, i);
    return id >= 0 && id < (int64_t)rows ? (uint32_t)id : rows;
}

// A wave's keys are 64 * kItems that follow one another, 64 at a time. `counts[digit]` of the wave
// grows; rank[] is a key's number among the wave's equal digits.
__device__ __forceinline__ void rank_keys(const uint32_t (&key)[kItems], uint32_t (&rank)[kItems], uint32_t valid, uint32_t shift,
                                          uint32_t bits, uint32_t *counts)
{
    const uint32_t lane = threadIdx.x & 63, mask = (1u << bits) - 1;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        if (i * 64u >= valid)   // the whole wave
            break;
        const bool in = i * 64u + lane < valid;
        const uint32_t d = key[i] >> shift & mask;
        uint64_t same = __ballot(in);
        for (uint32_t b = 0; b < bits; ++b) {
            const uint64_t v = __ballot(d >> b & 1);
            same &= d >> b & 1 ? v : ~v;
        }
        if (in) {
            rank[i] = counts[d] + (uint32_t)__popcll(same & ((1ull << lane) - 1));
            if (lane == (uint32_t)(63 - __clzll((long long)same)))   // the last of them
                counts[d] = rank[i] + 1;
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
    }
}

// counts[wave][digit] of a workgroup to where each wave's first key of a digit goes among the
// workgroup's; total[digit] of thread `digit` is returned. Threads past the digits bring 0.
__device__ __forceinline__ uint32_t digits_before(uint32_t (*counts)[kDigits], uint32_t *sums, uint32_t &before)
{
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6;
    uint32_t total = 0;
    if (t < kDigits) {
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

// All passes by one workgroup, up to kSortBlock ids. Keys and places go from pass to pass through
// LDS.
struct SortSmall {
    MxIds ids;
    uint32_t *keys_out, *places_out;
    uint32_t n, rows, bits, passes;   // bits of a digit
};

struct SortLds {
    uint32_t key[kSortBlock];
    uint16_t place[kSortBlock];
    uint32_t counts[kSortWaves][kDigits];
    uint32_t base[kDigits];
    uint32_t sums[kDigits / 64];
};

__device__ __forceinline__ void sort_small(const SortSmall &g, SortLds &l)
{
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const uint32_t per = (g.n + kSortThreads - 1) / kSortThreads * 64, w0 = wave * per;   // keys of a wave
    const uint32_t valid = w0 < g.n ? min(per, g.n - w0) : 0;
    uint32_t key[kItems], place[kItems], rank[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const uint32_t at = i * 64 + lane;
        place[i] = w0 + at;
        key[i] = at < valid ? key_of(g.ids, w0 + at, g.rows) : 0;
    }
    for (uint32_t p = 0; p < g.passes; ++p) {
        const uint32_t shift = p * g.bits, mask = (1u << g.bits) - 1;
        for (uint32_t i = t; i < kSortWaves * kDigits; i += kSortThreads)
            (&l.counts[0][0])[i] = 0;
        __syncthreads();
        rank_keys(key, rank, valid, shift, g.bits, l.counts[wave]);
        __syncthreads();
        uint32_t before;
        digits_before(l.counts, l.sums, before);
        if (t < kDigits)
            l.base[t] = before;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kItems; ++i)
            if (i * 64 + lane < valid) {
                const uint32_t d = key[i] >> shift & mask, to = l.base[d] + l.counts[wave][d] + rank[i];
                if (p + 1 < g.passes) {
                    l.key[to] = key[i];
                    l.place[to] = (uint16_t)place[i];
                } else {
                    g.keys_out[to] = key[i];
                    g.places_out[to] = place[i];
                }
            }
        __syncthreads();
        if (p + 1 < g.passes) {
#pragma unroll
            for (int i = 0; i < kItems; ++i)
                if (i * 64 + lane < valid) {
                    key[i] = l.key[w0 + i * 64 + lane];
                    place[i] = l.place[w0 + i * 64 + lane];
                }
        }
    }
}

// A pass of many workgroups: the digits of each block counted, the counts added up (digit by
// digit, block by block), the keys put where they go.
__device__ __forceinline__ void load_keys(const Sort &g, uint32_t w0, uint32_t valid, uint32_t (&key)[kItems])
{
    const uint32_t lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
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
    const uint64_t first = (uint64_t)blockIdx.x * kSortBlock + wave * (64 * kItems);
    const uint32_t w0 = (uint32_t)first, valid = first < g.n ? min(64u * kItems, g.n - w0) : 0;
    uint32_t key[kItems], rank[kItems];
    load_keys(g, w0, valid, key);
    for (uint32_t i = t; i < kSortWaves * kDigits; i += kSortThreads)
        (&counts[0][0])[i] = 0;
    __syncthreads();
    rank_keys(key, rank, valid, g.shift, g.bits, counts[wave]);
    __syncthreads();
    uint32_t before;
    const uint32_t total = digits_before(counts, sums, before);
    if (!PUT) {
        if (t <= mask)
            g.counts[(uint64_t)t * g.blocks + blockIdx.x] = total;
        return;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; ++i)
        if (i * 64 + lane < valid) {
            const uint32_t d = key[i] >> g.shift & mask;
            const uint32_t to = g.counts[(uint64_t)d * g.blocks + blockIdx.x] + counts[wave][d] + rank[i];
            g.keys_out[to] = key[i];
            g.places_out[to] = g.first ? w0 + i * 64 + lane : g.places[w0 + i * 64 + lane];
        }
}

// Each count becomes the sum of those before it; one workgroup.
__global__ __launch_bounds__(1024) void sums_before_kernel(uint32_t *counts, uint32_t n)
{
    __shared__ uint32_t sums[16];
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
    uint32_t type;
    MxRows dy;
    float scale;
    Out out;
    float *parts;                    // [chunks][2][cols]
};

constexpr uint32_t kChunk = 32, kSumThreads = 256, kTileCols = kSumThreads * 8;

__device__ __forceinline__ void put_row(const Out &o, uint64_t row, uint32_t c, uint32_t cols, float (&v)[8], float scale)
{
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] *= scale;
    const uint64_t at = row * o.ld;
    if (o.type == kFp32) {
        if (o.accumulate) {
            float w[8];
            load8<kFp32>(o.p, at, c, cols, w);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] += w[e];
        }
        store8<kFp32>(o.p, at, c, cols, v);
    } else if (o.type == kBf16) {
        store8<kBf16>(o.p, at, c, cols, v);
    } else {
        store8<kFp16>(o.p, at, c, cols, v);
    }
}

// The sums of kChunk sorted tokens, 8 columns to a thread. A sum that lies in the chunk whole is
// put out; one that goes on from the chunk before is left in part 0, one that begins here and
// goes on in part 1.
template <uint32_t T>
__global__ __launch_bounds__(kSumThreads) void sums_kernel(Sums g)
{
    const uint32_t chunk = blockIdx.x / g.tiles, c = (blockIdx.x - chunk * g.tiles) * kTileCols + threadIdx.x * 8;
    const uint32_t begin = chunk * kChunk, end = min(g.n, begin + kChunk);
    if (c >= g.cols)
        return;
    float sum[8] = {};
    bool here = begin == 0 || g.keys[begin] != g.keys[begin - 1];   // whether the running sum began in this chunk
    for (uint32_t i = begin; i < end; ++i) {
        const uint32_t key = g.keys[i];
        if (key >= g.rows)   // sorted last: no row's
            return;
        float v[8];
        load8<T>(g.dy.p, g.places[i] * g.dy.ld, c, g.cols, v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sum[e] += v[e];
        const bool last = i + 1 == g.n || g.keys[i + 1] != key;
        if (last && here)
            put_row(g.out, key, c, g.cols, sum, g.scale);
        else if (last || i + 1 == end)
            store8<kFp32>(g.parts, ((uint64_t)chunk * 2 + here) * g.cols, c, g.cols, sum);
        if (last) {
            here = true;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                sum[e] = 0.0f;
        }
    }
}

// The sums that go on from the chunk in which they began: its part 1, and part 0 of those after.
__global__ __launch_bounds__(kSumThreads) void join_sums_kernel(Sums g)
{
    const uint32_t chunk = blockIdx.x / g.tiles, c = (blockIdx.x - chunk * g.tiles) * kTileCols + threadIdx.x * 8;
    const uint32_t begin = chunk * kChunk, end = begin + kChunk;
    if (c >= g.cols || end >= g.n)
        return;
    const uint32_t key = g.keys[end - 1];
    if (key >= g.rows || g.keys[end] != key)
        return;
    if (g.keys[begin] == key && begin != 0 && g.keys[begin - 1] == key)
        return;   // it began before
    float sum[8], v[8];
    load8<kFp32>(g.parts, ((uint64_t)chunk * 2 + 1) * g.cols, c, g.cols, sum);
    for (uint32_t k = chunk + 1; k < g.chunks && g.keys[k * kChunk] == key; ++k) {
        load8<kFp32>(g.parts, (uint64_t)k * 2 * g.cols, c, g.cols, v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sum[e] += v[e];
    }
    put_row(g.out, key, c, g.cols, sum, g.scale);
}

// Zeros, 16 bytes to a thread and a step, in rows of `width` bytes.
__global__ __launch_bounds__(kThreads) void zero_kernel(uint8_t *p, uint64_t stride, uint64_t width, uint64_t rows)
{
    if (stride == width || rows == 1) {
        width *= rows;
        rows = 1;
    }
    for (uint64_t r = blockIdx.y; r < rows; r += gridDim.y) {
        uint8_t *row = p + r * stride;
        for (uint64_t at = (uint64_t)(blockIdx.x * kThreads + threadIdx.x) * 16; at < width; at += (uint64_t)gridDim.x * kThreads * 16) {
            if (at + 16 <= width) {
                const u32x4 zero = {0, 0, 0, 0};
                __builtin_memcpy(row + at, &zero, 16);
            } else {
                for (uint64_t b = at; b < width; b += 2)
                    *reinterpret_cast<uint16_t *>(row + b) = 0;
            }
        }
    }
}

__global__ __launch_bounds__(kSortThreads) void sort_small_kernel(SortSmall g)
{
    __shared__ SortLds l;
    sort_small(g, l);
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
    g.per_row = (uint32_t)((e.cols + 7) / 8);
    g.recip = div_recip_of(g.per_row);
    g.scale = e.scale;
    g.y = e.y;
    const uint64_t most = 0xFFFFFF00u / g.per_row;
    for (g.t0 = 0; g.t0 < e.m; g.t0 += most) {
        g.units = (uint32_t)((e.m - g.t0 < most ? e.m - g.t0 : most) * g.per_row);
        MX_TYPE(e.type, hipLaunchKernelGGL((lookup_kernel<T>), dim3((g.units + kThreads - 1) / kThreads), dim3(kThreads), 0, s, g));
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
    p.passes = (bits + 7) / 8;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.small = m <= kSortBlock;
    p.blocks = (uint32_t)((m + kSortBlock - 1) / kSortBlock);
    p.chunks = (uint32_t)((m + kChunk - 1) / kChunk);
    p.keys = round16(m * 4);
    p.counts = p.small ? 0 : round16(((uint64_t)p.blocks << p.bits) * 4);
    p.parts = p.chunks > 1 ? (uint64_t)p.chunks * 2 * cols * 4 : 0;
    return p;
}

}  // namespace

uint64_t mx_embedding_grad_work(uint64_t m, uint64_t rows, uint64_t cols)
{
    return m && rows && cols ? plan_of(m, rows, cols).bytes() : 0;
}

hipError_t launch_mx_embedding_grad(const EmbeddingGrad &e, int num_cu, hipStream_t s)
{
    if (e.rows == 0 || e.cols == 0)
        return hipSuccess;
    hipError_t err;
    if (!e.accumulate) {
        const uint64_t size = mx_type_size(e.otype), width = e.cols * size;
        const bool whole = e.dw.ld == e.cols || e.rows == 1;
        const uint64_t units = ((whole ? width * e.rows : width) + 16 * kThreads - 1) / (16 * kThreads);
        const uint32_t gx = (uint32_t)(units < 16u * num_cu ? units : 16u * num_cu), gy = whole ? 1 : (uint32_t)(e.rows < 8192 ? e.rows : 8192);
        hipLaunchKernelGGL(zero_kernel, dim3(gx, gy), dim3(kThreads), 0, s, reinterpret_cast<uint8_t *>(e.dw.p), e.dw.ld * size, width, e.rows);
        if ((err = hipGetLastError()) != hipSuccess)
            return err;
    }
    if (e.m == 0)
        return hipSuccess;
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
        hipLaunchKernelGGL(sort_small_kernel, dim3(1), dim3(kSortThreads), 0, s, g);
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
            hipLaunchKernelGGL(sums_before_kernel, dim3(1), dim3(1024), 0, s, g.counts, p.blocks << p.bits);
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
    g.out = {e.dw.p, e.dw.ld, e.otype, e.accumulate};
    g.parts = reinterpret_cast<float *>(at);
    const dim3 grid(g.chunks * g.tiles);
    MX_TYPE(e.type, hipLaunchKernelGGL((sums_kernel<T>), grid, dim3(kSumThreads), 0, s, g));
    if ((err = hipGetLastError()) != hipSuccess || g.chunks == 1)
        return err;
    hipLaunchKernelGGL(join_sums_kernel, grid, dim3(kSumThreads), 0, s, g);
    return hipGetLastError();
}

}  // namespace fastrack
