// Products with a microscaled operand where there are few outputs: one launch, no workspace
// for the float operand, every wave on its own.
//
// gemm_kernel (mx_gemm.hip) takes its time from the matrix unit only while tiles of 256 outputs
// a side fill the GPU. With fewer outputs the time is the latency of memory, of barriers and
// of launches. Here a workgroup has one small tile, its 8 waves each take every eighth piece of
// the sum without waiting for one another, and their results are added in LDS at the end, in
// the order of the waves.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mx.h"
#include "mx_dev.h"
#include "mx_gemm_dev.h"
#include "mx_small.h"

namespace fastrack {
namespace mx {

constexpr int kWaves = 8, kThreads = 64 * kWaves;

// The upper halves of eight floats: bf16 values cut, not rounded, so that what is left of each
// (left: v becomes it) has 8 significant bits less and the terms add up exactly.
__device__ __forceinline__ u32x4 upper_halves(const float (&v)[8])
{
    u32x4 h;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        h[i] = __builtin_amdgcn_perm(f32_bits(v[2 * i + 1]), f32_bits(v[2 * i]), 0x07060302u);
    return h;
}

__device__ __forceinline__ void leave_lower(float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] -= bits_f32(f32_bits(v[i]) & 0xFFFF0000u);
}

// The first term of values that have more, and what is left of them. An infinity goes into the
// first term whole (the subtraction alone would leave a NaN; of a NaN it leaves one rightly).
__device__ __forceinline__ u32x4 first_term(float (&v)[8])
{
    const u32x4 h = upper_halves(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float left = v[i] - bits_f32(f32_bits(v[i]) & 0xFFFF0000u);
        v[i] = __builtin_fabsf(v[i]) == __builtin_inff() ? 0.0f : left;
    }
    return h;
}

// Eight elements of a float operand as they lie in memory, and taken apart into bf16 terms.
template <uint32_t T> struct Unit8 {
    static constexpr int kTerms = T == kBf16 ? 1 : T == kFp16 ? 2 : 3;
    static constexpr int kWords = T == kFp32 ? 8 : 4, kSize = T == kFp32 ? 4 : 2;
    uint32_t w[kWords];

    // From any address of an element.
    __device__ __forceinline__ void load(const uint8_t *p)
    {
#pragma unroll
        for (int i = 0; i < kWords; i += 4) {
            u32x4 part;
            __builtin_memcpy(&part, p + 4 * i, 16);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w[i + j] = part[j];
        }
    }
    template <int N>
    __device__ __forceinline__ void move_words(bool yes)
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const uint32_t next = i + N < kWords ? w[(i + N) % kWords] : 0;
            w[i] = yes ? next : w[i];
        }
    }
    // The unit was read `by` elements before its place, because the row ends inside it: move them
    // down, zeros in at the top. 8 and more leave nothing.
    __device__ __forceinline__ void move_down(uint32_t by)
    {
        constexpr int kPer = 4 / kSize;   // elements to a word
        move_words<4 / kPer>(by & 4);
        move_words<2 / kPer>(by & 2);
        if (kPer == 1) {
            move_words<1>(by & 1);
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                const uint32_t next = i + 1 < kWords ? w[(i + 1) % kWords] : 0;
                w[i] = by & 1 ? w[i] >> 16 | next << 16 : w[i];
            }
        }
        keep(by < 8);
    }
    __device__ __forceinline__ void keep(bool yes)
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            w[i] = yes ? w[i] : 0;
    }
    __device__ __forceinline__ u32x4 bf16() const { return u32x4{w[0], w[1], w[2], w[3]}; }
    __device__ __forceinline__ void floats(float (&v)[8]) const
    {
        if (T == kFp32) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = bits_f32(w[i % kWords]);
        } else {
            typedef _Float16 h8 __attribute__((ext_vector_type(8)));
            const h8 h = __builtin_bit_cast(h8, bf16());
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = (float)h[i];
        }
    }
    // All terms at once.
    __device__ __forceinline__ void terms(u32x4 (&t)[kTerms]) const
    {
        if (T == kBf16) {
            t[0] = bf16();
            return;
        }
        float v[8];
        floats(v);
        t[0] = first_term(v);
        if (kTerms >= 2)
            t[kTerms >= 2 ? 1 : 0] = upper_halves(v);
        if (kTerms == 3) {
            leave_lower(v);
            t[kTerms - 1] = upper_halves(v);
        }
    }
};

// ---- one token, or up to 16 of them ---------------------------------------------------------
//
// y[m][n] = sum over k of x[m][k] w[n][k]. The weights are read once, 16 rows of them to a
// workgroup: lane l takes block l / 16 of every four of row l % 16, 16 bytes at once, and what
// it decodes is an operand of the 16 x 16 matrix instruction as it is (its lane holds 8
// consecutive values). x's values of the same places are the other operand; columns past m
// repeat the last token's. What bounds it is the reading of w: K / 2 + K / 32 bytes a row.
template <uint32_t T>
__global__ __launch_bounds__(kThreads, 4) void row_kernel(SmallProduct g)
{
    constexpr int NT = Unit8<T>::kTerms, U = T == kFp32 ? 2 : 4;   // chunks of 4 blocks read ahead
    __shared__ float part[kWaves][256];
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6, r = lane & 15, q = lane >> 4;
    const uint32_t n0 = blockIdx.x * 16;
    const uint64_t row = (uint64_t)min(n0 + r, g.n - 1) * g.nb;
    const u32x4 *codes = reinterpret_cast<const u32x4 *>(g.q.codes) + row;
    const uint8_t *scales = g.q.scales + row;
    constexpr uint32_t ES = Unit8<T>::kSize;
    const uint8_t *x = reinterpret_cast<const uint8_t *>(g.a.p) + min(r, g.m - 1) * g.a.ld * ES;
    const uint32_t chunks = (g.nb + 3) / 4, whole = g.k / 128;   // all of a chunk's values in the row

    f32x4 acc = {0, 0, 0, 0};
    u32x4 w[U];
    uint32_t e[U];
    Unit8<T> v[U][4];
    auto load = [&](int i, uint32_t c) {
        const uint32_t b = c * 4 + q;
        w[i] = codes[b];
        e[i] = scales[b];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[i][j].load(x + (uint64_t)(b * 32 + j * 8) * ES);
    };
    // The last chunk: a block past the end is 0, a unit that the row ends in is read from its end.
    auto load_last = [&](uint32_t c) {
        const uint32_t b = c * 4 + q;
        w[0] = codes[min(b, g.nb - 1)];
        e[0] = scales[min(b, g.nb - 1)];
        if (b >= g.nb) {
            w[0] = u32x4{0, 0, 0, 0};
            e[0] = 127;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t k = b * 32 + j * 8, from = min(k, g.k - 8);
            v[0][j].load(x + (uint64_t)from * ES);
            v[0][j].move_down(k - from);
        }
    };
    auto multiply = [&](int i) {
        const float s = scale4_f32(e[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bf16x8 d = __builtin_bit_cast(bf16x8, decode4_bf16(w[i][j], s));
            u32x4 terms[NT];
            v[i][j].terms(terms);
#pragma unroll
            for (int p = 0; p < NT; ++p)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(d, __builtin_bit_cast(bf16x8, terms[p]), acc, 0, 0, 0);
        }
    };
    uint32_t c = wave;
    for (; c + (U - 1) * kWaves < whole; c += U * kWaves) {
#pragma unroll
        for (int i = 0; i < U; ++i)
            load(i, c + i * kWaves);
        __builtin_amdgcn_sched_barrier(0);   // all of them on their way before the first is used
#pragma unroll
        for (int i = 0; i < U; ++i)
            multiply(i);
    }
    for (; c < chunks; c += kWaves) {
        if (c < whole)
            load(0, c);
        else
            load_last(c);
        multiply(0);
    }

    // Lane l holds token l % 16 of rows 4 (l / 16) + i.
#pragma unroll
    for (int i = 0; i < 4; ++i)
        part[wave][r * 16 + q * 4 + i] = acc[i];
    __syncthreads();
    if (t < 256) {
        const uint32_t m = t / 16, n = n0 + t % 16;
        float s = part[0][t];
#pragma unroll
        for (int i = 1; i < kWaves; ++i)
            s += part[i][t];
        if (m < g.m && n < g.n)
            put1(g.out, m, n, s);
    }
}

// ---- small tiles -----------------------------------------------------------------------------
//
// Tiles of 32 S x 32 S outputs. A wave has all of a tile's results and takes every eighth slice
// of 64 summed values of the workgroup's: it reads both operands (16 bytes of bf16 a lane),
// puts them into its own LDS as bf16 and reads the matrix instruction's operands back from
// there. Nothing waits for another wave. Terms of a 16 or 32-bit float go through the same
// bytes one after the other. The slice after is on its way from memory meanwhile. What bounds
// it is the issue of instructions: the splitting and decoding are repeated by every tile along
// the other axis.

// Place of chunk c (8 values) of row r: rows of 8 chunks as in at_k, rows of 4 with the chunks
// turned by bits 2 and 3 of the row, which again spreads 16 rows over all banks.
template <int CHUNKS>
__device__ __forceinline__ uint32_t at_small(uint32_t r, uint32_t c)
{
    return CHUNKS == 8 ? at_k(r, c) : r * 64 + ((c ^ ((r >> 2) & 3)) << 4);
}

template <uint32_t FMT, bool TA, bool TB, uint32_t T, int S>
__global__ __launch_bounds__(kThreads, S == 2 ? 2 : 4) void small_kernel(SmallProduct g)
{
    // Chunks to a row of an operand's tile (64 summed values, or 32 S outputs), rows that 64
    // lanes read at once, and how often they do.
    constexpr int CA = TA ? 4 * S : 8, CT = TB ? 4 * S : 8, RA = 64 / CA, RB = 64 / CT, U = 4 * S, SIDE = 32 * S;
    constexpr int NT = Unit8<T>::kTerms;
    constexpr uint32_t ES = Unit8<T>::kSize, CB = FMT == kMx4 ? 4 : 8, kTile = SIDE * 128;
    __shared__ __align__(16) uint8_t lds[kWaves * 2 * kTile];
    const uint32_t t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t tiles = g.tm * g.tn, cut = blockIdx.x / tiles, id = blockIdx.x - cut * tiles;
    const uint32_t m0 = id / g.tn * SIDE, n0 = id % g.tn * SIDE;
    const uint32_t s_end = min(g.slices, (cut + 1) * g.per);
    uint8_t *const la = lds + wave * 2 * kTile, *const lb = la + kTile;
    const uint32_t ar = lane / CA, ac = lane % CA, br = lane / CT, bc = lane % CT;

    // One address for the wave and 32-bit offsets of the lanes. Rows past the end of an output axis
    // are the last one again, and a unit that a row of a ends in is read from its end (`late`
    // elements before its place): along the output axis in every slice, along the sum in the
    // last one. What is past the end of the sum is made 0 before it is used.
    int32_t oa[U];
    uint32_t ob[U], oe[U], late = 0;
    if (TA) {
        const uint32_t from = min(m0 + ac * 8, g.m - 8);
        late = m0 + ac * 8 - from;
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const uint32_t r = i * RA + ar, q = i * RB + br;
        oa[i] = (int32_t)(((TA ? r : min(r, g.m - 1 - m0)) * (uint32_t)g.a.ld + ac * 8 - late) * ES);   // may be negative
        oe[i] = TB ? q * g.nb + min(bc / 4, g.nb - 1 - n0 / 32) : min(q, g.n - 1 - n0) * g.nb + bc / 4;
        ob[i] = oe[i] * (4 * CB) + bc % 4 * CB;
    }
    const uint32_t whole = g.k / 64;

    f32x16 acc[S][S] = {};
    Unit8<T> ra[U];
    u32x2 rb[U];
    uint32_t re[U];
    auto load = [&](uint32_t s) {
        const uint32_t k0 = s * 64;
        const uint64_t block0 = TB ? (uint64_t)k0 * g.nb + n0 / 32 : (uint64_t)n0 * g.nb + k0 / 32;
        const uint8_t *pa = reinterpret_cast<const uint8_t *>(g.a.p) + (TA ? k0 * g.a.ld + m0 : m0 * g.a.ld + k0) * ES;
        const uint8_t *pc = g.q.codes + block0 * (4 * CB), *ps = g.q.scales + block0;
        const bool last = s >= whole;
        uint32_t back = 0;   // of the last slice, where the sum runs along a's rows
        if (!TA && last) {
            const uint32_t k = k0 + ac * 8;
            late = k - min(k, g.k - 8);
            back = late * ES;
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            uint32_t b = ob[i], e = oe[i];
            int32_t a = oa[i] - (int32_t)back;
            if (last) {   // back to the last row or block of the sum
                const uint32_t r = k0 + i * RA + ar, q = TB ? k0 + i * RB + br : k0 / 32 + bc / 4, end = TB ? g.k : g.nb;
                const uint32_t over = q >= end ? (q - (end - 1)) * (TB ? g.nb : 1) : 0;
                b -= over * (4 * CB);
                e -= over;
                if (TA)
                    a -= (int32_t)((r >= g.k ? r - (g.k - 1) : 0) * (uint32_t)g.a.ld * ES);
            }
            if (FMT == kMx4)
                rb[i][0] = *reinterpret_cast<const uint32_t *>(pc + b);
            else
                rb[i] = *reinterpret_cast<const u32x2 *>(pc + b);
            re[i] = ps[e];
            ra[i].load(pa + a);
        }
    };
    // What was read past the end of the sum is 0.
    auto finish = [&](uint32_t s) {
        const uint32_t k0 = s * 64;
        if (TA ? m0 + SIDE > g.m : s >= whole)
#pragma unroll
            for (int i = 0; i < U; ++i)
                ra[i].move_down(late);
        if (s >= whole)
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const bool in = TB ? k0 + i * RB + br < g.k : k0 / 32 + bc / 4 < g.nb;
                if (TA)
                    ra[i].keep(k0 + i * RA + ar < g.k);
                rb[i][0] = in ? rb[i][0] : 0;
                rb[i][1] = in ? rb[i][1] : 0;
                re[i] = in ? re[i] : 127;
            }
    };
    // Reads of the operands; across rows as frag_t_at has it, from chunks turned by the row.
    auto frag = [&](uint8_t *tile, auto trans, auto chunks, int i, int ks) -> bf16x8 {
        constexpr int C = decltype(chunks)::value;
        if (!decltype(trans)::value)
            return read_k(tile + frag_k_at(i * 32, ks, lane));
        const uint32_t j = lane & 15, row = ks * 16 + (lane >> 5) * 8 + (j >> 2);
        const uint32_t col = i * 32 + ((lane >> 4) & 1) * 16 + (j & 3) * 4;
        return read_t2(tile + at_small<C>(row, col / 8) + col % 8 * 2, tile + at_small<C>(row + 4, col / 8) + col % 8 * 2);
    };

    uint32_t s = cut * g.per + wave;
    if (s < s_end)
        load(s);
    while (s < s_end) {
        finish(s);
#pragma unroll
        for (int i = 0; i < U; ++i)
            *reinterpret_cast<u32x4 *>(lb + at_small<CT>(i * RB + br, bc)) =
                FMT == kMx4 ? decode4_bf16(rb[i][0], scale4_f32(re[i])) : decode8_bf16(rb[i], scale8_f32(re[i]));
        constexpr int NV = T == kBf16 ? 1 : U;
        float v[NV][8];
        if (T != kBf16)
#pragma unroll
            for (int i = 0; i < U; ++i)
                ra[i].floats(v[i % NV]);
        auto term = [](float (&f)[8], int p) -> u32x4 {
            if (p == 0)
                return first_term(f);
            const u32x4 h = upper_halves(f);
            if (p + 1 < NT)
                leave_lower(f);
            return h;
        };
        const uint32_t next = s + kWaves;
#pragma unroll
        for (int p = 0; p < NT; ++p) {
#pragma unroll
            for (int i = 0; i < U; ++i)
                *reinterpret_cast<u32x4 *>(la + at_small<CA>(i * RA + ar, ac)) = T == kBf16 ? ra[i].bf16() : term(v[i % NV], p);
            wave_fence();
            if (p == NT - 1 && next < s_end)
                load(next);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                bf16x8 fa[S], fb[S];
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    fa[i] = frag(la, Const<TA>(), Const<CA>(), i, ks);
                    fb[i] = frag(lb, Const<TB>(), Const<CT>(), i, ks);
                }
#pragma unroll
                for (int i = 0; i < S; ++i)
#pragma unroll
                    for (int j = 0; j < S; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
            }
            wave_fence();
        }
        s = next;
    }

    // Each wave's results over its own tiles (4 bytes for two of bf16, the same number), then all of
    // them added in the order of the waves.
    float *mine = reinterpret_cast<float *>(la);
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
        for (int j = 0; j < S; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t y = i * 32 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4, x = j * 32 + (lane & 31);
                mine[y * SIDE + (S == 2 ? x ^ ((y & 4) << 3) : x)] = acc[i][j][r];
            }
    __syncthreads();
    const uint32_t y = t * 8 / SIDE, x = t * 8 % SIDE;
    if (y >= SIDE || m0 + y >= g.m || n0 + x >= g.n)
        return;
    float sum[8] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const f32x4 *p = reinterpret_cast<const f32x4 *>(reinterpret_cast<float *>(lds + w * 2 * kTile) + y * SIDE +
                                                         (S == 2 ? x ^ ((y & 4) << 3) : x));
        const f32x4 lo = p[0], hi = p[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum[i] += lo[i];
            sum[4 + i] += hi[i];
        }
    }
    Out o = g.out;
    if (g.cuts > 1)
        o = {g.parts + (uint64_t)cut * g.m * g.n, g.n, kFp32, 0};
    put8(o, m0 + y, n0 + x, g.n, sum);
}

}  // namespace mx

using namespace mx;

#define MX_TYPE(t, ...)                                                                            \
    do {                                                                                           \
        if ((t) == kBf16) { constexpr uint32_t T = kBf16; __VA_ARGS__; }                           \
        else if ((t) == kFp16) { constexpr uint32_t T = kFp16; __VA_ARGS__; }                      \
        else { constexpr uint32_t T = kFp32; __VA_ARGS__; }                                        \
    } while (0)

hipError_t launch_mx_rows(const SmallProduct &g, uint32_t type, hipStream_t s)
{
    const dim3 grid((g.n + 15) / 16);
    MX_TYPE(type, hipLaunchKernelGGL((row_kernel<T>), grid, dim3(kThreads), 0, s, g));
    return hipGetLastError();
}

hipError_t launch_mx_small(const SmallProduct &g, uint32_t op, uint32_t type, uint32_t side, hipStream_t s)
{
    const dim3 grid(g.tm * g.tn * g.cuts);
#define MX_SMALL(...)                                                                                       \
    MX_TYPE(type, {                                                                                         \
        if (side == 64)                                                                                     \
            hipLaunchKernelGGL((small_kernel<__VA_ARGS__, T, 2>), grid, dim3(kThreads), 0, s, g);           \
        else                                                                                                \
            hipLaunchKernelGGL((small_kernel<__VA_ARGS__, T, 1>), grid, dim3(kThreads), 0, s, g);           \
    })
    if (op == kLinear)
        MX_SMALL(kMx4, false, false);
    else if (op == kGradInput)
        MX_SMALL(kMx4, false, true);
    else
        MX_SMALL(kMx8, true, true);
#undef MX_SMALL
    return hipGetLastError();
}

}  // namespace fastrack
