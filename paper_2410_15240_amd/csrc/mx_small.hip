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

constexpr int kThreads = kSmallThreads, kWaves = kThreads / 64;

// Eight elements of a float operand as they lie in memory.
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
};

// ---- a few tokens ----------------------------------------------------------------------------
//
// y[m][n] = sum over k of x[m][k] w[n][k]. The weights as they lie in memory: a wave takes 64
// blocks of a row at once, one to a lane (1 KB of codes that follow one another), of R rows
// before it uses the first, and multiplies them with the x of those places, which it keeps in
// registers for all R. bf16 by the pairwise product, 16 and 32-bit floats in 32 bits. The
// lanes' sums meet in LDS. What bounds it is the reading of w, K / 2 + K / 32 bytes a row: 7.0
// us for 8192 x 8192, 5.1 TB/s, out of the last-level cache, and 9.4, 3.8 TB/s, out of memory
// (32 such layers in turn). (Lanes that read 64 bytes each of 16 rows, as the matrix
// instruction takes them, took twice that: rows a power of two apart are one memory channel's
// work at a time.)
constexpr int kDotWaves = 4;

// Rows at once: as many as leave the registers to 16 waves a CU.
template <uint32_t T, int M> constexpr int dot_rows() { return 8 / M; }

template <uint32_t T, int M>
__global__ __launch_bounds__(64 * kDotWaves, 4) void dot_kernel(SmallProduct g)
{
    constexpr int R = dot_rows<T, M>(), XW = T == kBf16 ? 16 : 32;
    constexpr uint32_t ES = Unit8<T>::kSize;
    __shared__ __align__(16) float part[kDotWaves][M][R][64];
    const uint32_t t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t n0 = blockIdx.x * R;
    float acc[M][R] = {};
    for (uint32_t b0 = wave * 64; b0 < g.nb; b0 += kDotWaves * 64) {
        const uint32_t b = min(b0 + lane, g.nb - 1);
        u32x4 w[R];
        uint32_t e[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const uint64_t at = (uint64_t)min(n0 + i, g.n - 1) * g.nb;
            w[i] = reinterpret_cast<const u32x4 *>(g.q.codes + at * 16)[b];
            e[i] = g.q.scales[at + b];
        }
        uint32_t x[M][XW];
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const uint8_t *row = reinterpret_cast<const uint8_t *>(g.a.p) + min((uint32_t)m, g.m - 1) * g.a.ld * ES;
            const bool end = (b0 + 64) * 32 > g.k;   // of the sum, in these blocks
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                Unit8<T> u;
                const uint32_t k = (b0 + lane) * 32 + j * 8, from = end ? min(k, g.k - 8) : k;
                u.load(row + (uint64_t)from * ES);
                if (end)
                    u.move_down(k - from);
                if (T == kBf16) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        x[m][j * 4 + i] = u.w[i];
                } else {
                    float f[8];
                    u.floats(f);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        x[m][(j * 8 + i) % XW] = f32_bits(f[i]);
                }
            }
        }
        const bool past = b0 + lane >= g.nb;   // no block: 0, whatever the last one holds
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float s = scale4_f32(past ? 127u : e[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t c = past ? 0u : w[i][j];
                if (T == kBf16) {
                    const u32x4 d = decode4_bf16(c, s);
#pragma unroll
                    for (int m = 0; m < M; ++m)
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            // (Left to see the conversion here, the compiler takes the
                            // first of the four pairs for all of them.)
                            uint32_t pair = d[y];
                            asm("" : "+v"(pair));
                            acc[m][i] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair),
                                                                        __builtin_bit_cast(bf16x2, x[m][j * 4 + y]),
                                                                        acc[m][i], false);
                        }
                } else {
                    float d[8];
                    decode4_f32(c, s, d);
#pragma unroll
                    for (int m = 0; m < M; ++m)
#pragma unroll
                        for (int y = 0; y < 8; ++y)
                            acc[m][i] = __builtin_fmaf(d[y], bits_f32(x[m][(j * 8 + y) % XW]), acc[m][i]);
                }
            }
        }
    }
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int i = 0; i < R; ++i)
            part[wave][m][i][lane] = acc[m][i];
    __syncthreads();
    // 16 lanes to a result.
    for (uint32_t i = t / 16; i < M * R; i += 4 * kDotWaves) {
        const uint32_t m = i / R, r = i % R;
        float s = 0.0f;
#pragma unroll
        for (int v = 0; v < kDotWaves; ++v) {
            const f32x4 p = *reinterpret_cast<const f32x4 *>(&part[v][m][r][t % 16 * 4]);
            s += (p[0] + p[1]) + (p[2] + p[3]);
        }
#pragma unroll
        for (int d = 1; d < 16; d *= 2)
            s += __shfl_xor(s, d, 64);
        if (t % 16 == 0 && m < g.m && n0 + r < g.n)
            put1(g.out, m, n0 + r, s);
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
// the other axis. 90 tokens and 700 x 700 weights of bf16 4.2 us (gemm_kernel and its joining of
// parts 12.4), 77 tokens of fp32 and 1000 x 1111 9.1 (20), 29 of fp16 and 2777 x 5003 13 (26).

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
        o = {g.parts + (uint64_t)cut * g.m * g.n, g.n, kFp32, 0, nullptr};
    if (o.scale) {
        const float scale = *o.scale;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            sum[i] *= scale;
    }
    put8(o, m0 + y, n0 + x, g.n, sum);
}

}  // namespace mx

using namespace mx;

template <uint32_t T, int M>
static hipError_t dot(SmallProduct g, hipStream_t s)
{
    constexpr uint32_t R = dot_rows<T, M>(), kMost = R << 23;   // rows of w: a launch has fewer than 2^32 threads
    for (uint32_t left = g.n;; left -= kMost) {
        g.n = left < kMost ? left : kMost;
        hipLaunchKernelGGL((dot_kernel<T, M>), dim3((g.n + R - 1) / R), dim3(64 * kDotWaves), 0, s, g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || left <= kMost)
            return e;
        g.q.codes += (uint64_t)kMost * g.nb * 16;
        g.q.scales += (uint64_t)kMost * g.nb;
        g.out.p = reinterpret_cast<uint8_t *>(g.out.p) + (uint64_t)kMost * mx_type_size(g.out.type);
    }
}

hipError_t launch_mx_dot(const SmallProduct &g, uint32_t type, hipStream_t s)
{
    MX_TYPE(type, return g.m == 1 ? dot<T, 1>(g, s) : dot<T, 2>(g, s));
}

template <uint32_t FMT, bool TA, bool TB>
static void small(const SmallProduct &g, uint32_t type, uint32_t side, hipStream_t s)
{
    const dim3 grid(g.tm * g.tn * g.cuts);
    if (side == 32)
        MX_TYPE(type, hipLaunchKernelGGL((small_kernel<FMT, TA, TB, T, 1>), grid, dim3(kThreads), 0, s, g));
    else if (type == kBf16)
        hipLaunchKernelGGL((small_kernel<FMT, TA, TB, kBf16, 2>), grid, dim3(kThreads), 0, s, g);
    else
        hipLaunchKernelGGL((small_kernel<FMT, TA, TB, kFp16, 2>), grid, dim3(kThreads), 0, s, g);
}

hipError_t launch_mx_small(const SmallProduct &g, uint32_t op, uint32_t type, uint32_t side, hipStream_t s)
{
    if (op == kLinear)
        small<kMx4, false, false>(g, type, side, s);
    else if (op == kGradInput)
        small<kMx4, false, true>(g, type, side, s);
    else
        small<kMx8, true, true>(g, type, side, s);
    return hipGetLastError();
}

}  // namespace fastrack
