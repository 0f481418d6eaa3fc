// Products with a microscaled operand, on the matrix cores.
//
// An MX value is exact in bf16 (2 or 7 significant bits and a power of two), so a product of
// a bf16 matrix with an MX one is a bf16 product with 32-bit sums and no rounding of its own.
// A 16-bit float with more significant bits, or a 32-bit one, is the exact sum of 2 or 3 bf16
// terms: its product is the sum of the terms' products, which the kernels run as a longer sum.
// (But for bits of a 32-bit float below bf16's smallest value, 2^-133, which are cut: floats
// below 2^-110 have them. Terms scaled up into range cost a sixth of the time, for bits that only
// MX scales near the top of theirs would show.)
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "launch.h"
#include "mx.h"
#include "mx_dev.h"
#include "mx_gemm_dev.h"
#include "mx_loss_dev.h"
#include "mx_small.h"

namespace fastrack {
namespace mx {

// The MX matrix decoded to bf16 beforehand: its blocks are 64 bytes, its scales not read.
constexpr uint32_t kDecoded = 16;

constexpr int kThreads = 256;   // 4 waves, 2 x 2 over the output tile
constexpr uint32_t kBK = 64;    // of the summed axis, at a time

struct Gemm {
    const uint16_t *a;       // bf16 terms of the float matrix, `planes` of them
    uint64_t a_plane;        // elements between them
    uint64_t lda;
    uint32_t a_cols;         // values of a row that may be read: laid-out rows end in zeros
    MxMatrix q;
    uint32_t nb;             // blocks in a row of q
    uint32_t m, n, k;        // output m x n, summed axis k
    uint32_t planes;
    uint32_t whole;          // whole stages of a term that are read unchecked
    uint32_t stages;         // planes * ceil(k / kBK)
    uint32_t splits, per;    // parts of the sum, stages in each
    uint32_t tm, tn;         // output tiles
    void *c;
    uint64_t ldc;
    uint32_t ctype;
    uint32_t accumulate;
    float *parts;            // [splits][m][n] where splits > 1
    const float *scale;      // of c (null: 1)
};

// Tile of workgroup `id`. Workgroups go to the 8 XCDs in turn, each with its own L2: an XCD
// takes a run of neighbouring tiles, in bands of 8 tile rows, so that the tiles it works on at
// one time share rows of both operands.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tm, uint32_t tn, uint32_t &m, uint32_t &n)
{
    constexpr uint32_t kXcds = 8, kBand = 8;
    const uint32_t tiles = tm * tn, q = tiles / kXcds, r = tiles % kXcds, x = id % kXcds;
    const uint32_t i = x * q + min(x, r) + id / kXcds;
    const uint32_t band = i / (kBand * tn), first = band * kBand, rows = min(kBand, tm - first), j = i - first * tn;
    m = first + j % rows;
    n = j / rows;
}

// A workgroup's results, 2 x 2 waves of N x N squares of 32: lane l of a wave holds column
// l % 32 of rows 8 (r / 4) + 4 (l / 32) + r % 4 of each. They pass through LDS, 64 rows at a
// time, so that c is written in whole rows of the tile. Rows whose bit 2 is set are turned by
// 32 columns: the two halves of a wave then write to different banks.
template <int N, bool SCALED = false>
__device__ __forceinline__ void put_tile(const f32x16 (&acc)[N][N], float *lds, uint32_t m0, uint32_t n0, uint32_t m,
                                         uint32_t n, const Out &o)
{
    constexpr uint32_t B = 64 * N;
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6;
    float scale = 1.0f;
    if (SCALED && o.scale)   // (a part of a sum has none)
        scale = *o.scale;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i)
            __syncthreads();
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t y = wave / 2 * 32 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4;
                const uint32_t x = wave % 2 * 32 * N + j * 32 + (lane & 31);
                lds[y * B + (x ^ ((y & 4) << 3))] = acc[i][j][r];
            }
        __syncthreads();
#pragma unroll 2
        for (uint32_t u = t; u < 64 * B / 8; u += kThreads) {
            const uint32_t y = u / (B / 8), x = u % (B / 8) * 8;
            const uint32_t row = m0 + (y >> 5) * 32 * N + i * 32 + (y & 31), col = n0 + x;
            const f32x4 *p = reinterpret_cast<const f32x4 *>(lds + y * B + (x ^ ((y & 4) << 3)));
            const f32x4 lo = p[0], hi = p[1];
            float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            if (SCALED)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[e] *= scale;
            if (row < m && col < n)
                put8(o, row, col, n, v);
        }
    }
}

// The end of a tile: its results to c, or to their part of a sum; SCALED: by g.scale. (Looking for a
// scale in every product costs a large one 1% of its time.)
template <bool SCALED>
struct Store {
    template <int N>
    __device__ __forceinline__ void finish(const f32x16 (&acc)[N][N], float *lds, uint32_t m0, uint32_t n0, uint32_t part,
                                           const Gemm &g) const
    {
        Out o = {g.c, g.ldc, g.ctype, g.accumulate, g.scale};
        if (g.splits > 1)
            o = {g.parts + (uint64_t)part * g.m * g.n, g.n, kFp32, 0, nullptr};
        put_tile<N, SCALED>(acc, lds, m0, n0, g.m, g.n, o);
    }
};

// 32 of each wave's rows of a tile (its squares i) to LDS, in rows as put_tile has them.
template <int N>
__device__ __forceinline__ void spread(const f32x16 (&acc)[N][N], int i, float *lds)
{
    constexpr uint32_t B = 64 * N;
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6;
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const uint32_t y = wave / 2 * 32 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4;
            const uint32_t x = wave % 2 * 32 * N + j * 32 + (lane & 31);
            lds[y * B + (x ^ ((y & 4) << 3))] = acc[i][j][r];
        }
}

// The end of a tile of logits, of which their largest and the sum of their exponentials are left.
// 64 rows at a time are in LDS, a quarter of a row to a thread, which holds it in registers between
// the two; threads begin at different places of their quarters, for the banks. An exponential is one fma and
// 2^v, with the largest value over ln 2 rounded; what that takes off it all have in common, and the sum is
// multiplied by it. What bounds it is
// v_exp_f32, 16 cycles of the 30 of a value: 7680 of a tile, whose products take 131072 with 4096
// inputs.
struct StatEnd {
    LossTile a;

    template <bool EDGE, uint32_t C>   // EDGE: only the first `left` columns of the quarter are classes
    __device__ __forceinline__ Stat stat(f32x4 (&v)[C], const uint32_t (&x)[C], uint32_t left) const
    {
        const float inf = __builtin_inff();
        float top = -inf;   // (a NaN shows in the sum)
#pragma unroll
        for (uint32_t k = 0; k < C; ++k)
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) {
                v[k][e] *= a.scale;
                top = fmaxf(top, EDGE && x[k] + e >= left ? -inf : v[k][e]);
            }
        top = fmaxf(top, quad_xor1(top));
        top = fmaxf(top, quad_xor2(top));
        float from = base_of(top), base = from * kLog2e;
        if (!near(base)) {   // (logits of 1e7 and more)
#pragma unroll
            for (uint32_t k = 0; k < C; ++k)
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e)
                    v[k][e] = minus(v[k][e], from);
            from = base = 0.0f;
        }
        float sum = 0.0f;
#pragma unroll
        for (uint32_t k = 0; k < C; ++k)
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(v[k][e], kLog2e, -base));
                sum += EDGE && x[k] + e >= left ? 0.0f : p;
            }
        sum += quad_xor1(sum);
        sum += quad_xor2(sum);
        return {top, sum * rounding_of(base, from)};
    }

    template <int N>
    __device__ __forceinline__ void finish(const f32x16 (&acc)[N][N], float *lds, uint32_t m0, uint32_t n0, uint32_t,
                                           const Gemm &g) const
    {
        constexpr uint32_t B = 64 * N, Q = B / 4, C = Q / 4;   // columns of a tile, of a quarter; chunks of 4 in it
        const uint32_t t = threadIdx.x, y = t / 4, q = t % 4, turn = (y & 4) << 3;
        const float *line = lds + y * B;
        uint32_t x[C];
#pragma unroll
        for (uint32_t k = 0; k < C; ++k)
            x[k] = (k + t) % C * 4;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t row = m0 + (y >> 5) * 32 * N + i * 32 + (y & 31);
            const int64_t at = row < g.m ? id_of(a.ids, row) - (int64_t)(a.v0 + n0) : -1;
            if (i)
                __syncthreads();
            spread<N>(acc, i, lds);
            __syncthreads();
            f32x4 v[C];
#pragma unroll
            for (uint32_t k = 0; k < C; ++k)
                v[k] = *reinterpret_cast<const f32x4 *>(line + ((q * Q + x[k]) ^ turn));
            const uint32_t classes = min(B, g.n - n0);
            const Stat s = classes == B ? stat<false, C>(v, x, 0) : stat<true, C>(v, x, classes > q * Q ? classes - q * Q : 0);
            if (q == 0 && row < g.m) {
                a.stats[(uint64_t)(a.part0 + n0 / B) * g.m + row] = s;
                if (at >= 0 && at < (int64_t)classes)
                    a.label[row] = line[(uint32_t)at ^ turn] * a.scale;
            }
        }
    }
};

// The end of a tile of logits that becomes their gradient, in bf16 terms, each the nearest to what
// those before leave: dloss (e^(z - lse) - [class = target]) times the scale.
// What it adds to a tile's products is v_exp_f32 and the writing of 128 KB of terms, which most
// workgroups do at once: 4096 tokens, 4096 x 32768, 883 us, the matrix unit busy 63% of the cycles
// (71% with StatEnd). With a row's values loaded for every 32 rows and the rounding's rest found after
// the last term too, 100 us more of the 6980 for loss and both gradients of 4096 tokens and 65536 classes. The
// scale and 1 / ln 2 in one factor would save 5, but logits have to be rounded as they were for lse: p of a class that
// has all of a row is off by lse's last digits otherwise.
struct SlopeEnd {
    LossTile a;

    template <int N>
    __device__ __forceinline__ void finish(const f32x16 (&acc)[N][N], float *lds, uint32_t m0, uint32_t n0, uint32_t,
                                           const Gemm &g) const
    {
        constexpr uint32_t B = 64 * N, U = B / 8, R = 64 * U / kThreads;   // units of a row; rows of a thread
        const uint32_t t = threadIdx.x, x = t % U * 8, classes = min(B, g.n - n0);
        // What a row needs, once for all, behind the 64 rows of logits: lse, its factor with what makes up
        // for the rounding of the third, lse over ln 2, and the target's column in the tile (-1: elsewhere,
        // -2: no target).
        f32x4 *const rows = reinterpret_cast<f32x4 *>(lds + 64 * B);
        if (B >= kThreads || t < B) {
            const uint32_t row = min(m0 + t, g.m - 1);
            const int64_t id = id_of(a.ids, row), d = id - (int64_t)(a.v0 + n0);
            const float lse = a.lse[row], base = lse * kLog2e, factor = factor_of(a, row);
            rows[t] = f32x4{lse, near(base) ? factor * rounding_of(base, lse) : factor, base, bits_f32(id < 0 ? -2u : d >= 0 && d < B ? (uint32_t)d : -1u)};
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i)
                __syncthreads();
            spread<N>(acc, i, lds);
            __syncthreads();
#pragma unroll
            for (uint32_t k = 0; k < R; ++k) {
                const uint32_t y = t / U + k * (kThreads / U), in = (y >> 5) * 32 * N + i * 32 + (y & 31), row = m0 + in;
                const f32x4 r = rows[in];
                const float lse = r[0], factor = r[1];
                float base = r[2];
                const int32_t target = (int32_t)f32_bits(r[3]), at = target - (int32_t)x;
                const f32x4 *p = reinterpret_cast<const f32x4 *>(lds + y * B + (x ^ ((y & 4) << 3)));
                const f32x4 lo = p[0], hi = p[1];
                float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[e] *= a.scale;
                if (!near(base)) {   // (logits of 1e7 and more)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        v[e] = minus(v[e], lse);
                    base = 0.0f;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[e] = factor * __builtin_amdgcn_exp2f(__builtin_fmaf(v[e], kLog2e, -base));
                if (target >= 0 && at >= 0 && at < 8) {
                    const float own = factor_of(a, row < g.m ? row : g.m - 1);
#pragma unroll
                    for (int e = 0; e < 8; ++e)   // (in one product: what e^0 - 1 leaves is not rounded away)
                        v[e] = at == e ? target_slope(minus(reinterpret_cast<const float *>(p)[e] * a.scale, lse), own) : v[e];
                }
                if (target == -2 || classes < B)
#pragma unroll
                    for (uint32_t e = 0; e < 8; ++e)   // no gradient, whatever the logits are; no class
                        v[e] = target == -2 || x + e >= classes ? 0.0f : v[e];
                if (row < g.m && n0 + x < a.ld)
                    put_terms(a.dz + row * a.ld + n0 + x, a.plane, a.terms, v);
            }
        }
    }
};

// One tile of c, or of one part of it, by 2 x 2 waves of 32 N x 32 N outputs each. TA: a is
// summed over its rows (a[k][m]) instead of along them (a[m][k]); TB: the same of the MX
// matrix. While a stage of 64 summed values is multiplied out of one half of the LDS, the next
// one is decoded from registers to bf16 in the other half, and the one after is on its way
// from memory.
//
// The large tile is 256 x 256 with four waves of 128 x 128, one on each SIMD: a stage's 2048
// cycles of products then need 1024 cycles of operand reads and 512 of writes from the LDS,
// where waves of 64 x 64 in a tile of 128 need 3072 (661 us instead of 414 for 4096 tokens and
// 8192 x 8192 weights of bf16; eight waves of 128 x 64, 414 too, and 572 instead of 490 where
// both operands are read across their rows). A wave alone on its SIMD has only its own work to
// put beside its products, so that is dealt out by hand, a few instructions after each
// (compiled in its own order: 514). Measured for that layer, on cards of different clocks:
// linear 403-443 us (1.24-1.36 PFLOP/s), input gradient 380-424 (1.30-1.45), weight gradient
// 439-487 with its decoding; the library's bf16 product of these sizes 398-421. The matrix unit is busy 70-76% of the cycles; what
// bounds them is power, which holds the clock near 1.7 GHz under this load.
//
// Stages of 64 whole values come first, of every term of a, then the terms' last, short ones.
// A whole stage is read without a check: rows and columns past the matrices' ends read the
// last ones again, for results that are not stored. (Rows so long that a tile spans 2^32
// bytes have no such stages; all of theirs are checked.)
template <uint32_t FMT, bool TA, bool TB, int N, class End>
__global__ __launch_bounds__(kThreads, N > 2 ? 1 : 2) void gemm_kernel(Gemm g, End end)
{
    constexpr int B = 64 * N, U = B * 8 / kThreads;   // outputs a side; units of 8 values that a thread copies of each operand
    constexpr uint32_t CB = FMT == kMx4 ? 4 : FMT == kMx8 ? 8 : 16;   // bytes of 8 codes, or bf16 values
    typedef uint32_t Codes __attribute__((ext_vector_type(FMT == kDecoded ? 4 : 2)));
    // Two stages: both tiles of a, then both of the MX matrix, so that a lane's offsets within
    // either are a register and a constant of 16 bits.
    constexpr uint32_t kTile = B * kBK * 2;
    __shared__ __align__(16) uint8_t lds[4 * kTile];
    const uint32_t t = threadIdx.x;
    const uint32_t lane = t & 63, wave = t >> 6;
    const uint32_t tiles = g.tm * g.tn, part = blockIdx.x / tiles;
    uint32_t tile_m, tile_n;
    tile_of(blockIdx.x - part * tiles, g.tm, g.tn, tile_m, tile_n);
    const uint32_t m0 = tile_m * B, n0 = tile_n * B;
    const uint32_t wm = wave / 2 * 32 * N, wn = wave % 2 * 32 * N;
    const uint32_t s_begin = part * g.per, s_end = min(g.stages, s_begin + g.per);
    const uint32_t full = g.whole, nfull = full * g.planes;   // whole stages of a term, of all

    f32x16 acc[N][N] = {};
    u32x4 ra[U];
    Codes rb[U];
    uint8_t re[U];

    // Offsets in the LDS: of the reads (see frag_k_at, frag_t_at), and of this thread's writes.
    uint32_t fa_at[4], fb_at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        fa_at[i] = TA ? frag_t_at<B>(wm + i % N * 32, lane) : frag_k_at(wm, i, lane);
        fb_at[i] = 2 * kTile + (TB ? frag_t_at<B>(wn + i % N * 32, lane) : frag_k_at(wn, i, lane));
    }
    const uint32_t wa_at = TA ? at_t<B>(t / (B / 8), t % (B / 8) * 8) : at_k(t / 8, t % 8);
    const uint32_t wb_at = 2 * kTile + (TB ? at_t<B>(t / (B / 8), t % (B / 8) * 8) : at_k(t / 8, t % 8));

    // A whole stage: one address for the workgroup and 32-bit offsets of the lanes, in bytes.
    uint32_t oa[U], ob[U], oe[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const uint32_t u = i * kThreads + t;
        if (TA)
            oa[i] = u / (B / 8) * (uint32_t)g.lda * 2 + min(u % (B / 8) * 8, (g.m - 1 - m0) & ~7u) * 2;
        else
            oa[i] = min(u / 8, g.m - 1 - m0) * (uint32_t)g.lda * 2 + u % 8 * 16;
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const uint32_t u = i * kThreads + t;
        const uint32_t row = TB ? u / (B / 8) : min(u / 8, g.n - 1 - n0);
        const uint32_t unit = TB ? min(u % (B / 8), (g.nb - n0 / 32) * 4 - 1) : u % 8;
        ob[i] = row * g.nb * (4 * CB) + unit * CB;
        oe[i] = row * g.nb + unit / 4;
    }
    // Where whole stage `at` of the terms' whole stages lies. Stages are visited in order: going on
    // to the next is an addition, and at the end of a term one back to the MX matrix's start.
    const uint64_t block0 = TB ? n0 / 32 : (uint64_t)n0 * g.nb, block_step = TB ? (uint64_t)kBK * g.nb : kBK / 32;
    const int64_t a_step = TA ? kBK * g.lda * 2 : kBK * 2;
    uint32_t at = 0;   // within its term
    const uint8_t *pa = nullptr, *pc = nullptr, *ps = nullptr;
    auto go_to = [&](uint32_t s) {
        const uint32_t plane = s / full;
        at = s - plane * full;
        pa = reinterpret_cast<const uint8_t *>(g.a + plane * g.a_plane + (TA ? (uint64_t)m0 : m0 * g.lda)) + at * a_step;
        pc = g.q.codes + (block0 + at * block_step) * (4 * CB);
        ps = g.q.scales + block0 + at * block_step;
    };
    const int64_t a_back = (int64_t)g.a_plane * 2 - (int64_t)(full - 1) * a_step, block_back = -(int64_t)(full - 1) * block_step;
    auto next = [&](int third) {
        if (third == 0) {
            at = at + 1 == full ? 0 : at + 1;
            pa += at ? a_step : a_back;
        } else if (third == 1) {
            pc += (at ? (int64_t)block_step : block_back) * (4 * CB);
        } else {
            ps += at ? (int64_t)block_step : block_back;
        }
    };
    auto load_a = [&](int i) { ra[i] = __builtin_amdgcn_raw_buffer_load_b128(buffer_at(pa), oa[i], 0, 0); };
    auto load_b = [&](int i) {
        if constexpr (FMT == kDecoded) {
            rb[i] = __builtin_amdgcn_raw_buffer_load_b128(buffer_at(pc), ob[i], 0, 0);
            return;
        } else if constexpr (FMT == kMx4) {
            rb[i][0] = __builtin_amdgcn_raw_buffer_load_b32(buffer_at(pc), ob[i], 0, 0);
        } else {
            rb[i] = __builtin_amdgcn_raw_buffer_load_b64(buffer_at(pc), ob[i], 0, 0);
        }
        re[i] = __builtin_amdgcn_raw_buffer_load_b8(buffer_at(ps), oe[i], 0, 0);
    };
    // The next stage's way from registers to the LDS, in small items, and its registers' next
    // load: per group a unit of the MX matrix (the scale, then the codes in pairs or all of
    // E2M1's, then the write) and one of a.
    constexpr int kPieces = FMT == kDecoded ? 1 : FMT == kMx4 ? 2 : 6, kGroup = kPieces + 1, kItems = kGroup * U;
    float scale;
    u32x4 dec;
    auto item = [&](uint32_t half, int y, bool again) {
        const int i = y / kGroup, p = y % kGroup;
        if (p == kGroup - 1) {
            *reinterpret_cast<u32x4 *>(lds + wa_at + half * kTile + i * kThreads * 16) = ra[i];
            if (again)
                load_a(i);
            return;
        }
        if (FMT != kDecoded && p == 0)
            scale = FMT == kMx4 ? scale4_f32(re[i]) : scale8_f32(re[i]);
        if (FMT == kMx8 && p >= 1 && p <= 4)
            dec[p - 1] = decode8_pair(rb[i][(p - 1) / 2], (p - 1) % 2, scale);
        if (p == kPieces - 1) {
            if constexpr (FMT == kDecoded)
                dec = rb[i];
            if (FMT == kMx4)
                dec = decode4_bf16(rb[i][0], scale);
            *reinterpret_cast<u32x4 *>(lds + wb_at + half * kTile + i * kThreads * 16) = dec;
            if (again)
                load_b(i);
        }
    };
    auto load_whole = [&](uint32_t s) {   // in the order of the main loop
        go_to(s);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            load_b(i);
            __builtin_amdgcn_sched_barrier(0);
            load_a(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Any stage, with every address checked; what lies outside is 0.
    auto load_short = [&](uint32_t i) {
        const uint32_t per = (g.k + kBK - 1) / kBK - full, plane = i / per, k0 = (full + i - plane * per) * kBK;
        const uint16_t *a = g.a + plane * g.a_plane;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const uint32_t u = i * kThreads + t;
            const uint32_t row = TA ? k0 + u / (B / 8) : m0 + u / 8, col = TA ? m0 + u % (B / 8) * 8 : k0 + u % 8 * 8;
            ra[i] = row < (TA ? g.k : g.m) ? chunk_at(a + row * g.lda, col, g.a_cols) : u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const uint32_t u = i * kThreads + t;
            const uint32_t row = TB ? k0 + u / (B / 8) : n0 + u / 8;
            const uint32_t unit = TB ? n0 / 8 + u % (B / 8) : k0 / 8 + u % 8;   // 8 codes, 4 to a block
            rb[i] = Codes(0);
            re[i] = 0;
            if (row < (TB ? g.k : g.n) && unit / 4 < g.nb) {
                const uint64_t at = (uint64_t)row * g.nb;
                if (FMT != kDecoded)
                    re[i] = g.q.scales[at + unit / 4];
                if (FMT == kMx4)
                    rb[i][0] = reinterpret_cast<const uint32_t *>(g.q.codes)[at * 4 + unit];
                else
                    rb[i] = reinterpret_cast<const Codes *>(g.q.codes)[at * 4 + unit];
            }
        }
    };
    auto load = [&](uint32_t s) {
        if (s < nfull) {
            load_whole(s);
        } else {
            load_short(s - nfull);
        }
    };
    bf16x8 fa[2][N], fb[2][N];
    auto read = [&](uint32_t half, int ks, int to, int r) {   // operand r of a step
        if (r < N)
            fa[to][r] = TA ? read_t<B>(lds + fa_at[r] + half * kTile + ks * 16 * B * 2) : read_k(lds + fa_at[ks] + half * kTile + r * 4096);
        else
            fb[to][r - N] = TB ? read_t<B>(lds + fb_at[r - N] + half * kTile + ks * 16 * B * 2)
                                : read_k(lds + fb_at[ks] + half * kTile + (r - N) * 4096);
    };
    // A step multiplies 16 values of the sum out of registers. `beside(x)` is what is issued
    // after product x: the matrix unit is busy 32 cycles with each, so the rest of the wave's work
    // is dealt out between them, in this order.
    constexpr int P = N * N, R = 2 * N;
    auto step = [&](int regs, auto beside) {
#pragma unroll
        for (int x = 0; x < P; ++x) {
            acc[x / N][x % N] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[regs][x / N], fb[regs][x % N],
                                                                          acc[x / N][x % N], 0, 0, 0);
            beside(x);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Item y of n dealt over the products [from, to): whether it comes after product x.
    auto turn = [](int x, int y, int n, int from, int to) { return from + y * (to - from) / n == x; };
    // One stage, out of `here`, whose first operands are in registers: each step multiplies what
    // the one before has read. The next stage goes to `there` beside the first three steps
    // (`beside(x)` after product x of their 3 P), and its first operands are read under the last.
    auto stage = [&](uint32_t here, uint32_t there, auto beside, auto last) {
#pragma unroll
        for (int ks = 0; ks < 3; ++ks)
            step(ks & 1, [&](int x) {
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (turn(x, r, R, 0, P / 2))
                        read(here, ks + 1, (ks + 1) & 1, r);
                beside(ks * P + x);
            });
        step(1, [&](int x) {
            if (x == P / 4)
                lds_barrier();
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (turn(x, r, R, P / 4, P * 3 / 4))
                    read(there, 0, 0, r);
            last(x);
        });
    };

    if (s_begin < s_end) {
        auto put = [&](uint32_t half) {
#pragma unroll
            for (int y = 0; y < kItems; ++y)
                item(half, y, false);
        };
        auto begin = [&](auto ld) {
            ld(s_begin);
            put(0);
            if (s_begin + 1 < s_end)
                ld(s_begin + 1);
            lds_barrier();
#pragma unroll
            for (int r = 0; r < R; ++r)
                read(0, 0, 0, r);
        };
        uint32_t s = s_begin;
        auto whole = [&](uint32_t here, uint32_t there) {
            stage(here, there, [&](int x) {
#pragma unroll
                for (int y = 0; y < kItems; ++y)
                    if (turn(x, y, kItems, 0, 3 * P))
                        item(there, y, true);
            }, [&](int x) {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (turn(x, i, 3, P / 2, P))
                        next(i);
            });
            ++s;
        };
        // (The main loop has a way in of its own: the waits it puts before its registers' use
        // count the loads issued since, on every way in.)
        if (s + 3 < min(s_end, nfull)) {
            begin(load_whole);
            go_to(s + 2);
            do {
                whole(0, 1);
                whole(1, 0);
            } while (s + 3 < min(s_end, nfull));
        } else {
            begin(load);
        }
        uint32_t h = 0;
        for (; s < s_end; ++s, h ^= 1) {
            stage(h, h ^ 1, [&](int x) {
                if (x == 3 * P - 1) {
                    if (s + 1 < s_end)
                        put(h ^ 1);
                    if (s + 2 < s_end)
                        load(s + 2);
                }
            }, [](int) {});
        }
        lds_barrier();
    }

    end.template finish<N>(acc, reinterpret_cast<float *>(lds), m0, n0, part, g);
}

// c = the sum of the parts, always in their order; four values of a row to a thread, or fewer at
// its end. (Products are cut only where they have fewer tiles than CUs: below 2^32 values.)
__global__ __launch_bounds__(kThreads) void join_kernel(const float *parts, uint32_t splits, uint32_t m, uint32_t n,
                                                        uint32_t per_row, uint32_t recip, Out o)
{
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x, row = div_recip(i, per_row, recip), c = (i - row * per_row) * 4;
    if (row >= m)
        return;
    const uint64_t total = (uint64_t)m * n;
    const float *p = parts + (uint64_t)row * n + c, scale = o.scale ? *o.scale : 1.0f;
    if (c + 4 <= n) {
        f32x4 v = {0, 0, 0, 0};
#pragma unroll 4
        for (uint32_t s = 0; s < splits; ++s) {
            f32x4 w;
            __builtin_memcpy(&w, p + s * total, 16);
            v += w;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            put1(o, row, c + j, v[j] * scale);
    } else {
        for (uint32_t j = c; j < n; ++j) {
            float v = 0.0f;
            for (uint32_t s = 0; s < splits; ++s)
                v += p[s * total + j - c];
            put1(o, row, j, v * scale);
        }
    }
}

// The bf16 terms of a float matrix, rows padded with zeros to ld (a multiple of 8): each term
// is what is left cut to its upper 16 bits, so that 3 terms of 8 significant bits (2 for
// 11 bits) add up to the value, down to its bit of 2^-133.
struct Terms {
    MxRows a;
    uint64_t row0;
    uint32_t units, per_row, recip, cols;   // 8 values each, of this launch; of a row
    uint16_t *out;
    uint64_t ld, plane;
};

template <uint32_t T>
__global__ __launch_bounds__(kThreads) void terms_kernel(Terms g)
{
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= g.units)
        return;
    const uint32_t r = div_recip(i, g.per_row, g.recip), c = (i - r * g.per_row) * 8;
    float v[8];
    load8<T>(g.a.p, (g.row0 + r) * g.a.ld, c, g.cols, v);
    uint16_t *out = g.out + (g.row0 + r) * g.ld + c;
    *reinterpret_cast<u32x4 *>(out) = T == kBf16 ? upper_halves(v) : first_term(v);
    if (T != kBf16)
        *reinterpret_cast<u32x4 *>(out + g.plane) = upper_halves(v);
    if (T == kFp32) {
        leave_lower(v);
        *reinterpret_cast<u32x4 *>(out + 2 * g.plane) = upper_halves(v);
    }
}

uint32_t planes_of(uint32_t type) { return type == kBf16 ? 1 : type == kFp16 ? 2 : 3; }

uint64_t round_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

// How a product runs.
enum Path : int {
    kDot,     // mx_small.hip, up to 2 tokens
    kSmall,   // mx_small.hip, tiles of 32 or 64
    kTiles,   // gemm_kernel, tiles of 128 or 256
};

struct Plan {
    Path path;
    uint32_t tile;                            // side of an output tile
    uint32_t tm, tn;                          // tiles
    uint64_t m, n, k;                         // output m x n, summed axis k
    uint64_t a_rows, a_cols;
    // Where a is read as bf16 terms from the workspace: their number, layout and bytes.
    bool laid_out;
    uint32_t planes;
    uint64_t a_ld, a_bytes;
    bool decoded;                             // the MX matrix is decoded there as well
    uint64_t q_bytes;
    uint32_t stages, splits, per;             // of 64 summed values; parts of the sum, stages in each
    uint64_t bytes() const { return a_bytes + q_bytes + (splits > 1 ? (uint64_t)splits * m * n * 4 : 0); }
};

// One way to run a product, its sum in up to `splits` parts.
Plan plan_as(const MxProduct &p, Path path, uint32_t tile, bool laid_out, uint64_t splits)
{
    Plan r = {};
    const bool ta = p.op == kWeightGrad;
    r.path = path;
    r.tile = tile;
    r.m = ta ? p.n : p.m;
    r.n = p.op == kLinear ? p.n : p.k;
    r.k = p.op == kLinear ? p.k : ta ? p.m : p.n;
    r.a_rows = p.m;
    r.a_cols = p.op == kLinear ? p.k : p.n;
    r.tm = (uint32_t)((r.m + tile - 1) / tile);
    r.tn = (uint32_t)((r.n + tile - 1) / tile);
    r.laid_out = laid_out && r.k;
    r.planes = p.terms ? p.terms : r.laid_out ? planes_of(p.type) : 1;
    r.a_ld = round_up(r.a_cols, 8);
    r.a_bytes = r.laid_out ? round_up(r.planes * r.a_rows * r.a_ld * 2, 256) : 0;
    r.stages = (uint32_t)((r.k + kBK - 1) / kBK) * r.planes;
    if (splits > r.stages)
        splits = r.stages;
    r.per = splits > 1 ? (uint32_t)((r.stages + splits - 1) / splits) : r.stages ? r.stages : 1;
    r.splits = r.stages ? (r.stages + r.per - 1) / r.per : 1;
    return r;
}

// A product's time in us beyond its ends when its sum is cut: the longest part, the parts in fp32
// written and read at 4 TB/s, and the joining launch.
double cut_us(double whole_us, uint64_t cuts, uint64_t outputs)
{
    return whole_us / (double)cuts + (cuts > 1 ? 3.0 + 8e-6 / 4.0 * (double)(outputs * cuts) : 0.0);
}

// The number of parts of a sum for which that is least, up to one part for every CU (a second
// round adds parts without shortening any) and down to 4 stages a part. (Parts: us. bf16 linear,
// 3000 tokens, 1000 x 1000, 192 tiles: 1: 16, 2: 27; 300 tokens, 5000 x 5000, 120 tiles: 1: 51, 2: 38,
// 4: 39. MX4 by MX4, 512 tokens, 4096 x 4096, 128 tiles: 1: 13, 2: 23, 4: 25; 64 tokens, 8192 x 8192,
// 64 tiles: 1: 20, 4: 15, 8: 18; 128 tokens, 16384 x 1024, 8 tiles: 1: 30, 8: 13, 16: 14.)
uint64_t cuts_of(double whole_us, uint64_t tiles, uint64_t stages, uint64_t outputs, uint64_t cu)
{
    uint64_t most = tiles ? cu / tiles : 1, best = 1;
    most = most < stages / 4 ? most : stages / 4;
    for (uint64_t c = 2; c <= most; c++)
        if (cut_us(whole_us, c, outputs) < cut_us(whole_us, best, outputs))
            best = c;
    return best;
}

Plan plan_of(const MxProduct &p, int num_cu)
{
    const uint64_t cu = (uint64_t)num_cu;
    const bool ta = p.op == kWeightGrad;
    const uint64_t m = ta ? p.n : p.m, n = p.op == kLinear ? p.n : p.k, a_cols = p.op == kLinear ? p.k : p.n;
    const uint64_t k = p.op == kLinear ? p.k : ta ? p.m : p.n;
    if (m == 0 || n == 0)
        return plan_as(p, kTiles, 128, false, 1);   // no outputs: nothing is launched
    if (p.op == kLinear && p.m <= 2 && p.k >= 512)
        return plan_as(p, kDot, 1, false, 1);
    const uint64_t span = 64 * (p.a.ld * 4 + mx_blocks(p.k) * 32) + 4096;   // a small tile's offsets in 31 bits
    // A loss's logits of up to 32 tokens, 64 of 16 bits: tiles of 128 and 256 are mostly empty, and
    // however many of them there are, small ones take less (us with the loss's kernels, as below and
    // small: 8 tokens of bf16, 4096 x 65536: 113, 57; fp32: 301, 134; 1024 x 32768: 22, 20; 64 of bf16, 4096 x
    // 65536: 114, 88; fp32: 305, 256, but 1024 x 32768: 40, 46).
    const uint64_t side = p.m <= 32 ? 32 : 64, few = (p.n + side - 1) / side;
    if (p.few && p.m <= (p.type == kFp32 ? 32 : 64) && p.k >= 8 && span < 1ull << 31 && few * kSmallThreads < 1ull << 32) {
        const uint64_t slices = (k + kBK - 1) / kBK, most = slices / 16 < cu / few ? slices / 16 : cu / few;
        return plan_as(p, kSmall, (uint32_t)side, false, few <= cu / 2 && most > 1 ? most : 1);
    }
    // gemm_kernel reads whole stages 16 bytes at a time at multiples of 4. Along its rows a may end
    // anywhere (the short stage looks at each value); across them, whole chunks.
    const bool in_place = p.terms || (p.type == kBf16 && reinterpret_cast<uintptr_t>(p.a.p) % 4 == 0 && (p.a.ld % 2 == 0 || p.m == 1) &&
                          (!ta || a_cols % 8 == 0));
    const uint64_t stages = (k + kBK - 1) / kBK, terms = p.terms ? p.terms : planes_of(p.type);

    // gemm_kernel: tiles of 256 where they give more than half the CUs work and the sum is long
    // enough to pay for a tile's ends (64 tokens' gradient of 8192 x 8192 weights: 67 us with tiles
    // of 128, 85 with 256; 300 tokens' of 4000 x 4000: 29.5 and 27.9), else of 128. Up to half the
    // CUs, tiles of 128, two to a CU, still fit in one round. (bf16 linear, 128 and 256: 2048
    // tokens, 4096 x 4096 79 and 92 us; 3000 tokens, 3000 x 4000 104 and 81; 1500 tokens, 6000 x
    // 6000 167 and 124.) A stage of a tile of 128 alone on its CU takes 0.4 us, 0.65 where the
    // operands are transposed, and the sum of each is cut where that pays.
    const uint64_t large = (m + 255) / 256 * ((n + 255) / 256);
    // (And where more tiles of 128 would be 2^32 threads, which no launch has.)
    const uint64_t tiles128 = (m + 127) / 128 * ((n + 127) / 128);
    const uint32_t tile = (large > cu / 2 && stages >= 4) || tiles128 * kThreads >= 1ull << 32 ? 256 : 128;
    const uint64_t tiles = (m + tile - 1) / tile * ((n + tile - 1) / tile), sum = stages * (in_place && !p.terms ? 1 : terms);
    const double whole_us = (ta ? 0.65 : 0.4) * (double)sum;
    const uint64_t splits = tile == 256 ? 1 : cuts_of(whole_us, tiles, sum, m * n, cu);
    Plan as_tiles = plan_as(p, kTiles, tile, !in_place, splits);
    // The kept input of a weight gradient is decoded by every row of tiles again, 24 instructions
    // for 8 values, which only partly fit between the matrix instructions. Where there are many
    // rows of tiles, once beforehand is less (8192 inputs, bf16, in the kernel and beforehand:
    // 4096 tokens and 8192 outputs 485 and 441 us, 4096 outputs 252 and 239; 1000 tokens and
    // 4096 outputs 92 and 87, 2048 outputs 46 and 49).
    if (p.op == kWeightGrad && tile == 256 && as_tiles.planes * m >= 4096) {
        as_tiles.decoded = true;
        as_tiles.q_bytes = p.m * mx_blocks(p.k) * 64;
    }
    if (tile == 256 || span >= 1ull << 31 || a_cols < 8 || k == 0 || p.terms > 1)
        return as_tiles;

    // Small tiles or gemm_kernel's of 128, by estimates of their times in us. A workgroup of small
    // tiles takes 3 and an eighth of what its slices were measured to take a wave; those of 32
    // run two to a CU. Where the MX matrix is read across its rows, 16 or 32 bytes of each, a slice
    // takes longer the more tiles read at once and the farther its rows lie apart (gradient of
    // 32 tokens, 4096 outputs of bf16, tiles of 32: 0.7 us in 16 and 32 tiles, 1.7 in 64 to 125; 2.1 in 128 with rows
    // of 128 blocks, 2.8 in 256, with gemm_kernel on the other side 15.7 and 16.0 us for 16.7 of 125 tiles
    // and 25.6 of 256): so the step at 64 tiles, and the one at rows of 128 blocks.
    // gemm_kernel takes 8, 4 more to lay out a's terms, and its sum's time as above, a quarter more
    // for every round of several. (Both sides: linear, 1000 x 2000 x 1000 of bf16: 12 and 26; 128 tokens, 8192 x
    // 8192 of fp32: 125 and 71; gradient of 32 tokens, 8192 x 8192 of bf16: 48 and 25; weight
    // gradient of 64 tokens, 8192 x 8192: 216 and 67, of 3000 tokens, 1000 x 1000: 20 and 27.)
    const uint64_t tiles64 = (m + 63) / 64 * ((n + 63) / 64), tiles32 = (m + 31) / 32 * ((n + 31) / 32);
    const bool by64 = tiles64 >= cu / 2 && p.type != kFp32;
    const uint64_t count = by64 ? tiles64 : tiles32, at_once = by64 ? cu : 2 * cu;
    if (count * kSmallThreads >= 1ull << 32)   // as many threads as no launch has
        return as_tiles;
    const double across = p.op == kWeightGrad ? 2.6 : mx_blocks(p.k) < 128 ? 1.5 : 2.6;
    const double slice = (p.op == kLinear ? (by64 ? 1.8 : 0.7) : by64 ? (p.op == kGradInput ? 2.2 : 3.0) : count <= 64 ? 1.0 : across) *
                         (p.type == kBf16 ? 1.0 : p.type == kFp16 ? 1.4 : p.op == kLinear ? 4.0 : 2.5);
    uint64_t cuts = count <= cu / 2 ? cu / count : 1;   // few tiles: parts of the sum, 16 slices each and more
    cuts = cuts < stages / 16 ? cuts : stages / 16;
    cuts = cuts < 1 ? 1 : cuts;
    const double small = (double)((count * cuts + at_once - 1) / at_once) * (3.0 + slice * (double)stages / (8.0 * (double)cuts)) +
                         (cuts > 1 ? 4.0 : 0.0);
    const double rounds = tiles <= cu ? 1.0 : 1.25 * (double)((tiles + cu - 1) / cu);
    const double large_us = 8.0 + (in_place ? 0.0 : 4.0) + cut_us(whole_us * rounds, splits, m * n);
    return small <= large_us ? plan_as(p, kSmall, by64 ? 64 : 32, false, cuts) : as_tiles;
}

// ---- MX4 x MX4 -------------------------------------------------------------------------

constexpr uint32_t kBK4 = 256;   // 8 blocks: rows of 128 bytes, as above

struct Gemm4 {
    MxMatrix x, w;
    uint32_t nb, m, n;
    uint32_t whole;          // stages of 8 blocks that are read unchecked
    uint32_t stages, splits, per, tm, tn;
    int tile;
    void *c;
    uint64_t ldc;
    uint32_t ctype;
    float *parts;
};

typedef int i32x8 __attribute__((ext_vector_type(8)));

// Both operands stay in 4 bits: the scaled matrix instruction takes 32 codes and their block's
// scale byte per lane, row l % 32, block l / 32. A stage of 8 blocks is laid out, copied and
// read like one of 64 bf16 values above (16 bytes are a block here), and its 8 scales of each
// row beside it. A lane reads its row's 8 scales at once, and the instruction picks the byte:
// blocks 2 ks of the lower lanes, 2 ks + 1 of the upper ones, whose words are shifted down by
// one byte. 141-155 us for 4096 tokens and 8192 x 8192 weights (3.7 PFLOP/s; tiles of 128 and one
// stage in LDS took 538), the matrix unit busy 57% of the cycles: a stage brings 68 KB to a
// workgroup in the time in which gemm_kernel brings 40 to 48, and its waits are what is left.
// (The checked last stages spill a few registers; the main loop does not.)
template <int N>
__global__ __launch_bounds__(kThreads, N > 2 ? 1 : 2) void gemm4_kernel(Gemm4 g)
{
    constexpr int B = 64 * N, U = B * 8 / kThreads, R = 2 * N, P = N * N;
    constexpr uint32_t kTile = B * 128, kS = 2 * B * 8;
    __shared__ __align__(16) uint8_t lds[2 * (2 * kTile + kS)];   // two stages: codes of x, of w, scales
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const uint32_t tiles = g.tm * g.tn, part = blockIdx.x / tiles;
    uint32_t tile_m, tile_n;
    tile_of(blockIdx.x - part * tiles, g.tm, g.tn, tile_m, tile_n);
    const uint32_t m0 = tile_m * B, n0 = tile_n * B;
    const uint32_t wm = (wave >> 1) * 32 * N, wn = (wave & 1) * 32 * N;
    const uint32_t s_begin = part * g.per, s_end = min(g.stages, s_begin + g.per);

    f32x16 acc[N][N] = {};
    u32x4 rc[2][U];            // codes on their way: of x, of w
    constexpr int S = 2 * B / kThreads;   // rows of scales that a thread copies
    u32x2 rsc[S];

    uint32_t frag_at[2][4], code_at[2][U], scale_at[S];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        frag_at[0][i] = frag_k_at(wm, i, lane);
        frag_at[1][i] = 2 * kTile + frag_k_at(wn, i, lane);
    }
    const uint32_t write_at = at_k(t / 8, t % 8), write_w = 2 * kTile + write_at;
#pragma unroll
    for (int i = 0; i < U; ++i) {
        code_at[0][i] = min(i * 32 + t / 8, g.m - 1 - m0) * g.nb * 16 + t % 8 * 16;
        code_at[1][i] = min(i * 32 + t / 8, g.n - 1 - n0) * g.nb * 16 + t % 8 * 16;
    }
    // Row r of the stage's scales: x's rows, then w's.
    auto row_of = [&](int i) { return (uint32_t)i * kThreads + t; };
#pragma unroll
    for (int i = 0; i < S; ++i) {
        const uint32_t r = row_of(i);
        scale_at[i] = r < B ? min(r, g.m - 1 - m0) * g.nb : min(r - B, g.n - 1 - n0) * g.nb;
    }
    const uint8_t *px = nullptr, *pw = nullptr, *sx = nullptr, *sw = nullptr;   // the next whole stage
    auto go_to = [&](uint32_t s) {
        const uint64_t x = (uint64_t)m0 * g.nb + s * 8, w = (uint64_t)n0 * g.nb + s * 8;
        px = g.x.codes + x * 16, sx = g.x.scales + x;
        pw = g.w.codes + w * 16, sw = g.w.scales + w;
    };
    auto load_code = [&](int o, int i) {
        rc[o][i] = __builtin_amdgcn_raw_buffer_load_b128(buffer_at(o ? pw : px), code_at[o][i], 0, 0);
    };
    auto load_scale = [&](int i) {   // 8 bytes of any alignment
        const uint8_t *base = (B % kThreads == 0 ? i * kThreads < B : t < B) ? sx : sw;
        __builtin_memcpy(&rsc[i], base + scale_at[i], 8);
    };
    constexpr int kItems = 2 * U + S;
    auto write = [&](uint32_t half, int y) {
        if (y < 2 * U)
            *reinterpret_cast<u32x4 *>(lds + (y & 1 ? write_w + half * kTile : write_at + half * kTile) + (y >> 1) * 4096) = rc[y & 1][y >> 1];
        else
            *reinterpret_cast<u32x2 *>(lds + 4 * kTile + half * kS + row_of(y - 2 * U) * 8) = rsc[y - 2 * U];
    };
    auto load_item = [&](int y) {
        if (y < 2 * U)
            load_code(y & 1, y >> 1);
        else
            load_scale(y - 2 * U);
    };
    auto load_whole = [&](uint32_t s) {
        go_to(s);
#pragma unroll
        for (int y = 0; y < kItems; ++y) {
            load_item(y);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Any stage, every address checked: blocks past the end are 0.
    auto load_short = [&](uint32_t s) {
        const uint32_t b0 = s * 8, block = b0 + t % 8;
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const uint32_t row = (o ? n0 : m0) + i * 32 + t / 8;
                rc[o][i] = u32x4{0, 0, 0, 0};
                if (row < (o ? g.n : g.m) && block < g.nb)
                    rc[o][i] = reinterpret_cast<const u32x4 *>(o ? g.w.codes : g.x.codes)[(uint64_t)row * g.nb + block];
            }
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const bool w = row_of(i) >= B;
            const uint32_t row = w ? n0 + row_of(i) - B : m0 + row_of(i);
            const uint8_t *p = (w ? g.w.scales : g.x.scales) + (uint64_t)row * g.nb + b0;
            uint64_t v = 0;   // a block of codes 0 is 0 at any scale but a NaN
            if (row < (w ? g.n : g.m))
#pragma unroll 1
                for (uint32_t j = 0; j < min(8u, g.nb - b0); ++j)
                    v |= (uint64_t)p[j] << (8 * j);
            rsc[i] = u32x2{(uint32_t)v, (uint32_t)(v >> 32)};
        }
    };
    auto load = [&](uint32_t s) {
        if (s < g.whole)
            load_whole(s);
        else
            load_short(s);
    };

    u32x4 fc[2][R];            // operands of two steps
    u32x2 next_scale[R];
    uint32_t scale[R][2];
    auto read = [&](uint32_t half, int ks, int to, int r) {
        fc[to][r] = *reinterpret_cast<const u32x4 *>(lds + (r < N ? frag_at[0][ks] + half * kTile + r * 4096 : frag_at[1][ks] + half * kTile + (r - N) * 4096));
    };
    auto read_scale = [&](uint32_t half, int r) {
        const uint32_t row = r < N ? wm + r * 32 : B + wn + (r - N) * 32;
        next_scale[r] = *reinterpret_cast<const u32x2 *>(lds + 4 * kTile + half * kS + (row + (lane & 31)) * 8);
    };
    const uint32_t shift = (lane >> 5) * 8;
    auto take_scale = [&](int r) {
        scale[r][0] = next_scale[r][0] >> shift;
        scale[r][1] = next_scale[r][1] >> shift;
    };
    auto wide = [](u32x4 v) { return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; };
    // As in gemm_kernel: other work is dealt out after each product.
    auto turn = [](int x, int y, int n, int from, int to) { return from + y * (to - from) / n == x; };
    auto step = [&](auto ks_, auto beside) {
        constexpr int ks = decltype(ks_)::value;
#pragma unroll
        for (int x = 0; x < P; ++x) {
            const int i = x / N, j = x % N;
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                wide(fc[ks & 1][i]), wide(fc[ks & 1][N + j]), acc[i][j], 4, 4, ks % 2 * 2, (int)scale[i][ks / 2],
                ks % 2 * 2, (int)scale[N + j][ks / 2]);
            beside(x);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto stage = [&](uint32_t here, uint32_t there, auto beside, auto last) {
        auto early = [&](auto ks_) {
            constexpr int ks = decltype(ks_)::value;
            step(ks_, [&](int x) {
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (turn(x, r, R, 0, P / 2))
                        read(here, ks + 1, (ks + 1) & 1, r);
                beside(ks * P + x);
            });
        };
        early(Const<0>());
        early(Const<1>());
        early(Const<2>());
        step(Const<3>(), [&](int x) {
            if (x == P / 4)
                lds_barrier();
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (turn(x, r, R, P / 4, P * 3 / 4)) {
                    read_scale(there, r);
                    read(there, 0, 0, r);
                }
            last(x);
        });
#pragma unroll
        for (int r = 0; r < R; ++r)
            take_scale(r);
    };

    if (s_begin < s_end) {
        auto put = [&](uint32_t half) {
#pragma unroll
            for (int y = 0; y < kItems; ++y)
                write(half, y);
        };
        auto begin = [&](auto ld) {
            ld(s_begin);
            put(0);
            if (s_begin + 1 < s_end)
                ld(s_begin + 1);
            lds_barrier();
#pragma unroll
            for (int r = 0; r < R; ++r) {
                read_scale(0, r);
                read(0, 0, 0, r);
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
                take_scale(r);
        };
        uint32_t s = s_begin;
        auto whole = [&](uint32_t here, uint32_t there) {
            stage(here, there, [&](int x) {
#pragma unroll
                for (int y = 0; y < kItems; ++y)
                    if (turn(x, y, kItems, 0, 3 * P)) {
                        write(there, y);
                        load_item(y);
                    }
            }, [&](int x) {
                if (x == P - 2) {
                    px += 128, pw += 128;
                    sx += 8, sw += 8;
                }
            });
            ++s;
        };
        if (s + 3 < min(s_end, g.whole)) {
            begin(load_whole);
            go_to(s + 2);
            do {
                whole(0, 1);
                whole(1, 0);
            } while (s + 3 < min(s_end, g.whole));
        } else {
            begin(load);
        }
        uint32_t h = 0;
        for (; s < s_end; ++s, h ^= 1) {
            stage(h, h ^ 1, [&](int x) {
                if (x == 3 * P - 1) {
                    if (s + 1 < s_end)
                        put(h ^ 1);
                    if (s + 2 < s_end)
                        load(s + 2);
                }
            }, [](int) {});
        }
        lds_barrier();
    }

    Out o = {g.c, g.ldc, g.ctype, 0, nullptr};
    if (g.splits > 1)
        o = {g.parts + (uint64_t)part * g.m * g.n, g.n, kFp32, 0, nullptr};
    put_tile<N>(acc, reinterpret_cast<float *>(lds), m0, n0, g.m, g.n, o);
}

Gemm4 plan4_of(const Mx4Product &p, int num_cu)
{
    Gemm4 g = {};
    g.x = p.x;
    g.w = p.w;
    g.nb = (uint32_t)mx_blocks(p.k);
    g.m = (uint32_t)p.m;
    g.n = (uint32_t)p.n;
    g.whole = 256ull * g.nb * 16 + 128 < 1ull << 32 ? g.nb / 8 : 0;   // a tile's offsets in 32 bits
    g.stages = (g.nb + 7) / 8;
    // Tiles of 256 where they give more than half the CUs work, as for gemm_kernel (128 and 256:
    // 2048 tokens, 4096 x 4096 29 and 36 us; 3000 tokens, 3000 x 4000 43 and 42; 1500 tokens, 6000 x
    // 6000 61 and 55), uncut. A stage of a tile of 128 takes 0.5 us.
    g.tile = (p.m + 255) / 256 * ((p.n + 255) / 256) > (uint64_t)num_cu / 2 ? 256 : 128;
    g.tm = (uint32_t)((p.m + g.tile - 1) / g.tile);
    g.tn = (uint32_t)((p.n + g.tile - 1) / g.tile);
    const uint64_t tiles = (uint64_t)g.tm * g.tn;
    const uint64_t splits =
        g.tile == 256 ? 1 : cuts_of(0.5 * (double)g.stages, tiles, g.stages, p.m * p.n, (uint64_t)num_cu);
    g.per = (uint32_t)((g.stages + splits - 1) / splits);
    if (g.per == 0)
        g.per = 1;
    g.splits = g.stages ? (g.stages + g.per - 1) / g.per : 1;
    return g;
}

}  // namespace mx

using namespace mx;

static hipError_t join(const float *parts, uint32_t splits, uint64_t m, uint64_t n, const Out &o, hipStream_t s)
{
    const uint32_t per_row = (uint32_t)((n + 3) / 4);
    hipLaunchKernelGGL(join_kernel, dim3((uint32_t)((m * per_row + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, parts,
                       splits, (uint32_t)m, (uint32_t)n, per_row, div_recip_of(per_row), o);
    return hipGetLastError();
}

// a's bf16 terms into the workspace.
static hipError_t lay_out(const MxProduct &p, const Plan &r, hipStream_t s)
{
    Terms g = {};
    g.a = p.a;
    g.per_row = (uint32_t)(r.a_ld / 8);
    g.recip = div_recip_of(g.per_row);
    g.cols = (uint32_t)r.a_cols;
    g.out = reinterpret_cast<uint16_t *>(p.work);
    g.ld = r.a_ld;
    g.plane = r.a_rows * r.a_ld;
    const uint64_t most = 0xFFFFFF00u / g.per_row;   // rows of a launch: thread indices in 32 bits
    for (g.row0 = 0; g.row0 < r.a_rows; g.row0 += most) {
        const uint64_t rows = r.a_rows - g.row0 < most ? r.a_rows - g.row0 : most;
        g.units = (uint32_t)(rows * g.per_row);
        const dim3 grid((g.units + kThreads - 1) / kThreads);
        if (p.type == kBf16)
            hipLaunchKernelGGL((terms_kernel<kBf16>), grid, dim3(kThreads), 0, s, g);
        else if (p.type == kFp16)
            hipLaunchKernelGGL((terms_kernel<kFp16>), grid, dim3(kThreads), 0, s, g);
        else
            hipLaunchKernelGGL((terms_kernel<kFp32>), grid, dim3(kThreads), 0, s, g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

static Gemm gemm_of(const MxProduct &p, const Plan &r, const MxRows &a, const MxMatrix &q, float *parts)
{
    Gemm g = {};
    g.a = reinterpret_cast<const uint16_t *>(a.p);
    g.lda = a.ld;
    g.a_cols = (uint32_t)(r.laid_out ? r.a_ld : p.terms ? round_up(r.a_cols, 8) : r.a_cols);
    g.a_plane = p.terms ? p.plane : r.a_rows * r.a_ld;
    g.q = q;
    g.nb = (uint32_t)mx_blocks(p.k);
    g.m = (uint32_t)r.m;
    g.n = (uint32_t)r.n;
    g.k = (uint32_t)r.k;
    g.stages = r.stages;
    g.planes = r.planes;
    const bool ta = p.op == kWeightGrad, tb = p.op != kLinear;
    const uint64_t span_a = (ta ? kBK : 256) * g.lda * 2 + 512, span_b = (tb ? kBK : 256) * (uint64_t)g.nb * (r.decoded ? 64 : 32) + 8192;
    g.whole = span_a < 1ull << 32 && span_b < 1ull << 32 ? g.k / kBK : 0;
    g.splits = r.splits;
    g.per = r.per;
    g.tm = r.tm;
    g.tn = r.tn;
    g.c = p.c.p;
    g.ldc = p.c.ld;
    g.ctype = p.ctype;
    g.accumulate = p.accumulate;
    g.scale = p.scale;
    g.parts = parts;
    return g;
}

template <class End>
static hipError_t launch_tiles(const MxProduct &p, const Plan &r, const MxRows &a, const MxMatrix &q, float *parts,
                               hipStream_t s)
{
    const End end;
    const Gemm g = gemm_of(p, r, a, q, parts);
    const dim3 grid(r.tm * r.tn * r.splits);
#define MX_GEMM(...)                                                                              \
    do {                                                                                          \
        if (r.tile == 256)                                                                        \
            hipLaunchKernelGGL((gemm_kernel<__VA_ARGS__, 4, End>), grid, dim3(kThreads), 0, s, g, end);     \
        else                                                                                      \
            hipLaunchKernelGGL((gemm_kernel<__VA_ARGS__, 2, End>), grid, dim3(kThreads), 0, s, g, end);     \
    } while (0)
    if (p.op == kLinear) {
        if constexpr (std::is_same<End, Store<false>>::value)   // (none is scaled)
            MX_GEMM(kMx4, false, false);
    } else if (p.op == kGradInput)
        MX_GEMM(kMx4, false, true);
    else if (!r.decoded)
        MX_GEMM(kMx8, true, true);
    else
        hipLaunchKernelGGL((gemm_kernel<kDecoded, true, true, 4, End>), grid, dim3(kThreads), 0, s, g, end);
#undef MX_GEMM
    return hipGetLastError();
}

// A head's logits, one tile after the other, to an end of their own.
template <class End>
static hipError_t launch_logits(const MxProduct &p, const LossTile &t, bool laid_out, int num_cu, hipStream_t s)
{
    const Plan r = plan_of(p, num_cu);
    MxRows a = p.a;
    if (r.laid_out) {
        const hipError_t e = laid_out ? hipSuccess : lay_out(p, r, s);
        if (e != hipSuccess)
            return e;
        a = {p.work, r.a_ld};
    }
    const End end = {t};
    const Gemm g = gemm_of(p, r, a, p.q, nullptr);
    const dim3 grid(r.tm * r.tn);
    if (r.tile == 256)
        hipLaunchKernelGGL((gemm_kernel<kMx4, false, false, 4, End>), grid, dim3(kThreads), 0, s, g, end);
    else
        hipLaunchKernelGGL((gemm_kernel<kMx4, false, false, 2, End>), grid, dim3(kThreads), 0, s, g, end);
    return hipGetLastError();
}

uint32_t mx_logits_tile(const MxProduct &p, int num_cu)
{
    const Plan r = plan_of(p, num_cu);
    return r.path == kTiles && r.splits == 1 ? r.tile : 0;
}

hipError_t launch_mx_logits_stats(const MxProduct &p, const LossTile &t, bool laid_out, int num_cu, hipStream_t s)
{
    return launch_logits<StatEnd>(p, t, laid_out, num_cu, s);
}

hipError_t launch_mx_logits_slopes(const MxProduct &p, const LossTile &t, bool laid_out, int num_cu, hipStream_t s)
{
    return launch_logits<SlopeEnd>(p, t, laid_out, num_cu, s);
}

uint64_t mx_product_work(const MxProduct &p, int num_cu) { return plan_of(p, num_cu).bytes(); }

hipError_t launch_mx_product(const MxProduct &p, int num_cu, hipStream_t s)
{
    const Plan r = plan_of(p, num_cu);
    if (r.m == 0 || r.n == 0)
        return hipSuccess;
    MxRows a = p.a;
    uint32_t type = p.type;
    float *parts = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(p.work) + r.a_bytes + r.q_bytes);
    MxMatrix q = p.q;
    if (r.decoded) {
        q = {reinterpret_cast<uint8_t *>(p.work) + r.a_bytes, nullptr};
        const hipError_t e = launch_mx_dequantize(kMx8, kBf16, p.q, p.m, p.k, {q.codes, mx_blocks(p.k) * kMxBlock}, s);
        if (e != hipSuccess)
            return e;
    }
    if (r.laid_out) {
        const hipError_t e = lay_out(p, r, s);
        if (e != hipSuccess)
            return e;
        a = {p.work, r.a_ld};
        type = kBf16;
    }
    hipError_t e;
    if (r.path == kTiles) {
        e = p.scale && r.splits == 1 ? launch_tiles<Store<true>>(p, r, a, q, parts, s)
                                     : launch_tiles<Store<false>>(p, r, a, q, parts, s);
    } else {
        SmallProduct g = {};
        g.a = a;
        g.q = p.q;
        g.nb = (uint32_t)mx_blocks(p.k);
        g.m = (uint32_t)r.m;
        g.n = (uint32_t)r.n;
        g.k = (uint32_t)r.k;
        g.tm = r.tm;
        g.tn = r.tn;
        g.slices = r.stages;
        g.cuts = r.splits;
        g.per = r.per;
        g.out = {p.c.p, p.c.ld, p.ctype, p.accumulate, p.scale};
        g.parts = parts;
        e = r.path == kDot ? launch_mx_dot(g, type, s) : launch_mx_small(g, p.op, type, r.tile, s);
    }
    return e == hipSuccess && r.splits > 1
               ? join(parts, r.splits, r.m, r.n, {p.c.p, p.c.ld, p.ctype, p.accumulate, p.scale}, s)
               : e;
}

uint64_t mx4_product_work(const Mx4Product &p, int num_cu)
{
    const Gemm4 g = plan4_of(p, num_cu);
    return g.splits > 1 ? (uint64_t)g.splits * p.m * p.n * 4 : 0;
}

hipError_t launch_mx4_product(const Mx4Product &p, int num_cu, hipStream_t s)
{
    Gemm4 g = plan4_of(p, num_cu);
    if (p.m == 0 || p.n == 0)
        return hipSuccess;
    g.c = p.c.p;
    g.ldc = p.c.ld;
    g.ctype = p.ctype;
    g.parts = reinterpret_cast<float *>(p.work);
    const dim3 grid(g.tm * g.tn * g.splits);
    if (g.tile == 256)
        hipLaunchKernelGGL((gemm4_kernel<4>), grid, dim3(kThreads), 0, s, g);
    else
        hipLaunchKernelGGL((gemm4_kernel<2>), grid, dim3(kThreads), 0, s, g);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess && g.splits > 1 ? join(g.parts, g.splits, p.m, p.n, {p.c.p, p.c.ld, p.ctype, 0, nullptr}, s) : e;
}

}  // namespace fastrack
