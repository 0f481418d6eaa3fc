// The norm between two blocks of a model, with what stands around it: the block's own norm, its
// gate, the residual and its scale. Forwards in one pass, with what the gradient needs kept in 8
// bits; backwards in one pass over that. Every value is read once and written once: what bounds it
// is HBM. 4096 rows of 8192 of bf16 with a norm, a gate and a residual: forwards 438 MB in 97-99 us,
// 4.4-4.5 TB/s (the VALU busy half of it), backwards 439 MB in 96-99 and 5 for the weights' sums; a
// device copy runs at 5.2.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "launch.h"
#include "mx_dev.h"
#include "mx_model.h"

namespace fastrack {
namespace mx {

// A row is shared by G threads: unit j of 8 columns belongs to thread j % G, U of them to a thread,
// which stay in its registers from the row's sum to its end. U = 0: rows of any length, read again
// after each sum.
template <int G> constexpr int threads_of() { return G < 128 ? 256 : G; }

// Which of a workgroup's rows is this thread's: the same for a whole wave, so that addresses are
// computed once for it.
template <int G>
__device__ __forceinline__ uint32_t part_of()
{
    return threads_of<G>() == G ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / G);
}

// The sum over the G threads of a row, to all of them. `slot` takes turns between 0 and 1: what one
// sum leaves in LDS is read until the next one's barrier.
template <int G>
__device__ __forceinline__ float row_sum(float v, float (*lds)[16], int slot)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
        v += __shfl_xor(v, d, 64);
    if (G > 64) {
        if (threadIdx.x % 64 == 0)
            lds[slot][threadIdx.x / 64] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < G / 64; ++w)
            v += lds[slot][w];
    }
    return v;
}

template <uint32_t T>
__device__ __forceinline__ void row8(const void *p, uint64_t row_off, uint32_t c, uint32_t cols, float (&v)[8])
{
    Raw8<T> r;
    r.load(p, row_off, c, cols);
    r.settle(c, cols);
    r.floats(v);
}

// Eight of a weight vector, in the rows' type or in 32 bits.
template <uint32_t T>
__device__ __forceinline__ void weights8(const void *w, uint32_t wtype, uint32_t c, uint32_t cols, float (&v)[8])
{
    if (T != kFp32 && wtype == kFp32)
        row8<kFp32>(w, 0, c, cols, v);
    else
        row8<T>(w, 0, c, cols, v);
}

__device__ __forceinline__ Unit unit_at(uint64_t row, uint32_t j, uint32_t units)
{
    return {row, j * 8, row * (units / 4) + j / 4, j & 3};
}

__device__ __forceinline__ float square_sum(const float (&v)[8])
{
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        s = __builtin_fmaf(v[i], v[i], s);
    return s;
}

// 1 / rms as the float next to it and what that leaves, from a row's threads' sums of squares. Those are
// in 32 bits, what is made of them in 64: a row's error would be in all of its values alike, and a
// value next to the border of two of its 8 bits' codes would go to the other one.
struct Inverse {
    float hi, lo;
    __device__ __forceinline__ float times(float v) const { return __builtin_fmaf(v, hi, v * lo); }
};

template <int G>
__device__ __forceinline__ Inverse inverse_rms(float squares, uint32_t cols, float eps, double (*lds)[16], int slot)
{
    double s = (double)squares;
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
        s += __shfl_xor(s, d, 64);
    if (G > 64) {
        if (threadIdx.x % 64 == 0)
            lds[slot][threadIdx.x / 64] = s;
        __syncthreads();
        s = 0.0;
#pragma unroll
        for (int w = 0; w < G / 64; ++w)
            s += lds[slot][w];
    }
    const double mean = s / (double)cols + (double)eps;
    // A Newton step of 1 / sqrt takes 32 bits' error to its square.
    const double near = (double)(1.0f / sqrtf((float)mean)), inv = near * (1.5 - 0.5 * mean * near * near);
    // (0, infinity and NaN as the first value has them)
    const float hi = near > 0.0 && near < (double)__builtin_inff() ? (float)inv : (float)near, lo = (float)(inv - (double)hi);
    return {hi, __builtin_fabsf(lo) < __builtin_fabsf(hi) ? lo : 0.0f};
}

template <uint32_t T, int G, int U>
__global__ __launch_bounds__(threads_of<G>()) void norm_kernel(Norm n, uint64_t row0)
{
    constexpr int N = U ? U : 1, R = threads_of<G>() / G;
    __shared__ double lds[2][16];
    const uint32_t t = threadIdx.x % G, cols = (uint32_t)n.cols, units = (uint32_t)(4 * mx_blocks(cols));
    const uint64_t row = row0 + (uint64_t)blockIdx.x * R + part_of<G>();
    if (row >= n.rows)   // (a whole wave, or a whole workgroup)
        return;
    auto each = [&](auto f) {
        if (U) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (t + i * G < units)
                    f(i, t + i * G);
        } else {
            for (uint32_t j = t; j < units; j += G)
                f(0, j);
        }
    };
    float h[N][8];
    Inverse inv1 = {1.0f, 0.0f};
    if (n.w1) {
        float s = 0.0f;
        each([&](int i, uint32_t j) {
            row8<T>(n.x.p, row * n.x.ld, j * 8, cols, h[i]);
            s += square_sum(h[i]);
        });
        inv1 = inverse_rms<G>(s, cols, n.eps, lds, 0);
        if (t == 0)
            n.inv1[row] = inv1.hi;
    }
    // h of a unit, and on the way (`keep`) what is kept of x and g.
    auto hidden = [&](int i, uint32_t j, bool keep) {
        const Unit u = unit_at(row, j, units);
        float f[8];
        if (!U || !n.w1)
            row8<T>(n.x.p, row * n.x.ld, u.c, cols, h[i]);
        if (n.w1)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                h[i][e] = inv1.times(h[i][e]);
        if (keep && n.v.codes)
            put<kMx8>(n.v, u, h[i]);
        if (n.w1) {
            weights8<T>(n.w1, n.wtype, u.c, cols, f);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                h[i][e] *= f[e];
        }
        if (n.g.p) {
            row8<T>(n.g.p, row * n.g.ld, u.c, cols, f);
            if (keep)
                put<kMx8>(n.gq, u, f);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                h[i][e] *= f[e];
        }
        if (n.r.p) {
            row8<T>(n.r.p, row * n.r.ld, u.c, cols, f);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                h[i][e] = __builtin_fmaf(h[i][e], n.scale, f[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                h[i][e] *= n.scale;
        }
    };
    float s = 0.0f;
    each([&](int i, uint32_t j) {
        hidden(i, j, true);
        s += square_sum(h[i]);
        if (n.h.p)
            store8<T>(n.h.p, row * n.h.ld, j * 8, cols, h[i]);
    });
    const Inverse inv2 = inverse_rms<G>(s, cols, n.eps, lds, 1);
    if (t == 0)
        n.inv2[row] = inv2.hi;
    each([&](int i, uint32_t j) {
        if (!U)
            hidden(i, j, false);
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            h[i][e] = inv2.times(h[i][e]);
        put<kMx8>(n.u, unit_at(row, j, units), h[i]);
        weights8<T>(n.w2, n.wtype, j * 8, cols, w);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            w[e] *= h[i][e];
        store8<T>(n.y.p, row * n.y.ld, j * 8, cols, w);
    });
}

// How rows of a length are shared out: threads of a row and units of a thread.
enum Way : int { kWave1, kWave, k128x1, k256x1, k256x2, k256x4, k512x1, k1024x1, k1024x2, k1024x4, kLoop };

// ---- backwards -----------------------------------------------------------------------------------
//
//   t = dy w2,  dh' = inv2 (t - u mean(t u)) + dh,  dw2 += dy u,  dr = dh'
//   db = scale dh',  dg = db (v w1),  db *= g,  dw1 += db v
//   dx = inv1 (db w1 - v mean(db w1 v))
// A group takes every P-th row and adds up its rows' parts of dw2 and dw1, in registers; the groups'
// sums are added in their order by columns_kernel. The next row is on its way from memory while
// one is worked on.

// What a thread reads of a row, as it lies in memory.
template <uint32_t T>
struct GradRow {
    Raw8<T> dy, dh;
    u32x2 u, v, g;
    uint8_t eu, ev, eg;
};

template <uint32_t T, int G, int U>
__global__ __launch_bounds__(threads_of<G>(), 4) void norm_grad_kernel(NormGrad n, uint32_t groups)
{
    constexpr int R = threads_of<G>() / G;
    // Two units leave no registers for a second row, for the weights, nor for the sums: these are in LDS.
    constexpr bool AHEAD = U == 1;
    __shared__ float lds[2][16];
    __shared__ f32x4 sums[AHEAD ? 1 : 2][AHEAD ? 1 : 2][AHEAD ? 1 : U * G];   // of dw2, dw1; halves of a unit
    const uint32_t t = threadIdx.x % G, cols = (uint32_t)n.cols, units = (uint32_t)(4 * mx_blocks(cols));
    const uint32_t group = blockIdx.x * R + part_of<G>();
    if (group >= groups)
        return;
    auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (t + i * G < units)
                f(i, t + i * G);
    };
    float sum2[U][8] = {}, sum1[U][8] = {}, w2[U][8], w1[U][8];
    if (!AHEAD)
        each([&](int, uint32_t j) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                sums[AHEAD ? 0 : k / 2][AHEAD ? 0 : k % 2][AHEAD ? 0 : j] = f32x4{0, 0, 0, 0};
        });
    // sum += x y, of the registers or of the LDS (each unit there is one thread's).
    auto add = [&](float (&sum)[8], int which, uint32_t j, const float (&x)[8], const float (&y)[8]) {
        if (AHEAD) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                sum[e] = __builtin_fmaf(x[e], y[e], sum[e]);
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4 &at = sums[AHEAD ? 0 : which][AHEAD ? 0 : h][AHEAD ? 0 : j];
                f32x4 v = at;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = __builtin_fmaf(x[4 * h + e], y[4 * h + e], v[e]);
                at = v;
            }
        }
    };
    auto weights = [&](int i, uint32_t j) {
        weights8<T>(n.w2, n.wtype, j * 8, cols, w2[i]);
        if (n.w1)
            weights8<T>(n.w1, n.wtype, j * 8, cols, w1[i]);
    };
    if (AHEAD)
        each(weights);
    auto fetch_first = [&](uint64_t row, GradRow<T> (&r)[U]) {
        each([&](int i, uint32_t j) {
            const Unit u = unit_at(row, j, units);
            r[i].dy.load(n.dy.p, row * n.dy.ld, u.c, cols);
            r[i].u = reinterpret_cast<const u32x2 *>(n.u.codes)[u.block * 4 + u.lane];
            r[i].eu = n.u.scales[u.block];
        });
    };
    auto fetch_rest = [&](uint64_t row, GradRow<T> &r, uint32_t j) {
        const Unit u = unit_at(row, j, units);
        if (n.dh.p)
            r.dh.load(n.dh.p, row * n.dh.ld, u.c, cols);
        if (n.v.codes) {
            r.v = reinterpret_cast<const u32x2 *>(n.v.codes)[u.block * 4 + u.lane];
            r.ev = n.v.scales[u.block];
        }
        if (n.gq.codes) {
            r.g = reinterpret_cast<const u32x2 *>(n.gq.codes)[u.block * 4 + u.lane];
            r.eg = n.gq.scales[u.block];
        }
    };
    GradRow<T> now[U], next[U];
    if (AHEAD && group < n.rows) {
        fetch_first(group, now);
        each([&](int i, uint32_t j) { fetch_rest(group, now[i], j); });
    }
    for (uint64_t row = group; row < n.rows; row += groups) {
        const float inv2 = n.inv2[row], inv1 = n.w1 ? n.inv1[row] : 0.0f;
        if (AHEAD && row + groups < n.rows) {
            fetch_first(row + groups, next);
            each([&](int i, uint32_t j) { fetch_rest(row + groups, next[i], j); });
        }
        float d[U][8], a[U][8];   // dy w2 and then what goes on; u and then v
        float s = 0.0f;
        each([&](int i, uint32_t j) {
            if (!AHEAD)
                weights8<T>(n.w2, n.wtype, j * 8, cols, w2[i]);
            if (AHEAD) {
                decode8_f32(now[i].u, scale8_f32(now[i].eu), a[i]);
                now[i].dy.settle(j * 8, cols);
                now[i].dy.floats(d[i]);
            } else {
                get<kMx8>(n.u, unit_at(row, j, units), a[i]);
                load8<T>(n.dy.p, row * n.dy.ld, j * 8, cols, d[i]);
            }
            add(sum2[i], 0, j, d[i], a[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                d[i][e] *= w2[i][e];
                s = __builtin_fmaf(d[i][e], a[i][e], s);
            }
        });
        const float along2 = row_sum<G>(s, lds, 0) / (float)cols;
        s = 0.0f;
        each([&](int i, uint32_t j) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                d[i][e] = inv2 * __builtin_fmaf(-along2, a[i][e], d[i][e]);
            if (n.dh.p) {
                float f[8];
                if (AHEAD) {
                    now[i].dh.settle(j * 8, cols);
                    now[i].dh.floats(f);
                } else {
                    load8<T>(n.dh.p, row * n.dh.ld, j * 8, cols, f);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    d[i][e] += f[e];
            }
            if (n.dr.p)
                store8<T>(n.dr.p, row * n.dr.ld, j * 8, cols, d[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                d[i][e] *= n.scale;
            if (n.v.codes) {
                if (AHEAD)
                    decode8_f32(now[i].v, scale8_f32(now[i].ev), a[i]);
                else
                    get<kMx8>(n.v, unit_at(row, j, units), a[i]);
            }
            if (!AHEAD && n.w1)
                weights8<T>(n.w1, n.wtype, j * 8, cols, w1[i]);
            if (n.gq.codes) {
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    f[e] = d[i][e] * (n.w1 ? a[i][e] * w1[i][e] : a[i][e]);
                store8<T>(n.dg.p, row * n.dg.ld, j * 8, cols, f);
                if (AHEAD)
                    decode8_f32(now[i].g, scale8_f32(now[i].eg), f);
                else
                    get<kMx8>(n.gq, unit_at(row, j, units), f);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    d[i][e] *= f[e];
            }
            if (!n.w1) {
                store8<T>(n.dx.p, row * n.dx.ld, j * 8, cols, d[i]);
                return;
            }
            add(sum1[i], 1, j, d[i], a[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                d[i][e] *= w1[i][e];
                s = __builtin_fmaf(d[i][e], a[i][e], s);
            }
        });
        if (n.w1) {
            const float along1 = row_sum<G>(s, lds, 1) / (float)cols;
            each([&](int i, uint32_t j) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    d[i][e] = inv1 * __builtin_fmaf(-along1, a[i][e], d[i][e]);
                store8<T>(n.dx.p, row * n.dx.ld, j * 8, cols, d[i]);
            });
        } else if (G > 64) {
            __syncthreads();   // (the next row's sum goes to the same place of the LDS)
        }
        if (AHEAD)
            now[0] = next[0];
    }
    float *const part2 = n.work + (uint64_t)group * cols, *const part1 = part2 + (uint64_t)groups * cols;
    each([&](int i, uint32_t j) {
        if (!AHEAD)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sum2[i][e] = sums[0][AHEAD ? 0 : e / 4][AHEAD ? 0 : j][e % 4];
                sum1[i][e] = sums[AHEAD ? 0 : 1][AHEAD ? 0 : e / 4][AHEAD ? 0 : j][e % 4];
            }
        store8<kFp32>(part2, 0, j * 8, cols, sum2[i]);
        if (n.w1)
            store8<kFp32>(part1, 0, j * 8, cols, sum1[i]);
    });
}

// Rows of any length: read again after each sum, and a group's sums of dw2 and dw1 kept in its part of
// the workspace.
template <uint32_t T>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(NormGrad n, uint32_t groups)
{
    __shared__ float lds[2][16];
    const uint32_t cols = (uint32_t)n.cols, units = (uint32_t)(4 * mx_blocks(cols)), group = blockIdx.x;
    float *const part2 = n.work + (uint64_t)group * cols, *const part1 = part2 + (uint64_t)groups * cols;
    auto add = [&](float *part, uint32_t j, const float (&x)[8], const float (&y)[8], bool first) {
        float s[8] = {};
        if (!first)
            load8<kFp32>(part, 0, j * 8, cols, s);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            s[e] = __builtin_fmaf(x[e], y[e], s[e]);
        store8<kFp32>(part, 0, j * 8, cols, s);
    };
    bool first = true;
    for (uint64_t row = group; row < n.rows; row += groups, first = false) {
        const float inv2 = n.inv2[row], inv1 = n.w1 ? n.inv1[row] : 0.0f;
        float along2 = 0.0f, d[8], a[8], w[8], s = 0.0f;
        auto begin = [&](uint32_t j, bool sums) {   // d = dy w2, a = u
            const Unit u = unit_at(row, j, units);
            row8<T>(n.dy.p, row * n.dy.ld, u.c, cols, d);
            get<kMx8>(n.u, u, a);
            weights8<T>(n.w2, n.wtype, u.c, cols, w);
            if (sums)
                add(part2, j, d, a, first);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                d[e] *= w[e];
        };
        auto middle = [&](uint32_t j, bool out) {   // d = db, without w1; a = v; w = w1
            const Unit u = unit_at(row, j, units);
            float f[8] = {};
            begin(j, false);
            if (n.dh.p)
                row8<T>(n.dh.p, row * n.dh.ld, u.c, cols, f);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                d[e] = inv2 * __builtin_fmaf(-along2, a[e], d[e]) + f[e];
            if (out && n.dr.p)
                store8<T>(n.dr.p, row * n.dr.ld, u.c, cols, d);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                d[e] *= n.scale;
            if (n.v.codes)
                get<kMx8>(n.v, u, a);
            if (n.w1)
                weights8<T>(n.w1, n.wtype, u.c, cols, w);
            if (n.gq.codes) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    f[e] = d[e] * (n.w1 ? a[e] * w[e] : a[e]);
                if (out)
                    store8<T>(n.dg.p, row * n.dg.ld, u.c, cols, f);
                get<kMx8>(n.gq, u, f);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    d[e] *= f[e];
            }
        };
        for (uint32_t j = threadIdx.x; j < units; j += 1024) {
            begin(j, true);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                s = __builtin_fmaf(d[e], a[e], s);
        }
        along2 = row_sum<1024>(s, lds, 0) / (float)cols;
        s = 0.0f;
        for (uint32_t j = threadIdx.x; j < units; j += 1024) {
            middle(j, true);
            if (!n.w1) {
                store8<T>(n.dx.p, row * n.dx.ld, j * 8, cols, d);
                continue;
            }
            add(part1, j, d, a, first);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                s = __builtin_fmaf(d[e] * w[e], a[e], s);
        }
        const float along1 = row_sum<1024>(s, lds, 1) / (float)cols;
        if (n.w1)
            for (uint32_t j = threadIdx.x; j < units; j += 1024) {
                middle(j, false);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    d[e] = inv1 * __builtin_fmaf(-along1, a[e], d[e] * w[e]);
                store8<T>(n.dx.p, row * n.dx.ld, j * 8, cols, d);
            }
    }
}

// Sums of 64 columns of `parts` rows, always in the same order: a wave takes every 16th row, the
// waves' sums are added in theirs. c0: the launch's first column.
__global__ __launch_bounds__(1024) void columns_kernel(const float *work, uint32_t parts, uint32_t cols, uint32_t c0, float *out0, float *out1)
{
    __shared__ float lds[16][64];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = c0 + blockIdx.x * 64 + lane;
    const float *p = work + (uint64_t)blockIdx.y * parts * cols;
    float s = 0.0f;
    if (c < cols)
#pragma unroll 8
        for (uint32_t r = wave; r < parts; r += 16)
            s += p[(uint64_t)r * cols + c];
    lds[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < cols) {
#pragma unroll
        for (int w = 1; w < 16; ++w)
            s += lds[w][lane];
        (blockIdx.y ? out1 : out0)[c] = s;
    }
}

}  // namespace mx

using namespace mx;

// Rows that fill the GPU: as few threads of a row as hold it (us, 4096 rows of bf16 with all operands: 1024
// columns a wave 13.7, 256 threads 17.3, 1024 42.8; 4096 columns 256 threads 43.6, 1024 66.4; 8192
// columns 96.7, 98.6). Few rows: more of them (1 row: 1024 columns a wave 6.5, 256 threads 5.1; 4096
// columns 256 threads 7.3, 1024 5.9; 8192 columns 11.5, 7.3; 100 rows of 2048 5.6, 6.0; 300 rows of 8192 16.1,
// 13.4).
static Way forward_way(uint64_t rows, uint64_t cols, int num_cu)
{
    const uint64_t units = 4 * mx_blocks(cols);
    if (units > 4096)
        return kLoop;
    if (units > 1024)
        return k1024x4;
    const bool few = rows < (uint64_t)num_cu;
    if (few ? units <= 256 : units <= 128)
        return few ? k256x1 : kWave;
    if (few || (units > 512 && rows <= 2 * (uint64_t)num_cu))
        return k1024x1;
    return units <= 256 ? k256x1 : units <= 512 ? k256x2 : k256x4;
}

hipError_t launch_mx_norm(const Norm &n, int num_cu, hipStream_t s)
{
    if (n.rows == 0 || n.cols == 0)
        return hipSuccess;
    const Way way = forward_way(n.rows, n.cols, num_cu);
    const uint64_t most = 1ull << 21;   // rows of a launch: fewer than 2^32 threads
    for (uint64_t row0 = 0; row0 < n.rows; row0 += most) {
        Norm p = n;
        p.rows = n.rows - row0 < most ? n.rows : row0 + most;
        const uint64_t rows = p.rows - row0;
#define NORM(G, U)                                                                                                   \
    MX_TYPE(n.type, hipLaunchKernelGGL((norm_kernel<T, G, U>), dim3((uint32_t)((rows * G + threads_of<G>() - 1) / threads_of<G>())), \
                                       dim3(threads_of<G>()), 0, s, p, row0))
        switch (way) {
        case kWave: NORM(64, 2); break;
        case k256x1: NORM(256, 1); break;
        case k256x2: NORM(256, 2); break;
        case k256x4: NORM(256, 4); break;
        case k1024x1: NORM(1024, 1); break;
        case k1024x4: NORM(1024, 4); break;
        default: NORM(1024, 0); break;
        }
#undef NORM
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

// A unit to a thread, which leaves registers for the next row (4096 rows of 4096: 512 threads 50.8 us, 1024
// 60.9); two up to 16384 columns (2048 such rows: 142 us, read again after each sum 240).
static Way backward_way(uint64_t cols)
{
    const uint64_t units = 4 * mx_blocks(cols);
    return units <= 64 ? kWave1 : units <= 128 ? k128x1 : units <= 256 ? k256x1 : units <= 512 ? k512x1 : units <= 1024 ? k1024x1 : units <= 2048 ? k1024x2 : kLoop;
}

// Groups that take the rows in turn: as many as run at once, 16 waves to a CU; of short rows fewer, since
// each leaves sums behind (4096 rows of 512: 1024 groups 19.1 us, 2048 21.5, 4096 29.1).
static uint32_t groups_of(uint64_t rows, uint64_t cols, int num_cu)
{
    const Way way = backward_way(cols);
    const uint64_t most = (uint64_t)num_cu * (way == k512x1 ? 2 : way == k1024x1 || way == k1024x2 || way == kLoop ? 1 : 4);
    return (uint32_t)(rows < most ? rows : most);
}

uint64_t mx_norm_grad_work(uint64_t rows, uint64_t cols, bool w1, int num_cu)
{
    return (uint64_t)groups_of(rows, cols, num_cu) * cols * (w1 ? 2 : 1);
}

hipError_t launch_mx_norm_grad(const NormGrad &n, int num_cu, hipStream_t s)
{
    if (n.cols == 0)
        return hipSuccess;
    const uint32_t groups = groups_of(n.rows, n.cols, num_cu);
    if (groups) {
#define NORM(G, U)                                                                                                        \
    MX_TYPE(n.type, hipLaunchKernelGGL((norm_grad_kernel<T, G, U>), dim3((groups * G + threads_of<G>() - 1) / threads_of<G>()), \
                                       dim3(threads_of<G>()), 0, s, n, groups))
        switch (backward_way(n.cols)) {
        case kWave1: NORM(64, 1); break;
        case k128x1: NORM(128, 1); break;
        case k256x1: NORM(256, 1); break;
        case k512x1: NORM(512, 1); break;
        case k1024x1: NORM(1024, 1); break;
        case k1024x2: NORM(1024, 2); break;
        default: MX_TYPE(n.type, hipLaunchKernelGGL((norm_grad_long_kernel<T>), dim3(groups), dim3(1024), 0, s, n, groups)); break;
        }
#undef NORM
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    const uint64_t most = 1ull << 26;   // columns of a launch: fewer than 2^32 threads for both weights
    for (uint64_t c0 = 0; c0 < n.cols; c0 += most) {
        const uint64_t c = n.cols - c0 < most ? n.cols - c0 : most;
        hipLaunchKernelGGL(columns_kernel, dim3((uint32_t)((c + 63) / 64), n.w1 ? 2 : 1), dim3(1024), 0, s, n.work, groups,
                           (uint32_t)n.cols, (uint32_t)c0, n.dw2, n.dw1);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace fastrack
