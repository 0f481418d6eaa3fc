// Quantisation to and from the microscaled formats, and the activation that keeps its inputs
// in 8 bits, forwards and backwards. All of it streams: one pass, every input read once and
// every output written once.
//
// Work is cut into units of 8 values; four neighbouring lanes hold a block of 32 and share
// its largest magnitude by two lane exchanges, so no value is read twice and nothing goes
// through LDS. What bounds it is HBM: 1 GiB of bf16 to MX4 in 223-258 us, back in 233-246 (5.3-6
// TB/s; a device copy of 1 GiB runs at 5.1); gated SiLU of 4096 x 16384 bf16 forwards 91-97 us and
// backwards 92-100 (5.8 TB/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "launch.h"
#include "mx.h"
#include "mx_dev.h"

namespace fastrack {
namespace mx {

constexpr int kThreads = 256;

// Where a thread's unit lies: units are numbered along the rows, 4 to a block.
struct Unit {
    uint64_t row;
    uint32_t c;      // first column
    uint64_t block;  // index of its block in the whole matrix
    uint32_t lane;   // which quarter of it
};

struct Shape {
    uint64_t row0;        // first row of this launch
    uint32_t units;       // of this launch, below 2^32
    uint32_t per_row;     // 4 blocks(cols)
    uint32_t recip;       // div_recip_of(per_row)
    uint32_t cols;
};

__device__ __forceinline__ bool unit_of(const Shape &sh, Unit &u)
{
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= sh.units)   // whole blocks: the four lanes of one leave together
        return false;
    const uint32_t r = div_recip(i, sh.per_row, sh.recip), j = i - r * sh.per_row;
    u.row = sh.row0 + r;
    u.c = j * 8;
    u.block = u.row * (sh.per_row / 4) + j / 4;
    u.lane = j & 3;
    return true;
}

template <uint32_t FMT>
__device__ __forceinline__ void put(const MxMatrix &q, const Unit &u, const float (&v)[8])
{
    const uint32_t e = block_scale<FMT>(block_top(v));
    if (FMT == kMx4)
        reinterpret_cast<uint32_t *>(q.codes)[u.block * 4 + u.lane] = encode4(v, e);
    else
        reinterpret_cast<u32x2 *>(q.codes)[u.block * 4 + u.lane] = encode8(v, e);
    if (u.lane == 0)
        q.scales[u.block] = (uint8_t)e;
}

template <uint32_t FMT>
__device__ __forceinline__ void get(const MxMatrix &q, const Unit &u, float (&v)[8])
{
    const uint32_t e = q.scales[u.block];
    if (FMT == kMx4)
        decode4_f32(reinterpret_cast<const uint32_t *>(q.codes)[u.block * 4 + u.lane], scale4_f32(e), v);
    else
        decode8_f32(reinterpret_cast<const u32x2 *>(q.codes)[u.block * 4 + u.lane], scale8_f32(e), v);
}

template <uint32_t FMT, uint32_t T>
__global__ __launch_bounds__(kThreads) void quantize_kernel(Shape sh, MxRows x, MxMatrix q)
{
    Unit u;
    if (!unit_of(sh, u))
        return;
    float v[8];
    load8<T>(x.p, u.row * x.ld, u.c, sh.cols, v);
    put<FMT>(q, u, v);
}

template <uint32_t FMT, uint32_t T>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(Shape sh, MxMatrix q, MxRows out)
{
    Unit u;
    if (!unit_of(sh, u))
        return;
    float v[8];
    get<FMT>(q, u, v);
    store8<T>(out.p, u.row * out.ld, u.c, sh.cols, v);
}

// The normal distribution above a >= 0, over e^(-a^2 / 2): a polynomial in t = 1 / (1 + c a) without a
// constant term, fitted for the least relative error over [0, 14.6] (2^-20.6 with 7 coefficients, 2^-28.5
// with 10). P of a negative x is that product and keeps its digits, where 1 + erf of it has none left
// from x = -5.5 down. (4096 x 16384 of bf16 with a gate: 97 us forwards and 101 backwards, with the
// library's erff 110 and 107, with its erfcf 133 and 137.)
template <bool FAST>
__device__ __forceinline__ float normal_tail(float a)
{
    constexpr int N = FAST ? 7 : 10;
    constexpr float c[10] = {FAST ? 0.105599828f : 0.0937371254f,   FAST ? 0.107836783f : 0.0940763354f,
                             FAST ? 0.0829465464f : 0.0853466466f,  FAST ? 0.142493442f : 0.0966654718f,
                             FAST ? -0.0663630813f : -0.00348356646f, FAST ? 0.195273235f : 0.207300872f,
                             FAST ? -0.0677870661f : -0.227627978f, 0.273647487f, -0.147487491f, 0.0278251003f};
    constexpr float k = FAST ? 0.265f : 0.235f;
    const float d = __builtin_fmaf(a, k, 1.0f);
    float t = __builtin_amdgcn_rcpf(d);
    if (!FAST) {   // the reciprocal's and d's own rounding, which count three times in the result
        const float low = __builtin_fmaf(a, k, 1.0f - d);
        t = __builtin_fmaf(t, __builtin_fmaf(-low, t, __builtin_fmaf(-d, t, 1.0f)), t);
    }
    float p = c[N - 1];
#pragma unroll
    for (int i = N - 2; i >= 0; --i)
        p = __builtin_fmaf(p, t, c[i]);
    return p * t;
}

// f and f' of the activation. FAST (16-bit types, whose own rounding is 2^-9 or 2^-12): the
// hardware's exponential and reciprocal, a few 2^-23 each.
template <uint32_t ACT, bool FAST>
__device__ __forceinline__ void act_of(float x, float &f, float &df)
{
    if (ACT == kSilu) {   // x s(x), s + x s (1 - s)
        const float d = 1.0f + (FAST ? __expf(-x) : expf(-x));
        const float s = FAST ? __builtin_amdgcn_rcpf(d) : 1.0f / d;
        f = x * s;
        df = s * (1.0f + x * (1.0f - s));
    } else {              // x P(x), P + x p(x); P the normal distribution, p its density
        const float a = fminf(__builtin_fabsf(x), 20.0f);   // (past which e is 0; a NaN goes on in x)
        constexpr float c = -0.7213475f, c_low = -9.629815e-9f;   // -log2(e) / 2
        const float sq = a * a, h = sq * c;
        float e = __builtin_amdgcn_exp2f(h);
        if (!FAST) {   // what the argument's roundings leave: a unit of it is worth as many as it is large
            const float low = __builtin_fmaf(sq, c_low, __builtin_fmaf(__builtin_fmaf(a, a, -sq), c, __builtin_fmaf(sq, c, -h)));
            e = __builtin_fmaf(e, low * 0.6931472f, e);
        }
        const float q = e * normal_tail<FAST>(a), P = x < 0.0f ? q : 1.0f - q;
        f = x * P;
        df = P + x * (e * 0.39894228f);
    }
}

template <uint32_t ACT, uint32_t T, bool GATE>
__global__ __launch_bounds__(kThreads) void act_kernel(Shape sh, MxRows x, MxRows gate, MxRows y, MxMatrix qx,
                                                       MxMatrix qg)
{
    Unit u;
    if (!unit_of(sh, u))
        return;
    float v[8], g[8], o[8];
    load8<T>(x.p, u.row * x.ld, u.c, sh.cols, v);
    if (GATE)
        load8<T>(gate.p, u.row * gate.ld, u.c, sh.cols, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float f, df;
        act_of<ACT, T != kFp32>(v[i], f, df);
        o[i] = GATE ? f * g[i] : f;
    }
    store8<T>(y.p, u.row * y.ld, u.c, sh.cols, o);
    put<kMx8>(qx, u, v);
    if (GATE)
        put<kMx8>(qg, u, g);
}

template <uint32_t ACT, uint32_t T, bool GATE>
__global__ __launch_bounds__(kThreads) void act_grad_kernel(Shape sh, MxRows dy, MxMatrix qx, MxMatrix qg, MxRows dx,
                                                            MxRows dgate)
{
    Unit u;
    if (!unit_of(sh, u))
        return;
    float v[8], g[8], d[8];
    load8<T>(dy.p, u.row * dy.ld, u.c, sh.cols, d);
    get<kMx8>(qx, u, v);
    if (GATE)
        get<kMx8>(qg, u, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float f, df;
        act_of<ACT, T != kFp32>(v[i], f, df);
        v[i] = GATE ? d[i] * g[i] * df : d[i] * df;
        g[i] = d[i] * f;
    }
    store8<T>(dx.p, u.row * dx.ld, u.c, sh.cols, v);
    if (GATE)
        store8<T>(dgate.p, u.row * dgate.ld, u.c, sh.cols, g);
}

// Calls launch(shape, grid) for row ranges of fewer than 2^32 units each.
template <class F>
hipError_t over_rows(uint64_t rows, uint64_t cols, F launch)
{
    if (rows == 0 || cols == 0)
        return hipSuccess;
    const uint32_t per_row = (uint32_t)(4 * mx_blocks(cols));
    const uint64_t most = 0xFFFFFF00u / per_row;   // the grid's last thread index stays below 2^32 too
    for (uint64_t r = 0; r < rows; r += most) {
        const uint64_t n = rows - r < most ? rows - r : most;
        const Shape sh = {r, (uint32_t)(n * per_row), per_row, div_recip_of(per_row), (uint32_t)cols};
        launch(sh, dim3((sh.units + kThreads - 1) / kThreads));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace mx

using namespace mx;

// A run-time choice as a template argument.
#define MX_BOOL(name, v, ...)                                                                      \
    do {                                                                                           \
        if (v) { constexpr bool name = true; __VA_ARGS__; }                                        \
        else { constexpr bool name = false; __VA_ARGS__; }                                         \
    } while (0)

hipError_t launch_mx_quantize(uint32_t fmt, uint32_t type, MxRows x, uint64_t rows, uint64_t cols, MxMatrix q,
                              hipStream_t s)
{
    return over_rows(rows, cols, [&](const Shape &sh, dim3 grid) {
        MX_TYPE(type, MX_BOOL(M4, fmt == kMx4, {
            constexpr uint32_t F = M4 ? kMx4 : kMx8;
            hipLaunchKernelGGL((quantize_kernel<F, T>), grid, dim3(kThreads), 0, s, sh, x, q);
        }));
    });
}

hipError_t launch_mx_dequantize(uint32_t fmt, uint32_t type, MxMatrix q, uint64_t rows, uint64_t cols, MxRows out,
                                hipStream_t s)
{
    return over_rows(rows, cols, [&](const Shape &sh, dim3 grid) {
        MX_TYPE(type, MX_BOOL(M4, fmt == kMx4, {
            constexpr uint32_t F = M4 ? kMx4 : kMx8;
            hipLaunchKernelGGL((dequantize_kernel<F, T>), grid, dim3(kThreads), 0, s, sh, q, out);
        }));
    });
}

hipError_t launch_mx_act(uint32_t act, uint32_t type, MxRows x, MxRows gate, uint64_t rows, uint64_t cols, MxRows y,
                         MxMatrix qx, MxMatrix qg, hipStream_t s)
{
    const bool has_gate = gate.p != nullptr;
    return over_rows(rows, cols, [&](const Shape &sh, dim3 grid) {
        MX_TYPE(type, MX_BOOL(GATE, has_gate, MX_BOOL(SILU, act == kSilu, {
            constexpr uint32_t A = SILU ? kSilu : kGelu;
            hipLaunchKernelGGL((act_kernel<A, T, GATE>), grid, dim3(kThreads), 0, s, sh, x, gate, y, qx, qg);
        })));
    });
}

hipError_t launch_mx_act_grad(uint32_t act, uint32_t type, MxRows dy, MxMatrix qx, MxMatrix qg, uint64_t rows,
                              uint64_t cols, MxRows dx, MxRows dgate, hipStream_t s)
{
    const bool has_gate = qg.codes != nullptr;
    return over_rows(rows, cols, [&](const Shape &sh, dim3 grid) {
        MX_TYPE(type, MX_BOOL(GATE, has_gate, MX_BOOL(SILU, act == kSilu, {
            constexpr uint32_t A = SILU ? kSilu : kGelu;
            hipLaunchKernelGGL((act_grad_kernel<A, T, GATE>), grid, dim3(kThreads), 0, s, sh, dy, qx, qg, dx,
                               dgate);
        })));
    });
}

}  // namespace fastrack
