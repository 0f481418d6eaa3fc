// Softmax cross entropy over a vocabulary whose head is an MX4 matrix, in pieces of the vocabulary:
// the logits are never kept. Forwards a piece's logits leave their largest value and the sum of
// their exponentials behind; backwards they are computed again, become the logits' gradient, and
// that is multiplied into the gradients of x and of the head.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "launch.h"
#include "mx_dev.h"
#include "mx_gemm_dev.h"
#include "mx_model.h"

namespace fastrack {
namespace mx {

constexpr int kThreads = 256;

__device__ __forceinline__ int64_t id_of(const MxIds &ids, uint64_t i)
{
    return ids.wide ? reinterpret_cast<const int64_t *>(ids.p)[i] : reinterpret_cast<const int32_t *>(ids.p)[i];
}

// A largest value and the sum of exponentials over it. An infinite largest value stands for none: e^z
// itself is summed then, which is 0 for -inf and inf for inf.
struct Stat {
    float top, sum;
};

__device__ __forceinline__ float base_of(float top) { return __builtin_fabsf(top) == __builtin_inff() ? 0.0f : top; }

// The larger one; NaN where either is (fmaxf would drop it).
__device__ __forceinline__ float larger(float a, float b) { return a > b || a != a ? a : b; }

__device__ __forceinline__ Stat join(const Stat &a, const Stat &b)
{
    const float top = larger(a.top, b.top), base = base_of(top);
    return {top, a.sum * expf(base_of(a.top) - base) + b.sum * expf(base_of(b.top) - base)};
}

struct Piece {
    const float *z;        // [m][n], unscaled
    uint32_t m, n;         // of this piece
    uint64_t v0;           // its first class
    float scale;
    MxIds ids;
    Stat *stats;           // [parts][m]
    float *label;          // [m]: the logit of the target
    uint32_t part0, parts; // of this piece
};

// One workgroup: kThreads * 8 classes of a row.
constexpr uint32_t kStatCols = kThreads * 8;

__global__ __launch_bounds__(kThreads) void stat_kernel(Piece g)
{
    __shared__ Stat lds[kThreads / 64];
    const uint32_t row = blockIdx.x / g.parts, part = blockIdx.x - row * g.parts, c = part * kStatCols + threadIdx.x * 8;
    Stat s = {-__builtin_inff(), 0.0f};
    if (c < g.n) {
        float v[8];
        load8<kFp32>(g.z, (uint64_t)row * g.n, c, g.n, v);
        const int64_t at = id_of(g.ids, row) - (int64_t)g.v0 - c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = c + i < g.n ? v[i] * g.scale : -__builtin_inff();
            s.top = larger(v[i], s.top);
            if (at == i && c + i < g.n)
                g.label[row] = v[i];
        }
        const float base = base_of(s.top);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            s.sum += expf(v[i] - base);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
        s = join(s, Stat{__shfl_xor(s.top, d, 64), __shfl_xor(s.sum, d, 64)});
    if (threadIdx.x % 64 == 0)
        lds[threadIdx.x / 64] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 64; ++w)
            s = join(s, lds[w]);
        g.stats[(uint64_t)(g.part0 + part) * g.m + row] = s;
    }
}

// The parts of 16 rows, in their order.
constexpr uint32_t kJoinRows = 16, kJoinLanes = kThreads / kJoinRows;

__global__ __launch_bounds__(kThreads) void loss_kernel(const Stat *stats, uint32_t parts, uint32_t m, uint32_t n, MxIds ids, const float *label,
                                                        float *loss, float *lse)
{
    __shared__ Stat lds[kJoinLanes][kJoinRows];
    const uint32_t r = threadIdx.x % kJoinRows, l = threadIdx.x / kJoinRows, row = blockIdx.x * kJoinRows + r;
    Stat s = {-__builtin_inff(), 0.0f};
    if (row < m)
        for (uint32_t p = l; p < parts; p += kJoinLanes)
            s = join(s, stats[(uint64_t)p * m + row]);
    lds[l][r] = s;
    __syncthreads();
    if (l == 0 && row < m) {
        for (uint32_t i = 1; i < kJoinLanes; ++i)
            s = join(s, lds[i][r]);
        const int64_t id = id_of(ids, row);
        // A target that is no class makes what comes of it a NaN.
        const float v = id >= (int64_t)n ? __builtin_nanf("") : base_of(s.top) + logf(s.sum);
        lse[row] = v;
        loss[row] = id < 0 ? 0.0f : v - label[row];
    }
}

// The logits' gradient, dloss (e^(z - lse) - [class = target]) times the scale, in rows of ld values
// that end in zeros.
struct Slope {
    const float *z;
    uint32_t m, n, per_row, recip;
    uint64_t row0, v0, ld;
    float scale;
    MxIds ids;
    const float *lse, *dloss;
    uint64_t dloss_step;
    void *dz;
};

__device__ __forceinline__ float slope(float z, float lse, float factor, bool target)
{
    return factor * (expf(z - lse) - (target ? 1.0f : 0.0f));
}

template <uint32_t T>
__global__ __launch_bounds__(kThreads) void slope_kernel(Slope g)
{
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x, r = div_recip(i, g.per_row, g.recip), c = (i - r * g.per_row) * 8;
    const uint64_t row = g.row0 + r;
    if (row >= g.m)
        return;
    float v[8];
    load8<kFp32>(g.z, row * g.n, c, g.n, v);
    const int64_t id = id_of(g.ids, row), at = id - (int64_t)g.v0 - c;
    const float lse = g.lse[row], factor = g.dloss[row * g.dloss_step] * g.scale;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        v[j] = id < 0 || c + j >= g.n ? 0.0f : slope(v[j] * g.scale, lse, factor, at == j);
    store8<T>(g.dz, row * g.ld, c, (uint32_t)g.ld, v);
}

// The result in its own type.
__global__ __launch_bounds__(kThreads) void round_kernel(const float *v, uint32_t m, uint32_t n, uint32_t per_row, uint32_t recip, uint64_t row0, Out o)
{
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x, r = div_recip(i, per_row, recip), c = (i - r * per_row) * 8;
    const uint64_t row = row0 + r;
    if (row >= m)
        return;
    float w[8];
    load8<kFp32>(v, row * n, c, n, w);
    put8(o, (uint32_t)row, c, n, w);
}

// launch(first row, threads) over rows of per_row threads, fewer than 2^32 in a launch.
template <class F>
hipError_t over(uint64_t rows, uint32_t per_row, F launch)
{
    const uint64_t most = 0xFFFFFF00u / per_row;
    for (uint64_t r = 0; r < rows; r += most) {
        const uint64_t left = rows - r < most ? rows - r : most;
        launch(r, dim3((uint32_t)((left * per_row + kThreads - 1) / kThreads)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

uint64_t round_to(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

// Classes of a piece, whole tiles of 256: 2^26 logits, which lie in the workspace.
constexpr uint64_t kPieceValues = 1ull << 26;
uint64_t piece_of(const Loss &l)
{
    const uint64_t most = round_to(l.n, 256), v = kPieceValues / (l.m ? l.m : 1) / 256 * 256;
    return v < 256 ? 256 : v < most ? v : most;
}

// Type of the logits' gradient: in 16 bits where that is what both results are rounded to.
uint32_t slope_type(const Loss &l)
{
    const bool x = !l.dx.p || l.dx_type == kBf16, w = !l.x8.codes || l.dw_type == kBf16;
    return x && w ? kBf16 : kFp32;
}

MxProduct logits(const Loss &l, uint64_t v0, uint64_t n, float *z)
{
    MxProduct p = {};
    const uint64_t nb = mx_blocks(l.k);
    p.op = kLinear;
    p.type = l.type;
    p.a = l.x;
    p.q = {l.w.codes + v0 * nb * 16, l.w.scales + v0 * nb};
    p.m = l.m, p.n = n, p.k = l.k;
    p.ctype = kFp32;
    p.c = {z, n};
    return p;
}

struct LossPlan {
    uint64_t piece, parts;
    uint64_t z, stats, label, product;   // bytes
    uint64_t dz, dx;
    uint64_t bytes() const { return z + stats + label + product + dz + dx; }
};

}  // namespace mx

using namespace mx;

namespace {

// What products of whole pieces and of the last one need.
template <class F>
uint64_t most_of(const Loss &l, uint64_t piece, F product, int num_cu)
{
    uint64_t most = 0;
    for (uint64_t n : {piece < l.n ? piece : l.n, l.n % piece ? l.n % piece : piece}) {
        const uint64_t need = mx_product_work(product(n), num_cu);
        most = need > most ? need : most;
    }
    return round_to(most, 256);
}

LossPlan plan_of(const Loss &l, int num_cu)
{
    LossPlan p = {};
    p.piece = piece_of(l);
    const uint64_t n = p.piece < l.n ? p.piece : l.n;
    p.parts = l.n / p.piece * ((p.piece + kStatCols - 1) / kStatCols) + (l.n % p.piece + kStatCols - 1) / kStatCols;
    p.z = round_to(l.m * n * 4, 256);
    p.stats = round_to(p.parts * l.m * sizeof(Stat), 256);
    p.label = round_to(l.m * 4, 256);
    p.product = most_of(l, p.piece, [&](uint64_t w) { return logits(l, 0, w, nullptr); }, num_cu);
    return p;
}

MxProduct back_x(const Loss &l, uint64_t v0, uint64_t n, void *dz, uint32_t type, uint64_t ld, const Out &o)
{
    MxProduct p = logits(l, v0, n, nullptr);
    p.op = kGradInput;
    p.type = type;
    p.a = {dz, ld};
    p.c = {o.p, o.ld};
    p.ctype = o.type;
    p.accumulate = o.accumulate;
    return p;
}

MxProduct back_w(const Loss &l, uint64_t v0, uint64_t n, void *dz, uint32_t type, uint64_t ld)
{
    MxProduct p = {};
    p.op = kWeightGrad;
    p.type = type;
    p.a = {dz, ld};
    p.q = l.x8;
    p.m = l.m, p.n = n, p.k = l.k;
    p.ctype = l.dw_type;
    p.c = {reinterpret_cast<uint8_t *>(l.dw.p) + v0 * l.dw.ld * mx_type_size(l.dw_type), l.dw.ld};
    p.accumulate = l.accumulate;
    return p;
}

// An address for a plan that asks where its float operand lies.
void *some_place() { return reinterpret_cast<void *>(256); }

LossPlan grad_plan_of(const Loss &l, int num_cu)
{
    LossPlan p = plan_of(l, num_cu);
    p.stats = p.label = 0;
    const uint32_t type = slope_type(l);
    const uint64_t n = p.piece < l.n ? p.piece : l.n;
    p.dz = round_to(l.m * round_to(n, 8) * mx_type_size(type), 256);
    p.dx = l.dx.p && l.dx_type != kFp32 && p.piece < l.n ? round_to(l.m * l.k * 4, 256) : 0;
    const uint64_t x = most_of(l, p.piece, [&](uint64_t w) { return back_x(l, 0, w, some_place(), type, round_to(w, 8), {}); }, num_cu);
    const uint64_t w = most_of(l, p.piece, [&](uint64_t w) { return back_w(l, 0, w, some_place(), type, round_to(w, 8)); }, num_cu);
    p.product = p.product > x ? p.product : x;
    p.product = p.product > w ? p.product : w;
    return p;
}

}  // namespace

uint64_t mx_loss_work(const Loss &l, int num_cu) { return l.m && l.n ? plan_of(l, num_cu).bytes() : 0; }

uint64_t mx_loss_grad_work(const Loss &l, int num_cu) { return l.m && l.n ? grad_plan_of(l, num_cu).bytes() : 0; }

static hipError_t multiply(MxProduct p, uint8_t *work, uint64_t bytes, int num_cu, hipStream_t s)
{
    p.work = work;
    p.work_bytes = bytes;
    return launch_mx_product(p, num_cu, s);
}

hipError_t launch_mx_loss(const Loss &l, int num_cu, hipStream_t s)
{
    if (l.m == 0)
        return hipSuccess;
    const LossPlan p = plan_of(l, num_cu);
    uint8_t *const work = reinterpret_cast<uint8_t *>(l.work);
    Piece g = {};
    g.z = reinterpret_cast<float *>(work + p.product);
    g.stats = reinterpret_cast<Stat *>(work + p.product + p.z);
    g.label = reinterpret_cast<float *>(work + p.product + p.z + p.stats);
    g.m = (uint32_t)l.m;
    g.scale = l.scale;
    g.ids = l.ids;
    for (g.v0 = 0; g.v0 < l.n; g.v0 += p.piece, g.part0 += g.parts) {
        g.n = (uint32_t)(l.n - g.v0 < p.piece ? l.n - g.v0 : p.piece);
        g.parts = (g.n + kStatCols - 1) / kStatCols;
        hipError_t e = multiply(logits(l, g.v0, g.n, const_cast<float *>(g.z)), work, p.product, num_cu, s);
        if (e != hipSuccess)
            return e;
        hipLaunchKernelGGL(stat_kernel, dim3(g.m * g.parts), dim3(kThreads), 0, s, g);
        if ((e = hipGetLastError()) != hipSuccess)
            return e;
    }
    hipLaunchKernelGGL(loss_kernel, dim3((g.m + kJoinRows - 1) / kJoinRows), dim3(kThreads), 0, s, g.stats, g.part0, g.m, (uint32_t)l.n, l.ids,
                       g.label, l.loss, l.lse);
    return hipGetLastError();
}

hipError_t launch_mx_loss_grad(const Loss &l, int num_cu, hipStream_t s)
{
    if (l.n == 0)
        return hipSuccess;
    hipError_t e;
    if (l.m == 0)   // no tokens: a head's gradient of zeros, or the one that is there
        return l.x8.codes ? multiply(back_w(l, 0, l.n, nullptr, kBf16, l.n), nullptr, 0, num_cu, s) : hipSuccess;
    const LossPlan p = grad_plan_of(l, num_cu);
    const uint32_t type = slope_type(l);
    uint8_t *const work = reinterpret_cast<uint8_t *>(l.work);
    Slope g = {};
    g.z = reinterpret_cast<float *>(work + p.product);
    g.dz = work + p.product + p.z;
    float *const dx = reinterpret_cast<float *>(work + p.product + p.z + p.dz);
    g.m = (uint32_t)l.m;
    g.scale = l.scale;
    g.ids = l.ids;
    g.lse = l.lse;
    g.dloss = l.dloss;
    g.dloss_step = l.dloss_step;
    for (g.v0 = 0; g.v0 < l.n; g.v0 += p.piece) {
        g.n = (uint32_t)(l.n - g.v0 < p.piece ? l.n - g.v0 : p.piece);
        g.ld = round_to(g.n, 8);
        if ((e = multiply(logits(l, g.v0, g.n, const_cast<float *>(g.z)), work, p.product, num_cu, s)) != hipSuccess)
            return e;
        g.per_row = (uint32_t)(g.ld / 8);
        g.recip = div_recip_of(g.per_row);
        e = over(l.m, g.per_row, [&](uint64_t row0, dim3 grid) {
            g.row0 = row0;
            if (type == kBf16)
                hipLaunchKernelGGL((slope_kernel<kBf16>), grid, dim3(kThreads), 0, s, g);
            else
                hipLaunchKernelGGL((slope_kernel<kFp32>), grid, dim3(kThreads), 0, s, g);
        });
        if (e != hipSuccess)
            return e;
        if (l.dx.p) {
            const Out o = p.dx ? Out{dx, l.k, kFp32, g.v0 != 0} : Out{l.dx.p, l.dx.ld, l.dx_type, g.v0 != 0};
            if ((e = multiply(back_x(l, g.v0, g.n, g.dz, type, g.ld, o), work, p.product, num_cu, s)) != hipSuccess)
                return e;
        }
        if (l.x8.codes)
            if ((e = multiply(back_w(l, g.v0, g.n, g.dz, type, g.ld), work, p.product, num_cu, s)) != hipSuccess)
                return e;
    }
    if (!p.dx)
        return hipSuccess;
    const uint32_t per_row = (uint32_t)((l.k + 7) / 8);
    return over(l.m, per_row, [&](uint64_t row0, dim3 grid) {
        hipLaunchKernelGGL(round_kernel, grid, dim3(kThreads), 0, s, dx, g.m, (uint32_t)l.k, per_row, div_recip_of(per_row), row0,
                           Out{l.dx.p, l.dx.ld, l.dx_type, 0});
    });
}

}  // namespace fastrack
