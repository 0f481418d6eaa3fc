// Softmax cross entropy over a vocabulary whose head is an MX4 matrix, in pieces of the vocabulary:
// the logits are never kept. Forwards a piece's logits leave their largest value and the sum of
// their exponentials behind; backwards they are computed again, become the logits' gradient, and
// that is multiplied into the gradients of x and of the head.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "launch.h"
#include "mx_dev.h"
#include "mx_gemm_dev.h"
#include "mx_loss_dev.h"
#include "mx_model.h"

namespace fastrack {
namespace mx {

constexpr int kThreads = 256;

// A token's loss, from the largest logit and not from lse, whose rounding would be all that is left of a small one.
// (What the sum of an exponential of 1 and others is off may be on the other side of 1.) A target that is no class
// makes what comes of it a NaN.
__device__ __forceinline__ void put_loss(const Stat &s, int64_t id, uint32_t n, float label, uint32_t row, float *loss, float *lse)
{
    const bool wrong = id >= (int64_t)n;
    const float base = base_of(s.top), above = logf(s.sum), v = minus(base, label) + above;
    lse[row] = wrong ? __builtin_nanf("") : base + above;
    loss[row] = id < 0 ? 0.0f : wrong ? __builtin_nanf("") : v < 0.0f ? 0.0f : v;
}

// One workgroup: kThreads * 8 classes of a row.
constexpr uint32_t kStatCols = kThreads * 8;

__global__ __launch_bounds__(kThreads) void stat_kernel(const float *z, uint32_t m, uint32_t n, uint32_t parts, LossTile a)
{
    __shared__ Stat lds[kThreads / 64];
    const uint32_t row = blockIdx.x / parts, part = blockIdx.x - row * parts, c = part * kStatCols + threadIdx.x * 8;
    Stat s = {-__builtin_inff(), 0.0f};
    if (c < n) {
        float v[8];
        load8<kFp32>(z, (uint64_t)row * n, c, n, v);
        const int64_t at = id_of(a.ids, row) - (int64_t)a.v0 - c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = c + i < n ? v[i] * a.scale : -__builtin_inff();
            s.top = larger(v[i], s.top);
            if (at == i && c + i < n)
                a.label[row] = v[i];
        }
        const float base = base_of(s.top);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            s.sum += exp_of(minus(v[i], base));
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
        a.stats[(uint64_t)(a.part0 + part) * m + row] = s;
    }
}

// A whole row's loss at once, by one workgroup, where its logits are all there and not too many for it: a
// launch less. (1 token, the whole call: 8192 classes 16 us, in parts 19; 32768 20 and 19; 65536 40 and
// 31: one CU reads 256 KB in 15 us.)
constexpr uint32_t kRowThreads = 1024, kRowMost = 1u << 14;

__global__ __launch_bounds__(kRowThreads) void row_loss_kernel(const float *z, uint32_t n, float scale, MxIds ids, float *loss, float *lse)
{
    constexpr int K = 4;   // units of 8 on their way at once
    __shared__ Stat lds[kRowThreads / 64];
    const uint32_t row = blockIdx.x;
    const int64_t id = id_of(ids, row);
    const float *line = z + (uint64_t)row * n;
    Stat s = {-__builtin_inff(), 0.0f};
    for (uint32_t c0 = threadIdx.x * 8; c0 < n; c0 += kRowThreads * 8 * K) {
        float v[K][8];
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (c0 + k * kRowThreads * 8 < n)
                load8<kFp32>(line, 0, c0 + k * kRowThreads * 8, n, v[k]);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t c = c0 + k * kRowThreads * 8;
            if (c >= n)
                break;
            Stat u = {-__builtin_inff(), 0.0f};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[k][i] = c + i < n ? v[k][i] * scale : -__builtin_inff();
                u.top = larger(v[k][i], u.top);
            }
            const float base = base_of(u.top);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                u.sum += exp_of(minus(v[k][i], base));
            s = join(s, u);
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
        s = join(s, Stat{__shfl_xor(s.top, d, 64), __shfl_xor(s.sum, d, 64)});
    if (threadIdx.x % 64 == 0)
        lds[threadIdx.x / 64] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (uint32_t w = 1; w < kRowThreads / 64; ++w)
            s = join(s, lds[w]);
        put_loss(s, id, n, id >= 0 && id < (int64_t)n ? line[id] * scale : 0.0f, row, loss, lse);
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
        put_loss(s, id_of(ids, row), n, label[row], row, loss, lse);
    }
}

// The scales of the kept x as the head's gradient takes them: the smallest one where a token is left out. Its dz is
// 0, but 0 times the NaN that a block of its stands for (x of a padded or masked token is anything) would be in
// the sum.
struct Kept {
    const uint8_t *scales;   // [m][blocks]
    uint8_t *counted;        // null: they are there already, or no such gradient is wanted
    uint32_t blocks;
    __device__ __forceinline__ void count(uint64_t row, int64_t id, uint32_t b, uint32_t step) const
    {
        for (; b < blocks; b += step)
            counted[row * blocks + b] = id < 0 ? 0 : scales[row * blocks + b];
    }
};

// The logits' gradient, dloss (e^(z - lse) - [class = target]) times the scale, as bf16 terms in rows of
// a.ld values that end in zeros.
__global__ __launch_bounds__(kThreads) void slope_kernel(const float *z, uint32_t m, uint32_t n, uint32_t per_row, uint32_t recip, uint64_t row0,
                                                         LossTile a, Kept kept)
{
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x, r = div_recip(i, per_row, recip), c = (i - r * per_row) * 8;
    const uint64_t row = row0 + r;
    if (row >= m)
        return;
    float v[8];
    load8<kFp32>(z, row * n, c, n, v);
    const int64_t id = id_of(a.ids, row), at = id - (int64_t)a.v0 - c;
    const float lse = a.lse[row], factor = factor_of(a, row);
    if (kept.counted)
        kept.count(row, id, c / 8, per_row);
#pragma unroll
    for (int j = 0; j < 8; ++j)   // (a token that is left out: no gradient, whatever its logits are)
        v[j] = id < 0 || c + j >= n ? 0.0f
               : at == j           ? target_slope(minus(v[j] * a.scale, lse), factor)
                                   : slope(minus(v[j] * a.scale, lse), factor);
    put_terms(a.dz + row * a.ld + c, a.plane, a.terms, v);
}

// The factor dloss * scale that all tokens have in common (a mean's or a sum's loss) does not have to be
// in the logits' gradient: out[1], 255 / 128, stands there for it, and out[0] makes up for that in the
// results. A token's largest gradient is that of its target, p - 1 of the factor. Rounded to bf16 with
// whatever factor, all of them would be off by the same part, up to 2^-8, while the model is unsure
// (p near 0); of 255 / 128 itself nothing is lost, and of what lies below it least. Where the tokens have
// several factors (or one far from 1, or none) out is 1 and 0, and each is rounded with its own.
__device__ __forceinline__ void find_common(const LossTile &a, uint32_t m, float *out)
{
    constexpr uint32_t K = 8;   // tokens of a thread at a time
    const uint32_t t = threadIdx.x;
    __shared__ uint32_t first;
    if (t == 0)
        first = m;
    __syncthreads();
    // The first token that counts, by the way whether those beside it have its dloss. (A NaN differs from all.)
    uint32_t f = m;
    float want = 0.0f;
    int differ = 0;
    for (uint32_t i0 = 0; i0 < m && !differ; i0 += 1024 * K) {
        float v[K];
        bool counts[K];
#pragma unroll
        for (uint32_t k = 0; k < K; ++k) {
            const uint32_t i = i0 + k * 1024 + t;
            counts[k] = i < m && id_of(a.ids, i) >= 0;
            v[k] = i < m ? a.dloss[i * a.dloss_step] : 0.0f;
        }
        if (f == m) {   // (the same in all threads)
#pragma unroll
            for (int k = (int)K - 1; k >= 0; --k)
                if (counts[k])
                    f = i0 + k * 1024 + t;
            if (f < m)
                atomicMin(&first, f);
            __syncthreads();
            f = first;
            want = f < m ? a.dloss[f * a.dloss_step] : 0.0f;
        }
        int other = 0;
#pragma unroll
        for (uint32_t k = 0; k < K; ++k)
            other |= counts[k] && v[k] != want;
        differ = __syncthreads_or(other);
    }
    if (t == 0) {
        const float factor = want * a.scale, size = __builtin_fabsf(factor), common = 255.0f / 128.0f;
        const bool one = !differ && size >= 0x1p-100f && size <= 0x1p100f;
        out[0] = one ? factor / common : 1.0f;
        out[1] = one ? common : 0.0f;
    }
}

// What goes before whole tiles: the first workgroup finds the common factor (`out` null: none), the others
// see to the tokens that are left out, one to a wave.
__global__ __launch_bounds__(1024) void before_kernel(LossTile a, uint32_t m, float *out, Kept kept)
{
    const uint32_t finds = out ? 1 : 0;
    if (blockIdx.x < finds) {
        find_common(a, m, out);
        return;
    }
    const uint32_t row = (blockIdx.x - finds) * 16 + threadIdx.x / 64;
    if (row < m)
        kept.count(row, id_of(a.ids, row), threadIdx.x % 64, 64);
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
hipError_t over_rows(uint64_t rows, uint32_t per_row, F launch)
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

// Classes of a piece of `values` logits, whole tiles of 256.
uint64_t piece_of(const Loss &l, uint64_t values)
{
    const uint64_t most = round_to(l.n, 256), v = values / (l.m ? l.m : 1) / 256 * 256;
    return v < 256 ? 256 : v < most ? v : most;
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
    p.few = true;
    return p;
}

// How the logits of a piece's width run: in whole tiles, whose ends do the rest, or (0: few
// outputs) into the workspace and through a kernel of their own.
struct Width {
    uint64_t n;
    uint32_t tile;
};

struct LossPlan {
    uint64_t piece;
    Width whole, rest;                   // of a piece; of the last one, n = 0 if there is none of its own
    uint64_t product, z, stats, label, dz, dx, common, counted;   // bytes
    uint32_t terms_x, terms_w;           // bf16 terms of the logits' gradient that the products take
    const float *common_at;              // the results' factor (null: 1)
    uint8_t *counted_at;                 // the kept x's scales, of the tokens that count
    const Width &width(uint64_t left) const { return left >= whole.n ? whole : rest; }
    uint64_t bytes() const { return product + z + stats + label + dz + dx + common + counted; }
};

uint64_t parts_of(const Width &w) { return w.tile ? (w.n + w.tile - 1) / w.tile : (w.n + kStatCols - 1) / kStatCols; }

// bf16 terms of the logits' gradient for a result of this type. One for bf16, whose own rounding is as
// large; but of few tokens, whose errors do not even out, two.
uint32_t terms_of(uint32_t type, uint64_t m) { return type == kBf16 ? (m <= 32 ? 2 : 1) : type == kFp16 ? 2 : 3; }

}  // namespace mx

using namespace mx;

namespace {

// Values of a piece: forwards no more than a launch has tiles for; backwards so many that the products
// of a piece fill the GPU and their sums over it are long (4096 tokens, 4096 x 65536, us: 2^26 6750,
// 2^27 6580, 2^28, which is all of them, 6580). Logits that go through the workspace, half as many.
constexpr uint64_t kForwardValues = 1ull << 34, kBackwardValues = 1ull << 27, kWorkspaceValues = 1ull << 26;

LossPlan plan_of(const Loss &l, int num_cu, uint64_t values)
{
    LossPlan p = {};
    const bool tiles = mx_logits_tile(logits(l, 0, l.n, nullptr), num_cu) != 0;
    p.piece = piece_of(l, tiles ? values : kWorkspaceValues);
    p.whole.n = p.piece < l.n ? p.piece : l.n;
    p.rest.n = l.n % p.whole.n;
    for (Width *w : {&p.whole, &p.rest}) {
        if (w->n == 0)
            continue;
        const MxProduct z = logits(l, 0, w->n, nullptr);
        w->tile = mx_logits_tile(z, num_cu);
        const uint64_t need = round_to(mx_product_work(z, num_cu), 256), own = w->tile ? 0 : round_to(l.m * w->n * 4, 256);
        p.product = need > p.product ? need : p.product;
        p.z = own > p.z ? own : p.z;
    }
    return p;
}

LossPlan forward_plan(const Loss &l, int num_cu)
{
    LossPlan p = plan_of(l, num_cu, kForwardValues);
    const uint64_t parts = l.n / p.whole.n * parts_of(p.whole) + (p.rest.n ? parts_of(p.rest) : 0);
    p.stats = round_to(parts * l.m * sizeof(Stat), 256);
    p.label = round_to(l.m * 4, 256);
    return p;
}

// A product with the logits' gradient, of which it takes as many terms as its result needs.
MxProduct slopes(const Loss &l, const LossPlan &p, const Width &w, void *dz, uint32_t terms)
{
    MxProduct r = {};
    r.type = kBf16;
    r.terms = terms;
    r.a = {dz, round_to(w.n, 8)};
    r.plane = l.m * r.a.ld;
    r.m = l.m, r.n = w.n, r.k = l.k;
    r.scale = p.common_at;
    return r;
}

MxProduct back_x(const Loss &l, const LossPlan &p, const Width &w, uint64_t v0, void *dz, const Out &o)
{
    MxProduct r = slopes(l, p, w, dz, p.terms_x);
    r.op = kGradInput;
    r.q = logits(l, v0, w.n, nullptr).q;
    r.c = {o.p, o.ld};
    r.ctype = o.type;
    r.accumulate = o.accumulate;
    return r;
}

MxProduct back_w(const Loss &l, const LossPlan &p, const Width &w, uint64_t v0, void *dz)
{
    MxProduct r = slopes(l, p, w, dz, p.terms_w);
    r.op = kWeightGrad;
    r.q = {l.x8.codes, p.counted_at};
    r.ctype = l.dw_type;
    r.c = {reinterpret_cast<uint8_t *>(l.dw.p) + v0 * l.dw.ld * mx_type_size(l.dw_type), l.dw.ld};
    r.accumulate = l.accumulate;
    return r;
}

LossPlan backward_plan(const Loss &l, int num_cu)
{
    LossPlan p = plan_of(l, num_cu, kBackwardValues);
    p.terms_x = l.dx.p ? terms_of(l.dx_type, l.m) : 0;
    p.terms_w = l.x8.codes ? terms_of(l.dw_type, l.m) : 0;
    const uint32_t terms = p.terms_x > p.terms_w ? p.terms_x : p.terms_w;
    p.common = p.terms_x == 1 || p.terms_w == 1 ? 256 : 0;   // (more terms round nothing that counts)
    p.counted = l.x8.codes ? round_to(l.m * mx_blocks(l.k), 256) : 0;
    p.dx = l.dx.p && l.dx_type != kFp32 && p.whole.n < l.n ? round_to(l.m * l.k * 4, 256) : 0;
    void *const some_place = reinterpret_cast<void *>(256);   // (a plan asks where its float operand lies)
    for (const Width *w : {&p.whole, &p.rest}) {
        if (w->n == 0)
            continue;
        const uint64_t dz = round_to(l.m * round_to(w->n, 8) * 2 * terms, 256);
        p.dz = dz > p.dz ? dz : p.dz;
        const uint64_t x = l.dx.p ? round_to(mx_product_work(back_x(l, p, *w, 0, some_place, {}), num_cu), 256) : 0;
        const uint64_t g = l.x8.codes ? round_to(mx_product_work(back_w(l, p, *w, 0, some_place), num_cu), 256) : 0;
        p.product = x > p.product ? x : p.product;
        p.product = g > p.product ? g : p.product;
    }
    return p;
}

hipError_t multiply(MxProduct p, uint8_t *work, uint64_t bytes, int num_cu, hipStream_t s)
{
    p.work = work;
    p.work_bytes = bytes;
    return launch_mx_product(p, num_cu, s);
}

}  // namespace

uint64_t mx_loss_work(const Loss &l, int num_cu) { return l.m && l.n ? forward_plan(l, num_cu).bytes() : 0; }

uint64_t mx_loss_grad_work(const Loss &l, int num_cu) { return l.m && l.n ? backward_plan(l, num_cu).bytes() : 0; }

hipError_t launch_mx_loss(const Loss &l, int num_cu, hipStream_t s)
{
    if (l.m == 0)
        return hipSuccess;
    const LossPlan p = forward_plan(l, num_cu);
    uint8_t *const work = reinterpret_cast<uint8_t *>(l.work);
    float *const z = reinterpret_cast<float *>(work + p.product);
    LossTile t = {};
    t.ids = l.ids;
    t.scale = l.scale;
    t.stats = reinterpret_cast<Stat *>(work + p.product + p.z);
    t.label = reinterpret_cast<float *>(work + p.product + p.z + p.stats);
    bool laid_out = false;
    hipError_t e;
    while (t.v0 < l.n) {
        const Width &w = p.width(l.n - t.v0);
        MxProduct g = logits(l, t.v0, w.n, z);
        if (w.tile) {
            g.work = work;
            if ((e = launch_mx_logits_stats(g, t, laid_out, num_cu, s)) != hipSuccess)
                return e;
            laid_out = true;
        } else {
            if ((e = multiply(g, work, p.product, num_cu, s)) != hipSuccess)
                return e;
            if (l.n <= kRowMost && w.n == l.n) {
                hipLaunchKernelGGL(row_loss_kernel, dim3((uint32_t)l.m), dim3(kRowThreads), 0, s, z, (uint32_t)l.n, l.scale, l.ids, l.loss, l.lse);
                return hipGetLastError();
            }
            const uint32_t parts = (uint32_t)parts_of(w);
            hipLaunchKernelGGL(stat_kernel, dim3((uint32_t)l.m * parts), dim3(kThreads), 0, s, z, (uint32_t)l.m, (uint32_t)w.n, parts, t);
            if ((e = hipGetLastError()) != hipSuccess)
                return e;
        }
        t.part0 += (uint32_t)parts_of(w);
        t.v0 += w.n;
    }
    hipLaunchKernelGGL(loss_kernel, dim3((uint32_t)((l.m + kJoinRows - 1) / kJoinRows)), dim3(kThreads), 0, s, t.stats, t.part0, (uint32_t)l.m,
                       (uint32_t)l.n, l.ids, t.label, l.loss, l.lse);
    return hipGetLastError();
}

hipError_t launch_mx_loss_grad(const Loss &l, int num_cu, hipStream_t s)
{
    if (l.n == 0 || (!l.dx.p && !l.x8.codes))
        return hipSuccess;
    if (l.m == 0) {   // no tokens: a head's gradient of zeros, or the one that is there
        LossPlan p = {};
        p.terms_w = 1;
        return l.x8.codes ? multiply(back_w(l, p, {l.n, 0}, 0, nullptr), nullptr, 0, num_cu, s) : hipSuccess;
    }
    LossPlan p = backward_plan(l, num_cu);
    uint8_t *const work = reinterpret_cast<uint8_t *>(l.work);
    float *const z = reinterpret_cast<float *>(work + p.product);
    uint8_t *const dz = work + p.product + p.z;
    float *const dx = reinterpret_cast<float *>(dz + p.dz);
    uint8_t *const tail = dz + p.dz + p.dx;
    p.common_at = p.common ? reinterpret_cast<float *>(tail) : nullptr;
    p.counted_at = p.counted ? tail + p.common : nullptr;
    LossTile t = {};
    t.ids = l.ids;
    t.scale = l.scale;
    t.lse = l.lse;
    t.dloss = l.dloss;
    t.dloss_step = l.dloss_step;
    t.dz = reinterpret_cast<uint16_t *>(dz);
    t.terms = p.terms_x > p.terms_w ? p.terms_x : p.terms_w;
    Kept kept = {l.x8.scales, p.counted_at, (uint32_t)mx_blocks(l.k)};
    hipError_t e;
    // (slope_kernel looks at the tokens itself.)
    const uint32_t counts = p.counted && p.whole.tile ? (uint32_t)((l.m + 15) / 16) : 0;
    if (p.common || counts) {
        float *const common = p.common ? reinterpret_cast<float *>(tail) : nullptr;
        hipLaunchKernelGGL(before_kernel, dim3((common ? 1 : 0) + counts), dim3(1024), 0, s, t, (uint32_t)l.m, common, kept);
        if ((e = hipGetLastError()) != hipSuccess)
            return e;
    }
    if (counts)
        kept.counted = nullptr;
    t.common = p.common_at;
    for (; t.v0 < l.n; t.v0 += p.width(l.n - t.v0).n) {
        const Width &w = p.width(l.n - t.v0);
        MxProduct g = logits(l, t.v0, w.n, z);
        t.ld = round_to(w.n, 8);
        t.plane = l.m * t.ld;
        if (w.tile) {
            g.work = work;
            if ((e = launch_mx_logits_slopes(g, t, false, num_cu, s)) != hipSuccess)
                return e;
        } else {
            if ((e = multiply(g, work, p.product, num_cu, s)) != hipSuccess)
                return e;
            const uint32_t per_row = (uint32_t)(t.ld / 8);
            e = over_rows(l.m, per_row, [&](uint64_t row0, dim3 grid) {
                hipLaunchKernelGGL(slope_kernel, grid, dim3(kThreads), 0, s, z, (uint32_t)l.m, (uint32_t)w.n, per_row,
                                   div_recip_of(per_row), row0, t, kept);
            });
            if (e != hipSuccess)
                return e;
            kept.counted = nullptr;
        }
        if (l.dx.p) {
            const Out o = p.dx ? Out{dx, l.k, kFp32, t.v0 != 0, nullptr} : Out{l.dx.p, l.dx.ld, l.dx_type, t.v0 != 0, nullptr};
            if ((e = multiply(back_x(l, p, w, t.v0, dz, o), work, p.product, num_cu, s)) != hipSuccess)
                return e;
        }
        if (l.x8.codes)
            if ((e = multiply(back_w(l, p, w, t.v0, dz), work, p.product, num_cu, s)) != hipSuccess)
                return e;
    }
    if (!p.dx)
        return hipSuccess;
    const uint32_t per_row = (uint32_t)((l.k + 7) / 8);
    return over_rows(l.m, per_row, [&](uint64_t row0, dim3 grid) {
        hipLaunchKernelGGL(round_kernel, grid, dim3(kThreads), 0, s, dx, (uint32_t)l.m, (uint32_t)l.k, per_row, div_recip_of(per_row), row0,
                           Out{l.dx.p, l.dx.ld, l.dx_type, 0, nullptr});
    });
}

}  // namespace fastrack
