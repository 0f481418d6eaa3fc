// Products with a microscaled operand, on the matrix cores.
//
// An MX value is exact in bf16 (2 or 7 significant bits and a power of two), so a product of
// a bf16 matrix with an MX one is a bf16 product with 32-bit sums and no rounding of its own.
// A 16-bit float with more significant bits, or a 32-bit one, is the exact sum of 2 or 3 bf16
// terms: its product is the sum of the terms' products, which the kernels run as a longer sum.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mx.h"
#include "mx_dev.h"

namespace fastrack {
namespace mx {

constexpr int kThreads = 256;   // 4 waves, 2 x 2 over the output tile
constexpr uint32_t kBK = 64;    // of the summed axis, at a time

struct Gemm {
    const uint16_t *a;       // bf16 terms of the float matrix, `planes` of them
    uint64_t a_plane;        // elements between them
    uint64_t lda;
    MxMatrix q;
    uint32_t nb;             // blocks in a row of q
    uint32_t m, n, k;        // output m x n, summed axis k
    uint32_t stages;         // planes * ceil(k / kBK)
    uint32_t kstages;        // ceil(k / kBK)
    uint32_t splits, per;    // parts of the sum, stages in each
    uint32_t tm, tn;         // output tiles
    void *c;
    uint64_t ldc;
    uint32_t ctype;
    uint32_t accumulate;
    float *parts;            // [splits][m][n] where splits > 1
};

// 16-byte chunk c of row r of a tile whose rows are 128 bytes: the low three bits of the row
// turn the chunk's place, so that a wave's reads of one chunk from 32 rows use every bank.
__device__ __forceinline__ uint32_t at_k(uint32_t r, uint32_t c) { return r * 128 + ((c ^ (r & 7)) << 4); }

// A tile stored along the output axis, rows of W columns: 64-byte groups of a row are turned
// by its low two bits, since a transposing read takes 4 rows of one 64-byte group at once.
template <int W>
__device__ __forceinline__ uint32_t at_t(uint32_t r, uint32_t col)
{
    return r * (W * 2) + ((col * 2) ^ ((r & 3) << 6));
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// A 32 x 16 operand of the matrix instruction: lane l holds 8 consecutive values of the
// summed axis, from 8 (l / 32), of row l % 32.
__device__ __forceinline__ bf16x8 frag_k(const uint8_t *t, uint32_t row0, uint32_t ks, uint32_t lane)
{
    return *reinterpret_cast<const bf16x8 *>(t + at_k(row0 + (lane & 31), ks * 2 + (lane >> 5)));
}

// The same from a tile stored along the output axis: in each group of 16 lanes, lane j gives
// the address of 4 columns of row j / 4 and receives column j of the 4 rows.
template <int W>
__device__ __forceinline__ bf16x8 frag_t(uint8_t *t, uint32_t col0, uint32_t ks, uint32_t lane)
{
    const uint32_t j = lane & 15, r = ks * 16 + (lane >> 5) * 8 + (j >> 2), c = col0 + ((lane >> 4) & 1) * 16 + (j & 3) * 4;
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(t + at_t<W>(r, c)));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(t + at_t<W>(r + 4, c)));
    return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// One 128 x 128 tile of c, or of one part of it. TA: a is summed over its rows (a[k][m])
// instead of along them (a[m][k]); TB: the same of the MX matrix.
template <uint32_t FMT, bool TA, bool TB>
__global__ __launch_bounds__(kThreads) void gemm_kernel(Gemm g)
{
    constexpr int BM = 128, BN = 128;
    __shared__ __align__(16) uint8_t sa[BM * kBK * 2], sb[BN * kBK * 2];
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6;
    uint32_t id = blockIdx.x;
    const uint32_t tiles = g.tm * g.tn, part = id / tiles;
    id -= part * tiles;
    const uint32_t m0 = id / g.tn * BM, n0 = id % g.tn * BN;
    const uint32_t s_begin = part * g.per, s_end = min(g.stages, s_begin + g.per);

    f32x16 acc[2][2] = {};
    u32x4 ra[4];
    u32x2 rb[4];
    uint32_t re[4];

    auto load = [&](uint32_t s) {
        const uint32_t plane = s / g.kstages, k0 = (s - plane * g.kstages) * kBK;
        const uint16_t *a = g.a + plane * g.a_plane;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u = i * kThreads + t;
            uint32_t row, col;   // of a
            bool in;
            if (TA) {
                row = k0 + u / (BM / 8), col = m0 + u % (BM / 8) * 8;
                in = row < g.k && col < g.m;
            } else {
                row = m0 + u / 8, col = k0 + u % 8 * 8;
                in = row < g.m && col < g.k;
            }
            ra[i] = in ? *reinterpret_cast<const u32x4 *>(a + row * g.lda + col) : u32x4{0, 0, 0, 0};
            const uint32_t qrow = TB ? k0 + u / (BN / 8) : n0 + u / 8;
            const uint32_t unit = TB ? n0 / 8 + u % (BN / 8) : k0 / 8 + u % 8;   // 8 codes, 4 to a block
            in = qrow < (TB ? g.k : g.n) && unit / 4 < g.nb;
            rb[i] = u32x2{0, 0};
            re[i] = 0;
            if (in) {
                const uint64_t at = (uint64_t)qrow * g.nb;
                re[i] = g.q.scales[at + unit / 4];
                if (FMT == kMx4)
                    rb[i][0] = reinterpret_cast<const uint32_t *>(g.q.codes)[at * 4 + unit];
                else
                    rb[i] = reinterpret_cast<const u32x2 *>(g.q.codes)[at * 4 + unit];
            }
        }
    };
    auto store = [&]() {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u = i * kThreads + t;
            const uint32_t pa = TA ? at_t<BM>(u / (BM / 8), u % (BM / 8) * 8) : at_k(u / 8, u % 8);
            *reinterpret_cast<u32x4 *>(sa + pa) = ra[i];
            const uint32_t pb = TB ? at_t<BN>(u / (BN / 8), u % (BN / 8) * 8) : at_k(u / 8, u % 8);
            *reinterpret_cast<u32x4 *>(sb + pb) =
                FMT == kMx4 ? decode4_bf16(rb[i][0], scale_f32(re[i])) : decode8_bf16(rb[i], scale8_f32(re[i]));
        }
    };

    if (s_begin < s_end)
        load(s_begin);
    for (uint32_t s = s_begin; s < s_end; ++s) {
        store();
        __syncthreads();
        if (s + 1 < s_end)
            load(s + 1);
        const uint32_t wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            bf16x8 fa[2], fb[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                fa[i] = TA ? frag_t<BM>(sa, wm + i * 32, ks, lane) : frag_k(sa, wm + i * 32, ks, lane);
                fb[i] = TB ? frag_t<BN>(sb, wn + i * 32, ks, lane) : frag_k(sb, wn + i * 32, ks, lane);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
        }
        __syncthreads();
    }

    // Lane l holds column l % 32 of rows 8 (r / 4) + 4 (l / 32) + r % 4.
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t row = m0 + (wave >> 1) * 64 + i * 32 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4;
                const uint32_t col = n0 + (wave & 1) * 64 + j * 32 + (lane & 31);
                if (row >= g.m || col >= g.n)
                    continue;
                const float v = acc[i][j][r];
                if (g.splits > 1) {
                    g.parts[((uint64_t)part * g.m + row) * g.n + col] = v;
                } else if (g.ctype == kFp32) {
                    float *p = reinterpret_cast<float *>(g.c) + row * g.ldc + col;
                    *p = g.accumulate ? *p + v : v;
                } else if (g.ctype == kBf16) {
                    reinterpret_cast<__bf16 *>(g.c)[row * g.ldc + col] = (__bf16)v;
                } else {
                    reinterpret_cast<_Float16 *>(g.c)[row * g.ldc + col] = (_Float16)v;
                }
            }
}

// c = the sum of the parts, always in the same order.
__global__ __launch_bounds__(kThreads) void join_kernel(const float *parts, uint32_t splits, uint32_t m, uint32_t n,
                                                        void *c, uint64_t ldc, uint32_t ctype, uint32_t accumulate)
{
    const uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x, total = (uint64_t)m * n;
    if (i >= total)
        return;
    float v = 0.0f;
    for (uint32_t s = 0; s < splits; ++s)
        v += parts[s * total + i];
    const uint64_t at = i / n * ldc + i % n;
    if (ctype == kFp32) {
        float *p = reinterpret_cast<float *>(c) + at;
        *p = accumulate ? *p + v : v;
    } else if (ctype == kBf16) {
        reinterpret_cast<__bf16 *>(c)[at] = (__bf16)v;
    } else {
        reinterpret_cast<_Float16 *>(c)[at] = (_Float16)v;
    }
}

// The bf16 terms of a float matrix, rows padded with zeros to ld (a multiple of 8): each term
// is what is left cut to its upper 16 bits, so that 3 terms of 8 significant bits (2 for
// 11 bits) add up to the value exactly. A NaN or an infinity is all in the first term.
template <uint32_t T, bool VEC>
__global__ __launch_bounds__(kThreads) void terms_kernel(MxRows a, uint64_t rows, uint32_t cols, uint16_t *out, uint64_t ld,
                                                         uint64_t plane)
{
    constexpr int P = T == kBf16 ? 1 : T == kFp16 ? 2 : 3;
    const uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x, per = ld / 8;
    const uint64_t r = i / per;
    if (r >= rows)
        return;
    const uint32_t c = (uint32_t)(i - r * per) * 8;
    float v[8];
    load8<T, VEC>(a.p, r * a.ld, c, cols, v);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        uint32_t h[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t u = f32_bits(v[j]);
            const bool odd = (u & 0x7F800000u) == 0x7F800000u;   // NaN or infinity
            h[j] = u >> 16;
            if (odd && (u & 0x007FFFFFu))
                h[j] |= 0x40u;   // stays a NaN
            v[j] = odd ? 0.0f : v[j] - bits_f32(u & 0xFFFF0000u);
        }
        *reinterpret_cast<u32x4 *>(out + p * plane + r * ld + c) =
            u32x4{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
    }
}

uint32_t planes_of(uint32_t type) { return type == kBf16 ? 1 : type == kFp16 ? 2 : 3; }

uint64_t round_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

// How a product runs: whether a is read in place, and into how many parts its sum is cut.
struct Plan {
    bool in_place;
    uint64_t a_rows, a_cols, a_ld, a_bytes;   // a's terms in the workspace, where not in place
    uint32_t kstages, stages, splits, per, tm, tn;
    uint64_t m, n, k;                         // output m x n, summed axis k
    uint64_t bytes() const { return a_bytes + (splits > 1 ? (uint64_t)splits * m * n * 4 : 0); }
};

Plan plan_of(const MxProduct &p, int num_cu)
{
    Plan r = {};
    const bool ta = p.op == kWeightGrad;
    r.m = ta ? p.n : p.m;
    r.n = p.op == kLinear ? p.n : p.k;
    r.k = p.op == kLinear ? p.k : ta ? p.m : p.n;
    r.a_rows = p.m;
    r.a_cols = p.op == kLinear ? p.k : p.n;
    // 16-byte chunks of a row: all of a chunk's values lie in the row, or none.
    r.in_place = p.type == kBf16 && reinterpret_cast<uintptr_t>(p.a.p) % 16 == 0 && p.a.ld % 8 == 0 && r.a_cols % 8 == 0;
    r.a_ld = round_up(r.a_cols, 8);
    r.a_bytes = r.in_place ? 0 : round_up(planes_of(p.type) * r.a_rows * r.a_ld * 2, 256);
    r.kstages = (uint32_t)((r.k + kBK - 1) / kBK);
    r.stages = r.kstages * (r.in_place ? 1 : planes_of(p.type));
    r.tm = (uint32_t)((r.m + 127) / 128);
    r.tn = (uint32_t)((r.n + 127) / 128);
    // Fewer tiles than CUs: cut the sum, down to 4 stages a part.
    const uint64_t tiles = (uint64_t)r.tm * r.tn;
    uint64_t splits = tiles >= (uint64_t)num_cu ? 1 : (uint64_t)num_cu * 2 / (tiles ? tiles : 1);
    if (splits > r.stages / 4)
        splits = r.stages / 4;
    if (splits < 1)
        splits = 1;
    r.per = (uint32_t)((r.stages + splits - 1) / splits);
    if (r.per == 0)
        r.per = 1;
    r.splits = (uint32_t)(r.stages ? (r.stages + r.per - 1) / r.per : 1);
    return r;
}

// ---- MX4 x MX4 -------------------------------------------------------------------------

constexpr uint32_t kBK4 = 128;

struct Gemm4 {
    MxMatrix x, w;
    uint32_t nb, m, n;
    uint32_t stages, splits, per, tm, tn;
    void *c;
    uint64_t ldc;
    uint32_t ctype;
    float *parts;
};

// Rows of 64 bytes (4 blocks): the chunk's place turned by bits 1 and 2 of the row.
__device__ __forceinline__ uint32_t at4(uint32_t r, uint32_t c) { return r * 64 + ((c ^ ((r >> 1) & 3)) << 4); }

// Both operands stay in 4 bits: the scaled matrix instruction takes 32 codes and their
// block's scale byte per lane, rows l % 32, block l / 32.
__global__ __launch_bounds__(kThreads) void gemm4_kernel(Gemm4 g)
{
    constexpr int BM = 128, BN = 128;
    typedef int i32x8 __attribute__((ext_vector_type(8)));
    __shared__ __align__(16) uint8_t sa[BM * kBK4 / 2], sb[BN * kBK4 / 2];
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6;
    uint32_t id = blockIdx.x;
    const uint32_t tiles = g.tm * g.tn, part = id / tiles;
    id -= part * tiles;
    const uint32_t m0 = id / g.tn * BM, n0 = id % g.tn * BN;
    const uint32_t wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
    const uint32_t s_begin = part * g.per, s_end = min(g.stages, s_begin + g.per);

    f32x16 acc[2][2] = {};
    u32x4 ra[2], rb[2];
    uint32_t ea[2][2], eb[2][2], na[2][2], nb[2][2];
    auto scale = [&](const MxMatrix &q, uint32_t row, uint32_t rows, uint32_t block) -> uint32_t {
        return row < rows && block < g.nb ? q.scales[(uint64_t)row * g.nb + block] : 127u;
    };
    auto load = [&](uint32_t s) {
        const uint32_t b0 = s * (kBK4 / 32);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t u = i * kThreads + t, row = u / 4, block = b0 + u % 4;
            ra[i] = rb[i] = u32x4{0, 0, 0, 0};
            if (m0 + row < g.m && block < g.nb)
                ra[i] = reinterpret_cast<const u32x4 *>(g.x.codes)[(uint64_t)(m0 + row) * g.nb + block];
            if (n0 + row < g.n && block < g.nb)
                rb[i] = reinterpret_cast<const u32x4 *>(g.w.codes)[(uint64_t)(n0 + row) * g.nb + block];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const uint32_t bl = b0 + ks * 2 + (lane >> 5);
                na[ks][i] = scale(g.x, m0 + wm + i * 32 + (lane & 31), g.m, bl);
                nb[ks][i] = scale(g.w, n0 + wn + i * 32 + (lane & 31), g.n, bl);
            }
        }
    };
    if (s_begin < s_end)
        load(s_begin);
    for (uint32_t s = s_begin; s < s_end; ++s) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t u = i * kThreads + t;
            *reinterpret_cast<u32x4 *>(sa + at4(u / 4, u % 4)) = ra[i];
            *reinterpret_cast<u32x4 *>(sb + at4(u / 4, u % 4)) = rb[i];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                ea[ks][i] = na[ks][i];
                eb[ks][i] = nb[ks][i];
            }
        }
        __syncthreads();
        if (s + 1 < s_end)
            load(s + 1);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            i32x8 fa[2] = {}, fb[2] = {};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u32x4 va = *reinterpret_cast<const u32x4 *>(sa + at4(wm + i * 32 + (lane & 31), ks * 2 + (lane >> 5)));
                const u32x4 vb = *reinterpret_cast<const u32x4 *>(sb + at4(wn + i * 32 + (lane & 31), ks * 2 + (lane >> 5)));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    fa[i][j] = (int)va[j];
                    fb[i][j] = (int)vb[j];
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fa[i], fb[j], acc[i][j], 4, 4, 0,
                                                                                (int)ea[ks][i], 0, (int)eb[ks][j]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t row = m0 + wm + i * 32 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4;
                const uint32_t col = n0 + wn + j * 32 + (lane & 31);
                if (row >= g.m || col >= g.n)
                    continue;
                const float v = acc[i][j][r];
                if (g.splits > 1)
                    g.parts[((uint64_t)part * g.m + row) * g.n + col] = v;
                else if (g.ctype == kFp32)
                    reinterpret_cast<float *>(g.c)[row * g.ldc + col] = v;
                else if (g.ctype == kBf16)
                    reinterpret_cast<__bf16 *>(g.c)[row * g.ldc + col] = (__bf16)v;
                else
                    reinterpret_cast<_Float16 *>(g.c)[row * g.ldc + col] = (_Float16)v;
            }
}

Gemm4 plan4_of(const Mx4Product &p, int num_cu)
{
    Gemm4 g = {};
    g.x = p.x;
    g.w = p.w;
    g.nb = (uint32_t)mx_blocks(p.k);
    g.m = (uint32_t)p.m;
    g.n = (uint32_t)p.n;
    g.stages = (uint32_t)((p.k + kBK4 - 1) / kBK4);
    g.tm = (uint32_t)((p.m + 127) / 128);
    g.tn = (uint32_t)((p.n + 127) / 128);
    const uint64_t tiles = (uint64_t)g.tm * g.tn;
    uint64_t splits = tiles >= (uint64_t)num_cu ? 1 : (uint64_t)num_cu * 2 / (tiles ? tiles : 1);
    if (splits > g.stages / 4)
        splits = g.stages / 4;
    if (splits < 1)
        splits = 1;
    g.per = (uint32_t)((g.stages + splits - 1) / splits);
    if (g.per == 0)
        g.per = 1;
    g.splits = g.stages ? (g.stages + g.per - 1) / g.per : 1;
    return g;
}

}  // namespace mx

using namespace mx;

uint64_t mx_product_work(const MxProduct &p, int num_cu) { return plan_of(p, num_cu).bytes(); }

hipError_t launch_mx_product(const MxProduct &p, int num_cu, hipStream_t s)
{
    const Plan r = plan_of(p, num_cu);
    if (r.m == 0 || r.n == 0)
        return hipSuccess;
    Gemm g = {};
    g.a = reinterpret_cast<const uint16_t *>(p.a.p);
    g.lda = p.a.ld;
    if (!r.in_place && r.k) {
        uint16_t *out = reinterpret_cast<uint16_t *>(p.work);
        g.a = out;
        g.lda = r.a_ld;
        g.a_plane = r.a_rows * r.a_ld;
        const uint64_t units = r.a_rows * (r.a_ld / 8);
        const bool vec = reinterpret_cast<uintptr_t>(p.a.p) % 16 == 0 && p.a.ld * mx_type_size(p.type) % 16 == 0;
        const dim3 grid((uint32_t)((units + kThreads - 1) / kThreads));
#define MX_TERMS(T)                                                                                                   \
    do {                                                                                                              \
        if (vec)                                                                                                      \
            hipLaunchKernelGGL((terms_kernel<T, true>), grid, dim3(kThreads), 0, s, p.a, r.a_rows, (uint32_t)r.a_cols, \
                               out, r.a_ld, g.a_plane);                                                               \
        else                                                                                                          \
            hipLaunchKernelGGL((terms_kernel<T, false>), grid, dim3(kThreads), 0, s, p.a, r.a_rows,                   \
                               (uint32_t)r.a_cols, out, r.a_ld, g.a_plane);                                           \
    } while (0)
        if (p.type == kBf16)
            MX_TERMS(kBf16);
        else if (p.type == kFp16)
            MX_TERMS(kFp16);
        else
            MX_TERMS(kFp32);
#undef MX_TERMS
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    g.q = p.q;
    g.nb = (uint32_t)mx_blocks(p.k);
    g.m = (uint32_t)r.m;
    g.n = (uint32_t)r.n;
    g.k = (uint32_t)r.k;
    g.stages = r.stages;
    g.kstages = r.kstages ? r.kstages : 1;
    g.splits = r.splits;
    g.per = r.per;
    g.tm = r.tm;
    g.tn = r.tn;
    g.c = p.c.p;
    g.ldc = p.c.ld;
    g.ctype = p.ctype;
    g.accumulate = p.accumulate;
    g.parts = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(p.work) + r.a_bytes);
    const dim3 grid(r.tm * r.tn * r.splits);
    if (p.op == kLinear)
        hipLaunchKernelGGL((gemm_kernel<kMx4, false, false>), grid, dim3(kThreads), 0, s, g);
    else if (p.op == kGradInput)
        hipLaunchKernelGGL((gemm_kernel<kMx4, false, true>), grid, dim3(kThreads), 0, s, g);
    else
        hipLaunchKernelGGL((gemm_kernel<kMx8, true, true>), grid, dim3(kThreads), 0, s, g);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || r.splits == 1)
        return e;
    const uint64_t total = r.m * r.n;
    hipLaunchKernelGGL(join_kernel, dim3((uint32_t)((total + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, g.parts,
                       r.splits, g.m, g.n, g.c, g.ldc, g.ctype, g.accumulate);
    return hipGetLastError();
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
    hipLaunchKernelGGL(gemm4_kernel, dim3(g.tm * g.tn * g.splits), dim3(kThreads), 0, s, g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || g.splits == 1)
        return e;
    const uint64_t total = p.m * p.n;
    hipLaunchKernelGGL(join_kernel, dim3((uint32_t)((total + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, g.parts,
                       g.splits, g.m, g.n, g.c, g.ldc, g.ctype, 0u);
    return hipGetLastError();
}

}  // namespace fastrack
