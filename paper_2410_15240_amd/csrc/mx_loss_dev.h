// What the loss's own kernels (mx_loss.hip) and the ends of its products' tiles (mx_gemm.hip) share.
#pragma once
#include "mx_dev.h"
#include "mx_model.h"

namespace fastrack {

// A largest value and the sum of exponentials over it. An infinite largest value stands for none: e^z
// itself is summed then, which is 0 for -inf and inf for inf.
struct Stat {
    float top, sum;
};

// What a tile of logits needs to know of the loss.
struct LossTile {
    MxIds ids;
    uint64_t v0;             // the piece's first class
    float scale;
    // Forwards:
    Stat *stats;             // [parts][m]
    float *label;            // [m]: the logit of the target
    uint32_t part0;          // of this piece
    // Backwards:
    const float *lse, *dloss;
    uint64_t dloss_step;
    uint16_t *dz;            // bf16 terms, rows of ld values
    uint64_t ld, plane;
    uint32_t terms;
    const float *common;     // [2], see find_common (null: no common factor)
};

// The side of the tiles in which `p` (kLinear) comes out whole, 0 where it does not.
uint32_t mx_logits_tile(const MxProduct &p, int num_cu);
// Its tiles to their end; `laid_out`: x's terms lie in the workspace already.
hipError_t launch_mx_logits_stats(const MxProduct &p, const LossTile &t, bool laid_out, int num_cu, hipStream_t s);
hipError_t launch_mx_logits_slopes(const MxProduct &p, const LossTile &t, bool laid_out, int num_cu, hipStream_t s);

namespace mx {

__device__ __forceinline__ float base_of(float top) { return __builtin_fabsf(top) == __builtin_inff() ? 0.0f : top; }

// The larger one; NaN where either is (fmaxf would drop it).
__device__ __forceinline__ float larger(float a, float b) { return a > b || a != a ? a : b; }

// a - b of a logit a as it is rounded to 32 bits. (Made one with the product that a comes from, as the compiler may,
// the difference of a logit and itself would be what the product's rounding takes off: hundreds, of logits of 1e10.)
__device__ __forceinline__ float minus(float a, float b)
{
#pragma clang fp contract(off)
    return a - b;
}

// e^v by the hardware's 2^v: off by 2^-23 of the result, and by |v| 2^-24 through the argument's rounding.
constexpr float kLog2e = 1.44269504f;
__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * kLog2e); }

// e^(v - from) for many v and one `from` as 2^(v log2e - base), one fma, with base = from log2e as it is rounded: that is
// off by the same factor for all v, 2 to what the rounding took off, and rounding_of() is the factor that makes up for it. As long
// as that is no more than 2^0.5; else from is taken off v first, exactly where it matters.
__device__ __forceinline__ bool near(float base) { return __builtin_fabsf(base) < 0x1p24f; }
__device__ __forceinline__ float rounding_of(float base, float from) { return __builtin_amdgcn_exp2f(__builtin_fmaf(-from, kLog2e, base)); }

// (Of no logits, or none but -inf, the sum is 0, whatever the other one's largest value makes of it.)
__device__ __forceinline__ float over(const Stat &s, float base) { return s.sum == 0.0f ? 0.0f : s.sum * exp_of(base_of(s.top) - base); }

__device__ __forceinline__ Stat join(const Stat &a, const Stat &b)
{
    const float top = larger(a.top, b.top), base = base_of(top);
    return {top, over(a, base) + over(b, base)};
}

// What a token's gradient is multiplied by: what stands for the tokens' common factor, or its own.
__device__ __forceinline__ float factor_of(const LossTile &a, uint64_t row)
{
    const float common = a.common ? a.common[1] : 0.0f;
    return common != 0.0f ? common : a.dloss[row * a.dloss_step] * a.scale;
}

// The gradient of a logit and of a target's, for v = z - lse.
__device__ __forceinline__ float slope(float v, float factor) { return factor * exp_of(v); }
__device__ __forceinline__ float target_slope(float v, float factor) { return factor * (exp_of(v) - 1.0f); }

// The value of the lane next to this one, and of the one two further, within four.
__device__ __forceinline__ float quad_xor1(float v)
{
    return bits_f32((uint32_t)__builtin_amdgcn_update_dpp(0, (int)f32_bits(v), 0xB1, 0xF, 0xF, true));
}
__device__ __forceinline__ float quad_xor2(float v)
{
    return bits_f32((uint32_t)__builtin_amdgcn_update_dpp(0, (int)f32_bits(v), 0x4E, 0xF, 0xF, true));
}

// Eight values as bf16 terms, each the nearest to what those before leave.
__device__ __forceinline__ void put_terms(uint16_t *p, uint64_t plane, uint32_t terms, float (&v)[8])
{
    for (uint32_t k = 0;; ++k) {
        bf16x8 h;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            h[e] = (__bf16)v[e];
        *reinterpret_cast<bf16x8 *>(p + k * plane) = h;
        if (k + 1 == terms)
            return;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = __builtin_fabsf((float)h[e]) == __builtin_inff() ? 0.0f : v[e] - (float)h[e];
    }
}

}  // namespace mx
}  // namespace fastrack
