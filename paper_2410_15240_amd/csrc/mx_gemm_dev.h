// Device pieces that the matrix products share: tiles in LDS, the matrix instruction's operands,
// results on their way out.
#pragma once
#include "mx_dev.h"
#include "mx_small.h"

namespace fastrack {
namespace mx {

// A constant as an argument of a lambda.
template <int V>
struct Const {
    static constexpr int value = V;
};

// 16-byte chunk c of row r of a tile whose rows are 128 bytes: bits 1 to 3 of the row turn the
// chunk's place, so that one chunk of 16 rows in turn lies in all 64 banks, once in each.
__device__ __forceinline__ uint32_t at_k(uint32_t r, uint32_t c) { return r * 128 + ((c ^ ((r >> 1) & 7)) << 4); }

// A tile stored along the output axis, rows of W columns: 64-byte groups of a row are turned
// by its low two bits, since a transposing read takes 4 rows of one 64-byte group at once.
template <int W>
__device__ __forceinline__ uint32_t at_t(uint32_t r, uint32_t col)
{
    return r * (W * 2) + ((col * 2) ^ ((r & 3) << 6));
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Offsets of a lane's reads of the matrix instruction's 32 x 16 operands, where lane l holds 8
// consecutive values of the summed axis, from 8 (l / 32), of row l % 32. In a tile stored along
// the summed axis they differ by the step (16 values) in the turned bits, and squares of 32
// rows follow each other.
__device__ __forceinline__ uint32_t frag_k_at(uint32_t row0, uint32_t ks, uint32_t lane)
{
    return at_k(row0 + (lane & 31), ks * 2 + (lane >> 5));
}

// In a tile stored along the output axis: in each group of 16 lanes, lane j gives the address
// of 4 columns of row j / 4 and receives column j of the 4 rows. Squares of 32 columns differ
// in the turned bits, and steps of 16 rows follow each other.
template <int W>
__device__ __forceinline__ uint32_t frag_t_at(uint32_t col0, uint32_t lane)
{
    const uint32_t j = lane & 15;
    return at_t<W>((lane >> 5) * 8 + (j >> 2), col0 + ((lane >> 4) & 1) * 16 + (j & 3) * 4);
}

__device__ __forceinline__ bf16x8 read_k(const uint8_t *p) { return *reinterpret_cast<const bf16x8 *>(p); }

__device__ __forceinline__ bf16x8 read_t2(uint8_t *first, uint8_t *second)
{
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)first);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)second);
    return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <int W>
__device__ __forceinline__ bf16x8 read_t(uint8_t *p) { return read_t2(p, p + 4 * W * 2); }

// 16-bit values [c, c + 8) of a row, zero past `cols`.
__device__ __forceinline__ u32x4 chunk_at(const uint16_t *row, uint32_t c, uint32_t cols)
{
    u32x4 v = {0, 0, 0, 0};
    if (c + 8 <= cols) {
        __builtin_memcpy(&v, row + c, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols)
                v[i / 2] |= (uint32_t)row[c + i] << (16 * (i % 2));
    }
    return v;
}

// Memory from one address for the whole wave, read at 32-bit offsets of its lanes. (Through
// plain pointers the compiler keeps every lane's offset in 64 bits and adds it to the address
// at each load.)
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_at(const void *p)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, 0xFFFFFFFFu, 0x00027000);
}

// This wave's LDS accesses before it come before those after it. (The LDS takes a wave's accesses
// in order; what is held back is the compiler.)
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// All waves' LDS accesses before it are done. (Loads from memory may still be on their way.)
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ void put1(const Out &o, uint32_t row, uint32_t c, float v)
{
    const uint64_t at = row * o.ld + c;
    if (o.type == kFp32) {
        float *p = reinterpret_cast<float *>(o.p) + at;
        *p = o.accumulate ? *p + v : v;
    } else if (o.type == kBf16) {
        reinterpret_cast<__bf16 *>(o.p)[at] = (__bf16)v;
    } else {
        reinterpret_cast<_Float16 *>(o.p)[at] = (_Float16)v;
    }
}

// Columns [c, c + 8) of a row.
__device__ __forceinline__ void put8(const Out &o, uint32_t row, uint32_t c, uint32_t cols, float (&v)[8])
{
    const uint64_t at = row * o.ld;
    if (o.type == kFp32) {
        if (o.accumulate) {
            float w[8];
            load8<kFp32>(o.p, at, c, cols, w);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] += w[i];
        }
        store8<kFp32>(o.p, at, c, cols, v);
    } else if (o.type == kBf16) {
        store8<kBf16>(o.p, at, c, cols, v);
    } else {
        store8<kFp16>(o.p, at, c, cols, v);
    }
}

}  // namespace mx
}  // namespace fastrack
