// Launch interface of the products with few outputs (mx_small.hip). Internal to the library.
#pragma once
#include "mx.h"

namespace fastrack {

// Where a product's results go: c itself, or parts of a sum as 32-bit floats.
struct Out {
    void *p;
    uint64_t ld;
    uint32_t type, accumulate;
};

struct SmallProduct {
    MxRows a;
    MxMatrix q;
    uint32_t nb;             // blocks in a row of q
    uint32_t m, n, k;        // output m x n, summed axis k
    uint32_t tm, tn;         // tiles (launch_mx_small)
    uint32_t slices;         // of 64 summed values
    uint32_t cuts, per;      // parts of the sum that workgroups of their own take, slices in each
    Out out;
    float *parts;            // [cuts][m][n] where cuts > 1
};

constexpr int kSmallThreads = 512;   // of a workgroup of launch_mx_small

// linear alone, m up to 2 and k from 8.
hipError_t launch_mx_dot(const SmallProduct &g, uint32_t type, hipStream_t s);
// Tiles of side 32, or of 64 where a is not fp32 (its terms of 64 rows do not fit the registers);
// a's rows of 8 values and more.
hipError_t launch_mx_small(const SmallProduct &g, uint32_t op, uint32_t type, uint32_t side, hipStream_t s);

}  // namespace fastrack
