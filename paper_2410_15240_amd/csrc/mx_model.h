// Launch interface of the microscaled operators around a model's layers: the norms between its
// blocks (mx_norm.hip), the lookup at its start (mx_embed.hip), the loss at its end
// (mx_loss.hip). Internal to the library.
#pragma once
#include "mx.h"

namespace fastrack {

// b = x / rms(x) * w1 (or x), h = r + scale * g * b, y = h / rms(h) * w2. Absent operands are null.
struct Norm {
    uint32_t type, wtype;   // of the rows; of w1 and w2: that, or fp32
    uint64_t rows, cols;
    MxRows x, r, g, y, h;
    const void *w2, *w1;
    float scale, eps;
    MxMatrix u, v, gq;      // kept in MX8: h / rms(h); x / rms(x), or x; g
    float *inv2, *inv1;     // 1 / rms
};
hipError_t launch_mx_norm(const Norm &n, int num_cu, hipStream_t s);

struct NormGrad {
    uint32_t type, wtype;
    uint64_t rows, cols;
    MxRows dy, dh, dx, dr, dg;
    const void *w2, *w1;
    float scale;
    MxMatrix u, v, gq;
    const float *inv2, *inv1;
    float *dw2, *dw1;
    float *work;
};
// Floats of workspace: a partial sum of dw2 (and dw1) of every group of rows.
uint64_t mx_norm_grad_work(uint64_t rows, uint64_t cols, bool w1, int num_cu);
hipError_t launch_mx_norm_grad(const NormGrad &n, int num_cu, hipStream_t s);

// y[t] = scale * table[id_t].
struct Embedding {
    MxIds ids;
    uint64_t m, rows, cols;
    MxMatrix table;
    float scale;
    uint32_t type;
    MxRows y;
};
hipError_t launch_mx_embedding(const Embedding &e, hipStream_t s);

// dw[i] (+)= scale * sum of dy[t] over the t with id_t = i, in the order of t.
struct EmbeddingGrad {
    MxIds ids;
    uint32_t type;
    MxRows dy;
    uint64_t m, rows, cols;
    float scale;
    uint32_t otype;
    MxRows dw;
    bool accumulate;
    void *work;
};
uint64_t mx_embedding_grad_work(uint64_t m, uint64_t rows, uint64_t cols);
hipError_t launch_mx_embedding_grad(const EmbeddingGrad &e, hipStream_t s);

// z = scale * x w^T [m, n]; lse = log sum exp z, loss = lse - z[id]; and from dloss the gradients
// dx [m, k] and dw [n, k] = scale dz^T x8.
struct Loss {
    uint32_t type;
    MxRows x;
    MxMatrix w;
    MxIds ids;
    uint64_t m, n, k;
    float scale;
    float *loss, *lse;      // (lse is read by the gradient)
    // The gradient:
    const float *dloss;
    uint64_t dloss_step;
    MxMatrix x8;            // null codes: no dw
    uint32_t dx_type, dw_type;
    MxRows dx, dw;          // null dx: none
    bool accumulate;        // dw += (fp32 only)
    void *work;
};
uint64_t mx_loss_work(const Loss &l, int num_cu);
hipError_t launch_mx_loss(const Loss &l, int num_cu, hipStream_t s);
uint64_t mx_loss_grad_work(const Loss &l, int num_cu);
hipError_t launch_mx_loss_grad(const Loss &l, int num_cu, hipStream_t s);

}  // namespace fastrack
