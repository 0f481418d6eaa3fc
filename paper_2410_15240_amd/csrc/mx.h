// Launch interface of the microscaled (MX) operators, between their C entries (mx_api.hip)
// and their kernels (mx.hip, mx_gemm.hip). Internal to the library.
//
// An MX matrix has rows of blocks of 32 values; a block is its codes (16 bytes of E2M1
// pairs in MX4, 32 int8 in MX8) and one scale byte e, worth 2^(e - 127), NaN for 255. The
// codes of a block start at a multiple of 16 bytes; rows are whole blocks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fastrack {

enum MxType : uint32_t { kBf16 = 0, kFp16 = 1, kFp32 = 2 };
enum MxFormat : uint32_t { kMx4 = 4, kMx8 = 8 };
enum MxAct : uint32_t { kSilu = 0, kGelu = 1 };

constexpr uint32_t kMxBlock = 32;

constexpr uint32_t mx_type_size(uint32_t t) { return t == kFp32 ? 4 : 2; }
constexpr uint64_t mx_blocks(uint64_t cols) { return (cols + kMxBlock - 1) / kMxBlock; }
constexpr uint32_t mx_block_bytes(uint32_t fmt) { return fmt == kMx4 ? 16 : 32; }

// A float matrix of a call: rows of ld elements, the first `cols` of each used.
struct MxRows {
    void *p;
    uint64_t ld;
};

struct MxMatrix {
    uint8_t *codes;
    uint8_t *scales;
};

hipError_t launch_mx_quantize(uint32_t fmt, uint32_t type, MxRows x, uint64_t rows, uint64_t cols, MxMatrix q,
                              hipStream_t s);
hipError_t launch_mx_dequantize(uint32_t fmt, uint32_t type, MxMatrix q, uint64_t rows, uint64_t cols, MxRows out,
                                hipStream_t s);
// y = f(x) [* gate]; x and gate kept in MX8. gate.p is null where there is none.
hipError_t launch_mx_act(uint32_t act, uint32_t type, MxRows x, MxRows gate, uint64_t rows, uint64_t cols, MxRows y,
                         MxMatrix qx, MxMatrix qg, hipStream_t s);
// dx = dy [* gate] f'(x), dgate = dy f(x), from the kept x and gate.
hipError_t launch_mx_act_grad(uint32_t act, uint32_t type, MxRows dy, MxMatrix qx, MxMatrix qg, uint64_t rows,
                              uint64_t cols, MxRows dx, MxRows dgate, hipStream_t s);

// The products. `op` says which axis of the MX matrix is summed over:
//   kLinear      c[m, n] = sum_k a[m, k] w[n, k]      w MX4, n rows
//   kGradInput   c[m, k] = sum_n a[m, n] w[n, k]      w MX4, n rows
//   kWeightGrad  c[n, k] = sum_m a[m, n] x[m, k]      x MX8, m rows
enum MxOp : uint32_t { kLinear = 0, kGradInput = 1, kWeightGrad = 2 };

struct MxProduct {
    uint32_t op;
    uint32_t type;          // of a
    MxRows a;
    MxMatrix q;
    uint64_t m, n, k;       // tokens, outputs and inputs of the layer
    uint32_t ctype;         // of c
    MxRows c;
    bool accumulate;        // c += (fp32 only)
    void *work;
    uint64_t work_bytes;
};

// Workspace that a product needs: the parts of a long sum, and a's bf16 terms where a is not
// read in place.
uint64_t mx_product_work(const MxProduct &p, int num_cu);
hipError_t launch_mx_product(const MxProduct &p, int num_cu, hipStream_t s);

// c[m, n] = sum_k x[m, k] w[n, k], both MX4.
struct Mx4Product {
    MxMatrix x, w;
    uint64_t m, n, k;
    uint32_t ctype;
    MxRows c;
    void *work;
    uint64_t work_bytes;
};
uint64_t mx4_product_work(const Mx4Product &p, int num_cu);
hipError_t launch_mx4_product(const Mx4Product &p, int num_cu, hipStream_t s);

// Errors of the C entries (api.hip): store the calling thread's message, return the code.
int set_error(int code, const char *msg);
void clear_error();

}  // namespace fastrack
