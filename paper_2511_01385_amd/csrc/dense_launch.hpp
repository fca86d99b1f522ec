// dense_launch.hpp -- host-side launchers of the operators around the block-circulant layer:
// 8-bit checkpoints, layer norm, and the dense product with its epilogue.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "launch.hpp"

namespace rdfft {

// An 8-bit checkpoint of [rows][n] values: codes [rows][n] and scales [rows][ceil(n/32)],
// contiguous.  Null pointers: none.
struct Checkpoint {
  int8_t* codes = nullptr;
  uint8_t* scales = nullptr;
};

hipError_t launch_act8_quantize(const void* x, int64_t ldx, int8_t* codes, uint8_t* scales, int64_t rows, int64_t n,
                                int storage, hipStream_t stream, int num_cu);
hipError_t launch_act8_dequantize(const int8_t* codes, const uint8_t* scales, void* out, int64_t ldo, int64_t rows,
                                  int64_t n, int storage, hipStream_t stream, int num_cu);

// Layer norm (norm_kernels.hip).  Row strides in elements; residual, bias, mean, rstd and the
// checkpoint may be null.
constexpr int64_t kNormMaxWidth = 16384;
struct NormArgs {
  const void* x;
  int64_t ldx;
  const void* residual;
  int64_t ldr;
  const float *weight, *bias;
  void* y;
  int64_t ldy;
  float *mean, *rstd;
  Checkpoint ck;
  int64_t rows, n;
  float eps;
  int storage;
};
hipError_t launch_layer_norm_forward(const NormArgs& a, hipStream_t stream, int num_cu);

// The norm's input is x (+ residual) or, with x null, the checkpoint.
struct NormGradArgs {
  const void* dy;
  int64_t ldg;
  const void* x;
  int64_t ldx;
  const void* residual;
  int64_t ldr;
  Checkpoint ck;
  const float *weight, *mean, *rstd;
  void* dx;
  int64_t ldd;
  float *dweight, *dbias;
  float* partials;  // norm_partials(rows, n) * 2n floats; unused where that is one
  int64_t rows, n;
  int storage;
};
int64_t norm_partials(int64_t rows, int64_t n);
hipError_t launch_layer_norm_backward(const NormGradArgs& a, hipStream_t stream);

// The second stage of a sum over rows (norm_kernels.hip): column c of out0 (c < n), or c - n of out1, is
// the sum over g < groups of partials[g * cols + c]; cols is n or 2n.
hipError_t launch_column_finish(const float* partials, int64_t groups, int64_t cols, int64_t n, void* out0, void* out1,
                                int storage, hipStream_t stream);

// The dense product (linear.hip).  Values of rdfft_activation_t:
constexpr int kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3;
// D (m x n) = A B^T with either operand along or across k (linear_kernels.hpp), k in `splits` ranges of
// k_split.  partial: each split's float32 sums, [splits][m][n], in place of D and its epilogue.
struct GemmArgs {
  const void* a;
  int64_t lda;
  const void* b;
  int64_t ldb;
  int64_t m, n, k;
  void* d;
  int64_t ldd;
  const void* bias;
  const void* residual;
  int64_t ldr;
  Checkpoint ck;
  int act;
  float* partial;
  int splits;
  int64_t k_split;
  int tiles_m, tiles_n;
};
// the instances for one storage type; null where one is not built.  Last index: 1 where
// both operands' memory rows hold whole chunks of 16 bytes, at addresses that can be loaded straight to LDS
enum LinearTile { kTile32x64, kTile64, kTile128, kTile128x256, kTile256, kLinearTiles };
enum LinearOperands { kForward, kGradX, kGradW, kLinearOperands };
using LinearFn = hipError_t (*)(const GemmArgs&, hipStream_t);
using LinearGradsFn = hipError_t (*)(const GemmArgs& dw, const GemmArgs& dx, hipStream_t);
constexpr int64_t kFewTokens = 64;
struct LinearTable {
  LinearFn fn[kLinearTiles][kLinearOperands][2];
  LinearGradsFn grads[kLinearTiles];  // dW and dx in one launch, of whole chunks
  LinearFn few[3][2][2];              // the forward of 16, 32, 64 tokens at most, 16 or 32 rows of W to a workgroup
};
LinearTable linear_table_f32();
LinearTable linear_table_bf16();
LinearTable linear_table_f16();

// Bytes of workspace that the calls below need for these sizes.
struct LinearSizes {
  int64_t d_in, d_out, tokens;
  int act, storage;
};
int64_t linear_forward_workspace(const LinearSizes& s);
int64_t linear_backward_workspace(const LinearSizes& s, bool dx, bool dw, bool db);

struct LinearForward {
  LinearSizes s;
  const void* x;
  int64_t ldx;
  const void* w;
  int64_t ldw;
  const void* bias;
  const void* residual;
  int64_t ldr;
  void* y;
  int64_t ldy;
  Checkpoint ck;
  void* workspace;
};
hipError_t launch_linear_forward(const LinearForward& a, hipStream_t stream);

struct LinearBackward {
  LinearSizes s;
  const void* dy;
  int64_t ldg;
  Checkpoint ck;
  const void* x;
  int64_t ldx;
  const void* w;
  int64_t ldw;
  const void* add;
  int64_t lda;
  void* dx;
  int64_t ldd;
  void* dw;
  int64_t lddw;
  void* db;
  void* workspace;
};
hipError_t launch_linear_backward(const LinearBackward& a, hipStream_t stream);

}  // namespace rdfft
