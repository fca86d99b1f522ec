// fp8_launch.hpp -- host-side launchers of the operators in 8-bit floating point and of RMS norm.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dense_launch.hpp"

namespace rdfft {

// [rows][n] values in 8-bit floating point (fp8_device.hpp).  Rows of codes are `ld` bytes apart and start at multiples of
// 16 bytes, rows of scales `lds` bytes at multiples of 4.  Row r's scales are row r >> shift: 0, or 7 for tiles.
struct Fp8Operand {
  uint8_t* codes = nullptr;
  int64_t ld = 0;
  uint8_t* scales = nullptr;
  int64_t lds = 0;
  int shift = 0;
};

// x [rows][n] (times the slope of `act` at what ck stands for) by rows into `held`, by columns into `columns`
// (either null); tiles: both with one scale for 128 x 128.  sums: [ceil(rows/128)][n], over each 128 rows; or
// total: of at most 128 rows, in the storage type.
struct Fp8Quantize {
  const void* x;
  int64_t ldx;
  int64_t rows, n;
  Fp8Operand held, columns;
  bool tiles;
  int act;
  Checkpoint ck;
  float* sums;
  void* total;
  int storage;
};
hipError_t launch_fp8_quantize(const Fp8Quantize& q, hipStream_t stream);
hipError_t launch_fp8_dequantize(const Fp8Operand& from, void* out, int64_t ldo, int64_t rows, int64_t n, int storage,
                                 hipStream_t stream, int num_cu);

// RMS norm (rms_norm_kernels.hip).  residual, y, summed, rstd, ck and y8 may be null.
struct RmsArgs {
  const void* x;
  int64_t ldx;
  const void* residual;
  int64_t ldr;
  const float* weight;
  void* y;
  int64_t ldy;
  void* summed;
  int64_t lds;
  float* rstd;
  Checkpoint ck;
  Fp8Operand y8;
  int64_t rows, n;
  float eps;
  int storage;
};
hipError_t launch_rms_norm_forward(const RmsArgs& a, hipStream_t stream, int num_cu);

// The norm's input is u or, with u null, the checkpoint.  add and dweight may be null.
struct RmsGradArgs {
  const void* dy;
  int64_t ldg;
  const void* u;
  int64_t ldu;
  Checkpoint ck;
  const float *weight, *rstd;
  const void* add;
  int64_t lda;
  void* dx;
  int64_t ldd;
  float* dweight;
  float* partials;  // rms_partials(rows, n) * n floats; unused where that is one
  int64_t rows, n;
  int storage;
};
int64_t rms_partials(int64_t rows, int64_t n);
hipError_t launch_rms_norm_backward(const RmsGradArgs& a, hipStream_t stream);

// The product in 8 bits (linear_fp8.hip): D (m x n) = A B^T, both operands along k, with GemmArgs' epilogue.
struct Gemm8Args {
  GemmArgs g;  // (a, b, lda and ldb are not used)
  Fp8Operand a, b;
};
// K2, K4: two or four groups of waves, each with stages of its own
enum Linear8Tile {
  kTile8_32x64,
  kTile8_64,
  kTile8_64x128,
  kTile8_32x64K4,
  kTile8_64x128K2,
  kTile8_128,
  kTile8_128K2,
  kTile8_128x256,
  kTile8_256,
  kLinear8Tiles
};
using Linear8Fn = hipError_t (*)(const Gemm8Args&, hipStream_t);
using Linear8PairFn = hipError_t (*)(const Gemm8Args&, const Gemm8Args&, hipStream_t);
struct Linear8Table {
  Linear8Fn fn[kLinear8Tiles];  // null where one is not built
  Linear8PairFn pair[kLinear8Tiles];
  Linear8Fn few[3][2];          // 16, 32, 64 rows of A at most; 16 or 32 rows of B to a workgroup
};
Linear8Table linear_fp8_table_f32();
Linear8Table linear_fp8_table_bf16();
Linear8Table linear_fp8_table_f16();

int64_t linear_fp8_forward_workspace(const LinearSizes& s);
int64_t linear_fp8_backward_workspace(const LinearSizes& s, bool dx, bool dw, bool db);

struct LinearFp8Forward {
  LinearSizes s;
  Fp8Operand x, w;
  const void* bias;
  const void* residual;
  int64_t ldr;
  void* y;
  int64_t ldy;
  Checkpoint ck;
  void* workspace;
};
hipError_t launch_linear_fp8_forward(const LinearFp8Forward& a, hipStream_t stream);

// x: [d_in][tokens], w: [d_in][d_out]
struct LinearFp8Backward {
  LinearSizes s;
  const void* dy;
  int64_t ldg;
  Checkpoint ck;
  Fp8Operand x, w;
  const void* add;
  int64_t lda;
  void* dx;
  int64_t ldd;
  void* dw;
  int64_t lddw;
  void* db;
  void* workspace;
};
hipError_t launch_linear_fp8_backward(const LinearFp8Backward& a, hipStream_t stream);

}  // namespace rdfft
