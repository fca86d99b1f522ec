// act8_kernels.hip -- activations into 8-bit checkpoints (dense_device.hpp) and back.
//
// Both directions move bytes and little else: S * n in and n * 33/32 out a row (or the reverse), S the
// storage size.  A thread takes eight values, four lanes a block of 32, so the block's
// maximum is two cross-lane moves and nothing goes through LDS.  Rows that follow each other
// without a gap and end with a block are one long row, which needs no index arithmetic.
//
// 16384 x 4096 bf16 values: quantize 39 us (203 MB, 5.2 TB/s), dequantize 31 us (6.6 TB/s); a copy of 1 GiB runs at
// 5.2 TB/s.  128 x 256 floats: 2.9 us each, a launch's length.
#include <hip/hip_runtime.h>

#include "dense_device.hpp"
#include "dense_launch.hpp"

namespace rdfft {

constexpr int kActWG = 256;

// lanes: threads along a row, a power of two from 4 to kActWG; kActWG / lanes rows to a workgroup.
// The quads stay whole in the loop: a row is gone through in whole blocks.
template <class E>
__global__ void __launch_bounds__(kActWG) act8_quantize_kernel(const typename E::T* __restrict__ x, int64_t ldx,
                                                               int8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                                               int64_t rows, int64_t n, int64_t blocks, int lanes) {
  const int64_t row = (int64_t)blockIdx.y * (kActWG / lanes) + threadIdx.x / lanes;
  if (row >= rows) return;
  const int lane = threadIdx.x & (lanes - 1);
  x += row * ldx;
  codes += row * n;
  scales += row * blocks;
  const int64_t step = (int64_t)gridDim.x * lanes * kVec;
  for (int64_t i = ((int64_t)blockIdx.x * lanes + lane) * kVec; i < blocks * kCkBlock; i += step) {
    float v[kVec];
    read_group<E>(x, i, n, v);
    write_checkpoint(codes, scales, i, n, v);
  }
}

template <class E>
__global__ void __launch_bounds__(kActWG) act8_dequantize_kernel(const int8_t* __restrict__ codes,
                                                                 const uint8_t* __restrict__ scales,
                                                                 typename E::T* __restrict__ out, int64_t ldo,
                                                                 int64_t rows, int64_t n, int64_t blocks, int lanes) {
  const int64_t row = (int64_t)blockIdx.y * (kActWG / lanes) + threadIdx.x / lanes;
  if (row >= rows) return;
  const int lane = threadIdx.x & (lanes - 1);
  out += row * ldo;
  codes += row * n;
  scales += row * blocks;
  const int64_t step = (int64_t)gridDim.x * lanes * kVec;
  for (int64_t i = ((int64_t)blockIdx.x * lanes + lane) * kVec; i < n; i += step) {
    const Bytes8 c = i + kVec <= n ? *reinterpret_cast<const Bytes8*>(codes + i) : tail_codes(codes, i, n);
    float v[kVec];
    ck_decode<E>(c, ck_scale(scales[i / kCkBlock]), v);
    write_group<E>(out, i, n, v);
  }
}

// fn(grid, lanes, first row, rows) for launches that cover `rows` rows of n values
template <class F>
static hipError_t act8_launches(int64_t rows, int64_t n, int num_cu, F&& fn) {
  const int64_t groups = (n + kCkBlock - 1) / kCkBlock * kCkLanes;
  int lanes = kCkLanes;
  while (lanes < kActWG && lanes < groups) lanes *= 2;
  const int per = kActWG / lanes;
  constexpr int64_t kMaxY = 65535;
  for (int64_t r0 = 0; r0 < rows; r0 += kMaxY * per) {
    const int64_t r = std::min(rows - r0, kMaxY * per), gy = (r + per - 1) / per;
    // one long row spreads over the chip, several times over
    const int64_t most = std::max<int64_t>(1, (int64_t)num_cu * 32 / gy);
    const int64_t gx = std::min((groups + lanes - 1) / lanes, most);
    fn(dim3((unsigned)gx, (unsigned)gy), lanes, r0, r);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class E>
static hipError_t quantize(const void* x, int64_t ldx, int8_t* codes, uint8_t* scales, int64_t rows, int64_t n,
                           hipStream_t stream, int num_cu) {
  if (ldx == n && n % kCkBlock == 0) {
    n *= rows;
    rows = 1;
    ldx = n;
  }
  const int64_t blocks = (n + kCkBlock - 1) / kCkBlock;
  return act8_launches(rows, n, num_cu, [&](dim3 grid, int lanes, int64_t r0, int64_t r) {
    hipLaunchKernelGGL(act8_quantize_kernel<E>, grid, dim3(kActWG), 0, stream,
                       static_cast<const typename E::T*>(x) + r0 * ldx, ldx, codes + r0 * n, scales + r0 * blocks, r, n,
                       blocks, lanes);
  });
}

template <class E>
static hipError_t dequantize(const int8_t* codes, const uint8_t* scales, void* out, int64_t ldo, int64_t rows, int64_t n,
                             hipStream_t stream, int num_cu) {
  if (ldo == n && n % kCkBlock == 0) {
    n *= rows;
    rows = 1;
    ldo = n;
  }
  const int64_t blocks = (n + kCkBlock - 1) / kCkBlock;
  return act8_launches(rows, n, num_cu, [&](dim3 grid, int lanes, int64_t r0, int64_t r) {
    hipLaunchKernelGGL(act8_dequantize_kernel<E>, grid, dim3(kActWG), 0, stream, codes + r0 * n, scales + r0 * blocks,
                       static_cast<typename E::T*>(out) + r0 * ldo, ldo, r, n, blocks, lanes);
  });
}

hipError_t launch_act8_quantize(const void* x, int64_t ldx, int8_t* codes, uint8_t* scales, int64_t rows, int64_t n,
                                int storage, hipStream_t stream, int num_cu) {
  return with_elem(storage, [&](auto e) { return quantize<decltype(e)>(x, ldx, codes, scales, rows, n, stream, num_cu); });
}

hipError_t launch_act8_dequantize(const int8_t* codes, const uint8_t* scales, void* out, int64_t ldo, int64_t rows,
                                  int64_t n, int storage, hipStream_t stream, int num_cu) {
  return with_elem(storage,
                   [&](auto e) { return dequantize<decltype(e)>(codes, scales, out, ldo, rows, n, stream, num_cu); });
}

}  // namespace rdfft
