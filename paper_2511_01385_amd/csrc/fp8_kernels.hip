// fp8_kernels.hip -- matrices into 8-bit floating point (fp8_device.hpp) and back.
//
// A product in 8 bits needs its operands in blocks along k: activations by rows for y = x W^T, by columns (the rows
// of the transpose) for dW = dz^T x, a weight both ways.  One pass reads the matrix and leaves whichever are
// wanted; in a backward pass it also takes dy through the activation's slope and sums dz over the rows.
//
// A workgroup holds a tile of 128 x 128 values in registers, eight rows by eight columns to a thread: a block
// along the row is then 16 lanes of a DPP row, a block along the column all the threads with the same columns (four
// in a wave, by LDS from wave to wave), and a thread has eight consecutive codes in either direction.
#include <hip/hip_runtime.h>

#include "fp8_device.hpp"
#include "fp8_launch.hpp"
#include "linear_kernels.hpp"

namespace rdfft {

constexpr int kFp8WG = 256, kFp8Waves = kFp8WG / 64;

// the maximum and the sum over the four lanes of a wave that are equal modulo 16, in a fixed order
__device__ __forceinline__ uint32_t across_rows_max(uint32_t v) {
  v = max(v, (uint32_t)__shfl_xor((int)v, 16));
  return max(v, (uint32_t)__shfl_xor((int)v, 32));
}
__device__ __forceinline__ float across_rows_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

template <class E, bool EXACT>
__global__ void __launch_bounds__(kFp8WG) fp8_quantize_kernel(Fp8Quantize q) {
  using T = typename E::T;
  __shared__ uint32_t top[kFp8Waves][kFp8Block];
  __shared__ float sums[kFp8Waves][kFp8Block];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  const int64_t row0 = ((int64_t)blockIdx.y * kFp8Block) + threadIdx.x / kFp8Lanes * kVec;
  const int64_t col0 = (int64_t)blockIdx.x * kFp8Block, col = col0 + threadIdx.x % kFp8Lanes * kVec;
  const int64_t rows = q.rows, n = q.n;
  const T* const x = static_cast<const T*>(q.x);

  float v[kVec][kVec];
  if constexpr (EXACT) {
    // (rows and columns past the ends load what is near, without a branch)
    typename E::Raw raw[kVec];
    const int64_t c = min(col, n - kVec);
#pragma unroll
    for (int r = 0; r < kVec; ++r) raw[r] = E::load(x + min(row0 + r, rows - 1) * q.ldx + c);
#pragma unroll
    for (int r = 0; r < kVec; ++r) {
      E::widen(raw[r], v[r]);
      const bool in = row0 + r < rows && col < n;
#pragma unroll
      for (int i = 0; i < kVec; ++i) v[r][i] = in ? v[r][i] : 0.f;
    }
  } else {
#pragma unroll
    for (int r = 0; r < kVec; ++r) {
      if (row0 + r < rows && col < n) {
        read_group<E>(x + (row0 + r) * q.ldx, col, n, v[r]);
      } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[r][i] = 0.f;
      }
    }
  }
  if (q.act != kActNone) {
    const int64_t blocks = (n + kCkBlock - 1) / kCkBlock;
#pragma unroll
    for (int r = 0; r < kVec; ++r) {
      if (row0 + r >= rows || col >= n) continue;
      float z[kVec];
      const int8_t* const codes = q.ck.codes + (row0 + r) * n;
      const Bytes8 code = col + kVec <= n ? *reinterpret_cast<const Bytes8*>(codes + col) : tail_codes(codes, col, n);
      ck_decode<ElemF32>(code, ck_scale(q.ck.scales[(row0 + r) * blocks + col / kCkBlock]), z);
      times_slope8(q.act, z, v[r]);
    }
  }
  if (q.sums != nullptr) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      float s = v[0][i];
#pragma unroll
      for (int r = 1; r < kVec; ++r) s += v[r][i];
      s = across_rows_sum(s);
      if (lane < kFp8Lanes) sums[wave][lane * kVec + i] = s;
    }
  }
  // the largest of each column
  const bool by_column = q.columns.codes != nullptr || q.tiles;
  if (by_column) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      uint32_t m = abs_bits(v[0][i]);
#pragma unroll
      for (int r = 1; r < kVec; ++r) m = max(m, abs_bits(v[r][i]));
      m = across_rows_max(m);
      if (lane < kFp8Lanes) top[wave][lane * kVec + i] = m;
    }
  }
  if (by_column || q.sums != nullptr) __syncthreads();
  if (q.sums != nullptr && threadIdx.x < kFp8Block && col0 + threadIdx.x < n) {
    float s = sums[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < kFp8Waves; ++w) s += sums[w][threadIdx.x];
    q.sums[(int64_t)blockIdx.y * n + col0 + threadIdx.x] = s;
  }
  uint32_t column_top[kVec];
  int tile = 0;
  if (by_column) {
    uint32_t all = 0;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      uint32_t m = 0;
#pragma unroll
      for (int w = 0; w < kFp8Waves; ++w) m = max(m, top[w][threadIdx.x % kFp8Lanes * kVec + i]);
      column_top[i] = m;
      all = max(all, m);
    }
    tile = fp8_scale_byte(row_max(all));
  }
  if (q.held.codes != nullptr) {
#pragma unroll
    for (int r = 0; r < kVec; ++r) {
      const int s = q.tiles ? tile : fp8_scale_byte(row_max(max_bits8(v[r])));
      if (row0 + r >= rows || col >= n) continue;
      write_bytes(q.held.codes + (row0 + r) * q.held.ld, col, n, fp8_encode(v[r], s));
      if (threadIdx.x % kFp8Lanes == 0 && (!q.tiles || (threadIdx.x == 0 && r == 0)))
        q.held.scales[(q.tiles ? (int64_t)blockIdx.y : row0 + r) * q.held.lds + blockIdx.x] = (uint8_t)s;
    }
  }
  if (q.columns.codes != nullptr) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      if (row0 >= rows || col + i >= n) continue;
      const int s = q.tiles ? tile : fp8_scale_byte(column_top[i]);
      float t[kVec];
#pragma unroll
      for (int r = 0; r < kVec; ++r) t[r] = v[r][i];
      write_bytes(q.columns.codes + (col + i) * q.columns.ld, row0, rows, fp8_encode(t, s));
      if (threadIdx.x < kFp8Lanes && (!q.tiles || (threadIdx.x == 0 && i == 0)))
        q.columns.scales[(q.tiles ? (int64_t)blockIdx.x : col + i) * q.columns.lds + blockIdx.y] = (uint8_t)s;
    }
  }
}

template <class E>
__global__ void __launch_bounds__(kFp8WG) fp8_dequantize_kernel(Fp8Operand from, typename E::T* __restrict__ out, int64_t ldo,
                                                                int64_t row0, int64_t rows, int64_t n, int lanes) {
  const int64_t row = row0 + (int64_t)blockIdx.y * (kFp8WG / lanes) + threadIdx.x / lanes;
  if (row >= rows) return;
  const int lane = threadIdx.x & (lanes - 1);
  out += row * ldo;
  const int8_t* const codes = reinterpret_cast<const int8_t*>(from.codes) + row * from.ld;
  const uint8_t* const scales = from.scales + (row >> from.shift) * from.lds;
  const int64_t step = (int64_t)gridDim.x * lanes * kVec;
  for (int64_t i = ((int64_t)blockIdx.x * lanes + lane) * kVec; i < n; i += step) {
    const Bytes8 c = i + kVec <= n ? *reinterpret_cast<const Bytes8*>(codes + i) : tail_codes(codes, i, n);
    float v[kVec];
    fp8_decode<E>(c, scales[i / kFp8Block], v);
    write_group<E>(out, i, n, v);
  }
}

hipError_t launch_fp8_quantize(const Fp8Quantize& q, hipStream_t stream) {
  const int64_t tx = (q.n + kFp8Block - 1) / kFp8Block, ty = (q.rows + kFp8Block - 1) / kFp8Block;
  return with_elem(q.storage, [&](auto e) {
    using E = decltype(e);
    const auto go = [&](auto kernel) {
      // (a grid has at most 65535 rows of workgroups)
      constexpr int64_t kMaxY = 65535;
      for (int64_t t0 = 0; t0 < ty; t0 += kMaxY) {
        Fp8Quantize p = q;
        const int64_t r0 = t0 * kFp8Block, bands = std::min(ty - t0, kMaxY);
        p.x = static_cast<const typename E::T*>(q.x) + r0 * q.ldx;
        p.rows = std::min(q.rows - r0, bands * kFp8Block);
        if (q.ck.codes != nullptr) {
          p.ck.codes += r0 * q.n;
          p.ck.scales += r0 * ((q.n + kCkBlock - 1) / kCkBlock);
        }
        if (q.sums != nullptr) p.sums += t0 * q.n;
        if (q.held.codes != nullptr) {
          p.held.codes += r0 * q.held.ld;
          p.held.scales += (q.tiles ? t0 : r0) * q.held.lds;
        }
        if (q.columns.codes != nullptr) {
          p.columns.codes += r0;
          p.columns.scales += t0;
        }
        hipLaunchKernelGGL(kernel, dim3((unsigned)tx, (unsigned)bands), dim3(kFp8WG), 0, stream, p);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
      }
      return hipSuccess;
    };
    return q.n % kVec == 0 ? go(fp8_quantize_kernel<E, true>) : go(fp8_quantize_kernel<E, false>);
  });
}

hipError_t launch_fp8_dequantize(const Fp8Operand& from, void* out, int64_t ldo, int64_t rows, int64_t n, int storage,
                                 hipStream_t stream, int num_cu) {
  return with_elem(storage, [&](auto e) {
    using E = decltype(e);
    const int64_t groups = (n + kVec - 1) / kVec;
    int lanes = 1;
    while (lanes < kFp8WG && lanes < groups) lanes *= 2;
    const int per = kFp8WG / lanes;
    constexpr int64_t kMaxY = 65535;
    for (int64_t r0 = 0; r0 < rows; r0 += kMaxY * per) {
      const int64_t gy = (std::min(rows - r0, kMaxY * per) + per - 1) / per;
      const int64_t gx = std::min((groups + lanes - 1) / lanes, std::max<int64_t>(1, (int64_t)num_cu * 32 / gy));
      hipLaunchKernelGGL(fp8_dequantize_kernel<E>, dim3((unsigned)gx, (unsigned)gy), dim3(kFp8WG), 0, stream, from,
                         static_cast<typename E::T*>(out), ldo, r0, rows, n, lanes);
      const hipError_t err = hipGetLastError();
      if (err != hipSuccess) return err;
    }
    return hipSuccess;
  });
}

}  // namespace rdfft
