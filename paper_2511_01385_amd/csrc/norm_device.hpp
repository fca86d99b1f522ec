// norm_device.hpp -- what the norms over rows share: sums over the threads of a row, rows in groups of eight values,
// and how many threads take a row.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "dense_device.hpp"

namespace rdfft {

// Sums of K values over the TPR threads of a group, in each of them.  Groups longer than a wave are a
// workgroup's only ones or run in step; `red` holds [2][waves][K] and `turn` alternates.
template <int TPR, int K>
__device__ __forceinline__ void group_sums(float* v, float* red, int& turn) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = wave_sum(v[k]);
  if constexpr (TPR > 64) {
    const int waves = (int)blockDim.x / 64, wave = threadIdx.x / 64;
    float* const r = red + turn * waves * K;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) r[wave * K + k] = v[k];
    }
    turn ^= 1;
    __syncthreads();
    const float* const mine = r + wave / (TPR / 64) * (TPR / 64) * K;
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = mine[k];
#pragma unroll
    for (int w = 1; w < TPR / 64; ++w)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += mine[w * K + k];
  }
}

// Eight values of a row from i0, zeros past its end.  EXACT: n is a multiple of eight, so a group is in the
// row or out of it and its load needs no branch (an absent group's reads the row's start).
template <class E, bool EXACT>
struct RowGroup {
  using T = typename E::T;
  typename E::Raw raw;
  __device__ __forceinline__ void load(const T* row, int i0, int n) {
    if constexpr (EXACT) raw = E::load(row + (i0 < n ? i0 : 0));
  }
  __device__ __forceinline__ void widen(const T* row, int i0, int n, float* v) const {
    if constexpr (EXACT) {
      E::widen(raw, v);
#pragma unroll
      for (int k = 0; k < kVec; ++k) v[k] = i0 < n ? v[k] : 0.f;
    } else {
      read_group<E>(row, i0, n, v);
    }
  }
};
// The same for rows of any length of at least eight, loaded without a branch: a group that the row's end cuts is loaded so
// as to end there and shifted into place by the lanes that hold it.
template <class E>
struct ShiftedGroup {
  using T = typename E::T;
  typename E::Raw raw;
  __device__ __forceinline__ void load(const T* row, int i0, int n) { raw = E::load(row + min(i0, n - kVec)); }
  __device__ __forceinline__ void widen(const T*, int i0, int n, float* v) const {
    E::widen(raw, v);
    int past = i0 + kVec - n;
    if (past > 0) {
      asm volatile("" : "+v"(past));  // (what follows from it is not worth registers from row to row)
#pragma unroll
      for (int by = 4; by > 0; by /= 2)
#pragma unroll
        for (int k = 0; k < kVec; ++k) v[k] = past >= kVec ? 0.f : !(past & by) ? v[k] : k + by < kVec ? v[k + by] : 0.f;
    }
  }
};
// Eight codes of such a row's checkpoint, zeros past its end.
__device__ __forceinline__ Bytes8 shifted_codes(const int8_t* row, int i0, int n) {
  const Bytes8 c = *reinterpret_cast<const Bytes8*>(row + min(i0, n - kVec));
  const int past = min(max(i0 + kVec - n, 0), kVec);
  const uint64_t w = past == kVec ? 0 : ((uint64_t)c.w[1] << 32 | c.w[0]) >> (8 * past);
  return {{(uint32_t)w, (uint32_t)(w >> 32)}};
}

template <class E, bool EXACT>
__device__ __forceinline__ void store_group(typename E::T* row, int i0, int n, const float* v) {
  if constexpr (EXACT) {
    if (i0 < n) E::store(row + i0, v);
  } else {
    write_group<E>(row, i0, n, v);
  }
}

// fn(threads of a row, groups of eight per thread) by the row's length
template <class F>
hipError_t with_row(int64_t n, F&& fn) {
  using std::integral_constant;
  const auto go = [&](auto tpr, auto c) { return fn(tpr, c); };
  if (n <= 512) return go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (n <= 1024) return go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  if (n <= 2048) return go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (n <= 4096) return go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  if (n <= 8192) return go(integral_constant<int, 512>{}, integral_constant<int, 2>{});
  return go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}

// the same for the backward, whose threads also hold sums
template <class F>
hipError_t with_row_backward(int64_t n, F&& fn) {
  using std::integral_constant;
  const auto go = [&](auto tpr, auto c) { return fn(tpr, c); };
  if (n <= 512) return go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (n <= 1024) return go(integral_constant<int, 128>{}, integral_constant<int, 1>{});
  if (n <= 2048) return go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (n <= 4096) return go(integral_constant<int, 512>{}, integral_constant<int, 1>{});
  if (n <= 8192) return go(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
  return go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}

// whether rows are loaded and stored in whole groups only
inline bool exact_rows(int64_t n) { return n % kVec == 0; }
template <class F>
hipError_t with_exact(int64_t n, F&& fn) {
  return exact_rows(n) ? fn(std::true_type{}) : fn(std::false_type{});
}

}  // namespace rdfft
