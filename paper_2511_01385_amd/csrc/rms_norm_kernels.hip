// rms_norm_kernels.hip -- root-mean-square norm of rows of n values, forward and backward.
//
//   u = round(x + r),  rstd = (mean(u^2) + eps)^-1/2,  y = u rstd w
//   xh = u rstd,  g = dy w,  dx = rstd (g - xh mean(g xh)) + add,  dw = sum over rows of dy xh
//
// The sum is rounded to the storage type first: the residual stream is kept in that type, and the norm is of what is
// kept, so that the backward's gradient is that of the function that was computed.
//
// Both are bound by HBM.  As in the layer norm TPR threads hold a row in registers, C groups of eight values each,
// so that every tensor is read once and the sum, y, y in 8-bit floating point (16 lanes to a block of 128) and the
// checkpoint all leave in the same pass.  Weights, and in the backward the sums of dw, stay in
// registers from row to row; the partial sums of dw are joined by a second launch in a fixed order (no atomics).
//
// 16384 x 4096 bf16 with the sum, y and a checkpoint written: forward 103 us (606 MB, 5.9 TB/s), backward from the checkpoint
// with a gradient added 104 us and 5 for the join (472 MB, 4.5 TB/s; a copy of 1 GiB runs at 5.1).  2045 x 769 float32: 8.4,
// 7.8 and 3.0 us; with a branch to each group of an odd row 12.9, 10.0 and 3.9.  One token of 4096: 2.9 us, a launch's length.
// Rows of more than 8192 values spill in the backward: u, g, the next row's values, w and dw of two groups do not fit the 128
// registers of a thread among 1024 (24 to 41 of them are spilled for 16-bit types, 66 to 111 for float32).  4096 x 16384 bf16
// with a gradient added takes 107 us from the sum (5.0 TB/s; 8192 x 8192, as many values, 99) and 125 from a checkpoint (86);
// float32 223 and 233 (195, 158).
#include <hip/hip_runtime.h>

#include "fp8_device.hpp"
#include "fp8_launch.hpp"
#include "norm_device.hpp"

namespace rdfft {

template <int TPR>
constexpr int rms_fwd_wg() {
  return TPR > 256 ? TPR : 256;
}

// Rows of whole groups, of any length of at least eight, and shorter ones (value by value)
enum RowsOf { kWholeGroups, kCutGroups, kShort };
template <class E, RowsOf ROWS>
using RmsGroup = std::conditional_t<ROWS == kCutGroups, ShiftedGroup<E>, RowGroup<E, ROWS == kWholeGroups>>;

// eight values as the storage type holds them
template <class E>
__device__ __forceinline__ void round_group(float* v) {
  if constexpr (E::kId != kStorageF32) {
    typename E::T t[kVec];
    E::store(t, v);
    E::widen(E::load(t), v);
  }
}

template <class E, int TPR, int C, RowsOf ROWS>
__global__ void __launch_bounds__(rms_fwd_wg<TPR>()) rms_norm_forward_kernel(RmsArgs a) {
  using T = typename E::T;
  constexpr int WG = rms_fwd_wg<TPR>(), GROUPS = TPR > 64 ? 1 : WG / TPR;
  static_assert(TPR == 64 || TPR == WG, "groups longer than a wave are alone in their workgroup");
  __shared__ float red[2 * (WG / 64)];
  int turn = 0;
  const int lane = threadIdx.x % TPR;
  const int n = (int)a.n, blocks = (n + kCkBlock - 1) / kCkBlock;
  const float count = (float)n;
  int at[C];
  float w[C][kVec];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    at[c] = (c * TPR + lane) * kVec;
    read_group<ElemF32>(a.weight, at[c], n, w[c]);
  }
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  // (a wave lies in one row: addresses of rows are scalar)
  for (int64_t row = (int64_t)blockIdx.x * GROUPS + __builtin_amdgcn_readfirstlane((int)threadIdx.x / TPR); row < a.rows;
       row += step) {
    const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* const r = static_cast<const T*>(a.residual) + row * a.ldr;
    float u[C][kVec];
    RmsGroup<E, ROWS> xs[C], rs[C];
#pragma unroll
    for (int c = 0; c < C; ++c) xs[c].load(x, at[c], n);
    if (a.residual != nullptr) {
#pragma unroll
      for (int c = 0; c < C; ++c) rs[c].load(r, at[c], n);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) xs[c].widen(x, at[c], n, u[c]);
    if (a.residual != nullptr) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float v[kVec];
        rs[c].widen(r, at[c], n, v);
#pragma unroll
        for (int k = 0; k < kVec; ++k) u[c][k] += v[k];
        round_group<E>(u[c]);
      }
    }
    float s[1] = {0.f}, unit = 1.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < kVec; ++k) s[0] = fmaf(u[c][k], u[c][k], s[0]);
    group_sums<TPR, 1>(s, red, turn);
    // squares that leave float32's range are taken of the values times a power of two (the sum is the same in all
    // threads; with an infinity among them it is infinite again: the infinity becomes NaN, the row's other values 0)
    if (!(s[0] <= 0x1.fffffep127f) || (s[0] < 0x1p-80f && a.eps < 0x1p-100f)) {
      unit = s[0] < 1.f ? 0x1p100f : 0x1p-80f;
      s[0] = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int k = 0; k < kVec; ++k) s[0] = fmaf(u[c][k] * unit, u[c][k] * unit, s[0]);
      group_sums<TPR, 1>(s, red, turn);
    }
    const float root = sqrtf(s[0] / count + a.eps * unit * unit), rstd = unit / root;
    if (lane == 0 && a.rstd != nullptr) a.rstd[row] = rstd;
    if (a.summed != nullptr) {
      T* const h = static_cast<T*>(a.summed) + row * a.lds;
#pragma unroll
      for (int c = 0; c < C; ++c) store_group<E, ROWS == kWholeGroups>(h, at[c], n, u[c]);
    }
    if (a.ck.codes != nullptr) {
#pragma unroll
      for (int c = 0; c < C; ++c) write_checkpoint(a.ck.codes + row * n, a.ck.scales + row * blocks, at[c], n, u[c]);
    }
    float times = rstd;
    if (unit > 1.f) {  // rstd may be past the largest number; values as small can be scaled without loss
      times = 1.f / root;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int k = 0; k < kVec; ++k) u[c][k] *= unit;
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < kVec; ++k) u[c][k] = u[c][k] * times * w[c][k];
    if (a.y != nullptr) {
      T* const y = static_cast<T*>(a.y) + row * a.ldy;
#pragma unroll
      for (int c = 0; c < C; ++c) store_group<E, ROWS == kWholeGroups>(y, at[c], n, u[c]);
    }
    if (a.y8.codes != nullptr) {
#pragma unroll
      for (int c = 0; c < C; ++c) write_fp8(a.y8.codes + row * a.y8.ld, a.y8.scales + row * a.y8.lds, at[c], n, u[c]);
    }
  }
}

constexpr int kRmsBwdWG = 1024;
// Groups that take a row each.  (With more threads to a row than a workgroup has there would be none, and no end to the rows.)
template <int TPR>
constexpr int rms_bwd_groups() {
  static_assert(kRmsBwdWG % TPR == 0, "a workgroup holds whole rows");
  return kRmsBwdWG / TPR;
}
template <int TPR, int C>
constexpr int rms_bwd_lds() {
  constexpr int groups = rms_bwd_groups<TPR>();
  return groups == 1 ? 0 : groups * TPR * C * kVec * 4;
}

// A row's dy, what is added to dx, and the norm's input (or its checkpoint), on their way from memory
template <class E, int TPR, int C, bool CK, RowsOf ROWS>
struct RmsRow {
  using T = typename E::T;
  RmsGroup<E, ROWS> dy[C], u[CK ? 1 : C], add[C];
  Bytes8 codes[CK ? C : 1];
  int scale[CK ? C : 1];
  float rstd;

  __device__ __forceinline__ void load(const RmsGradArgs& a, int64_t row, const int* at, int n, int blocks) {
    rstd = a.rstd[row];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      dy[c].load(static_cast<const T*>(a.dy) + row * a.ldg, at[c], n);
      if constexpr (CK) {
        const int i = at[c] < n ? at[c] : 0;
        if constexpr (ROWS == kWholeGroups) codes[c] = *reinterpret_cast<const Bytes8*>(a.ck.codes + row * n + i);
        else if constexpr (ROWS == kCutGroups) codes[c] = shifted_codes(a.ck.codes + row * n, at[c], n);
        else codes[c] = tail_codes(a.ck.codes + row * n, at[c], n);
        scale[c] = a.ck.scales[row * blocks + i / kCkBlock];
      } else {
        u[c].load(static_cast<const T*>(a.u) + row * a.ldu, at[c], n);
      }
      if (a.add != nullptr) add[c].load(static_cast<const T*>(a.add) + row * a.lda, at[c], n);
    }
  }
  __device__ __forceinline__ void widen(const RmsGradArgs& a, int64_t row, const int* at, int n, int blocks,
                                        float (*g)[kVec], float (*v)[kVec]) const {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      dy[c].widen(static_cast<const T*>(a.dy) + row * a.ldg, at[c], n, g[c]);
      if constexpr (CK) {
        ck_decode<ElemF32>(codes[c], ck_scale(scale[c]), v[c]);
#pragma unroll
        for (int k = 0; k < kVec; ++k) v[c][k] = at[c] < n ? v[c][k] : 0.f;
      } else {
        u[c].widen(static_cast<const T*>(a.u) + row * a.ldu, at[c], n, v[c]);
      }
    }
  }
};

// Each workgroup's sums go to dw_out + blockIdx.x * n.
template <class E, int TPR, int C, bool CK, RowsOf ROWS>
__global__ void __launch_bounds__(kRmsBwdWG) rms_norm_backward_kernel(RmsGradArgs a, float* dw_out) {
  using T = typename E::T;
  constexpr int WG = kRmsBwdWG, GROUPS = rms_bwd_groups<TPR>();
  __shared__ float red[2 * (WG / 64)];
  int turn = 0;
  const int lane = threadIdx.x % TPR, grp = __builtin_amdgcn_readfirstlane((int)threadIdx.x / TPR);  // (one in a wave)
  const int n = (int)a.n, blocks = (n + kCkBlock - 1) / kCkBlock;
  const float inv_n = 1.0f / (float)n;
  int at[C];
  float w[C][kVec], dw[C][kVec];
  const int64_t step = (int64_t)gridDim.x * GROUPS;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    at[c] = (c * TPR + lane) * kVec;
    read_group<ElemF32>(a.weight, at[c], n, w[c]);
#pragma unroll
    for (int k = 0; k < kVec; ++k) dw[c][k] = 0.f;
  }
  int64_t row = (int64_t)blockIdx.x * GROUPS + grp;
  using Row = RmsRow<E, TPR, C, CK, ROWS>;
  // (the groups of a workgroup take the same number of rows: they meet at barriers)
  const auto work = [&](const Row& in, bool act, auto&& loads) {
    float u[C][kVec], g[C][kVec], more[C][kVec];
    float rstd = 0.f;
    if (act) {
      rstd = in.rstd;
      in.widen(a, row, at, n, blocks, g, u);
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int k = 0; k < kVec; ++k) g[c][k] = u[c][k] = 0.f;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (act && a.add != nullptr) {
        in.add[c].widen(static_cast<const T*>(a.add) + row * a.lda, at[c], n, more[c]);
      } else {
#pragma unroll
        for (int k = 0; k < kVec; ++k) more[c][k] = 0.f;
      }
    }
    loads();  // of a later row, into the registers that are free now
    float s[1] = {0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        u[c][k] *= rstd;
        dw[c][k] = fmaf(g[c][k], u[c][k], dw[c][k]);
        g[c][k] *= w[c][k];
        s[0] = fmaf(g[c][k], u[c][k], s[0]);
      }
    group_sums<TPR, 1>(s, red, turn);
    if (act) {
      const float mean = s[0] * inv_n;
      T* const dx = static_cast<T*>(a.dx) + row * a.ldd;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float v[kVec];
#pragma unroll
        for (int k = 0; k < kVec; ++k) v[k] = fmaf(rstd, g[c][k] - u[c][k] * mean, more[c][k]);
        store_group<E, ROWS == kWholeGroups>(dx, at[c], n, v);
      }
    }
    row += step;
  };
  int64_t row0 = (int64_t)blockIdx.x * GROUPS;
  // rows that are on their way while one is worked on, as far as the registers go
  constexpr int AHEAD = C > 1 ? 0 : E::kId == kStorageF32 && !CK ? 1 : 2;
  Row in[AHEAD > 1 ? 2 : 1];
  const auto load = [&](Row& to, int64_t r) {
    if (r < a.rows) to.load(a, r, at, n, blocks);
  };
#pragma unroll
  for (int q = 0; q < AHEAD; ++q) load(in[q], row + q * step);
  for (; row0 < a.rows; row0 += step) {
    if constexpr (AHEAD == 0) load(in[0], row);
    work(in[0], row < a.rows, [&] {
      if constexpr (AHEAD > 0) load(in[0], row + AHEAD * step);
    });
    if constexpr (AHEAD > 1) {
      row0 += step;
      if (row0 >= a.rows) break;
      work(in[1], row < a.rows, [&] { load(in[1], row + AHEAD * step); });
    }
  }
  if (dw_out == nullptr) return;
  dw_out += blockIdx.x * a.n;
  if constexpr (GROUPS == 1) {
#pragma unroll
    for (int c = 0; c < C; ++c) write_group<ElemF32>(dw_out, at[c], n, dw[c]);
  } else {
    constexpr int COLS = TPR * C * kVec;
    extern __shared__ float sums[];  // [GROUPS][COLS]
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < kVec; ++k)  // value k of all lanes side by side: no two lanes of a wave meet in a bank
        sums[grp * COLS + (c * kVec + k) * TPR + lane] = dw[c][k];
    __syncthreads();
    for (int p = threadIdx.x; p < COLS; p += WG) {
      float v = sums[p];
#pragma unroll
      for (int o = 1; o < GROUPS; ++o) v += sums[o * COLS + p];
      const int i = (p / TPR / kVec * TPR + p % TPR) * kVec + p / TPR % kVec;
      if (i < n) dw_out[i] = v;
    }
  }
}

// fn(storage type, threads of a row, groups of eight per thread, RowsOf); pick: with_row or with_row_backward
template <class Pick, class F>
static hipError_t with_rows(int storage, int64_t n, Pick&& pick, F&& fn) {
  using std::integral_constant;
  return with_elem(storage, [&](auto e) {
    if (n < kVec) return fn(e, integral_constant<int, 64>{}, integral_constant<int, 1>{}, integral_constant<RowsOf, kShort>{});
    return pick(n, [&](auto tpr, auto c) {
      return n % kVec == 0 ? fn(e, tpr, c, integral_constant<RowsOf, kWholeGroups>{})
                           : fn(e, tpr, c, integral_constant<RowsOf, kCutGroups>{});
    });
  });
}

hipError_t launch_rms_norm_forward(const RmsArgs& a, hipStream_t stream, int num_cu) {
  const auto pick = [](int64_t n, auto&& fn) { return with_row(n, fn); };
  return with_rows(a.storage, a.n, pick, [&](auto e, auto tpr, auto c, auto of) {
    constexpr int TPR = decltype(tpr)::value, C = decltype(c)::value, WG = rms_fwd_wg<TPR>();
    constexpr int groups = TPR > 64 ? 1 : WG / TPR;
    // as many workgroups as are on the chip at once
    const int64_t grid = std::min((a.rows + groups - 1) / groups, (int64_t)num_cu * (2048 / WG));
    hipLaunchKernelGGL((rms_norm_forward_kernel<decltype(e), TPR, C, decltype(of)::value>), dim3((unsigned)grid), dim3(WG), 0,
                       stream, a);
    return hipGetLastError();
  });
}

// Workgroups of the backward, each leaving one row of partial sums: one per CU of the largest device at most.  Rows that
// one workgroup goes through in two turns are left to it, whose sums are the result: that saves the second launch.
constexpr int64_t kRmsMaxPartials = 256;
int64_t rms_partials(int64_t rows, int64_t n) {
  int64_t groups = 1;
  (void)with_row_backward(n, [&](auto tpr, auto) {
    groups = rms_bwd_groups<decltype(tpr)::value>();
    return hipSuccess;
  });
  return rows <= 2 * groups ? 1 : std::min((rows + groups - 1) / groups, kRmsMaxPartials);
}

template <class E, int TPR, int C, bool CK, RowsOf ROWS>
static hipError_t rms_backward_launch(const RmsGradArgs& a, int64_t grid, float* dw, hipStream_t stream) {
  constexpr int lds = rms_bwd_lds<TPR, C>();
  const auto kernel = rms_norm_backward_kernel<E, TPR, C, CK, ROWS>;
  static const hipError_t ready = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                      hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (ready != hipSuccess) return ready;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kRmsBwdWG), lds, stream, a, dw);
  return hipGetLastError();
}

hipError_t launch_rms_norm_backward(const RmsGradArgs& a, hipStream_t stream) {
  const int64_t grid = rms_partials(a.rows, a.n);
  // a single workgroup's sums are the result
  float* const dw = a.dweight == nullptr ? nullptr : grid == 1 ? a.dweight : a.partials;
  const auto pick = [](int64_t n, auto&& fn) { return with_row_backward(n, fn); };
  const hipError_t err = with_rows(a.storage, a.n, pick, [&](auto e, auto tpr, auto c, auto of) {
    using E = decltype(e);
    constexpr int TPR = decltype(tpr)::value, C = decltype(c)::value;
    constexpr RowsOf ROWS = decltype(of)::value;
    return a.u == nullptr ? rms_backward_launch<E, TPR, C, true, ROWS>(a, grid, dw, stream)
                          : rms_backward_launch<E, TPR, C, false, ROWS>(a, grid, dw, stream);
  });
  if (err != hipSuccess || grid == 1 || dw == nullptr) return err;
  return launch_column_finish(a.partials, grid, a.n, a.n, a.dweight, nullptr, kStorageF32, stream);
}

}  // namespace rdfft
