// norm_kernels.hip -- layer norm of rows of n values, forward and backward.
//
//   u = x (+ r),  mu = mean(u),  rstd = (mean((u - mu)^2) + eps)^-1/2,  y = (u - mu) rstd w + b
//   xh = (u - mu) rstd,  g = dy w,  dx = rstd (g - mean(g) - xh mean(g xh)),
//   dw = sum over rows of dy xh,  db = sum over rows of dy
//
// Both are bound by HBM.  TPR threads hold a row in registers, C groups of eight values each, so that a
// row is read once: the variance is taken around the mean in a second look at the registers (no
// difference of large numbers).  The forward may leave u as an 8-bit checkpoint, of the float32 sum
// where there is a residual; the backward then reads n * 33/32 bytes a row in place of S * n (or 2 S n).
//
// A group of threads goes through rows one after another and keeps w (and b) in registers, and in
// the backward the sums of dw and db over its rows.  The groups of a workgroup are added in LDS
// in a fixed order and each workgroup leaves one row of partial sums (2n floats); a second launch adds
// those.  No atomics: results do not depend on the order of execution.
//
// 16384 x 4096 bf16 with a residual and a checkpoint: forward 91 us (472 MB, 5.2 TB/s), backward 76 us after forwards
// and 68 after itself (337 MB, 4.4 and 4.9 TB/s) and 5 us for the join; from x and the residual, without a checkpoint, 79 us
// (403 MB) and 99 (537 MB).  4096 x 768: 7.7, 8.4 and 3.5 us, two or three trips to memory one after another.  One wave per
// row up to 1024 values (no barrier), a workgroup beyond.  Rows of more than 8192 values run at half the rate in the
// backward, whose threads then hold two groups each and spill (4096 x 16384: forward 98 us, backward 137).
#include <hip/hip_runtime.h>

#include "dense_device.hpp"
#include "dense_launch.hpp"

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
template <class E, bool EXACT>
__device__ __forceinline__ void store_group(typename E::T* row, int i0, int n, const float* v) {
  if constexpr (EXACT) {
    if (i0 < n) E::store(row + i0, v);
  } else {
    write_group<E>(row, i0, n, v);
  }
}

template <int TPR>
constexpr int norm_fwd_wg() {
  return TPR > 256 ? TPR : 256;
}

template <class E, int TPR, int C, bool EXACT>
__global__ void __launch_bounds__(norm_fwd_wg<TPR>()) layer_norm_forward_kernel(NormArgs a) {
  using T = typename E::T;
  constexpr int WG = norm_fwd_wg<TPR>(), GROUPS = TPR > 64 ? 1 : WG / TPR;
  static_assert(TPR == 64 || TPR == WG, "groups longer than a wave are alone in their workgroup");
  __shared__ float red[2 * (WG / 64)];
  int turn = 0;
  const int lane = threadIdx.x % TPR;
  const int n = (int)a.n, blocks = (n + kCkBlock - 1) / kCkBlock;
  const float count = (float)n;
  int at[C];
  float w[C][kVec], b[C][kVec];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    at[c] = (c * TPR + lane) * kVec;
    read_group<ElemF32>(a.weight, at[c], n, w[c]);
    if (a.bias != nullptr) read_group<ElemF32>(a.bias, at[c], n, b[c]);
    else
#pragma unroll
      for (int k = 0; k < kVec; ++k) b[c][k] = 0.f;
  }
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  // (a wave lies in one row: addresses of rows are scalar)
  for (int64_t row = (int64_t)blockIdx.x * GROUPS + __builtin_amdgcn_readfirstlane((int)threadIdx.x / TPR); row < a.rows;
       row += step) {
    const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* const r = static_cast<const T*>(a.residual) + row * a.ldr;
    float u[C][kVec];
    RowGroup<E, EXACT> xs[C], rs[C];
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
      }
    }
    float s[1] = {0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < kVec; ++k) s[0] += u[c][k];
    group_sums<TPR, 1>(s, red, turn);
    const float mean = s[0] / count;  // (not times 1 / n: a constant row's mean is its value)
    if (a.ck.codes != nullptr) {
      int8_t* const codes = a.ck.codes + row * n;
      uint8_t* const scales = a.ck.scales + row * blocks;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int byte = ck_scale_byte(quad_max(max_bits8(u[c])));
        if (at[c] < n) {
          if constexpr (EXACT) *reinterpret_cast<Bytes8*>(codes + at[c]) = ck_encode(u[c], byte);
          else write_codes(codes, at[c], n, ck_encode(u[c], byte));
          if (at[c] % kCkBlock == 0) scales[at[c] / kCkBlock] = (uint8_t)byte;
        }
      }
    }
    s[0] = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        const bool in = EXACT ? at[c] < n : at[c] + k < n;
        u[c][k] = in ? u[c][k] - mean : 0.f;
        s[0] = fmaf(u[c][k], u[c][k], s[0]);
      }
    group_sums<TPR, 1>(s, red, turn);
    const float rstd = 1.0f / sqrtf(s[0] / count + a.eps);
    if (lane == 0) {
      if (a.mean != nullptr) a.mean[row] = mean;
      if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
    T* const y = static_cast<T*>(a.y) + row * a.ldy;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float v[kVec];
#pragma unroll
      for (int k = 0; k < kVec; ++k) v[k] = fmaf(u[c][k] * rstd, w[c][k], b[c][k]);
      store_group<E, EXACT>(y, at[c], n, v);
    }
  }
}

constexpr int kNormBwdWG = 1024;
template <int TPR, int C>
constexpr int norm_bwd_lds() {
  const int groups = kNormBwdWG / TPR;
  return groups == 1 ? 0 : groups * 2 * TPR * C * kVec * 4;
}

// A row's dy and the norm's input (or its checkpoint), on their way from memory
template <class E, int TPR, int C, bool CK, bool EXACT>
struct NormRow {
  using T = typename E::T;
  RowGroup<E, EXACT> dy[C], x[CK ? 1 : C], r[CK ? 1 : C];
  Bytes8 codes[CK ? C : 1];
  int scale[CK ? C : 1];
  float mean, rstd;

  __device__ __forceinline__ void load(const NormGradArgs& a, int64_t row, const int* at, int n, int blocks) {
    mean = a.mean[row];
    rstd = a.rstd[row];
    if constexpr (EXACT) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        dy[c].load(static_cast<const T*>(a.dy) + row * a.ldg, at[c], n);
        const int i = at[c] < n ? at[c] : 0;
        if constexpr (CK) {
          codes[c] = *reinterpret_cast<const Bytes8*>(a.ck.codes + row * n + i);
          scale[c] = a.ck.scales[row * blocks + i / kCkBlock];
        } else {
          x[c].load(static_cast<const T*>(a.x) + row * a.ldx, at[c], n);
          if (a.residual != nullptr) r[c].load(static_cast<const T*>(a.residual) + row * a.ldr, at[c], n);
        }
      }
    }
  }
  // g: dy, u: the norm's input
  __device__ __forceinline__ void widen(const NormGradArgs& a, int64_t row, const int* at, int n, int blocks,
                                        float (*g)[kVec], float (*u)[kVec]) const {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      dy[c].widen(static_cast<const T*>(a.dy) + row * a.ldg, at[c], n, g[c]);
      if constexpr (CK && EXACT) {
        ck_decode<ElemF32>(codes[c], ck_scale(scale[c]), u[c]);
      } else if constexpr (CK) {
        const int s = at[c] < n ? a.ck.scales[row * blocks + at[c] / kCkBlock] : 0;
        ck_decode<ElemF32>(tail_codes(a.ck.codes + row * n, at[c], n), ck_scale(s), u[c]);
      } else {
        x[c].widen(static_cast<const T*>(a.x) + row * a.ldx, at[c], n, u[c]);
        if (a.residual != nullptr) {
          float v[kVec];
          r[c].widen(static_cast<const T*>(a.residual) + row * a.ldr, at[c], n, v);
#pragma unroll
          for (int k = 0; k < kVec; ++k) u[c][k] += v[k];
        }
      }
    }
  }
};

// Each workgroup's sums go to dw_out + blockIdx.x * stride and db_out + blockIdx.x * stride.
template <class E, int TPR, int C, bool CK, bool EXACT>
__global__ void __launch_bounds__(kNormBwdWG)
    layer_norm_backward_kernel(NormGradArgs a, float* dw_out, float* db_out, int64_t stride) {
  using T = typename E::T;
  constexpr int WG = kNormBwdWG, GROUPS = WG / TPR;
  __shared__ float red[4 * (WG / 64)];
  int turn = 0;
  const int lane = threadIdx.x % TPR, grp = __builtin_amdgcn_readfirstlane((int)threadIdx.x / TPR);  // (one in a wave)
  const int n = (int)a.n, blocks = (n + kCkBlock - 1) / kCkBlock;
  const float inv_n = 1.0f / (float)n;
  int at[C];
  float w[C][kVec], dw[C][kVec], db[C][kVec];
  const int64_t step = (int64_t)gridDim.x * GROUPS;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    at[c] = (c * TPR + lane) * kVec;
    read_group<ElemF32>(a.weight, at[c], n, w[c]);
#pragma unroll
    for (int k = 0; k < kVec; ++k) dw[c][k] = db[c][k] = 0.f;
  }
  int64_t row = (int64_t)blockIdx.x * GROUPS + grp;
  const auto work = [&](const NormRow<E, TPR, C, CK, EXACT>& in, bool act, auto&& loads) {
    float u[C][kVec], g[C][kVec];
    float mean = 0.f, rstd = 0.f;
    if (act) {
      mean = in.mean;
      rstd = in.rstd;
      in.widen(a, row, at, n, blocks, g, u);
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int k = 0; k < kVec; ++k) g[c][k] = u[c][k] = 0.f;
    }
    loads();  // of a later row, into the registers that are free now
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        u[c][k] = (u[c][k] - mean) * rstd;
        dw[c][k] = fmaf(g[c][k], u[c][k], dw[c][k]);
        db[c][k] += g[c][k];
        g[c][k] *= w[c][k];
        s[0] += g[c][k];
        s[1] = fmaf(g[c][k], u[c][k], s[1]);
      }
    group_sums<TPR, 2>(s, red, turn);
    if (act) {
      const float m0 = s[0] * inv_n, m1 = s[1] * inv_n;
      T* const dx = static_cast<T*>(a.dx) + row * a.ldd;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float v[kVec];
#pragma unroll
        for (int k = 0; k < kVec; ++k) v[k] = rstd * (g[c][k] - m0 - u[c][k] * m1);
        store_group<E, EXACT>(dx, at[c], n, v);
      }
    }
    row += step;
  };
  // (the groups of a workgroup take the same number of rows: they meet at barriers)
  int64_t row0 = (int64_t)blockIdx.x * GROUPS;
  // rows that are on their way while one is worked on, as far as the registers go
  constexpr int AHEAD = C > 1 ? 0 : E::kId == kStorageF32 && !CK ? 1 : 2;
  NormRow<E, TPR, C, CK, EXACT> in[AHEAD > 1 ? 2 : 1];
  const auto load = [&](NormRow<E, TPR, C, CK, EXACT>& to, int64_t r) {
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
  dw_out += blockIdx.x * stride;
  db_out += blockIdx.x * stride;
  if constexpr (GROUPS == 1) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      write_group<ElemF32>(dw_out, at[c], n, dw[c]);
      write_group<ElemF32>(db_out, at[c], n, db[c]);
    }
  } else {
    constexpr int COLS = TPR * C * kVec;
    extern __shared__ float sums[];  // [GROUPS][2][COLS]
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        // value k of all lanes side by side: no two lanes of a wave meet in a bank
        sums[grp * 2 * COLS + (c * kVec + k) * TPR + lane] = dw[c][k];
        sums[grp * 2 * COLS + COLS + (c * kVec + k) * TPR + lane] = db[c][k];
      }
    __syncthreads();
    for (int p = threadIdx.x; p < 2 * COLS; p += WG) {
      float v = sums[p];
#pragma unroll
      for (int o = 1; o < GROUPS; ++o) v += sums[o * 2 * COLS + p];
      const int q = p % COLS, i = (q / TPR / kVec * TPR + q % TPR) * kVec + q / TPR % kVec;
      if (i < n) (p < COLS ? dw_out : db_out)[i] = v;
    }
  }
}

// 32 threads along the columns (a cache line), 32 of them to a column: thread k adds rows k, k + 32, ...
constexpr int kFinishCols = 32, kFinishRows = 32;
template <class E>
__global__ void __launch_bounds__(kFinishCols * kFinishRows)
    column_finish_kernel(const float* __restrict__ partials, int64_t groups, int64_t cols, int64_t n,
                         typename E::T* __restrict__ out0, typename E::T* __restrict__ out1) {
  __shared__ float part[kFinishRows][kFinishCols + 1];
  const int x = threadIdx.x % kFinishCols, y = threadIdx.x / kFinishCols;
  const int64_t c = (int64_t)blockIdx.x * kFinishCols + x;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int64_t g = y; g < groups; g += kFinishRows) s += partials[g * cols + c];
  }
  part[y][x] = s;
  __syncthreads();
  if (y != 0 || c >= cols) return;
#pragma unroll
  for (int w = 1; w < kFinishRows; ++w) s += part[w][x];
  if (c < n) E::put(out0 + c, s);
  else E::put(out1 + (c - n), s);
}

hipError_t launch_column_finish(const float* partials, int64_t groups, int64_t cols, int64_t n, void* out0, void* out1,
                                int storage, hipStream_t stream) {
  return with_elem(storage, [&](auto e) {
    using E = decltype(e);
    hipLaunchKernelGGL(column_finish_kernel<E>, dim3((unsigned)((cols + kFinishCols - 1) / kFinishCols)),
                       dim3(kFinishCols * kFinishRows), 0, stream,
                       partials, groups, cols, n, static_cast<typename E::T*>(out0), static_cast<typename E::T*>(out1));
    return hipGetLastError();
  });
}

// fn(threads of a row, groups of eight per thread) by the row's length
template <class F>
static hipError_t with_row(int64_t n, F&& fn) {
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
static hipError_t with_row_backward(int64_t n, F&& fn) {
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
static bool exact_rows(int64_t n) { return n % kVec == 0; }
template <class F>
static hipError_t with_exact(int64_t n, F&& fn) {
  return exact_rows(n) ? fn(std::true_type{}) : fn(std::false_type{});
}

hipError_t launch_layer_norm_forward(const NormArgs& a, hipStream_t stream, int num_cu) {
  return with_elem(a.storage, [&](auto e) {
    return with_row(a.n, [&](auto tpr, auto c) {
      return with_exact(a.n, [&](auto exact) {
        constexpr int TPR = decltype(tpr)::value, C = decltype(c)::value, WG = norm_fwd_wg<TPR>();
        constexpr int groups = TPR > 64 ? 1 : WG / TPR;
        // as many workgroups as are on the chip at once
        const int64_t grid = std::min((a.rows + groups - 1) / groups, (int64_t)num_cu * (2048 / WG));
        hipLaunchKernelGGL((layer_norm_forward_kernel<decltype(e), TPR, C, decltype(exact)::value>),
                           dim3((unsigned)grid), dim3(WG), 0, stream, a);
        return hipGetLastError();
      });
    });
  });
}

// Workgroups of the backward, each leaving one row of partial sums: one per CU of the largest device
// at most.  More would fill the chip no better (16 waves each) and cost 8n bytes of traffic apiece, twice.  Rows that
// one workgroup goes through in two turns are left to it, whose sums are the result: that saves the second launch.
constexpr int64_t kNormMaxPartials = 256;
int64_t norm_partials(int64_t rows, int64_t n) {
  int64_t groups = 1;
  (void)with_row_backward(n, [&](auto tpr, auto) {
    groups = kNormBwdWG / decltype(tpr)::value;
    return hipSuccess;
  });
  return rows <= 2 * groups ? 1 : std::min((rows + groups - 1) / groups, kNormMaxPartials);
}

template <class E, int TPR, int C, bool CK, bool EXACT>
static hipError_t backward_launch(const NormGradArgs& a, int64_t grid, float* dw, float* db, hipStream_t stream) {
  constexpr int lds = norm_bwd_lds<TPR, C>();
  const auto kernel = layer_norm_backward_kernel<E, TPR, C, CK, EXACT>;
  static const hipError_t ready = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                      hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (ready != hipSuccess) return ready;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kNormBwdWG), lds, stream, a, dw, db, 2 * a.n);
  return hipGetLastError();
}

hipError_t launch_layer_norm_backward(const NormGradArgs& a, hipStream_t stream) {
  const int64_t grid = norm_partials(a.rows, a.n);
  // a single workgroup's sums are the result
  float* const dw = grid == 1 ? a.dweight : a.partials;
  float* const db = grid == 1 ? a.dbias : a.partials + a.n;
  const hipError_t err = with_elem(a.storage, [&](auto e) {
    return with_row_backward(a.n, [&](auto tpr, auto c) {
      return with_exact(a.n, [&](auto exact) {
        using E = decltype(e);
        constexpr int TPR = decltype(tpr)::value, C = decltype(c)::value;
        constexpr bool EXACT = decltype(exact)::value;
        return a.x == nullptr ? backward_launch<E, TPR, C, true, EXACT>(a, grid, dw, db, stream)
                              : backward_launch<E, TPR, C, false, EXACT>(a, grid, dw, db, stream);
      });
    });
  });
  if (err != hipSuccess || grid == 1) return err;
  return launch_column_finish(a.partials, grid, 2 * a.n, a.n, a.dweight, a.dbias, kStorageF32, stream);
}

}  // namespace rdfft
