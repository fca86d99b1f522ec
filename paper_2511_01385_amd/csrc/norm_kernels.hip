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

template <int TPR>
constexpr int norm_fwd_wg() {
  return TPR > 256 ? TPR : 256;
}

template <class E, int TPR, int C>
__global__ void __launch_bounds__(norm_fwd_wg<TPR>()) layer_norm_forward_kernel(NormArgs a) {
  using T = typename E::T;
  constexpr int WG = norm_fwd_wg<TPR>(), GROUPS = TPR > 64 ? 1 : WG / TPR;
  static_assert(TPR == 64 || TPR == WG, "groups longer than a wave are alone in their workgroup");
  __shared__ float red[2 * (WG / 64)];
  int turn = 0;
  const int lane = threadIdx.x % TPR;
  const int64_t n = a.n;
  const float count = (float)n;
  float w[C][kVec], b[C][kVec];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int64_t i = (int64_t)(c * TPR + lane) * kVec;
    read_group<ElemF32>(a.weight, i, n, w[c]);
    if (a.bias != nullptr) read_group<ElemF32>(a.bias, i, n, b[c]);
    else
#pragma unroll
      for (int k = 0; k < kVec; ++k) b[c][k] = 0.f;
  }
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  for (int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / TPR; row < a.rows; row += step) {
    const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
    float u[C][kVec];
    if (n >= kVec) {
      typename E::Raw raw[C], more[C];
#pragma unroll
      for (int c = 0; c < C; ++c) raw[c] = load_group<E>(x, (int64_t)(c * TPR + lane) * kVec, n);
      if (a.residual != nullptr) {
        const T* const r = static_cast<const T*>(a.residual) + row * a.ldr;
#pragma unroll
        for (int c = 0; c < C; ++c) more[c] = load_group<E>(r, (int64_t)(c * TPR + lane) * kVec, n);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const int64_t i = (int64_t)(c * TPR + lane) * kVec;
          float v[kVec];
          widen_group<E>(raw[c], x, i, n, u[c]);
          widen_group<E>(more[c], r, i, n, v);
#pragma unroll
          for (int k = 0; k < kVec; ++k) u[c][k] += v[k];
        }
      } else {
#pragma unroll
        for (int c = 0; c < C; ++c) widen_group<E>(raw[c], x, (int64_t)(c * TPR + lane) * kVec, n, u[c]);
      }
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int64_t i = (int64_t)(c * TPR + lane) * kVec;
        read_group<E>(x, i, n, u[c]);
        if (a.residual != nullptr) {
          float v[kVec];
          read_group<E>(static_cast<const T*>(a.residual) + row * a.ldr, i, n, v);
#pragma unroll
          for (int k = 0; k < kVec; ++k) u[c][k] += v[k];
        }
      }
    }
    float s[1] = {0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < kVec; ++k) s[0] += u[c][k];
    group_sums<TPR, 1>(s, red, turn);
    const float mean = s[0] / count;
    if (a.ck.codes != nullptr) {
      const int64_t blocks = (n + kCkBlock - 1) / kCkBlock;
#pragma unroll
      for (int c = 0; c < C; ++c)
        write_checkpoint(a.ck.codes + row * n, a.ck.scales + row * blocks, (int64_t)(c * TPR + lane) * kVec, n, u[c]);
    }
    s[0] = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t i = (int64_t)(c * TPR + lane) * kVec;
      if (i + kVec <= n) {
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
          u[c][k] -= mean;
          s[0] = fmaf(u[c][k], u[c][k], s[0]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
          u[c][k] = i + k < n ? u[c][k] - mean : 0.f;
          s[0] = fmaf(u[c][k], u[c][k], s[0]);
        }
      }
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
      write_group<E>(y, (int64_t)(c * TPR + lane) * kVec, n, v);
    }
  }
}

template <int TPR>
constexpr int norm_bwd_wg() {
  return TPR > 256 ? TPR : 1024;
}

// Each workgroup's sums go to dw_out + blockIdx.x * stride and db_out + blockIdx.x * stride.
template <class E, int TPR, int C, bool CK>
__global__ void __launch_bounds__(norm_bwd_wg<TPR>())
    layer_norm_backward_kernel(NormGradArgs a, float* dw_out, float* db_out, int64_t stride) {
  using T = typename E::T;
  constexpr int WG = norm_bwd_wg<TPR>(), GROUPS = WG / TPR;
  __shared__ float red[4 * (WG / 64)];
  int turn = 0;
  const int lane = threadIdx.x % TPR, grp = threadIdx.x / TPR;
  const int64_t n = a.n, blocks = (n + kCkBlock - 1) / kCkBlock;
  const float count = (float)n;
  float w[C][kVec], dw[C][kVec], db[C][kVec];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    read_group<ElemF32>(a.weight, (int64_t)(c * TPR + lane) * kVec, n, w[c]);
#pragma unroll
    for (int k = 0; k < kVec; ++k) dw[c][k] = db[c][k] = 0.f;
  }
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  // (the groups of a workgroup take the same number of rows: they meet at barriers)
  for (int64_t row0 = (int64_t)blockIdx.x * GROUPS; row0 < a.rows; row0 += step) {
    const int64_t row = row0 + grp;
    const bool act = row < a.rows;
    float xh[C][kVec], g[C][kVec];
    float mean = 0.f, rstd = 0.f;
    const T* const dy = static_cast<const T*>(a.dy) + (act ? row : 0) * a.ldg;
    if (act) {
      mean = a.mean[row];
      rstd = a.rstd[row];
      if constexpr (CK) {
        const int8_t* const codes = a.ck.codes + row * n;
        const uint8_t* const scales = a.ck.scales + row * blocks;
        if (n >= kVec) {
          typename E::Raw raw[C];
          Bytes8 held[C];
          int sc[C];
#pragma unroll
          for (int c = 0; c < C; ++c) {
            const int64_t i = (int64_t)(c * TPR + lane) * kVec;
            raw[c] = load_group<E>(dy, i, n);
            held[c] = load_codes(codes, i, n);
            sc[c] = scales[i < n ? i / kCkBlock : 0];
          }
#pragma unroll
          for (int c = 0; c < C; ++c) {
            const int64_t i = (int64_t)(c * TPR + lane) * kVec;
            widen_group<E>(raw[c], dy, i, n, g[c]);
            if (i + kVec > n) held[c] = tail_codes(codes, i, n);
            ck_decode(held[c], ck_scale(sc[c]), xh[c]);
          }
        } else {
#pragma unroll
          for (int c = 0; c < C; ++c) {
            const int64_t i = (int64_t)(c * TPR + lane) * kVec;
            read_group<E>(dy, i, n, g[c]);
            ck_decode(tail_codes(codes, i, n), ck_scale(scales[0]), xh[c]);
          }
        }
      } else {
        const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const int64_t i = (int64_t)(c * TPR + lane) * kVec;
          read_group<E>(dy, i, n, g[c]);
          read_group<E>(x, i, n, xh[c]);
        }
        if (a.residual != nullptr) {
          const T* const r = static_cast<const T*>(a.residual) + row * a.ldr;
#pragma unroll
          for (int c = 0; c < C; ++c) {
            float v[kVec];
            read_group<E>(r, (int64_t)(c * TPR + lane) * kVec, n, v);
#pragma unroll
            for (int k = 0; k < kVec; ++k) xh[c][k] += v[k];
          }
        }
      }
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int k = 0; k < kVec; ++k) g[c][k] = xh[c][k] = 0.f;
    }
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        xh[c][k] = (xh[c][k] - mean) * rstd;
        dw[c][k] = fmaf(g[c][k], xh[c][k], dw[c][k]);
        db[c][k] += g[c][k];
        g[c][k] *= w[c][k];
        s[0] += g[c][k];
        s[1] = fmaf(g[c][k], xh[c][k], s[1]);
      }
    group_sums<TPR, 2>(s, red, turn);
    if (!act) continue;
    const float m0 = s[0] / count, m1 = s[1] / count;
    T* const dx = static_cast<T*>(a.dx) + row * a.ldd;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float v[kVec];
#pragma unroll
      for (int k = 0; k < kVec; ++k) v[k] = rstd * (g[c][k] - m0 - xh[c][k] * m1);
      write_group<E>(dx, (int64_t)(c * TPR + lane) * kVec, n, v);
    }
  }
  dw_out += blockIdx.x * stride;
  db_out += blockIdx.x * stride;
  if constexpr (GROUPS == 1) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t i = (int64_t)(c * TPR + lane) * kVec;
      write_group<ElemF32>(dw_out, i, n, dw[c]);
      write_group<ElemF32>(db_out, i, n, db[c]);
    }
  } else {
    constexpr int COLS = TPR * C * kVec;
    __shared__ float sums[2 * COLS];
    for (int o = 0; o < GROUPS; ++o) {
      if (grp == o) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int k = 0; k < kVec; ++k) {
            // value k of all lanes side by side: no two lanes of a wave meet in a bank
            const int at = (c * kVec + k) * TPR + lane;
            sums[at] = o == 0 ? dw[c][k] : sums[at] + dw[c][k];
            sums[COLS + at] = o == 0 ? db[c][k] : sums[COLS + at] + db[c][k];
          }
      }
      __syncthreads();
    }
    for (int64_t i = threadIdx.x; i < n; i += WG) {
      const int at = (int)((i / (TPR * kVec) * kVec + i % kVec) * TPR + i / kVec % TPR);
      dw_out[i] = sums[at];
      db_out[i] = sums[COLS + at];
    }
  }
}

// Sixteen waves share 64 columns; wave k adds rows k, k + 16, ...
constexpr int kFinishWaves = 16;
template <class E>
__global__ void __launch_bounds__(64 * kFinishWaves)
    column_finish_kernel(const float* __restrict__ partials, int64_t groups, int64_t cols, int64_t n,
                         typename E::T* __restrict__ out0, typename E::T* __restrict__ out1) {
  __shared__ float part[kFinishWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  const int64_t c = (int64_t)blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int64_t g = wave; g < groups; g += kFinishWaves) s += partials[g * cols + c];
  }
  part[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || c >= cols) return;
#pragma unroll
  for (int w = 1; w < kFinishWaves; ++w) s += part[w][lane];
  if (c < n) E::put(out0 + c, s);
  else E::put(out1 + (c - n), s);
}

hipError_t launch_column_finish(const float* partials, int64_t groups, int64_t cols, int64_t n, void* out0, void* out1,
                                int storage, hipStream_t stream) {
  return with_elem(storage, [&](auto e) {
    using E = decltype(e);
    hipLaunchKernelGGL(column_finish_kernel<E>, dim3((unsigned)((cols + 63) / 64)), dim3(64 * kFinishWaves), 0, stream,
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

hipError_t launch_layer_norm_forward(const NormArgs& a, hipStream_t stream, int num_cu) {
  return with_elem(a.storage, [&](auto e) {
    return with_row(a.n, [&](auto tpr, auto c) {
      constexpr int TPR = decltype(tpr)::value, C = decltype(c)::value, WG = norm_fwd_wg<TPR>();
      constexpr int groups = TPR > 64 ? 1 : WG / TPR;
      // as many workgroups as are on the chip at once
      const int64_t grid = std::min((a.rows + groups - 1) / groups, (int64_t)num_cu * (2048 / WG));
      hipLaunchKernelGGL((layer_norm_forward_kernel<decltype(e), TPR, C>), dim3((unsigned)grid), dim3(WG), 0, stream, a);
      return hipGetLastError();
    });
  });
}

// Workgroups of the backward, each leaving one row of partial sums: one per CU of the largest device
// at most.  More would fill the chip no better (16 waves each) and cost 8n bytes of traffic apiece, twice.
constexpr int64_t kNormMaxPartials = 256;
int64_t norm_partials(int64_t rows, int64_t n) {
  int64_t groups = 1;
  (void)with_row(n, [&](auto tpr, auto) {
    constexpr int TPR = decltype(tpr)::value;
    groups = norm_bwd_wg<TPR>() / TPR;
    return hipSuccess;
  });
  return std::max<int64_t>(1, std::min((rows + groups - 1) / groups, kNormMaxPartials));
}

hipError_t launch_layer_norm_backward(const NormGradArgs& a, hipStream_t stream) {
  const int64_t grid = norm_partials(a.rows, a.n);
  // a single workgroup's sums are the result
  float* const dw = grid == 1 ? a.dweight : a.partials;
  float* const db = grid == 1 ? a.dbias : a.partials + a.n;
  const int64_t stride = 2 * a.n;
  const hipError_t err = with_elem(a.storage, [&](auto e) {
    return with_row(a.n, [&](auto tpr, auto c) {
      constexpr int TPR = decltype(tpr)::value, C = decltype(c)::value, WG = norm_bwd_wg<TPR>();
      if (a.x == nullptr)
        hipLaunchKernelGGL((layer_norm_backward_kernel<decltype(e), TPR, C, true>), dim3((unsigned)grid), dim3(WG), 0,
                           stream, a, dw, db, stride);
      else
        hipLaunchKernelGGL((layer_norm_backward_kernel<decltype(e), TPR, C, false>), dim3((unsigned)grid), dim3(WG), 0,
                           stream, a, dw, db, stride);
      return hipGetLastError();
    });
  });
  if (err != hipSuccess || grid == 1) return err;
  return launch_column_finish(a.partials, grid, 2 * a.n, a.n, a.dweight, a.dbias, kStorageF32, stream);
}

}  // namespace rdfft
