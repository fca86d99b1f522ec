// fp8_kernels.hip -- matrices into 8-bit floating point (fp8_device.hpp) and back.
//
// A product in 8 bits needs its operands in blocks along k: activations by rows for y = x W^T, by columns (the rows
// of the transpose) for dW = dz^T x, a weight both ways.  One pass reads the matrix and leaves whichever are
// wanted; in a backward pass it also takes dy through the activation's slope and sums dz over the rows.
//
// A workgroup of 512 threads holds a tile of 128 x 128 values in registers, four rows by eight columns to a thread.  A
// block along the row is 16 lanes (a DPP row).  A block along the column is the 32 threads with the same columns: four in
// a wave, reached by lane swaps, and by LDS from wave to wave; its codes are turned in LDS so that they leave in
// whole cache lines too.  The conversion instructions divide by the power of two themselves.
//
// Bound by HBM where the matrix is large: 8192 x 4096 bf16 16.7 us by rows (6.0 TB/s, part of it from the Infinity Cache),
// 23.4 both ways (with 256 threads of eight rows each, shuffles through LDS and eight-byte stores down the columns 37.4).
// dz = dy gelu'(z) of 8192 x 8192 both ways with its sums: 92 us (346 MB), of which the slope's arithmetic is a fifth.  A
// small matrix takes the time of one tile on one CU, 4 us.  Back: 16.5 us for 8192 x 4096 bf16 (103 MB).
#include <hip/hip_runtime.h>

#include "fp8_device.hpp"
#include "fp8_launch.hpp"
#include "linear_kernels.hpp"

namespace rdfft {

constexpr int kFp8WG = 512, kFp8Waves = kFp8WG / 64, kFp8Rows = kFp8Block * kFp8Lanes / kFp8WG;
constexpr int kFp8Pitch = kFp8Block / 4 + 1;  // words of a column's codes in LDS: the 16 columns of a write on most banks
static_assert(kFp8Rows == 4, "a thread's codes of a column are a word");

// fn over the four lanes that are equal modulo 16, in each of them and in a fixed order
template <class F>
__device__ __forceinline__ uint32_t across_rows(uint32_t v, F&& fn) {
  const auto near = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = fn(near[0], near[1]);
  const auto far = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return fn(far[0], far[1]);
}

// A thread's four rows by eight columns: as floats, or 16-bit values in the pairs they come in, for which the largest, the
// conversion and the turn take two values an instruction.
struct FloatRows {
  static constexpr int kMaxima = kVec;  // words that hold eight columns' maxima
  using Top = uint32_t;
  float v[kFp8Rows][kVec];
  __device__ __forceinline__ static uint32_t bits(uint32_t m) { return m; }  // a maximum as a float's bits
  __device__ __forceinline__ uint32_t row_top(int r) const { return max_bits8(v[r]); }
  __device__ __forceinline__ uint32_t column_tops(int i) const {
    uint32_t m = abs_bits(v[0][i]);
#pragma unroll
    for (int r = 1; r < kFp8Rows; ++r) m = max(m, abs_bits(v[r][i]));
    return across_rows(m, [](uint32_t a, uint32_t b) { return max(a, b); });
  }
  __device__ __forceinline__ Bytes8 row_codes(int r, int s) const { return fp8_encode(v[r], s); }
  __device__ __forceinline__ uint32_t column_codes(int i, float scale) const {
    return fp8_word(v[0][i], v[1][i], v[2][i], v[3][i], scale);
  }
  __device__ __forceinline__ void column_sums(float* s) const {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      s[i] = v[0][i];
#pragma unroll
      for (int r = 1; r < kFp8Rows; ++r) s[i] += v[r][i];
    }
  }
};
template <class E>
struct PairRows {
  typedef unsigned short Pair __attribute__((ext_vector_type(2)));
  static constexpr int kMaxima = kVec / 2;
  using Top = uint16_t;
  uint32_t p[kFp8Rows][kVec / 2];
  __device__ __forceinline__ static uint32_t larger(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(Pair, a), __builtin_bit_cast(Pair, b)));
  }
  __device__ __forceinline__ static uint32_t size(uint32_t w) { return w & 0x7fff7fffu; }
  __device__ __forceinline__ static uint32_t bits(uint32_t m) {
    if constexpr (E::kId == ElemBF16::kId) return m << 16;
    else return __float_as_uint(E::get(reinterpret_cast<const uint16_t*>(&m)));
  }
  __device__ __forceinline__ uint32_t row_top(int r) const {
    const uint32_t m = larger(larger(size(p[r][0]), size(p[r][1])), larger(size(p[r][2]), size(p[r][3])));
    return bits(max(m & 0xffffu, m >> 16));
  }
  __device__ __forceinline__ uint32_t column_tops(int i) const {
    uint32_t m = size(p[0][i]);
#pragma unroll
    for (int r = 1; r < kFp8Rows; ++r) m = larger(m, size(p[r][i]));
    return across_rows(m, [](uint32_t a, uint32_t b) { return larger(a, b); });
  }
  __device__ __forceinline__ Bytes8 row_codes(int r, int s) const {
    const float scale = fp8_scale(s);
    const Bytes8 c = {{fp8_word<E>(p[r][0], p[r][1], scale), fp8_word<E>(p[r][2], p[r][3], scale)}};
    return s == kCkNaN ? Bytes8{{kFp8NaNs, kFp8NaNs}} : c;
  }
  __device__ __forceinline__ uint32_t column_codes(int i, float scale) const {
    const uint32_t half = i % 2 ? 0x07060302u : 0x05040100u;
    return fp8_word<E>(__builtin_amdgcn_perm(p[1][i / 2], p[0][i / 2], half), __builtin_amdgcn_perm(p[3][i / 2], p[2][i / 2], half),
                       scale);
  }
  __device__ __forceinline__ void column_sums(float* s) const {
    float v[kVec];
#pragma unroll
    for (int r = 0; r < kFp8Rows; ++r) {
      E::widen(typename E::Raw{{p[r][0], p[r][1], p[r][2], p[r][3]}}, v);
#pragma unroll
      for (int i = 0; i < kVec; ++i) s[i] = r == 0 ? v[i] : s[i] + v[i];
    }
  }
};

template <class E, bool EXACT, bool SLOPE>
__global__ void __launch_bounds__(kFp8WG) fp8_quantize_kernel(Fp8Quantize q) {
  using T = typename E::T;
  constexpr bool PAIRS = sizeof(T) == 2 && !SLOPE;
  using Rows = std::conditional_t<PAIRS, PairRows<E>, FloatRows>;
  using Top = typename Rows::Top;
  __shared__ uint32_t top[kFp8Waves][kFp8Block * sizeof(Top) / 4];
  __shared__ float sums[kFp8Waves][kFp8Block];
  __shared__ float scale_of[kFp8Block];
  __shared__ uint32_t tile_top[2], turned[kFp8Block * kFp8Pitch];
  const int thread = threadIdx.x, lane = thread & 63, wave = thread / 64;
  const int64_t first_row = (int64_t)blockIdx.y * kFp8Block, row0 = first_row + thread / kFp8Lanes * kFp8Rows;
  const int64_t col0 = (int64_t)blockIdx.x * kFp8Block, col = col0 + thread % kFp8Lanes * kVec;
  const int64_t rows = q.rows, n = q.n;
  const T* const x = static_cast<const T*>(q.x);

  Rows m;
  Bytes8 code[SLOPE ? kFp8Rows : 1];
  int byte[SLOPE ? kFp8Rows : 1];
  if constexpr (EXACT || PAIRS) {
    // (rows and columns past the ends load what is near, without a branch)
    typename E::Raw raw[kFp8Rows];
    const int64_t c = min(col, n - kVec);
    if (EXACT || n >= kVec) {
#pragma unroll
      for (int r = 0; r < kFp8Rows; ++r) raw[r] = E::load(x + min(row0 + r, rows - 1) * q.ldx + c);
    }
    if constexpr (SLOPE) {
      const int64_t blocks = (n + kCkBlock - 1) / kCkBlock;
#pragma unroll
      for (int r = 0; r < kFp8Rows; ++r) {
        const int64_t at = min(row0 + r, rows - 1);
        code[r] = *reinterpret_cast<const Bytes8*>(q.ck.codes + at * n + c);
        byte[r] = q.ck.scales[at * blocks + c / kCkBlock];
      }
    }
#pragma unroll
    for (int r = 0; r < kFp8Rows; ++r) {
      const bool in = row0 + r < rows && col < n;
      if constexpr (PAIRS) {
        u32x4 w = {raw[r].w[0], raw[r].w[1], raw[r].w[2], raw[r].w[3]};
        if constexpr (!EXACT) {
          if (n < kVec) {
            const T* const row = x + min(row0 + r, rows - 1) * q.ldx;
#pragma unroll
            for (int i = 0; i < kVec; i += 2) {
              const uint32_t a = i < n ? row[min((int64_t)i, n - 1)] : 0, b = i + 1 < n ? row[min((int64_t)i + 1, n - 1)] : 0;
              w[i / 2] = a | b << 16;
            }
          } else if (col + kVec > n) {  // the row's end cuts this group: it was loaded so as to end there
            w = drop_bytes(w, (int)min(col + kVec - n, (int64_t)(kVec - 1)) * 2);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) m.p[r][i] = in ? w[i] : 0u;
      } else {
        E::widen(raw[r], m.v[r]);
#pragma unroll
        for (int i = 0; i < kVec; ++i) m.v[r][i] = in ? m.v[r][i] : 0.f;
      }
    }
  } else {
#pragma unroll
    for (int r = 0; r < kFp8Rows; ++r) {
      const bool in = row0 + r < rows && col < n;
      if (in) {
        read_group<E>(x + (row0 + r) * q.ldx, col, n, m.v[r]);
      } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) m.v[r][i] = 0.f;
      }
      if constexpr (SLOPE) {
        code[r] = {{0, 0}};
        byte[r] = 0;
        if (in) {
          code[r] = tail_codes(q.ck.codes + (row0 + r) * n, col, n);
          byte[r] = q.ck.scales[(row0 + r) * ((n + kCkBlock - 1) / kCkBlock) + col / kCkBlock];
        }
      }
    }
  }
  if constexpr (SLOPE) {
#pragma unroll
    for (int r = 0; r < kFp8Rows; ++r) {
      if (row0 + r >= rows || col >= n) continue;
      float z[kVec];
      ck_decode<ElemF32>(code[r], ck_scale(byte[r]), z);
      times_slope8(q.act, z, m.v[r]);
    }
  }
  const bool by_sums = q.sums != nullptr || q.total != nullptr;
  if (by_sums) {
    float s[kVec];
    m.column_sums(s);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      s[i] = __uint_as_float(across_rows(__float_as_uint(s[i]), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
      }));
    }
    if (lane < kFp8Lanes) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) sums[wave][lane * kVec + i] = s[i];
    }
  }
  // the largest of each column
  const bool by_column = q.columns.codes != nullptr || q.tiles;
  if (by_column) {
    uint32_t t[Rows::kMaxima];
#pragma unroll
    for (int i = 0; i < Rows::kMaxima; ++i) t[i] = m.column_tops(i);
    if (lane < kFp8Lanes) {
#pragma unroll
      for (int i = 0; i < Rows::kMaxima; ++i) top[wave][lane * Rows::kMaxima + i] = t[i];
    }
  }
  if (by_column || by_sums) __syncthreads();
  if (thread < kFp8Block) {
    if (by_sums && col0 + thread < n) {
      float s = sums[0][thread];
#pragma unroll
      for (int w = 1; w < kFp8Waves; ++w) s += sums[w][thread];
      if (q.total != nullptr) E::put(static_cast<T*>(q.total) + col0 + thread, s);
      else q.sums[(int64_t)blockIdx.y * n + col0 + thread] = s;
    }
    if (by_column) {
      uint32_t t = reinterpret_cast<const Top*>(top[0])[thread];
#pragma unroll
      for (int w = 1; w < kFp8Waves; ++w) t = max(t, (uint32_t)reinterpret_cast<const Top*>(top[w])[thread]);
      t = Rows::bits(t);
      if (q.tiles) {
        t = row_max(t);
        t = across_rows(t, [](uint32_t a, uint32_t b) { return max(a, b); });
        if (lane == 0) tile_top[wave] = t;
      } else {
        const int s = fp8_scale_byte(t);
        scale_of[thread] = fp8_scale(s);
        if (col0 + thread < n) q.columns.scales[(col0 + thread) * q.columns.lds + blockIdx.y] = (uint8_t)s;
      }
    }
  }
  int tile = 0;
  if (by_column) {
    __syncthreads();
    if (q.tiles) {
      tile = fp8_scale_byte(max(tile_top[0], tile_top[1]));
      if (thread == 0) {
        if (q.held.codes != nullptr) q.held.scales[(int64_t)blockIdx.y * q.held.lds + blockIdx.x] = (uint8_t)tile;
        if (q.columns.codes != nullptr) q.columns.scales[(int64_t)blockIdx.x * q.columns.lds + blockIdx.y] = (uint8_t)tile;
      }
    }
  }
  if (q.columns.codes != nullptr) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int c = thread % kFp8Lanes * kVec + i;
      const float scale = q.tiles ? fp8_scale(tile) : scale_of[c];
      const uint32_t w = m.column_codes(i, scale);
      turned[c * kFp8Pitch + thread / kFp8Lanes] = scale == __builtin_inff() ? kFp8NaNs : w;  // (byte 255)
    }
  }
  if (q.held.codes != nullptr) {
#pragma unroll
    for (int r = 0; r < kFp8Rows; ++r) {
      const int s = q.tiles ? tile : fp8_scale_byte(row_max(m.row_top(r)));
      if (row0 + r >= rows || col >= n) continue;
      write_bytes(q.held.codes + (row0 + r) * q.held.ld, col, n, m.row_codes(r, s));
      if (!q.tiles && thread % kFp8Lanes == 0) q.held.scales[(row0 + r) * q.held.lds + blockIdx.x] = (uint8_t)s;
    }
  }
  if (q.columns.codes == nullptr) return;
  __syncthreads();
  // a quarter of a column to a thread
  const int c = thread / 4, part = thread % 4 * 8;
  const int64_t left = min(rows - first_row - part * 4, (int64_t)32);
  if (col0 + c >= n || left <= 0) return;
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = turned[c * kFp8Pitch + part + i];
  uint8_t* const to = q.columns.codes + (col0 + c) * q.columns.ld + first_row + part * 4;
  if (left == 32) {
    *reinterpret_cast<Bytes16*>(to) = {{w[0], w[1], w[2], w[3]}};
    *reinterpret_cast<Bytes16*>(to + 16) = {{w[4], w[5], w[6], w[7]}};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (i * 4 + e < left) to[i * 4 + e] = (uint8_t)(w[i] >> (8 * e));
  }
}

constexpr int kDequantizeWG = 256;
template <class E>
__global__ void __launch_bounds__(kDequantizeWG) fp8_dequantize_kernel(Fp8Operand from, typename E::T* __restrict__ out, int64_t ldo,
                                                                int64_t row0, int64_t rows, int64_t n, int lanes) {
  const int64_t row = row0 + (int64_t)blockIdx.y * (kDequantizeWG / lanes) + threadIdx.x / lanes;
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
    if (q.act != kActNone)
      return q.n % kVec == 0 ? go(fp8_quantize_kernel<E, true, true>) : go(fp8_quantize_kernel<E, false, true>);
    return q.n % kVec == 0 ? go(fp8_quantize_kernel<E, true, false>) : go(fp8_quantize_kernel<E, false, false>);
  });
}

hipError_t launch_fp8_dequantize(const Fp8Operand& from, void* out, int64_t ldo, int64_t rows, int64_t n, int storage,
                                 hipStream_t stream, int num_cu) {
  return with_elem(storage, [&](auto e) {
    using E = decltype(e);
    const int64_t groups = (n + kVec - 1) / kVec;
    int lanes = 1;
    while (lanes < kDequantizeWG && lanes < groups) lanes *= 2;
    const int per = kDequantizeWG / lanes;
    constexpr int64_t kMaxY = 65535;
    for (int64_t r0 = 0; r0 < rows; r0 += kMaxY * per) {
      const int64_t gy = (std::min(rows - r0, kMaxY * per) + per - 1) / per;
      const int64_t gx = std::min((groups + lanes - 1) / lanes, std::max<int64_t>(1, (int64_t)num_cu * 32 / gy));
      hipLaunchKernelGGL(fp8_dequantize_kernel<E>, dim3((unsigned)gx, (unsigned)gy), dim3(kDequantizeWG), 0, stream, from,
                         static_cast<typename E::T*>(out), ldo, r0, rows, n, lanes);
      const hipError_t err = hipGetLastError();
      if (err != hipSuccess) return err;
    }
    return hipSuccess;
  });
}

}  // namespace rdfft
