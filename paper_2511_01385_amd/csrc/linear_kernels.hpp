// linear_kernels.hpp -- the dense product with its epilogue on the matrix cores, as templates over
// the storage type (linear_{f32,bf16,f16}.hip instantiate them).
//
//   D(m, n) = sum over k of A(m, k) B(n, k)
//
// Three products have this form: y = x W^T (A = x, B = W), dx = dz W (A = dz, B = W with its
// rows along k) and dW = dz^T x (both with their rows along k).  An operand is "along k" when
// its rows in memory are runs of k (element (m, k) at a[m * lda + k]) and "across k" when they
// are runs of m (a[k * lda + m]).
//
// A workgroup computes a BM x BN tile of D; a stage of 128 bytes of k (64 16-bit values, 32
// floats) of both operands lies in LDS, two or three stages in turn.  The stages after the one being
// multiplied are under way in the meantime: by loads that go straight to LDS (16 bytes a lane), or
// through registers where a row of a 16-bit operand does not start at a multiple of 16 bytes.
//
// LDS layouts (units of 16 bytes, `pos` of a row holding chunk `pos ^ swizzle`):
//   along k:   [BM rows][8 chunks], swizzle row & 7: the 16 rows of a fragment, read at one chunk,
//              fall on all banks evenly;
//   across k:  [k rows][BM * S / 16 chunks].  16-bit fragments are read transposed, four k rows of 16
//              values (32 bytes) at a time, k and k + 8 together: swizzle (k & 3) * 2 + (k / 8 & 1) * 8
//              spreads them over all banks ((k & 3 ^ k / 8 & 1) * 2 in rows of 128 bytes; without the
//              k / 8 a third to a half of the LDS cycles of dx and dW were conflicts).  Floats are read
//              one by one in runs of 16 at four k rows: (k / 4 & 3) * 4.
//
// The matrix instructions take n as their row and m as their column, so that a lane's four
// results are consecutive in n, the direction in which D, the bias, the residual and the 8-bit
// blocks run.  k is spread over a fragment's four lane groups in runs of one chunk, for both
// operands alike.  Sums are float32 throughout.
//
// What bounds it: dx and dW of 8192 tokens, 4096 -> 8192 (bf16, normal values) take 397 and 405 us, 1390 and
// 1360 TFLOP/s (the library's bare products 413 and 515); the matrix cores are busy 74 % of the CUs' cycles, at a
// clock that such work takes down to about 1.9 GHz.  The forward takes 418 us without anything in its epilogue (library
// 370), 451 with gelu, 444 with the checkpoint, 469 with both and 494 with a residual besides: the epilogues of a round
// of tiles coincide.  (Averages of 60 launches of each in random order; what ran before moves the clock, and one of
// these by up to 10 %.)
#pragma once

#include <hip/hip_runtime.h>

#include "dense_device.hpp"
#include "dense_launch.hpp"

namespace rdfft {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// One chunk of k (16 bytes a lane and lane group): 16 x 16 results
template <class E>
__device__ __forceinline__ f32x4 mfma_chunk(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (E::kId == kStorageBF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                   0);
  } else if constexpr (E::kId == kStorageF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
    return c;
  }
}

// ----------------------------------------------------------------------------------
// activations.  erf by Abramowitz and Stegun's 7.1.26 (absolute error 1.5e-7), whose exp(-x^2) is
// also the density in gelu's slope.  For float32 storage too: gelu is 9e-8 of its norm off, where a
// correctly rounded erf leaves 4e-8; relatively it loses most where it is next to nothing (5e-4 at -4).

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rcp_fast(float x) { return __builtin_amdgcn_rcpf(x); }
constexpr float kLog2e = 1.44269504088896341f;

// normal distribution function of z, and e = exp(-z^2 / 2)
__device__ __forceinline__ float normal_cdf(float z, float* e) {
  const float x = fabsf(z) * 0.70710678118654752f;
  const float t = rcp_fast(fmaf(0.3275911f, x, 1.f));
  const float g = exp2_fast(-kLog2e * x * x);
  float p = fmaf(1.061405429f, t, -1.453152027f);
  p = fmaf(p, t, 1.421413741f);
  p = fmaf(p, t, -0.284496736f);
  p = fmaf(p, t, 0.254829592f);
  *e = g;
  const float tail = 0.5f * p * t * g;  // 1 - cdf(|z|)
  return z < 0.f ? tail : 1.f - tail;
}

__device__ __forceinline__ float activate(int act, float z) {
  if (act == kActRelu) return z < 0.f ? 0.f : z;  // (a NaN stays)
  if (act == kActGelu) {
    float e;
    const float c = normal_cdf(z, &e);
    return c == 0.f ? c * 0.f : z * c;  // -infinity to zero, not NaN
  }
  if (act == kActSilu) {
    const float d = 1.f + exp2_fast(-kLog2e * z);
    return z * rcp_fast(d);
  }
  return z;
}

__device__ __forceinline__ float activation_slope(int act, float z) {
  if (act == kActRelu) return z != z ? z : z > 0.f ? 1.f : 0.f;
  if (act == kActGelu) {
    float e;
    const float c = normal_cdf(z, &e);
    return fmaf(z * 0.39894228040143268f, e, c);
  }
  if (act == kActSilu) {
    const float s = rcp_fast(1.f + exp2_fast(-kLog2e * z));
    return s * fmaf(z, 1.f - s, 1.f);
  }
  return 1.f;
}

// eight values; act is the same for the whole launch
__device__ __forceinline__ void activate8(int act, float* z) {
  const auto each = [&](auto which) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) z[i] = activate(decltype(which)::value, z[i]);
  };
  using std::integral_constant;
  if (act == kActRelu) each(integral_constant<int, kActRelu>{});
  else if (act == kActGelu) each(integral_constant<int, kActGelu>{});
  else if (act == kActSilu) each(integral_constant<int, kActSilu>{});
}
// g *= act'(z)
__device__ __forceinline__ void times_slope8(int act, const float* z, float* g) {
  const auto each = [&](auto which) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) g[i] *= activation_slope(decltype(which)::value, z[i]);
  };
  using std::integral_constant;
  if (act == kActRelu) each(integral_constant<int, kActRelu>{});
  else if (act == kActGelu) each(integral_constant<int, kActGelu>{});
  else if (act == kActSilu) each(integral_constant<int, kActSilu>{});
}

// ----------------------------------------------------------------------------------
// operands

constexpr int kStageBytes = 128;  // of k, per row and stage

// Loads that go straight to LDS: 64 lanes of 16 bytes (or four) from `base` + their offset to consecutive
// LDS bytes from `lds`.  A lane whose offset is not under `records`, such as kNowhere, stores zeros.  They are written as assembly
// because the compiler, which cannot tell the stages apart, would wait for them before each LDS
// read; stage_wait() and loads_wait() are the waits.  (No register receives anything.)
constexpr uint32_t kNowhere = 0x80000000u;
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int BYTES = 16>
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t offset, uint32_t lds, int records = (int)(kNowhere - 1)) {
  // (base and lds are the same in all lanes, which the compiler does not always see)
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  const uint64_t u = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(p >> 32)) << 32 |
                     (uint32_t)__builtin_amdgcn_readfirstlane((int)p);
  lds = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds);
  const __amdgpu_buffer_rsrc_t r =
      __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<char*>(u), 0, records, 0x00020000);
  if constexpr (BYTES == 16)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(r)
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(r)
                 : "memory", "m0");
}
#pragma clang diagnostic pop
// all but the last LEFT of this wave's loads to LDS done, its LDS reads done, every wave here
template <int LEFT>
__device__ __forceinline__ void stage_wait() {
  static_assert(LEFT < 64);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((LEFT & 15) | 7 << 4 | (LEFT >> 4) << 14);  // vmcnt(LEFT) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// the same within a wave: all but the last LEFT loads to LDS done; its LDS reads done
template <int LEFT>
__device__ __forceinline__ void loads_wait() {
  static_assert(LEFT < 64);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((LEFT & 15) | 7 << 4 | 15 << 8 | (LEFT >> 4) << 14);  // vmcnt(LEFT)
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void reads_wait() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(15 | 7 << 4 | 3 << 14);  // lgkmcnt(0)
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ void wave_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// 16 bytes without the first `bytes` (0 ... 15), the rest moved up
__device__ __forceinline__ u32x4 drop_bytes(u32x4 v, int bytes) {
  uint64_t lo = (uint64_t)v[1] << 32 | v[0], hi = (uint64_t)v[3] << 32 | v[2];
  if (bytes >= 8) {
    lo = hi;
    hi = 0;
  }
  const int bits = (bytes & 7) * 8;
  lo = lo >> bits | hi << 1 << (63 - bits);
  hi >>= bits;
  return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// what a chunk's place in memory row k of a stage across k is xored with
template <int S, int CPR>
__device__ __forceinline__ int across_swizzle(int k) {
  if (S == 4) return (k >> 2 & 3) << 2;
  return CPR >= 16 ? (k & 3) << 1 | (k >> 3 & 1) << 3 : ((k & 3) ^ (k >> 3 & 1)) << 1;
}

// R rows (m or n) of one operand's stage.  ACROSS: memory rows run along m.  kDirect: straight to LDS, for which
// memory rows hold whole chunks and, of 16-bit values, start at multiples of 16 bytes (these loads take any address that
// is a multiple of four).  kDirectCut, floats only: the same where chunks may be cut, by the end of k or by the
// operand's last row across k; such a stage is loaded value by value.  kByRegisters, 16-bit values only: the rest.
enum LoadPath { kByRegisters, kDirect, kDirectCut };
template <class E, int R, int WAVES, bool ACROSS, LoadPath PATH>
struct Operand {
  using T = typename E::T;
  static constexpr bool DMA = PATH != kByRegisters;
  static constexpr int S = sizeof(T), EPC = 16 / S, BK = kStageBytes / S;
  static constexpr int CPR = ACROSS ? R * S / 16 : 8;  // chunks of an LDS row
  static constexpr int BYTES = R * kStageBytes;
  static constexpr int LINES = BYTES / 1024 / WAVES;   // 64 chunks each, a wave's share
  static_assert(LINES * WAVES * 1024 == BYTES && 64 % CPR == 0);
  static_assert(PATH == kDirect || (PATH == kByRegisters) == (S == 2), "floats go straight to LDS in any case");
  static_assert(!ACROSS || CPR >= (S == 2 ? 8 : 16), "the swizzle stays in the row");

  const T* base;    // row 0 and k 0 of this workgroup's tile
  int64_t ld;
  int rows, depth;  // rows of the tile that exist, k that is left
  int before;       // values of a memory row in front of the tile, or of the k that is left
  int wave, lane;
  uint32_t offset[DMA ? LINES : 1];
  u32x4 held[2][DMA ? 1 : LINES];  // two stages on their way through registers,
  int held_along[2], held_lines[2];  // and what of them exists where that is not all of it

  // LDS row and chunk of this lane's part of line j
  __device__ __forceinline__ int row_of(int j) const { return (wave * LINES + j) * (64 / CPR) + lane / CPR; }
  // whether every stage has chunks that the operand's last row (across k) cuts
  __device__ __forceinline__ bool cut() const { return PATH == kDirectCut && ACROSS && rows < R && rows % EPC != 0; }
  __device__ __forceinline__ int chunk_of(int j) const {
    return (lane % CPR) ^ (ACROSS ? across_swizzle<S, CPR>(row_of(j)) : row_of(j) & 7);
  }

  __device__ __forceinline__ void init(const T* origin, int64_t ld_, int64_t r0, int64_t r_end, int64_t k0, int64_t k_end,
                                       int wave_, int lane_) {
    ld = ld_;
    base = origin + (ACROSS ? k0 * ld + r0 : r0 * ld + k0);
    rows = (int)(r_end - r0 < R ? r_end - r0 : R);
    depth = (int)(k_end - k0);
    before = ACROSS ? (int)(r0 < kVec ? r0 : kVec) : (int)(k0 < kVec ? k0 : kVec);
    wave = wave_;
    lane = lane_;
    if constexpr (DMA) {
#pragma unroll
      for (int j = 0; j < LINES; ++j) {
        const int r = row_of(j), c = chunk_of(j);
        const bool in = ACROSS ? c * EPC < rows : r < rows;
        offset[j] = in ? (uint32_t)r * (uint32_t)(ld * S) + (uint32_t)c * 16u : kNowhere;
      }
    }
  }

  // line j of a stage in front of the end of k, straight to LDS; step() after the last
  __device__ __forceinline__ void fetch_line(int j, uint32_t lds) const {
    load_to_lds(reinterpret_cast<const char*>(base), offset[j], lds + (uint32_t)(wave * LINES + j) * 1024u);
  }
  __device__ __forceinline__ void step() {
    base += ACROSS ? BK * ld : BK;
    depth -= BK;
  }
  // starts the loads of the next stage (to the LDS region `lds` for DMA, else to held[SLOT]) and steps on.
  template <int SLOT = 0>
  __device__ __forceinline__ void fetch(uint32_t lds) {
    if constexpr (DMA) {
      const char* const p = reinterpret_cast<const char*>(base);
      if (PATH == kDirectCut && (cut() || (!ACROSS && depth < BK && depth % EPC != 0))) {
#pragma unroll
        for (int q = 0; q < LINES * 4; ++q) {  // 64 values each
          const int place = q * 16 + lane / 4, line = wave * LINES * (64 / CPR) + place / CPR;
          const int c = place % CPR ^ (ACROSS ? across_swizzle<S, CPR>(line) : line & 7);
          const int i = c * EPC + lane % 4, r = ACROSS ? i : line, k = ACROSS ? line : i;
          const uint32_t at = (uint32_t)line * (uint32_t)(ld * S) + (uint32_t)i * 4u;
          load_to_lds<4>(p, r < rows && k < depth ? at : kNowhere, lds + (uint32_t)(wave * LINES) * 1024u + (uint32_t)q * 256u);
        }
      } else if (depth >= BK) {
#pragma unroll
        for (int j = 0; j < LINES; ++j) load_to_lds(p, offset[j], lds + (uint32_t)(wave * LINES + j) * 1024u);
      } else {
#pragma unroll
        for (int j = 0; j < LINES; ++j) {
          const int k = ACROSS ? row_of(j) : chunk_of(j) * EPC;
          load_to_lds(p, k < depth ? offset[j] : kNowhere, lds + (uint32_t)(wave * LINES + j) * 1024u);
        }
      }
    } else {
      // Whole chunks without branches: a chunk that the end of its memory row cuts is loaded so as to end there, then
      // shifted into place.  k beyond its end is zero; a row of the tile beyond the last is of no account (its
      // results are not stored) and repeats what is near.
      const int along = ACROSS ? rows : min(depth, BK), lines = ACROSS ? min(depth, BK) : rows;
      const auto chunk = [](const T* p) {
        const Bytes16 v = *reinterpret_cast<const Bytes16*>(p);
        return u32x4{v.w[0], v.w[1], v.w[2], v.w[3]};
      };
      bool mend = false;
      if (along == (ACROSS ? R : BK) && lines == (ACROSS ? BK : R)) {
#pragma unroll
        for (int j = 0; j < LINES; ++j) held[SLOT][j] = chunk(base + row_of(j) * ld + chunk_of(j) * EPC);
      } else if (along + before >= EPC) {
        const int last = along - EPC;
#pragma unroll
        for (int j = 0; j < LINES; ++j)
          held[SLOT][j] = chunk(base + min(row_of(j), lines - 1) * ld + min(chunk_of(j) * EPC, last));
        mend = true;
      } else {
#pragma unroll
        for (int j = 0; j < LINES; ++j) {
          const int r = row_of(j), i = chunk_of(j) * EPC;
          const int r_end = ACROSS ? min(depth, BK) : rows, i_end = ACROSS ? rows : min(depth, BK);
          const T* const p = base + r * ld + i;
          u32x4 h = {0, 0, 0, 0};
          if (r < r_end) {
            if (i + EPC <= i_end) {
              const Bytes16 v = *reinterpret_cast<const Bytes16*>(p);
              h = u32x4{v.w[0], v.w[1], v.w[2], v.w[3]};
            } else {
#pragma unroll
              for (int e = 0; e < EPC; ++e)
                if (i + e < i_end) h[e / 2] |= (uint32_t)p[e] << (16 * (e % 2));
            }
          }
          held[SLOT][j] = h;
        }
      }
      held_along[SLOT] = mend ? along : kVec << 20;
      held_lines[SLOT] = lines;
    }
    step();
    if constexpr (!ACROSS && !DMA) before = kVec;
  }
  // puts held[SLOT] into LDS
  template <int SLOT>
  __device__ __forceinline__ void commit(char* lds) {
    if constexpr (!DMA) {
      const int along = held_along[SLOT], last = along - EPC;
      if (along <= (ACROSS ? R : BK)) {
#pragma unroll
        for (int j = 0; j < LINES; ++j) {
          const int i = chunk_of(j) * EPC;
          const u32x4 h = drop_bytes(held[SLOT][j], i > last && i < along ? (i - last) * S : 0);
          const bool out = ACROSS ? row_of(j) >= held_lines[SLOT] : i >= along;
#pragma unroll
          for (int e = 0; e < 4; ++e) held[SLOT][j][e] = out ? 0 : h[e];
        }
      }
#pragma unroll
      for (int j = 0; j < LINES; ++j)
        *reinterpret_cast<u32x4*>(lds + (wave * LINES + j) * 1024 + lane * 16) = held[SLOT][j];
    }
  }
};

// Fragments of one operand: 16 rows at row0 + 16 f, k chunk group kk (of two).
template <class E, int R, bool ACROSS>
struct Fragments {
  static constexpr int S = sizeof(typename E::T), ROWB = R * S;
  uint32_t at[ACROSS ? 4 : 2];
  __device__ __forceinline__ void init(int row0, int lane) {
    const int g = lane >> 4, j = lane & 15;
    if constexpr (!ACROSS) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
        at[kk] = (uint32_t)((row0 + j) * kStageBytes + ((kk * 4 + g) ^ (j & 7)) * 16);
    } else if constexpr (S == 2) {
      // (all k that a lane reads have its group's bit 3 and its own bits 0 and 1)
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const int chunk = (row0 / 8 + f * 2 + ((j & 3) >> 1)) ^ across_swizzle<S, ROWB / 16>(g * 8 + (j >> 2));
        at[f] = (uint32_t)((g * 8 + (j >> 2)) * ROWB + chunk * 16 + (j & 1) * 8);
      }
    } else {
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const int chunk = (row0 / 4 + f * 4 + (j >> 2)) ^ (g << 2);
        at[f] = (uint32_t)(g * 4 * ROWB + chunk * 16 + (j & 3) * 4);
      }
    }
  }
  __device__ __forceinline__ u32x4 read(const char* lds, int f, int kk) const {
    if constexpr (!ACROSS) {
      return *reinterpret_cast<const u32x4*>(lds + at[kk] + f * 16 * kStageBytes);
    } else if constexpr (S == 2) {
      // the second four groups of 16 rows are 128 bytes on, a bit of its own in the place (row0 is a multiple of 128 there)
      const char* const p = lds + (at[f & 3] ^ ((f >> 2) * 128)) + kk * 32 * ROWB;
      typedef __attribute__((address_space(3))) s16x4 Lds;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)p));
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(p + 4 * ROWB)));
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
      const char* const p = lds + at[f & 3] + (f >> 2) * 256 + kk * 16 * ROWB;
      u32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint32_t*>(p + i * ROWB);
      return v;
    }
  }
};

// ----------------------------------------------------------------------------------
// epilogue of eight consecutive results z of row m, from column n (a multiple of eight); four
// consecutive lanes hold an 8-bit block, all of them here.  bias: of these columns.
template <class E>
__device__ __forceinline__ void finish_group(const GemmArgs& g, int64_t m, int64_t n, const float* bias, float* z) {
  using T = typename E::T;
  const bool in = m < g.m && n < g.n;
  if (g.partial != nullptr) {
    if (in) write_group<ElemF32>(g.partial + m * g.n, n, g.n, z);
    return;
  }
  const int left = in ? (int)min(g.n - n, (int64_t)kVec) : 0;
#pragma unroll
  for (int i = 0; i < kVec; ++i) z[i] = i < left ? z[i] + bias[i] : 0.f;
  if (g.ck.codes != nullptr) {
    const int s = ck_scale_byte(quad_max(max_bits8(z)));
    if (in) {
      write_codes(g.ck.codes + m * g.n, n, g.n, ck_encode(z, s));
      if (n % kCkBlock == 0) g.ck.scales[m * ((g.n + kCkBlock - 1) / kCkBlock) + n / kCkBlock] = (uint8_t)s;
    }
  }
  if (!in) return;
  activate8(g.act, z);
  if (g.residual != nullptr) {
    float add[kVec];
    read_group<E>(static_cast<const T*>(g.residual) + m * g.ldr, n, g.n, add);
#pragma unroll
    for (int i = 0; i < kVec; ++i) z[i] += add[i];
  }
  write_group<E>(static_cast<T*>(g.d) + m * g.ldd, n, g.n, z);
}
// The same for COUNT rows m, m + step, ... that lie in D with all their columns; take(b, z) gives row b's
// results.  The residual's loads are all under way before the first row is worked on.
template <class E, int COUNT, class Take>
__device__ __forceinline__ void finish_rows(const GemmArgs& g, int64_t m, int step, int64_t n, const float* bias, Take&& take) {
  using T = typename E::T;
  float z[kVec];
  if (g.partial != nullptr) {
    float* const p = g.partial + m * g.n + n;
#pragma unroll
    for (int b = 0; b < COUNT; ++b) {
      take(b, z);
      ElemF32::store(p + (int64_t)(b * step) * g.n, z);
    }
    return;
  }
  typename E::Raw add[COUNT];
  if (g.residual != nullptr) {
    const T* const p = static_cast<const T*>(g.residual) + m * g.ldr + n;
#pragma unroll
    for (int b = 0; b < COUNT; ++b) add[b] = E::load(p + (int64_t)(b * step) * g.ldr);
  }
  T* const d = static_cast<T*>(g.d) + m * g.ldd + n;
  const int64_t blocks = (g.n + kCkBlock - 1) / kCkBlock;
#pragma unroll
  for (int b = 0; b < COUNT; ++b) {
    take(b, z);
#pragma unroll
    for (int i = 0; i < kVec; ++i) z[i] += bias[i];
    if (g.ck.codes != nullptr) {
      const int s = ck_scale_byte(quad_max(max_bits8(z)));
      const int64_t row = m + b * step;
      *reinterpret_cast<Bytes8*>(g.ck.codes + row * g.n + n) = ck_encode(z, s);
      if (n % kCkBlock == 0) g.ck.scales[row * blocks + n / kCkBlock] = (uint8_t)s;
    }
    activate8(g.act, z);
    if (g.residual != nullptr) {
      float v[kVec];
      E::widen(add[b], v);
#pragma unroll
      for (int i = 0; i < kVec; ++i) z[i] += v[i];
    }
    E::store(d + (int64_t)(b * step) * g.ldd, z);
  }
}

template <class E>
__device__ __forceinline__ void read_bias(const GemmArgs& g, int64_t n, float* bias) {
  if (g.bias != nullptr && n < g.n) {
    read_group<E>(static_cast<const typename E::T*>(g.bias), n, g.n, bias);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) bias[i] = 0.f;
  }
}

// D's tile (or split) of this workgroup.  Workgroups are dealt to the eight XCDs in turn; each XCD
// takes a run of tiles, ordered so that eight rows of tiles share the columns that its L2 holds.
struct TileAt {
  int tm, tn, split;
};
__device__ __forceinline__ TileAt tile_of(int id, int tiles_m, int tiles_n, int splits) {
  const int total = tiles_m * tiles_n * splits;
  constexpr int XCDS = 8, GROUP = 8;
  const int each = total / XCDS, more = total % XCDS;
  const int x = id % XCDS;
  int t = x * each + min(x, more) + id / XCDS;
  const int split = t / (tiles_m * tiles_n);
  t -= split * tiles_m * tiles_n;
  const int band = t / (GROUP * tiles_n), first = band * GROUP;
  const int high = min(GROUP, tiles_m - first);
  t -= band * GROUP * tiles_n;
  return {first + t % high, t / high, split};
}

template <class E, int BM, int BN, int WM, int WN, int STAGES, bool AX, bool BX, LoadPath PATH>
__device__ __forceinline__ void linear_tile(GemmArgs g, int id) {
  using T = typename E::T;
  constexpr int WAVES = WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
  constexpr int BK = kStageBytes / (int)sizeof(T);
  static_assert(FN % 2 == 0, "a wave holds whole blocks of 32 values");
  constexpr bool DMA = PATH != kByRegisters;
  using OpA = Operand<E, BM, WAVES, AX, PATH>;
  using OpB = Operand<E, BN, WAVES, BX, PATH>;
  constexpr int STAGE = OpA::BYTES + OpB::BYTES;
  extern __shared__ __attribute__((aligned(1024))) char linear_lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
  const int wm = wave / WN, wn = wave % WN;
  const TileAt at = tile_of(id, g.tiles_m, g.tiles_n, g.splits);
  const int64_t m0 = (int64_t)at.tm * BM, n0 = (int64_t)at.tn * BN;
  const int64_t k0 = (int64_t)at.split * g.k_split, k1 = min(k0 + g.k_split, g.k);

  OpA a;
  OpB b;
  a.init(static_cast<const T*>(g.a), g.lda, m0, g.m, k0, k1, wave, lane);
  b.init(static_cast<const T*>(g.b), g.ldb, n0, g.n, k0, k1, wave, lane);
  Fragments<E, BM, AX> fa;
  Fragments<E, BN, BX> fb;
  fa.init(wm * TM, lane);
  fb.init(wn * TN, lane);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)linear_lds;

  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Half a stage's fragments (chunk group kk), and their products.  A half is read while the one before it
  // is multiplied: reads and products are dealt out in turn.
  struct Half {
    u32x4 a[FM], b[FN];
  };
  const auto read = [&](Half& h, const char* la, int kk) {
#pragma unroll
    for (int j = 0; j < FN; ++j) h.b[j] = fb.read(la + OpA::BYTES, j, kk);
#pragma unroll
    for (int i = 0; i < FM; ++i) h.a[i] = fa.read(la, i, kk);
  };
  const auto multiply = [&](const Half& h) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = mfma_chunk<E>(h.b[j], h.a[i], acc[i][j]);
  };
  // instructions of a half, for the scheduler
  constexpr int PRODUCTS = FM * FN * (E::kId == kStorageF32 ? 4 : 1);
  constexpr int READS = FM * (!AX ? 1 : sizeof(T) == 2 ? 2 : 4) + FN * (!BX ? 1 : sizeof(T) == 2 ? 2 : 4);
  const auto interleave = [&] {
    constexpr int GROUPS = READS < PRODUCTS ? READS : PRODUCTS;
#pragma unroll
    for (int q = 0; q < GROUPS; ++q) {
      __builtin_amdgcn_sched_group_barrier(0x008, PRODUCTS / GROUPS, 0);  // matrix instructions
      __builtin_amdgcn_sched_group_barrier(0x100, READS / GROUPS, 0);    // LDS reads
    }
  };
  const int steps = (int)((k1 - k0 + BK - 1) / BK);
  if constexpr (DMA) {
    // STAGES - 1 stages are under way ahead of the one being multiplied.  The barrier sits
    // between a stage's two halves: every wave has read all of the stage by then, so that its
    // region can be loaded anew, and the next stage's first half is read under the second's products.
    constexpr int EACH = OpA::LINES + OpB::LINES;  // (a stage that is loaded value by value has more: its waits are longer)
    const auto fetch = [&](int slot) {
      a.fetch(lds0 + (uint32_t)slot * STAGE);
      b.fetch(lds0 + (uint32_t)slot * STAGE + OpA::BYTES);
    };
    // One half's products with the other's reads and a stage's loads between them, a row of fragments at a time:
    // loads that set out together wait for each other and hold up the products behind them.
    const auto weave = [&](const Half& h, Half& to, const char* from, int slot) {
      constexpr int TOTAL = FM + FN;
      const uint32_t la = lds0 + (uint32_t)slot * STAGE, lb = la + OpA::BYTES;
#pragma unroll
      for (int i = 0; i < FM; ++i) {
#pragma unroll
        for (int e = i * EACH / FM; e < (i + 1) * EACH / FM; ++e) {
          if (e < OpA::LINES) a.fetch_line(e, la);
          else b.fetch_line(e - OpA::LINES, lb);
        }
#pragma unroll
        for (int e = i * TOTAL / FM; e < (i + 1) * TOTAL / FM; ++e) {
          if (e < FN) to.b[e] = fb.read(from + OpA::BYTES, e, 0);
          else to.a[e - FN] = fa.read(from, e - FN, 0);
        }
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = mfma_chunk<E>(h.b[j], h.a[i], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
      }
      a.step();
      b.step();
    };
    Half h0, h1;
#pragma unroll
    for (int q = 0; q < STAGES; ++q)
      if (q < steps) fetch(q);
    if (steps > 0) {
      if (steps >= STAGES) stage_wait<(STAGES - 1) * EACH>();
      else stage_wait<0>();
      read(h0, linear_lds, 0);
    }
    int cur = 0, t = 0;
    const auto next = [](int slot) { return slot + 1 == STAGES ? 0 : slot + 1; };
    const int steady = a.cut() || b.cut() ? 0 : steps - 1 - STAGES;
    for (; t < steady; ++t) {  // (the stage that is fetched is not the last)
      read(h1, linear_lds + cur * STAGE, 1);
      multiply(h0);
      interleave();
      stage_wait<(STAGES - 2) * EACH>();
      if constexpr (E::kId != kStorageF32) {
        weave(h1, h0, linear_lds + next(cur) * STAGE, cur);
        cur = next(cur);
      } else {
        // (four products a pair of fragments: the loads are out of their way)
        const uint32_t la = lds0 + (uint32_t)cur * STAGE;
#pragma unroll
        for (int e = 0; e < OpA::LINES; ++e) a.fetch_line(e, la);
#pragma unroll
        for (int e = 0; e < OpB::LINES; ++e) b.fetch_line(e, la + OpA::BYTES);
        a.step();
        b.step();
        cur = next(cur);
        read(h0, linear_lds + cur * STAGE, 0);
        multiply(h1);
        interleave();
      }
    }
    for (; t < steps; ++t) {
      read(h1, linear_lds + cur * STAGE, 1);
      multiply(h0);
      if (t + 1 < steps) {
        // this stage is read; the next has landed when those after it are all that is left
        if (STAGES > 2 && t + STAGES - 1 < steps) stage_wait<(STAGES - 2) * EACH>();
        else stage_wait<0>();
        if (t + STAGES < steps) fetch(cur);
        cur = next(cur);
        read(h0, linear_lds + cur * STAGE, 0);
      }
      multiply(h1);
    }
  } else {
    // The same with two stages on their way through registers: stage t + 1 goes to LDS between the halves of stage t,
    // into the region that every wave has left at the last barrier, and stage t + 3 sets out.
    static_assert(DMA || STAGES == 2);
    const auto fetch = [&](auto slot) {
      a.template fetch<decltype(slot)::value>(0);
      b.template fetch<decltype(slot)::value>(0);
    };
    const auto commit = [&](auto slot) {
      constexpr int S = decltype(slot)::value;
      a.template commit<S>(linear_lds + S * STAGE);
      b.template commit<S>(linear_lds + S * STAGE + OpA::BYTES);
    };
    using std::integral_constant;
    Half h0, h1;
    const auto step = [&](int t, auto cur) {
      constexpr int C = decltype(cur)::value;
      constexpr integral_constant<int, C ^ 1> other{};
      read(h1, linear_lds + C * STAGE, 1);
      multiply(h0);
      if (t + 1 < steps) {
        commit(other);
        if (t + 3 < steps) fetch(other);
        reads_wait();
        wave_barrier();
        read(h0, linear_lds + (C ^ 1) * STAGE, 0);
      }
      multiply(h1);
    };
    constexpr integral_constant<int, 0> even{};
    constexpr integral_constant<int, 1> odd{};
    if (steps > 0) {
      fetch(even);
      if (steps > 1) fetch(odd);
      commit(even);
      if (steps > 2) fetch(even);
      reads_wait();
      wave_barrier();
      read(h0, linear_lds, 0);
    }
    for (int t = 0; t < steps; t += 2) {
      step(t, even);
      if (t + 1 < steps) step(t + 1, odd);
    }
  }
  stage_wait<0>();

  // Each wave turns its results through LDS of its own (no wave reads stages any more), PART blocks of 16 rows at a
  // time, into runs of eight along n: the lanes of a row then read and write whole cache lines.  16 bytes c of a row lie
  // at (c / 2, odd ones in the second half) xor row: neither side meets in a bank.
  constexpr int PART = FM >= 4 && WAVES * 4 * 16 * TN * 4 <= STAGES * STAGE ? 4 : FM >= 2 ? 2 : 1;
  constexpr int CH = TN / 4, RUNS = TN / kVec, ROWS = 64 / RUNS, PASSES = 16 * PART / ROWS;
  static_assert(WAVES * PART * 16 * TN * 4 <= STAGES * STAGE && FM % PART == 0);
  char* const turn = linear_lds + wave * (PART * 16 * TN * 4);
  const auto slot = [](int row, int c) { return (row * CH + (((c >> 1) | (c & 1) * (CH / 2)) ^ (row & (CH - 1)))) * 16; };
  const int64_t n = n0 + wn * TN + lane % RUNS * kVec;
  float bias[kVec];
  read_bias<E>(g, n, bias);
  if (g.partial != nullptr) g.partial += (int64_t)at.split * g.m * g.n;
  const bool inner = m0 + BM <= g.m && n0 + BN <= g.n;  // no result outside D
#pragma unroll
  for (int p = 0; p < FM; p += PART) {
#pragma unroll
    for (int i = 0; i < PART; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
        *reinterpret_cast<f32x4*>(turn + slot(i * 16 + (lane & 15), j * 4 + (lane >> 4))) = acc[p + i][j];
    const int r = lane / RUNS;
    const int64_t m = m0 + wm * TM + p * 16 + r;
    const auto take = [&](int row, float* z) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(turn + slot(row, lane % RUNS * 2 + q));
#pragma unroll
        for (int e = 0; e < 4; ++e) z[q * 4 + e] = v[e];
      }
    };
    if (inner) {
      constexpr int BATCH = PASSES < 4 ? PASSES : 4;
#pragma unroll 1
      for (int h = 0; h < PASSES; h += BATCH)
        finish_rows<E, BATCH>(g, m + h * ROWS, ROWS, n, bias, [&](int b, float* z) { take((h + b) * ROWS + r, z); });
    } else {
#pragma unroll 1
      for (int h = 0; h < PASSES; ++h) {
        float z[kVec];
        take(h * ROWS + r, z);
        finish_group<E>(g, m + h * ROWS, n, bias, z);
      }
    }
  }
}

template <class E, int BM, int BN, int WM, int WN, int STAGES, bool AX, bool BX, LoadPath PATH>
__global__ void __launch_bounds__(WM * WN * 64) __attribute__((amdgpu_waves_per_eu(2)))  // 256 registers, no second file
    linear_kernel(GemmArgs g) {
  linear_tile<E, BM, BN, WM, WN, STAGES, AX, BX, PATH>(g, (int)blockIdx.x);
}

template <class E, int BM, int BN, int WM, int WN, int STAGES, bool AX, bool BX, LoadPath PATH>
hipError_t linear_launch(const GemmArgs& g, hipStream_t stream) {
  constexpr int lds = STAGES * (BM + BN) * kStageBytes;
  const auto kernel = linear_kernel<E, BM, BN, WM, WN, STAGES, AX, BX, PATH>;
  static const hipError_t ready = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                      hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (ready != hipSuccess) return ready;
  GemmArgs t = g;
  t.tiles_m = (int)((g.m + BM - 1) / BM);
  t.tiles_n = (int)((g.n + BN - 1) / BN);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(t.tiles_m * t.tiles_n * t.splits)), dim3(WM * WN * 64), lds, stream, t);
  return hipGetLastError();
}

// dW and dx in one launch, neither with its k split: the first workgroups take the tiles of the one with the longer k.
// Where each alone leaves CUs idle they fill each other's rounds.
template <class E, int BM, int BN, int WM, int WN, int STAGES, LoadPath PATH>
__global__ void __launch_bounds__(WM * WN * 64) __attribute__((amdgpu_waves_per_eu(2)))
    linear_grads_kernel(GemmArgs dw, GemmArgs dx) {
  const bool dw_first = dw.k >= dx.k;
  const int id = (int)blockIdx.x, first = dw_first ? dw.tiles_m * dw.tiles_n : dx.tiles_m * dx.tiles_n;
  const int at = id < first ? id : id - first;
  if ((id < first) == dw_first) linear_tile<E, BM, BN, WM, WN, STAGES, true, true, PATH>(dw, at);
  else linear_tile<E, BM, BN, WM, WN, STAGES, false, true, PATH>(dx, at);
}

template <class E, int BM, int BN, int WM, int WN, int STAGES, LoadPath PATH>
hipError_t grads_launch(const GemmArgs& dw, const GemmArgs& dx, hipStream_t stream) {
  constexpr int lds = STAGES * (BM + BN) * kStageBytes;
  const auto kernel = linear_grads_kernel<E, BM, BN, WM, WN, STAGES, PATH>;
  static const hipError_t ready = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                      hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (ready != hipSuccess) return ready;
  GemmArgs t[2] = {dw, dx};
  for (GemmArgs& g : t) {
    g.tiles_m = (int)((g.m + BM - 1) / BM);
    g.tiles_n = (int)((g.n + BN - 1) / BN);
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)(t[0].tiles_m * t[0].tiles_n + t[1].tiles_m * t[1].tiles_n)),
                     dim3(WM * WN * 64), lds, stream, t[0], t[1]);
  return hipGetLastError();
}

// ----------------------------------------------------------------------------------
// Few tokens (at most 16 MT): y = act(x W^T + b) + r is bound by reading W once.  A workgroup takes 16 NT of
// W's rows, each of its waves a range of k.  With direct loads a wave streams its part of both operands through LDS
// of its own, STAGES stages of 128 bytes of k a row, without a barrier: whole cache lines, many of them in
// flight, and no registers held for them.  Without (rows that start anywhere) the fragments come from
// memory, half a line a row and instruction.  The waves' sums meet in LDS.  One token of 4096 x 4096, with a residual:
// 5.9 us (33.6 MB that the Infinity Cache holds: 5.7 TB/s), 7.7 without; 61 tokens, 1024 -> 4096, gelu: 5.3 and 7.7.
template <class E, int MT, int NT, int WAVES, int STAGES, LoadPath PATH>
__global__ void __launch_bounds__(WAVES * 64) __attribute__((amdgpu_waves_per_eu(2))) linear_few_kernel(GemmArgs g) {
  using T = typename E::T;
  constexpr bool DMA = PATH != kByRegisters;
  constexpr int BK = kStageBytes / (int)sizeof(T), STAGE = 16 * (MT + NT) * kStageBytes;
  constexpr int PRIVATE = DMA ? STAGES * STAGE : NT * MT * 1024;
  static_assert(PRIVATE >= NT * MT * 1024);
  extern __shared__ __attribute__((aligned(1024))) char linear_lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
  char* const mine = linear_lds + wave * PRIVATE;
  const int64_t n0 = (int64_t)blockIdx.x * (16 * NT);
  f32x4 acc[NT][MT];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const auto multiply = [&](const u32x4* w, const u32x4* x) {
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i) acc[j][i] = mfma_chunk<E>(w[j], x[i], acc[j][i]);
  };
  const int64_t stages = (g.k + BK - 1) / BK, per = (stages + WAVES - 1) / WAVES * BK;
  const int64_t k0 = min(wave * per, g.k), k1 = min(k0 + per, g.k);

  if constexpr (DMA) {
    Operand<E, 16 * NT, 1, false, PATH> w;
    Operand<E, 16 * MT, 1, false, PATH> x;
    w.init(static_cast<const T*>(g.b), g.ldb, n0, g.n, k0, k1, 0, lane);
    x.init(static_cast<const T*>(g.a), g.lda, 0, g.m, k0, k1, 0, lane);
    Fragments<E, 16, false> f;
    f.init(0, lane);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine;
    const int steps = (int)((k1 - k0 + BK - 1) / BK);
    constexpr int EACH = w.LINES + x.LINES;
    const auto fetch = [&](int slot) {
      w.fetch(lds0 + (uint32_t)slot * STAGE);
      x.fetch(lds0 + (uint32_t)slot * STAGE + w.BYTES);
    };
#pragma unroll
    for (int q = 0; q < STAGES; ++q)
      if (q < steps) fetch(q);
    int slot = 0;
    for (int t = 0; t < steps; ++t) {
      if (t + STAGES <= steps) loads_wait<(STAGES - 1) * EACH>();
      else loads_wait<0>();
      const char* const at = mine + slot * STAGE;
      u32x4 vw[2][NT], vx[2][MT];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
        for (int j = 0; j < NT; ++j) vw[kk][j] = f.read(at, j, kk);
#pragma unroll
        for (int i = 0; i < MT; ++i) vx[kk][i] = f.read(at + w.BYTES, i, kk);
      }
      if (t + STAGES < steps) {
        reads_wait();
        fetch(slot);
      }
      slot = slot + 1 == STAGES ? 0 : slot + 1;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) multiply(vw[kk], vx[kk]);
    }
    reads_wait();
  } else {
    // rows beyond the last stand for it; their results are not stored
    constexpr int EPC = 16 / (int)sizeof(T), HALF = BK / 2, U = NT + MT > 4 ? 4 : 8;
    const int r = lane & 15, grp = lane >> 4;
    const T *wp[NT], *xp[MT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
      wp[j] = static_cast<const T*>(g.b) + min(n0 + j * 16 + r, g.n - 1) * g.ldb + k0 + grp * EPC;
#pragma unroll
    for (int i = 0; i < MT; ++i)
      xp[i] = static_cast<const T*>(g.a) + min((int64_t)(i * 16 + r), g.m - 1) * g.lda + k0 + grp * EPC;
    const auto whole = [](const T* p) {
      const Bytes16 v = *reinterpret_cast<const Bytes16*>(p);
      return u32x4{v.w[0], v.w[1], v.w[2], v.w[3]};
    };
    const int depth = (int)(k1 - k0);
    const auto step = [&](int s, int count, auto load) {
      u32x4 vw[U][NT], vx[U][MT];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u >= count) break;
#pragma unroll
        for (int j = 0; j < NT; ++j) vw[u][j] = load(wp[j] + (s + u) * HALF, s + u);
#pragma unroll
        for (int i = 0; i < MT; ++i) vx[u][i] = load(xp[i] + (s + u) * HALF, s + u);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u >= count) break;
        multiply(vw[u], vx[u]);
      }
    };
    int s = 0;
    for (; (s + U) * HALF <= depth; s += U) step(s, U, [&](const T* p, int) { return whole(p); });
    for (; s * HALF < depth; ++s)
      step(s, 1, [&](const T* p, int at) {
        const int left = depth - at * HALF - grp * EPC;
        if (left >= EPC) return whole(p);
        u32x4 h = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < EPC; ++e)
          if (e < left) h[e / 2] |= (uint32_t)p[e] << (16 * (e % 2));
        return h;
      });
  }
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i) reinterpret_cast<f32x4*>(mine)[(j * MT + i) * 64 + lane] = acc[j][i];
  __syncthreads();
  // eight results of one token to a thread, groups of a row side by side
  constexpr int UNITS = MT * 16 * NT * 2;
  static_assert(UNITS <= WAVES * 64);
  const int unit = threadIdx.x;
  if (unit >= UNITS) return;
  const int q = unit % (NT * 2), m = unit / (NT * 2);
  const int at = (q / 2 * MT + m / 16) * 64 + (q & 1) * 32 + (m & 15);
  float z[kVec] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, bias[kVec];
  read_bias<E>(g, n0 + q * kVec, bias);
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const f32x4* const part = reinterpret_cast<const f32x4*>(linear_lds + w * PRIVATE);
    const f32x4 lo = part[at], hi = part[at + 16];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      z[e] += lo[e];
      z[4 + e] += hi[e];
    }
  }
  finish_group<E>(g, m, n0 + q * kVec, bias, z);
}

template <class E, int MT, int NT, int WAVES, int STAGES, LoadPath PATH>
hipError_t few_launch(const GemmArgs& g, hipStream_t stream) {
  constexpr int lds = WAVES * (PATH != kByRegisters ? STAGES * 16 * (MT + NT) * kStageBytes : NT * MT * 1024);
  const auto kernel = linear_few_kernel<E, MT, NT, WAVES, STAGES, PATH>;
  static const hipError_t ready = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                      hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (ready != hipSuccess) return ready;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((g.n + 16 * NT - 1) / (16 * NT))), dim3(WAVES * 64), lds, stream, g);
  return hipGetLastError();
}

template <class E>
LinearTable make_linear_table() {
  LinearTable t{};
  constexpr bool F32 = E::kId == kStorageF32;
  // the loads of whole chunks, and those of anything else
  constexpr LoadPath W = kDirect, ANY = F32 ? kDirectCut : kByRegisters;
  const auto operands = [&](auto ax, auto bx, LinearOperands o) {
    constexpr bool AX = decltype(ax)::value, BX = decltype(bx)::value;
    t.fn[kTile64][o][0] = linear_launch<E, 64, 64, 2, 2, F32 ? 3 : 2, AX, BX, ANY>;
    t.fn[kTile64][o][1] = linear_launch<E, 64, 64, 2, 2, 3, AX, BX, W>;
    if constexpr (!AX) {
      t.fn[kTile32x64][o][1] = linear_launch<E, 32, 64, 2, 2, 3, AX, BX, W>;
      if constexpr (F32) t.fn[kTile32x64][o][0] = linear_launch<E, 32, 64, 2, 2, 3, AX, BX, ANY>;
    }
    // (float32 products are bound by the matrix cores in the smallest tiles already: 4096 x 4096 x 4096 takes 970 to 1010 us
    // in 64 x 64, 136 to 141 TFLOP/s, the library 960 to 1000)
    if constexpr (!F32) {
      t.fn[kTile128][o][0] = linear_launch<E, 128, 128, 2, 4, 2, AX, BX, ANY>;
      // (both operands across k need more than the 256 registers there are)
      if constexpr (!AX) t.fn[kTile128x256][o][0] = linear_launch<E, 128, 256, 2, 4, 2, AX, BX, ANY>;
      t.fn[kTile128][o][1] = linear_launch<E, 128, 128, 2, 4, 2, AX, BX, W>;
      t.fn[kTile128x256][o][1] = linear_launch<E, 128, 256, 2, 4, 3, AX, BX, W>;
      t.fn[kTile256][o][1] = linear_launch<E, 256, 256, 2, 4, 2, AX, BX, W>;
    }
  };
  operands(std::false_type{}, std::false_type{}, kForward);
  operands(std::false_type{}, std::true_type{}, kGradX);
  operands(std::true_type{}, std::true_type{}, kGradW);
  t.grads[kTile64] = grads_launch<E, 64, 64, 2, 2, 3, W>;
  if constexpr (!F32) t.grads[kTile128] = grads_launch<E, 128, 128, 2, 4, 2, W>;
  t.few[0][0][1] = few_launch<E, 1, 1, 8, 4, W>;
  t.few[0][1][1] = few_launch<E, 1, 2, 4, 6, W>;
  t.few[1][0][1] = few_launch<E, 2, 1, 4, 6, W>;
  t.few[1][1][1] = few_launch<E, 2, 2, 4, 4, W>;
  t.few[2][0][1] = few_launch<E, 4, 1, 4, 4, W>;
  t.few[2][1][1] = few_launch<E, 4, 2, 4, 3, W>;
  t.few[0][0][0] = few_launch<E, 1, 1, 8, F32 ? 4 : 0, ANY>;
  t.few[0][1][0] = few_launch<E, 1, 2, F32 ? 4 : 8, F32 ? 6 : 0, ANY>;
  t.few[1][0][0] = few_launch<E, 2, 1, F32 ? 4 : 8, F32 ? 6 : 0, ANY>;
  t.few[1][1][0] = few_launch<E, 2, 2, F32 ? 4 : 8, F32 ? 4 : 0, ANY>;
  t.few[2][0][0] = few_launch<E, 4, 1, F32 ? 4 : 8, F32 ? 4 : 0, ANY>;
  t.few[2][1][0] = few_launch<E, 4, 2, F32 ? 4 : 8, F32 ? 3 : 0, ANY>;
  return t;
}

}  // namespace rdfft
