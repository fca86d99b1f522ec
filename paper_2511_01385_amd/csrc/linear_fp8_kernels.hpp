// linear_fp8_kernels.hpp -- the dense product of operands in 8-bit floating point, with the epilogue of
// linear_kernels.hpp, as templates over the storage type of D (linear_fp8_{f32,bf16,f16}.hip instantiate them).
//
//   D(m, n) = sum over k of A(m, k) B(n, k),  A(m, k) = code * 2^(scale byte of its block of 128 k - 127)
//
// Both operands run along k: quantize has left each as the product at hand needs it.  A stage is 128 bytes of k, so one
// block of the format, and lies in LDS as in linear_kernels.hpp.  The scaled matrix instructions take a
// scale byte per row of a fragment with it, so that the blocks' scales cost no arithmetic.  Bytes come four stages at
// a time: a dword per row goes straight to LDS beside the stages, one group of four ahead, from there to a register of
// the lane that holds the row, and is shifted by a byte from stage to stage.
//
// The order of k within a stage is free, as long as both operands have the same: a fragment's lane takes whole
// chunks of 16 bytes, and all of a stage's k share a scale per row.
//
// Sums.  The accumulators are float32, but the 8-bit matrix instructions add their products after aligning them to the
// largest, about 16 bits down: results are 1.5e-5 of their norm off (5e-5 for codes spread evenly over all exponents),
// next to a rounding of 2.1e-4 (float16) or 1.7e-3 (bfloat16).  A float32 D is worth more than that: its operands' codes are
// widened to bfloat16, exactly, for the 16-bit instructions, whose sums are float32 throughout (4e-7 of the norm); a block's sum
// takes its scales (any two of them: their product alone has to be a float32 number) on its way to the accumulator.  The
// instructions run at half the rate; with the conversions and the scales a product takes 3.3 times as long (below).
//
// What bounds it: 8192 tokens, 8192 -> 4096 (normal values) takes 198 us, 2770 TFLOP/s (the library's product, without
// block scales, 182), and 154 us with operands of zeros: power takes the clock to 1.9 GHz, at which the matrix cores are busy
// 62 to 70 % of the cycles.  4096 -> 8192: 212 to 221 us (library 225), with bias, gelu and checkpoint in the epilogue 41 more.
// Two halves of a stage in registers, as the 16-bit kernels hold them, spill in a tile of 256 x 256 (five times the time):
// there the fragments of A come one by one, which leaves 3 of 256 registers spilled.  Four waves of 128 x 128 with accumulators
// in the second register file took 209 us, 177 with zeros.  float32 results: 8192 x 4096 -> 4096 363 to 381 us (16-bit results
// 113), 720 to 757 TFLOP/s: the arithmetic of the scales and conversions.
#pragma once

#include "fp8_device.hpp"
#include "fp8_launch.hpp"
#include "linear_kernels.hpp"

namespace rdfft {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// codes as the fragments' elements
struct ElemCode {
  using T = uint8_t;
};

// Which chunk of LDS row r holds the row's chunk c: c ^ code_swizzle(r).  A read of 16 bytes a lane is done 16 lanes at a
// time, lanes 0-3, 12-15, 20-27 and the like: with 32 rows to a fragment those are rows of which two agree modulo eight, and
// bit 3 of the row keeps them apart (without it half of the cycles that the LDS was busy were conflicts).  With 16 rows to a
// fragment the lanes' two chunks do.
template <int FRAGMENT>
__device__ __forceinline__ int code_swizzle(int r) {
  return FRAGMENT == 32 ? (r & 7) ^ (r >> 3 & 1) : r & 7;
}

// R rows of one operand's stage on their way to LDS, as Operand of linear_kernels.hpp loads them, in fewer registers:
// a lane's part of line j lies 8 j rows below that of line 0, in the same chunk or its neighbour, and rows past the last are
// out of the buffer's bounds.
// GROUPS: the stages that a step takes.
template <int R, int WAVES, int FRAGMENT, int GROUPS = 1>
struct CodeOperand {
  static constexpr int BYTES = R * kStageBytes, LINES = BYTES / 1024 / WAVES;
  static_assert(LINES * WAVES * 1024 == BYTES && LINES % 2 == 0, "lines' parities are those of j");
  const uint8_t* base;  // row 0 and this stage's k 0 of the tile
  uint32_t ld, offset;  // bytes from row to row; of this lane's part of line 0
  uint32_t above;       // bytes of the rows that exist but for the last
  int depth;            // k that is left
  int chunk, wave;      // chunk: of line 0

  __device__ __forceinline__ void init(const Fp8Operand& o, int64_t r0, int64_t r_end, int64_t k0, int64_t k_end, int wave_,
                                       int lane) {
    base = o.codes + r0 * o.ld + k0;
    ld = (uint32_t)o.ld;
    const int rows = (int)min(r_end - r0, (int64_t)R);
    above = (uint32_t)(rows - 1) * ld;
    depth = (int)(k_end - k0);
    wave = wave_;
    chunk = (lane & 7) ^ (lane >> 3);
    offset = (uint32_t)(wave * LINES * 8 + lane / 8) * ld + (uint32_t)chunk * 16u;
  }
  // (a row's last chunk counts whole)
  __device__ __forceinline__ int records() const { return depth > 0 ? (int)(above + ((uint32_t)depth + 15) / 16 * 16) : 0; }
  // line j of a stage in front of the end of k; step() after the last
  __device__ __forceinline__ void fetch_line(int j, uint32_t lds) const {
    load_to_lds<16>(reinterpret_cast<const char*>(base), at(j), lds + (uint32_t)(wave * LINES + j) * 1024u, records());
  }
  __device__ __forceinline__ int chunk_of(int j) const { return FRAGMENT == 32 ? chunk ^ (j & 1) : chunk; }
  __device__ __forceinline__ uint32_t at(int j) const {
    return offset + (uint32_t)(8 * j) * ld + (uint32_t)((chunk_of(j) - chunk) * 16);
  }
  __device__ __forceinline__ void step() {
    base += GROUPS * kStageBytes;
    depth -= GROUPS * kStageBytes;
  }
  // any stage: chunks past the end of k are zeros
  __device__ __forceinline__ void fetch(uint32_t lds) {
#pragma unroll
    for (int j = 0; j < LINES; ++j)
      load_to_lds<16>(reinterpret_cast<const char*>(base), chunk_of(j) * 16 < depth ? at(j) : kNowhere,
                      lds + (uint32_t)(wave * LINES + j) * 1024u, records());
    step();
  }
};

// bytes 8q ... 8q+7 of a lane's 32 as bfloat16 values (exact)
__device__ __forceinline__ bf16x8 widen_codes(i32x8 v, int q) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  union {
    bf16x2 pair[4];
    bf16x8 all;
  } u;
  u.pair[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * q], 1.f, false);
  u.pair[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * q], 1.f, true);
  u.pair[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * q + 1], 1.f, false);
  u.pair[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * q + 1], 1.f, true);
  return u.all;
}

// 32 x 32 results of 64 k: lane l holds row l % 32 of either operand and k chunks l / 32, l / 32 + 2 of four.
// Scale bytes are the lowest of sa and sb; the wide form leaves them out.
__device__ __forceinline__ f32x16 product32(i32x8 a, i32x8 b, f32x16 c, uint32_t sa, uint32_t sb) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, (int)sa, 0, (int)sb);
}
__device__ __forceinline__ f32x16 product32_wide(i32x8 a, i32x8 b, f32x16 c) {
#pragma unroll
  for (int q = 0; q < 4; ++q)
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen_codes(a, q), widen_codes(b, q), c, 0, 0, 0);
  return c;
}
// 16 x 16 results of 128 k: row l % 16, chunks l / 16 and l / 16 + 4 of eight
__device__ __forceinline__ f32x4 product16(i32x8 a, i32x8 b, f32x4 c, uint32_t sa, uint32_t sb) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, (int)sa, 0, (int)sb);
}
__device__ __forceinline__ f32x4 product16_wide(i32x8 a, i32x8 b) {
  f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int q = 0; q < 4; ++q)
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen_codes(a, q), widen_codes(b, q), c, 0, 0, 0);
  return c;
}
// whether one of a dword's bytes is the scale of a block that is not finite
__device__ __forceinline__ bool has_nan_scale(uint32_t v) { return (((v & 0x7f7f7f7fu) + 0x01010101u) & v & 0x80808080u) != 0; }
// a block's sum of codes' products times its two powers of two, or NaN
__device__ __forceinline__ float scaled_or_nan(float v, int a, int b) {
  return a == kCkNaN || b == kCkNaN ? __uint_as_float(0x7fc00000u) : ldexpf(v, a + b - 254);
}

__device__ __forceinline__ i32x8 join_chunks(u32x4 lo, u32x4 hi) {
  return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// Fragments of 32 rows at row0 + 32 f, half kk of a stage.
struct Fragments32 {
  uint32_t first;  // half 0's first chunk: the others' places differ in two bits
  __device__ __forceinline__ void init(int row0, int lane) {
    first = (uint32_t)((row0 + (lane & 31)) * kStageBytes + ((lane >> 5) ^ code_swizzle<32>(lane & 31)) * 16);
  }
  __device__ __forceinline__ i32x8 read(const char* lds, int f, int kk) const {
    const char* const p = lds + f * 32 * kStageBytes;
    return join_chunks(*reinterpret_cast<const u32x4*>(p + (first ^ (uint32_t)(kk * 64))),
                       *reinterpret_cast<const u32x4*>(p + (first ^ (uint32_t)(kk * 64 + 32))));
  }
};

// Keeps what is computed from v inside the loop that this stands in: else it would lie in registers all along.
__device__ __forceinline__ void recompute(uint32_t& v) { asm volatile("" : "+v"(v)); }

// Zeros in place of what follows the last `left` bytes of k in a stage's rows (left % 16 != 0; whole chunks past the
// end are zeros already): what lies behind a row's end may be anything.
template <int FRAGMENT>
__device__ __forceinline__ void cut_stage(char* lds, int rows, int left, int thread, int threads) {
  const int c = left / 16, keep = left % 16;
  for (int r = thread; r < rows; r += threads) {
    u32x4* const p = reinterpret_cast<u32x4*>(lds + r * kStageBytes + (c ^ code_swizzle<FRAGMENT>(r)) * 16);
    u32x4 v = *p;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int bytes = keep - w * 4;
      v[w] = bytes >= 4 ? v[w] : bytes <= 0 ? 0u : v[w] & ((1u << (8 * bytes)) - 1);
    }
    *p = v;
  }
}

// The scale bytes of an operand's rows r0 ... for the four stages of a group: a dword for each of 64 rows from `row`
// on, straight to LDS.
__device__ __forceinline__ void fetch_scales(const Fp8Operand& o, int64_t r0, int64_t r_end, int row, int group, uint32_t lds,
                                             int lane) {
  const int64_t first = r0 >> o.shift;
  const int64_t r = r0 + row + lane;
  const uint32_t at = (uint32_t)((r >> o.shift) - first) * (uint32_t)o.lds + (uint32_t)group * 4u;
  load_to_lds<4>(reinterpret_cast<const char*>(o.scales) + first * o.lds, r < r_end ? at : kNowhere, lds);
}

template <class E, int BM, int BN, int WM, int WN, int STAGES, int KG>
struct Fp8Tile {
  static constexpr int THREADS = WM * WN * KG * 64;
  static constexpr int STAGE = (BM + BN) * kStageBytes;
  // rows of scales, in whole loads of 64
  static constexpr int SA = (BM + 63) / 64 * 64, SB = (BN + 63) / 64 * 64, SLOT = (SA + SB) * 4;
  static constexpr int SLOTS = 4;
  static constexpr int LDS = STAGES * KG * STAGE + SLOTS * SLOT;
  static_assert(LDS <= 160 * 1024);
};

// KG groups of WM x WN waves share the tile: of a step's KG stages each multiplies its own, and their sums meet in LDS at
// the end.  A step of several stages costs little more than one where nothing but its own latency holds it up: where a CU
// has one workgroup, and small tiles.
template <class E, int BM, int BN, int WM, int WN, int STAGES, int KG>
__device__ __forceinline__ void linear_fp8_tile(const Gemm8Args& args, int id) {
  using Tile = Fp8Tile<E, BM, BN, WM, WN, STAGES, KG>;
  GemmArgs g = args.g;
  constexpr bool WIDE = E::kId == kStorageF32;
  constexpr int WAVES = WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 32, FN = TN / 32;
  constexpr int BK = kStageBytes, STAGE = Tile::STAGE;
  constexpr bool STREAM = FM >= 4 && !WIDE;  // fragments of A one at a time: two halves of a stage take too many registers
  using OpA = CodeOperand<BM, WAVES, 32, KG>;
  using OpB = CodeOperand<BN, WAVES, 32, KG>;
  extern __shared__ __attribute__((aligned(1024))) char linear_lds[];
  const int lane = threadIdx.x & 63, any_wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
  const int kg = any_wave / WAVES, wave = any_wave % WAVES;
  const int wm = wave / WN, wn = wave % WN;
  const TileAt at = tile_of(id, g.tiles_m, g.tiles_n, g.splits);
  const int64_t m0 = (int64_t)at.tm * BM, n0 = (int64_t)at.tn * BN;
  const int64_t k0 = (int64_t)at.split * g.k_split, k1 = min(k0 + g.k_split, g.k);

  OpA a;
  OpB b;
  a.init(args.a, m0, g.m, k0 + kg * BK, k1, wave, lane);
  b.init(args.b, n0, g.n, k0 + kg * BK, k1, wave, lane);
  Fragments32 fa, fb;
  fa.init(wm * TM, lane);
  fb.init(wn * TN, lane);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)linear_lds;

  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  // Half a stage's fragments.  A half is read while the one before it is multiplied.
  struct Half {
    i32x8 a[FM], b[FN];
  };
  // This stage's scale bytes in the lowest place, the group's later ones above: of the rows of A and B that a lane
  // holds, or (wide) of the row of A and the sixteen of B that its results belong to.
  constexpr int SBS = WIDE ? 16 : 1;
  uint32_t sa[FM], sb[FN][SBS];
  f32x16 block[WIDE ? FM : 1][WIDE ? FN : 1];  // wide: this stage's sums
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
      for (int j = 0; j < FN; ++j) {
        if constexpr (WIDE) block[i][j] = product32_wide(h.b[j], h.a[i], block[i][j]);
        else acc[i][j] = product32(h.b[j], h.a[i], acc[i][j], sb[j][0], sa[i]);
      }
  };
  const auto clear_block = [&] {
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) block[i][j][e] = 0.f;
    }
  };
  int odd_scales = 0;  // wide: whether this wave has a block that is not finite in this group of stages
  const auto add_block = [&] {
    if constexpr (WIDE) {
      const auto each = [&](auto&& times) {
#pragma unroll
        for (int i = 0; i < FM; ++i) {
          const int of_a = (int)(sa[i] & 255), power = of_a - 254;
#pragma unroll
          for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] += times(block[i][j][e], of_a, power, (int)(sb[j][e] & 255));
        }
      };
      if (__builtin_amdgcn_readfirstlane(odd_scales)) each([](float v, int a, int, int b) { return scaled_or_nan(v, a, b); });
      else each([](float v, int, int power, int b) { return ldexpf(v, power + b); });
    }
  };
  const int stages = (int)((k1 - k0 + BK - 1) / BK), steps = (stages + KG - 1) / KG, s0 = (int)(k0 / BK);
  const int groups = (int)((k1 + 4 * BK - 1) / (4 * BK));
  constexpr int SCALES = STAGES * KG * STAGE;  // where they lie in LDS
  // the scales of a group of four stages on their way to its slot
  const auto fetch_group = [&](int group) {
    if (group >= groups) return;
    const uint32_t slot = lds0 + SCALES + (uint32_t)(group & (Tile::SLOTS - 1)) * Tile::SLOT;
    for (int q = any_wave; q < (Tile::SA + Tile::SB) / 64; q += WAVES * KG) {
      if (q < Tile::SA / 64) fetch_scales(args.a, m0, g.m, q * 64, group, slot + (uint32_t)q * 256u, lane);
      else fetch_scales(args.b, n0, g.n, q * 64 - Tile::SA, group, slot + (uint32_t)q * 256u, lane);
    }
  };
  const auto take_group = [&](int group) {
    const uint32_t* const p = reinterpret_cast<const uint32_t*>(linear_lds + SCALES + (group & (Tile::SLOTS - 1)) * Tile::SLOT);
#pragma unroll
    for (int i = 0; i < FM; ++i) sa[i] = p[wm * TM + i * 32 + (lane & 31)];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const uint32_t* const of = p + Tile::SA + wn * TN + j * 32;
#pragma unroll
      for (int e = 0; e < SBS; ++e) sb[j][e] = of[WIDE ? 8 * (e / 4) + 4 * (lane >> 5) + e % 4 : lane & 31];
    }
    if constexpr (WIDE) {
      bool odd = false;
#pragma unroll
      for (int i = 0; i < FM; ++i) odd |= has_nan_scale(sa[i]);
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < SBS; ++e) odd |= has_nan_scale(sb[j][e]);
      odd_scales = __any(odd);
    }
  };
  const auto shift_scales = [&](int bits) {
#pragma unroll
    for (int i = 0; i < FM; ++i) sa[i] >>= bits;
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < SBS; ++e) sb[j][e] >>= bits;
  };
  // Step t's scales into the lowest place.  Three groups beyond the one that the step begins in are there or on their way, in
  // four slots: a step and the next reach into two of them, and the slot that is filled anew was last read at the
  // start of the step before, with a barrier since.
  const auto scales_of = [&](int t) {
    if (t == 0) return;
    const int first = s0 + t * KG, s = first + kg;
    if ((s & 3) < KG) {
      take_group(s >> 2);
      if (KG > 1) shift_scales((s & 3) * 8);
    } else {
      shift_scales(8 * KG);
    }
    if ((first & 3) < KG) fetch_group((first >> 2) + 3);
  };
  static_assert(STAGES <= 3, "a group of scales has landed by the step that takes it");
  // STAGES - 1 stages are under way ahead of the one being multiplied; the barrier sits between a stage's halves.
  constexpr int EACH = OpA::LINES + OpB::LINES;
  const auto fetch = [&](int slot) {
    a.fetch(lds0 + (uint32_t)(slot * KG + kg) * STAGE);
    b.fetch(lds0 + (uint32_t)(slot * KG + kg) * STAGE + OpA::BYTES);
  };
  const int tail = (int)((k1 - k0) % BK);
  const auto cut = [&](int slot) {
    if (tail % 16 == 0) return;
    cut_stage<32>(linear_lds + (slot * KG + (stages - 1) % KG) * STAGE, BM + BN, tail, (int)threadIdx.x,
                  Tile::THREADS);  // (BM is a multiple of 16 rows)
    reads_wait();
    wave_barrier();
  };
  // One half's products with the other's reads and a stage's loads between them, a row of fragments at a time.
  const auto weave = [&](const Half& h, Half& to, const char* from, int slot) {
    constexpr int TOTAL = FM + FN;
    const uint32_t la = lds0 + (uint32_t)(slot * KG + kg) * STAGE, lb = la + OpA::BYTES;
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
      for (int j = 0; j < FN; ++j) {
        if constexpr (WIDE) block[i][j] = product32_wide(h.b[j], h.a[i], block[i][j]);
        else acc[i][j] = product32(h.b[j], h.a[i], acc[i][j], sb[j][0], sa[i]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    a.step();
    b.step();
  };
  constexpr bool SMALL = FM * FN <= 2;
  constexpr int PRODUCTS = FM * FN * (WIDE ? 4 : 1), READS = 2 * (FM + FN);
  const auto interleave = [&] {
    constexpr int GROUPS = READS < PRODUCTS ? READS : PRODUCTS;
#pragma unroll
    for (int q = 0; q < GROUPS; ++q) {
      __builtin_amdgcn_sched_group_barrier(0x008, PRODUCTS / GROUPS, 0);  // matrix instructions
      __builtin_amdgcn_sched_group_barrier(0x100, READS / GROUPS, 0);    // LDS reads
    }
  };
  if (steps > 0) {
    // (older than the stages, so that the waits for those cover them)
    for (int q = 0; q < Tile::SLOTS; ++q) fetch_group((s0 >> 2) + q);
  }
#pragma unroll
  for (int q = 0; q < STAGES; ++q)
    if (q < steps) fetch(q);
  if (steps > 0) {
    if (steps >= STAGES) stage_wait<(STAGES - 1) * EACH>();
    else stage_wait<0>();
    if (steps == 1) cut(0);
    take_group((s0 + kg) >> 2);
    shift_scales(((s0 + kg) & 3) * 8);
  }
  int cur = 0, t = 0;
  const auto next = [](int slot) { return slot + 1 == STAGES ? 0 : slot + 1; };
  const int steady = steps - 1 - STAGES;  // (the stage that is fetched is not the last)
  if constexpr (STREAM) {
    static_assert(KG == 1);
    // Fragments of A come one at a time, AHEAD steps before their products, into a ring; those of B half a stage
    // before.  The barrier comes when the stage's last fragment is read, AHEAD steps before its end.
    constexpr int STEPS = 2 * FM, AHEAD = 3, RING = 4, LAST = STEPS - AHEAD;
    static_assert(STEPS % RING == 0 && FN <= LAST);
    i32x8 ring[RING], hb[2][FN];
    const auto stage = [&](auto is_steady) {
      constexpr bool STEADY = decltype(is_steady)::value;
      const char* const here = linear_lds + cur * STAGE;
      const char* const there = linear_lds + next(cur) * STAGE;
      const uint32_t la = lds0 + (uint32_t)cur * STAGE, lb = la + OpA::BYTES;
      recompute(a.offset);
      recompute(b.offset);
      recompute(fa.first);
      recompute(fb.first);
      scales_of(t);
      const bool more = STEADY || t + 1 < steps;
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        if (s == LAST) {
          if constexpr (STEADY) {
            stage_wait<(STAGES - 2) * EACH>();
          } else if (more) {
            stage_wait<0>();
            if (t + STAGES < steps) fetch(cur);
            if (t + 2 == steps) cut(next(cur));
          }
        }
        if constexpr (STEADY) {
          if (s >= LAST) {
#pragma unroll
            for (int e = (s - LAST) * EACH / AHEAD; e < (s - LAST + 1) * EACH / AHEAD; ++e) {
              if (e < OpA::LINES) a.fetch_line(e, la);
              else b.fetch_line(e - OpA::LINES, lb);
            }
          }
        }
        const int to = s + AHEAD;
        if (s < FN) hb[1][s] = fb.read(here + OpA::BYTES, s, 1);
        if (s < LAST) {
          ring[to % RING] = fa.read(here, to % FM, to / FM);
        } else if (more) {
#pragma unroll
          for (int j = (s - LAST) * FN / AHEAD; j < (s - LAST + 1) * FN / AHEAD; ++j) hb[0][j] = fb.read(there + OpA::BYTES, j, 0);
          ring[to % RING] = fa.read(there, (to - STEPS) % FM, (to - STEPS) / FM);
        }
#pragma unroll
        for (int j = 0; j < FN; ++j)
          acc[s % FM][j] = product32(hb[s / FM][j], ring[s % RING], acc[s % FM][j], sb[j][0], sa[s % FM]);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (STEADY) {
        a.step();
        b.step();
      }
      cur = next(cur);
    };
    if (steps > 0) {
#pragma unroll
      for (int j = 0; j < FN; ++j) hb[0][j] = fb.read(linear_lds + OpA::BYTES, j, 0);
#pragma unroll
      for (int s = 0; s < AHEAD; ++s) ring[s] = fa.read(linear_lds, s % FM, s / FM);
    }
    for (; t < steady; ++t) stage(std::true_type{});
#pragma unroll 1
    for (; t < steps; ++t) stage(std::false_type{});
  } else {
    const auto place = [&](int slot) { return linear_lds + (slot * KG + kg) * STAGE; };
    Half h0, h1;
    if (steps > 0) read(h0, place(0), 0);
    for (; t < steady; ++t) {
      // (few products: the reads go first, else they would set out behind products that wait for the half before)
      if (SMALL) {
        read(h1, place(cur), 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      scales_of(t);
      clear_block();
      if (!SMALL) read(h1, place(cur), 1);
      multiply(h0);
      if (!SMALL) interleave();
      stage_wait<(STAGES - 2) * EACH>();
      weave(h1, h0, place(next(cur)), cur);
      add_block();
      cur = next(cur);
    }
    for (; t < steps; ++t) {
      const bool mine = KG == 1 || t * KG + kg < stages;  // (the last step may have no stage for this group)
      read(h1, place(cur), 1);
      scales_of(t);
      clear_block();
      if (mine) multiply(h0);
      if (t + 1 < steps) {
        // this stage is read; the next has landed when those after it are all that is left
        if (STAGES > 2 && t + STAGES - 1 < steps) stage_wait<(STAGES - 2) * EACH>();
        else stage_wait<0>();
        if (t + STAGES < steps) fetch(cur);
        cur = next(cur);
        if (t + 2 == steps) cut(cur);
        read(h0, place(cur), 0);
      }
      if (mine) {
        multiply(h1);
        add_block();
      }
    }
  }
  stage_wait<0>();

  // the groups' sums, in their order
  constexpr int MEET = (KG - 1) * BM * BN * 4;
  if constexpr (KG > 1) {
    const auto sums_of = [&](int group) {
      return reinterpret_cast<f32x4*>(linear_lds + ((group - 1) * WAVES + wave) * (TM * TN * 4)) + lane;
    };
    if (kg > 0) {
      f32x4* const p = sums_of(kg);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            p[((i * FN + j) * 4 + q) * 64] =
                f32x4{acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int o = 1; o < KG; ++o) {
      const f32x4* const p = sums_of(o);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x4 v = p[((i * FN + j) * 4 + q) * 64];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][q * 4 + e] += v[e];
          }
    }
  }

  // Each wave turns its results through LDS of its own, 32 rows at a time, into runs of eight along n: the lanes of a row
  // then read and write whole cache lines.  16 bytes c of a row lie at (c / 2, odd ones in the second half) xor row.
  constexpr int CH = TN / 4, RUNS = TN / kVec, ROWS = 64 / RUNS, PASSES = 32 / ROWS;
  static_assert(MEET + WAVES * 32 * TN * 4 <= STAGES * KG * STAGE && 32 % ROWS == 0);
  char* const turn = linear_lds + MEET + wave * (32 * TN * 4);
  const auto slot = [](int row, int c) { return (row * CH + (((c >> 1) | (c & 1) * (CH / 2)) ^ (row & (CH - 1)))) * 16; };
  const int64_t n = n0 + wn * TN + lane % RUNS * kVec;
  float bias[kVec];
  read_bias<E>(g, n, bias);
  if (g.partial != nullptr) g.partial += (int64_t)at.split * g.m * g.n;
  const bool inner = m0 + BM <= g.m && n0 + BN <= g.n;  // no result outside D
#pragma unroll
  for (int i = 0; i < FM; ++i) {
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(turn + slot(lane & 31, j * 8 + q * 2 + (lane >> 5))) =
            f32x4{acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
    const int r = lane / RUNS;
    const int64_t m = m0 + wm * TM + i * 32 + r;
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
        finish_rows<E, BATCH>(g, m + h * ROWS, ROWS, n, bias, [&](int p, float* z) { take((h + p) * ROWS + r, z); });
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

template <class E, int BM, int BN, int WM, int WN, int STAGES, int KG>
__global__ void __launch_bounds__(WM * WN * KG * 64) __attribute__((amdgpu_waves_per_eu(2)))
    linear_fp8_kernel(Gemm8Args args) {
  linear_fp8_tile<E, BM, BN, WM, WN, STAGES, KG>(args, (int)blockIdx.x);
}

template <class E, int BM, int BN, int WM, int WN, int STAGES, int KG = 1>
hipError_t linear_fp8_launch(const Gemm8Args& args, hipStream_t stream) {
  constexpr int lds = Fp8Tile<E, BM, BN, WM, WN, STAGES, KG>::LDS;
  const auto kernel = linear_fp8_kernel<E, BM, BN, WM, WN, STAGES, KG>;
  static const hipError_t ready = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                      hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (ready != hipSuccess) return ready;
  Gemm8Args t = args;
  t.g.tiles_m = (int)((args.g.m + BM - 1) / BM);
  t.g.tiles_n = (int)((args.g.n + BN - 1) / BN);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(t.g.tiles_m * t.g.tiles_n * t.g.splits)), dim3(WM * WN * KG * 64), lds, stream, t);
  return hipGetLastError();
}

// Two products in one launch, neither with its k split: where each alone leaves CUs idle they fill each other's rounds.
// The first workgroups take the tiles of the first.
template <class E, int BM, int BN, int WM, int WN, int STAGES>
__global__ void __launch_bounds__(WM * WN * 64) __attribute__((amdgpu_waves_per_eu(2)))
    linear_fp8_pair_kernel(Gemm8Args first, Gemm8Args second) {
  const int id = (int)blockIdx.x, tiles = first.g.tiles_m * first.g.tiles_n;
  // (the same code for both: they differ in their arguments alone)
  linear_fp8_tile<E, BM, BN, WM, WN, STAGES, 1>(id < tiles ? first : second, id < tiles ? id : id - tiles);
}

template <class E, int BM, int BN, int WM, int WN, int STAGES>
hipError_t linear_fp8_pair_launch(const Gemm8Args& first, const Gemm8Args& second, hipStream_t stream) {
  constexpr int lds = Fp8Tile<E, BM, BN, WM, WN, STAGES, 1>::LDS;
  const auto kernel = linear_fp8_pair_kernel<E, BM, BN, WM, WN, STAGES>;
  static const hipError_t ready = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                      hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (ready != hipSuccess) return ready;
  Gemm8Args t[2] = {first, second};
  for (Gemm8Args& p : t) {
    p.g.tiles_m = (int)((p.g.m + BM - 1) / BM);
    p.g.tiles_n = (int)((p.g.n + BN - 1) / BN);
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)(t[0].g.tiles_m * t[0].g.tiles_n + t[1].g.tiles_m * t[1].g.tiles_n)),
                     dim3(WM * WN * 64), lds, stream, t[0], t[1]);
  return hipGetLastError();
}

// ----------------------------------------------------------------------------------
// Few rows of A (at most 16 MT): bound by reading B once.  A workgroup takes 16 NT of B's rows, each of its waves a range of
// k, which it streams through LDS of its own without a barrier; the waves' sums meet in LDS.  Scales come for sixteen
// stages at a time.  One row of 4096 x 4096 4.5 us (16.8 MB that the Infinity Cache holds: 3.7 TB/s), of 8192 x 8192 13.0 us
// (5.2 TB/s); 61 rows of 1024 -> 4096 3.8.  Four stages, and one workgroup to a CU, took 4.53 and 13.6.
// of a wave: [4 groups][64 rows of B, then of A] dwords
constexpr int few_scale_bytes() { return 4 * 128 * 4; }

template <class E, int MT, int NT, int WAVES, int STAGES>
__global__ void __launch_bounds__(WAVES * 64) __attribute__((amdgpu_waves_per_eu(2))) linear_fp8_few_kernel(Gemm8Args args) {
  const GemmArgs& g = args.g;
  constexpr bool WIDE = E::kId == kStorageF32;
  constexpr int BK = kStageBytes, STAGE = 16 * (MT + NT) * kStageBytes;
  constexpr int PRIVATE = STAGES * STAGE + few_scale_bytes();
  static_assert(STAGES * STAGE >= NT * MT * 1024);
  extern __shared__ __attribute__((aligned(1024))) char linear_lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
  char* const mine = linear_lds + wave * PRIVATE;
  const int64_t n0 = (int64_t)blockIdx.x * (16 * NT);
  f32x4 acc[NT][MT];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t stages = (g.k + BK - 1) / BK, per = (stages + WAVES - 1) / WAVES * BK;
  const int64_t k0 = min(wave * per, g.k), k1 = min(k0 + per, g.k);

  CodeOperand<16 * NT, 1, 16> w;
  CodeOperand<16 * MT, 1, 16> x;
  w.init(args.b, n0, g.n, k0, k1, 0, lane);
  x.init(args.a, 0, g.m, k0, k1, 0, lane);
  Fragments<ElemCode, 16, false> f;
  f.init(0, lane);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine;
  const int steps = (int)((k1 - k0 + BK - 1) / BK), s0 = (int)(k0 / BK), tail = (int)((k1 - k0) % BK);
  const int groups = (int)((k1 + 4 * BK - 1) / (4 * BK));
  constexpr int EACH = w.LINES + x.LINES;
  const auto fetch = [&](int slot) {
    w.fetch(lds0 + (uint32_t)slot * STAGE);
    x.fetch(lds0 + (uint32_t)slot * STAGE + w.BYTES);
  };
  // the scales of the sixteen stages that stage s is one of
  const auto fetch_all = [&](int s) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int group = (s >> 4) * 4 + q;
      if (group >= groups) break;
      const uint32_t to = lds0 + STAGES * STAGE + (uint32_t)q * 512u;
      fetch_scales(args.b, n0, min(n0 + 16 * NT, g.n), 0, group, to, lane);
      fetch_scales(args.a, 0, g.m, 0, group, to + 256u, lane);
    }
  };
  // as above: of the rows that a lane holds, or of those that its results belong to
  constexpr int SBS = WIDE ? 4 : 1;
  uint32_t sw[NT][SBS], sx[MT];
  if (steps > 0) fetch_all(s0);
#pragma unroll
  for (int q = 0; q < STAGES; ++q)
    if (q < steps) fetch(q);
  int slot = 0;
  for (int t = 0; t < steps; ++t) {
    const int s = s0 + t;
    if (t > 0 && (s & 15) == 0) {
      reads_wait();
      fetch_all(s);
      loads_wait<0>();
    }
    if (t + STAGES <= steps) loads_wait<(STAGES - 1) * EACH>();
    else loads_wait<0>();
    if (t == 0 || (s & 3) == 0) {
      const uint32_t* const p = reinterpret_cast<const uint32_t*>(mine + STAGES * STAGE + (s >> 2 & 3) * 512);
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < SBS; ++e) sw[j][e] = p[j * 16 + (WIDE ? (lane >> 4) * 4 + e : lane & 15)] >> ((s & 3) * 8);
#pragma unroll
      for (int i = 0; i < MT; ++i) sx[i] = p[64 + i * 16 + (lane & 15)] >> ((s & 3) * 8);
    } else {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < SBS; ++e) sw[j][e] >>= 8;
#pragma unroll
      for (int i = 0; i < MT; ++i) sx[i] >>= 8;
    }
    char* const at = mine + slot * STAGE;
    if (t + 1 == steps && tail % 16 != 0) {
      cut_stage<16>(at, 16 * (MT + NT), tail, lane, 64);
      reads_wait();
    }
    i32x8 vw[NT], vx[MT];
#pragma unroll
    for (int j = 0; j < NT; ++j) vw[j] = join_chunks(f.read(at, j, 0), f.read(at, j, 1));
#pragma unroll
    for (int i = 0; i < MT; ++i) vx[i] = join_chunks(f.read(at + w.BYTES, i, 0), f.read(at + w.BYTES, i, 1));
    if (t + STAGES < steps) {
      reads_wait();
      fetch(slot);
    }
    slot = slot + 1 == STAGES ? 0 : slot + 1;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        if constexpr (WIDE) {
          const f32x4 block = product16_wide(vw[j], vx[i]);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[j][i][e] += scaled_or_nan(block[e], (int)(sx[i] & 255), (int)(sw[j][e] & 255));
        } else {
          acc[j][i] = product16(vw[j], vx[i], acc[j][i], sw[j][0], sx[i]);
        }
      }
  }
  reads_wait();
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i) reinterpret_cast<f32x4*>(mine)[(j * MT + i) * 64 + lane] = acc[j][i];
  __syncthreads();
  // eight results of one row of A to a thread, groups of a row side by side
  constexpr int UNITS = MT * 16 * NT * 2;
  static_assert(UNITS <= WAVES * 64);
  const int unit = threadIdx.x;
  if (unit >= UNITS) return;
  const int q = unit % (NT * 2), m = unit / (NT * 2);
  const int at = (q / 2 * MT + m / 16) * 64 + (q & 1) * 32 + (m & 15);
  float z[kVec] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, bias[kVec];
  read_bias<E>(g, n0 + q * kVec, bias);
#pragma unroll
  for (int v = 0; v < WAVES; ++v) {
    const f32x4* const part = reinterpret_cast<const f32x4*>(linear_lds + v * PRIVATE);
    const f32x4 lo = part[at], hi = part[at + 16];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      z[e] += lo[e];
      z[4 + e] += hi[e];
    }
  }
  finish_group<E>(g, m, n0 + q * kVec, bias, z);
}

template <class E, int MT, int NT, int WAVES, int STAGES>
hipError_t few_fp8_launch(const Gemm8Args& args, hipStream_t stream) {
  constexpr int lds = WAVES * (STAGES * 16 * (MT + NT) * kStageBytes + few_scale_bytes());
  static_assert(lds <= 160 * 1024);
  const auto kernel = linear_fp8_few_kernel<E, MT, NT, WAVES, STAGES>;
  static const hipError_t ready = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                      hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (ready != hipSuccess) return ready;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((args.g.n + 16 * NT - 1) / (16 * NT))), dim3(WAVES * 64), lds, stream, args);
  return hipGetLastError();
}

template <class E>
Linear8Table make_linear_fp8_table() {
  Linear8Table t{};
  t.fn[kTile8_32x64] = linear_fp8_launch<E, 32, 64, 1, 2, 3>;
  t.fn[kTile8_64] = linear_fp8_launch<E, 64, 64, 2, 2, 3>;
  t.fn[kTile8_64x128] = linear_fp8_launch<E, 64, 128, 2, 2, 3>;
  t.fn[kTile8_32x64K4] = linear_fp8_launch<E, 32, 64, 1, 2, 2, 4>;
  t.fn[kTile8_64x128K2] = linear_fp8_launch<E, 64, 128, 2, 2, 2, 2>;
  t.pair[kTile8_64] = linear_fp8_pair_launch<E, 64, 64, 2, 2, 3>;
  t.pair[kTile8_64x128] = linear_fp8_pair_launch<E, 64, 128, 2, 2, 3>;
  // (the wide form needs registers for a block's sums and scales)
  if constexpr (E::kId != kStorageF32) {
    t.fn[kTile8_128] = linear_fp8_launch<E, 128, 128, 2, 2, 2>;
    t.fn[kTile8_128K2] = linear_fp8_launch<E, 128, 128, 2, 2, 2, 2>;
    t.fn[kTile8_128x256] = linear_fp8_launch<E, 128, 256, 2, 4, 3>;
    t.fn[kTile8_256] = linear_fp8_launch<E, 256, 256, 2, 4, 2>;
    t.pair[kTile8_128] = linear_fp8_pair_launch<E, 128, 128, 2, 2, 2>;
  }
  t.few[0][0] = few_fp8_launch<E, 1, 1, 8, 2>;
  t.few[0][1] = few_fp8_launch<E, 1, 2, 8, 2>;
  t.few[1][0] = few_fp8_launch<E, 2, 1, 4, 6>;
  t.few[1][1] = few_fp8_launch<E, 2, 2, 4, 4>;
  t.few[2][0] = few_fp8_launch<E, 4, 1, 4, 3>;
  t.few[2][1] = few_fp8_launch<E, 4, 2, 4, 3>;
  return t;
}

}  // namespace rdfft
