// linear.hip -- the dense product y = act(x W^T + b) + r and its gradients: which kernel of
// linear_kernels.hpp runs, in how many parts, and the two passes beside it, the join of a
// product whose k is split and the gradient through the activation with its column sums.
#include <hip/hip_runtime.h>

#include <cmath>

#include "linear_kernels.hpp"

namespace rdfft {

// The plans count on this many CUs (an MI355X has them all; fewer only take longer), so that a
// workspace's size follows from the sizes of a call alone.
constexpr int64_t kCUs = 256;

// ----------------------------------------------------------------------------------
// the join of a split product: one thread sums eight columns over the splits
constexpr int kJoinWG = 256;
template <class E>
__global__ void __launch_bounds__(kJoinWG) linear_join_kernel(GemmArgs g, const float* __restrict__ partial, int lanes) {
  const int64_t m = (int64_t)blockIdx.y * (kJoinWG / lanes) + threadIdx.x / lanes;
  const int64_t n = ((int64_t)blockIdx.x * lanes + threadIdx.x % lanes) * kVec;
  float z[kVec] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, bias[kVec];
  read_bias<E>(g, n, bias);
  if (m < g.m && n < g.n) {
#pragma unroll 4
    for (int s = 0; s < g.splits; ++s) {
      float v[kVec];
      read_group<ElemF32>(partial + ((int64_t)s * g.m + m) * g.n, n, g.n, v);
#pragma unroll
      for (int i = 0; i < kVec; ++i) z[i] += v[i];
    }
  }
  finish_group<E>(g, m, n, bias, z);
}

hipError_t launch_linear_join(GemmArgs g, int storage, hipStream_t stream) {
  const float* const partial = g.partial;
  g.partial = nullptr;
  int lanes = kCkLanes;
  const int64_t groups = (g.n + kCkBlock - 1) / kCkBlock * kCkLanes;
  while (lanes < kJoinWG && lanes < groups) lanes *= 2;
  const int64_t per = kJoinWG / lanes, gx = (groups + lanes - 1) / lanes;
  constexpr int64_t kMaxY = 65535;
  const int64_t gy = (g.m + per - 1) / per;
  if (gy > kMaxY) return hipErrorInvalidValue;  // (a product of so many rows is never split)
  return with_elem(storage, [&](auto e) {
    hipLaunchKernelGGL(linear_join_kernel<decltype(e)>, dim3((unsigned)gx, (unsigned)gy), dim3(kJoinWG), 0, stream, g, partial,
                       lanes);
    return hipGetLastError();
  });
}

// ----------------------------------------------------------------------------------
// dz = dy act'(z), z from its checkpoint, rounded once to the storage type (it is a matrix operand), in rows
// of slope_pitch values, so that it is loaded like an aligned operand whatever d_out; and the column sums
// of the unrounded dz.  A workgroup takes a strip of 512 columns, its four waves every fourth row of its
// range; partials[blockIdx.y][n] receive the sums, or db where there is one range.
// 8192 x 8192 bf16: 72 to 78 us (346 MB, 4.4 to 4.8 TB/s), 4096 x 768: 8.8 us.
constexpr int kSlopeWG = 256, kSlopeWaves = 4, kSlopeStrip = 64 * kVec, kSlopeAhead = 4;
constexpr int64_t kSlopeMaxParts = 256;

template <class E, bool EXACT>
__global__ void __launch_bounds__(kSlopeWG)
    linear_slope_kernel(const typename E::T* __restrict__ dy, int64_t ldg, Checkpoint ck, typename E::T* __restrict__ dz,
                        int64_t ldz, float* __restrict__ partials, typename E::T* __restrict__ db, int rows, int per, int n,
                        int act) {
  __shared__ float sums[kSlopeWaves][kSlopeStrip];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  const int i = blockIdx.x * kSlopeStrip + lane * kVec;
  const int blocks = (n + kCkBlock - 1) / kCkBlock;
  const int r0 = blockIdx.y * per + wave, r1 = min(rows, (int)(blockIdx.y + 1) * per);
  float s[kVec] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (i < n) {
    const auto row = [&](int r, float* g, const Bytes8& code, int byte) {
      if (act != kActNone) {
        float z[kVec];
        ck_decode<ElemF32>(code, ck_scale(byte), z);
        times_slope8(act, z, g);
        E::store(dz + r * ldz + i, g);  // (rows are padded to whole groups, with zeros)
      }
#pragma unroll
      for (int k = 0; k < kVec; ++k) s[k] += g[k];
    };
    int r = r0;
    if constexpr (EXACT) {
      // several rows under way at once
      for (; r + (kSlopeAhead - 1) * kSlopeWaves < r1; r += kSlopeAhead * kSlopeWaves) {
        typename E::Raw raw[kSlopeAhead];
        Bytes8 code[kSlopeAhead];
        int byte[kSlopeAhead];
#pragma unroll
        for (int u = 0; u < kSlopeAhead; ++u) raw[u] = E::load(dy + (int64_t)(r + u * kSlopeWaves) * ldg + i);
        if (act != kActNone) {
#pragma unroll
          for (int u = 0; u < kSlopeAhead; ++u) {
            code[u] = *reinterpret_cast<const Bytes8*>(ck.codes + (int64_t)(r + u * kSlopeWaves) * n + i);
            byte[u] = ck.scales[(int64_t)(r + u * kSlopeWaves) * blocks + i / kCkBlock];
          }
        }
#pragma unroll
        for (int u = 0; u < kSlopeAhead; ++u) {
          float g[kVec];
          E::widen(raw[u], g);
          row(r + u * kSlopeWaves, g, code[u], byte[u]);
        }
      }
    }
#pragma unroll 1
    for (; r < r1; r += kSlopeWaves) {
      float g[kVec];
      Bytes8 code = {{0, 0}};
      int byte = 0;
      read_group<E>(dy + (int64_t)r * ldg, i, n, g);
      if (act != kActNone) {
        code = tail_codes(ck.codes + (int64_t)r * n, i, n);
        byte = ck.scales[(int64_t)r * blocks + i / kCkBlock];
      }
      row(r, g, code, byte);
    }
  }
  if (partials == nullptr && db == nullptr) return;
#pragma unroll
  for (int k = 0; k < kVec; ++k) sums[wave][k * 64 + lane] = s[k];
  __syncthreads();
  for (int c = threadIdx.x; c < kSlopeStrip; c += kSlopeWG) {
    const int col = blockIdx.x * kSlopeStrip + c;
    if (col >= n) break;
    const int at = c % kVec * 64 + c / kVec;
    float v = sums[0][at];
#pragma unroll
    for (int w = 1; w < kSlopeWaves; ++w) v += sums[w][at];
    if (db != nullptr) E::put(db + col, v);
    else partials[(int64_t)blockIdx.y * n + col] = v;
  }
}

static int64_t slope_pitch(int64_t n) { return (n + kVec - 1) / kVec * kVec; }

// row ranges that fill the chip's wave slots (eight workgroups a CU), of sixteen rows at least
static int64_t slope_parts(int64_t rows, int64_t n) {
  const int64_t strips = (n + kSlopeStrip - 1) / kSlopeStrip;
  return std::max<int64_t>(1, std::min({(kCUs * 8 + strips - 1) / strips, (rows + 15) / 16, kSlopeMaxParts}));
}

// ----------------------------------------------------------------------------------
// plans

// What a tile costs, in us, fitted to products of 128 to 8192: a stage (128 bytes of k) where a CU has one workgroup
// of them, a stage of each where it has more (`together` fit), and what comes before and after.  16-bit values: the largest
// tile is the fastest where its tiles fill the chip in whole rounds (1390 TFLOP/s); the smaller ones leave fewer CUs idle.
// Unsplit, in the kernel, averages in turn: 4096 x 768 x 768 (12 stages) 11.6 us in tiles of 128, 12.0 in 64, 15.4 in
// 32 x 64, 15.6 and 22.9 in the larger two; 2045 x 4096 x 4096 59 us in 128 x 256, 64, 88 and 97 in 128, 256 and 64;
// 128 x 4096 x 4096 17 us in 32 x 64, 18 in 64, 40 in 128.  float32: 4096 x 4096 x 4096 1013 us in 64, 1055 in 32 x 64;
// 300 x 768 x 768 11.4 us in 32 x 64, 16.7 in 64.
struct TileCost {
  int bm, bn, together;
  double alone, each, ends;
};
constexpr TileCost kCost16[kLinearTiles] = {{32, 64, 4, 0.19, 0.14, 3.4},   {64, 64, 3, 0.235, 0.175, 3.6},
                                            {128, 128, 2, 0.50, 0.445, 4.0}, {128, 256, 1, 0.82, 0.82, 4.8},
                                            {256, 256, 1, 1.30, 1.30, 13.0}};
constexpr TileCost kCost32[] = {{32, 64, 4, 0.285, 0.256, 3.6}, {64, 64, 3, 0.53, 0.50, 4.0}};

struct Plan {
  LinearTile tile;
  int64_t splits, k_split;
  double cost;
};

// The tile and the number of k ranges that cost least.  The join of s ranges costs a launch (4 us) and 8 s bytes a
// result, at 4 TB/s.
static Plan plan_of(int64_t m, int64_t n, int64_t k, LinearOperands kind, int storage, bool direct) {
  const bool f32 = storage == kStorageF32;
  const int64_t bk = kStageBytes / (f32 ? 4 : 2), stages = std::max<int64_t>(1, (k + bk - 1) / bk);
  Plan best{kTile64, 1, stages * bk, 0};
  for (int t = 0; t < kLinearTiles; ++t) {
    // what is not built
    if (f32 ? t > kTile64 : !direct && (t == kTile32x64 || t == kTile256)) continue;
    if (kind == kGradW && (t == kTile32x64 || (!direct && t == kTile128x256))) continue;
    const TileCost& c = f32 ? kCost32[t] : kCost16[t];
    const int64_t tiles = ((m + c.bm - 1) / c.bm) * ((n + c.bn - 1) / c.bn);
    for (int64_t want = 1; want <= 16; ++want) {
      const int64_t each = (stages + want - 1) / want, splits = (stages + each - 1) / each;
      if (splits != want) continue;  // (as many ranges of another length)
      if (splits > 1 && (each < 2 || tiles * splits > 4 * kCUs)) break;
      const int64_t per_cu = std::max<int64_t>(1, (tiles * splits + kCUs - 1) / kCUs);
      const double stage = per_cu == 1 ? c.alone : c.each * (double)per_cu;
      double cost = (double)each * stage + c.ends * (double)((per_cu + c.together - 1) / c.together);
      if (splits > 1) cost += 4.0 + 8.0 * (double)splits * (double)m * (double)n / 4e6;
      if (best.cost == 0 || cost < best.cost) best = {(LinearTile)t, splits, each * bk, cost};
    }
  }
  return best;
}
// (whether rows are aligned is not known here: the larger of both plans' needs)
static int64_t split_bytes(int64_t m, int64_t n, int64_t k, LinearOperands kind, int storage) {
  int64_t most = 0;
  for (const bool direct : {false, true}) {
    const Plan p = plan_of(m, n, k, kind, storage, direct);
    if (p.splits > 1) most = std::max(most, p.splits * m * n * 4);
  }
  return most;
}

static int64_t round_up(int64_t bytes) { return (bytes + 255) & ~(int64_t)255; }
static int storage_bytes(int storage) { return storage == kStorageF32 ? 4 : 2; }

int64_t linear_forward_workspace(const LinearSizes& s) {
  return s.tokens <= kFewTokens ? 0 : split_bytes(s.tokens, s.d_out, s.d_in, kForward, s.storage);
}

// dz, then the partial sums of whichever pass runs (they follow each other on the stream)
static int64_t slope_bytes(const LinearSizes& s) {
  return s.act == kActNone ? 0 : round_up(s.tokens * slope_pitch(s.d_out) * storage_bytes(s.storage));
}
int64_t linear_backward_workspace(const LinearSizes& s, bool dx, bool dw, bool db) {
  int64_t parts = 0;
  if (db && slope_parts(s.tokens, s.d_out) > 1) parts = std::max(parts, slope_parts(s.tokens, s.d_out) * s.d_out * 4);
  if (dx) parts = std::max(parts, split_bytes(s.tokens, s.d_in, s.d_out, kGradX, s.storage));
  if (dw) parts = std::max(parts, split_bytes(s.d_out, s.d_in, s.tokens, kGradW, s.storage));
  return slope_bytes(s) + parts;
}

// Whether an operand's memory rows of `len` values hold whole chunks of 16 bytes and, of 16-bit values, start at
// multiples of 16 bytes (floats may start anywhere).
static bool whole_chunks(const void* p, int64_t ld, int64_t len, int storage) {
  if (storage == kStorageF32) return len % 4 == 0;
  return (reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * 2) | (uintptr_t)(len * 2)) % 16 == 0;
}

static const LinearTable& table_of(int storage) {
  static const LinearTable tables[] = {linear_table_f32(), linear_table_bf16(), linear_table_f16()};
  return tables[storage];
}

// a_len: values in a memory row of A that may be loaded (those past its end are zeros)
static bool whole_operands(const GemmArgs& g, int64_t a_len, LinearOperands kind, int storage) {
  return whole_chunks(g.a, g.lda, a_len, storage) && whole_chunks(g.b, g.ldb, kind == kForward ? g.k : g.n, storage);
}

static hipError_t product(GemmArgs& g, int64_t a_len, LinearOperands kind, int storage, void* workspace,
                          hipStream_t stream) {
  const LinearTable& t = table_of(storage);
  const bool direct = whole_operands(g, a_len, kind, storage);
  g.splits = 1;
  if (kind == kForward && g.m <= kFewTokens) {
    // 32 rows of W to a workgroup where that still fills the chip (x is read half as often: 64 tokens of 8192 x 8192
    // 22.8 us, else 31.3) or a checkpoint's blocks ask for it; 16 otherwise (one token of 4096 x 4096 5.9 us, else 7.2)
    const bool wide = g.ck.codes != nullptr || g.n >= 32 * kCUs;
    return t.few[g.m <= 16 ? 0 : g.m <= 32 ? 1 : 2][wide][direct](g, stream);
  }
  const Plan p = plan_of(g.m, g.n, g.k, kind, storage, direct);
  g.splits = (int)p.splits;
  g.k_split = p.k_split;
  g.partial = p.splits > 1 ? static_cast<float*>(workspace) : nullptr;
  const hipError_t e = t.fn[p.tile][kind][direct](g, stream);
  if (e != hipSuccess || g.partial == nullptr) return e;
  return launch_linear_join(g, storage, stream);
}

// Which tile dW and dx share in one launch, or kLinearTiles where two launches cost less.  The product with the longer k
// goes first.  Where it has a workgroup for every CU the rounds are simply full; where it has fewer, its CUs deal
// part of their time to the other's tiles until those run out, and finish alone.  Its times are good to about 8 % for most
// sizes, so one launch has to take that much less.
// One launch and two, us in the kernels (tokens x d_in x d_out): 1021 x 1024 x 768 float32 35.7 and 42.7; bf16 512 x 768 x
// 768 6.8 and 11.5, 2045 x 2048 x 2048 38.9 and 54.9, 4096 x 768 x 2560 44.1 and 64.7.  Two stay: 2048 x 4096 x 4096 (123
// and 124), 8192 x 768 x 768 (40.7 and 40.2, its dW's k split), and 4096 x 768 x 768, where the model is wrong (23.5 and 30.2).
static LinearTile together_of(const GemmArgs& dw, const GemmArgs& dx, int storage) {
  const bool f32 = storage == kStorageF32;
  const int64_t bk = kStageBytes / (f32 ? 4 : 2);
  LinearTile best = kLinearTiles;
  double least = 0.92 * (plan_of(dw.m, dw.n, dw.k, kGradW, storage, true).cost +
                         plan_of(dx.m, dx.n, dx.k, kGradX, storage, true).cost);
  const GemmArgs& first = dw.k >= dx.k ? dw : dx;
  const GemmArgs& second = dw.k >= dx.k ? dx : dw;
  const double cus = (double)kCUs, k1 = (double)((first.k + bk - 1) / bk), k2 = (double)((second.k + bk - 1) / bk);
  for (const LinearTile t : {kTile64, kTile128}) {
    if (table_of(storage).grads[t] == nullptr) continue;
    const TileCost& c = f32 ? kCost32[t] : kCost16[t];
    const auto tiles = [&](const GemmArgs& g) { return (double)((g.m + c.bm - 1) / c.bm * ((g.n + c.bn - 1) / c.bn)); };
    const double n1 = tiles(first), n2 = tiles(second), per_cu = std::ceil((n1 + n2) / cus);
    const double full = (n1 * k1 + n2 * k2) / cus * c.each;
    double cost = std::max(full, k1 * c.alone);
    if (n1 < cus && per_cu > 1) {
      const double share = 1 / std::min((double)c.together, per_cu);  // of such a CU that the longer k has
      const double until = n2 * k2 / cus * c.each / (1 - n1 / cus * share);
      cost = std::max(full, until + std::max(0.0, k1 - until * share / c.each) * c.alone);
    }
    cost += c.ends * std::ceil(per_cu / c.together);
    if (cost < least) {
      least = cost;
      best = t;
    }
  }
  return best;
}

hipError_t launch_linear_forward(const LinearForward& a, hipStream_t stream) {
  GemmArgs g{};
  g.a = a.x;
  g.lda = a.ldx;
  g.b = a.w;
  g.ldb = a.ldw;
  g.m = a.s.tokens;
  g.n = a.s.d_out;
  g.k = a.s.d_in;
  g.d = a.y;
  g.ldd = a.ldy;
  g.bias = a.bias;
  g.residual = a.residual;
  g.ldr = a.ldr;
  g.ck = a.ck;
  g.act = a.s.act;
  return product(g, g.k, kForward, a.s.storage, a.workspace, stream);
}

hipError_t launch_linear_backward(const LinearBackward& a, hipStream_t stream) {
  const int64_t T = a.s.tokens, n = a.s.d_out;
  const int storage = a.s.storage;
  char* const parts = static_cast<char*>(a.workspace) + slope_bytes(a.s);
  const void* dz = a.dy;
  int64_t ldz = a.ldg, dz_len = n;
  hipError_t e = hipSuccess;
  if (a.s.act != kActNone || a.db != nullptr) {
    const int64_t count = slope_parts(T, n), per = (T + count - 1) / count;
    float* const partials = a.db == nullptr || count == 1 ? nullptr : reinterpret_cast<float*>(parts);
    void* const db = count == 1 ? a.db : nullptr;
    e = with_elem(storage, [&](auto elem) {
      using E = decltype(elem);
      const auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)((n + kSlopeStrip - 1) / kSlopeStrip), (unsigned)count), dim3(kSlopeWG),
                           0, stream, static_cast<const typename E::T*>(a.dy), a.ldg, a.ck,
                           static_cast<typename E::T*>(a.workspace), slope_pitch(n), partials,
                           static_cast<typename E::T*>(db), (int)T, (int)per, (int)n, a.s.act);
        return hipGetLastError();
      };
      return n % kVec == 0 ? go(linear_slope_kernel<E, true>) : go(linear_slope_kernel<E, false>);
    });
    if (e == hipSuccess && partials != nullptr)
      e = launch_column_finish(partials, count, n, n, a.db, nullptr, storage, stream);
    if (e != hipSuccess) return e;
    if (a.s.act != kActNone) {
      dz = a.workspace;
      ldz = dz_len = slope_pitch(n);
    }
  }
  GemmArgs x{}, w{};
  const bool dx = a.dx != nullptr && T > 0, dw = a.dw != nullptr;
  x.a = dz;
  x.lda = ldz;
  x.b = a.w;
  x.ldb = a.ldw;
  x.m = T;
  x.n = a.s.d_in;
  x.k = n;
  x.d = a.dx;
  x.ldd = a.ldd;
  x.residual = a.add;
  x.ldr = a.lda;
  w.a = dz;
  w.lda = ldz;
  w.b = a.x;
  w.ldb = a.ldx;
  w.m = n;
  w.n = a.s.d_in;
  w.k = T;
  w.d = a.dw;
  w.ldd = a.lddw;
  if (dx && dw && whole_operands(x, dz_len, kGradX, storage) && whole_operands(w, dz_len, kGradW, storage)) {
    const LinearTile t = together_of(w, x, storage);
    if (t != kLinearTiles) {
      x.splits = w.splits = 1;
      x.k_split = x.k;
      w.k_split = w.k;
      return table_of(storage).grads[t](w, x, stream);
    }
  }
  if (dx) e = product(x, dz_len, kGradX, storage, parts, stream);
  if (e == hipSuccess && dw) e = product(w, dz_len, kGradW, storage, parts, stream);
  return e;
}

}  // namespace rdfft
