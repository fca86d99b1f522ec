// linear.hip -- the dense product y = act(x W^T + b) + r and its gradients: which kernel of
// linear_kernels.hpp runs, in how many parts, and the two passes beside it, the join of a
// product whose k is split and the gradient through the activation with its column sums.
#include <hip/hip_runtime.h>

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

template <class E>
static hipError_t join(GemmArgs g, hipStream_t stream) {
  const float* const partial = g.partial;
  g.partial = nullptr;
  int lanes = kCkLanes;
  const int64_t groups = (g.n + kCkBlock - 1) / kCkBlock * kCkLanes;
  while (lanes < kJoinWG && lanes < groups) lanes *= 2;
  const int64_t per = kJoinWG / lanes, gx = (groups + lanes - 1) / lanes;
  constexpr int64_t kMaxY = 65535;
  const int64_t gy = (g.m + per - 1) / per;
  if (gy > kMaxY) return hipErrorInvalidValue;  // (a product of so many rows is never split)
  hipLaunchKernelGGL(linear_join_kernel<E>, dim3((unsigned)gx, (unsigned)gy), dim3(kJoinWG), 0, stream, g, partial, lanes);
  return hipGetLastError();
}

// ----------------------------------------------------------------------------------
// dz = dy act'(z), z from its checkpoint, rounded once to the storage type (it is a matrix operand),
// and the column sums of the unrounded dz.  A workgroup takes a strip of 512 columns, its four
// waves every fourth row of its range; partials[blockIdx.y][n] receive the sums.
constexpr int kSlopeWG = 256, kSlopeWaves = 4, kSlopeStrip = 64 * kVec;
constexpr int64_t kSlopeMaxParts = 128;

template <class E>
__global__ void __launch_bounds__(kSlopeWG)
    linear_slope_kernel(const typename E::T* __restrict__ dy, int64_t ldg, Checkpoint ck, typename E::T* __restrict__ dz,
                        float* __restrict__ partials, int64_t rows, int64_t per, int64_t n, int act) {
  __shared__ float sums[kSlopeWaves][kSlopeStrip];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  const int64_t i = (int64_t)blockIdx.x * kSlopeStrip + lane * kVec;
  const int64_t blocks = (n + kCkBlock - 1) / kCkBlock;
  const int64_t r1 = min(rows, (int64_t)(blockIdx.y + 1) * per);
  float s[kVec] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (i < n) {
#pragma unroll 2
    for (int64_t r = (int64_t)blockIdx.y * per + wave; r < r1; r += kSlopeWaves) {
      float g[kVec];
      read_group<E>(dy + r * ldg, i, n, g);
      if (ck.codes != nullptr) {
        const int8_t* const row = ck.codes + r * n;
        const Bytes8 c = i + kVec <= n ? *reinterpret_cast<const Bytes8*>(row + i) : tail_codes(row, i, n);
        float z[kVec];
        ck_decode(c, ck_scale(ck.scales[r * blocks + i / kCkBlock]), z);
#pragma unroll
        for (int k = 0; k < kVec; ++k) g[k] *= activation_slope(act, z[k]);
        write_group<E>(dz + r * n, i, n, g);
      }
#pragma unroll
      for (int k = 0; k < kVec; ++k) s[k] += g[k];
    }
  }
  if (partials == nullptr) return;
#pragma unroll
  for (int k = 0; k < kVec; ++k) sums[wave][k * 64 + lane] = s[k];
  __syncthreads();
  for (int c = threadIdx.x; c < kSlopeStrip; c += kSlopeWG) {
    const int64_t col = (int64_t)blockIdx.x * kSlopeStrip + c;
    if (col >= n) break;
    const int at = c % kVec * 64 + c / kVec;
    float v = sums[0][at];
#pragma unroll
    for (int w = 1; w < kSlopeWaves; ++w) v += sums[w][at];
    partials[blockIdx.y * n + col] = v;
  }
}

// row ranges that fill the chip a few times over, of eight rows at least
static int64_t slope_parts(int64_t rows, int64_t n) {
  const int64_t strips = (n + kSlopeStrip - 1) / kSlopeStrip;
  return std::max<int64_t>(1, std::min({(kCUs * 8 + strips - 1) / strips, (rows + 7) / 8, kSlopeMaxParts}));
}

// ----------------------------------------------------------------------------------
// plans

struct Plan {
  LinearTile tile;
  int64_t splits, k_split;
};

// Tiles of 256 where they fill the chip, else of 128; k is split where even those leave CUs without
// work, into ranges of four stages at least.
static Plan plan_of(int64_t m, int64_t n, int64_t k, int storage) {
  const int64_t bk = kStageBytes / (storage == kStorageF32 ? 4 : 2), stages = (k + bk - 1) / bk;
  const auto tiles = [&](int64_t b) { return ((m + b - 1) / b) * ((n + b - 1) / b); };
  if (storage != kStorageF32 && tiles(256) >= kCUs * 3 / 4) return {kTile256, 1, std::max<int64_t>(k, 1)};
  const int64_t t = std::max<int64_t>(tiles(128), 1);
  int64_t splits = std::max<int64_t>(1, std::min(kCUs * 2 / t, stages / 4));
  const int64_t each = std::max<int64_t>(1, (stages + splits - 1) / splits);
  splits = std::max<int64_t>(1, (stages + each - 1) / each);
  return {kTile128, splits, each * bk};
}
static int64_t split_bytes(int64_t m, int64_t n, int64_t k, int storage) {
  const Plan p = plan_of(m, n, k, storage);
  return p.splits > 1 ? p.splits * m * n * 4 : 0;
}

static int64_t round_up(int64_t bytes) { return (bytes + 255) & ~(int64_t)255; }
static int storage_bytes(int storage) { return storage == kStorageF32 ? 4 : 2; }

int64_t linear_forward_workspace(const LinearSizes& s) { return split_bytes(s.tokens, s.d_out, s.d_in, s.storage); }

// dz, then the partial sums of whichever pass runs (they follow each other on the stream)
static int64_t slope_bytes(const LinearSizes& s) {
  return s.act == kActNone ? 0 : round_up(s.tokens * s.d_out * storage_bytes(s.storage));
}
int64_t linear_backward_workspace(const LinearSizes& s, bool dx, bool dw, bool db) {
  int64_t parts = 0;
  if (db) parts = std::max(parts, slope_parts(s.tokens, s.d_out) * s.d_out * 4);
  if (dx) parts = std::max(parts, split_bytes(s.tokens, s.d_in, s.d_out, s.storage));
  if (dw) parts = std::max(parts, split_bytes(s.d_out, s.d_in, s.tokens, s.storage));
  return slope_bytes(s) + parts;
}

// Whether an operand's memory rows of `len` values start at multiples of 16 bytes and hold whole chunks.
static bool whole_chunks(const void* p, int64_t ld, int64_t len, int storage) {
  const int64_t s = storage_bytes(storage);
  return (reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * s) | (uintptr_t)(len * s)) % 16 == 0;
}

static hipError_t product(GemmArgs& g, LinearOperands kind, int storage, void* workspace, hipStream_t stream) {
  static const LinearTable tables[] = {linear_table_f32(), linear_table_bf16(), linear_table_f16()};
  const Plan p = plan_of(g.m, g.n, g.k, storage);
  g.splits = (int)p.splits;
  g.k_split = p.k_split;
  g.partial = p.splits > 1 ? static_cast<float*>(workspace) : nullptr;
  const bool direct = whole_chunks(g.a, g.lda, kind == kGradW ? g.m : g.k, storage) &&
                      whole_chunks(g.b, g.ldb, kind == kForward ? g.k : g.n, storage);
  const LinearTable& t = tables[storage];
  LinearFn fn = t.fn[p.tile][kind][direct];
  if (fn == nullptr) fn = t.fn[kTile128][kind][direct];
  const hipError_t e = fn(g, stream);
  if (e != hipSuccess || g.partial == nullptr) return e;
  return with_elem(storage, [&](auto elem) { return join<decltype(elem)>(g, stream); });
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
  return product(g, kForward, a.s.storage, a.workspace, stream);
}

hipError_t launch_linear_backward(const LinearBackward& a, hipStream_t stream) {
  const int64_t T = a.s.tokens, n = a.s.d_out;
  const int storage = a.s.storage;
  char* const parts = static_cast<char*>(a.workspace) + slope_bytes(a.s);
  const void* dz = a.dy;
  int64_t ldz = a.ldg;
  hipError_t e = hipSuccess;
  if (a.s.act != kActNone || a.db != nullptr) {
    const int64_t count = slope_parts(T, n), per = (T + count - 1) / count;
    float* const partials = a.db == nullptr ? nullptr : reinterpret_cast<float*>(parts);
    e = with_elem(storage, [&](auto elem) {
      using E = decltype(elem);
      hipLaunchKernelGGL(linear_slope_kernel<E>, dim3((unsigned)((n + kSlopeStrip - 1) / kSlopeStrip), (unsigned)count),
                         dim3(kSlopeWG), 0, stream, static_cast<const typename E::T*>(a.dy), a.ldg,
                         a.s.act == kActNone ? Checkpoint{} : a.ck, static_cast<typename E::T*>(a.workspace), partials, T,
                         per, n, a.s.act);
      return hipGetLastError();
    });
    if (e == hipSuccess && a.db != nullptr)
      e = launch_column_finish(partials, count, n, n, a.db, nullptr, storage, stream);
    if (e != hipSuccess) return e;
    if (a.s.act != kActNone) {
      dz = a.workspace;
      ldz = n;
    }
  }
  if (a.dx != nullptr && T > 0) {
    GemmArgs g{};
    g.a = dz;
    g.lda = ldz;
    g.b = a.w;
    g.ldb = a.ldw;
    g.m = T;
    g.n = a.s.d_in;
    g.k = n;
    g.d = a.dx;
    g.ldd = a.ldd;
    g.residual = a.add;
    g.ldr = a.lda;
    e = product(g, kGradX, storage, parts, stream);
    if (e != hipSuccess) return e;
  }
  if (a.dw != nullptr) {
    GemmArgs g{};
    g.a = dz;
    g.lda = ldz;
    g.b = a.x;
    g.ldb = a.ldx;
    g.m = n;
    g.n = a.s.d_in;
    g.k = T;
    g.d = a.dw;
    g.ldd = a.lddw;
    e = product(g, kGradW, storage, parts, stream);
  }
  return e;
}

}  // namespace rdfft
