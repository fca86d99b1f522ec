// linear_fp8.hip -- the dense product of operands in 8-bit floating point and its gradients: which kernel of
// linear_fp8_kernels.hpp runs, in how many parts, and the order of a backward's passes.
//
// All three products are one kernel, because each operand comes in blocks along its own k: y = x W^T takes the rows of
// x and W, dx = dz W the rows of dz and the columns of W, dW = dz^T x the columns of dz and x.
#include <hip/hip_runtime.h>

#include <cmath>

#include "fp8_launch.hpp"

namespace rdfft {

// the plans count on this many CUs, so that a workspace's size follows from the sizes of a call alone
constexpr int64_t kCUs = 256;
constexpr int64_t kStage = 128;  // k to a stage

// What a tile costs, in us, fitted to products of 100 to 8192: a stage where a CU has one workgroup of them, a stage of
// each where it has more (`together` fit), and what comes before and after.  The largest tile is the fastest where its tiles
// fill the chip in whole rounds; the smaller ones leave fewer CUs idle; groups of waves with stages of their own
// shorten the way through k where a CU has one workgroup.  In the call (us): 8192 x 8192 -> 4096 199 in 256, 220 in 128 x 256,
// 240 in 128; 2045 x 4096 -> 4096 34 in 128 x 256, 36 in 128; 1021 x 4096 -> 4096 22.8 in 128 of two groups, 25.9 in 128, 23.4 in
// 64 x 128; 300 x 4096 -> 4096 13.2 in 64 x 128 of two groups, 14.3 of one; 128 x 4096 -> 4096 8.6 in 32 x 64 of four groups, 10.6
// of one; 4093 x 768 -> 768 9.0 in 64, 13.0 in 32 x 64.  float32 results: 4096 x 2048 -> 2048 56 in 64 x 128, 63 in 64.
struct TileCost {
  int log_m, log_n, together;
  double alone, each, ends;
  int bm = 1 << log_m, bn = 1 << log_n;
};
constexpr TileCost kCost16[kLinear8Tiles] = {{5, 6, 4, 0.20, 0.13, 1.6},   {6, 6, 3, 0.205, 0.18, 1.8},
                                             {6, 7, 2, 0.26, 0.29, 2.5},  {5, 6, 1, 0.12, 0.19, 2.0},
                                             {6, 7, 1, 0.235, 0.35, 2.8}, {7, 7, 2, 0.60, 0.48, 3.5},
                                             {7, 7, 1, 0.50, 0.58, 3.8}, {7, 8, 1, 0.77, 0.77, 4.9},
                                             {8, 8, 1, 1.42, 1.42, 7.2}};
// float32 results
constexpr TileCost kCost32[] = {{5, 6, 4, 0.50, 0.31, 2.0}, {6, 6, 3, 0.60, 0.45, 2.0}, {6, 7, 2, 0.85, 0.80, 2.5},
                                {5, 6, 1, 0.22, 0.50, 2.5}, {6, 7, 1, 0.78, 0.85, 3.0}};
static const TileCost* costs_of(int storage) { return storage == kStorageF32 ? kCost32 : kCost16; }

static const Linear8Table& table_of(int storage) {
  static const Linear8Table tables[] = {linear_fp8_table_f32(), linear_fp8_table_bf16(), linear_fp8_table_f16()};
  return tables[storage];
}

struct Plan {
  Linear8Tile tile;
  int64_t splits, k_split;
  double cost;
};

// The tile and the number of k ranges that cost least.  The join of s ranges costs a launch (4 us) and 8 s bytes a
// result, at 4 TB/s; a product that takes less than that whole is not looked at in ranges.
static Plan plan_of(int64_t m, int64_t n, int64_t k, int storage) {
  // (a call works this out several times over, for the workspace's size too: 32 bits, which the sizes fit, and no
  // divisions that the host would wait for)
  const int stages = std::max(1, (int)((k + kStage - 1) / kStage)), cus = (int)kCUs;
  const Linear8Table& table = table_of(storage);
  const TileCost* const costs = costs_of(storage);
  const double join = 8.0 * (double)m * (double)n / 4e6;
  Linear8Tile tile = kLinear8Tiles;
  int best_splits = 1, best_each = stages;
  double least = 0;
  const auto look = [&](int t, int tiles, int splits, int each) {
    const TileCost& c = costs[t];
    const int per_cu = std::max(1, (tiles * splits + cus - 1) / cus);
    const int rounds = (int)(((double)per_cu + c.together - 1) / c.together);
    const double stage = per_cu == 1 ? c.alone : c.each * per_cu;
    double cost = each * stage + c.ends * rounds;
    if (splits > 1) cost += 4.0 + join * splits;
    if (tile == kLinear8Tiles || cost < least) {
      tile = (Linear8Tile)t;
      best_splits = splits;
      best_each = each;
      least = cost;
    }
  };
  int tiles[kLinear8Tiles];
  for (int t = 0; t < kLinear8Tiles; ++t) {
    if (table.fn[t] == nullptr) continue;  // (not built)
    tiles[t] = (int)((uint32_t)(m + costs[t].bm - 1) >> costs[t].log_m) * (int)((uint32_t)(n + costs[t].bn - 1) >> costs[t].log_n);
    look(t, tiles[t], 1, stages);
  }
  for (int t = 0; t < kLinear8Tiles; ++t) {
    if (table.fn[t] == nullptr) continue;
    for (int want = 2; want <= 16; ++want) {
      if (tiles[t] * want > 4 * cus || stages < 2 * want || 4.0 + costs[t].ends + join * want >= least) break;
      const int each = (stages + want - 1) / want, splits = (stages + each - 1) / each;
      if (splits == want) look(t, tiles[t], splits, each);  // (else as many ranges of another length)
    }
  }
  return {tile, best_splits, best_each * kStage, least};
}
static int64_t split_bytes(int64_t m, int64_t n, int64_t k, int storage) {
  if (m <= kFewTokens) return 0;
  const Plan p = plan_of(m, n, k, storage);
  return p.splits > 1 ? p.splits * m * n * 4 : 0;
}

// Which tile two products share in one launch, the first one's k being the longer, or kLinear8Tiles where two launches
// cost less.  Where the first has a workgroup for every CU the rounds are simply full; where it has fewer, its CUs deal
// part of their time to the second's tiles until those run out, and finish alone.  4 us: the launch that is saved.
// One launch and two, with the pass that quantizes dz (us, tokens x d_in x d_out): 1000 x 768 x 768 14.0 and 17.6, 4093 x 768 x
// 768 26 and 32, 2045 x 2048 x 2048 34 and 42; two stay for 30 x 4096 x 4096 (25.8, one 26.9) and 16384 x 512 x 512.
static Linear8Tile together_of(const GemmArgs& first, const GemmArgs& second, int storage) {
  const double k1 = (double)((first.k + kStage - 1) / kStage), k2 = (double)((second.k + kStage - 1) / kStage);
  // (the few rows' kernel: B's bytes at the rate of memory, 3 us before and after.  That holds where its workgroups, one for
  // 16 or 32 rows of B, are many and k is no longer than a layer is wide; the few of dW with few outputs over many tokens take
  // longer, 64 x 64 over 16384 17 us where this says 3.2)
  const auto alone = [&](const GemmArgs& g) {
    return g.m <= kFewTokens ? 3.0 + (double)g.n * (double)g.k / 5e6 : plan_of(g.m, g.n, g.k, storage).cost;
  };
  Linear8Tile best = kLinear8Tiles;
  double least = 4.0 + alone(first) + alone(second);
  for (int t = 0; t < kLinear8Tiles; ++t) {
    if (table_of(storage).pair[t] == nullptr) continue;
    const TileCost& c = costs_of(storage)[t];
    const auto tiles = [&](const GemmArgs& g) { return (double)((g.m + c.bm - 1) / c.bm * ((g.n + c.bn - 1) / c.bn)); };
    const double cus = (double)kCUs, n1 = tiles(first), n2 = tiles(second), per_cu = std::ceil((n1 + n2) / cus);
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
      best = (Linear8Tile)t;
    }
  }
  return best;
}

static hipError_t product(Gemm8Args& args, int storage, void* workspace, hipStream_t stream) {
  GemmArgs& g = args.g;
  const Linear8Table& t = table_of(storage);
  g.splits = 1;
  if (g.m <= kFewTokens) {
    // 32 rows of B to a workgroup where 16 make more workgroups than CUs (one row of 4096 -> 6144 4.8 us, else 5.7; 64 rows of
    // 2048 -> 6144 5.2, else 8.1; one row of 4096 -> 4096 4.8, with 16 4.5), or a checkpoint's blocks ask for it.  (dW of 64
    // outputs and less comes here too, and does not split k over workgroups: 64 x 64 over 16384 tokens takes 17 us, 72 x 64
    // in a tile whose k is split 9.3 with its join; 64 x 4096 18, 72 x 4096 23; 64 x 64 over 4096 tokens 6.5, 72 x 64 8.5)
    const bool wide = g.ck.codes != nullptr || g.n > 16 * kCUs;
    return t.few[g.m <= 16 ? 0 : g.m <= 32 ? 1 : 2][wide](args, stream);
  }
  const Plan p = plan_of(g.m, g.n, g.k, storage);
  g.splits = (int)p.splits;
  g.k_split = p.k_split;
  g.partial = p.splits > 1 ? static_cast<float*>(workspace) : nullptr;
  const hipError_t e = t.fn[p.tile](args, stream);
  return e != hipSuccess || g.partial == nullptr ? e : launch_linear_join(g, storage, stream);
}

int64_t linear_fp8_forward_workspace(const LinearSizes& s) { return split_bytes(s.tokens, s.d_out, s.d_in, s.storage); }

hipError_t launch_linear_fp8_forward(const LinearFp8Forward& a, hipStream_t stream) {
  Gemm8Args p{};
  p.a = a.x;
  p.b = a.w;
  p.g.m = a.s.tokens;
  p.g.n = a.s.d_out;
  p.g.k = a.s.d_in;
  p.g.d = a.y;
  p.g.ldd = a.ldy;
  p.g.bias = a.bias;
  p.g.residual = a.residual;
  p.g.ldr = a.ldr;
  p.g.ck = a.ck;
  p.g.act = a.s.act;
  return product(p, a.s.storage, a.workspace, stream);
}

// ----------------------------------------------------------------------------------
// the backward's workspace: dz by rows, dz by columns, then the partial sums of whichever pass runs (they follow
// each other on the stream)
static int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

struct BackwardSpace {
  Fp8Operand rows, columns;
  char* parts;
  int64_t bytes;  // before the parts
};
static BackwardSpace space_of(const LinearSizes& s, bool dx, bool dw, void* workspace) {
  char* p = static_cast<char*>(workspace);
  BackwardSpace b{};
  const auto take = [&](int64_t rows, int64_t n) {
    Fp8Operand o;
    o.ld = round_up(n, 16);
    o.lds = round_up((n + kStage - 1) / kStage, 4);
    o.codes = reinterpret_cast<uint8_t*>(p + b.bytes);
    b.bytes += round_up(rows * o.ld, 256);
    o.scales = reinterpret_cast<uint8_t*>(p + b.bytes);
    b.bytes += round_up(rows * o.lds, 256);
    return o;
  };
  if (dx) b.rows = take(s.tokens, s.d_out);
  if (dw) b.columns = take(s.d_out, s.tokens);
  b.parts = p + b.bytes;
  return b;
}

int64_t linear_fp8_backward_workspace(const LinearSizes& s, bool dx, bool dw, bool db) {
  int64_t parts = 0;
  if (db && s.tokens > kStage) parts = std::max(parts, (s.tokens + kStage - 1) / kStage * s.d_out * 4);
  if (dx) parts = std::max(parts, split_bytes(s.tokens, s.d_in, s.d_out, s.storage));
  if (dw) parts = std::max(parts, split_bytes(s.d_out, s.d_in, s.tokens, s.storage));
  return space_of(s, dx, dw, nullptr).bytes + parts;
}

hipError_t launch_linear_fp8_backward(const LinearFp8Backward& a, hipStream_t stream) {
  const int64_t T = a.s.tokens, n = a.s.d_out;
  const int storage = a.s.storage;
  const bool dx = a.dx != nullptr && T > 0, dw = a.dw != nullptr;
  const BackwardSpace space = space_of(a.s, a.dx != nullptr, dw, a.workspace);
  hipError_t e = hipSuccess;
  if (T > 0) {
    Fp8Quantize q{};
    q.x = a.dy;
    q.ldx = a.ldg;
    q.rows = T;
    q.n = n;
    if (dx) q.held = space.rows;
    if (dw) q.columns = space.columns;
    q.act = a.s.act;
    q.ck = a.s.act == kActNone ? Checkpoint{} : a.ck;
    // (the sums of a single band are db itself)
    if (a.db != nullptr && T <= kStage) q.total = a.db;
    else if (a.db != nullptr) q.sums = reinterpret_cast<float*>(space.parts);
    q.storage = storage;
    e = launch_fp8_quantize(q, stream);
    if (e != hipSuccess) return e;
  }
  if (a.db != nullptr && (T == 0 || T > kStage)) {
    e = launch_column_finish(reinterpret_cast<const float*>(space.parts), (T + kStage - 1) / kStage, n, n, a.db, nullptr,
                             storage, stream);
    if (e != hipSuccess) return e;
  }
  Gemm8Args x{}, w{};
  x.a = space.rows;
  x.b = a.w;
  x.g.m = T;
  x.g.n = a.s.d_in;
  x.g.k = n;
  x.g.d = a.dx;
  x.g.ldd = a.ldd;
  x.g.residual = a.add;
  x.g.ldr = a.lda;
  w.a = space.columns;
  w.b = a.x;
  w.g.m = n;
  w.g.n = a.s.d_in;
  w.g.k = T;
  w.g.d = a.dw;
  w.g.ldd = a.lddw;
  if (dx && dw) {
    const bool dw_first = T >= n;  // (the longer k)
    Gemm8Args &first = dw_first ? w : x, &second = dw_first ? x : w;
    const Linear8Tile t = together_of(first.g, second.g, storage);
    if (t != kLinear8Tiles) {
      for (GemmArgs* g : {&first.g, &second.g}) {
        g->splits = 1;
        g->k_split = g->k;
      }
      return table_of(storage).pair[t](first, second, stream);
    }
  }
  if (dx) e = product(x, storage, space.parts, stream);
  if (e == hipSuccess && dw) e = product(w, storage, space.parts, stream);
  return e;
}

}  // namespace rdfft
