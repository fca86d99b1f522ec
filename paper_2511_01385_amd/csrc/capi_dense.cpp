// capi_dense.cpp -- the C entry points of the operators around the block-circulant layer: 8-bit
// checkpoints, the norms, the dense product and its form in 8-bit floating point (declared in include/rdfft.h).  As in
// capi.cpp, arguments are checked on the host before any HIP call and nothing allocates device memory.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <initializer_list>

#include "capi_util.hpp"
#include "dense_launch.hpp"
#include "fp8_launch.hpp"
#include "rdfft.h"

namespace {

using rdfft::aligned16;
using rdfft::elem_bytes;
using rdfft::ensure_device;
using rdfft::mul_ok;

constexpr int64_t kMaxFeatures = (int64_t)1 << 20, kMaxStride = (int64_t)1 << 21, kMaxTokens = (int64_t)1 << 22;
constexpr int64_t kMaxTiles = (int64_t)1 << 22;  // of 128 x 128 results
constexpr int64_t kMaxFp8Width = (int64_t)1 << 29;  // (a row of 2^22 tiles to quantize)

bool known(int dtype) { return dtype == RDFFT_F32 || dtype == RDFFT_BF16 || dtype == RDFFT_F16; }

// rows of `len` bytes, `pitch` bytes apart
struct Rows {
  const void* p = nullptr;
  int64_t rows = 0, len = 0, pitch = 0;
  bool empty() const { return p == nullptr || rows <= 0 || len <= 0; }
  int64_t span() const { return (rows - 1) * pitch + len; }
};

// whether a byte belongs to both; rows of one pitch may lie side by side
bool overlap(const Rows& a, const Rows& b) {
  if (a.empty() || b.empty() || !rdfft::overlaps(a.p, a.span(), b.p, b.span())) return false;
  if (a.rows == 1 || b.rows == 1 || a.pitch != b.pitch) return true;
  const int64_t d = (int64_t)(reinterpret_cast<intptr_t>(b.p) - reinterpret_cast<intptr_t>(a.p));
  const int64_t off = ((d % a.pitch) + a.pitch) % a.pitch;  // where b's rows start in a's
  return !(off >= a.len && off + b.len <= a.pitch);
}
bool same(const Rows& a, const Rows& b) { return a.p == b.p && a.pitch == b.pitch; }

// fills `out` from a tensor of elements of `item` bytes; false: null (unless it may be), misaligned, a
// stride shorter than the row, or sizes beyond 63 bits.  The stride of a single row reaches nothing: it counts as the row.
bool tensor(const void* p, int64_t rows, int64_t n, int64_t ld, int item, bool may_be_null, Rows* out) {
  if (p == nullptr || rows == 0) {
    *out = Rows{};
    return p != nullptr || may_be_null || rows == 0;
  }
  int64_t bytes = 0, all = 0;
  if (ld < n || reinterpret_cast<uintptr_t>(p) % (uintptr_t)item != 0) return false;
  if (!mul_ok(rows == 1 ? n : ld, item, &bytes) || !mul_ok(rows, bytes, &all)) return false;
  *out = Rows{p, rows, n * item, bytes};
  return true;
}
bool contiguous(const void* p, int64_t count, int item, bool may_be_null, Rows* out) {
  return tensor(p, count > 0 ? 1 : 0, count, count, item, may_be_null, out);
}

// a tensor's row stride in elements of `item` bytes
int64_t stride(const Rows& r, int item) { return r.pitch / item; }

int64_t ck_blocks(int64_t n) { return (n + 31) / 32; }
bool checkpoint(const act8_t& c, int64_t rows, int64_t n, bool may_be_null, Rows* codes, Rows* scales) {
  if (may_be_null && c.codes == nullptr && c.scales == nullptr) return true;
  return tensor(c.codes, rows, n, n, 1, false, codes) && tensor(c.scales, rows, ck_blocks(n), ck_blocks(n), 1, false, scales);
}

// An 8-bit floating point matrix [rows][n] as the launchers take it; false: null, misaligned, or strides too short.
bool fp8(const fp8_t& o, int64_t rows, int64_t n, Rows* codes, Rows* scales, rdfft::Fp8Operand* out) {
  const int64_t blocks = (n + 127) / 128, bands = o.block_rows == 1 ? rows : (rows + 127) / 128;
  if (o.block_rows != 1 && o.block_rows != 128) return false;
  if (!tensor(o.codes, rows, n, rows == 1 ? n : o.ld, 1, false, codes) ||
      !tensor(o.scales, bands, blocks, bands == 1 ? blocks : o.lds, 1, false, scales))
    return false;
  if (rows == 0 || n == 0) return true;
  if (!aligned16(o.codes) || reinterpret_cast<uintptr_t>(o.scales) % 4 != 0) return false;
  if ((rows > 1 && o.ld % 16 != 0) || (bands > 1 && o.lds % 4 != 0)) return false;
  // (a single row's strides are such as a next row's would be)
  *out = {o.codes, rows == 1 ? (n + 15) / 16 * 16 : codes->pitch, o.scales,
          bands == 1 ? (blocks + 3) / 4 * 4 : scales->pitch, o.block_rows == 1 ? 0 : 7};
  return true;
}

// no output overlaps an input or another output
bool apart(std::initializer_list<Rows> outputs, std::initializer_list<Rows> inputs) {
  for (const Rows* o = outputs.begin(); o != outputs.end(); ++o) {
    for (const Rows& i : inputs)
      if (overlap(*o, i)) return false;
    for (const Rows* p = outputs.begin(); p != o; ++p)
      if (overlap(*o, *p)) return false;
  }
  return true;
}

bool workspace(const void* p, int64_t bytes, int64_t need, Rows* out) {
  if (need == 0) return true;
  if (p == nullptr || bytes < need || !aligned16(p)) return false;
  *out = Rows{p, 1, need, need};
  return true;
}

int status(hipError_t e) { return e == hipSuccess ? RDFFT_OK : RDFFT_ELAUNCH; }

int device(int* num_cu) {
  const float2* tw = nullptr;
  return ensure_device(&tw, num_cu);
}

int act8_sizes(int64_t rows, int64_t n, int dtype) {
  int64_t all = 0, bytes = 0;
  if (!known(dtype) || rows < 0 || n < 1) return RDFFT_EINVAL;
  return mul_ok(rows, n, &all) && mul_ok(all, 4, &bytes) ? RDFFT_OK : RDFFT_EINVAL;
}

int norm_sizes(int64_t rows, int64_t n, int dtype) {
  const int st = act8_sizes(rows, n, dtype);
  return st == RDFFT_OK && n > rdfft::kNormMaxWidth ? RDFFT_EUNSUPPORTED : st;
}

int linear_sizes(int64_t d_in, int64_t d_out, int64_t tokens, int act, int dtype) {
  if (!known(dtype) || d_in < 1 || d_out < 1 || tokens < 0) return RDFFT_EINVAL;
  if (act < RDFFT_ACT_NONE || act > RDFFT_ACT_SILU) return RDFFT_EINVAL;
  if (d_in > kMaxFeatures || d_out > kMaxFeatures || tokens > kMaxTokens) return RDFFT_EUNSUPPORTED;
  const auto tiles = [](int64_t a, int64_t b) { return ((a + 127) / 128) * ((b + 127) / 128); };
  if (tiles(tokens, d_out) > kMaxTiles || tiles(tokens, d_in) > kMaxTiles || tiles(d_out, d_in) > kMaxTiles)
    return RDFFT_EUNSUPPORTED;
  return RDFFT_OK;
}

}  // namespace

extern "C" {

int act8_quantize(const void* x, int64_t ldx, const act8_t* to, int64_t rows, int64_t n, rdfft_dtype_t dtype,
                  rdfft_stream_t stream) {
  int st = act8_sizes(rows, n, dtype);
  if (st != RDFFT_OK) return st;
  if (rows == 0) return RDFFT_OK;
  Rows in, codes, scales;
  if (to == nullptr || !tensor(x, rows, n, ldx, elem_bytes(dtype), false, &in) ||
      !checkpoint(*to, rows, n, false, &codes, &scales) || !apart({codes, scales}, {in}))
    return RDFFT_EINVAL;
  int num_cu = 0;
  st = device(&num_cu);
  if (st != RDFFT_OK) return st;
  return status(rdfft::launch_act8_quantize(x, ldx, to->codes, to->scales, rows, n, dtype,
                                            reinterpret_cast<hipStream_t>(stream), num_cu));
}

int act8_dequantize(const act8_t* from, void* out, int64_t ldo, int64_t rows, int64_t n, rdfft_dtype_t dtype,
                    rdfft_stream_t stream) {
  int st = act8_sizes(rows, n, dtype);
  if (st != RDFFT_OK) return st;
  if (rows == 0) return RDFFT_OK;
  Rows to, codes, scales;
  if (from == nullptr || !tensor(out, rows, n, ldo, elem_bytes(dtype), false, &to) ||
      !checkpoint(*from, rows, n, false, &codes, &scales) || !apart({to}, {codes, scales}))
    return RDFFT_EINVAL;
  int num_cu = 0;
  st = device(&num_cu);
  if (st != RDFFT_OK) return st;
  return status(rdfft::launch_act8_dequantize(from->codes, from->scales, out, ldo, rows, n, dtype,
                                              reinterpret_cast<hipStream_t>(stream), num_cu));
}

int layer_norm_forward(const layer_norm_forward_t* a, int64_t rows, int64_t n, float eps, rdfft_dtype_t dtype,
                       rdfft_stream_t stream) {
  int st = norm_sizes(rows, n, dtype);
  if (st != RDFFT_OK) return st;
  if (!(eps >= 0.f) || isinf(eps)) return RDFFT_EINVAL;
  if (rows == 0) return RDFFT_OK;
  if (a == nullptr) return RDFFT_EINVAL;
  const int s = elem_bytes(dtype);
  Rows x, r, w, b, y, mean, rstd, codes, scales;
  if (!tensor(a->x, rows, n, a->ldx, s, false, &x) || !tensor(a->residual, rows, n, a->ldr, s, true, &r) ||
      !contiguous(a->weight, n, 4, false, &w) || !contiguous(a->bias, n, 4, true, &b) ||
      !tensor(a->y, rows, n, a->ldy, s, false, &y) || !contiguous(a->mean, rows, 4, true, &mean) ||
      !contiguous(a->rstd, rows, 4, true, &rstd) || !checkpoint(a->checkpoint, rows, n, true, &codes, &scales))
    return RDFFT_EINVAL;
  // a row is read whole before it is written
  if ((overlap(y, x) && !same(y, x)) || (overlap(y, r) && !same(y, r)) || !apart({y, mean, rstd, codes, scales}, {w, b}) ||
      !apart({mean, rstd, codes, scales}, {x, r}))
    return RDFFT_EINVAL;
  int num_cu = 0;
  st = device(&num_cu);
  if (st != RDFFT_OK) return st;
  const rdfft::NormArgs k{a->x, a->ldx, a->residual, a->ldr, a->weight, a->bias, a->y, a->ldy, a->mean, a->rstd,
                          {a->checkpoint.codes, a->checkpoint.scales}, rows, n, eps, dtype};
  return status(rdfft::launch_layer_norm_forward(k, reinterpret_cast<hipStream_t>(stream), num_cu));
}

int64_t layer_norm_backward_workspace(int64_t rows, int64_t n) {
  const int st = norm_sizes(rows, n, RDFFT_F32);
  if (st != RDFFT_OK) return st;
  const int64_t parts = rdfft::norm_partials(rows, n);
  return parts == 1 ? 0 : parts * 2 * n * 4;
}

int layer_norm_backward(const layer_norm_backward_t* a, int64_t rows, int64_t n, rdfft_dtype_t dtype,
                        rdfft_stream_t stream) {
  int st = norm_sizes(rows, n, dtype);
  if (st != RDFFT_OK) return st;
  if (a == nullptr) return RDFFT_EINVAL;
  const int s = elem_bytes(dtype);
  Rows dy, x, r, w, mean, rstd, codes, scales, dx, dw, db, ws;
  const bool held = a->x == nullptr;
  if (!tensor(a->dy, rows, n, a->ldg, s, false, &dy) || !tensor(a->x, rows, n, a->ldx, s, true, &x) ||
      !tensor(a->residual, rows, n, a->ldr, s, true, &r) || !contiguous(a->weight, n, 4, false, &w) ||
      !contiguous(a->mean, rows, 4, false, &mean) || !contiguous(a->rstd, rows, 4, false, &rstd) ||
      !tensor(a->dx, rows, n, a->ldd, s, false, &dx) || !contiguous(a->dweight, n, 4, false, &dw) ||
      !contiguous(a->dbias, n, 4, false, &db))
    return RDFFT_EINVAL;
  if (held && (a->residual != nullptr || !checkpoint(a->checkpoint, rows, n, rows == 0, &codes, &scales)))
    return RDFFT_EINVAL;
  if (!workspace(a->workspace, a->workspace_bytes, layer_norm_backward_workspace(rows, n), &ws)) return RDFFT_EINVAL;
  if ((overlap(dx, dy) && !same(dx, dy)) || !apart({dx, dw, db, ws}, {x, r, codes, scales, w, mean, rstd}) ||
      !apart({dw, db, ws}, {dy}))
    return RDFFT_EINVAL;
  st = device(nullptr);
  if (st != RDFFT_OK) return st;
  const rdfft::NormGradArgs k{a->dy, a->ldg, a->x, a->ldx, a->residual, a->ldr,
                              {held ? a->checkpoint.codes : nullptr, held ? a->checkpoint.scales : nullptr},
                              a->weight, a->mean, a->rstd, a->dx, a->ldd, a->dweight, a->dbias,
                              static_cast<float*>(a->workspace), rows, n, dtype};
  return status(rdfft::launch_layer_norm_backward(k, reinterpret_cast<hipStream_t>(stream)));
}

int64_t linear_forward_workspace(int64_t d_in, int64_t d_out, int64_t tokens, rdfft_dtype_t dtype) {
  const int st = linear_sizes(d_in, d_out, tokens, RDFFT_ACT_NONE, dtype);
  if (st != RDFFT_OK) return st;
  return tokens == 0 ? 0 : rdfft::linear_forward_workspace({d_in, d_out, tokens, RDFFT_ACT_NONE, dtype});
}

int linear_forward(const linear_forward_t* a, int64_t d_in, int64_t d_out, int64_t tokens, rdfft_activation_t act,
                   rdfft_dtype_t dtype, rdfft_stream_t stream) {
  int st = linear_sizes(d_in, d_out, tokens, act, dtype);
  if (st != RDFFT_OK) return st;
  if (tokens == 0) return RDFFT_OK;
  if (a == nullptr) return RDFFT_EINVAL;
  const int s = elem_bytes(dtype);
  Rows x, w, b, r, y, codes, scales, ws;
  if (!tensor(a->x, tokens, d_in, a->ldx, s, false, &x) || !tensor(a->w, d_out, d_in, a->ldw, s, false, &w) ||
      !contiguous(a->bias, d_out, s, true, &b) || !tensor(a->residual, tokens, d_out, a->ldr, s, true, &r) ||
      !tensor(a->y, tokens, d_out, a->ldy, s, false, &y) || !checkpoint(a->checkpoint, tokens, d_out, true, &codes, &scales) ||
      !workspace(a->workspace, a->workspace_bytes, linear_forward_workspace(d_in, d_out, tokens, dtype), &ws))
    return RDFFT_EINVAL;
  if (stride(x, s) > kMaxStride || stride(w, s) > kMaxStride) return RDFFT_EUNSUPPORTED;
  if ((overlap(y, r) && !same(y, r)) || !apart({y, codes, scales, ws}, {x, w, b}) || !apart({codes, scales, ws}, {r}))
    return RDFFT_EINVAL;
  st = device(nullptr);
  if (st != RDFFT_OK) return st;
  const rdfft::LinearForward k{{d_in, d_out, tokens, act, dtype}, a->x, stride(x, s), a->w, stride(w, s), a->bias,
                               a->residual, a->ldr, a->y, a->ldy, {a->checkpoint.codes, a->checkpoint.scales}, a->workspace};
  return status(rdfft::launch_linear_forward(k, reinterpret_cast<hipStream_t>(stream)));
}

int64_t linear_backward_workspace(int64_t d_in, int64_t d_out, int64_t tokens, int dx, int dw, int db,
                                  rdfft_activation_t act, rdfft_dtype_t dtype) {
  const int st = linear_sizes(d_in, d_out, tokens, act, dtype);
  if (st != RDFFT_OK) return st;
  return rdfft::linear_backward_workspace({d_in, d_out, tokens, act, dtype}, dx != 0, dw != 0, db != 0);
}

int linear_backward(const linear_backward_t* a, int64_t d_in, int64_t d_out, int64_t tokens, rdfft_activation_t act,
                    rdfft_dtype_t dtype, rdfft_stream_t stream) {
  int st = linear_sizes(d_in, d_out, tokens, act, dtype);
  if (st != RDFFT_OK) return st;
  if (a == nullptr) return RDFFT_EINVAL;
  const int s = elem_bytes(dtype);
  const bool wants_dx = a->dx != nullptr, wants_dw = a->dw != nullptr, wants_db = a->db != nullptr;
  if (!wants_dx && !wants_dw && !wants_db) return RDFFT_OK;
  Rows dy, codes, scales, x, w, add, dx, dw, db, ws;
  if (!tensor(a->dy, tokens, d_out, a->ldg, s, false, &dy) ||
      !tensor(a->dx, tokens, d_in, a->ldd, s, true, &dx) || !tensor(a->dw, d_out, d_in, a->lddw, s, true, &dw) ||
      !contiguous(a->db, d_out, s, true, &db))
    return RDFFT_EINVAL;
  if (act != RDFFT_ACT_NONE && !checkpoint(a->checkpoint, tokens, d_out, tokens == 0, &codes, &scales)) return RDFFT_EINVAL;
  if (wants_dw && !tensor(a->x, tokens, d_in, a->ldx, s, false, &x)) return RDFFT_EINVAL;
  if (wants_dx &&
      (!tensor(a->w, d_out, d_in, a->ldw, s, false, &w) || !tensor(a->add, tokens, d_in, a->lda, s, true, &add)))
    return RDFFT_EINVAL;
  if (!workspace(a->workspace, a->workspace_bytes,
                 linear_backward_workspace(d_in, d_out, tokens, wants_dx, wants_dw, wants_db, act, dtype), &ws))
    return RDFFT_EINVAL;
  if (stride(dy, s) > kMaxStride || stride(x, s) > kMaxStride || stride(w, s) > kMaxStride) return RDFFT_EUNSUPPORTED;
  if ((overlap(dx, add) && !same(dx, add)) || !apart({dx, dw, db, ws}, {dy, codes, scales, x, w}) ||
      !apart({dw, db, ws}, {add}))
    return RDFFT_EINVAL;
  st = device(nullptr);
  if (st != RDFFT_OK) return st;
  const rdfft::LinearBackward k{{d_in, d_out, tokens, act, dtype}, a->dy, stride(dy, s),
                                {a->checkpoint.codes, a->checkpoint.scales}, a->x, stride(x, s), a->w, stride(w, s), a->add,
                                a->lda, a->dx, a->ldd, a->dw, a->lddw, a->db, a->workspace};
  return status(rdfft::launch_linear_backward(k, reinterpret_cast<hipStream_t>(stream)));
}

int fp8_quantize(const void* x, int64_t ldx, const fp8_t* held, const fp8_t* columns, int64_t rows, int64_t n,
                 rdfft_dtype_t dtype, rdfft_stream_t stream) {
  int st = act8_sizes(rows, n, dtype);
  if (st != RDFFT_OK) return st;
  if (rows == 0) return RDFFT_OK;
  Rows in, hc, hs, cc, cs;
  rdfft::Fp8Quantize q{};
  if ((held == nullptr && columns == nullptr) || !tensor(x, rows, n, ldx, elem_bytes(dtype), false, &in) ||
      (held != nullptr && !fp8(*held, rows, n, &hc, &hs, &q.held)) ||
      (columns != nullptr && !fp8(*columns, n, rows, &cc, &cs, &q.columns)) || !apart({hc, hs, cc, cs}, {in}))
    return RDFFT_EINVAL;
  // (a single row's blocks are tiles just as well)
  const bool by_held = held != nullptr && rows > 1, by_columns = columns != nullptr && n > 1;
  if (by_held && by_columns && held->block_rows != columns->block_rows) return RDFFT_EINVAL;
  if (n > kMaxFp8Width) return RDFFT_EUNSUPPORTED;
  st = device(nullptr);
  if (st != RDFFT_OK) return st;
  q.x = x;
  q.ldx = ldx;
  q.rows = rows;
  q.n = n;
  q.tiles = (by_held && held->block_rows != 1) || (by_columns && columns->block_rows != 1);
  q.storage = dtype;
  return status(rdfft::launch_fp8_quantize(q, reinterpret_cast<hipStream_t>(stream)));
}

int fp8_dequantize(const fp8_t* from, void* out, int64_t ldo, int64_t rows, int64_t n, rdfft_dtype_t dtype,
                   rdfft_stream_t stream) {
  int st = act8_sizes(rows, n, dtype);
  if (st != RDFFT_OK) return st;
  if (rows == 0) return RDFFT_OK;
  Rows to, codes, scales;
  rdfft::Fp8Operand o;
  if (from == nullptr || !tensor(out, rows, n, ldo, elem_bytes(dtype), false, &to) ||
      !fp8(*from, rows, n, &codes, &scales, &o) || !apart({to}, {codes, scales}))
    return RDFFT_EINVAL;
  int num_cu = 0;
  st = device(&num_cu);
  if (st != RDFFT_OK) return st;
  return status(rdfft::launch_fp8_dequantize(o, out, ldo, rows, n, dtype, reinterpret_cast<hipStream_t>(stream), num_cu));
}

int rms_norm_forward(const rms_norm_forward_t* a, int64_t rows, int64_t n, float eps, rdfft_dtype_t dtype,
                     rdfft_stream_t stream) {
  int st = norm_sizes(rows, n, dtype);
  if (st != RDFFT_OK) return st;
  if (!(eps >= 0.f) || isinf(eps)) return RDFFT_EINVAL;
  if (rows == 0) return RDFFT_OK;
  if (a == nullptr) return RDFFT_EINVAL;
  const int s = elem_bytes(dtype);
  const bool wants8 = a->y8.codes != nullptr || a->y8.scales != nullptr;
  Rows x, r, w, y, u, rstd, codes, scales, c8, s8;
  rdfft::Fp8Operand y8;
  if (!tensor(a->x, rows, n, a->ldx, s, false, &x) || !tensor(a->residual, rows, n, a->ldr, s, true, &r) ||
      !contiguous(a->weight, n, 4, false, &w) || !tensor(a->y, rows, n, a->ldy, s, true, &y) ||
      !tensor(a->summed, rows, n, a->lds, s, true, &u) || !contiguous(a->rstd, rows, 4, true, &rstd) ||
      !checkpoint(a->checkpoint, rows, n, true, &codes, &scales) ||
      (wants8 && (a->y8.block_rows != 1 || !fp8(a->y8, rows, n, &c8, &s8, &y8))))
    return RDFFT_EINVAL;
  // a row is read whole before it is written
  for (const Rows& o : {y, u})
    if ((overlap(o, x) && !same(o, x)) || (overlap(o, r) && !same(o, r))) return RDFFT_EINVAL;
  if (!apart({y, u, rstd, codes, scales, c8, s8}, {w}) || !apart({rstd, codes, scales, c8, s8}, {x, r})) return RDFFT_EINVAL;
  int num_cu = 0;
  st = device(&num_cu);
  if (st != RDFFT_OK) return st;
  const rdfft::RmsArgs k{a->x, a->ldx, a->residual, a->ldr, a->weight, a->y, a->ldy, a->summed, a->lds, a->rstd,
                         {a->checkpoint.codes, a->checkpoint.scales}, y8, rows, n, eps, dtype};
  return status(rdfft::launch_rms_norm_forward(k, reinterpret_cast<hipStream_t>(stream), num_cu));
}

int64_t rms_norm_backward_workspace(int64_t rows, int64_t n) {
  const int st = norm_sizes(rows, n, RDFFT_F32);
  if (st != RDFFT_OK) return st;
  const int64_t parts = rdfft::rms_partials(rows, n);
  return parts == 1 ? 0 : parts * n * 4;
}

int rms_norm_backward(const rms_norm_backward_t* a, int64_t rows, int64_t n, rdfft_dtype_t dtype, rdfft_stream_t stream) {
  int st = norm_sizes(rows, n, dtype);
  if (st != RDFFT_OK) return st;
  if (a == nullptr) return RDFFT_EINVAL;
  const int s = elem_bytes(dtype);
  Rows dy, u, w, rstd, add, codes, scales, dx, dw, ws;
  const bool held = a->u == nullptr;
  if (!tensor(a->dy, rows, n, a->ldg, s, false, &dy) || !tensor(a->u, rows, n, a->ldu, s, true, &u) ||
      !contiguous(a->weight, n, 4, false, &w) || !contiguous(a->rstd, rows, 4, false, &rstd) ||
      !tensor(a->add, rows, n, a->lda, s, true, &add) || !tensor(a->dx, rows, n, a->ldd, s, false, &dx) ||
      !contiguous(a->dweight, n, 4, true, &dw))
    return RDFFT_EINVAL;
  if (held && !checkpoint(a->checkpoint, rows, n, rows == 0, &codes, &scales)) return RDFFT_EINVAL;
  if (a->dweight != nullptr && !workspace(a->workspace, a->workspace_bytes, rms_norm_backward_workspace(rows, n), &ws))
    return RDFFT_EINVAL;
  if ((overlap(dx, dy) && !same(dx, dy)) || (overlap(dx, add) && !same(dx, add)) ||
      !apart({dx, dw, ws}, {u, codes, scales, w, rstd}) || !apart({dw, ws}, {dy, add}))
    return RDFFT_EINVAL;
  if (rows == 0 && a->dweight == nullptr) return RDFFT_OK;
  st = device(nullptr);
  if (st != RDFFT_OK) return st;
  const rdfft::RmsGradArgs k{a->dy, a->ldg, a->u, a->ldu,
                             {held ? a->checkpoint.codes : nullptr, held ? a->checkpoint.scales : nullptr},
                             a->weight, a->rstd, a->add, a->lda, a->dx, a->ldd, a->dweight,
                             static_cast<float*>(a->workspace), rows, n, dtype};
  return status(rdfft::launch_rms_norm_backward(k, reinterpret_cast<hipStream_t>(stream)));
}

int64_t linear_fp8_forward_workspace(int64_t d_in, int64_t d_out, int64_t tokens, rdfft_dtype_t dtype) {
  const int st = linear_sizes(d_in, d_out, tokens, RDFFT_ACT_NONE, dtype);
  if (st != RDFFT_OK) return st;
  return tokens == 0 ? 0 : rdfft::linear_fp8_forward_workspace({d_in, d_out, tokens, RDFFT_ACT_NONE, dtype});
}

int linear_fp8_forward(const linear_fp8_forward_t* a, int64_t d_in, int64_t d_out, int64_t tokens, rdfft_activation_t act,
                       rdfft_dtype_t dtype, rdfft_stream_t stream) {
  int st = linear_sizes(d_in, d_out, tokens, act, dtype);
  if (st != RDFFT_OK) return st;
  if (tokens == 0) return RDFFT_OK;
  if (a == nullptr) return RDFFT_EINVAL;
  const int s = elem_bytes(dtype);
  Rows xc, xs, wc, wsc, b, r, y, codes, scales, ws;
  rdfft::LinearFp8Forward k{};
  if (!fp8(a->x, tokens, d_in, &xc, &xs, &k.x) || !fp8(a->w, d_out, d_in, &wc, &wsc, &k.w) ||
      !contiguous(a->bias, d_out, s, true, &b) || !tensor(a->residual, tokens, d_out, a->ldr, s, true, &r) ||
      !tensor(a->y, tokens, d_out, a->ldy, s, false, &y) || !checkpoint(a->checkpoint, tokens, d_out, true, &codes, &scales) ||
      !workspace(a->workspace, a->workspace_bytes, linear_fp8_forward_workspace(d_in, d_out, tokens, dtype), &ws))
    return RDFFT_EINVAL;
  if (xc.pitch > kMaxStride || wc.pitch > kMaxStride || xs.pitch > kMaxStride || wsc.pitch > kMaxStride)
    return RDFFT_EUNSUPPORTED;
  if ((overlap(y, r) && !same(y, r)) || !apart({y, codes, scales, ws}, {xc, xs, wc, wsc, b}) ||
      !apart({codes, scales, ws}, {r}))
    return RDFFT_EINVAL;
  st = device(nullptr);
  if (st != RDFFT_OK) return st;
  k.s = {d_in, d_out, tokens, act, dtype};
  k.bias = a->bias;
  k.residual = a->residual;
  k.ldr = a->ldr;
  k.y = a->y;
  k.ldy = a->ldy;
  k.ck = {a->checkpoint.codes, a->checkpoint.scales};
  k.workspace = a->workspace;
  return status(rdfft::launch_linear_fp8_forward(k, reinterpret_cast<hipStream_t>(stream)));
}

int64_t linear_fp8_backward_workspace(int64_t d_in, int64_t d_out, int64_t tokens, int dx, int dw, int db,
                                      rdfft_dtype_t dtype) {
  const int st = linear_sizes(d_in, d_out, tokens, RDFFT_ACT_NONE, dtype);
  if (st != RDFFT_OK) return st;
  return rdfft::linear_fp8_backward_workspace({d_in, d_out, tokens, RDFFT_ACT_NONE, dtype}, dx != 0, dw != 0, db != 0);
}

int linear_fp8_backward(const linear_fp8_backward_t* a, int64_t d_in, int64_t d_out, int64_t tokens, rdfft_activation_t act,
                        rdfft_dtype_t dtype, rdfft_stream_t stream) {
  int st = linear_sizes(d_in, d_out, tokens, act, dtype);
  if (st != RDFFT_OK) return st;
  if (a == nullptr) return RDFFT_EINVAL;
  const int s = elem_bytes(dtype);
  const bool wants_dx = a->dx != nullptr, wants_dw = a->dw != nullptr, wants_db = a->db != nullptr;
  if (!wants_dx && !wants_dw && !wants_db) return RDFFT_OK;
  Rows dy, codes, scales, xc, xs, wc, wsc, add, dx, dw, db, ws;
  rdfft::LinearFp8Backward k{};
  if (!tensor(a->dy, tokens, d_out, a->ldg, s, false, &dy) || !tensor(a->dx, tokens, d_in, a->ldd, s, true, &dx) ||
      !tensor(a->dw, d_out, d_in, a->lddw, s, true, &dw) || !contiguous(a->db, d_out, s, true, &db))
    return RDFFT_EINVAL;
  if (act != RDFFT_ACT_NONE && !checkpoint(a->checkpoint, tokens, d_out, tokens == 0, &codes, &scales)) return RDFFT_EINVAL;
  if (wants_dw && tokens > 0 && !fp8(a->x, d_in, tokens, &xc, &xs, &k.x)) return RDFFT_EINVAL;
  if (wants_dx && tokens > 0 &&
      (!fp8(a->w, d_in, d_out, &wc, &wsc, &k.w) || !tensor(a->add, tokens, d_in, a->lda, s, true, &add)))
    return RDFFT_EINVAL;
  if (!workspace(a->workspace, a->workspace_bytes,
                 linear_fp8_backward_workspace(d_in, d_out, tokens, wants_dx, wants_dw, wants_db, dtype), &ws))
    return RDFFT_EINVAL;
  if (stride(dy, s) > kMaxStride || xc.pitch > kMaxTokens || wc.pitch > kMaxStride || xs.pitch > kMaxStride ||
      wsc.pitch > kMaxStride)
    return RDFFT_EUNSUPPORTED;
  if ((overlap(dx, add) && !same(dx, add)) || !apart({dx, dw, db, ws}, {dy, codes, scales, xc, xs, wc, wsc}) ||
      !apart({dw, db, ws}, {add}))
    return RDFFT_EINVAL;
  st = device(nullptr);
  if (st != RDFFT_OK) return st;
  k.s = {d_in, d_out, tokens, act, dtype};
  k.dy = a->dy;
  k.ldg = a->ldg;
  k.ck = {a->checkpoint.codes, a->checkpoint.scales};
  k.add = a->add;
  k.lda = a->lda;
  k.dx = a->dx;
  k.ldd = a->ldd;
  k.dw = a->dw;
  k.lddw = a->lddw;
  k.db = a->db;
  k.workspace = a->workspace;
  return status(rdfft::launch_linear_fp8_backward(k, reinterpret_cast<hipStream_t>(stream)));
}

}  // extern "C"
