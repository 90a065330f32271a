// C ABI of the attention block: argument checks of layer norm, the linear layers and cross attention.

#include <hip/hip_runtime.h>

#include <cmath>
#include <string>

#include "checks.h"
#include "common.h"
#include "cross.h"
#include "internal.h"

using namespace fold;

namespace {

size_t vector_bytes(int64_t n) { return (size_t)n * sizeof(float); }

int check_norm(const std::string& who, int dtype, int64_t rows, int width) {
  if (!known_type(dtype)) return api_fail(FOLD_E_INVALID, who + ": unknown dtype");
  if (rows < 0 || rows > INT32_MAX) return api_fail(FOLD_E_INVALID, who + ": rows out of range");
  if (width < 1 || width > kMaxHidden) return api_fail(FOLD_E_INVALID, who + ": width out of range (1 .. 4096)");
  return FOLD_OK;
}

template <class F>
int check_linear(const std::string& who, int dtype, int64_t rows, int in_dim, int out_dim, F&& tiles) {
  if (!known_type(dtype)) return api_fail(FOLD_E_INVALID, who + ": unknown dtype");
  if (rows < 0 || rows > INT32_MAX) return api_fail(FOLD_E_INVALID, who + ": rows out of range");
  if (in_dim < 1 || in_dim > kMaxLinear || out_dim < 1 || out_dim > kMaxLinear)
    return api_fail(FOLD_E_INVALID, who + ": in_dim and out_dim must be 1 .. 16384");
  if (tiles(dtype, rows, in_dim, out_dim) >= kMaxTiles)
    return api_fail(FOLD_E_INVALID, who + ": too many tiles for one launch (rows times the widths)");
  return FOLD_OK;
}

// A matrix of cross attention: columns of rows that are ld elements apart.
struct Cols {
  const void* p;
  int64_t ld, rows;
  int width;  // elements
};
// Whether two of them share an element.  Different columns of rows with one stride (k and v side by side) do not.
bool share(const Cols& a, const Cols& b, int es) {
  const auto bytes = [&](const Cols& c) { return c.rows > 0 ? (size_t)((c.rows - 1) * c.ld + c.width) * es : (size_t)0; };
  if (!overlap({a.p, bytes(a)}, {b.p, bytes(b)})) return false;
  if (a.ld != b.ld) return true;
  if (reinterpret_cast<uintptr_t>(b.p) < reinterpret_cast<uintptr_t>(a.p)) return share(b, a, es);
  const int64_t row = a.ld * es;
  const int64_t d = (int64_t)((reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p)) % (uintptr_t)row);
  return !(d >= (int64_t)a.width * es && d + (int64_t)b.width * es <= row);
}

// a gradient's type: the operator's own, or fp32
bool grad_type(int type, int dtype) { return type == FOLD_F32 || type == dtype; }

}  // namespace

extern "C" {

int32_t fold_layer_norm(int32_t dtype, int64_t rows, int32_t width, const void* x, const float* gamma, const float* beta,
                        float eps, void* y, float* mean, float* rstd, hipStream_t st) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_layer_norm");
    const int rc = check_norm(who, dtype, rows, width);
    if (rc != FOLD_OK) return rc;
    if (!(eps > 0.f) || !std::isfinite(eps)) return api_fail(FOLD_E_INVALID, who + ": eps must be finite and above 0");
    if (rows == 0) return FOLD_OK;
    if (!x || !y) return api_fail(FOLD_E_INVALID, who + ": NULL buffer");
    if (misaligned(x) || misaligned(y)) return api_fail(FOLD_E_INVALID, who + ": x and y must be 16-byte aligned");
    const size_t m = bytes_of(dtype, rows, width), v = vector_bytes(width), r = vector_bytes(rows);
    const Span out[] = {{y, m}, {mean, r}, {rstd, r}};
    const Span in[] = {{y == x ? nullptr : x, m}, {gamma, v}, {beta, v}};
    if (any_overlap(out, 3, in, 3)) return api_fail(FOLD_E_INVALID, who + ": an output overlaps another buffer");
    launch_norm(dtype, rows, width, x, gamma, beta, eps, y, mean, rstd, st);
    FOLD_HIP_CHECK(hipGetLastError());
    return FOLD_OK;
  });
}

int32_t fold_layer_norm_workspace_size(int32_t dtype, int64_t rows, int32_t width, size_t* bytes) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_layer_norm_workspace_size");
    if (!bytes) return api_fail(FOLD_E_INVALID, who + ": NULL argument");
    const int rc = check_norm(who, dtype, rows, width);
    if (rc != FOLD_OK) return rc;
    *bytes = norm_backward_bytes(dtype, rows, width);
    return FOLD_OK;
  });
}

int32_t fold_layer_norm_backward(int32_t dtype, int64_t rows, int32_t width, const void* x, const float* gamma,
                                 const float* mean, const float* rstd, int32_t dy_dtype, const void* dy,
                                 int32_t residual_dtype, const void* residual, int32_t dx_dtype, void* dx, float* dgamma,
                                 float* dbeta, int32_t flags, void* ws, size_t ws_bytes, hipStream_t st) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_layer_norm_backward");
    const int rc = check_norm(who, dtype, rows, width);
    if (rc != FOLD_OK) return rc;
    if (!grad_type(dy_dtype, dtype) || !grad_type(dx_dtype, dtype) || (residual && !grad_type(residual_dtype, dtype)))
      return api_fail(FOLD_E_INVALID, who + ": gradients are of the states' type, or fp32");
    if (flags & ~FOLD_BLOCK_ACCUMULATE) return api_fail(FOLD_E_INVALID, who + ": unknown flag");
    if ((!dx || rows == 0) && !dgamma && !dbeta) return FOLD_OK;
    if (rows > 0 && (!x || !mean || !rstd || !dy)) return api_fail(FOLD_E_INVALID, who + ": NULL buffer");
    if (misaligned(x) || misaligned(dy) || misaligned(residual) || misaligned(dx) || misaligned(ws))
      return api_fail(FOLD_E_INVALID, who + ": matrices and the workspace must be 16-byte aligned");
    const size_t need = dgamma || dbeta ? norm_backward_bytes(dtype, rows, width) : 0;
    if (need > 0 && (!ws || ws_bytes < need))
      return api_fail(FOLD_E_MISMATCH, who + ": workspace smaller than fold_layer_norm_workspace_size");
    const size_t v = vector_bytes(width), r = vector_bytes(rows);
    const Span out[] = {{dx, bytes_of(dx_dtype, rows, width)}, {dgamma, v}, {dbeta, v}, {ws, need}};
    const Span in[] = {{x, bytes_of(dtype, rows, width)},
                       {dx == dy && dx_dtype == dy_dtype ? nullptr : dy, bytes_of(dy_dtype, rows, width)},
                       {dx == residual && dx_dtype == residual_dtype ? nullptr : residual, bytes_of(residual_dtype, rows, width)},
                       {gamma, v},
                       {mean, r},
                       {rstd, r}};
    if (any_overlap(out, 4, in, 6)) return api_fail(FOLD_E_INVALID, who + ": an output overlaps another buffer");
    launch_norm_backward(dtype, rows, width, x, gamma, mean, rstd, dy_dtype, dy, dx_dtype, residual_dtype, residual, dx, dgamma,
                         dbeta, flags & FOLD_BLOCK_ACCUMULATE, ws, st);
    FOLD_HIP_CHECK(hipGetLastError());
    return FOLD_OK;
  });
}

int32_t fold_linear(int32_t dtype, int64_t rows, int32_t in_dim, int32_t out_dim, const void* x, const void* W,
                    const float* bias, int32_t act, const void* residual, void* out, void* pre, void* ws, size_t ws_bytes,
                    hipStream_t st) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_linear");
    const int rc = check_linear(who, dtype, rows, in_dim, out_dim, linear_tiles);
    if (rc != FOLD_OK) return rc;
    if (act < FOLD_ACT_NONE || act > FOLD_ACT_GELU) return api_fail(FOLD_E_INVALID, who + ": unknown activation");
    if (rows == 0) return FOLD_OK;
    if (!x || !W || !out) return api_fail(FOLD_E_INVALID, who + ": NULL buffer");
    if (misaligned(x) || misaligned(W) || misaligned(residual) || misaligned(out) || misaligned(pre) || misaligned(ws))
      return api_fail(FOLD_E_INVALID, who + ": matrices must be 16-byte aligned");
    const size_t m = bytes_of(dtype, rows, out_dim);
    const size_t need = linear_bytes(dtype, rows, in_dim, out_dim);
    if (need > 0 && (!ws || ws_bytes < need))
      return api_fail(FOLD_E_MISMATCH, who + ": workspace smaller than fold_linear_workspace_size");
    const Span outs[] = {{out, m}, {pre, m}, {ws, need}};
    const Span in[] = {{x, bytes_of(dtype, rows, in_dim)}, {W, bytes_of(dtype, out_dim, in_dim)},
                       {bias, vector_bytes(out_dim)}, {residual == out ? nullptr : residual, m}};
    if (any_overlap(outs, 3, in, 4)) return api_fail(FOLD_E_INVALID, who + ": an output overlaps another buffer");
    launch_linear(dtype, rows, in_dim, out_dim, x, W, bias, act, residual, out, pre, ws, st);
    FOLD_HIP_CHECK(hipGetLastError());
    return FOLD_OK;
  });
}

int32_t fold_linear_workspace_size(int32_t dtype, int64_t rows, int32_t in_dim, int32_t out_dim, size_t* fwd_bytes,
                                   size_t* bwd_bytes) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_linear_workspace_size");
    if (!fwd_bytes || !bwd_bytes) return api_fail(FOLD_E_INVALID, who + ": NULL argument");
    int rc = check_linear(who, dtype, rows, in_dim, out_dim, linear_tiles);
    if (rc == FOLD_OK) rc = check_linear(who, dtype, rows, in_dim, out_dim, linear_backward_tiles);
    if (rc != FOLD_OK) return rc;
    *fwd_bytes = linear_bytes(dtype, rows, in_dim, out_dim);
    *bwd_bytes = linear_backward_bytes(dtype, rows, in_dim, out_dim);
    return FOLD_OK;
  });
}

int32_t fold_linear_backward(int32_t dtype, int64_t rows, int32_t in_dim, int32_t out_dim, const void* x, const void* W,
                             int32_t act, const void* pre, const void* dout, void* dpre, int32_t dx_dtype, void* dx,
                             int32_t dw_dtype, void* dW, float* dbias, int32_t flags, void* ws, size_t ws_bytes,
                             hipStream_t st) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_linear_backward");
    const int rc = check_linear(who, dtype, rows, in_dim, out_dim, linear_backward_tiles);
    if (rc != FOLD_OK) return rc;
    if (act < FOLD_ACT_NONE || act > FOLD_ACT_GELU) return api_fail(FOLD_E_INVALID, who + ": unknown activation");
    if (!grad_type(dx_dtype, dtype) || !grad_type(dw_dtype, dtype))
      return api_fail(FOLD_E_INVALID, who + ": gradients are of the layer's type, or fp32");
    if (flags & ~FOLD_BLOCK_ACCUMULATE) return api_fail(FOLD_E_INVALID, who + ": unknown flag");
    if ((flags & FOLD_BLOCK_ACCUMULATE) && dW && dw_dtype != FOLD_F32)
      return api_fail(FOLD_E_INVALID, who + ": a dW that is added to is fp32");
    const bool bent = act != FOLD_ACT_NONE;
    if (((!dx && !(bent && dpre)) || rows == 0) && !dW && !dbias) return FOLD_OK;
    if (rows > 0 && (!dout || (dW && !x) || (dx && !W) || (bent && (!pre || !dpre))))
      return api_fail(FOLD_E_INVALID, who + ": NULL buffer");
    if (!bent && (pre || dpre)) return api_fail(FOLD_E_INVALID, who + ": pre and dpre belong to an activation");
    if (misaligned(x) || misaligned(W) || misaligned(pre) || misaligned(dout) || misaligned(dpre) || misaligned(dx) ||
        misaligned(dW) || misaligned(ws))
      return api_fail(FOLD_E_INVALID, who + ": matrices and the workspace must be 16-byte aligned");
    const size_t need = linear_backward_bytes(dtype, rows, in_dim, out_dim);
    if (need > 0 && (!ws || ws_bytes < need))
      return api_fail(FOLD_E_MISMATCH, who + ": workspace smaller than fold_linear_workspace_size");
    const size_t m = bytes_of(dtype, rows, out_dim);
    const Span out[] = {{dpre, m}, {dx, bytes_of(dx_dtype, rows, in_dim)}, {dW, bytes_of(dw_dtype, out_dim, in_dim)},
                        {dbias, vector_bytes(out_dim)}, {ws, need}};
    const Span others[] = {{x, bytes_of(dtype, rows, in_dim)}, {W, bytes_of(dtype, out_dim, in_dim)},
                           {dpre == pre ? nullptr : pre, m}, {dpre == dout ? nullptr : dout, m}};
    // what dpre may be, the other outputs may not
    const Span elementwise[] = {{pre, m}, {dout, m}};
    if (any_overlap(out, 5, others, 4) || any_overlap(out + 1, 4, elementwise, 2))
      return api_fail(FOLD_E_INVALID, who + ": an output overlaps another buffer");
    launch_linear_backward(dtype, rows, in_dim, out_dim, x, W, act, pre, dout, dpre, dx_dtype, dx, dw_dtype, dW, dbias,
                           flags & FOLD_BLOCK_ACCUMULATE, ws, st);
    FOLD_HIP_CHECK(hipGetLastError());
    return FOLD_OK;
  });
}

int32_t fold_cross_create(const fold_cross_batch* batch, hipStream_t st, fold_cross** out) {
  return guarded([&]() -> int32_t {
    if (!out) return api_fail(FOLD_E_INVALID, "fold_cross_create: out is NULL");
    *out = nullptr;
    if (!batch) return api_fail(FOLD_E_INVALID, "fold_cross_create: batch is NULL");
    return cross_create(batch, st, out);
  });
}

int32_t fold_cross_free(fold_cross* cross) {
  return guarded([&]() -> int32_t {
    cross_destroy(cross);
    return FOLD_OK;
  });
}

int32_t fold_cross_workspace_size(const fold_cross* cross, size_t* fwd_bytes, size_t* bwd_bytes) {
  return guarded([&]() -> int32_t {
    if (!cross || !fwd_bytes || !bwd_bytes) return api_fail(FOLD_E_INVALID, "fold_cross_workspace_size: NULL argument");
    *fwd_bytes = cross_forward_bytes(cross->c);
    *bwd_bytes = cross_backward_bytes(cross->c);
    return FOLD_OK;
  });
}

}  // extern "C"

namespace {

// the checks that both directions share
int check_cross(const std::string& who, const fold_cross* cross, const Cols* in, int nin, const Cols* out, int nout,
                const uint8_t* mask, float scale, const void* stats, const void* ws, size_t need, size_t ws_bytes,
                bool stats_written) {
  const Cross& c = cross->c;
  int dev = -1;
  FOLD_HIP_CHECK(hipGetDevice(&dev));
  if (dev != c.device) return api_fail(FOLD_E_MISMATCH, who + ": the plan belongs to another device");
  // (below 2^127: the kernels multiply it by log2 e)
  if (!(scale > 0.f) || scale >= 0x1p127f) return api_fail(FOLD_E_INVALID, who + ": scale must be above 0 and below 2^127");
  const int es = c.dtype == FOLD_BF16 ? 2 : 4;
  const auto bad = [&](const Cols& m, bool needed) {
    if (!m.p) return needed && m.rows > 0;
    return m.ld < m.width || m.ld * es > INT32_MAX || (reinterpret_cast<uintptr_t>(m.p) & (es - 1)) != 0;
  };
  for (int i = 0; i < nin; ++i)
    if (bad(in[i], true)) return api_fail(FOLD_E_INVALID, who + ": NULL or misaligned matrix, or a stride below its width");
  for (int i = 0; i < nout; ++i)
    if (bad(out[i], false)) return api_fail(FOLD_E_INVALID, who + ": misaligned output, or a stride below its width");
  if (misaligned(ws)) return api_fail(FOLD_E_INVALID, who + ": the workspace must be 16-byte aligned");
  if (need > 0 && (!ws || ws_bytes < need))
    return api_fail(FOLD_E_MISMATCH, who + ": workspace smaller than fold_cross_workspace_size");
  const Cols lists{mask, 1, c.num_keys, 1};
  const Cols scratch{ws, 1, (int64_t)need, 1};
  const Cols stat{stats, c.heads, c.query_rows, c.heads};
  const auto meets = [&](const Cols& a, int ea, const Cols& b, int eb) {  // as plain runs of bytes
    const auto bytes = [](const Cols& m, int e) { return m.rows > 0 ? (size_t)((m.rows - 1) * m.ld + m.width) * e : (size_t)0; };
    return overlap({a.p, bytes(a, ea)}, {b.p, bytes(b, eb)});
  };
  for (int i = 0; i < nout; ++i) {
    for (int j = i + 1; j < nout; ++j)
      if (out[j].p && out[i].p && share(out[i], out[j], es)) return api_fail(FOLD_E_INVALID, who + ": outputs overlap");
    for (int j = 0; j < nin; ++j)
      if (out[i].p && in[j].p && share(out[i], in[j], es))
        return api_fail(FOLD_E_INVALID, who + ": an output overlaps another buffer");
    if (meets(out[i], es, lists, 1) || meets(out[i], es, scratch, 1) || meets(out[i], es, stat, 4))
      return api_fail(FOLD_E_INVALID, who + ": an output overlaps another buffer");
  }
  for (int j = 0; j < nin; ++j)
    if (meets(in[j], es, scratch, 1) || (stats_written && meets(in[j], es, stat, 4)))
      return api_fail(FOLD_E_INVALID, who + ": an output overlaps another buffer");
  if (meets(lists, 1, scratch, 1) || meets(stat, 4, scratch, 1) || (stats_written && meets(stat, 4, lists, 1)))
    return api_fail(FOLD_E_INVALID, who + ": an output overlaps another buffer");
  return FOLD_OK;
}

}  // namespace

extern "C" {

int32_t fold_cross_attend(const fold_cross* cross, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v,
                          int64_t ldv, const uint8_t* key_mask, float scale, void* out, int64_t ldo, float* lse, void* ws,
                          size_t ws_bytes, hipStream_t st) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_cross_attend");
    if (!cross) return api_fail(FOLD_E_INVALID, who + ": cross is NULL");
    const Cross& c = cross->c;
    const int wq = c.heads * c.head_dim, wk = c.kv_heads * c.head_dim;
    const Cols in[] = {{q, ldq, c.query_rows, wq}, {k, ldk, c.key_rows, wk}, {v, ldv, c.key_rows, wk}};
    const Cols outs[] = {{out, ldo, c.query_rows, wq}};
    const int rc = check_cross(who, cross, in, 3, outs, 1, key_mask, scale, lse, ws, cross_forward_bytes(c), ws_bytes, true);
    if (rc != FOLD_OK) return rc;
    if (c.num_queries == 0) return FOLD_OK;
    if (!out) return api_fail(FOLD_E_INVALID, who + ": NULL buffer");
    launch_cross(c, {q, ldq}, {k, ldk}, {v, ldv}, key_mask, scale, out, ldo, lse, ws, st);
    FOLD_HIP_CHECK(hipGetLastError());
    return FOLD_OK;
  });
}

int32_t fold_cross_backward(const fold_cross* cross, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v,
                            int64_t ldv, const uint8_t* key_mask, float scale, const void* out, int64_t ldo,
                            const float* lse, const void* dout, int64_t lddo, void* dq, int64_t lddq, void* dk, int64_t lddk,
                            void* dv, int64_t lddv, void* ws, size_t ws_bytes, hipStream_t st) {
  return guarded([&]() -> int32_t {
    const std::string who("fold_cross_backward");
    if (!cross) return api_fail(FOLD_E_INVALID, who + ": cross is NULL");
    const Cross& c = cross->c;
    if (!dq && !dk && !dv) return FOLD_OK;
    const int wq = c.heads * c.head_dim, wk = c.kv_heads * c.head_dim;
    const Cols in[] = {{q, ldq, c.query_rows, wq}, {k, ldk, c.key_rows, wk}, {v, ldv, c.key_rows, wk},
                       {out, ldo, c.query_rows, wq}, {dout, lddo, c.query_rows, wq}};
    const Cols outs[] = {{dq, lddq, c.query_rows, wq}, {dk, lddk, c.key_rows, wk}, {dv, lddv, c.key_rows, wk}};
    const int rc = check_cross(who, cross, in, 5, outs, 3, key_mask, scale, lse, ws, cross_backward_bytes(c), ws_bytes, false);
    if (rc != FOLD_OK) return rc;
    if (c.num_queries > 0 && !lse) return api_fail(FOLD_E_INVALID, who + ": NULL lse");
    launch_cross_backward(c, {q, ldq}, {k, ldk}, {v, ldv}, key_mask, scale, {out, ldo}, lse, {dout, lddo}, dq, lddq, dk, lddk,
                          dv, lddv, ws, st);
    FOLD_HIP_CHECK(hipGetLastError());
    return FOLD_OK;
  });
}

}  // extern "C"
