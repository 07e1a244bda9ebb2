// C ABI of the operators of a model's end (include/adapm.h): argument checks, workspace layouts and launches.  The calls keep
// nothing between them, allocate nothing and never wait for the device, so they can be captured into a HIP graph.
#include "ops_plan.h"

#include <cmath>

using namespace adapm;

namespace {

#define HIP_TRY(expr)                                                                      \
  do {                                                                                     \
    hipError_t e_ = (expr);                                                                \
    if (e_ != hipSuccess) return fail(ADAPM_EHIP, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

int esize(int32_t dt) { return dt == ADAPM_BF16 ? 2 : dt == ADAPM_E4M3 ? 1 : 4; }
bool is_float(int32_t dt) { return dt == ADAPM_F32 || dt == ADAPM_BF16; }

// a matrix of activations that has to be there (rows > 0) with `cols` elements a row
adapm_status_t check_rows(const char* name, const adapm_rows_t& r, int64_t rows, int64_t cols, int32_t dtype) {
  if (rows == 0) return ADAPM_OK;
  if (!r.data) return fail(ADAPM_EINVAL, "%s is null", name);
  if ((uintptr_t)r.data & (esize(dtype) - 1)) return fail(ADAPM_EINVAL, "%s is not aligned to its elements", name);
  if (r.stride < cols || r.stride >= (1ll << 40)) return fail(ADAPM_EINVAL, "%s: row stride %lld, rows of %lld", name, (long long)r.stride, (long long)cols);
  return ADAPM_OK;
}
adapm_status_t check_ptr(const char* name, const void* p, size_t align) {
  if (!p) return fail(ADAPM_EINVAL, "%s is null", name);
  if ((uintptr_t)p & (align - 1)) return fail(ADAPM_EINVAL, "%s is not %zu-byte aligned", name, align);
  return ADAPM_OK;
}
Rows rows_of(const adapm_rows_t& r) { return Rows{r.data, r.stride}; }

#define TRY(expr)                               \
  do {                                          \
    const adapm_status_t s_ = (expr);           \
    if (s_ != ADAPM_OK) return s_;              \
  } while (0)

// null: no dropout
adapm_status_t drop_of(const adapm_dropout_t* d, int64_t rows, int64_t cols, DropDev* out) {
  *out = DropDev{0, 0, 0, nullptr, 0, 1.f};
  if (!d) return ADAPM_OK;
  if (!(d->p >= 0.f && d->p < 1.f)) return fail(ADAPM_EINVAL, "dropout probability %g not in [0, 1)", (double)d->p);
  if (d->reserved) return fail(ADAPM_EINVAL, "dropout: reserved is %d, 0 is wanted", d->reserved);
  if ((uintptr_t)d->offset_dev & 7) return fail(ADAPM_EINVAL, "offset_dev is not 8-byte aligned");
  if (rows > (1ll << 32) || cols > (1ll << 34)) return fail(ADAPM_EINVAL, "dropout: too many rows or columns for its counter");
  // 16 random bits decide: the probability is the nearest multiple of 2^-16, and the scale is that probability's
  const double t = std::floor(65536.0 * (double)d->p + 0.5);
  out->thr = t > 65535.0 ? 65535u : (uint32_t)t;
  out->scale = (float)(65536.0 / (65536.0 - out->thr));
  out->k0 = (uint32_t)d->seed;
  out->k1 = (uint32_t)(d->seed >> 32);
  out->offset = d->offset;
  out->offset_dev = d->offset_dev;
  return ADAPM_OK;
}

constexpr int64_t NORM_COLS = 16384;      // a row stays in the registers of one workgroup

adapm_status_t check_norm(const adapm_norm_t* n) {
  if (!n) return fail(ADAPM_EINVAL, "norm is null");
  if (n->rows < 0 || n->rows > (1ll << 31)) return fail(ADAPM_EINVAL, "rows %lld out of range", (long long)n->rows);
  if (n->cols < 1 || n->cols > NORM_COLS) return fail(ADAPM_EINVAL, "cols %lld not in [1, %lld]", (long long)n->cols, (long long)NORM_COLS);
  if (!is_float(n->dtype) || !is_float(n->weight_dtype)) return fail(ADAPM_EINVAL, "unknown dtype");
  if (n->reserved) return fail(ADAPM_EINVAL, "norm: reserved is %d, 0 is wanted", n->reserved);
  if (!(n->eps >= 0.f) || !std::isfinite(n->eps)) return fail(ADAPM_EINVAL, "eps must be finite and >= 0");
  return ADAPM_OK;
}

adapm_status_t check_head(const adapm_head_t* h) {
  if (!h) return fail(ADAPM_EINVAL, "head is null");
  if (h->rows < 0 || h->rows > (1ll << 22)) return fail(ADAPM_EINVAL, "rows %lld not in [0, 2^22]", (long long)h->rows);
  if (h->vocab < 1 || h->vocab > (1ll << 21)) return fail(ADAPM_EINVAL, "vocab %lld not in [1, 2^21]", (long long)h->vocab);
  if (h->cols < 1 || h->cols > (1ll << 16)) return fail(ADAPM_EINVAL, "cols %lld not in [1, 2^16]", (long long)h->cols);
  if (!is_float(h->dtype)) return fail(ADAPM_EINVAL, "unknown dtype %d", h->dtype);
  if (h->reduction != ADAPM_REDUCE_SUM && h->reduction != ADAPM_REDUCE_MEAN) return fail(ADAPM_EINVAL, "unknown reduction %d", h->reduction);
  if (h->reserved) return fail(ADAPM_EINVAL, "head: reserved is %d, 0 is wanted", h->reserved);
  if (!std::isfinite(h->scale)) return fail(ADAPM_EINVAL, "scale is not finite");
  return ADAPM_OK;
}

// The products' tiles are one dimension of a grid, which holds less than 2^32 threads.
constexpr int64_t GRID_THREADS = 1ll << 32;

// Rows that are whole 16-byte vectors are read where they are; others are copied into the workspace.
bool in_place(const adapm_head_t* h, const adapm_rows_t& w) {
  const int v = 16 / esize(h->dtype);
  return h->cols % v == 0 && w.stride % v == 0 && ((uintptr_t)w.data & 15) == 0;
}

adapm_status_t head_args(const adapm_head_t* h, adapm_rows_t x, adapm_rows_t weight, const int64_t* targets, const float* row_weight,
                         const void* workspace, size_t workspace_bytes, bool backward, bool want_dx, HeadDev* out) {
  TRY(check_rows("x", x, h->rows, h->cols, h->dtype));
  TRY(check_rows("weight", weight, 1, h->cols, h->dtype));
  if (weight.stride > (1ll << 21)) return fail(ADAPM_EINVAL, "weight: row stride %lld above 2^21", (long long)weight.stride);
  if (h->rows) {
    TRY(check_ptr("targets", targets, 8));
    if (row_weight) TRY(check_ptr("row_weight", row_weight, 4));
    TRY(check_ptr("workspace", workspace, 256));
  }
  HeadDev d;
  d.rows = h->rows;
  d.vocab = h->vocab;
  d.cols = (int)h->cols;
  d.bf16 = h->dtype == ADAPM_BF16;
  const int step = 128 / esize(h->dtype);
  d.pitch = (int)((h->cols + step - 1) / step * step);
  d.mean = h->reduction == ADAPM_REDUCE_MEAN;
  d.scale = h->scale;
  d.x = rows_of(x);
  d.w = rows_of(weight);
  d.dx = d.dw = Rows{nullptr, 0};
  d.targets = targets;
  d.row_weight = row_weight;
  d.upstream = nullptr;
  d.loss = d.row_loss = d.lse = nullptr;
  d.ws = (char*)const_cast<void*>(workspace);
  d.w_packed = !in_place(h, weight);
  d.twin_rows = backward ? head_twin_rows(d.bf16, row_weight != nullptr) : 0;
  const bool as_it_is = in_place(h, x) && x.stride <= (1ll << 21);
  d.direct = !backward && head_direct(h->rows) && as_it_is;
  d.whole = head_whole(h->rows) && as_it_is;
  d.lay = head_layout(h->rows, h->vocab, h->cols, d.bf16, d.w_packed, backward, want_dx, d.twin_rows);
  if (d.lay.threads >= GRID_THREADS) return fail(ADAPM_EINVAL, "rows %lld x vocab %lld: too many for one call", (long long)h->rows, (long long)h->vocab);
  if (h->rows && workspace_bytes < (size_t)d.lay.bytes)
    return fail(ADAPM_EINVAL, "workspace of %zu bytes, %lld are needed", workspace_bytes, (long long)d.lay.bytes);
  *out = d;
  return ADAPM_OK;
}

}  // namespace

extern "C" {

adapm_status_t adapm_dropout(adapm_rows_t y, adapm_rows_t x, adapm_rows_t residual, int64_t rows, int64_t cols, int32_t dtype,
                             const adapm_dropout_t* drop, void* stream) {
  if (rows < 0 || cols < 1 || rows > (1ll << 32) || cols > (1ll << 34) || (rows && cols > (1ll << 46) / rows))
    return fail(ADAPM_EINVAL, "rows %lld / cols %lld out of range", (long long)rows, (long long)cols);
  if (!is_float(dtype)) return fail(ADAPM_EINVAL, "unknown dtype %d", dtype);
  if (!drop) return fail(ADAPM_EINVAL, "drop is null");
  TRY(check_rows("y", y, rows, cols, dtype));
  TRY(check_rows("x", x, rows, cols, dtype));
  if (residual.data) TRY(check_rows("residual", residual, rows, cols, dtype));
  DropDev d;
  TRY(drop_of(drop, rows, cols, &d));
  if (!rows) return ADAPM_OK;
  launch_dropout(dtype == ADAPM_BF16, rows_of(y), rows_of(x), rows_of(residual), rows, cols, d, (hipStream_t)stream);
  HIP_TRY(hipGetLastError());
  return ADAPM_OK;
}

adapm_status_t adapm_norm_forward(const adapm_norm_t* n, adapm_rows_t x, adapm_rows_t residual, adapm_rows_t h, const void* weight,
                                  adapm_rows_t y, float* y_scale, float* rstd, const adapm_dropout_t* drop, void* stream) {
  TRY(check_norm(n));
  if (!is_float(n->y_dtype) && n->y_dtype != ADAPM_E4M3) return fail(ADAPM_EINVAL, "unknown y_dtype %d", n->y_dtype);
  if (is_float(n->y_dtype) && n->y_dtype != n->dtype) return fail(ADAPM_EINVAL, "y_dtype has to be dtype or ADAPM_E4M3");
  TRY(check_rows("x", x, n->rows, n->cols, n->dtype));
  if (residual.data) TRY(check_rows("residual", residual, n->rows, n->cols, n->dtype));
  NormDev d = {};
  TRY(drop_of(drop, n->rows, n->cols, &d.drop));
  if (h.data) TRY(check_rows("h", h, n->rows, n->cols, n->dtype));
  else if (n->rows && (residual.data || d.drop.thr)) return fail(ADAPM_EINVAL, "h is null: the sum with the residual, or what dropout leaves, is needed by the backward pass");
  TRY(check_ptr("weight", weight, esize(n->weight_dtype)));
  TRY(check_rows("y", y, n->rows, n->cols, n->y_dtype));
  if (n->rows) {
    TRY(check_ptr("rstd", rstd, 4));
    if (n->y_dtype == ADAPM_E4M3) TRY(check_ptr("y_scale", y_scale, 4));
  }
  if (!n->rows) return ADAPM_OK;
  if (y.data == h.data) return fail(ADAPM_EINVAL, "y is h");
  d.rows = n->rows;
  d.cols = (int)n->cols;
  d.eps = n->eps;
  d.x = rows_of(x);
  d.residual = rows_of(residual);
  d.h = rows_of(h);
  d.y = rows_of(y);
  d.weight = weight;
  d.y_scale = y_scale;
  d.rstd = rstd;
  d.w_bf16 = n->weight_dtype == ADAPM_BF16;
  d.out8 = n->y_dtype == ADAPM_E4M3;
  launch_norm_forward(n->dtype == ADAPM_BF16, d, (hipStream_t)stream);
  HIP_TRY(hipGetLastError());
  return ADAPM_OK;
}

size_t adapm_norm_workspace_bytes(const adapm_norm_t* n) {
  if (check_norm(n) != ADAPM_OK) return 0;
  return (size_t)norm_backward_groups(n->rows, n->cols) * (size_t)n->cols * 4;
}

adapm_status_t adapm_norm_backward(const adapm_norm_t* n, adapm_rows_t dy, adapm_rows_t dh, adapm_rows_t h, const void* weight,
                                   const float* rstd, adapm_rows_t dx, adapm_rows_t dresidual, void* dweight,
                                   const adapm_dropout_t* drop, void* workspace_dev, void* stream) {
  TRY(check_norm(n));
  if (!is_float(n->grad_dtype)) return fail(ADAPM_EINVAL, "unknown grad_dtype %d", n->grad_dtype);
  TRY(check_rows("dy", dy, n->rows, n->cols, n->dtype));
  TRY(check_rows("h", h, n->rows, n->cols, n->dtype));
  TRY(check_rows("dx", dx, n->rows, n->cols, n->dtype));
  if (dh.data) TRY(check_rows("dh", dh, n->rows, n->cols, n->dtype));
  if (dresidual.data) TRY(check_rows("dresidual", dresidual, n->rows, n->cols, n->dtype));
  TRY(check_ptr("weight", weight, esize(n->weight_dtype)));
  TRY(check_ptr("dweight", dweight, esize(n->grad_dtype)));
  if (n->rows) TRY(check_ptr("rstd", rstd, 4));
  TRY(check_ptr("workspace_dev", workspace_dev, 256));
  NormDev d = {};
  TRY(drop_of(drop, n->rows, n->cols, &d.drop));
  if (n->rows && d.drop.thr && dx.data == dresidual.data) return fail(ADAPM_EINVAL, "with dropout dx and dresidual differ");
  d.rows = n->rows;
  d.cols = (int)n->cols;
  d.dy = rows_of(dy);
  d.dh = rows_of(dh);
  d.h = rows_of(h);
  d.dx = rows_of(dx);
  d.dres = rows_of(dresidual);
  d.weight = weight;
  d.dweight = dweight;
  d.rstd = const_cast<float*>(rstd);
  d.partial = (float*)workspace_dev;
  d.w_bf16 = n->weight_dtype == ADAPM_BF16;
  d.g_bf16 = n->grad_dtype == ADAPM_BF16;
  launch_norm_backward(n->dtype == ADAPM_BF16, d, (hipStream_t)stream);
  HIP_TRY(hipGetLastError());
  return ADAPM_OK;
}

size_t adapm_head_workspace_bytes(const adapm_head_t* h, adapm_rows_t weight, int32_t backward) {
  if (check_head(h) != ADAPM_OK) return 0;
  // for a call with or without weights on its rows
  const bool bf16 = h->dtype == ADAPM_BF16, packed = !in_place(h, weight);
  int64_t bytes = 0;
  for (int weighted = 0; weighted < (backward ? 2 : 1); ++weighted) {
    const HeadLayout l = head_layout(h->rows, h->vocab, h->cols, bf16, packed, backward != 0, true, backward ? head_twin_rows(bf16, weighted != 0) : 0);
    if (l.threads >= GRID_THREADS) return 0;
    bytes = l.bytes > bytes ? l.bytes : bytes;
  }
  return (size_t)bytes;
}

adapm_status_t adapm_head_loss(const adapm_head_t* h, adapm_rows_t x, adapm_rows_t weight, const int64_t* targets,
                               const float* row_weight, float* loss, float* row_loss, float* lse, void* workspace_dev,
                               size_t workspace_bytes, void* stream) {
  TRY(check_head(h));
  HeadDev d;
  TRY(head_args(h, x, weight, targets, row_weight, workspace_dev, workspace_bytes, false, false, &d));
  TRY(check_ptr("loss", loss, 4));
  if (h->rows) {
    TRY(check_ptr("row_loss", row_loss, 4));
    TRY(check_ptr("lse", lse, 4));
  }
  d.loss = loss;
  d.row_loss = row_loss;
  d.lse = lse;
  launch_head_loss(d, (hipStream_t)stream);
  HIP_TRY(hipGetLastError());
  return ADAPM_OK;
}

adapm_status_t adapm_head_backward(const adapm_head_t* h, adapm_rows_t x, adapm_rows_t weight, const int64_t* targets,
                                   const float* row_weight, const float* lse, const float* upstream, adapm_rows_t dx,
                                   adapm_rows_t dweight, void* workspace_dev, size_t workspace_bytes, void* stream) {
  TRY(check_head(h));
  if (!dx.data && !dweight.data) return fail(ADAPM_EINVAL, "dx and dweight are both null");
  HeadDev d;
  TRY(head_args(h, x, weight, targets, row_weight, workspace_dev, workspace_bytes, true, dx.data != nullptr, &d));
  if (h->rows) TRY(check_ptr("lse", lse, 4));
  if (upstream) TRY(check_ptr("upstream", upstream, 4));
  if (dx.data) TRY(check_rows("dx", dx, h->rows, h->cols, h->dtype));
  if (dweight.data) TRY(check_rows("dweight", dweight, 1, h->cols, h->dtype));
  // W and the packed x are read while gradients are written
  if (dweight.data && (dweight.data == weight.data || (h->rows && dweight.data == x.data))) return fail(ADAPM_EINVAL, "dweight is an input");
  if (dx.data && h->rows && (dx.data == weight.data || dx.data == dweight.data)) return fail(ADAPM_EINVAL, "dx is W or dweight");
  d.lse = const_cast<float*>(lse);
  d.upstream = upstream;
  d.dx = rows_of(dx);
  d.dw = rows_of(dweight);
  launch_head_backward(d, (hipStream_t)stream);
  HIP_TRY(hipGetLastError());
  return ADAPM_OK;
}

}  // extern "C"
