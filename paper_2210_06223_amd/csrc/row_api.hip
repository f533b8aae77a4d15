// extern "C" boundary of the row operators: argument validation and launches only.
#include <initializer_list>

#include "row_ops.hpp"

using namespace lasnet;

namespace {

constexpr int64_t kMaxRows = 1ll << 30;          // row and slot numbers are 32-bit inside the kernels, with room for a tile beyond the last
constexpr int32_t kMaxCols = 1 << 20;
constexpr int kMaxExperts = 4096, kMaxSlots = 64;

int bytes_of(int dtype) { return dtype == LASNET_F32 ? 4 : dtype == LASNET_BF16 ? 2 : 1; }

// Rows of one of the allowed types (bits 1 << dtype).
int check_rows(const lasnet_rows* t, unsigned types) {
  if (!t) return LASNET_EINVAL;
  if (t->dtype < 0 || t->dtype > 2) return LASNET_EINVAL;
  if (!(types >> t->dtype & 1)) return LASNET_EUNSUPPORTED;
  if (t->rows < 0 || t->cols <= 0) return LASNET_ESHAPE;
  if (t->stride != 0 && t->stride < t->cols) return LASNET_ESHAPE;
  if (t->rows > 0 && !t->data) return LASNET_EINVAL;
  if (t->rows > kMaxRows || t->cols > kMaxCols || t->stride > (1ll << 40)) return LASNET_EUNSUPPORTED;
  return LASNET_OK;
}
// ... of the type and shape of another
int check_like(const lasnet_rows* t, const lasnet_rows* as) {
  const int s = check_rows(t, 7);
  if (s != LASNET_OK) return s;
  return t->dtype != as->dtype || t->rows != as->rows || t->cols != as->cols ? LASNET_ESHAPE : LASNET_OK;
}
int check_experts(int k, int E) {
  if (k <= 0 || E <= 0) return LASNET_EINVAL;
  return k > kMaxSlots || E > kMaxExperts ? LASNET_EUNSUPPORTED : LASNET_OK;
}
RowsArg arg(const lasnet_rows* t) {
  if (!t) return RowsArg{nullptr, 0};
  return RowsArg{(unsigned char*)t->data, (t->stride ? t->stride : t->cols) * bytes_of(t->dtype)};
}
constexpr unsigned kFloats = 1u << LASNET_F32 | 1u << LASNET_BF16;

bool same(const lasnet_rows* a, const lasnet_rows* b) { return a && b && a->data && a->data == b->data; }
// in place: the same rows, not merely the same address
bool may_share(const lasnet_rows* a, const lasnet_rows* b) {
  return !same(a, b) || (arg(a).pitch == arg(b).pitch && a->dtype == b->dtype);
}
const void* at(const lasnet_rows* t) { return t ? t->data : nullptr; }
// whether an output lies where another one or an input does (pairs that may be the same rows are left out of the call)
bool clash(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs) {
  for (const void* const* o = outputs.begin(); o != outputs.end(); ++o) {
    if (!*o) continue;
    for (const void* const* p = o + 1; p != outputs.end(); ++p)
      if (*p == *o) return true;
    for (const void* i : inputs)
      if (i == *o) return true;
  }
  return false;
}
int enqueued(hipError_t e) { return e == hipSuccess ? LASNET_OK : LASNET_EHIP; }

#define CHECK(call)                      \
  do {                                   \
    const int s_ = (call);               \
    if (s_ != LASNET_OK) return s_;      \
  } while (0)

// tiles of a product's grid, in all
int check_tiles(int64_t rows, int E, int32_t ni, int32_t nj) {
  const int64_t by_rows = rows / 128 + E + 1, by_matrix = (int64_t)E * ((nj + 127) / 128);
  const int64_t most = (by_rows > by_matrix ? by_rows : by_matrix) * ((ni + 127) / 128);
  return most < (1 << 23) ? LASNET_OK : LASNET_EUNSUPPORTED;
}

}  // namespace

extern "C" {

int lasnet_norm_rows(const lasnet_rows* x, const lasnet_rows* residual, const float* weight, float eps, const lasnet_rows* sum_out,
                     const lasnet_rows* out, uint8_t* scale, float* rstd_out, void* hip_stream) {
  CHECK(check_rows(x, kFloats));
  if (residual) CHECK(check_like(residual, x));
  if (sum_out) CHECK(check_like(sum_out, x));
  CHECK(check_rows(out, 7));
  const bool q = out->dtype == LASNET_E4M3;
  if (out->rows != x->rows || out->cols != x->cols || (!q && out->dtype != x->dtype)) return LASNET_ESHAPE;
  if (!weight || !(eps >= 0.f)) return LASNET_EINVAL;
  if (x->rows > 0 && q != (scale != nullptr)) return LASNET_EINVAL;
  if (x->cols > kNormCols) return LASNET_EUNSUPPORTED;
  if (!may_share(out, x) || !may_share(out, residual) || !may_share(sum_out, x) || !may_share(sum_out, residual) ||
      clash({at(out), at(sum_out), scale, rstd_out}, {weight}) || clash({scale, rstd_out}, {at(x), at(residual)}))
    return LASNET_EALIAS;
  if (!device_ok()) return LASNET_EHIP;
  if (x->rows == 0) return LASNET_OK;
  return enqueued(launch_norm_rows(x->dtype, out->dtype, x->rows, x->cols, arg(x), arg(residual), weight, eps, arg(sum_out), arg(out), scale,
                                   rstd_out, (hipStream_t)hip_stream));
}

size_t lasnet_norm_rows_backward_workspace_bytes(int64_t rows, int cols) {
  if (rows <= 0 || rows > kMaxRows || cols <= 0 || cols > kNormCols) return 0;
  return norm_backward_workspace_bytes(rows, cols);
}

int lasnet_norm_rows_backward(const lasnet_rows* dy, const lasnet_rows* s, const float* weight, const float* rstd, const lasnet_rows* dsum,
                              const lasnet_rows* dx, float* dweight, void* workspace, size_t workspace_bytes, void* hip_stream) {
  CHECK(check_rows(s, kFloats));
  CHECK(check_like(dy, s));
  if (dsum) CHECK(check_like(dsum, s));
  CHECK(check_like(dx, s));
  if (!weight || !dweight || (s->rows > 0 && !rstd)) return LASNET_EINVAL;
  if (s->cols > kNormCols) return LASNET_EUNSUPPORTED;
  const size_t need = lasnet_norm_rows_backward_workspace_bytes(s->rows, s->cols);
  if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))) return LASNET_EINVAL;
  if (!may_share(dx, dy) || !may_share(dx, dsum) || clash({at(dx), dweight, workspace}, {at(s), weight, rstd}) ||
      clash({dweight, workspace}, {at(dy), at(dsum)}))
    return LASNET_EALIAS;
  if (!device_ok()) return LASNET_EHIP;
  return enqueued(launch_norm_rows_backward(s->dtype, s->rows, s->cols, arg(dy), arg(s), weight, rstd, arg(dsum), arg(dx), dweight, workspace,
                                            (hipStream_t)hip_stream));
}

size_t lasnet_route_workspace_bytes(int64_t tokens, int k, int E) {
  if (tokens <= 0 || tokens > kMaxRows || check_experts(k, E) != LASNET_OK || tokens * k > kMaxRows) return 0;
  return route_workspace_bytes(tokens * k, E);
}

int lasnet_route(const int32_t* experts, int64_t tokens, int k, int E, int32_t* offsets, int32_t* order, int32_t* position, void* workspace,
                 size_t workspace_bytes, void* hip_stream) {
  if (tokens < 0) return LASNET_ESHAPE;
  CHECK(check_experts(k, E));
  if (tokens > kMaxRows || tokens * k > kMaxRows) return LASNET_EUNSUPPORTED;
  if (!offsets || (tokens > 0 && (!experts || !position))) return LASNET_EINVAL;
  const size_t need = lasnet_route_workspace_bytes(tokens, k, E);
  if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))) return LASNET_EINVAL;
  if (tokens > 0 && clash({offsets, order, position, workspace}, {experts})) return LASNET_EALIAS;
  if (!device_ok()) return LASNET_EHIP;
  return enqueued(launch_route(experts, tokens * k, E, offsets, order, position, workspace, (hipStream_t)hip_stream));
}

int lasnet_dispatch_rows(const lasnet_rows* x, const uint8_t* scale, const int32_t* position, const int32_t* offsets, int k, int E,
                         const lasnet_rows* out, uint8_t* out_scale, void* hip_stream) {
  CHECK(check_rows(x, 7));
  CHECK(check_rows(out, 7));
  CHECK(check_experts(k, E));
  if (out->dtype != x->dtype || out->cols != x->cols || out->rows != x->rows * k) return LASNET_ESHAPE;
  if (x->rows > 0 && (!position || !offsets || (scale != nullptr) != (out_scale != nullptr))) return LASNET_EINVAL;
  if (clash({at(out), out_scale}, {at(x), scale, position, offsets})) return LASNET_EALIAS;
  if (!device_ok()) return LASNET_EHIP;
  if (x->rows == 0) return LASNET_OK;
  return enqueued(launch_dispatch(x->rows, k, E, x->cols * bytes_of(x->dtype), arg(x), scale, position, offsets, arg(out), out_scale,
                                  (hipStream_t)hip_stream));
}

int lasnet_combine_rows(const lasnet_rows* y, const float* weights, const int32_t* position, int k, const lasnet_rows* base,
                        const lasnet_rows* out, void* hip_stream) {
  CHECK(check_rows(y, kFloats));
  CHECK(check_rows(out, kFloats));
  CHECK(check_experts(k, 1));
  if (base) CHECK(check_like(base, out));
  if (out->dtype != y->dtype || out->cols != y->cols || y->rows != out->rows * k) return LASNET_ESHAPE;
  if (out->rows > 0 && !position) return LASNET_EINVAL;
  if (!may_share(out, base) || clash({at(out)}, {at(y), weights, position})) return LASNET_EALIAS;
  if (!device_ok()) return LASNET_EHIP;
  if (out->rows == 0) return LASNET_OK;
  return enqueued(launch_combine(y->dtype, out->rows, k, y->cols, arg(y), weights, position, arg(base), arg(out), (hipStream_t)hip_stream));
}

int lasnet_combine_rows_backward(const lasnet_rows* dout, const lasnet_rows* y, const float* weights, const int32_t* position,
                                 const int32_t* offsets, int k, int E, const lasnet_rows* dy, float* dweights, void* hip_stream) {
  CHECK(check_rows(dout, kFloats));
  CHECK(check_rows(y, kFloats));
  CHECK(check_experts(k, E));
  CHECK(check_like(dy, y));
  if (dout->dtype != y->dtype || dout->cols != y->cols || y->rows != dout->rows * k) return LASNET_ESHAPE;
  if (dout->rows > 0 && (!position || !offsets)) return LASNET_EINVAL;
  if (!may_share(dy, y) || clash({at(dy), dweights}, {at(dout), weights, position, offsets}) || clash({dweights}, {at(y)})) return LASNET_EALIAS;
  if (!device_ok()) return LASNET_EHIP;
  if (dout->rows == 0) return LASNET_OK;
  return enqueued(launch_combine_backward(y->dtype, dout->rows, k, E, y->cols, arg(dout), arg(y), weights, position, offsets, arg(dy), dweights,
                                          (hipStream_t)hip_stream));
}

int lasnet_expert_product(const lasnet_rows* x, const uint8_t* scale, const int32_t* offsets, int E, const void* W, const float* wscale,
                          const lasnet_rows* out, uint32_t flags, void* hip_stream) {
  CHECK(check_rows(x, 1u << LASNET_BF16 | 1u << LASNET_E4M3));
  CHECK(check_rows(out, 1u << LASNET_BF16));
  CHECK(check_experts(1, E));
  if (out->rows != x->rows) return LASNET_ESHAPE;
  if (!offsets || !W || (flags & ~(uint32_t)LASNET_POST_RELU)) return LASNET_EINVAL;
  if (x->dtype != LASNET_E4M3 && (scale || wscale)) return LASNET_EINVAL;
  CHECK(check_tiles(x->rows, E, out->cols, 0));
  if (clash({at(out)}, {at(x), scale, offsets, W, wscale})) return LASNET_EALIAS;
  if (!device_ok()) return LASNET_EHIP;
  if (x->rows == 0) return LASNET_OK;
  return enqueued(launch_expert_product(x->dtype, x->rows, E, out->cols, x->cols, arg(x), scale, offsets, W, wscale, arg(out),
                                        (flags & LASNET_POST_RELU) != 0, (hipStream_t)hip_stream));
}

int lasnet_expert_product_dx(const lasnet_rows* dy, const int32_t* offsets, int E, const void* W, const lasnet_rows* dx, void* hip_stream) {
  CHECK(check_rows(dy, 1u << LASNET_BF16));
  CHECK(check_rows(dx, 1u << LASNET_BF16));
  CHECK(check_experts(1, E));
  if (dx->rows != dy->rows) return LASNET_ESHAPE;
  if (!offsets || !W) return LASNET_EINVAL;
  CHECK(check_tiles(dy->rows, E, dx->cols, 0));
  if (clash({at(dx)}, {at(dy), offsets, W})) return LASNET_EALIAS;
  if (!device_ok()) return LASNET_EHIP;
  if (dy->rows == 0) return LASNET_OK;
  return enqueued(launch_expert_product_dx(dy->rows, E, dy->cols, dx->cols, arg(dy), offsets, W, arg(dx), (hipStream_t)hip_stream));
}

size_t lasnet_expert_product_dw_workspace_bytes(int64_t rows, int E, int n, int k) {
  if (rows <= 0 || rows > kMaxRows || check_experts(1, E) != LASNET_OK || n <= 0 || k <= 0 || check_tiles(rows, E, k, n) != LASNET_OK) return 0;
  return product_dw_workspace_bytes(rows, E, n, k);
}

int lasnet_expert_product_dw_ex(const lasnet_rows* dy, const lasnet_rows* x, const int32_t* offsets, int E, void* dW, int dw_dtype,
                                void* workspace, size_t workspace_bytes, void* hip_stream) {
  CHECK(check_rows(dy, 1u << LASNET_BF16));
  CHECK(check_rows(x, 1u << LASNET_BF16));
  CHECK(check_experts(1, E));
  if (x->rows != dy->rows) return LASNET_ESHAPE;
  if (!offsets || !dW || (dw_dtype != LASNET_F32 && dw_dtype != LASNET_BF16)) return LASNET_EINVAL;
  CHECK(check_tiles(x->rows, E, x->cols, dy->cols));
  if (workspace && (workspace_bytes < lasnet_expert_product_dw_workspace_bytes(x->rows, E, dy->cols, x->cols) || ((uintptr_t)workspace & 255))) return LASNET_EINVAL;
  if (clash({dW, workspace}, {at(x), at(dy), offsets})) return LASNET_EALIAS;
  if (!device_ok()) return LASNET_EHIP;
  return enqueued(launch_expert_product_dw(x->rows, E, dy->cols, x->cols, arg(dy), arg(x), offsets, dW, dw_dtype == LASNET_F32, workspace,
                                           (hipStream_t)hip_stream));
}

int lasnet_expert_product_dw(const lasnet_rows* dy, const lasnet_rows* x, const int32_t* offsets, int E, void* dW, int dw_dtype,
                             void* hip_stream) {
  return lasnet_expert_product_dw_ex(dy, x, offsets, E, dW, dw_dtype, nullptr, 0, hip_stream);
}

}  // extern "C"
