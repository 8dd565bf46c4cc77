// Host-only argument checks of the gradient norm, AdamW and 8-bit entry points. Plain C++ with no HIP dependency.
#include "update_checks.h"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <initializer_list>

namespace dit {

namespace {
constexpr int32_t MOST_TENSORS = 1 << 20;
constexpr int64_t MOST_ELEMENTS = int64_t(1) << 44;

dit_status check_dtype(int32_t dtype) {
  if (dtype != DIT_F32 && dtype != DIT_BF16) return set_error(DIT_ERR_INVALID_ARG, "dtype %d invalid", dtype);
  return DIT_OK;
}
bool aligned_to(const void* p, int32_t dtype) { return (uintptr_t)p % (dtype == DIT_BF16 ? 2 : 4) == 0; }

dit_status check_list(const void* list, int32_t n) {
  if (n < 0) return set_error(DIT_ERR_INVALID_ARG, "%d tensors", n);
  if (n > 0 && !list) return set_error(DIT_ERR_INVALID_ARG, "the list of tensors is NULL");
  if (n > MOST_TENSORS) return set_error(DIT_ERR_UNSUPPORTED, "%d tensors (at most 2^20)", n);
  return DIT_OK;
}
dit_status check_count(int64_t count, int32_t i, int64_t* total) {
  if (count < 0) return set_error(DIT_ERR_INVALID_ARG, "tensor %d has %lld elements", i, (long long)count);
  if (count > MOST_ELEMENTS || (*total += count) > MOST_ELEMENTS)
    return set_error(DIT_ERR_UNSUPPORTED, "more than 2^44 elements in all");
  return DIT_OK;
}
}  // namespace

int64_t update_chunk(int64_t total) {
  const int64_t unit = 2048;
  return unit * std::max<int64_t>(1, (total + unit * 8192 - 1) / (unit * 8192));
}

dit_status check_gradients(const dit_gradient* g, int32_t n, bool data, int64_t* total) {
  *total = 0;
  dit_status st = check_list(g, n);
  for (int32_t i = 0; !st && i < n; i++) {
    if ((st = check_dtype(g[i].dtype)) || (st = check_count(g[i].count, i, total))) return st;
    if (g[i].reserved) return set_error(DIT_ERR_INVALID_ARG, "tensor %d: reserved is not 0", i);
    if (data && g[i].count > 0 && (!g[i].data || !aligned_to(g[i].data, g[i].dtype)))
      return set_error(DIT_ERR_INVALID_ARG, "tensor %d is NULL or not aligned to its type", i);
  }
  return st;
}

dit_status check_adamw(const dit_adamw_config* c, const dit_adamw_tensor* t, int32_t n, bool step_dev, int64_t* total) {
  *total = 0;
  if (!c) return set_error(DIT_ERR_INVALID_ARG, "config is NULL");
  // (the kernel's numbers are fp32: an eps that rounds to 0 there would make 0 / 0 of a weight that has had no gradient)
  if (!(std::fabs(c->lr) <= FLT_MAX) || !(std::fabs(c->weight_decay) <= FLT_MAX))
    return set_error(DIT_ERR_DOMAIN, "lr or weight_decay not finite in fp32");
  // (a mean in fp32 times a beta that rounds to 1 there stays as it is)
  for (double beta : {c->beta1, c->beta2})
    if (!(beta >= 0.0 && beta < 1.0) || !((float)beta < 1.f))
      return set_error(DIT_ERR_DOMAIN, "beta1 and beta2 must be in [0, 1), also as fp32 numbers");
  if (c->eps != 0.0 && !(c->eps >= FLT_MIN && c->eps <= FLT_MAX))
    return set_error(DIT_ERR_DOMAIN, "eps must be 0 or a positive normal fp32 number");
  if (!step_dev && c->step < 1) return set_error(DIT_ERR_DOMAIN, "step %lld (from 1 on)", (long long)c->step);
  dit_status st = check_list(t, n);
  for (int32_t i = 0; !st && i < n; i++) {
    if ((st = check_dtype(t[i].param_dtype)) || (st = check_dtype(t[i].grad_dtype)) || (st = check_count(t[i].count, i, total)))
      return st;
    if (t[i].count == 0) continue;
    if (!t[i].param || !t[i].grad || !t[i].m || !t[i].v) return set_error(DIT_ERR_INVALID_ARG, "tensor %d: param/grad/m/v NULL", i);
    if (!aligned_to(t[i].param, t[i].param_dtype) || !aligned_to(t[i].grad, t[i].grad_dtype) || !aligned_to(t[i].m, DIT_F32) ||
        !aligned_to(t[i].v, DIT_F32) || !aligned_to(t[i].copy, DIT_BF16))
      return set_error(DIT_ERR_INVALID_ARG, "tensor %d is not aligned to its type", i);
  }
  return st;
}

dit_status check_quantize(int32_t rows, int32_t cols, int64_t x_row, int32_t dtype, int64_t q_row, bool values, int64_t values_row) {
  dit_status st = check_dtype(dtype);
  if (st) return st;
  if (rows < 0 || cols < 0) return set_error(DIT_ERR_INVALID_ARG, "negative size");
  const int64_t most = int64_t(1) << 40;   // (further than the device's memory: products with 2^31 rows do not overflow)
  for (int64_t r : {x_row, q_row, values ? values_row : (int64_t)cols}) {
    if (r < cols) return set_error(DIT_ERR_INVALID_ARG, "a row stride is below cols");
    if (r >= most / 1024) return set_error(DIT_ERR_UNSUPPORTED, "a row stride is 2^30 or more");
  }
  return DIT_OK;
}

dit_status check_int8(const dit_int8_config* c, bool given) {
  if (!c) return set_error(DIT_ERR_INVALID_ARG, "config is NULL");
  dit_status st = check_dtype(c->dtype);
  if (st) return st;
  if (c->act != DIT_ACT_NONE && c->act != DIT_ACT_GELU_TANH) return set_error(DIT_ERR_INVALID_ARG, "activation %d invalid", c->act);
  if (c->rows < 0 || c->out_features < 0) return set_error(DIT_ERR_INVALID_ARG, "negative size");
  if (c->in_features < 1) return set_error(DIT_ERR_SHAPE, "in_features %d must be positive", c->in_features);
  // 128 * 128 * 131071 is the largest sum that an int32 holds
  if (c->in_features >= 1 << 17) return set_error(DIT_ERR_UNSUPPORTED, "in_features %d (at most 131071)", c->in_features);
  if (c->x_row < c->in_features || c->w_row < c->in_features || c->y_row < c->out_features)
    return set_error(DIT_ERR_INVALID_ARG, "a row stride is below the row's elements");
  if (c->w_row % 16 || (given && c->x_row % 16)) return set_error(DIT_ERR_INVALID_ARG, "strides of int8 rows must be multiples of 16");
  // a tile's rows lie within 31 bits of its first
  if (c->w_row >= 1 << 23 || (given && c->x_row >= 1 << 23) || c->x_row >= 1 << 30 || c->y_row >= 1 << 30)
    return set_error(DIT_ERR_UNSUPPORTED, "a row stride is too large (int8 rows: below 2^23, others: below 2^30)");
  return DIT_OK;
}

}  // namespace dit
