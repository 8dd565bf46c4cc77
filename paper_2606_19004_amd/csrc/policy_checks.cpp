// Host-only argument checks of packed attention, the gated norm and the policy loss. Plain C++ with no HIP dependency.
#include "policy_checks.h"

#include <cmath>
#include <initializer_list>

namespace dit {

namespace {
int64_t esize_of(int32_t dtype) { return dtype == DIT_BF16 ? 2 : 4; }

dit_status check_strides(const char* name, int64_t row, int64_t head, int32_t d, int32_t dtype) {
  if (row < d || head < 0) return set_error(DIT_ERR_INVALID_ARG, "%s_row must be at least head_dim, %s_head >= 0", name, name);
  // (bounded before anything is multiplied by them; 2^40 elements are further than the device's memory)
  if (row >= (1 << 24)) return set_error(DIT_ERR_UNSUPPORTED, "%s_row %lld is 2^24 or more", name, (long long)row);
  if (head >= (int64_t(1) << 40)) return set_error(DIT_ERR_UNSUPPORTED, "%s_head %lld is 2^40 or more", name, (long long)head);
  if ((row * esize_of(dtype)) % 16 || (head * esize_of(dtype)) % 16)
    return set_error(DIT_ERR_INVALID_ARG, "%s strides must keep 16-byte rows", name);
  return DIT_OK;
}

// whether the (row, head) pieces of a written tensor are apart
dit_status check_apart(const char* name, int64_t row, int64_t head, int32_t d, int64_t rows, int64_t heads) {
  if (heads <= 1 || rows <= 0) return DIT_OK;
  const bool heads_inside = head >= d && head <= row && row >= (heads - 1) * head + d;   // (row is below 2^24: no overflow)
  const bool rows_inside = head >= (rows - 1) * row + d;
  if (heads_inside || rows_inside || (rows == 1 && head >= d)) return DIT_OK;
  return set_error(DIT_ERR_INVALID_ARG, "%s strides make rows of different heads overlap", name);
}
}  // namespace

dit_status check_packed(const dit_packed_config* c) {
  if (!c) return set_error(DIT_ERR_INVALID_ARG, "config is NULL");
  if (c->dtype != DIT_F32 && c->dtype != DIT_BF16) return set_error(DIT_ERR_INVALID_ARG, "dtype %d invalid", c->dtype);
  if (c->sequences < 0 || c->total_q < 0 || c->total_k < 0 || c->max_q < 0)
    return set_error(DIT_ERR_INVALID_ARG, "negative size");
  if (c->heads <= 0 || c->kv_heads <= 0 || c->heads % c->kv_heads)
    return set_error(DIT_ERR_SHAPE, "heads %d must be a positive multiple of kv_heads %d", c->heads, c->kv_heads);
  if (c->head_dim != 64 && c->head_dim != 128) return set_error(DIT_ERR_UNSUPPORTED, "head_dim %d (64 or 128)", c->head_dim);
  if (!(c->scale > 0.f) || !std::isfinite(c->scale)) return set_error(DIT_ERR_INVALID_ARG, "scale must be positive and finite");
  // (row, head) pairs and tiles are counted in 32 bits
  if ((int64_t)c->total_q * c->heads >= (1 << 30) || (int64_t)c->total_k * c->kv_heads >= (1 << 30) || c->sequences >= (1 << 20) ||
      (int64_t)c->sequences * c->heads >= (1 << 28))
    return set_error(DIT_ERR_UNSUPPORTED, "rows x heads of 2^30 or more, or too many sequences");
  dit_status st;
  if ((st = check_strides("q", c->q_row, c->q_head, c->head_dim, c->dtype))) return st;
  if ((st = check_strides("k", c->k_row, c->k_head, c->head_dim, c->dtype))) return st;
  if ((st = check_strides("v", c->v_row, c->v_head, c->head_dim, c->dtype))) return st;
  if ((st = check_strides("o", c->o_row, c->o_head, c->head_dim, c->dtype))) return st;
  return check_apart("o", c->o_row, c->o_head, c->head_dim, c->total_q, c->heads);
}

dit_status check_packed_gradients(const dit_packed_config* c) {
  dit_status st;
  if ((st = check_apart("q", c->q_row, c->q_head, c->head_dim, c->total_q, c->heads))) return st;
  if ((st = check_apart("k", c->k_row, c->k_head, c->head_dim, c->total_k, c->kv_heads))) return st;
  return check_apart("v", c->v_row, c->v_head, c->head_dim, c->total_k, c->kv_heads);
}

dit_status check_lengths(const char* what, const void* offsets, int32_t rows, int32_t sequences) {
  if (!offsets && sequences > 0 && rows % sequences)
    return set_error(DIT_ERR_SHAPE, "%s: %d rows are not %d sequences of equal length, and there are no offsets", what, rows,
                     sequences);
  return DIT_OK;
}

dit_status check_gated_norm(const dit_gated_norm_config* c) {
  if (!c) return set_error(DIT_ERR_INVALID_ARG, "config is NULL");
  if (c->dtype != DIT_F32 && c->dtype != DIT_BF16) return set_error(DIT_ERR_INVALID_ARG, "dtype %d invalid", c->dtype);
  if (c->rows < 0 || c->sequences < 0) return set_error(DIT_ERR_INVALID_ARG, "negative size");
  if (c->rows > 0 && c->sequences == 0) return set_error(DIT_ERR_SHAPE, "%d rows of no sequence", c->rows);
  if (c->hidden <= 0) return set_error(DIT_ERR_SHAPE, "hidden %d must be positive", c->hidden);
  if (c->hidden > 8192) return set_error(DIT_ERR_UNSUPPORTED, "hidden %d > 8192", c->hidden);
  if (c->sequences >= (1 << 20)) return set_error(DIT_ERR_UNSUPPORTED, "%d sequences (at most 2^20 - 1)", c->sequences);
  // (chunks of a sequence, of 8 rows at least where there are many, are counted up to 2^25)
  if (c->rows > (1 << 28)) return set_error(DIT_ERR_UNSUPPORTED, "%d rows (at most 2^28)", c->rows);
  for (int32_t k : {c->post_norm, c->pre_norm})
    if (k < DIT_NORM_NONE || k > DIT_NORM_RMS) return set_error(DIT_ERR_INVALID_ARG, "norm kind %d invalid", k);
  if (!(c->eps > 0.f) || !std::isfinite(c->eps)) return set_error(DIT_ERR_INVALID_ARG, "eps must be positive");
  if (!std::isfinite(c->residual_scale)) return set_error(DIT_ERR_INVALID_ARG, "residual_scale not finite");
  for (int64_t r : {c->x_row, c->y_row, c->h_row, c->mod_row})
    if (r < c->hidden) return set_error(DIT_ERR_INVALID_ARG, "a row stride is below hidden");
  return DIT_OK;
}

dit_status flow_density_terms(int64_t n, double t, double t_next, double noise_level, double* cx, double* cv, double* var,
                              double* cst) {
  if (!(noise_level > 0.0) || !std::isfinite(noise_level))
    return set_error(DIT_ERR_DOMAIN, "the density needs a finite noise_level > 0 (the ODE step has none)");
  if (!(t > 0.0 && t < 1.0) || !std::isfinite(t_next) || !(t_next < t))
    return set_error(DIT_ERR_DOMAIN, "the density needs 0 < t < 1 and t_next < t (t=%g, t_next=%g)", t, t_next);
  const double h = t_next - t;
  const double k1 = 0.5 * noise_level * noise_level / (1.0 - t);   // sigma^2 / (2 t)
  *var = noise_level * noise_level * t / (1.0 - t) * -h;
  *cx = 1.0 + h * k1;
  *cv = h * (1.0 + k1 * (1.0 - t));
  *cst = -0.5 * (double)n * std::log(2.0 * M_PI * *var);
  return DIT_OK;
}

dit_status check_policy_loss(int32_t batch, int64_t n, double logp_scale, double clip_low, double clip_high,
                             double kl_weight) {
  if (batch < 0 || n < 0) return set_error(DIT_ERR_INVALID_ARG, "batch %d / n_per_sample %lld < 0", batch, (long long)n);
  if (!(logp_scale > 0.0) || !std::isfinite(logp_scale)) return set_error(DIT_ERR_DOMAIN, "logp_scale must be positive and finite");
  if (!(clip_low >= 0.0 && clip_low <= 1.0) || !(clip_high >= 0.0) || !std::isfinite(clip_high))
    return set_error(DIT_ERR_DOMAIN, "clip_low must be in [0, 1], clip_high >= 0 and finite");
  if (!(kl_weight >= 0.0) || !std::isfinite(kl_weight)) return set_error(DIT_ERR_DOMAIN, "kl_weight must be >= 0 and finite");
  return DIT_OK;
}

}  // namespace dit
