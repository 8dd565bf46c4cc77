// Host-only argument checks of the entry points of ditpolicy.h (defined in policy_checks.cpp).
#pragma once
#include "../../include/ditpolicy.h"
#include "status.h"

namespace dit {
// DIT_OK or the first violated rule (message set).
dit_status check_packed(const dit_packed_config* c);
// The strides of the gradients written like q, k and v.
dit_status check_packed_gradients(const dit_packed_config* c);
dit_status check_gated_norm(const dit_gated_norm_config* c);
// Equal lengths where the offsets are NULL.
dit_status check_lengths(const char* what, const void* offsets, int32_t rows, int32_t sequences);
// mean = cx x + cv v, the variance and the constant of the log-density of n elements
dit_status flow_density_terms(int64_t n, double t, double t_next, double noise_level, double* cx, double* cv, double* var,
                              double* cst);
dit_status check_policy_loss(int32_t batch, int64_t n, double logp_scale, double clip_low, double clip_high,
                             double kl_weight);
}  // namespace dit
