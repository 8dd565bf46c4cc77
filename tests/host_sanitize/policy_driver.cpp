// Drives the argument checks of the policy-update entry points through valid, boundary and absurd values.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include <limits>

#include "policy_checks.h"

using namespace dit;

#define EXPECT(cond)                                                     \
  do {                                                                   \
    if (!(cond)) {                                                       \
      std::fprintf(stderr, "line %d: %s\n", __LINE__, #cond);            \
      std::exit(1);                                                      \
    }                                                                    \
  } while (0)

namespace {
const int64_t STRIDES[] = {0, 1, 63, 64, 128, 256, 512, 513, (1 << 24) - 8, 1 << 24, (int64_t(1) << 40) - 64, int64_t(1) << 40, int64_t(1) << 60, int64_t(1) << 61,
                           int64_t(1) << 62, std::numeric_limits<int64_t>::max(), -1, -64, std::numeric_limits<int64_t>::min()};
const int32_t SIZES[] = {0, 1, 2, 7, 100, (1 << 20) - 1, 1 << 20, 1 << 28, std::numeric_limits<int32_t>::max(), -1,
                         std::numeric_limits<int32_t>::min()};

dit_packed_config packed() {
  dit_packed_config c{};
  c.sequences = 2;
  c.heads = 4;
  c.kv_heads = 2;
  c.head_dim = 64;
  c.total_q = c.total_k = 100;
  c.dtype = DIT_BF16;
  c.scale = 0.125f;
  c.q_row = c.k_row = c.v_row = 512;
  c.o_row = 256;
  c.q_head = c.k_head = c.v_head = c.o_head = 64;
  return c;
}

void packed_configs() {
  EXPECT(check_packed(nullptr) == DIT_ERR_INVALID_ARG);
  EXPECT(check_packed_gradients([] { static dit_packed_config c = packed(); return &c; }()) == DIT_OK);
  int64_t dit_packed_config::* const strides[] = {&dit_packed_config::q_row, &dit_packed_config::q_head, &dit_packed_config::k_row,
                                                 &dit_packed_config::k_head, &dit_packed_config::v_row, &dit_packed_config::v_head,
                                                 &dit_packed_config::o_row, &dit_packed_config::o_head};
  for (int32_t heads : {1, 2, 4, 1 << 20})
    for (int32_t dtype : {(int32_t)DIT_BF16, (int32_t)DIT_F32})
      for (auto field : strides)
        for (int64_t value : STRIDES) {
          dit_packed_config c = packed();
          c.heads = c.kv_heads = heads;
          c.dtype = dtype;
          c.*field = value;
          if (check_packed(&c) == DIT_OK) check_packed_gradients(&c);
          // a head further off than any tensor reaches is refused, not wrapped round
          const bool head = field == strides[1] || field == strides[3] || field == strides[5] || field == strides[7];
          if (value < 0 || (head && value >= (int64_t(1) << 60))) EXPECT(check_packed(&c) != DIT_OK);
        }
  for (int64_t head : STRIDES) {   // as many heads as one row may have
    dit_packed_config c = packed();
    c.sequences = c.total_q = c.total_k = 1;
    c.heads = c.kv_heads = (1 << 28) - 1;
    c.q_head = c.k_head = c.v_head = c.o_head = head;
    if (check_packed(&c) == DIT_OK) check_packed_gradients(&c);
    c.total_q = c.total_k = 2;
    if (head >= 0 && head < 512) EXPECT(check_packed(&c) != DIT_OK);
  }
  int32_t dit_packed_config::* const sizes[] = {&dit_packed_config::sequences, &dit_packed_config::heads, &dit_packed_config::kv_heads,
                                               &dit_packed_config::head_dim, &dit_packed_config::total_q, &dit_packed_config::total_k,
                                               &dit_packed_config::max_q};
  for (auto field : sizes)
    for (int32_t value : SIZES) {
      dit_packed_config c = packed();
      c.*field = value;
      if (check_packed(&c) == DIT_OK) {
        check_packed_gradients(&c);
        check_lengths("q", nullptr, c.total_q, c.sequences);
      }
      if (value < 0) EXPECT(check_packed(&c) != DIT_OK);
    }
}

void norms_and_losses() {
  dit_gated_norm_config c{};
  EXPECT(check_gated_norm(nullptr) == DIT_ERR_INVALID_ARG);
  c.sequences = 2;
  c.rows = 10;
  c.hidden = 64;
  c.dtype = DIT_F32;
  c.eps = 1e-6f;
  c.residual_scale = 1.f;
  c.x_row = c.y_row = c.h_row = c.mod_row = 64;
  EXPECT(check_gated_norm(&c) == DIT_OK);
  int64_t dit_gated_norm_config::* const strides[] = {&dit_gated_norm_config::x_row, &dit_gated_norm_config::y_row,
                                                     &dit_gated_norm_config::h_row, &dit_gated_norm_config::mod_row};
  for (auto field : strides)
    for (int64_t value : STRIDES) {
      dit_gated_norm_config b = c;
      b.*field = value;
      EXPECT((check_gated_norm(&b) == DIT_OK) == (value >= 64));
    }
  const double nan = std::nan(""), inf = std::numeric_limits<double>::infinity();
  double cx, cv, var, cst;
  for (double t : {-1.0, 0.0, 1e-300, 0.5, 1.0 - 1e-16, 1.0, 2.0, nan, inf})
    for (double tn : {-1.0, 0.0, 0.25, 0.5, 1.0, nan, -inf})
      for (double level : {0.0, 1e-300, 0.7, 1e300, nan, inf}) {
        const dit_status st = flow_density_terms(64, t, tn, level, &cx, &cv, &var, &cst);
        EXPECT((st == DIT_OK) == (t > 0.0 && t < 1.0 && std::isfinite(tn) && tn < t && level > 0.0 && std::isfinite(level)));
      }
  for (int64_t n : {int64_t(0), int64_t(1), int64_t(-1), std::numeric_limits<int64_t>::max()})
    for (int32_t batch : SIZES)
      EXPECT((check_policy_loss(batch, n, 1.0, 0.2, 0.2, 0.0) == DIT_OK) == (batch >= 0 && n >= 0));
  EXPECT(check_policy_loss(1, 1, nan, 0.2, 0.2, 0.0) == DIT_ERR_DOMAIN && check_policy_loss(1, 1, 1.0, nan, 0.2, 0.0) == DIT_ERR_DOMAIN);
}
}  // namespace

int main() {
  packed_configs();
  norms_and_losses();
  std::puts("all checks passed");
  return 0;
}
