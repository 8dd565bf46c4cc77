// Drives the argument checks of the gradient norm, AdamW and 8-bit entry points through valid, boundary and absurd values.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include <limits>

#include "update_checks.h"

using namespace dit;

#define EXPECT(cond)                                                     \
  do {                                                                   \
    if (!(cond)) {                                                       \
      std::fprintf(stderr, "line %d: %s\n", __LINE__, #cond);            \
      std::exit(1);                                                      \
    }                                                                    \
  } while (0)

namespace {
const int64_t LONG[] = {0, 1, 15, 16, 100, 112, 131072, (1 << 23) - 16, 1 << 23, 1 << 30, (int64_t)1 << 44, ((int64_t)1 << 44) + 1,
                        std::numeric_limits<int64_t>::max(), -1, std::numeric_limits<int64_t>::min()};
const int32_t SHORT[] = {0, 1, 2, 100, 131071, 131072, std::numeric_limits<int32_t>::max(), -1, std::numeric_limits<int32_t>::min()};

void lists() {
  float x[4];
  int64_t total;
  for (int64_t a : LONG)
    for (int64_t b : LONG) {
      dit_gradient g[2] = {{x, a, DIT_F32, 0}, {x, b, DIT_BF16, 0}};
      const bool ok = check_gradients(g, 2, true, &total) == DIT_OK;
      EXPECT(ok == (a >= 0 && b >= 0 && a <= (int64_t)1 << 44 && b <= ((int64_t)1 << 44) - a));
      if (!ok) continue;
      const int64_t chunk = update_chunk(total);
      EXPECT(chunk % 2048 == 0 && chunk >= 2048 && (total + chunk - 1) / chunk <= 8192);
      dit_adamw_config c{1e-3, 0.9, 0.999, 1e-8, 0.0, 1};
      dit_adamw_tensor t[2] = {{x, x, x, x, nullptr, a, DIT_F32, DIT_F32}, {x, x, x, x, x, b, DIT_BF16, DIT_BF16}};
      EXPECT(check_adamw(&c, t, 2, false, &total) == DIT_OK);
    }
  for (int32_t n : SHORT) check_gradients(nullptr, n, true, &total);
  for (double v : {0.0, -0.0, 1.0, 0.5, -1.0, 1e308, (double)INFINITY, (double)NAN})
    for (double dit_adamw_config::*f : {&dit_adamw_config::lr, &dit_adamw_config::beta1, &dit_adamw_config::beta2, &dit_adamw_config::eps,
                                        &dit_adamw_config::weight_decay}) {
      dit_adamw_config c{1e-3, 0.9, 0.999, 1e-8, 0.0, 1};
      c.*f = v;
      const dit_status st = check_adamw(&c, nullptr, 0, false, &total);
      EXPECT(std::isfinite(v) || st == DIT_ERR_DOMAIN);
    }
  EXPECT(check_adamw(nullptr, nullptr, 0, false, &total) == DIT_ERR_INVALID_ARG);
}

void rows() {
  for (int32_t n : SHORT)
    for (int32_t cols : SHORT)
      for (int64_t x : LONG)
        for (int64_t q : LONG) {
          const dit_status st = check_quantize(n, cols, x, DIT_BF16, q, true, x);
          EXPECT((st == DIT_OK) == (n >= 0 && cols >= 0 && x >= cols && q >= cols && x < 1 << 30 && q < 1 << 30));
        }
}

void products() {
  EXPECT(check_int8(nullptr, true) == DIT_ERR_INVALID_ARG);
  for (int32_t m : SHORT)
    for (int32_t k : SHORT)
      for (int64_t x : LONG)
        for (int64_t w : LONG)
          for (bool given : {true, false}) {
            const dit_int8_config c{m, k, 50, DIT_F32, DIT_ACT_NONE, x, w, 50};
            const bool ok = check_int8(&c, given) == DIT_OK;
            const bool want = m >= 0 && k >= 1 && k < 1 << 17 && x >= k && w >= k && w % 16 == 0 && w < 1 << 23 &&
                              (given ? x % 16 == 0 && x < 1 << 23 : x < 1 << 30);
            EXPECT(ok == want);
          }
}
}  // namespace

int main() {
  lists();
  rows();
  products();
  std::puts("all checks passed");
  return 0;
}
