// Host-only argument checks of the entry points of ditupdate.h and ditint8.h (defined in update_checks.cpp).
#pragma once
#include "../../include/ditint8.h"
#include "../../include/ditupdate.h"
#include "status.h"

namespace dit {
// Elements of the tensors that one workgroup takes, for `total` elements in all: a multiple of 2048.
int64_t update_chunk(int64_t total);
// DIT_OK or the first violated rule (message set); *total: elements of all tensors. data: whether the pointers are there too.
dit_status check_gradients(const dit_gradient* g, int32_t n, bool data, int64_t* total);
dit_status check_adamw(const dit_adamw_config* c, const dit_adamw_tensor* t, int32_t n, bool step_dev, int64_t* total);
dit_status check_quantize(int32_t rows, int32_t cols, int64_t x_row, int32_t dtype, int64_t q_row, bool values, int64_t values_row);
// given: x is int8
dit_status check_int8(const dit_int8_config* c, bool given);
}  // namespace dit
