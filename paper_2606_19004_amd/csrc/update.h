// Entry points of k_update.hip and k_int8.hip.
#pragma once
#include "../../include/ditint8.h"
#include "../../include/ditupdate.h"
#include "internal.h"

namespace dit {

// Partial sums of a list's norm: one for every chunk of a tensor.
int64_t grad_norm_parts(const dit_gradient* g, int n, int64_t chunk);
hipError_t grad_norm_sums(const dit_gradient* g, int n, int64_t chunk, double* parts, hipStream_t s);
hipError_t grad_norm_finish(const double* parts, int64_t nparts, double max_norm, double* norm, float* scale, hipStream_t s);
hipError_t grad_clip_launch(const dit_gradient* g, int n, int64_t chunk, const float* scale, hipStream_t s);
hipError_t adamw_launch(const dit_adamw_config& c, const dit_adamw_tensor* t, int n, int64_t chunk, const float* scale,
                        const int64_t* step_dev, hipStream_t s);

struct QuantArgs {
  const void* x; int8_t* q; float* scale; void* values;
  int rows, cols;
  int64_t x_row, q_row, values_row;
};
hipError_t quantize_rows_launch(const QuantArgs& a, int dtype, hipStream_t s);

struct Int8Args {
  const int8_t* x; const float* x_scale; const int8_t* w; const float* w_scale; const void* bias; void* y;
  int M, N, K;
  int64_t x_row, w_row, y_row;
  const void* raw; int64_t raw_row;   // rows that are not integers yet, in place of x and x_scale (where int8_takes_raw), or null
};
// How a product runs: one or two rows by dot products; tiles of 32 or 64 whose waves share k; of 64 or 128 with rings of LDS stages; of 256 x 192
// or 256 x 256
enum Int8Form { INT8_FEW_ROWS, INT8_KSPLIT_32, INT8_KSPLIT_64, INT8_RING_64, INT8_RING_128, INT8_LARGE_192, INT8_LARGE_256 };
Int8Form int8_form(int M, int N, int K);
int64_t int8_matmul_threads(int M, int N, int K);   // of the product's launch: one takes fewer than 2^32
bool int8_takes_raw(int M, int N, int K);    // whether a product rounds its rows by itself
hipError_t int8_matmul_launch(const Int8Args& a, int dtype, int act, hipStream_t s);

}  // namespace dit
