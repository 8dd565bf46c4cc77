// The end of a policy update: the 2-norm over the gradients of all weights, clipping, and the weights' AdamW step. All are
// bound by memory (a large copy runs at 5.0 TB/s). 340 M weights, bf16 gradients, fp32 master weights with bf16 copies: norm 118-123 us (5.5 TB/s), clip
// 271 (5.0), AdamW 1895 (5.0), of bf16 weights without masters 1497 (5.0). Tensors come as tables in the kernels' arguments (no copy to the device,
// nothing kept between calls); a workgroup takes one chunk of one tensor. About 8192 chunks, of 2048 elements at least:
// 2.4 M fp32 weights in 20 tensors: AdamW 12.4-14.0 us (4.7-5.3 TB/s; chunks of 4096 15.3), norm 6.3, clip 5.2.
#include <algorithm>
#include <cmath>

#include "update.h"
#include "vectors.h"

namespace dit {
namespace {

constexpr int THREADS = 256;

// ---- tables of tensors ----
// first[e]: the workgroup that takes tensor e's first chunk; unused entries are past every workgroup.
// A launch's arguments stay below 4 KB: 192 gradients, 64 weights. Short lists take smaller tables, which the host copies faster (20 tensors: norm
// and clip 15.1 -> 13.1 us). Long lists of small tensors pay for their launches: 1200 tensors, 9 M weights, AdamW 111-133 us in 19 of them.
constexpr int GRADS = 192, WEIGHTS = 64, FEW = 24;
template <int N> struct GradTable {
  void* data[N];
  int64_t count[N];   // elements, bf16 ones negated
  int first[N];
};
template <int N> struct WeightTable {
  void* param[N];
  const void* grad[N];
  float* m[N];
  float* v[N];
  void* copy[N];
  int64_t count[N];
  int first[N];
  int types[N];       // bit 0: bf16 param, bit 1: bf16 grad
};
static_assert(sizeof(GradTable<GRADS>) + 64 <= 4096 && sizeof(WeightTable<WEIGHTS>) + 96 <= 4096, "a launch's arguments");

// The tensor that workgroup b works on: every lane looks at entries of its own, so that the search is one load long.
template <int N> __device__ __forceinline__ int entry_of(const int* first, int b) {
  constexpr int LOADS = (N + 63) / 64;
  const int lane = threadIdx.x & 63;
  int f[LOADS], e = -1;
#pragma unroll
  for (int i = 0; i < LOADS; i++) f[i] = first[min(64 * i + lane, N - 1)];
#pragma unroll
  for (int i = 0; i < LOADS; i++) e += __popcll(__ballot(64 * i + lane < N && f[i] <= b));
  return e;
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// ---- norm ----
// Two launches: sums of the chunks, then one workgroup that adds them up (2-5 us, most of it the launch; joining them needs counters that start at zero).
// Squares are taken and summed in fp64 (a bf16 or fp32 value's square is exact there, and finite): four sums per thread in flight,
// whose order is given by the chunk.
template <typename T> __device__ double chunk_squares(const T* p, int64_t begin, int64_t end) {
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  constexpr int U = 4;
  int64_t at = begin + 8 * threadIdx.x;
  for (; at + (U - 1) * 8 * THREADS + 8 <= end; at += U * 8 * THREADS) {
    float f[U][8];
#pragma unroll
    for (int u = 0; u < U; u++) load8_any(p + at + u * 8 * THREADS, f[u]);
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
      for (int i = 0; i < 8; i++) s[i & 3] = fma((double)f[u][i], (double)f[u][i], s[i & 3]);
  }
  for (; at < end; at += 8 * THREADS) {
    if (at + 8 <= end) {
      float f[8];
      load8_any(p + at, f);
#pragma unroll
      for (int i = 0; i < 8; i++) s[i & 3] = fma((double)f[i], (double)f[i], s[i & 3]);
    } else {
      for (int i = 0; at + i < end; i++) {
        const double d = to_f32(p[at + i]);
        s[0] = fma(d, d, s[0]);
      }
    }
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}

template <int N>
__global__ void __launch_bounds__(THREADS) norm_kernel(const GradTable<N> t, int64_t chunk, double* parts) {
  __shared__ double red[THREADS / 64];
  const int b = blockIdx.x, e = entry_of<N>(t.first, b);
  const int64_t n = t.count[e], count = n < 0 ? -n : n;
  const int64_t begin = (b - t.first[e]) * chunk, end = min(begin + chunk, count);
  double s = n < 0 ? chunk_squares((const u16*)t.data[e], begin, end) : chunk_squares((const float*)t.data[e], begin, end);
  s = wave_sum64(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) parts[b] = (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ void __launch_bounds__(1024) norm_finish_kernel(const double* parts, int64_t n, double max_norm, double* norm, float* scale) {
  __shared__ double red[16];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += parts[i];
  s = wave_sum64(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  s = 0.0;
#pragma unroll
  for (int w = 0; w < 16; w++) s += red[w];
  const double r = sqrt(s);
  if (norm) *norm = r;
  if (scale) *scale = r < INFINITY ? (float)fmin(1.0, max_norm / (r + 1e-6)) : NAN;
}

// ---- clipping ----
template <typename T> __device__ void chunk_scale(T* p, int64_t begin, int64_t end, float k) {
  for (int64_t at = begin + 8 * threadIdx.x; at < end; at += 8 * THREADS) {
    if (at + 8 <= end) {
      float f[8];
      load8_any(p + at, f);
#pragma unroll
      for (int i = 0; i < 8; i++) f[i] *= k;
      store8_any(p + at, f);
    } else {
      for (int i = 0; at + i < end; i++) p[at + i] = from_f32<T>(to_f32(p[at + i]) * k);
    }
  }
}
template <int N>
__global__ void __launch_bounds__(THREADS) clip_kernel(const GradTable<N> t, int64_t chunk, const float* scale) {
  const float k = *scale;
  if (k == 1.f) return;
  const int b = blockIdx.x, e = entry_of<N>(t.first, b);
  const int64_t n = t.count[e], count = n < 0 ? -n : n;
  const int64_t begin = (b - t.first[e]) * chunk, end = min(begin + chunk, count);
  if (n < 0) chunk_scale((u16*)t.data[e], begin, end, k);
  else chunk_scale((float*)t.data[e], begin, end, k);
}

// ---- AdamW ----
// One pass: 28 bytes move for a weight of the master form. The step's number on the device, from which every thread computes its two factors in
// fp64, costs 0.5 us of 12.4 (2.4 M fp32 weights) and nothing of 1895 (340 M). Rounding to bf16 weights is to nearest: without master weights a step below
// half a unit in the last place is lost.
// A beta is the sum of two fp32 numbers, so that what a mean keeps and what is added to it have the weights beta and 1 - beta to 2^-24 of 1 - beta.
// (One fp32 number is off by up to 1.7e-4 of 1 - 0.9999, in every step to the same side.)
struct Adam {
  float beta1, low1, rest1, beta2, low2, rest2, eps, lr, decay, mean1, root2;
  // with s = *scale: m = (beta1 + low1) m + rest1 s g, v = (beta2 + low2) v + rest2 (s g)^2, p -= lr (mean1 m / (sqrt(v) root2 + eps) + decay p),
  // mean1 = 1 / (1 - beta1^t), root2 = 1 / sqrt(1 - beta2^t). (p (1 - lr decay) would lose every decay below 2^-25.)
  __device__ __forceinline__ void apply(float g, float& m, float& v, float& p) const {
    m = fmaf(rest1, g, fmaf(beta1, m, low1 * m));
    v = fmaf(rest2 * g, g, fmaf(beta2, v, low2 * v));
    p = fmaf(-lr, fmaf(decay, p, mean1 * m / fmaf(sqrtf(v), root2, eps)), p);
  }
};
struct AdamArgs {
  Adam a;                          // of the host's step number
  const int64_t* step_dev;         // where that is on the device: with the logarithms of the betas (-inf for 0)
  double log_beta1, log_beta2;
  const float* scale;
};
// mean1 and root2 from t, in fp64: 1 - beta^t loses what a beta near 1 has
__host__ __device__ __forceinline__ void set_step(Adam& a, double t, double log_beta1, double log_beta2) {
  a.mean1 = (float)(1.0 / -expm1(t * log_beta1));
  a.root2 = (float)(1.0 / sqrt(-expm1(t * log_beta2)));
}

template <typename P, typename G>
__device__ void chunk_adam(const Adam& a, float k, P* p, const G* g, float* m, float* v, u16* copy, int64_t begin, int64_t end) {
  for (int64_t at = begin + 8 * threadIdx.x; at < end; at += 8 * THREADS) {
    if (at + 8 <= end) {
      float fp[8], fg[8], fm[8], fv[8];
      load8_any(p + at, fp);
      load8_any(g + at, fg);
      load8_any(m + at, fm);
      load8_any(v + at, fv);
#pragma unroll
      for (int i = 0; i < 8; i++) a.apply(k * fg[i], fm[i], fv[i], fp[i]);
      store8_any(p + at, fp);
      store8_any(m + at, fm);
      store8_any(v + at, fv);
      if (copy) store8_any(copy + at, fp);
    } else {
      for (int64_t i = at; i < end; i++) {
        float fp = to_f32(p[i]), fm = m[i], fv = v[i];
        a.apply(k * to_f32(g[i]), fm, fv, fp);
        p[i] = from_f32<P>(fp);
        m[i] = fm;
        v[i] = fv;
        if (copy) copy[i] = from_f32<u16>(fp);
      }
    }
  }
}
template <int N>
__global__ void __launch_bounds__(THREADS) adamw_kernel(const WeightTable<N> t, int64_t chunk, const AdamArgs args) {
  const float k = args.scale ? *args.scale : 1.f;
  if (k != k) return;
  const int b = blockIdx.x, e = entry_of<N>(t.first, b);
  const int64_t begin = (b - t.first[e]) * chunk, end = min(begin + chunk, t.count[e]);
  Adam a = args.a;
  if (args.step_dev) {
    const int64_t step = *args.step_dev;
    if (step < 1) return;   // (1 - beta^t is 0 or negative)
    set_step(a, (double)step, args.log_beta1, args.log_beta2);
  }
  void* p = t.param[e];
  const void* g = t.grad[e];
  float *m = t.m[e], *v = t.v[e];
  u16* copy = (u16*)t.copy[e];
  switch (t.types[e]) {
    case 0: return chunk_adam(a, k, (float*)p, (const float*)g, m, v, copy, begin, end);
    case 1: return chunk_adam(a, k, (u16*)p, (const float*)g, m, v, copy, begin, end);
    case 2: return chunk_adam(a, k, (float*)p, (const u16*)g, m, v, copy, begin, end);
    default: return chunk_adam(a, k, (u16*)p, (const u16*)g, m, v, copy, begin, end);
  }
}

int64_t chunks_of(int64_t count, int64_t chunk) { return (count + chunk - 1) / chunk; }

// Tables of successive tensors that have elements, a launch for each: launch(table, workgroups).
template <int N, typename F> hipError_t for_each_table(const dit_gradient* g, int n, int64_t chunk, F&& launch) {
  for (int i = 0; i < n;) {
    GradTable<N> t{};
    int used = 0;
    int64_t blocks = 0;
    for (; i < n && used < N; i++) {
      if (g[i].count == 0) continue;
      t.data[used] = g[i].data;
      t.count[used] = g[i].dtype == DIT_BF16 ? -g[i].count : g[i].count;
      t.first[used++] = (int)blocks;
      blocks += chunks_of(g[i].count, chunk);
    }
    if (used == 0) break;
    for (int k = used; k < N; k++) t.first[k] = 0x7fffffff;
    const hipError_t e = launch(t, (int)blocks);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int N> hipError_t norm_sums(const dit_gradient* g, int n, int64_t chunk, double* parts, hipStream_t s) {
  return for_each_table<N>(g, n, chunk, [&](const GradTable<N>& t, int blocks) {
    norm_kernel<N><<<blocks, THREADS, 0, s>>>(t, chunk, parts);
    parts += blocks;
    return hipGetLastError();
  });
}
template <int N> hipError_t clip(const dit_gradient* g, int n, int64_t chunk, const float* scale, hipStream_t s) {
  return for_each_table<N>(g, n, chunk, [&](const GradTable<N>& t, int blocks) {
    clip_kernel<N><<<blocks, THREADS, 0, s>>>(t, chunk, scale);
    return hipGetLastError();
  });
}
template <int N> hipError_t adamw(const AdamArgs& a, const dit_adamw_tensor* w, int n, int64_t chunk, hipStream_t s) {
  for (int i = 0; i < n;) {
    WeightTable<N> t{};
    int used = 0;
    int64_t blocks = 0;
    for (; i < n && used < N; i++) {
      if (w[i].count == 0) continue;
      t.param[used] = w[i].param;
      t.grad[used] = w[i].grad;
      t.m[used] = w[i].m;
      t.v[used] = w[i].v;
      t.copy[used] = w[i].copy;
      t.count[used] = w[i].count;
      t.types[used] = (w[i].param_dtype == DIT_BF16) | (w[i].grad_dtype == DIT_BF16) << 1;
      t.first[used++] = (int)blocks;
      blocks += chunks_of(w[i].count, chunk);
    }
    if (used == 0) break;
    for (int k = used; k < N; k++) t.first[k] = 0x7fffffff;
    adamw_kernel<N><<<(int)blocks, THREADS, 0, s>>>(t, chunk, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

int64_t grad_norm_parts(const dit_gradient* g, int n, int64_t chunk) {
  int64_t parts = 0;
  for (int i = 0; i < n; i++) parts += chunks_of(g[i].count, chunk);
  return parts;
}

hipError_t grad_norm_sums(const dit_gradient* g, int n, int64_t chunk, double* parts, hipStream_t s) {
  return n <= FEW ? norm_sums<FEW>(g, n, chunk, parts, s) : norm_sums<GRADS>(g, n, chunk, parts, s);
}

hipError_t grad_norm_finish(const double* parts, int64_t nparts, double max_norm, double* norm, float* scale, hipStream_t s) {
  norm_finish_kernel<<<1, 1024, 0, s>>>(parts, nparts, max_norm, norm, scale);
  return hipGetLastError();
}

hipError_t grad_clip_launch(const dit_gradient* g, int n, int64_t chunk, const float* scale, hipStream_t s) {
  return n <= FEW ? clip<FEW>(g, n, chunk, scale, s) : clip<GRADS>(g, n, chunk, scale, s);
}

hipError_t adamw_launch(const dit_adamw_config& c, const dit_adamw_tensor* w, int n, int64_t chunk, const float* scale,
                        const int64_t* step_dev, hipStream_t s) {
  auto low = [](double beta) { return (float)(beta - (double)(float)beta); };
  AdamArgs a{{(float)c.beta1, low(c.beta1), (float)(1.0 - c.beta1), (float)c.beta2, low(c.beta2), (float)(1.0 - c.beta2), (float)c.eps,
              (float)c.lr, (float)c.weight_decay, 0.f, 0.f},
             step_dev, std::log(c.beta1), std::log(c.beta2), scale};
  set_step(a.a, (double)c.step, a.log_beta1, a.log_beta2);
  return n <= FEW ? adamw<FEW>(a, w, n, chunk, s) : adamw<WEIGHTS>(a, w, n, chunk, s);
}

}  // namespace dit
