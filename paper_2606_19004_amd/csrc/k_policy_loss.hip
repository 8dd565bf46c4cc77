// The clipped policy loss of one SDE step and its gradient for the velocity, in two passes over the samples:
//   sums    per (sample, chunk): sum (x_next - mean)^2 and, with a reference, sum (v - v_ref)^2
//   finish  every workgroup adds its sample's sums up (the same order everywhere), forms the ratio and the slope of the
//           loss in logp, and writes its chunk of dv; the first one also writes the loss
// Everything is fp64 from the fp32 inputs: x_next - mean is a difference of near values, the sums run over millions
// of terms. Bound by memory: 12 (16 with a reference) bytes per element read by each pass, 4 written by the second (24 samples of
// 409600 elements with a reference: 71 us, 5.0 TB/s; a large copy 4.9; 59 us where the inputs are in the last-level cache). dv
// needs the finished sum of its sample. One pass would keep a sample's elements on the chip while its workgroups wait for each
// other, which takes all of them running at once and counters that start each call at zero.
// Small calls are bound by their two launches, and in the second by what comes before its first element: the sums of its sample, their
// reduction and an exponential (16 samples of 65536 elements: 10.6 us).
#include <algorithm>

#include "packed.h"

namespace dit {
namespace {

constexpr int THREADS = 256;

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// Sum over the workgroup, in every thread.
__device__ double block_sum(double v, double* red) {
  v = wave_sum64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; w++) s += red[w];
  return s;
}

// Elements [begin, end) of a sample that chunk c covers (multiples of 4 from the sample's start).
__device__ __forceinline__ void chunk_range(const PolicyLossArgs& a, int c, int64_t& begin, int64_t& end) {
  const int64_t quads = (a.n + 3) / 4, per = (quads + a.chunks - 1) / a.chunks;
  begin = min((int64_t)c * per * 4, a.n);
  end = min(begin + per * 4, a.n);
}

template <bool VEC, bool REF>
__global__ void __launch_bounds__(THREADS) sums_kernel(PolicyLossArgs a) {
  __shared__ double red[THREADS / 64];
  const int b = blockIdx.x / a.chunks, c = blockIdx.x - b * a.chunks;
  const int64_t base = (int64_t)b * a.n;
  int64_t begin, end;
  chunk_range(a, c, begin, end);
  double se = 0.0, sr = 0.0;
  auto term = [&](float x, float v, float n, float r) {
    const double e = (double)n - fma(a.cv, (double)v, a.cx * (double)x);
    se = fma(e, e, se);
    if (REF) {
      const double k = (double)v - (double)r;
      sr = fma(k, k, sr);
    }
  };
  if (VEC) {
    for (int64_t i = begin + 4 * threadIdx.x; i < end; i += 4 * THREADS) {
      const float4 x = *(const float4*)(a.x + base + i), v = *(const float4*)(a.v + base + i);
      const float4 n = *(const float4*)(a.xn + base + i);
      float4 r = v;
      if (REF) r = *(const float4*)(a.v_ref + base + i);
      term(x.x, v.x, n.x, r.x);
      term(x.y, v.y, n.y, r.y);
      term(x.z, v.z, n.z, r.z);
      term(x.w, v.w, n.w, r.w);
    }
  } else {
    for (int64_t i = begin + threadIdx.x; i < end; i += THREADS)
      term(a.x[base + i], a.v[base + i], a.xn[base + i], REF ? a.v_ref[base + i] : 0.f);
  }
  se = block_sum(se, red);
  if (REF) sr = block_sum(sr, red);
  if (threadIdx.x == 0) {
    double* p = a.parts + 2 * ((int64_t)b * a.chunks + c);
    p[0] = se;
    p[1] = sr;
  }
}

// What sample b's sums give. `lanes` lanes that are neighbours work on the same sample.
struct Sample {
  double logp, ratio, loss, slope;   // slope: d loss / d logp
};
__device__ Sample sample_of(const PolicyLossArgs& a, int b, int lanes) {
  double se = 0.0, sr = 0.0;
  for (int c = threadIdx.x & (lanes - 1); c < a.chunks; c += lanes) {
    const double2 p = *(const double2*)(a.parts + 2 * ((int64_t)b * a.chunks + c));
    se += p.x;
    sr += p.y;
  }
  for (int o = lanes >> 1; o > 0; o >>= 1) {
    se += __shfl_xor(se, o, 64);
    sr += __shfl_xor(sr, o, 64);
  }
  Sample s;
  s.logp = a.cst - se / (2.0 * a.var);
  s.ratio = exp(a.logp_scale * (s.logp - a.logp_old[b]));
  const double adv = a.adv[b];
  // adv = 0 adds nothing, also where the ratio has overflowed
  const double free_ = adv == 0.0 ? 0.0 : s.ratio * adv;
  const double clipped = fmin(fmax(s.ratio, 1.0 - a.clip_low), 1.0 + a.clip_high) * adv;
  const bool open = !(free_ > clipped);   // (a NaN stays one)
  s.loss = -(open ? free_ : clipped) + a.kl_weight * a.logp_scale * a.cv * a.cv / (2.0 * a.var) * sr;
  s.slope = open ? -free_ * a.logp_scale / a.batch : 0.0;
  return s;
}

template <bool VEC, bool REF>
__global__ void __launch_bounds__(THREADS) finish_kernel(PolicyLossArgs a) {
  __shared__ double red[THREADS / 64];
  const int b = blockIdx.x / a.chunks, c = blockIdx.x - b * a.chunks;
  const Sample s = sample_of(a, b, 64);
  if (c == 0 && threadIdx.x == 0) {
    if (a.logp) a.logp[b] = s.logp;
    if (a.ratio) a.ratio[b] = s.ratio;
  }
  if (a.dv) {
    const int64_t base = (int64_t)b * a.n;
    int64_t begin, end;
    chunk_range(a, c, begin, end);
    const double ke = s.slope * a.cv / a.var;
    const double kr = a.kl_weight * a.logp_scale * a.cv * a.cv / (a.var * a.batch);
    auto term = [&](float x, float v, float n, float r) {
      double d = s.slope == 0.0 ? 0.0 : ke * ((double)n - fma(a.cv, (double)v, a.cx * (double)x));
      if (REF) d = fma(kr, (double)v - (double)r, d);
      return (float)d;
    };
    if (VEC) {
      for (int64_t i = begin + 4 * threadIdx.x; i < end; i += 4 * THREADS) {
        const float4 x = *(const float4*)(a.x + base + i), v = *(const float4*)(a.v + base + i);
        const float4 n = *(const float4*)(a.xn + base + i);
        float4 r = v;
        if (REF) r = *(const float4*)(a.v_ref + base + i);
        *(float4*)(a.dv + base + i) = make_float4(term(x.x, v.x, n.x, r.x), term(x.y, v.y, n.y, r.y),
                                                  term(x.z, v.z, n.z, r.z), term(x.w, v.w, n.w, r.w));
      }
    } else {
      for (int64_t i = begin + threadIdx.x; i < end; i += THREADS)
        a.dv[base + i] = term(a.x[base + i], a.v[base + i], a.xn[base + i], REF ? a.v_ref[base + i] : 0.f);
    }
  }
  if (a.loss && c == 0 && b == 0) {
    int lanes = 1;   // of a sample
    while (lanes < 64 && lanes < a.chunks) lanes *= 2;
    double total = 0.0;
    for (int i = threadIdx.x / lanes; i - (int)threadIdx.x / lanes < a.batch; i += THREADS / lanes) {
      const double l = sample_of(a, min(i, a.batch - 1), lanes).loss;
      if (i < a.batch && (threadIdx.x & (lanes - 1)) == 0) total += l;
    }
    total = block_sum(total, red);
    if (threadIdx.x == 0) *a.loss = total / a.batch;
  }
}

bool vectors(const PolicyLossArgs& a) {
  return a.n % 4 == 0 && ((uintptr_t)a.x | (uintptr_t)a.v | (uintptr_t)a.xn | (uintptr_t)a.v_ref | (uintptr_t)a.dv) % 16 == 0;
}

}  // namespace

// Enough workgroups to fill the chip, of at least 2048 elements each: 1024 (24 samples of 409600 elements with a reference, inputs in
// the last-level cache, us with 512 / 1024 / 2048 / 4096: 57.1 / 58.9 / 59.3 / 58.2; 16 samples of 65536: 9.8 to 9.9 with each).
int policy_loss_chunks(int batch, int64_t n) {
  const int64_t fill = 1024 / std::max(batch, 1);
  return (int)std::max<int64_t>(1, std::min<int64_t>(fill, n / 2048));
}

#define POLICY_LAUNCH(kernel)                                                        \
  do {                                                                               \
    const int grid = a.chunks * a.batch;                                             \
    if (vectors(a) && a.v_ref) kernel<true, true><<<grid, THREADS, 0, s>>>(a);       \
    else if (vectors(a)) kernel<true, false><<<grid, THREADS, 0, s>>>(a);            \
    else if (a.v_ref) kernel<false, true><<<grid, THREADS, 0, s>>>(a);               \
    else kernel<false, false><<<grid, THREADS, 0, s>>>(a);                           \
  } while (0)

hipError_t policy_loss_sums(const PolicyLossArgs& a, hipStream_t s) {
  POLICY_LAUNCH(sums_kernel);
  return hipGetLastError();
}
hipError_t policy_loss_finish(const PolicyLossArgs& a, hipStream_t s) {
  POLICY_LAUNCH(finish_kernel);
  return hipGetLastError();
}

}  // namespace dit
