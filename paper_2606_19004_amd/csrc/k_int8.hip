// Linear layers in 8-bit integers on gfx950: rows to integers with a scale each, and the product of two such row sets.
#include <algorithm>

#include "gemm_common.h"
#include "update.h"
#include "vectors.h"

namespace dit {
namespace {

// ---------------------------------------------------------------------------
// rows to integers
// ---------------------------------------------------------------------------
// scale = max |x| / 127, correctly rounded and at least the smallest normal number, so that its reciprocal is finite.
// q = the integer nearest to x / scale: r = rint(x (1 / scale)) is off by one at most, and only next to a half. What is left,
// x - r scale, is exact in fp32: both are multiples of half a unit in the last place of scale, and their difference is below
// 2^24 of these. Comparing it with scale / 2 decides, a tie for the even one.
struct RowScale {
  float scale, inv, half;
  bool bad;   // the row holds a NaN or an infinity: scale NaN, integers 0
};
// top: the largest |x| of the row, as bits (which order like the values, NaN last)
__device__ __forceinline__ RowScale row_scale(uint32_t top) {
  RowScale r;
  r.bad = top >= 0x7f800000u;
  r.scale = fmaxf(__uint_as_float(r.bad ? 0u : top) / 127.f, 0x1p-126f);
  r.inv = 1.f / r.scale;
  r.half = 0.5f * r.scale;
  return r;
}
__device__ __forceinline__ float to_integer(float x, const RowScale& r) {
  const float q = rintf(x * r.inv), left = fmaf(-q, r.scale, x), d = fabsf(left);
  const bool odd = (int)q & 1;
  return d > r.half || (d == r.half && odd) ? q + copysignf(1.f, left) : q;
}
__device__ __forceinline__ uint32_t pack4(const float* q) {
  return ((uint32_t)(int)q[0] & 0xff) | ((uint32_t)(int)q[1] & 0xff) << 8 | ((uint32_t)(int)q[2] & 0xff) << 16 | (uint32_t)(int)q[3] << 24;
}
typedef unsigned u32x2_any1 __attribute__((ext_vector_type(2), aligned(1)));

__device__ __forceinline__ uint32_t top_of(uint32_t top, const float* f) {
#pragma unroll
  for (int i = 0; i < 8; i++) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
  return top;
}
template <typename T>
__device__ __forceinline__ void load_row8(const T* x, int at, int cols, float* f) {
  if (at + 8 <= cols) {
    load8_any(x + at, f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) f[i] = at + i < cols ? to_f32(x[at + i]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store_row8(const RowScale& r, const float* f, int at, int cols, int8_t* q, T* values) {
  float z[8], v[8];
#pragma unroll
  for (int i = 0; i < 8; i++) {
    z[i] = r.bad ? 0.f : to_integer(f[i], r);
    v[i] = r.bad ? NAN : z[i] * r.scale;
  }
  if (at + 8 <= cols) {
    *(u32x2_any1*)(q + at) = u32x2_any1{pack4(z), pack4(z + 4)};
    if (values) store8_any(values + at, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (at + i < cols) {
        q[at + i] = (int8_t)(int)z[i];
        if (values) values[at + i] = from_f32<T>(v[i]);
      }
  }
}

// LANES (64: a wave, 256: a workgroup) take a row, VECTORS x 8 elements each, in registers: one read.
template <typename T, int LANES, int VECTORS>
__global__ void __launch_bounds__(256) quantize_kernel(const QuantArgs a) {
  __shared__ uint32_t red[4];
  const int lane = threadIdx.x & (LANES - 1), per = 256 / LANES;
  for (int64_t row = (int64_t)blockIdx.x * per + threadIdx.x / LANES; row < a.rows; row += (int64_t)gridDim.x * per) {
    const T* x = (const T*)a.x + row * a.x_row;
    float f[VECTORS][8];
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < VECTORS; k++) load_row8(x, 8 * (lane + LANES * k), a.cols, f[k]);
#pragma unroll
    for (int k = 0; k < VECTORS; k++) top = top_of(top, f[k]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    if (LANES == 256) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
      __syncthreads();
      top = max(max(red[0], red[1]), max(red[2], red[3]));
    }
    const RowScale r = row_scale(top);
    if (lane == 0) a.scale[row] = r.bad ? NAN : r.scale;
#pragma unroll
    for (int k = 0; k < VECTORS; k++)
      store_row8<T>(r, f[k], 8 * (lane + LANES * k), a.cols, a.q + row * a.q_row,
                    a.values ? (T*)a.values + row * a.values_row : nullptr);
  }
}
// Rows past 16384 elements: a workgroup reads them twice.
template <typename T>
__global__ void __launch_bounds__(256) quantize_long_kernel(const QuantArgs a) {
  __shared__ uint32_t red[4];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = (const T*)a.x + row * a.x_row;
    uint32_t top = 0;
    for (int64_t at = 8 * threadIdx.x; at < a.cols; at += 8 * 256) {
      float f[8];
      load_row8(x, (int)at, a.cols, f);
      top = top_of(top, f);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
    __syncthreads();
    const RowScale r = row_scale(max(max(red[0], red[1]), max(red[2], red[3])));
    if (threadIdx.x == 0) a.scale[row] = r.bad ? NAN : r.scale;
    for (int64_t at = 8 * threadIdx.x; at < a.cols; at += 8 * 256) {
      float f[8];
      load_row8(x, (int)at, a.cols, f);
      store_row8<T>(r, f, (int)at, a.cols, a.q + row * a.q_row, a.values ? (T*)a.values + row * a.values_row : nullptr);
    }
  }
}

template <typename T, int LANES, int VECTORS> void quantize(const QuantArgs& a, hipStream_t s) {
  const int grid = (int)std::min<int64_t>(((int64_t)a.rows + 256 / LANES - 1) / (256 / LANES), 1 << 20);
  quantize_kernel<T, LANES, VECTORS><<<grid, 256, 0, s>>>(a);
}
template <typename T> hipError_t quantize_any(const QuantArgs& a, hipStream_t s) {
  if (a.cols <= 512) quantize<T, 64, 1>(a, s);
  else if (a.cols <= 1024) quantize<T, 64, 2>(a, s);
  else if (a.cols <= 2048) quantize<T, 256, 1>(a, s);
  else if (a.cols <= 4096) quantize<T, 256, 2>(a, s);
  else if (a.cols <= 8192) quantize<T, 256, 4>(a, s);
  else if (a.cols <= 16384) quantize<T, 256, 8>(a, s);
  else quantize_long_kernel<T><<<std::min(a.rows, 1 << 20), 256, 0, s>>>(a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------
// As in the bf16 GEMM, y^T = w x^T: matrix operand "A" = rows of w, "B" = rows of x, 16 bytes of k per lane and instruction
// (v_mfma_i32_16x16x64_i8), whose byte layout is that of the bf16 form: lane l gives bytes 16 (l / 16) .. + 15 of row l % 16 of both
// operands, so the order in which the instruction sums over k does not matter. Accumulator register q of lane l is
// feature 4 (l / 16) + q, row l % 16.
//
// A k-tile is 128 bytes of every row. In the last one, chunks of 16 bytes past the row's end have an offset past the
// buffer's records, which reads zeros, and x's bytes past in_features are masked, so that whatever w holds there does not count.
typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x4 mfma_i8(i32x4 w, i32x4 x, i32x4 c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, c, 0, 0, 0); }

// mask of the 16 bytes that start at byte `at` of a row of K
__device__ __forceinline__ i32x4 row_mask(int at, int K) {
  i32x4 m;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const int left = K - at - 4 * i;   // bytes of this word that count
    m[i] = left >= 4 ? -1 : left <= 0 ? 0 : (int)((1u << (8 * left)) - 1);
  }
  return m;
}

// buffer descriptor of up to `rows` rows from p on, `row` bytes apart, of which the last reaches to its 16-byte end
__device__ __forceinline__ u32x4_t rows_rsrc(const int8_t* p, int rows, int64_t row, int K) {
  const uint64_t u = (uint64_t)p;
  const uint32_t records = (uint32_t)((rows - 1) * row + ((K + 15) & ~15));
  return u32x4_t{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)u),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(u >> 32) & 0xffffu)),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)records), 0x00020000u};
}

// y of row m at features n .. n + 3 from their sums
template <int ACT, typename T>
__device__ __forceinline__ void finish4(const Int8Args& a, i32x4 c, int m, int n) {
  const float xs = a.x_scale[m];
  float v[4];
#pragma unroll
  for (int q = 0; q < 4; q++) {
    const int nq = min(n + q, a.N - 1);
    v[q] = (float)c[q] * xs * a.w_scale[nq];
    if (a.bias) v[q] += to_f32(((const T*)a.bias)[nq]);
    if (ACT) v[q] = gelu_tanh_f(v[q]);
  }
  T* y = (T*)a.y + (int64_t)m * a.y_row + n;
  if (n + 4 <= a.N) {
    store4_any(y, v);
  } else {
#pragma unroll
    for (int q = 0; q < 4; q++)
      if (n + q < a.N) y[q] = from_f32<T>(v[q]);
  }
}

// 64 x 64 tile, 4 waves of 32 x 32, k-tiles in a ring of three LDS stages (48 KB, three workgroups per CU).
template <int ACT, typename T>
__global__ void __launch_bounds__(256) int8_tile64_kernel(const Int8Args a, int total_tiles) {
  constexpr int B = 64, STAGE = 2 * B * 128;
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[3 * STAGE];
  const int per = gridDim.x >> 3;
  const int t = (blockIdx.x & 7) * per + (blockIdx.x >> 3);   // XCD-aware, as in the bf16 kernel
  if (t >= total_tiles) return;
  int tm, tn;
  tile_coords(t, cdiv(a.M, B), cdiv(a.N, B), tm, tn);
  const int m0 = tm * B, n0 = tn * B;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const u32x4_t rx = rows_rsrc(a.x + (int64_t)m0 * a.x_row, min(B, a.M - m0), a.x_row, a.K);
  const u32x4_t rw = rows_rsrc(a.w + (int64_t)n0 * a.w_row, min(B, a.N - n0), a.w_row, a.K);
  const uint32_t OOB = 0x80000000u;
  // a wave load fills 8 rows: lane -> row lane / 8, slot lane % 8, which holds chunk slot ^ swz(row)
  uint32_t xoff[2], woff[2];
  int chunk[2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int r = 8 * (wave * 2 + i) + (lane >> 3);
    chunk[i] = ((lane & 7) ^ swz(r)) * 16;
    xoff[i] = m0 + r < a.M ? (uint32_t)(r * a.x_row) + chunk[i] : OOB;
    woff[i] = n0 + r < a.N ? (uint32_t)(r * a.w_row) + chunk[i] : OOB;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem;
  auto issue = [&](int kt, int st) {
    const uint32_t base = lds0 + st * STAGE + wave * 2048;
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const bool in = kt * 128 + chunk[i] < a.K;
      dma_b128(rx, base + i * 1024, in ? xoff[i] : OOB, kt * 128);
      dma_b128(rw, base + B * 128 + i * 1024, in ? woff[i] : OOB, kt * 128);
    }
  };
  const int wm = wave >> 1, wn = wave & 1, r16 = lane & 15, kq = lane >> 4;
  i32x4 acc[2][2] = {};
  const int nk = (a.K + 127) / 128;
  issue(0, 0);
  if (nk > 1) issue(1, 1);
  int st = 0;
  for (int kt = 0; kt < nk; kt++) {
    // tile kt has landed (the 4 loads of tile kt + 1 may be in flight) in every wave, and every wave is done reading
    // tile kt - 1, whose stage takes tile kt + 2
    if (kt + 1 < nk) __builtin_amdgcn_s_waitcnt(0x0f74);
    else __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();
    if (kt + 2 < nk) issue(kt + 2, st == 0 ? 2 : st - 1);
    const char* sx = smem + st * STAGE;
    const char* sw = sx + B * 128;
#pragma unroll
    for (int s = 0; s < 2; s++) {
      i32x4 fw[2], fx[2];
#pragma unroll
      for (int i = 0; i < 2; i++) {
        const int rw_ = 32 * wn + 16 * i + r16, rx_ = 32 * wm + 16 * i + r16;
        fw[i] = *(const i32x4*)(sw + rw_ * 128 + (((4 * s + kq) ^ swz(rw_)) << 4));
        fx[i] = *(const i32x4*)(sx + rx_ * 128 + (((4 * s + kq) ^ swz(rx_)) << 4));
      }
      if (kt + 1 == nk) {
        const i32x4 mask = row_mask(kt * 128 + 64 * s + 16 * kq, a.K);
#pragma unroll
        for (int i = 0; i < 2; i++) fx[i] &= mask;
      }
#pragma unroll
      for (int i = 0; i < 2; i++)
#pragma unroll
        for (int j = 0; j < 2; j++) acc[i][j] = mfma_i8(fw[i], fx[j], acc[i][j]);
    }
    st = st == 2 ? 0 : st + 1;
  }
#pragma unroll
  for (int j = 0; j < 2; j++) {
    const int m = m0 + 32 * wm + 16 * j + r16;
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const int n = n0 + 32 * wn + 16 * i + 4 * kq;
      if (m < a.M && n < a.N) finish4<ACT, T>(a, acc[i][j], m, n);
    }
  }
#endif
}

template <int ACT, typename T> hipError_t matmul(const Int8Args& a, hipStream_t s) {
  const int64_t tiles = (int64_t)cdiv(a.M, 64) * cdiv(a.N, 64);
  int8_tile64_kernel<ACT, T><<<8 * cdiv(tiles, 8), 256, 0, s>>>(a, (int)tiles);
  return hipGetLastError();
}

}  // namespace

hipError_t quantize_rows_launch(const QuantArgs& a, int dtype, hipStream_t s) {
  return dtype == DT_BF16 ? quantize_any<u16>(a, s) : quantize_any<float>(a, s);
}

int64_t int8_matmul_threads(int M, int N) { return 256 * 8 * (((int64_t)cdiv(M, 64) * cdiv(N, 64) + 7) / 8); }

hipError_t int8_matmul_launch(const Int8Args& a, int dtype, int act, hipStream_t s) {
  if (dtype == DT_BF16) return act ? matmul<1, u16>(a, s) : matmul<0, u16>(a, s);
  return act ? matmul<1, float>(a, s) : matmul<0, float>(a, s);
}

}  // namespace dit
