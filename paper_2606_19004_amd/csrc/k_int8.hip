// Linear layers in 8-bit integers on gfx950: rows to integers with a scale each, and the product of two such row sets.
//   q_ij = nearest integer to x_ij / s_i, s_i = max_j |x_ij| / 127;   y_in = act((sum_k xq_ik wq_nk) xs_i ws_n + b_n)
// Integer sums are exact, so every form of the product gives the same bits.
#include <algorithm>
#include <type_traits>

#include "gemm_common.h"
#include "packed.h"
#include "update.h"
#include "vectors.h"

namespace dit {
namespace {

// ---------------------------------------------------------------------------
// rows to integers
// ---------------------------------------------------------------------------
// scale = max |x| / 127, correctly rounded and at least the smallest normal number, so that its reciprocal is finite.
// q = the integer nearest to x / scale. x (1 / scale), rounded once to an integer, is that or its neighbour, which happens next to a half
// only. What is left, x - q scale, is exact in fp32: both are multiples of half a unit in the last place of scale, and their
// difference is below 2^24 of these. Where twice that is below scale, q is right; elsewhere, which is rare, a tie goes to the even one. (What is
// left is doubled, which is exact. Half of the scale is not: below 2^-125 a scale is a multiple of 2^-149, the smallest unit there is.)
struct RowScale {
  float scale, inv;
  bool bad;   // the row holds a NaN or an infinity: scale NaN, integers 0
};
// top: the largest |x| of the row, as bits (which order like the values, NaN last)
__device__ __forceinline__ RowScale row_scale(uint32_t top) {
  RowScale r;
  r.bad = top >= 0x7f800000u;
  r.scale = fmaxf(__uint_as_float(r.bad ? 0u : top) / 127.f, 0x1p-126f);
  r.inv = 1.f / r.scale;
  return r;
}
constexpr float MAGIC = 12582912.f;   // 1.5 2^23: MAGIC + q has the integer q in its low bits
// the low bytes of four words
__device__ __forceinline__ uint32_t low_bytes(const float* t) {
  const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(t[1]), __float_as_uint(t[0]), 0x0c0c0400u);
  const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(t[3]), __float_as_uint(t[2]), 0x04000c0cu);
  return lo | hi;
}
typedef unsigned u32x2_any1 __attribute__((ext_vector_type(2), aligned(1)));

// 8 successive elements of a row as they are stored, and the largest of their absolute values' bits
template <typename T> struct Eight;
template <> struct Eight<u16> {
  uint32_t w[4];
  __device__ __forceinline__ void load(const u16* x) {
    const u32x4_any2 u = *(const u32x4_any2*)x;
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = u[i];
  }
  __device__ __forceinline__ void set(int i, u16 v) { w[i >> 1] = i & 1 ? w[i >> 1] | (uint32_t)v << 16 : v; }
  __device__ __forceinline__ uint32_t top() const {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = __builtin_bit_cast(u16x2, w[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; i++) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
    return (uint32_t)max(m[0], m[1]) << 16;
  }
  __device__ __forceinline__ void get(float* f) const { unpack8(w, f); }
};
template <> struct Eight<float> {
  float v[8];
  __device__ __forceinline__ void load(const float* x) { load8_any(x, v); }
  __device__ __forceinline__ void set(int i, float f) { v[i] = f; }
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
  }
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int i = 0; i < 8; i++) f[i] = v[i];
  }
};
template <typename T>
__device__ __forceinline__ void load_row8(const T* x, int at, int cols, Eight<T>& e) {
  if (at + 8 <= cols) {
    e.load(x + at);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) e.set(i, at + i < cols ? x[at + i] : (T)0);
  }
}
// t: MAGIC + q of 8 elements
__device__ __forceinline__ void to_integers(const RowScale& r, const float* f, float* t) {
  float far = 0.f;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    t[i] = fmaf(f[i], r.inv, MAGIC);
    far = fmaxf(far, fabsf(fmaf(MAGIC - t[i], r.scale, f[i])));
  }
  if (2.f * far >= r.scale) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float left = fmaf(MAGIC - t[i], r.scale, f[i]), d = 2.f * fabsf(left);
      if (d > r.scale || (d == r.scale && (__float_as_uint(t[i]) & 1))) t[i] += copysignf(1.f, left);
    }
  }
}
template <typename T>
__device__ __forceinline__ void store_row8(const RowScale& r, const Eight<T>& e, int at, int cols, int8_t* q, T* values) {
  if (at >= cols) return;
  float f[8], t[8];
  e.get(f);
  to_integers(r, f, t);
  if (r.bad) {
#pragma unroll
    for (int i = 0; i < 8; i++) t[i] = MAGIC;
  }
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; i++) v[i] = r.bad ? NAN : (t[i] - MAGIC) * r.scale;
  if (at + 8 <= cols) {
    *(u32x2_any1*)(q + at) = u32x2_any1{low_bytes(t), low_bytes(t + 4)};
    if (values) store8_any(values + at, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (at + i < cols) {
        q[at + i] = (int8_t)__float_as_uint(t[i]);
        if (values) values[at + i] = from_f32<T>(v[i]);
      }
  }
}
// the largest over LANES: part of a wave, or a workgroup of several
template <int LANES> __device__ __forceinline__ uint32_t row_top(uint32_t top, uint32_t* red) {
  constexpr int WAVES = LANES / 64;
#pragma unroll
  for (int o = LANES < 64 ? LANES / 2 : 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  if (WAVES > 1) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; w++) top = max(top, red[w]);
  }
  return top;
}

// LANES (a wave or part of one, or a whole workgroup) take a row, VECTORS x 8 elements each, in registers: one read. Bound by memory: 20480 bf16
// rows of 12288 with their values 230 us, 5.5 TB/s (a large copy 5.0); 12288 fp32 rows of 3072 62 us; 20480 bf16 rows of 3072 without
// values 41 us. One row of 12288 takes 3.3 us on the device, most of it the launch.
template <typename T, int LANES, int VECTORS>
__global__ void __launch_bounds__(LANES < 256 ? 256 : LANES) quantize_kernel(const QuantArgs a) {
  __shared__ uint32_t red[LANES < 64 ? 1 : LANES / 64];
  constexpr int PER = LANES < 256 ? 256 / LANES : 1;   // rows of a workgroup
  const int lane = threadIdx.x % LANES;
  for (int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / LANES; row < a.rows; row += (int64_t)gridDim.x * PER) {
    const T* x = (const T*)a.x + row * a.x_row;
    Eight<T> e[VECTORS];
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < VECTORS; k++) load_row8(x, 8 * (lane + LANES * k), a.cols, e[k]);
#pragma unroll
    for (int k = 0; k < VECTORS; k++) top = max(top, e[k].top());
    const RowScale r = row_scale(row_top<LANES>(top, red));
    if (lane == 0) a.scale[row] = r.bad ? NAN : r.scale;
#pragma unroll
    for (int k = 0; k < VECTORS; k++)
      store_row8<T>(r, e[k], 8 * (lane + LANES * k), a.cols, a.q + row * a.q_row,
                    a.values ? (T*)a.values + row * a.values_row : nullptr);
  }
}
// Longer rows: a workgroup reads them twice.
template <typename T>
__global__ void __launch_bounds__(1024) quantize_long_kernel(const QuantArgs a) {
  __shared__ uint32_t red[16];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = (const T*)a.x + row * a.x_row;
    Eight<T> e;
    uint32_t top = 0;
    for (int64_t at = 8 * threadIdx.x; at < a.cols; at += 8 * 1024) {
      load_row8(x, (int)at, a.cols, e);
      top = max(top, e.top());
    }
    const RowScale r = row_scale(row_top<1024>(top, red));
    if (threadIdx.x == 0) a.scale[row] = r.bad ? NAN : r.scale;
    for (int64_t at = 8 * threadIdx.x; at < a.cols; at += 8 * 1024) {
      load_row8(x, (int)at, a.cols, e);
      store_row8<T>(r, e, (int)at, a.cols, a.q + row * a.q_row, a.values ? (T*)a.values + row * a.values_row : nullptr);
    }
  }
}

template <typename T, int LANES, int VECTORS> void quantize(const QuantArgs& a, hipStream_t s) {
  constexpr int PER = LANES < 256 ? 256 / LANES : 1;
  const int grid = (int)std::min<int64_t>(((int64_t)a.rows + PER - 1) / PER, 1 << 20);
  quantize_kernel<T, LANES, VECTORS><<<grid, LANES < 256 ? 256 : LANES, 0, s>>>(a);
}
// As many lanes as fill the row with few vectors each (rows of 12288 by 256 lanes of 8 vectors: 20480 of them 350 us, one 9.6; rows of 256 by a
// whole wave: 100000 of them 36 us, by half a wave 21).
template <typename T> hipError_t quantize_any(const QuantArgs& a, hipStream_t s) {
  if (a.cols <= 128) quantize<T, 16, 1>(a, s);
  else if (a.cols <= 256) quantize<T, 32, 1>(a, s);
  else if (a.cols <= 512) quantize<T, 64, 1>(a, s);
  else if (a.cols <= 1024) quantize<T, 64, 2>(a, s);
  else if (a.cols <= 2048) quantize<T, 256, 1>(a, s);
  else if (a.cols <= 4096) quantize<T, 256, 2>(a, s);
  else if (a.cols <= 8192) quantize<T, 512, 2>(a, s);
  else if (a.cols <= 12288) quantize<T, 512, 3>(a, s);
  else if (a.cols <= 16384) quantize<T, 512, 4>(a, s);
  else if (a.cols <= 32768) quantize<T, 1024, 4>(a, s);
  else quantize_long_kernel<T><<<std::min(a.rows, 1 << 20), 1024, 0, s>>>(a);
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

// What a feature contributes to its results.
struct Channel {
  float scale, bias;
};
template <typename T> __device__ __forceinline__ Channel channel(const Int8Args& a, int n) {
  return Channel{a.w_scale[n], a.bias ? to_f32(((const T*)a.bias)[n]) : 0.f};
}
template <int ACT> __device__ __forceinline__ float finish(int sum, float x_scale, Channel c) {
  // (two products and a sum, each rounded by itself in every form of the product)
#pragma clang fp contract(off)
  const float v = (float)sum * x_scale * c.scale + c.bias;
  return ACT ? gelu_tanh_f(v) : v;
}
// four successive features of a row, as far as it goes
template <typename T> __device__ __forceinline__ void store_features(const Int8Args& a, const float* v, int m, int n) {
  T* y = (T*)a.y + (int64_t)m * a.y_row + n;
  if (n + 4 <= a.N) {
    store4_any(y, v);
  } else {
#pragma unroll
    for (int q = 0; q < 4; q++)
      if (n + q < a.N) y[q] = from_f32<T>(v[q]);
  }
}

constexpr uint32_t OUTSIDE = 0xC0000000u;   // an offset past any tile's records, also with what a burst adds

// RING = 0 (256-row tiles): three LDS stages of x and two of w (160 KB), the pipeline of the bf16 GEMM's large tile, at
// twice its depth per byte. RING > 0: a ring of RING stages of both.
// Bound by the matrix units, at the clock that the chip's power leaves: 20480 x 3072 -> 12288 in 610 us (590-640 from card to card), 2540
// TOP/s (a library product of these integers: 720 us), with gelu 640. A 256 x 256 tile takes 2380 cycles per k-tile, 2048 of them the products'
// (one of 128 x 128: 1030 and 512; more stages, fewer LDS reads per product or two tiles to a barrier did not help), 2.3 GHz on few CUs and 1.6-1.75 on all.
// bf16 rows of y that do not start at multiples of 4 bytes cost stores of parts of a word: on one card 20480 x 3072 -> 12288 624 us, -> 12284 634,
// -> 12287 752.
template <int BM, int BN, int WM, int WN, int RING, int ACT, typename T>
__global__ void __launch_bounds__(WM * WN * 64) int8_gemm_kernel(const Int8Args a, int total_tiles) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr bool TRI = RING == 0;
  constexpr int NW = WM * WN, NT = NW * 64;
  constexpr int WTM = BM / WM, WTN = BN / WN, TJ = WTM / 16, TI = WTN / 16;   // wave tile, its blocks along rows and features
  constexpr int X_LOADS = BM / 8 / NW, W_LOADS = BN / 8 / NW;                 // 8-row groups that a wave loads per k-tile
  constexpr int X_BYTES = BM * 128, W_BYTES = BN * 128;
  static_assert(X_LOADS >= 1 && W_LOADS >= 1, "every wave loads at least one row group");
  static_assert(TI % 2 == 0, "the paired store joins blocks 2p and 2p + 1");
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int per = gridDim.x >> 3;
  const int t = (blockIdx.x & 7) * per + (blockIdx.x >> 3);   // XCD-aware, as in the bf16 kernel
  if (t >= total_tiles) return;
  int tm, tn;
  tile_coords(t, cdiv(a.M, BM), cdiv(a.N, BN), tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int K = a.K, nk = (K + 127) / 128;

  // a wave load fills 8 rows: lane -> row lane / 8, slot lane % 8, which holds chunk slot ^ swz(row); bursts carry -1024 i in
  // their offsets and 4 KB that the base lacks
  constexpr bool BX = X_LOADS == 3 || X_LOADS == 4, BW = W_LOADS == 3 || W_LOADS == 4;
  const int lrow = lane >> 3;
  u32x4_t rx = rows_rsrc(a.x + (int64_t)m0 * a.x_row - (BX ? 4096 : 0), min(BM, a.M - m0), a.x_row, K);
  u32x4_t rw = rows_rsrc(a.w + (int64_t)n0 * a.w_row - (BW ? 4096 : 0), min(BN, a.N - n0), a.w_row, K);
  if (BX) rx[2] += 4096;
  if (BW) rw[2] += 4096;
  uint32_t xoff[X_LOADS], woff[W_LOADS];
  int xchunk[X_LOADS], wchunk[W_LOADS];
#pragma unroll
  for (int i = 0; i < X_LOADS; i++) {
    const int r = 8 * (wave * X_LOADS + i) + lrow;
    xchunk[i] = ((lane & 7) ^ swz(r)) * 16;
    xoff[i] = m0 + r < a.M ? (uint32_t)(r * a.x_row) + xchunk[i] + (BX ? 4096u - 1024u * i : 0u) : OUTSIDE;
  }
#pragma unroll
  for (int i = 0; i < W_LOADS; i++) {
    const int r = 8 * (wave * W_LOADS + i) + lrow;
    wchunk[i] = ((lane & 7) ^ swz(r)) * 16;
    woff[i] = n0 + r < a.N ? (uint32_t)(r * a.w_row) + wchunk[i] + (BW ? 4096u - 1024u * i : 0u) : OUTSIDE;
  }
  // RING = 0: [W0][W1][X0][X1][X2], tile kt uses w stage kt % 2 and x stage kt % 3; else stage kt % RING of [W][X] pairs
  auto stage_w = [&](int kt) -> uint32_t { return TRI ? (kt & 1) * W_BYTES : (kt % (RING + TRI)) * (X_BYTES + W_BYTES); };
  auto stage_x = [&](int kt) -> uint32_t {
    return TRI ? 2 * W_BYTES + (kt % 3) * X_BYTES : (kt % (RING + TRI)) * (X_BYTES + W_BYTES) + W_BYTES;
  };
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem;
  // END: the tile may be the last one, whose chunks past the row's end read zeros
  auto issue_x = [&](int kt, auto end_c) {
    constexpr bool END = decltype(end_c)::value;
    const uint32_t to = lds0 + stage_x(kt) + wave * X_LOADS * 1024;
    uint32_t off[X_LOADS];
#pragma unroll
    for (int i = 0; i < X_LOADS; i++) off[i] = END && kt * 128 + xchunk[i] >= K ? OUTSIDE : xoff[i];
    if constexpr (BX) {
      dma_burst<X_LOADS>(rx, to, off, kt * 128);
    } else {
#pragma unroll
      for (int i = 0; i < X_LOADS; i++) dma_b128(rx, to + i * 1024, off[i], kt * 128);
    }
  };
  auto issue_w = [&](int kt, auto end_c) {
    constexpr bool END = decltype(end_c)::value;
    const uint32_t to = lds0 + stage_w(kt) + wave * W_LOADS * 1024;
    uint32_t off[W_LOADS];
#pragma unroll
    for (int i = 0; i < W_LOADS; i++) off[i] = END && kt * 128 + wchunk[i] >= K ? OUTSIDE : woff[i];
    if constexpr (BW) {
      dma_burst<W_LOADS>(rw, to, off, kt * 128);
    } else {
#pragma unroll
      for (int i = 0; i < W_LOADS; i++) dma_b128(rw, to + i * 1024, off[i], kt * 128);
    }
  };
  using End = std::true_type;

  i32x4 acc[TI][TJ];
#pragma unroll
  for (int i = 0; i < TI; i++)
#pragma unroll
    for (int j = 0; j < TJ; j++) acc[i][j] = i32x4{0, 0, 0, 0};
  const int wm = wave / WN, wn = wave % WN;
  const int frow = lane & 15, lkc = lane >> 4;   // row inside a 16-row block, 16-byte chunk inside a 64-byte step
  int fwk[TI], fxk[TJ];
#pragma unroll
  for (int i = 0; i < TI; i++) fwk[i] = swz(wn * WTN + 16 * i + frow);
#pragma unroll
  for (int j = 0; j < TJ; j++) fxk[j] = swz(wm * WTM + 16 * j + frow);
  const int wrow0 = (wn * WTN + frow) * 128, xrow0 = (wm * WTM + frow) * 128;
  // fragments of step s, register-double-buffered so that step s + 1 loads while step s multiplies
  i32x4 fw[2][TI], fx[2][TJ];
  auto frags = [&](int kt, int s, int rb) {
    const char* sx = smem + stage_x(kt);
    const char* sw = smem + stage_w(kt);
    const int c = 4 * s + lkc;
#pragma unroll
    for (int i = 0; i < TI; i++) fw[rb][i] = *(const i32x4*)(sw + wrow0 + i * 2048 + ((c ^ fwk[i]) << 4));
#pragma unroll
    for (int j = 0; j < TJ; j++) fx[rb][j] = *(const i32x4*)(sx + xrow0 + j * 2048 + ((c ^ fxk[j]) << 4));
  };
  auto mask_last = [&](int s) {   // of the last tile's step s, once its fragments are there
    const i32x4 mask = row_mask((nk - 1) * 128 + 64 * s + 16 * lkc, K);
#pragma unroll
    for (int j = 0; j < TJ; j++) fx[s][j] &= mask;
  };
  auto multiply = [&](int rb, int i0, int i1) {
#pragma unroll
    for (int i = i0; i < i1; i++)
#pragma unroll
      for (int j = 0; j < TJ; j++) acc[i][j] = mfma_i8(fw[rb][i], fx[rb][j], acc[i][j]);
  };

  // What the epilogue needs of the features and rows, requested before the last k-tile: a feature for each thread, a row of each block.
  // Branch-free: past the end they read the last one's.
  static_assert(BN <= NT, "a thread for each feature");
  Channel pre_c{0.f, 0.f};
  float pre_x[TJ];
  auto prefetch = [&]() {
    pre_c = channel<T>(a, min(n0 + min(tid, BN - 1), a.N - 1));
#pragma unroll
    for (int j = 0; j < TJ; j++) pre_x[j] = a.x_scale[min(m0 + wm * WTM + 16 * j + frow, a.M - 1)];
  };

  if constexpr (TRI) {
    // as in the bf16 kernel: the refill of an x stage in the first step, of a w stage after the barrier, which sits at the last step,
    // whose fragments are in registers; a wave's issue priority falls from barrier to barrier
    constexpr int NM = TI * TJ;
    auto ktile = [&](int kt, auto ph_c) {
      constexpr int PH = decltype(ph_c)::value;   // 0, 1: refill tile kt + 2 (1: the last one); 2: none; 3: last tile
      using Kind = std::integral_constant<bool, PH == 1>;
#pragma unroll
      for (int s = 0; s < 2; s++) {
        const int rb = s;
        if (s == 0) {
          __builtin_amdgcn_s_setprio(1);
          frags(kt, 1, 1);
          if constexpr (PH <= 1) issue_x(kt + 2, Kind());
        } else if constexpr (PH < 3) {
          if (PH < 2) __builtin_amdgcn_s_waitcnt(0x0070 | X_LOADS);
          else __builtin_amdgcn_s_waitcnt(0);
          __syncthreads();
          __builtin_amdgcn_s_setprio(3);
          if constexpr (PH <= 1) issue_w(kt + 2, Kind());
          frags(kt + 1, 0, 0);
        }
        if constexpr (PH == 3) mask_last(s);
        multiply(rb, 0, TI / 2);
        if constexpr (PH < 3) {
          if (s == 0) sched_step<NM / 2, PH <= 1 ? X_LOADS : 0, TI + TJ>();
          else sched_step<NM / 2, PH <= 1 ? W_LOADS : 0, TI + TJ>();
        }
        if (s == 1) __builtin_amdgcn_s_setprio(2);
        else __builtin_amdgcn_s_setprio(0);
        multiply(rb, TI / 2, TI);
      }
    };
    issue_x(0, End());
    issue_w(0, End());
    if (nk > 1) issue_x(1, End());
    if (nk > 1) __builtin_amdgcn_s_waitcnt(0x0070 | X_LOADS);
    else __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (nk > 1) issue_w(1, End());
    frags(0, 0, 0);
    for (int kt = 0; kt + 3 < nk; kt++) ktile(kt, std::integral_constant<int, 0>());
    if (nk >= 3) ktile(nk - 3, std::integral_constant<int, 1>());
    if (nk >= 2) ktile(nk - 2, std::integral_constant<int, 2>());
    prefetch();
    ktile(nk - 1, std::integral_constant<int, 3>());
    __builtin_amdgcn_s_setprio(0);
  } else {
    // All stages are filled up front. The hand-over from tile kt to kt + 1 sits before the last step's products, whose fragments are in
    // registers: tile kt + 1 has landed (the loads of the RING - 2 tiles after it stay in flight), barrier. Stage kt % RING then takes tile
    // kt + RING. SPREAD: w between the products of that step, x between those of the next, so that the loads' issue does not stand before the
    // products (128 x 12288 -> 3072 48 -> 43 us, 512 x 4096 -> 4096 20.5 -> 17.7; where the whole chip is busy its clock falls to 1.6 GHz
    // and nothing is gained: 1280 x 12288 -> 3072 62 and 63). Tiles of 64, of which a CU holds three, are faster without (28 and 31).
    constexpr int L = X_LOADS + W_LOADS;
    constexpr bool SPREAD = BM * BN > 64 * 64;
    static_assert(RING <= 4 && (RING - 2) * L <= 15 && (RING - 1) * L <= 63 && X_LOADS <= TI && W_LOADS <= TI, "the waits and places below");
    auto wait_tiles = [&](int n) {   // at most the loads of n tiles in flight, LDS reads done
      if (n >= RING - 2) __builtin_amdgcn_s_waitcnt(0x0070 | ((RING - 2) * L & 15));
      else if (n == 1) __builtin_amdgcn_s_waitcnt(0x0070 | (L & 15));
      else __builtin_amdgcn_s_waitcnt(0x0070);
    };
    // the products of a step, with the refill of one operand by tile `to` between them
    auto products = [&](int rb, auto op_c, int to) {
      constexpr int OP = decltype(op_c)::value;   // 0: none, 1: w, 2: x
#pragma unroll
      for (int i = 0; i < TI; i++) {
        multiply(rb, i, i + 1);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (OP == 1)
          if (i < W_LOADS) dma_b128(rw, lds0 + stage_w(to) + (wave * W_LOADS + i) * 1024, to * 128 + wchunk[i] >= K ? OUTSIDE : woff[i], to * 128);
        if constexpr (OP == 2)
          if (i < X_LOADS) dma_b128(rx, lds0 + stage_x(to) + (wave * X_LOADS + i) * 1024, to * 128 + xchunk[i] >= K ? OUTSIDE : xoff[i], to * 128);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    using None = std::integral_constant<int, 0>;
    using OfW = std::integral_constant<int, 1>;
    using OfX = std::integral_constant<int, 2>;
    auto step = [&](int kt, auto x_c, auto w_c) {   // a tile that is not the last
      constexpr bool REFILL = decltype(w_c)::value != 0;
      frags(kt, 1, 1);
      if constexpr (SPREAD) {
        __builtin_amdgcn_sched_barrier(0);
        products(0, x_c, kt - 1 + RING);
      } else {
        multiply(0, 0, TI);
      }
      wait_tiles(REFILL ? RING - 2 : nk - 2 - kt);
      __syncthreads();
      if constexpr (REFILL && !SPREAD) {
        issue_x(kt + RING, End());
        issue_w(kt + RING, End());
      }
      frags(kt + 1, 0, 0);
      if constexpr (SPREAD) {
        __builtin_amdgcn_sched_barrier(0);
        products(1, w_c, kt + RING);
      } else {
        multiply(1, 0, TI);
      }
    };
    for (int kt = 0; kt < RING && kt < nk; kt++) {
      issue_x(kt, End());
      issue_w(kt, End());
    }
    if (nk >= RING) __builtin_amdgcn_s_waitcnt(0x0070 | ((RING - 1) * L & 15) | (((RING - 1) * L >> 4) << 14));
    else wait_tiles(nk - 1);
    __syncthreads();
    frags(0, 0, 0);
    int kt = 0;
    if constexpr (SPREAD) {
      if (nk > RING) {
        step(0, None(), OfW());
        for (kt = 1; kt + RING < nk; kt++) step(kt, OfX(), OfW());
        step(kt++, OfX(), None());
      }
    } else {
      for (; kt + RING < nk; kt++) step(kt, OfX(), OfW());
    }
    for (; kt + 1 < nk; kt++) step(kt, None(), None());
    prefetch();
    frags(nk - 1, 1, 1);
    mask_last(0);
    multiply(0, 0, TI);
    mask_last(1);
    multiply(1, 0, TI);
  }

  __syncthreads();   // every wave is done with the operand tiles
  Channel* sc = (Channel*)smem;
  if (tid < BN) sc[tid] = pre_c;
  __syncthreads();
  // block (i, j), register q: feature 16 i + 4 (lane / 16) + q, row 16 j + lane % 16. bf16: blocks i and i + 1 are regrouped so that a lane
  // holds 8 adjacent features, stored with one 16-byte store at any alignment.
  constexpr bool PAIRS = sizeof(T) == 2;
  const int pair_col = 16 * (lkc & 1) + 8 * (lkc >> 1);
  auto values = [&](int i, int j, float* v) {
    const int nl = wn * WTN + 16 * i + 4 * lkc;
#pragma unroll
    for (int q = 0; q < 4; q++) v[q] = finish<ACT>(acc[i][j][q], pre_x[j], sc[nl + q]);
  };
#pragma unroll
  for (int j = 0; j < TJ; j++) {
    const int m = m0 + wm * WTM + 16 * j + frow;
    if (m >= a.M) continue;   // the swap partners (lanes l and l ^ 16) share the row m
    if constexpr (PAIRS) {
#pragma unroll
      for (int p = 0; p < TI / 2; p++) {
        uint32_t w[2][2];
#pragma unroll
        for (int e = 0; e < 2; e++) {
          float v[4];
          values(2 * p + e, j, v);
          w[e][0] = pack_bf16x2(v[0], v[1]);
          w[e][1] = pack_bf16x2(v[2], v[3]);
        }
        swap16(w[0][0], w[1][0]);
        swap16(w[0][1], w[1][1]);
        const int n = n0 + wn * WTN + 32 * p + pair_col;
        u16* y = (u16*)a.y + (int64_t)m * a.y_row + n;
        if (n + 8 <= a.N) {
          *(u32x4_any2*)y = u32x4_any2{w[0][0], w[0][1], w[1][0], w[1][1]};
        } else {
#pragma unroll
          for (int e = 0; e < 8; e++)
            if (n + e < a.N) y[e] = (u16)(w[e >> 2][(e >> 1) & 1] >> (16 * (e & 1)));
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < TI; i++) {
        const int n = n0 + wn * WTN + 16 * i + 4 * lkc;
        float v[4];
        values(i, j, v);
        if (n < a.N) store_features<T>(a, v, m, n);
      }
    }
  }
#endif
}

// B x B tile for few tiles: each of the 4 waves takes every 4th 128-byte slice of the whole tile, with two LDS stages of its own, so no barrier
// stands in the k loop; the partial tiles meet in LDS. A quarter of the chain of the other forms per tile.
template <int B, int ACT, typename T>
__global__ void __launch_bounds__(256) int8_ksplit_kernel(const Int8Args a, int total_tiles) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int NB = B / 16, LD = B / 8, STAGE = 2 * B * 128;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int per = gridDim.x >> 3;
  const int t = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if (t >= total_tiles) return;
  int tm, tn;
  tile_coords(t, cdiv(a.M, B), cdiv(a.N, B), tm, tn);
  const int m0 = tm * B, n0 = tn * B;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int K = a.K, nk = (K + 127) / 128;
  const u32x4_t rx = rows_rsrc(a.x + (int64_t)m0 * a.x_row, min(B, a.M - m0), a.x_row, K);
  const u32x4_t rw = rows_rsrc(a.w + (int64_t)n0 * a.w_row, min(B, a.N - n0), a.w_row, K);
  uint32_t xoff[LD], woff[LD];
#pragma unroll
  for (int i = 0; i < LD; i++) {
    const int r = 8 * i + (lane >> 3);
    const uint32_t chunk = ((lane & 7) ^ swz(r)) * 16;
    xoff[i] = m0 + r < a.M ? (uint32_t)(r * a.x_row) + chunk : OUTSIDE;
    woff[i] = n0 + r < a.N ? (uint32_t)(r * a.w_row) + chunk : OUTSIDE;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem + wave * 2 * STAGE;
  auto issue = [&](int kt, int st) {
    const uint32_t base = lds0 + st * STAGE;
#pragma unroll
    for (int i = 0; i < LD; i++) {
      const bool in = kt * 128 + ((lane & 7) ^ swz(8 * i + (lane >> 3))) * 16 < K;
      dma_b128(rx, base + i * 1024, in ? xoff[i] : OUTSIDE, kt * 128);
      dma_b128(rw, base + B * 128 + i * 1024, in ? woff[i] : OUTSIDE, kt * 128);
    }
  };
  const int r16 = lane & 15, kq = lane >> 4;
  i32x4 acc[NB][NB];
#pragma unroll
  for (int i = 0; i < NB; i++)
#pragma unroll
    for (int j = 0; j < NB; j++) acc[i][j] = i32x4{0, 0, 0, 0};
  if (wave < nk) issue(wave, 0);
  if (wave + 4 < nk) issue(wave + 4, 1);
  int st = 0;
  for (int kt = wave; kt < nk; kt += 4) {
    // this wave's slice kt has landed (the 2 LD loads of its next slice may be in flight)
    if (kt + 4 >= nk) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    else if (LD == 4) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
    const char* sx = smem + wave * 2 * STAGE + st * STAGE;
    const char* sw = sx + B * 128;
    i32x4 fw[2][NB], fx[2][NB];
#pragma unroll
    for (int s = 0; s < 2; s++)
#pragma unroll
      for (int i = 0; i < NB; i++) {
        const int r = 16 * i + r16;
        fw[s][i] = *(const i32x4*)(sw + r * 128 + (((4 * s + kq) ^ swz(r)) << 4));
        fx[s][i] = *(const i32x4*)(sx + r * 128 + (((4 * s + kq) ^ swz(r)) << 4));
      }
    if (kt + 8 < nk) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the fragments are in registers: the stage is free
      issue(kt + 8, st);
    }
    if (kt + 1 == nk) {
#pragma unroll
      for (int s = 0; s < 2; s++) {
        const i32x4 mask = row_mask(kt * 128 + 64 * s + 16 * kq, K);
#pragma unroll
        for (int i = 0; i < NB; i++) fx[s][i] &= mask;
      }
    }
#pragma unroll
    for (int s = 0; s < 2; s++)
#pragma unroll
      for (int i = 0; i < NB; i++)
#pragma unroll
        for (int j = 0; j < NB; j++) acc[i][j] = mfma_i8(fw[s][i], fx[s][j], acc[i][j]);
    st ^= 1;
  }
  __syncthreads();   // every wave's loads have landed and been read
  i32x4* part = (i32x4*)smem;   // [block][wave][lane]
#pragma unroll
  for (int i = 0; i < NB; i++)
#pragma unroll
    for (int j = 0; j < NB; j++) part[((NB * i + j) * 4 + wave) * 64 + lane] = acc[i][j];
  __syncthreads();
#pragma unroll
  for (int q = 0; q < NB * NB / 4; q++) {
    const int blk = wave * (NB * NB / 4) + q, i = blk / NB, j = blk % NB;
    i32x4 c = part[(blk * 4) * 64 + lane];
#pragma unroll
    for (int g = 1; g < 4; g++) c += part[(blk * 4 + g) * 64 + lane];
    const int m = m0 + 16 * j + r16, n = n0 + 16 * i + 4 * kq;
    if (m < a.M && n < a.N) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; e++) v[e] = finish<ACT>(c[e], a.x_scale[m], channel<T>(a, min(n + e, a.N - 1)));
      store_features<T>(a, v, m, n);
    }
  }
#endif
}

// Small products of rows that are not integers yet, in one launch: a 32 x 32 tile as above, whose workgroup first rounds its 32 rows of x into
// LDS, eight lanes to a row, while its slices of w are on their way. Bound by latency: the launch, x, w, the sums. Against a launch that
// rounds the rows and one that multiplies (us, as eager calls and in a graph): 3 x 256 -> 256 6.6 and 4.0 for 9.6 and 6.1, 500 x 256 -> 1024 6.7 and
// 6.4 for 9.6 and 8.7, 500 x 512 -> 1024 9.5 and 9.3 for 10.1 and 9.2; rows of 1001 (333 of them, 515 features) took 12.4 for 10.0 and 7.9.
constexpr int RAW_K = 512;   // longest rows: four k-tiles, one for each wave
static_assert(RAW_K <= 4 * 128, "a wave has one slice of k at most");
template <int VECTORS, int ACT, typename T>
__global__ void __launch_bounds__(256) int8_small_kernel(const Int8Args a, int total_tiles) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int B = 32, STAGE = B * 128;
  extern __shared__ __attribute__((aligned(1024))) char smem[];   // x [k-tile][row][128], then each wave's slice of w
  __shared__ float scales[B];
  const int per = gridDim.x >> 3;
  const int t = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if (t >= total_tiles) return;
  int tm, tn;
  tile_coords(t, cdiv(a.M, B), cdiv(a.N, B), tm, tn);
  const int m0 = tm * B, n0 = tn * B;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int K = a.K, nk = (K + 127) / 128;
  const u32x4_t rw = rows_rsrc(a.w + (int64_t)n0 * a.w_row, min(B, a.N - n0), a.w_row, K);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem + (nk + wave) * STAGE;
  auto issue = [&](int kt) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int r = 8 * i + (lane >> 3), chunk = ((lane & 7) ^ swz(r)) * 16;
      const bool in = kt * 128 + chunk < K && n0 + r < a.N;
      dma_b128(rw, lds0 + i * 1024, in ? (uint32_t)(r * a.w_row) + chunk : OUTSIDE, kt * 128);
    }
  };
  const int row = tid >> 3, part = tid & 7;   // elements 8 (part + 8 v) .. + 7 of a row; rows past the end repeat the last and are not stored
  const T* x = (const T*)a.raw + min(m0 + row, a.M - 1) * a.raw_row;
  Eight<T> e[VECTORS];
#pragma unroll
  for (int v = 0; v < VECTORS; v++) {
    const int at = 8 * (part + 8 * v);
    if (K % 8 == 0) e[v].load(x + min(at, K - 8));   // (past the end: repeats the last ones, which does not change the largest)
    else load_row8(x, at, K, e[v]);
  }
  if (wave < nk) issue(wave);
  uint32_t top = 0;
#pragma unroll
  for (int v = 0; v < VECTORS; v++) top = max(top, e[v].top());
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  const RowScale r = row_scale(top);
  if (part == 0) scales[row] = r.bad ? NAN : r.scale;
#pragma unroll
  for (int v = 0; v < VECTORS; v++) {
    const int at = 8 * (part + 8 * v);
    if (at >= nk * 128) break;
    float f[8], z[8];
    e[v].get(f);
    to_integers(r, f, z);
    const bool none = r.bad || at >= K;
    *(uint2*)(smem + (at >> 7) * STAGE + row * 128 + ((((at >> 4) & 7) ^ swz(row)) << 4) + (at & 8)) =
        none ? make_uint2(0, 0) : make_uint2(low_bytes(z), low_bytes(z + 4));
  }
  __syncthreads();

  const int r16 = lane & 15, kq = lane >> 4;
  i32x4 acc[2][2] = {};
  if (wave < nk) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const char* sx = smem + wave * STAGE;
    const char* sw = smem + (nk + wave) * STAGE;
    i32x4 fw[2][2], fx[2][2];
#pragma unroll
    for (int s = 0; s < 2; s++)
#pragma unroll
      for (int i = 0; i < 2; i++) {
        const int fr = 16 * i + r16;
        fw[s][i] = *(const i32x4*)(sw + fr * 128 + (((4 * s + kq) ^ swz(fr)) << 4));
        fx[s][i] = *(const i32x4*)(sx + fr * 128 + (((4 * s + kq) ^ swz(fr)) << 4));
      }
#pragma unroll
    for (int s = 0; s < 2; s++)
#pragma unroll
      for (int i = 0; i < 2; i++)
#pragma unroll
        for (int j = 0; j < 2; j++) acc[i][j] = mfma_i8(fw[s][i], fx[s][j], acc[i][j]);
  }
  __syncthreads();   // x and w have been read
  i32x4* sums = (i32x4*)smem;   // [block][wave][lane]
#pragma unroll
  for (int i = 0; i < 2; i++)
#pragma unroll
    for (int j = 0; j < 2; j++) sums[((2 * i + j) * 4 + wave) * 64 + lane] = acc[i][j];
  __syncthreads();
  i32x4 c = sums[(wave * 4) * 64 + lane];   // wave q finishes block (q / 2, q % 2)
#pragma unroll
  for (int g = 1; g < 4; g++) c += sums[(wave * 4 + g) * 64 + lane];
  const int ml = 16 * (wave & 1) + r16, m = m0 + ml, n = n0 + 16 * (wave >> 1) + 4 * kq;
  if (m < a.M && n < a.N) {
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] = finish<ACT>(c[e], scales[ml], channel<T>(a, min(n + e, a.N - 1)));
    store_features<T>(a, v, m, n);
  }
#endif
}

// One or two rows: bound by reading w once. A wave takes F features, 1 KB of each per step (16 bytes a lane), by v_dot4; x lies in LDS as
// integers, zeros behind its end. SHARE: the four waves of a workgroup share the k of the same features (few features).
// RAW: x comes in its own type and every workgroup rounds it by itself while its first weights are on their way: no launch before this one.
// 3072 -> 12288 (37.8 MB): one row 8.9 us, two 10.5, a launch that rounds and the 32 x 32 tiles above 12.2; rows that are integers 7.4 and 8.2,
// tiles 8.5 (four rows 10.4, tiles 8.7: only up to two). SHARE where there are fewer than 512 workgroups otherwise: 12288 -> 3072 8.4 us for 10.2 in
// tiles.
constexpr int F = 4, STEP = 1024;
constexpr int RAW_ELEMENTS = 16384;   // of all rows
template <int ROWS, bool SHARE, bool RAW, int ACT, typename T>
__global__ void __launch_bounds__(256) int8_few_rows_kernel(const Int8Args a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ int part[4][F][ROWS];
  __shared__ uint32_t red[ROWS][4];
  __shared__ float scales[ROWS];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int K = a.K, steps = (K + STEP - 1) / STEP, pad = steps * STEP;
  const int n0 = blockIdx.x * (SHARE ? F : 4 * F), mine = SHARE ? n0 : n0 + wave * F;
  const int8_t* w[F];
#pragma unroll
  for (int f = 0; f < F; f++) w[f] = a.w + (int64_t)min(mine + f, a.N - 1) * a.w_row;   // (features past the end repeat the last, unused)
  constexpr int AHEAD = 4, STRIDE = SHARE ? 4 : 1;
  const int first = SHARE ? wave : 0;
  i32x4 fw[AHEAD][F];
  auto load = [&](int step, i32x4* to) {
    const int at = min(step * STEP + 16 * lane, (K - 1) & ~15);
#pragma unroll
    for (int f = 0; f < F; f++) to[f] = *(const i32x4*)(w[f] + at);
  };
  // (branch-free, so that what was requested before can be waited for alone; steps past the end repeat the last)
  auto load_ahead = [&]() {
#pragma unroll
    for (int u = 0; u < AHEAD; u++) load(min(first + u * STRIDE, steps - 1), fw[u]);
  };

  // x to LDS
  if constexpr (RAW) {
    constexpr int VECTORS = RAW_ELEMENTS / (ROWS * 2048);   // of 8 elements of a row that a thread holds
    Eight<T> e[ROWS][VECTORS];
#pragma unroll
    for (int m = 0; m < ROWS; m++) {
      const T* x = (const T*)a.raw + min(m, a.M - 1) * a.raw_row;
#pragma unroll
      for (int v = 0; v < VECTORS; v++) {
        const int at = 8 * (tid + 256 * v);
        if (K % 8 == 0) e[m][v].load(x + min(at, K - 8));   // (past the end: repeats the last ones, which does not change the largest)
        else load_row8(x, at, K, e[m][v]);
      }
    }
    load_ahead();
#pragma unroll
    for (int m = 0; m < ROWS; m++) {
      uint32_t top = 0;
#pragma unroll
      for (int v = 0; v < VECTORS; v++) top = max(top, e[m][v].top());
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
      if (lane == 0) red[m][wave] = top;
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < ROWS; m++) {
      const RowScale r = row_scale(max(max(red[m][0], red[m][1]), max(red[m][2], red[m][3])));
      if (tid == 0) scales[m] = r.bad ? NAN : r.scale;
#pragma unroll
      for (int v = 0; v < VECTORS; v++) {
        const int at = 8 * (tid + 256 * v);
        if (at >= pad) break;
        float f[8], t[8];
        e[m][v].get(f);
        to_integers(r, f, t);
        const bool none = r.bad || at >= K;   // (K % 8: the elements past the end were read as zeros)
        *(uint2*)(smem + m * pad + at) = none ? make_uint2(0, 0) : make_uint2(low_bytes(t), low_bytes(t + 4));
      }
    }
  } else {
#pragma unroll
    for (int m = 0; m < ROWS; m++) {
      const int8_t* x = a.x + min(m, a.M - 1) * a.x_row;
      for (int at = 16 * tid; at < pad; at += 16 * 256)
        *(i32x4*)(smem + m * pad + at) = *(const i32x4*)(x + min(at, (K - 1) & ~15)) & row_mask(at, K);
      if (tid == 0) scales[m] = a.x_scale[min(m, a.M - 1)];
    }
    load_ahead();
  }
  __syncthreads();

  int acc[F][ROWS];
#pragma unroll
  for (int f = 0; f < F; f++)
#pragma unroll
    for (int m = 0; m < ROWS; m++) acc[f][m] = 0;
  for (int s = first; s < steps; s += AHEAD * STRIDE) {
#pragma unroll
    for (int u = 0; u < AHEAD; u++) {
      const int step = s + u * STRIDE;
      if (step < steps) {
#pragma unroll
        for (int m = 0; m < ROWS; m++) {
          const i32x4 x = *(const i32x4*)(smem + m * pad + step * STEP + 16 * lane);
#pragma unroll
          for (int f = 0; f < F; f++)
#pragma unroll
            for (int i = 0; i < 4; i++) acc[f][m] = __builtin_amdgcn_sdot4(fw[u][f][i], x[i], acc[f][m], false);
        }
        if (step + AHEAD * STRIDE < steps) load(step + AHEAD * STRIDE, fw[u]);
      }
    }
  }
#pragma unroll
  for (int f = 0; f < F; f++)
#pragma unroll
    for (int m = 0; m < ROWS; m++) {
      const int total = (int)wave_scan((unsigned)acc[f][m]);   // in the last lane
      if (lane == 63) part[wave][f][m] = total;
    }
  __syncthreads();
  constexpr int WIDTH = SHARE ? F : 4 * F;   // features of the workgroup
  if (tid >= WIDTH * ROWS) return;
  const int m = tid / WIDTH, f = tid % WIDTH, n = n0 + f;
  if (m >= a.M || n >= a.N) return;
  const int sum = SHARE ? part[0][f][m] + part[1][f][m] + part[2][f][m] + part[3][f][m] : part[f / F][f % F][m];
  ((T*)a.y)[(int64_t)m * a.y_row + n] = from_f32<T>(finish<ACT>(sum, scales[m], channel<T>(a, n)));
}

int64_t tiles_of(int M, int N, int bm, int bn) { return (int64_t)cdiv(M, bm) * cdiv(N, bn); }

// rows of x in LDS
size_t few_rows_lds(int M, int K) { return (size_t)M * ((K + STEP - 1) / STEP * STEP); }

// of one or two rows: whether waves of a workgroup share k, and its workgroups
bool few_rows_share(int N) { return cdiv(N, 4 * F) < 2 * cu_count(); }
int few_rows_blocks(int N) { return cdiv(N, few_rows_share(N) ? F : 4 * F); }

int64_t tile_blocks(int M, int N, int bm, int bn) { return (tiles_of(M, N, bm, bn) + 7) / 8 * 8; }

int64_t form_threads(Int8Form f, int M, int N) {
  switch (f) {
    case INT8_FEW_ROWS: return 256 * (int64_t)few_rows_blocks(N);
    case INT8_KSPLIT_32: return 256 * tile_blocks(M, N, 32, 32);
    case INT8_KSPLIT_64:
    case INT8_RING_64: return 256 * tile_blocks(M, N, 64, 64);
    case INT8_RING_128: return 512 * tile_blocks(M, N, 128, 128);
    case INT8_LARGE_192: return 512 * tile_blocks(M, N, 256, 192);
    case INT8_LARGE_256: return 512 * tile_blocks(M, N, 256, 256);
  }
  return INT64_MAX;
}
// a launch takes fewer than 2^32 threads
bool fits(Int8Form f, int M, int N) { return form_threads(f, M, N) < int64_t(1) << 32; }

}  // namespace

Int8Form int8_form(int M, int N, int K) {
  if (M <= 2 && few_rows_lds(M, K) <= 61440 && fits(INT8_FEW_ROWS, M, N)) return INT8_FEW_ROWS;
  // Estimated times, us. What a CU takes per k-tile: 1.25 for a 256 x 256 tile (near the matrix rate), 0.5 for 128 x 128 and 0.24 for 64 x 64
  // (LDS reads), 0.23 and 0.09 for those whose waves share k; beside it each round's first loads and stores. Measured (us, in this order: 32 and 64
  // with shared k, 64, 128, 256 x 192, 256): 128 x 12288 -> 3072: 19 / 22 / 28 / 43 / 77 / 97; 333 x 3072 -> 9216: 35 / 35 / 22 / 16 / 25 / 31;
  // 512 x 4096 -> 4096: 26 / 21 / 16 / 18 / 31 / 38; 1280 x 3072 -> 9216: 120 / 116 / 69 / 56 / 35 / 38; 1280 x 12288 -> 3072:
  // 137 / 100 / 94 / 62 / 98 / 117; 20480 x 3072 -> 12288: 2307 / 2043 / 1181 / 962 / 640 / 610.
  const double kt = (K + 127) / 128;
  const int64_t cus = cu_count();
  auto rounds = [&](int bm, int bn) { return (double)((tiles_of(M, N, bm, bn) + cus - 1) / cus); };
  auto shares = [&](int b, double slots) { return std::max(1.0, tiles_of(M, N, b, b) / (slots * cus)); };
  double best = rounds(256, 256) * (1.25 * kt + 11.0);
  Int8Form pick = INT8_LARGE_256;
  auto consider = [&](Int8Form f, double cost) {
    if (cost < best && fits(f, M, N)) best = cost, pick = f;
  };
  consider(INT8_LARGE_192, rounds(256, 192) * (1.09 * kt + 8.5));
  consider(INT8_RING_128, rounds(128, 128) * (0.5 * kt + 4.5));
  consider(INT8_RING_64, 3.0 + std::max(0.27 * kt, shares(64, 1) * std::max(0.235 * kt, 0.9 + 0.1 * kt)));
  consider(INT8_KSPLIT_64, rounds(64, 64) * (0.23 * kt + 3.0));
  consider(INT8_KSPLIT_32, 2.5 + shares(32, 2) * (0.185 * kt + 0.7));
  return pick;
}

namespace {

template <int BM, int BN, int WM, int WN, int RING, int ACT, typename T> hipError_t launch_tiles(const Int8Args& a, hipStream_t s) {
  constexpr size_t lds = RING == 0 ? (size_t)(2 * BN + 3 * BM) * 128 : (size_t)RING * (BM + BN) * 128;
  static std::atomic<bool> attr_set[64] = {};
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(&int8_gemm_kernel<BM, BN, WM, WN, RING, ACT, T>), lds, attr_set);
  if (e != hipSuccess) return e;
  const int64_t tiles = tiles_of(a.M, a.N, BM, BN);
  int8_gemm_kernel<BM, BN, WM, WN, RING, ACT, T><<<(int)tile_blocks(a.M, a.N, BM, BN), WM * WN * 64, lds, s>>>(a, (int)tiles);
  return hipGetLastError();
}
template <int B, int ACT, typename T> hipError_t launch_ksplit(const Int8Args& a, hipStream_t s) {
  constexpr size_t lds = (size_t)16 * B * 128;
  static std::atomic<bool> attr_set[64] = {};
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(&int8_ksplit_kernel<B, ACT, T>), lds, attr_set);
  if (e != hipSuccess) return e;
  const int64_t tiles = tiles_of(a.M, a.N, B, B);
  int8_ksplit_kernel<B, ACT, T><<<(int)tile_blocks(a.M, a.N, B, B), 256, lds, s>>>(a, (int)tiles);
  return hipGetLastError();
}
template <int ROWS, bool RAW, int ACT, typename T> hipError_t launch_few(const Int8Args& a, hipStream_t s) {
  const size_t lds = few_rows_lds(a.M, a.K);
  if (few_rows_share(a.N)) int8_few_rows_kernel<ROWS, true, RAW, ACT, T><<<few_rows_blocks(a.N), 256, lds, s>>>(a);
  else int8_few_rows_kernel<ROWS, false, RAW, ACT, T><<<few_rows_blocks(a.N), 256, lds, s>>>(a);
  return hipGetLastError();
}
template <bool RAW, int ACT, typename T> hipError_t launch_few_rows(const Int8Args& a, hipStream_t s) {
  return a.M == 1 ? launch_few<1, RAW, ACT, T>(a, s) : launch_few<2, RAW, ACT, T>(a, s);
}

template <int VECTORS, int ACT, typename T> hipError_t launch_small(const Int8Args& a, hipStream_t s) {
  const size_t lds = (size_t)((a.K + 127) / 128 + 4) * 4096;   // 20 to 32 KB (the sums take 16)
  const int64_t tiles = tiles_of(a.M, a.N, 32, 32);
  int8_small_kernel<VECTORS, ACT, T><<<(int)tile_blocks(a.M, a.N, 32, 32), 256, lds, s>>>(a, (int)tiles);
  return hipGetLastError();
}
template <int ACT, typename T> hipError_t launch_raw(const Int8Args& a, hipStream_t s) {
  if (a.M <= 2) return launch_few_rows<true, ACT, T>(a, s);
  return a.K <= RAW_K / 2 ? launch_small<RAW_K / 128, ACT, T>(a, s) : launch_small<RAW_K / 64, ACT, T>(a, s);
}

template <int ACT, typename T> hipError_t matmul(const Int8Args& a, hipStream_t s) {
  switch (int8_form(a.M, a.N, a.K)) {
    case INT8_FEW_ROWS: return launch_few_rows<false, ACT, T>(a, s);
    case INT8_KSPLIT_32: return launch_ksplit<32, ACT, T>(a, s);
    case INT8_KSPLIT_64: return launch_ksplit<64, ACT, T>(a, s);
    case INT8_RING_64: return launch_tiles<64, 64, 2, 2, 3, ACT, T>(a, s);
    case INT8_RING_128: return launch_tiles<128, 128, 2, 4, 4, ACT, T>(a, s);
    case INT8_LARGE_192: return launch_tiles<256, 192, 4, 2, 0, ACT, T>(a, s);
    case INT8_LARGE_256: return launch_tiles<256, 256, 4, 2, 0, ACT, T>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t quantize_rows_launch(const QuantArgs& a, int dtype, hipStream_t s) {
  return dtype == DT_BF16 ? quantize_any<u16>(a, s) : quantize_any<float>(a, s);
}

// (a product that rounds its own rows has the threads of this form, or 512 small tiles)
int64_t int8_matmul_threads(int M, int N, int K) { return form_threads(int8_form(M, N, K), M, N); }

bool int8_takes_raw(int M, int N, int K) {
  if (M <= 2) return (int64_t)M * K <= RAW_ELEMENTS && fits(INT8_FEW_ROWS, M, N);
  return K <= RAW_K && tiles_of(M, N, 32, 32) <= 2 * cu_count();
}

hipError_t int8_matmul_launch(const Int8Args& a, int dtype, int act, hipStream_t s) {
  if (a.raw) {
    if (dtype == DT_BF16) return act ? launch_raw<1, u16>(a, s) : launch_raw<0, u16>(a, s);
    return act ? launch_raw<1, float>(a, s) : launch_raw<0, float>(a, s);
  }
  if (dtype == DT_BF16) return act ? matmul<1, u16>(a, s) : matmul<0, u16>(a, s);
  return act ? matmul<1, float>(a, s) : matmul<0, float>(a, s);
}

}  // namespace dit
