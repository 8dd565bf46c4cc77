// Pieces that the attention kernels share: exchanges between the halves of a wave, loads that go straight
// into LDS, and the tile layout whose rows are read both as they are and transposed.
#pragma once
#include <type_traits>

#include "internal.h"

namespace dit {

typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));

// Combine the values of lanes l and l ^ 32 through v_permlane32_swap (a VALU exchange of the two
// 32-lane halves) instead of an LDS permute. With both operands v, the swap's two results hold, in
// every lane, v[l] and v[l ^ 32] (which of the two is which depends on the half), so only symmetric
// combinations are formed from them.
__device__ __forceinline__ void half_pair(float v, float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}
__device__ __forceinline__ float pair_max(float v) {
  float a, b;
  half_pair(v, a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float pair_sum(float v) {
  float a, b;
  half_pair(v, a, b);
  return a + b;
}

typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));

// Four direct-to-LDS loads under one M0 value: destination M0 + 1024 i + 16 lane, global offset
// v[i] + 1024 i (the instruction offset moves both addresses). Issued back to back they hold the
// wave's issue for less than four separately issued loads, each of which sets M0 on its own.
// Inline assembly, so the compiler does not track these loads: the wait before the barrier that
// hands a stage over is the explicit s_waitcnt(0) of the loop.
__device__ __forceinline__ void dma4_b128(u32x4_t rsrc, uint32_t m0v, uint32_t v0, uint32_t v1, uint32_t v2,
                                          uint32_t v3) {
  uint32_t saved;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
               "buffer_load_dwordx4 %2, %6, 0 offen lds\n\t"
               "buffer_load_dwordx4 %3, %6, 0 offen offset:1024 lds\n\t"
               "buffer_load_dwordx4 %4, %6, 0 offen offset:2048 lds\n\t"
               "buffer_load_dwordx4 %5, %6, 0 offen offset:3072 lds\n\t"
               "s_mov_b32 m0, %0"
               : "=&s"(saved) : "s"(m0v), "v"(v0), "v"(v1), "v"(v2), "v"(v3), "s"(rsrc) : "memory");
}

// One or two such loads.
__device__ __forceinline__ void dma1_b128(u32x4_t rsrc, uint32_t m0v, uint32_t v0) {
  uint32_t saved;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
               "buffer_load_dwordx4 %2, %3, 0 offen lds\n\t"
               "s_mov_b32 m0, %0"
               : "=&s"(saved) : "s"(m0v), "v"(v0), "s"(rsrc) : "memory");
}
__device__ __forceinline__ void dma2_b128(u32x4_t rsrc, uint32_t m0v, uint32_t v0, uint32_t v1) {
  uint32_t saved;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
               "buffer_load_dwordx4 %2, %4, 0 offen lds\n\t"
               "buffer_load_dwordx4 %3, %4, 0 offen offset:1024 lds\n\t"
               "s_mov_b32 m0, %0"
               : "=&s"(saved) : "s"(m0v), "v"(v0), "v"(v1), "s"(rsrc) : "memory");
}

template <int N> __device__ __forceinline__ void wait_loads() {   // until at most N of this wave's loads are in flight
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}

// A tile of ROWS rows of D bf16 in LDS, loaded by NW waves straight from global memory. 16-byte chunk c of
// row r sits in slot c ^ tile_swizzle<D>(r): sixteen successive rows (eight, two to a 256-byte line, at D = 64)
// put the same chunk into different banks, which serves the b128 reads of rows, and any four aligned rows put
// a 64-byte piece into four different quarters of the banks, which serves the transposing reads.
template <int D> __device__ __forceinline__ int tile_swizzle(int r) {
  return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}
template <int D, int ROWS, int NW> struct RowTile {
  static constexpr int CH = D / 8, RB = D * 2, BYTES = ROWS * RB;
  static constexpr int KPI = 64 / CH, LOADS = ROWS / KPI / NW;   // rows per 1 KB wave load, loads per wave
  static_assert(LOADS >= 1 && LOADS <= 8, "");
  uint32_t off[LOADS];   // global offset of this lane's chunk of load i, less the instruction's own offset
  uint32_t dst, stride;
  // (the descriptor starts 4 KB early so that no offset goes negative)
  __device__ __forceinline__ void init(int wave, int lane, int64_t row_stride) {
    stride = (uint32_t)(row_stride * 2);
    dst = (uint32_t)(__builtin_amdgcn_readfirstlane(wave) * LOADS * 1024);
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      const int row = (wave * LOADS + i) * KPI + lane / CH, slot = lane % CH;
      off[i] = row * stride + ((slot ^ tile_swizzle<D>(row)) << 4) + 4096u - 1024u * (i & 3);
    }
  }
  // rows: how many of the tile's rows exist (uniform); the others read as zeros
  __device__ __forceinline__ void load(const u16* base, int rows, uint32_t lds) const {
    const uint64_t b = (uint64_t)base - 4096;
    const uint32_t nrec = rows > 0 ? (uint32_t)(min(rows, ROWS) - 1) * stride + RB + 4096u : 0u;
    const u32x4_t rs = {(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b),
                        (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32) & 0xffffu),
                        (uint32_t)__builtin_amdgcn_readfirstlane(nrec), 0x00020000u};
    const uint32_t d = lds + dst;
    if constexpr (LOADS == 1) dma1_b128(rs, d, off[0]);
    else if constexpr (LOADS == 2) dma2_b128(rs, d, off[0], off[1]);
    else
#pragma unroll
      for (int i = 0; i < LOADS; i += 4) dma4_b128(rs, d + 1024u * i, off[i], off[i + 1], off[i + 2], off[i + 3]);
  }
  // 8 elements of row `row`, chunk c
  static __device__ __forceinline__ bf16x8 read(const char* tile, int row, int c) {
    return *(const bf16x8*)(tile + row * RB + ((c ^ tile_swizzle<D>(row)) << 4));
  }
};

// Four rows k0..k0+3 of one dim each, transposed: lane s of 16 gives the address of 4 dims of row k0 + s / 4 and gets
// rows k0..k0+3 of dim s of the 16 dims that the group covers.
__device__ __forceinline__ i16x4 read_tr(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p));
}
__device__ __forceinline__ bf16x8 join_tr(i16x4 lo, i16x4 hi) {
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Between accesses to LDS by which the lanes of one wave hand data to each other without a barrier. The unit keeps a wave's accesses
// in order; this keeps the compiler from moving a lane's own across it. No instruction.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// fp32 on v_mfma_f32_16x16x4_f32: 16 owned rows per wave (fragments own[c]: dims 16 c + 4 g4 + 0..3 of row lane % 16, g4 = lane / 16)
// against a walked tile of 16 rows of two tensors, staged through registers into LDS by LANES lanes (a workgroup, or a wave
// with tiles of its own).
template <int D, int LANES> struct WalkF32 {
  static constexpr int NROW = 16, LD = D + 4, CPT = NROW * D / 4 / LANES;
  f32x4 ra[CPT], rb[CPT];
  // rows past `left` are zeros (what they are multiplied with is 0, but 0 times an infinity would be NaN)
  __device__ __forceinline__ void fetch(const float* a, int64_t as, const float* b, int64_t bs, int left) {
#pragma unroll
    for (int i = 0; i < CPT; i++) {
      const int idx = threadIdx.x % LANES + LANES * i, r = idx / (D / 4), c = idx % (D / 4), rr = min(r, left - 1);
      ra[i] = *(const f32x4*)(a + rr * as + 4 * c);
      rb[i] = *(const f32x4*)(b + rr * bs + 4 * c);
      if (r >= left) ra[i] = rb[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  __device__ __forceinline__ void stage(float* sa, float* sb) const {
#pragma unroll
    for (int i = 0; i < CPT; i++) {
      const int idx = threadIdx.x % LANES + LANES * i, r = idx / (D / 4), c = idx % (D / 4);
      *(f32x4*)(sa + r * LD + 4 * c) = ra[i];
      *(f32x4*)(sb + r * LD + 4 * c) = rb[i];
    }
  }
  // [walked row 4 g4 + r][owned row lane % 16] products
  static __device__ __forceinline__ f32x4 dot(const float* st, const f32x4* own, int l16, int g4) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < D / 16; c++) {
      const f32x4 w = *(const f32x4*)(st + l16 * LD + 16 * c + 4 * g4);
#pragma unroll
      for (int e = 0; e < 4; e++) s = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], own[c][e], s, 0, 0, 0);
    }
    return s;
  }
  // acc[dim][owned] += sum over the walked rows of st[row][dim] w[row][owned]
  static __device__ __forceinline__ void add(f32x4* acc, const float* st, const f32x4& w, int l16, int g4) {
#pragma unroll
    for (int r = 0; r < 4; r++)
#pragma unroll
      for (int i = 0; i < D / 16; i++)
        acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(st[(4 * g4 + r) * LD + l16 + 16 * i], w[r], acc[i], 0, 0, 0);
  }
};
// The sums of four waves that own the same rows, in wave 0, through LDS of 3 x 16 x (D + 4) floats.
template <int D> __device__ __forceinline__ void join_waves(float* lds, f32x4* acc, int wave, int l16, int g4) {
  __syncthreads();
  if (wave > 0)
#pragma unroll
    for (int i = 0; i < D / 16; i++) *(f32x4*)(lds + ((wave - 1) * 16 + l16) * (D + 4) + 16 * i + 4 * g4) = acc[i];
  __syncthreads();
  if (wave == 0)
#pragma unroll
    for (int w = 0; w < 3; w++)
#pragma unroll
      for (int i = 0; i < D / 16; i++) acc[i] += *(const f32x4*)(lds + (w * 16 + l16) * (D + 4) + 16 * i + 4 * g4);
}

}  // namespace dit
