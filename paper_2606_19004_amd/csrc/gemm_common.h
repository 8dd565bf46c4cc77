// What the matrix product kernels of k_gemm.hip and k_int8.hip share: direct-to-LDS loads, the LDS swizzle, the order of
// tiles, scheduling hints, and host helpers of their launches.
#pragma once
#include <atomic>

#include "internal.h"

namespace dit {

__device__ __forceinline__ float gelu_tanh_f(float z) {
  // 0.5 z (1 + tanh(u)) = z * sigmoid(2u), u = sqrt(2/pi) (z + 0.044715 z^3), and
  // sigmoid(2u) = 1 / (1 + 2^(-2u log2 e)) with -2u log2 e = z (K1 + K2 z^2)
  constexpr float K1 = -2.0f * 0.7978845608028654f * 1.4426950408889634f;
  constexpr float K2 = K1 * 0.044715f;
  return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * fmaf(K2, z * z, K1)));
}

typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));

// Direct-to-LDS 16-byte-per-lane buffer load (M0 = LDS destination of lane 0), written as inline
// assembly so that the compiler does not track it: with LDS addresses chosen at run time it cannot
// prove that a later LDS read does not alias the load, and would wait for all loads in flight. The
// caller's explicit s_waitcnt vmcnt is the only synchronisation for these loads. M0 is reserved by
// the compiler, so the sequence saves it in a scratch SGPR and restores it after issuing the load
// (the destination is taken from M0 when the load issues). rsrc is a raw buffer descriptor (base,
// stride 0, num_records, flags).
__device__ __forceinline__ void dma_b128(u32x4_t rsrc, uint32_t m0v, uint32_t voff, uint32_t soff) {
  uint32_t saved;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, %4 offen lds\n\t"
               "s_mov_b32 m0, %0"
               : "=&s"(saved) : "s"(m0v), "v"(voff), "s"(rsrc), "s"(soff) : "memory");
}

// N (3 or 4) direct-to-LDS loads sharing one M0: destination M0 + 1024 i + 16 lane, global offset
// v[i] + 1024 i (the instruction offset moves both addresses)
template <int N>
__device__ __forceinline__ void dma_burst(u32x4_t rsrc, uint32_t m0v, const uint32_t* v, uint32_t soff) {
  uint32_t saved;
  if constexpr (N == 4)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                 "buffer_load_dwordx4 %2, %6, %7 offen lds\n\t"
                 "buffer_load_dwordx4 %3, %6, %7 offen offset:1024 lds\n\t"
                 "buffer_load_dwordx4 %4, %6, %7 offen offset:2048 lds\n\t"
                 "buffer_load_dwordx4 %5, %6, %7 offen offset:3072 lds\n\t"
                 "s_mov_b32 m0, %0"
                 : "=&s"(saved) : "s"(m0v), "v"(v[0]), "v"(v[1]), "v"(v[2]), "v"(v[3]), "s"(rsrc), "s"(soff) : "memory");
  else
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                 "buffer_load_dwordx4 %2, %5, %6 offen lds\n\t"
                 "buffer_load_dwordx4 %3, %5, %6 offen offset:1024 lds\n\t"
                 "buffer_load_dwordx4 %4, %5, %6 offen offset:2048 lds\n\t"
                 "s_mov_b32 m0, %0"
                 : "=&s"(saved) : "s"(m0v), "v"(v[0]), "v"(v[1]), "v"(v[2]), "s"(rsrc), "s"(soff) : "memory");
}

// Exchange lanes 16-31 of x with lanes 0-15 of y and lanes 48-63 of x with lanes 32-47 of y.
__device__ __forceinline__ void swap16(uint32_t& x, uint32_t& y) {
  const auto r = __builtin_amdgcn_permlane16_swap(x, y, false, false);
  x = r[0];
  y = r[1];
}

__device__ __forceinline__ void tile_coords(int tl, int mt, int nt, int& tm, int& tn) {
  constexpr int GROUP_M = 8;
  int per_group = GROUP_M * nt;
  int group = tl / per_group;
  int first_m = group * GROUP_M;
  int gm = min(mt - first_m, GROUP_M);
  int in_group = tl - group * per_group;
  tm = first_m + in_group % gm;
  tn = in_group / gm;
}

// LDS swizzle key of tile row r (rows of 128 bytes = 64 bf16 of k): chunk c of row r lives in
// 16-byte slot c ^ f(r). Measured service rule of ds_read_b128 on this chip: the 64 lanes are
// served as four groups of 16, a group being the lanes that agree in lane bit 5 and in the
// parity of lane bits 2..4; a group takes as many cycles as the largest number of its lanes
// that hit one 16-byte bank group ((address / 16) mod 16) at different addresses. With
// f(r) = (r / 2) mod 8 every group of a 16x16x32 or a 32x32x16 fragment read hits 16 distinct
// bank groups, so a wave's read takes the minimum four cycles.
__device__ __forceinline__ int swz(int r) { return (r >> 1) & 7; }

// Instructions of one kind placed after MFMA q when n of them are spread evenly over the first
// `span` MFMAs of a k step.
__host__ __device__ constexpr int spread(int q, int n, int span) {
  return span <= 0 ? (q == 0 ? n : 0) : ((q + 1 < span ? q + 1 : span) * n) / span - ((q < span ? q : span) * n) / span;
}

// Scheduling hints for one k step of NM MFMAs: NV direct-to-LDS loads spread over the first half
// of the MFMAs, ND fragment reads over the first three quarters.
template <int NM, int NV, int ND, int Q = 0>
__device__ __forceinline__ void sched_step() {
  if constexpr (Q < NM) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // one MFMA
    constexpr int v = spread(Q, NV, NM / 2), d = spread(Q, ND, 3 * NM / 4);
    if constexpr (v > 0) __builtin_amdgcn_sched_group_barrier(0x020, v, 0);   // VMEM loads
    if constexpr (d > 0) __builtin_amdgcn_sched_group_barrier(0x100, d, 0);   // LDS reads
    sched_step<NM, NV, ND, Q + 1>();
  }
}

// buffer descriptor of a tile's operand rows, starting at the tile's first row
__device__ __forceinline__ u32x4_t tile_rsrc(const void* p) {
  const uint64_t u = (uint64_t)p;
  return u32x4_t{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)u),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(u >> 32) & 0xffffu)), 0x7fffffffu, 0x00020000u};
}

// Raises a kernel's dynamic-LDS limit once per device and kernel instance (the flags belong to it).
// Two host threads may reach this at once; setting the attribute twice is harmless, and the flags are
// atomics so the check itself is race-free.
inline hipError_t allow_lds(const void* kernel, size_t lds, std::atomic<bool>* attr_set) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) dev = 0;
  if (lds > 65536 && (dev < 0 || dev >= 64 || !attr_set[dev].load(std::memory_order_acquire))) {
    hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    if (dev >= 0 && dev < 64) attr_set[dev].store(true, std::memory_order_release);
  }
  return hipSuccess;
}

// Compute units of the current device (one 256 x 256 workgroup fills a CU: 160 KB of LDS and the
// whole register file), read once per device.
inline int cu_count() {
  static std::atomic<int> cus[64] = {};   // 0 = not read yet; concurrent first reads store the same value
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  int n = cus[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    cus[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

}  // namespace dit
