// Gated norm on gfx950: the boundary between two sublayers of a block,
//   x_out = alpha x + gate u, u = post(y) post_w;   h = pre(x_out) pre_w (1 + scale) + shift,
// and its gradients. Bound by memory: 4 row tensors pass forward, 6 backward (bf16 rows of 3072, with all operands: 20480 rows forward in
// 102 us, 4.9 TB/s; about 10900 rows backward with all vector gradients in 97 us, 4.1 TB/s; a large copy runs at 4.9).
//
// A row is held in registers, 8 elements per lane, so that the two passes of its mean and variance need no second read.
#include <algorithm>

#include "packed.h"

namespace dit {
namespace {

// The 8 successive elements of a row that a lane holds. VEC: D is a multiple of 8 and everything 16-byte aligned. Otherwise a lane
// takes 16 bytes at the alignment of an element, which the memory unit allows; the one at the row's end loads its elements one by one
// (the vectors of a chunk, and rows of up to 256 elements; longer rows: Raw) and stores 4, 2 and 1 of them.
typedef unsigned u32x4_any2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void unpack8(const uint32_t* w, float* f) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8_any(const u16* p, float* f) {
  const u32x4_any2 u = *(const u32x4_any2*)p;
  const uint32_t w[4] = {u[0], u[1], u[2], u[3]};
  unpack8(w, f);
}
__device__ __forceinline__ void load8_any(const float* p, float* f) {
  const f32x4_any4 u = *(const f32x4_any4*)p, v = *(const f32x4_any4*)(p + 4);
#pragma unroll
  for (int i = 0; i < 4; i++) {
    f[i] = u[i];
    f[4 + i] = v[i];
  }
}
__device__ __forceinline__ void store8_any(u16* p, const float* f) {
  *(u32x4_any2*)p = u32x4_any2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
}
__device__ __forceinline__ void store8_any(float* p, const float* f) {
  *(f32x4_any4*)p = f32x4_any4{f[0], f[1], f[2], f[3]};
  *(f32x4_any4*)(p + 4) = f32x4_any4{f[4], f[5], f[6], f[7]};
}
typedef unsigned u32x2_any2 __attribute__((ext_vector_type(2), aligned(2)));
typedef unsigned u32_any2 __attribute__((aligned(2)));
typedef float f32x2_any4 __attribute__((ext_vector_type(2), aligned(4)));
__device__ __forceinline__ void store4_any(u16* p, const float* f) { *(u32x2_any2*)p = u32x2_any2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])}; }
__device__ __forceinline__ void store4_any(float* p, const float* f) { *(f32x4_any4*)p = f32x4_any4{f[0], f[1], f[2], f[3]}; }
__device__ __forceinline__ void store2_any(u16* p, const float* f) { *(u32_any2*)p = pack_bf16x2(f[0], f[1]); }
__device__ __forceinline__ void store2_any(float* p, const float* f) { *(f32x2_any4*)p = f32x2_any4{f[0], f[1]}; }
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, int at, int D, float* f) {
#pragma unroll
  for (int i = 0; i < 8; i++) f[i] = 0.f;
  if (VEC) {
    if (at < D) {
      load4<T>(p + at, f);
      load4<T>(p + at + 4, f + 4);
    }
  } else if (at + 8 <= D) {
    load8_any(p + at, f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (at + i < D) f[i] = to_f32(p[at + i]);
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* p, int at, int D, const float* f) {
  if (VEC) {
    if (at < D) {
      store4<T>(p + at, f);
      store4<T>(p + at + 4, f + 4);
    }
  } else if (at + 8 <= D) {
    store8_any(p + at, f);
  } else if (at < D) {   // 4, 2 and 1 of the elements left
    const int left = D - at;
    float g[4] = {f[0], f[1], f[2], f[3]};
    p += at;
    if (left & 4) {
      store4_any(p, g);
      p += 4;
#pragma unroll
      for (int i = 0; i < 4; i++) g[i] = f[4 + i];
    }
    if (left & 2) {
      store2_any(p, g);
      p += 2;
      g[0] = g[2];
    }
    if (left & 1) *p = from_f32<T>(g[0]);
  }
}
// The same as it was loaded, for rows of more than 8: a row on its way while the one before it is worked on. Without VEC every lane
// loads 16 bytes: the ones at the row's end and past it its last 8 elements, less the first `skip` of them, which are other lanes'
// (20480 bf16 rows of 3068 forward 107 us, 10400 backward 98; the end element by element 142 and 152).
template <bool VEC> __device__ __forceinline__ int skip_of(int at, int D) { return VEC ? 0 : min(max(at + 8 - D, 0), 8); }
// w's elements from `by` on, zeros behind them; PER: elements of a word
template <int WORDS, int PER> __device__ __forceinline__ void skip_first(uint32_t* w, int by) {
#pragma unroll
  for (int step = WORDS; step >= 1; step /= 2)   // words
    if (by & (step * PER))
#pragma unroll
      for (int i = 0; i < WORDS; i++) w[i] = i + step < WORDS ? w[i + step] : 0;
  if (PER == 2 && (by & 1))
#pragma unroll
    for (int i = 0; i < WORDS; i++) w[i] = w[i] >> 16 | (i + 1 < WORDS ? w[i + 1] << 16 : 0);
}
template <typename T, bool VEC> struct Raw {
  static constexpr int PER = 4 / sizeof(T), WORDS = 8 / PER;
  uint32_t w[WORDS];
  __device__ __forceinline__ void load(const T* p, int at, int D) {
    if (VEC && at >= D) {
#pragma unroll
      for (int i = 0; i < WORDS; i++) w[i] = 0;
      return;
    }
    const T* from = p + (VEC ? at : min(at, D - 8));
#pragma unroll
    for (int i = 0; i < WORDS; i += 4) {
      if constexpr (VEC) {
        const uint4 u = *(const uint4*)(from + PER * i);
        w[i] = u.x; w[i + 1] = u.y; w[i + 2] = u.z; w[i + 3] = u.w;
      } else {
        const u32x4_any2 u = *(const u32x4_any2*)(from + PER * i);
        w[i] = u[0]; w[i + 1] = u[1]; w[i + 2] = u[2]; w[i + 3] = u[3];
      }
    }
  }
  __device__ __forceinline__ void get(float* o, int skip) const {
    uint32_t x[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; i++) x[i] = w[i];
    if (!VEC) skip_first<WORDS, PER>(x, skip);
    if constexpr (PER == 2) unpack8(x, o);
    else
#pragma unroll
      for (int i = 0; i < 8; i++) o[i] = __uint_as_float(x[i]);
  }
};

// ky = gate post_w, kh = (1 + scale) pre_w; 0 past the row
template <typename T, bool VEC>
__device__ __forceinline__ void gains(const GatedNormArgs& a, int64_t mo, int at, float* ky, float* kh) {
  // (all loads go out before the first is used)
  float pw[8], rw[8];
#pragma unroll
  for (int i = 0; i < 8; i++) {
    ky[i] = pw[i] = rw[i] = 1.f;
    kh[i] = 0.f;
  }
  if (a.gate) load8<float, VEC>(a.gate + mo, at, a.D, ky);
  if (a.scale) load8<float, VEC>(a.scale + mo, at, a.D, kh);
  if (a.post_w) load8<T, VEC>((const T*)a.post_w, at, a.D, pw);
  if (a.pre_w) load8<T, VEC>((const T*)a.pre_w, at, a.D, rw);
#pragma unroll
  for (int i = 0; i < 8; i++) {
    ky[i] *= pw[i];
    kh[i] = (1.f + kh[i]) * rw[i];
  }
#pragma unroll
  for (int i = 0; i < 8; i++)
    if (at + i >= a.D) ky[i] = kh[i] = 0.f;
}

__device__ __forceinline__ float lanes_sum(float v, int lpr) {
  for (int o = lpr >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// The sequence of a row, or -1. All lanes call it; `row` may differ between them.
__device__ __forceinline__ int sequence_of(const GatedNormArgs& a, int row) {
  if (!a.pr.off) return row / a.pr.len;
  const int lane = threadIdx.x & 63;
  const int first = __builtin_amdgcn_readfirstlane(row);
  int seq = 0;   // sequences that end at or before the first lane's row
  for (int base = 0; base < a.nseq; base += 64) {
    const int end = base + lane < a.nseq ? a.pr.off[base + lane + 1] : 0x7fffffff;
    const int past = __popcll(__ballot(end <= first));
    seq += past;
    if (past < 64) break;
  }
  while (seq < a.nseq && a.pr.off[seq + 1] <= row) seq++;
  if (seq >= a.nseq) return -1;
  const RowSpan r = a.pr.span(seq);
  return row >= r.begin && row < r.begin + r.count ? seq : -1;
}

// the sequence, and its chunk of chunk_rows rows, that this workgroup works on
__device__ __forceinline__ bool find_chunk(const GatedNormArgs& a, int chunk_rows, int& seq, int& chunk, RowSpan& rows) {
  return find_unit(a.nseq, blockIdx.x, [&](int i) { return a.pr.span(i); },
                   [&](const RowSpan& r) { return cdiv(r.count, chunk_rows); }, seq, chunk, rows);
}

struct Norm {
  float mean, r;
};
// of a row of up to 256 elements, held by lpr lanes; at: this lane's first element
__device__ __forceinline__ Norm statistics(int kind, const float* v, const GatedNormArgs& a, int at, int lpr) {
  Norm n{0.f, 1.f};
  if (kind == NORM_NONE) return n;
  if (kind == NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) s += v[i];
    n.mean = lanes_sum(s, lpr) / (float)a.D;
  }
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const float d = at + i < a.D ? v[i] - n.mean : 0.f;
    q = fmaf(d, d, q);
  }
  n.r = rsqrtf(lanes_sum(q, lpr) / (float)a.D + a.eps);
  return n;
}

// Rows of up to 256 elements: 64 / lpr rows per wave, 4 waves.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) forward_narrow(GatedNormArgs a, int lpr) {
  const int lane = threadIdx.x & 63, per = 64 / lpr, l = lane & (lpr - 1);
  const int64_t row64 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * per + lane / lpr;
  const int row = (int)min(row64, (int64_t)a.rows - 1);
  const int seq = sequence_of(a, row);
  if (row64 >= a.rows || seq < 0) return;   // (whole groups of lpr lanes: the sums below stay inside a group)
  const int D = a.D, at = 8 * l;
  const int64_t mo = seq * a.mod_row;
  float v[8], w[8];
  load8<T, VEC>((const T*)a.x + row * a.x_row, at, D, v);
#pragma unroll
  for (int i = 0; i < 8; i++) v[i] *= a.alpha;
  if (a.y) {
    float u[8];
    load8<T, VEC>((const T*)a.y + row * a.y_row, at, D, u);
    const Norm n = statistics(a.post, u, a, at, lpr);
#pragma unroll
    for (int i = 0; i < 8; i++) u[i] = (u[i] - n.mean) * n.r;
    if (a.post_w) {
      load8<T, VEC>((const T*)a.post_w, at, D, w);
#pragma unroll
      for (int i = 0; i < 8; i++) u[i] *= w[i];
    }
    if (a.gate) {
      load8<float, VEC>(a.gate + mo, at, D, w);
#pragma unroll
      for (int i = 0; i < 8; i++) u[i] *= w[i];
    }
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = at + i < D ? v[i] + u[i] : 0.f;
  }
  if (a.x_out) store8<T, VEC>((T*)a.x_out + row * a.x_row, at, D, v);
  if (!a.h) return;
  const Norm n = statistics(a.pre, v, a, at, lpr);
#pragma unroll
  for (int i = 0; i < 8; i++) v[i] = (v[i] - n.mean) * n.r;
  if (a.pre_w) {
    load8<T, VEC>((const T*)a.pre_w, at, D, w);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] *= w[i];
  }
  if (a.scale) {
    load8<float, VEC>(a.scale + mo, at, D, w);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = fmaf(v[i], w[i], v[i]);
  }
  if (a.shift) {
    load8<float, VEC>(a.shift + mo, at, D, w);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] += w[i];
  }
  store8<T, VEC>((T*)a.h + row * a.h_row, at, D, v);
}

// ---------------------------------------------------------------------------
// Longer rows take a workgroup of D / 8 lanes, which walks a chunk of rows of one sequence: gate, scale, shift and weights stay in
// registers (read per row they are half again as many bytes as the rows, from L2), and the next row is on its way while the
// sums of a row pass their barriers.
// ---------------------------------------------------------------------------
constexpr int MAX_WAVES = 16;   // of 8192 / 8 lanes

// v of the lane that a step of a sum over the wave takes it from (0 where there is none): 1, 2, 4, 8 lanes before, which puts the sum of
// a row of 16 lanes into its lane 15, then the rows before. VALU moves, no LDS.
template <int CTRL, int ROWS> __device__ __forceinline__ float moved(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xf, false));
}
template <int STEP> __device__ __forceinline__ float before(float v) {
  if constexpr (STEP < 4) return moved<0x110 + (1 << STEP), 0xf>(v);
  else if constexpr (STEP == 4) return moved<0x142, 0xa>(v);
  else return moved<0x143, 0xc>(v);
}
__device__ __forceinline__ float lane_of(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
// sum over the wave, and over its first 16 lanes, in every lane
__device__ __forceinline__ float row_sum(float v) {
  v += before<0>(v);
  v += before<1>(v);
  v += before<2>(v);
  v += before<3>(v);
  return v;
}
__device__ __forceinline__ float wave_total(float v) {
  v = row_sum(v);
  v += before<4>(v);
  v += before<5>(v);
  return lane_of(v, 63);
}
__device__ __forceinline__ float first_row_total(float v) { return lane_of(row_sum(v), 15); }

// What is known of a set of row elements v with weights g: sum v, sum (v - m)^2 and sum g (v - m) about the set's own mean m (rms: 0),
// sum g. Sets are joined by the formulas for the sums about another point, which lose nothing where the mean is large.
struct Moments {
  float s, q, sg, c;
};
// one step of the sum over a wave: a lane's set of n elements and another of as many
template <int STEP, bool WITH_G> __device__ __forceinline__ void join_equal(bool layer, Moments& m, float half_inverse) {
  const float s = before<STEP>(m.s), sg = WITH_G ? before<STEP>(m.sg) : 0.f;
  m.q += before<STEP>(m.q);
  if (WITH_G) m.c += before<STEP>(m.c);
  if (layer) {   // half_inverse = 1 / (2 n)
    const float d = m.s - s;
    m.q = fmaf(d * d, half_inverse, m.q);
    if (WITH_G) m.c = fmaf(d * (m.sg - sg), half_inverse, m.c);
    m.s += s;
  }
  if (WITH_G) m.sg += sg;
}
template <bool WITH_G>
__device__ __forceinline__ Moments wave_moments(int kind, const float* v, const float* g, const bool* in, float count) {
  Moments m{0.f, 0.f, 0.f, 0.f};
  const bool layer = kind == NORM_LAYER;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    if (layer) m.s += v[i];
    if (WITH_G) m.sg += g[i];
  }
  if (count == 512.f) {
    const float mean = m.s * 0.125f;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float d = v[i] - mean;
      m.q = fmaf(d, d, m.q);
      if (WITH_G) m.c = fmaf(g[i], d, m.c);
    }
    join_equal<0, WITH_G>(layer, m, 1.f / 16);
    join_equal<1, WITH_G>(layer, m, 1.f / 32);
    join_equal<2, WITH_G>(layer, m, 1.f / 64);
    join_equal<3, WITH_G>(layer, m, 1.f / 128);
    join_equal<4, WITH_G>(layer, m, 1.f / 256);
    join_equal<5, WITH_G>(layer, m, 1.f / 512);
    return m;   // (lane 63 has the wave's)
  }
  // a wave at the end of the row: its mean first
  if (WITH_G) m.sg = wave_total(m.sg);
  float mean = 0.f;
  if (layer) {
    m.s = wave_total(m.s);
    mean = count > 0.f ? m.s / count : 0.f;
  }
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const float d = in[i] ? v[i] - mean : 0.f;
    m.q = fmaf(d, d, m.q);
    if (WITH_G) m.c = fmaf(g[i], d, m.c);
  }
  m.q = wave_total(m.q);
  if (WITH_G) m.c = wave_total(m.c);
  return m;
}
// mean, 1 / deviation, sum g, sum g (v - mean) r of a row from its waves' moments (m: [MAX_WAVES], zeros past the last), each of `count`
// elements; lane w looks at wave w's
struct RowStats {
  float mean, r, sg, c;
};
template <bool WITH_G>
__device__ __forceinline__ RowStats join_moments(int kind, const float4* m, float count, float inv_d, float eps) {
  const float4 x = m[threadIdx.x & 15];
  RowStats o{0.f, 1.f, 0.f, 0.f};
  float off = 0.f;
  if (kind == NORM_LAYER) {
    o.mean = first_row_total(x.x) * inv_d;
    off = count > 0.f ? x.x / count - o.mean : 0.f;
  }
  if (kind != NORM_NONE) o.r = rsqrtf(first_row_total(fmaf(count * off, off, x.y)) * inv_d + eps);
  if (WITH_G) {
    o.sg = first_row_total(x.z);
    o.c = first_row_total(fmaf(x.z, off, x.w)) * o.r;
  }
  return o;
}
// elements of the row in wave w = lane % 16
__device__ __forceinline__ float wave_count(int D) { return (float)min(max(D - 512 * (int)(threadIdx.x & 15), 0), 512); }

// A barrier for what the waves exchange through LDS. __syncthreads() would also wait for the loads of the next row and the stores of
// the last one, which no other wave looks at (8 x about 1300 rows of 3072, backward: 97 us, with __syncthreads() 99; forward the same).
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <typename T, bool VEC>
__global__ void __launch_bounds__(1024) forward_wide(GatedNormArgs a, int chunk_rows) {
  __shared__ float4 red[2][MAX_WAVES];
  int seq, chunk;
  RowSpan rows;
  if (!find_chunk(a, chunk_rows, seq, chunk, rows)) return;
  // every chunks-th row: the workgroups that run together then work on neighbouring rows
  const int begin = rows.begin + chunk, end = rows.begin + rows.count, step = cdiv(rows.count, chunk_rows);
  const int D = a.D, l = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), at = 8 * l, skip = skip_of<VEC>(at, D);
  const int64_t mo = seq * a.mod_row;
  const bool has_y = a.y, has_xo = a.x_out, has_h = a.h;
  Raw<T, VEC> nx, ny;
  auto fetch = [&](int64_t row) {
    nx.load((const T*)a.x + row * a.x_row, at, D);
    if (has_y) ny.load((const T*)a.y + row * a.y_row, at, D);
  };
  fetch(begin);
  bool in[8];
#pragma unroll
  for (int i = 0; i < 8; i++) in[i] = at + i < D;
  if (l < 2 * MAX_WAVES) red[l >> 4][l & 15] = make_float4(0.f, 0.f, 0.f, 0.f);
  __syncthreads();
  const float counts = wave_count(D), count = lane_of(counts, wave), inv_d = 1.f / (float)D;
  float ky[8], kh[8], sh[8];   // gate post_w; (1 + scale) pre_w; shift
  gains<T, VEC>(a, mo, at, ky, kh);
#pragma unroll
  for (int i = 0; i < 8; i++) sh[i] = 0.f;
  if (a.shift && has_h) load8<float, VEC>(a.shift + mo, at, D, sh);
  int turn = 0;   // (a buffer is written again two barriers after it was)
  auto stats = [&](int kind, const float* v) {
    const Moments m = wave_moments<false>(kind, v, nullptr, in, count);
    if ((l & 63) == 63) red[turn][wave] = make_float4(m.s, m.q, 0.f, 0.f);
    lds_barrier();
    const RowStats n = join_moments<false>(kind, red[turn], counts, inv_d, a.eps);
    turn ^= 1;
    return n;
  };
  for (int64_t row = begin; row < end; row += step) {
    float v[8], u[8];
    nx.get(v, skip);
    if (has_y) ny.get(u, skip);
    fetch(row + step < end ? row + step : row);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] *= a.alpha;
    if (has_y) {
      if (a.post != NORM_NONE) {
        const RowStats n = stats(a.post, u);
#pragma unroll
        for (int i = 0; i < 8; i++) u[i] = (u[i] - n.mean) * n.r;
      }
#pragma unroll
      for (int i = 0; i < 8; i++) v[i] = fmaf(u[i], ky[i], v[i]);   // (past the row ky is 0)
    }
    if (has_xo) store8<T, VEC>((T*)a.x_out + row * a.x_row, at, D, v);
    if (!has_h) continue;
    RowStats n{0.f, 1.f, 0.f, 0.f};
    if (a.pre != NORM_NONE) n = stats(a.pre, v);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = fmaf((v[i] - n.mean) * n.r, kh[i], sh[i]);
    store8<T, VEC>((T*)a.h + row * a.h_row, at, D, v);
  }
}

// ---------------------------------------------------------------------------
// Backward. A workgroup takes a chunk of rows of one sequence and adds its column sums up in registers: a lane holds the
// same 8 columns of every row. With xh = pre(x_out), yh = post(y) the normalised rows and t = dx_out + pre'(dh (1 + scale) pre_w),
//   dx = alpha t,  dy = post'(gate post_w t),  norm'(g) = r (g - [mean g] - xh mean(g xh));
// the sums over the rows are R = sum dh, P = sum dh xh, Q = sum t yh, from which every vector's gradient follows
// (columns_kernel). R, P and Q of a chunk go to the workspace.
// ---------------------------------------------------------------------------
// What both kernels do with a row once its statistics are known. t: dx_out, becomes its total; xv, yv: become the normalised rows.
struct RowGradient {
  float mean, r, mg, mgx;   // of x_out: mean, 1 / deviation, mean g, mean g xh (0 where the norm has none)
};
__device__ __forceinline__ RowGradient row_gradient(int kind, const RowStats& n, float inv_d) {
  return RowGradient{n.mean, n.r, kind == NORM_LAYER ? n.sg * inv_d : 0.f, kind != NORM_NONE ? n.c * inv_d : 0.f};
}
struct Columns {
  float R[8], P[8], Q[8];   // sums of dh, dh xh, t yh over the chunk's rows
};
// g = dh kh; t += pre'(g), and the columns' shares
__device__ __forceinline__ void add_pre(const RowGradient& n, float* xv, const float* dh, const float* kh, float* t, bool live, Columns& s) {
#pragma unroll
  for (int i = 0; i < 8; i++) {
    xv[i] = (xv[i] - n.mean) * n.r;   // (past the row dh and the gains are 0, and t is not kept)
    t[i] += n.r * (dh[i] * kh[i] - n.mg - xv[i] * n.mgx);
    if (live) {
      s.R[i] += dh[i];
      s.P[i] = fmaf(dh[i], xv[i], s.P[i]);
    }
  }
}

template <bool VEC>
__device__ __forceinline__ void store_columns(const GatedNormArgs& a, int at, const Columns& s) {
  float* out = a.parts + (int64_t)blockIdx.x * 3 * a.D;
  store8<float, VEC>(out, at, a.D, s.R);
  store8<float, VEC>(out + a.D, at, a.D, s.P);
  store8<float, VEC>(out + 2 * a.D, at, a.D, s.Q);
}
template <typename T, bool VEC>
__device__ __forceinline__ void load_rows(const GatedNormArgs& a, int64_t row, int at, float* xv, float* yv, float* t, float* dh) {
#pragma unroll
  for (int i = 0; i < 8; i++) yv[i] = t[i] = dh[i] = 0.f;
  load8<T, VEC>((const T*)a.x + row * a.x_row, at, a.D, xv);
  if (a.y) load8<T, VEC>((const T*)a.y + row * a.y_row, at, a.D, yv);
  if (a.dx_out) load8<T, VEC>((const T*)a.dx_out + row * a.x_row, at, a.D, t);
  if (a.dh) load8<T, VEC>((const T*)a.dh + row * a.h_row, at, a.D, dh);
}

// Rows of up to 256 elements: groups of lpr lanes take a row each.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) rows_narrow(GatedNormArgs a, int lpr, int chunk_rows) {
  __shared__ float cols[256 * 25];   // (25: an odd stride keeps lanes on different banks)
  int seq, chunk;
  RowSpan rows;
  if (!find_chunk(a, chunk_rows, seq, chunk, rows)) return;
  const int begin = rows.begin + chunk * chunk_rows, end = min(begin + chunk_rows, rows.begin + rows.count);
  const int D = a.D, groups = 256 / lpr, l = threadIdx.x & (lpr - 1), grp = threadIdx.x / lpr, at = 8 * l;
  float ky[8], kh[8];
  gains<T, VEC>(a, seq * a.mod_row, at, ky, kh);
  bool in[8];
  Columns cs;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    in[i] = at + i < D;
    cs.R[i] = cs.P[i] = cs.Q[i] = 0.f;
  }
  const float inv_d = 1.f / (float)D;
  // (a turn without a row works on the chunk's last one and keeps nothing: every lane takes part in the sums)
  for (int r0 = begin; r0 < end; r0 += groups) {
    const bool live = r0 + grp < end;
    const int64_t row = min(r0 + grp, end - 1);
    float xv[8], yv[8], t[8], dh[8];
    load_rows<T, VEC>(a, row, at, xv, yv, t, dh);
    if (a.dh) {
      const Norm n = statistics(a.pre, xv, a, at, lpr);
      RowStats st{n.mean, n.r, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float g = dh[i] * kh[i];
        st.sg += g;
        st.c = fmaf(g, (xv[i] - n.mean) * n.r, st.c);
      }
      st.sg = lanes_sum(st.sg, lpr);
      st.c = lanes_sum(st.c, lpr);
      add_pre(row_gradient(a.pre, st, inv_d), xv, dh, kh, t, live, cs);
    }
    if (a.y) {
      const Norm n = statistics(a.post, yv, a, at, lpr);
      float g[8], u = 0.f, w = 0.f;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        yv[i] = in[i] ? (yv[i] - n.mean) * n.r : 0.f;
        if (live) cs.Q[i] = fmaf(t[i], yv[i], cs.Q[i]);
        g[i] = in[i] ? t[i] * ky[i] : 0.f;
        u += g[i];
        w = fmaf(g[i], yv[i], w);
      }
      if (a.dy) {
        u = a.post == NORM_LAYER ? lanes_sum(u, lpr) * inv_d : 0.f;
        w = a.post != NORM_NONE ? lanes_sum(w, lpr) * inv_d : 0.f;
#pragma unroll
        for (int i = 0; i < 8; i++) g[i] = n.r * (g[i] - u - yv[i] * w);
        if (live) store8<T, VEC>((T*)a.dy + row * a.y_row, at, D, g);
      }
    }
    if (a.dx && live) {
#pragma unroll
      for (int i = 0; i < 8; i++) t[i] *= a.alpha;
      store8<T, VEC>((T*)a.dx + row * a.x_row, at, D, t);
    }
  }
  if (!a.parts) return;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    cols[threadIdx.x * 25 + i] = cs.R[i];
    cols[threadIdx.x * 25 + 8 + i] = cs.P[i];
    cols[threadIdx.x * 25 + 16 + i] = cs.Q[i];
  }
  __syncthreads();
  if (grp > 0) return;
  for (int g = 1; g < groups; g++)   // the groups in order
#pragma unroll
    for (int i = 0; i < 8; i++) {
      cs.R[i] += cols[(g * lpr + l) * 25 + i];
      cs.P[i] += cols[(g * lpr + l) * 25 + 8 + i];
      cs.Q[i] += cols[(g * lpr + l) * 25 + 16 + i];
    }
  store_columns<VEC>(a, at, cs);
}

// FULL: every row tensor is there. The number of loads and stores of a row is then known to the compiler, which waits for the next
// row's loads without waiting for the last row's stores (8 x about 1300 rows of 3072: 101 us without, 97 with; forward the same).
template <typename T, bool VEC, bool FULL>
__global__ void __launch_bounds__(1024) rows_wide(GatedNormArgs a, int chunk_rows) {
  __shared__ float4 redx[2][MAX_WAVES], redy[2][MAX_WAVES];
  __shared__ float2 redg[2][MAX_WAVES];
  int seq, chunk;
  RowSpan rows;
  if (!find_chunk(a, chunk_rows, seq, chunk, rows)) return;
  // every chunks-th row: the workgroups that run together then work on neighbouring rows
  const int begin = rows.begin + chunk, end = rows.begin + rows.count, step = cdiv(rows.count, chunk_rows);
  const int D = a.D, l = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), at = 8 * l, skip = skip_of<VEC>(at, D);
  const bool has_y = FULL || a.y, has_dxo = FULL || a.dx_out, has_dh = FULL || a.dh, has_dx = FULL || a.dx, has_dy = FULL || a.dy;
  Raw<T, VEC> nx, ny, nt, nh;
  auto fetch = [&](int64_t row) {
    nx.load((const T*)a.x + row * a.x_row, at, D);
    if (has_y) ny.load((const T*)a.y + row * a.y_row, at, D);
    if (has_dxo) nt.load((const T*)a.dx_out + row * a.x_row, at, D);
    if (has_dh) nh.load((const T*)a.dh + row * a.h_row, at, D);
  };
  fetch(begin);
  float ky[8], kh[8];
  gains<T, VEC>(a, seq * a.mod_row, at, ky, kh);
  bool in[8];
  Columns cs;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    in[i] = at + i < D;
    cs.R[i] = cs.P[i] = cs.Q[i] = 0.f;
  }
  if (l < 2 * MAX_WAVES) {
    redx[l >> 4][l & 15] = redy[l >> 4][l & 15] = make_float4(0.f, 0.f, 0.f, 0.f);
    redg[l >> 4][l & 15] = make_float2(0.f, 0.f);
  }
  __syncthreads();
  const float counts = wave_count(D), count = lane_of(counts, wave), inv_d = 1.f / (float)D;
  int turn = 0;   // (a buffer is written again two barriers after it was)
  for (int64_t row = begin; row < end; row += step, turn ^= 1) {
    float xv[8], yv[8], t[8], dh[8];
#pragma unroll
    for (int i = 0; i < 8; i++) yv[i] = t[i] = dh[i] = 0.f;
    nx.get(xv, skip);
    if (has_y) ny.get(yv, skip);
    if (has_dxo) nt.get(t, skip);
    if (has_dh) nh.get(dh, skip);
    fetch(row + step < end ? row + step : row);
    if (has_dh) {
      float g[8];
#pragma unroll
      for (int i = 0; i < 8; i++) g[i] = dh[i] * kh[i];
      const Moments m = wave_moments<true>(a.pre, xv, g, in, count);
      if ((l & 63) == 63) redx[turn][wave] = make_float4(m.s, m.q, m.sg, m.c);
    }
    if (has_y && a.post != NORM_NONE) {
      const Moments m = wave_moments<false>(a.post, yv, nullptr, in, count);
      if ((l & 63) == 63) redy[turn][wave] = make_float4(m.s, m.q, 0.f, 0.f);
    }
    lds_barrier();
    if (has_dh) add_pre(row_gradient(a.pre, join_moments<true>(a.pre, redx[turn], counts, inv_d, a.eps), inv_d), xv, dh, kh, t, true, cs);
    if (has_dx) {
      float o[8];
#pragma unroll
      for (int i = 0; i < 8; i++) o[i] = t[i] * a.alpha;
      store8<T, VEC>((T*)a.dx + row * a.x_row, at, D, o);
    }
    if (!has_y) continue;
    RowStats n{0.f, 1.f, 0.f, 0.f};
    if (a.post != NORM_NONE) n = join_moments<false>(a.post, redy[turn], counts, inv_d, a.eps);
#pragma unroll
    for (int i = 0; i < 8; i++) {
      yv[i] = (yv[i] - n.mean) * n.r;
      cs.Q[i] = fmaf(t[i], yv[i], cs.Q[i]);
      t[i] *= ky[i];   // (past the row ky is 0)
    }
    if (!has_dy) continue;
    float u = 0.f, w = 0.f;
    if (a.post != NORM_NONE) {
#pragma unroll
      for (int i = 0; i < 8; i++) {
        u += t[i];
        w = fmaf(t[i], yv[i], w);
      }
      u = wave_total(u);
      w = wave_total(w);
      if ((l & 63) == 63) redg[turn][wave] = make_float2(u, w);
      lds_barrier();
      const float2 x = redg[turn][threadIdx.x & 15];
      u = a.post == NORM_LAYER ? first_row_total(x.x) * inv_d : 0.f;
      w = first_row_total(x.y) * inv_d;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) t[i] = n.r * (t[i] - u - yv[i] * w);
    store8<T, VEC>((T*)a.dy + row * a.y_row, at, D, t);
  }
  if (a.parts) store_columns<VEC>(a, at, cs);
}

// Sums of the chunks of one sequence, 64 columns per workgroup, whose WAVES waves share the chunks:
//   dshift = R, dscale = P pre_w, dgate = Q post_w.
// P and Q stay behind for the weights' gradients (in the sequence's place after the chunks).
template <typename T, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) columns_kernel(GatedNormArgs a, int chunk_rows) {
  __shared__ float red[3][WAVES][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = a.D;
  const int blocks = cdiv(D, 64), seq = blockIdx.x / blocks, col = (blockIdx.x - seq * blocks) * 64 + lane;
  int64_t before = 0;
  for (int i = lane; i < seq; i += 64) before += cdiv(a.pr.span(i).count, chunk_rows);
  for (int o = 32; o > 0; o >>= 1) before += __shfl_xor(before, o, 64);
  // (offsets that are not increasing can promise more chunks than there are)
  const int n = (int)min((int64_t)cdiv(a.pr.span(seq).count, chunk_rows), a.chunks - before);
  float s[3] = {0.f, 0.f, 0.f};
  if (col < D)
#pragma unroll 4   // (loads of several chunks in flight)
    for (int c = wave; c < n; c += WAVES) {
      const float* p = a.parts + (before + c) * 3 * D + col;
#pragma unroll
      for (int k = 0; k < 3; k++) s[k] += p[(int64_t)k * D];
    }
#pragma unroll
  for (int k = 0; k < 3; k++) red[k][wave][lane] = s[k];
  __syncthreads();
  if (wave > 0 || col >= D) return;
  for (int w = 1; w < WAVES; w++)
#pragma unroll
    for (int k = 0; k < 3; k++) s[k] += red[k][w][lane];
  const int64_t at = seq * a.mod_row + col;
  if (a.dshift) a.dshift[at] = s[0];
  if (a.dscale) a.dscale[at] = a.pre_w ? s[1] * to_f32(((const T*)a.pre_w)[col]) : s[1];
  if (a.dgate) a.dgate[at] = a.post_w ? s[2] * to_f32(((const T*)a.post_w)[col]) : s[2];
  if (a.dpre_w || a.dpost_w) {
    float* keep = a.parts + ((int64_t)a.chunks * 3 + 2 * seq) * D + col;
    keep[0] = s[1];
    keep[D] = s[2];
  }
}

// dpre_w = sum over the sequences of (1 + scale) P, dpost_w of gate Q: 64 columns per workgroup, its 16 waves share the sequences.
__global__ void __launch_bounds__(1024) weights_kernel(GatedNormArgs a) {
  constexpr int WAVES = 16;
  __shared__ float red[2][WAVES][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane, D = a.D;
  float p = 0.f, q = 0.f;
  if (col < D)
#pragma unroll 4
    for (int s = wave; s < a.nseq; s += WAVES) {
      const float* k = a.parts + ((int64_t)a.chunks * 3 + 2 * s) * D + col;
      const int64_t at = s * a.mod_row + col;
      p = fmaf(a.scale ? 1.f + a.scale[at] : 1.f, k[0], p);
      q = fmaf(a.gate ? a.gate[at] : 1.f, k[D], q);
    }
  red[0][wave][lane] = p;
  red[1][wave][lane] = q;
  __syncthreads();
  if (wave > 0 || col >= D) return;
  for (int w = 1; w < WAVES; w++) {
    p += red[0][w][lane];
    q += red[1][w][lane];
  }
  if (a.dpre_w) a.dpre_w[col] = p;
  if (a.dpost_w) a.dpost_w[col] = q;
}

bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool vectors(const GatedNormArgs& a) {
  const void* all[] = {a.x, a.y, a.post_w, a.pre_w, a.gate, a.scale, a.shift, a.x_out, a.h, a.dx_out, a.dh, a.dx, a.dy};
  for (const void* p : all)
    if (!aligned(p)) return false;
  return a.D % 8 == 0 && a.x_row % 8 == 0 && a.y_row % 8 == 0 && a.h_row % 8 == 0 && a.mod_row % 8 == 0;
}
// lanes of a row of up to 256 elements
int lanes_of(int D) {
  int l = 8;
  while (l * 8 < D) l *= 2;
  return l;
}

// Rows of up to 256 elements share a wave; longer ones take the waves of a workgroup (20000 rows of 512: forward 19.5 us, backward 43;
// as one row per wave of the narrow kernels 23 and 62. Of 256: 14 and 43 either way).
bool narrow(int D) { return D <= 256; }
int wide_threads(int D) { return cdiv(cdiv(D, 8), 64) * 64; }

// Rows of a chunk of the backward pass: as many as let all chunks run at once (16 waves per CU, which their registers allow). Half as
// many rows need another round of workgroups for what the first leaves over and write twice the sums (8 sequences of about 1300
// rows of 3072: 120 us where all at once take 97). At least, for long rows, what costs less than the sums of more chunks (a row costs
// its chunk 2 us; gradients in all, us with 8 / 4 / 2 / 1 at least): 64 rows of 1024 22 / 16 / 13 / 12, 512 of 3072 28 / 23 / 22 / 22;
// 616 of 3072 29 / 23 / 26 / 25, 4000 of 1024 32 / 27 / 33 / 32, 3000 of 512 in one sequence 27 / 25 / 33 / 50. Short rows: 8, which
// the waves of a workgroup take at once.
int chunk_rows_of(int nseq, int rows, int D) {
  const int waves = narrow(D) ? 4 : wide_threads(D) / 64, slots = 256 * std::max(16 / waves, 1);
  return std::max(narrow(D) ? 8 : rows <= 512 ? 2 : 4, cdiv(rows, std::max(slots - nseq, slots / 2)));
}

// rows a workgroup walks forward: up to 8 (20480 rows of 3072: 103 us; 20, one round of workgroups: 109), as long as that leaves enough
// workgroups for the 32 waves a CU can hold
int forward_rows_of(int rows, int D) { return std::min(8, std::max(1, rows / (256 * 32 / (wide_threads(D) / 64)))); }

// Threads of a launch.
struct Launch {
  int64_t groups;
  int threads;
  int64_t total() const { return groups * threads; }
};
Launch forward_of(const GatedNormArgs& a) {
  if (narrow(a.D)) return {cdiv(a.rows, 4 * (64 / lanes_of(a.D))), 256};
  return {(int64_t)a.rows / forward_rows_of(a.rows, a.D) + a.nseq, wide_threads(a.D)};
}
Launch rows_of(const GatedNormArgs& a) { return {a.chunks, narrow(a.D) ? 256 : wide_threads(a.D)}; }
Launch columns_of(const GatedNormArgs& a) {
  return {(int64_t)cdiv(a.D, 64) * a.nseq, a.chunks <= 8 * (int64_t)a.nseq ? 256 : 1024};   // few chunks per sequence: 4 waves
}

template <typename T>
void forward_launch(const GatedNormArgs& a, hipStream_t s) {
  const bool vec = vectors(a);
  const Launch l = forward_of(a);
  const int grid = (int)l.groups;
  if (narrow(a.D)) {
    const int lpr = lanes_of(a.D);
    if (vec) forward_narrow<T, true><<<grid, 256, 0, s>>>(a, lpr);
    else forward_narrow<T, false><<<grid, 256, 0, s>>>(a, lpr);
  } else {
    const int cr = forward_rows_of(a.rows, a.D);
    if (vec) forward_wide<T, true><<<grid, l.threads, 0, s>>>(a, cr);
    else forward_wide<T, false><<<grid, l.threads, 0, s>>>(a, cr);
  }
}

template <typename T>
void rows_launch(const GatedNormArgs& a, hipStream_t s) {
  const int cr = chunk_rows_of(a.nseq, a.rows, a.D);
  const bool vec = vectors(a);
  if (narrow(a.D)) {
    const int lpr = lanes_of(a.D);
    if (vec) rows_narrow<T, true><<<a.chunks, 256, 0, s>>>(a, lpr, cr);
    else rows_narrow<T, false><<<a.chunks, 256, 0, s>>>(a, lpr, cr);
  } else {
    const int threads = rows_of(a).threads;
    if (vec && a.y && a.dx_out && a.dh && a.dx && a.dy) rows_wide<T, true, true><<<a.chunks, threads, 0, s>>>(a, cr);
    else if (vec) rows_wide<T, true, false><<<a.chunks, threads, 0, s>>>(a, cr);
    else rows_wide<T, false, false><<<a.chunks, threads, 0, s>>>(a, cr);
  }
}

}  // namespace

int64_t gated_norm_forward_threads(const GatedNormArgs& a) { return forward_of(a).total(); }
int64_t gated_norm_backward_threads(const GatedNormArgs& a) {
  return std::max(a.rows > 0 ? rows_of(a).total() : 0, a.parts ? columns_of(a).total() : 0);
}

hipError_t gated_norm_fwd(const GatedNormArgs& a, int dtype, hipStream_t s) {
  if (dtype == DT_BF16) forward_launch<u16>(a, s);
  else forward_launch<float>(a, s);
  return hipGetLastError();
}

int gated_norm_chunks(int nseq, int rows, int D) { return rows / chunk_rows_of(nseq, rows, D) + nseq; }
size_t gated_norm_ws(int nseq, int rows, int D) {
  return ((size_t)gated_norm_chunks(nseq, rows, D) * 3 + 2 * (size_t)nseq) * D * 4;
}

hipError_t gated_norm_rows_bwd(const GatedNormArgs& a, int dtype, hipStream_t s) {
  if (dtype == DT_BF16) rows_launch<u16>(a, s);
  else rows_launch<float>(a, s);
  return hipGetLastError();
}

template <typename T>
static void columns_launch(const GatedNormArgs& a, int cr, hipStream_t s) {
  const Launch l = columns_of(a);
  if (l.threads == 256) columns_kernel<T, 4><<<l.groups, 256, 0, s>>>(a, cr);
  else columns_kernel<T, 16><<<l.groups, 1024, 0, s>>>(a, cr);
}
hipError_t gated_norm_columns_bwd(const GatedNormArgs& a, int dtype, hipStream_t s) {
  const int cr = chunk_rows_of(a.nseq, a.rows, a.D);
  if (a.nseq > 0) {
    if (dtype == DT_BF16) columns_launch<u16>(a, cr, s);
    else columns_launch<float>(a, cr, s);
  }
  if (a.dpre_w || a.dpost_w) weights_kernel<<<cdiv(a.D, 64), 1024, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace dit
