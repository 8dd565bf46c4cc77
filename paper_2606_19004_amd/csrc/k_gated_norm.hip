// Gated norm on gfx950: the boundary between two sublayers of a block,
//   x_out = alpha x + gate u, u = post(y) post_w;   h = pre(x_out) pre_w (1 + scale) + shift,
// and its gradients. Bound by memory: 4 row tensors pass forward, 6 backward.
//
// Forward: a row is held by 64 lanes (fewer where it is short), 8 elements per lane and chunk, so that the two-pass mean
// and variance need no second read. Backward: see rows_kernel.
#include <algorithm>

#include "packed.h"

namespace dit {
namespace {

// Elements of a row that a lane holds: 8 successive ones per chunk (VEC: D a multiple of 8, everything 16-byte
// aligned) or 8 that are LPR apart.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, int at, int step, int D, float* f) {
  if (VEC) {
    if (at < D) {
      load4<T>(p + at, f);
      load4<T>(p + at + 4, f + 4);
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++) f[i] = 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) f[i] = at + i * step < D ? to_f32(p[at + i * step]) : 0.f;
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* p, int at, int step, int D, const float* f) {
  if (VEC) {
    if (at < D) {
      store4<T>(p + at, f);
      store4<T>(p + at + 4, f + 4);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (at + i * step < D) p[at + i * step] = from_f32<T>(f[i]);
  }
}
// place of a lane's first element of chunk c, of the LPR lanes of a row
template <bool VEC>
__device__ __forceinline__ int place(int c, int l, int lpr) { return VEC ? (c * lpr + l) * 8 : c * lpr * 8 + l; }

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
  const int b = a.pr.begin(seq);
  return row >= b && row < b + a.pr.count(seq) ? seq : -1;
}

struct Norm {
  float mean, r;
};
template <int CH>
__device__ __forceinline__ Norm statistics(int kind, const float (*v)[8], const GatedNormArgs& a, int l, int lpr, bool vec) {
  Norm n{0.f, 1.f};
  if (kind == NORM_NONE) return n;
  if (kind == NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < CH; c++)
#pragma unroll
      for (int i = 0; i < 8; i++) s += v[c][i];
    n.mean = lanes_sum(s, lpr) / (float)a.D;
  }
  float q = 0.f;
#pragma unroll
  for (int c = 0; c < CH; c++)
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const int at = vec ? (c * lpr + l) * 8 + i : c * lpr * 8 + l + i * lpr;
      const float d = at < a.D ? v[c][i] - n.mean : 0.f;
      q = fmaf(d, d, q);
    }
  n.r = rsqrtf(lanes_sum(q, lpr) / (float)a.D + a.eps);
  return n;
}

template <typename T, int CH, bool VEC>
__global__ void __launch_bounds__(256) forward_kernel(GatedNormArgs a, int lpr) {
  const int lane = threadIdx.x & 63, per = 64 / lpr, l = lane & (lpr - 1);
  const int64_t row64 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * per + lane / lpr;
  const int row = (int)min(row64, (int64_t)a.rows - 1);
  const int seq = sequence_of(a, row);
  const bool real = row64 < a.rows && seq >= 0;
  if (!real) return;   // (whole groups of lpr lanes: the sums below stay inside a group)
  const int D = a.D;
  const T* x = (const T*)a.x + row * a.x_row;
  const int64_t mo = seq * a.mod_row;
  float v[CH][8];
  if (a.y) {
    const T* y = (const T*)a.y + row * a.y_row;
#pragma unroll
    for (int c = 0; c < CH; c++) load8<T, VEC>(y, place<VEC>(c, l, lpr), lpr, D, v[c]);
    const Norm n = statistics<CH>(a.post, v, a, l, lpr, VEC);
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const int at = place<VEC>(c, l, lpr);
      float xv[8], w[8], g[8];
      load8<T, VEC>(x, at, lpr, D, xv);
      if (a.post_w) load8<T, VEC>((const T*)a.post_w, at, lpr, D, w);
      if (a.gate) load8<float, VEC>(a.gate + mo, at, lpr, D, g);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        float u = (v[c][i] - n.mean) * n.r;
        if (a.post_w) u *= w[i];
        if (a.gate) u *= g[i];
        v[c][i] = fmaf(a.alpha, xv[i], u);
      }
    }
  } else {
#pragma unroll
    for (int c = 0; c < CH; c++) {
      load8<T, VEC>(x, place<VEC>(c, l, lpr), lpr, D, v[c]);
#pragma unroll
      for (int i = 0; i < 8; i++) v[c][i] *= a.alpha;
    }
  }
  if (!VEC) {   // lanes past the row hold what the mean of y left there
#pragma unroll
    for (int c = 0; c < CH; c++)
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (place<VEC>(c, l, lpr) + i * lpr >= D) v[c][i] = 0.f;
  } else {
#pragma unroll
    for (int c = 0; c < CH; c++)
      if (place<VEC>(c, l, lpr) >= D)
#pragma unroll
        for (int i = 0; i < 8; i++) v[c][i] = 0.f;
  }
  if (a.x_out) {
    T* xo = (T*)a.x_out + row * a.x_row;
#pragma unroll
    for (int c = 0; c < CH; c++) store8<T, VEC>(xo, place<VEC>(c, l, lpr), lpr, D, v[c]);
  }
  if (!a.h) return;
  const Norm n = statistics<CH>(a.pre, v, a, l, lpr, VEC);
  T* h = (T*)a.h + row * a.h_row;
#pragma unroll
  for (int c = 0; c < CH; c++) {
    const int at = place<VEC>(c, l, lpr);
    float w[8], sc[8], sh[8], o[8];
    if (a.pre_w) load8<T, VEC>((const T*)a.pre_w, at, lpr, D, w);
    if (a.scale) load8<float, VEC>(a.scale + mo, at, lpr, D, sc);
    if (a.shift) load8<float, VEC>(a.shift + mo, at, lpr, D, sh);
#pragma unroll
    for (int i = 0; i < 8; i++) {
      o[i] = (v[c][i] - n.mean) * n.r;
      if (a.pre_w) o[i] *= w[i];
      if (a.scale) o[i] *= 1.f + sc[i];
      if (a.shift) o[i] += sh[i];
    }
    store8<T, VEC>(h, at, lpr, D, o);
  }
}

// ---------------------------------------------------------------------------
// Backward. A workgroup takes a chunk of rows of one sequence, so that its gate and scale are read once, and adds
// the column sums of the chunk up in registers: a lane holds the same 8 columns of every row. Rows of up to 512
// elements share a wave (lpr lanes each); longer ones take the whole workgroup, D / 8 lanes. With xh = pre(x_out), yh = post(y) the
// normalised rows and t = dx_out + pre'(dh (1 + scale) pre_w),
//   dx = alpha t,  dy = post'(gate post_w t),  norm'(g) = r (g - [mean g] - xh mean(g xh));
// the sums over the rows are R = sum dh, P = sum dh xh, Q = sum t yh, from which every vector's gradient follows
// (columns_kernel). R, P and Q of a chunk go to the workspace.
// ---------------------------------------------------------------------------
// Sums of two values over the lanes of a row.
template <bool WIDE>
__device__ __forceinline__ void row_sums(float& u, float& v, int lpr, float2* red) {
  if (!WIDE) {
    u = lanes_sum(u, lpr);
    v = lanes_sum(v, lpr);
    return;
  }
  u = lanes_sum(u, 64);
  v = lanes_sum(v, 64);
  const int waves = blockDim.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = make_float2(u, v);
  __syncthreads();
  u = v = 0.f;
  for (int w = 0; w < waves; w++) {
    u += red[w].x;
    v += red[w].y;
  }
}

template <typename T, bool VEC, bool WIDE>
__global__ void __launch_bounds__(WIDE ? 1024 : 256) rows_kernel(GatedNormArgs a, int lpr, int chunk_rows) {
  __shared__ float2 red[16];
  __shared__ float cols[WIDE ? 1 : 256 * 24];
  int seq, chunk;
  if (!find_unit(a.nseq, blockIdx.x, [&](int i) { return cdiv(a.pr.count(i), chunk_rows); }, seq, chunk)) return;
  const int begin = a.pr.begin(seq) + chunk * chunk_rows;
  const int end = min(begin + chunk_rows, a.pr.begin(seq) + a.pr.count(seq));
  const int D = a.D, groups = WIDE ? 1 : blockDim.x / lpr, l = WIDE ? (int)threadIdx.x : (int)threadIdx.x & (lpr - 1);
  const int grp = WIDE ? 0 : threadIdx.x / lpr;
  const int at = l < lpr ? place<VEC>(0, l, lpr) : a.D;
  const int64_t mo = seq * a.mod_row;
  float kh[8], ky[8], R[8], P[8], Q[8];   // (1 + scale) pre_w; gate post_w
  bool in[8];
  {
    float w[8], m[8];
#pragma unroll
    for (int i = 0; i < 8; i++) kh[i] = ky[i] = 1.f;
    if (a.scale) {
      load8<float, VEC>(a.scale + mo, at, lpr, D, m);
#pragma unroll
      for (int i = 0; i < 8; i++) kh[i] += m[i];
    }
    if (a.pre_w) {
      load8<T, VEC>((const T*)a.pre_w, at, lpr, D, w);
#pragma unroll
      for (int i = 0; i < 8; i++) kh[i] *= w[i];
    }
    if (a.gate) {
      load8<float, VEC>(a.gate + mo, at, lpr, D, m);
#pragma unroll
      for (int i = 0; i < 8; i++) ky[i] *= m[i];
    }
    if (a.post_w) {
      load8<T, VEC>((const T*)a.post_w, at, lpr, D, w);
#pragma unroll
      for (int i = 0; i < 8; i++) ky[i] *= w[i];
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
      in[i] = VEC ? at < D : at + i * lpr < D;
      R[i] = P[i] = Q[i] = 0.f;
    }
  }
  const float inv_d = 1.f / (float)D;
  // (every group makes the same number of turns, so that barriers meet; a turn without a row works on the last one and keeps nothing)
  for (int r0 = begin; r0 < end; r0 += groups) {
    const bool live = r0 + grp < end;
    const int64_t row = min(r0 + grp, end - 1);
    float xv[8], yv[8], t[8], dh[8];
    load8<T, VEC>((const T*)a.x + row * a.x_row, at, lpr, D, xv);
    if (a.y) load8<T, VEC>((const T*)a.y + row * a.y_row, at, lpr, D, yv);
    if (a.dx_out) load8<T, VEC>((const T*)a.dx_out + row * a.x_row, at, lpr, D, t);
    if (a.dh) load8<T, VEC>((const T*)a.dh + row * a.h_row, at, lpr, D, dh);
#pragma unroll
    for (int i = 0; i < 8; i++) {
      if (!a.y) yv[i] = 0.f;
      if (!a.dx_out) t[i] = 0.f;
      if (!a.dh) dh[i] = 0.f;
    }
    float u = 0.f, w = 0.f, mx = 0.f, my = 0.f, rx = 1.f, ry = 1.f;
    if (a.pre == NORM_LAYER || a.post == NORM_LAYER) {
#pragma unroll
      for (int i = 0; i < 8; i++) {
        u += xv[i];
        w += yv[i];
      }
      row_sums<WIDE>(u, w, lpr, red);
      if (a.pre == NORM_LAYER) mx = u * inv_d;
      if (a.post == NORM_LAYER) my = w * inv_d;
    }
    u = w = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      xv[i] = in[i] ? xv[i] - mx : 0.f;
      yv[i] = in[i] ? yv[i] - my : 0.f;
      u = fmaf(xv[i], xv[i], u);
      w = fmaf(yv[i], yv[i], w);
    }
    if (a.pre != NORM_NONE || a.post != NORM_NONE) {
      row_sums<WIDE>(u, w, lpr, red);
      if (a.pre != NORM_NONE) rx = rsqrtf(u * inv_d + a.eps);
      if (a.post != NORM_NONE) ry = rsqrtf(w * inv_d + a.eps);
    }
    if (a.dh) {
      u = w = 0.f;
      float gx[8];
#pragma unroll
      for (int i = 0; i < 8; i++) {
        xv[i] *= rx;
        gx[i] = dh[i] * kh[i];
        u += gx[i];
        w = fmaf(gx[i], xv[i], w);
      }
      if (a.pre != NORM_NONE) row_sums<WIDE>(u, w, lpr, red);
      const float mg = a.pre == NORM_LAYER ? u * inv_d : 0.f, mgx = a.pre != NORM_NONE ? w * inv_d : 0.f;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        t[i] += rx * (gx[i] - mg - xv[i] * mgx);
        if (live) {
          R[i] += dh[i];
          P[i] = fmaf(dh[i], xv[i], P[i]);
        }
      }
    }
    if (a.y) {
#pragma unroll
      for (int i = 0; i < 8; i++) {
        yv[i] *= ry;
        if (live) Q[i] = fmaf(t[i], yv[i], Q[i]);
      }
      if (a.dy) {
        float gy[8];
        u = w = 0.f;
#pragma unroll
        for (int i = 0; i < 8; i++) {
          gy[i] = in[i] ? t[i] * ky[i] : 0.f;
          u += gy[i];
          w = fmaf(gy[i], yv[i], w);
        }
        if (a.post != NORM_NONE) row_sums<WIDE>(u, w, lpr, red);
        const float mg = a.post == NORM_LAYER ? u * inv_d : 0.f, mgy = a.post != NORM_NONE ? w * inv_d : 0.f;
#pragma unroll
        for (int i = 0; i < 8; i++) gy[i] = ry * (gy[i] - mg - yv[i] * mgy);
        if (live) store8<T, VEC>((T*)a.dy + row * a.y_row, at, lpr, D, gy);
      }
    }
    if (a.dx && live) {
#pragma unroll
      for (int i = 0; i < 8; i++) t[i] *= a.alpha;
      store8<T, VEC>((T*)a.dx + row * a.x_row, at, lpr, D, t);
    }
  }
  if (!a.parts) return;
  float* out = a.parts + (int64_t)blockIdx.x * 3 * D;
  if (!WIDE) {   // the groups of rows, in order
#pragma unroll
    for (int i = 0; i < 8; i++) {
      cols[threadIdx.x * 24 + i] = R[i];
      cols[threadIdx.x * 24 + 8 + i] = P[i];
      cols[threadIdx.x * 24 + 16 + i] = Q[i];
    }
    __syncthreads();
    if (grp > 0) return;
    for (int g = 1; g < groups; g++)
#pragma unroll
      for (int i = 0; i < 8; i++) {
        R[i] += cols[(g * lpr + l) * 24 + i];
        P[i] += cols[(g * lpr + l) * 24 + 8 + i];
        Q[i] += cols[(g * lpr + l) * 24 + 16 + i];
      }
  }
  store8<float, VEC>(out, at, lpr, D, R);
  store8<float, VEC>(out + D, at, lpr, D, P);
  store8<float, VEC>(out + 2 * D, at, lpr, D, Q);
}

// Sums of the chunks of one sequence, 64 columns per workgroup, its 4 waves sharing the chunks:
//   dshift = R, dscale = P pre_w, dgate = Q post_w.
// P and Q stay behind for the weights' gradients (in the sequence's place after the chunks).
template <typename T>
__global__ void __launch_bounds__(256) columns_kernel(GatedNormArgs a, int chunk_rows) {
  __shared__ float red[3][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = a.D;
  const int blocks = cdiv(D, 64), seq = blockIdx.x / blocks, col = (blockIdx.x - seq * blocks) * 64 + lane;
  int64_t before = 0;
  for (int i = lane; i < seq; i += 64) before += cdiv(a.pr.count(i), chunk_rows);
  for (int o = 32; o > 0; o >>= 1) before += __shfl_xor(before, o, 64);
  // (offsets that are not increasing can promise more chunks than there are)
  const int n = (int)min((int64_t)cdiv(a.pr.count(seq), chunk_rows), a.chunks - before);
  float s[3] = {0.f, 0.f, 0.f};
  if (col < D)
    for (int c = wave; c < n; c += 4) {
      const float* p = a.parts + (before + c) * 3 * D + col;
#pragma unroll
      for (int k = 0; k < 3; k++) s[k] += p[(int64_t)k * D];
    }
#pragma unroll
  for (int k = 0; k < 3; k++) red[k][wave][lane] = s[k];
  __syncthreads();
  if (wave > 0 || col >= D) return;
#pragma unroll
  for (int k = 0; k < 3; k++) s[k] = red[k][0][lane] + red[k][1][lane] + red[k][2][lane] + red[k][3][lane];
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

// dpre_w = sum over the sequences of (1 + scale) P, dpost_w of gate Q.
__global__ void __launch_bounds__(256) weights_kernel(GatedNormArgs a) {
  const int col = blockIdx.x * 256 + threadIdx.x, D = a.D;
  if (col >= D) return;
  float p = 0.f, q = 0.f;
  for (int s = 0; s < a.nseq; s++) {
    const float* k = a.parts + ((int64_t)a.chunks * 3 + 2 * s) * D + col;
    const int64_t at = s * a.mod_row + col;
    p = fmaf(a.scale ? 1.f + a.scale[at] : 1.f, k[0], p);
    q = fmaf(a.gate ? a.gate[at] : 1.f, k[D], q);
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
// lanes of a row of D elements in a wave
int lanes_of(int D) {
  int l = 8;
  while (l < 64 && l * 8 < D) l *= 2;
  return l;
}

template <typename T, int CH>
void forward_launch(const GatedNormArgs& a, hipStream_t s) {
  const int lpr = lanes_of(a.D);
  const int grid = cdiv(a.rows, 4 * (64 / lpr));
  if (vectors(a)) forward_kernel<T, CH, true><<<grid, 256, 0, s>>>(a, lpr);
  else forward_kernel<T, CH, false><<<grid, 256, 0, s>>>(a, lpr);
}
template <typename T>
void forward_chunks(const GatedNormArgs& a, hipStream_t s) {
  const int ch = cdiv(a.D, 512);
  if (ch <= 1) forward_launch<T, 1>(a, s);
  else if (ch <= 2) forward_launch<T, 2>(a, s);
  else if (ch <= 4) forward_launch<T, 4>(a, s);
  else if (ch <= 6) forward_launch<T, 6>(a, s);
  else if (ch <= 8) forward_launch<T, 8>(a, s);
  else forward_launch<T, 16>(a, s);
}

// Rows of a chunk: enough chunks to fill the chip, long enough that their sums (3 fp32 rows out and in again) stay
// small beside their rows.
int chunk_rows_of(int rows) { return std::min(64, std::max(8, rows / 1024)); }

template <typename T>
void rows_launch(const GatedNormArgs& a, hipStream_t s) {
  const int lpr = a.D > 512 ? cdiv(a.D, 8) : lanes_of(a.D), cr = chunk_rows_of(a.rows);
  const bool vec = vectors(a);
  if (a.D > 512) {
    const int threads = cdiv(lpr, 64) * 64;
    if (vec) rows_kernel<T, true, true><<<a.chunks, threads, 0, s>>>(a, lpr, cr);
    else rows_kernel<T, false, true><<<a.chunks, threads, 0, s>>>(a, lpr, cr);
  } else if (vec) {
    rows_kernel<T, true, false><<<a.chunks, 256, 0, s>>>(a, lpr, cr);
  } else {
    rows_kernel<T, false, false><<<a.chunks, 256, 0, s>>>(a, lpr, cr);
  }
}

}  // namespace

hipError_t gated_norm_fwd(const GatedNormArgs& a, int dtype, hipStream_t s) {
  if (dtype == DT_BF16) forward_chunks<u16>(a, s);
  else forward_chunks<float>(a, s);
  return hipGetLastError();
}

int gated_norm_chunks(int nseq, int rows) { return (int)std::min<int64_t>((int64_t)rows / chunk_rows_of(rows) + nseq, 0x7fffffff); }
size_t gated_norm_ws(int nseq, int rows, int D) {
  return ((size_t)gated_norm_chunks(nseq, rows) * 3 + 2 * (size_t)nseq) * D * 4;
}

hipError_t gated_norm_rows_bwd(const GatedNormArgs& a, int dtype, hipStream_t s) {
  if (dtype == DT_BF16) rows_launch<u16>(a, s);
  else rows_launch<float>(a, s);
  return hipGetLastError();
}

hipError_t gated_norm_columns_bwd(const GatedNormArgs& a, int dtype, hipStream_t s) {
  const int64_t grid = (int64_t)cdiv(a.D, 64) * a.nseq;
  const int cr = chunk_rows_of(a.rows);
  if (grid == 0) {
  } else if (dtype == DT_BF16) columns_kernel<u16><<<grid, 256, 0, s>>>(a, cr);
  else columns_kernel<float><<<grid, 256, 0, s>>>(a, cr);
  if (a.dpre_w || a.dpost_w) weights_kernel<<<cdiv(a.D, 256), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace dit
