// Gradients of packed attention on gfx950. With s = scale q k^T, p = exp(s - lse) and delta = rowsum(do o),
//   dv = p^T do,   ds = p (do v^T - delta),   dq = scale ds k,   dk = scale ds^T q.
//
// Two kinds of workgroup recompute p, so that every gradient is summed in a fixed order without atomics: one owns
// query rows and walks the keys (dq: 3 products), one owns keys and walks the query rows of all heads that share them
// (dk, dv: 4 products). That is 7 products where 5 would do with atomics on dq.
// Bound by the matrix instructions: causal, 8192 tokens of 32 over 8 heads in 1730 to 1860 us from card to
// card, in which the 7 products run at 1030 to 1110 TFLOP/s.
//
// bf16, v_mfma_f32_32x32x16_bf16, 4 waves: an owned row (or key) is a column of the score block, so that p and ds
// of a lane belong to one owned row and are operand B of the next product as they stand, rounded to bf16 (up to 2^-8 of each term,
// which the sums average to the size of the outputs' own rounding: the gradients are off by 0.0024 of themselves in the 2-norm, by 0.0017
// were only they rounded). The walked rows are in LDS twice over time, never in two
// layouts: a tile is read by rows for the scores and by columns (transposing reads) for the gradients.
#include <algorithm>

#include "attn_common.h"
#include "packed.h"

namespace dit {

namespace {
constexpr float LOG2E = 1.4426950408889634f;

// What p is formed with, or what makes every p of a row without visible keys 0. bf16: lse in log2 units, p = exp2(c s - lse2) in one
// operation; the rounding of lse2 is below that of p to bf16 (2^-8) while |lse| < 2^16. fp32: lse itself, and the difference
// from it is taken before it goes to the exponential's base, which rounds it no further.
template <typename T> __device__ __forceinline__ float lse_of(float lse) {
  return lse == -INFINITY ? INFINITY : sizeof(T) == 2 ? lse * LOG2E : lse;
}
__device__ __forceinline__ float p_f32(float s, float lse) { return __builtin_amdgcn_exp2f((s - lse) * LOG2E); }

// stats[head][tok] = (lse as above, delta = sum_e do o): D / 8 (bf16) or D / 4 lanes per row, 16 bytes each. By head, so that the
// rows a key tile walks read theirs in one piece ([tok][head] as lse comes: 1273 us for dk, dv of 8192 keys, 8 of 32 heads).
template <typename T, int D>
__global__ void __launch_bounds__(256) stats_kernel(PackedArgs a) {
  constexpr int EL = 16 / sizeof(T), LPR = D / EL;
  const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LPR;
  const int c = threadIdx.x % LPR;
  if (row >= (int64_t)a.qr.total * a.H) return;
  const int head = row / a.qr.total, tok = row - (int64_t)head * a.qr.total;
  const int64_t at = (int64_t)tok * a.o_row + (int64_t)head * a.o_head + EL * c;
  const T* x = (const T*)a.o + at;
  const T* y = (const T*)a.d_o + at;
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < EL; i += 4) {
    float f[4], g[4];
    load4<T>(x + i, f);
    load4<T>(y + i, g);
#pragma unroll
    for (int j = 0; j < 4; j++) s = fmaf(f[j], g[j], s);
  }
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (c == 0) a.stats[row] = make_float2(lse_of<T>(a.lse[(int64_t)tok * a.H + head]), s);
}
__device__ __forceinline__ float2 stats_of(const PackedArgs& a, int64_t tok, int64_t head) { return a.stats[head * a.qr.total + tok]; }

// Address parts of a transposing read of a tile: this lane's 4 dims of dim block db, row 4 half + (lane >> 2) % 4 + 8 e of a step
template <int D>
__device__ __forceinline__ void tr_bases(int lane, int (*base)[2]) {
  const int r = 4 * (lane >> 5) + ((lane >> 2) & 3);
#pragma unroll
  for (int db = 0; db < D / 32; db++) {
    const int ch = 4 * db + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
#pragma unroll
    for (int e = 0; e < 2; e++)
      base[db][e] = (r + 8 * e) * (2 * D) + ((ch ^ tile_swizzle<D>(r + 8 * e)) << 4) + 8 * (lane & 1);
  }
}

// acc[dim][column] of this wave's 32 columns, times f, to rows of bf16 through 32 rows of LDS: store(column, chunk, value)
template <int D, typename F>
__device__ __forceinline__ void store_columns(char* so, const f32x16* acc, float f, int lane, F&& store) {
  constexpr int CH = D / 8, RB = D * 2;
  const int half = lane >> 5, l32 = lane & 31;
#pragma unroll
  for (int db = 0; db < D / 32; db++)
#pragma unroll
    for (int g = 0; g < 4; g++) {
      uint2 u;
      u.x = pack_bf16x2(acc[db][4 * g] * f, acc[db][4 * g + 1] * f);
      u.y = pack_bf16x2(acc[db][4 * g + 2] * f, acc[db][4 * g + 3] * f);
      *(uint2*)(so + l32 * RB + (((4 * db + g) ^ (l32 % CH)) << 4) + 8 * half) = u;
    }
  wave_fence();
  constexpr int RPI = 64 / CH;
#pragma unroll
  for (int i = 0; i < 32 / RPI; i++) {
    const int r = i * RPI + lane / CH, ch = lane % CH;
    store(r, ch, *(const uint4*)(so + r * RB + ((ch ^ (r % CH)) << 4)));
  }
  wave_fence();   // (the rows may be written again)
}

// Both kinds of workgroup are in one launch, those of the keys, which are the longer, first. In a launch each, every CU waits between
// them for the last workgroup of the first (all gradients, graph replays, us in two launches / one: fp32 3 x 80..333 tokens 26.1 / 19.8,
// joint attention of 512 tokens 312 / 297, causal 8192 tokens 1905 / 1862).
template <int D> constexpr int GRAD_LDS = 4 * 64 * 2 * D + 512;

template <int ROWS> __device__ __forceinline__ bool find_row_tile(const PackedArgs& a, int block, int& seq, int& tile, PackedSeq& s) {
  return find_unit(a.nseq, block / a.Hkv, [&](int i) { return a.sequence(i); },
                   [&](const PackedSeq& x) { return (x.m * a.G + ROWS - 1) / ROWS; }, seq, tile, s);
}
template <int KEYS> __device__ __forceinline__ bool find_key_tile(const PackedArgs& a, int block, int shares, int& seq, int& tile, PackedSeq& s) {
  return find_unit(a.nseq, block / (a.Hkv * shares), [&](int i) { return a.sequence(i); },
                   [&](const PackedSeq& x) { return (x.n + KEYS - 1) / KEYS; }, seq, tile, s);
}

// ---------------------------------------------------------------------------
// dq: 128 query rows (row r: query r / G, head r % G of the group) against 64-key tiles
// ---------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ void dq_bf16(const PackedArgs& a, int block, char* smem) {   // [K0][K1][V0][V1]
  constexpr int ROWS = 128, KB = 64, NDB = D / 32, NKS = D / 16;
  using Tile = RowTile<D, KB, 4>;
  constexpr int TILE = Tile::BYTES, RB = Tile::RB;
  static_assert(4 * TILE <= GRAD_LDS<D>, "");
  const int g = block % a.Hkv;
  int seq, rt;
  PackedSeq sq;
  if (!find_row_tile<ROWS>(a, block, seq, rt, sq)) return;
  const int m = sq.m, n = sq.n;
  const int rows = m * a.G;
  if (a.causal) rt = cdiv(rows, ROWS) - 1 - rt;
  const int row0 = rt * ROWS;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int half = lane >> 5, l32 = lane & 31;
  const int q0 = sq.q0;
  const int64_t k0 = sq.k0;
  const u16* Kg = (const u16*)a.k + k0 * a.k_row + (int64_t)g * a.k_head;
  const u16* Vg = (const u16*)a.v + k0 * a.v_row + (int64_t)g * a.v_head;
  const int row = min(row0 + wave * 32 + l32, rows - 1);
  const int tok = row / a.G, head = g * a.G + (row - tok * a.G);
  const int vis = a.causal ? min(tok + n - m + 1, n) : n;
  bf16x8 qf[NKS], df[NKS];
  {
    const u16* qrow = (const u16*)a.q + (int64_t)(q0 + tok) * a.q_row + (int64_t)head * a.q_head;
    const u16* drow = (const u16*)a.d_o + (int64_t)(q0 + tok) * a.o_row + (int64_t)head * a.o_head;
#pragma unroll
    for (int s = 0; s < NKS; s++) {
      qf[s] = *(const bf16x8*)(qrow + 16 * s + 8 * half);
      df[s] = *(const bf16x8*)(drow + 16 * s + 8 * half);
    }
  }
  const float2 st = stats_of(a, q0 + tok, head);
  const float lse2 = st.x, delta = st.y;
  const int last_tok = (min(row0 + ROWS, rows) - 1) / a.G;
  const int nvis = a.causal ? min(max(last_tok + n - m + 1, 0), n) : n;
  const int all_vis = __builtin_amdgcn_readfirstlane(vis);
  const int nt = cdiv(nvis, KB);
  Tile tk, tv;
  tk.init(wave, lane, a.k_row);
  tv.init(wave, lane, a.v_row);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem;
  auto issue = [&](int kt) {
    tk.load(Kg + (int64_t)kt * KB * a.k_row, n - kt * KB, lds0 + (kt & 1) * TILE);
    tv.load(Vg + (int64_t)kt * KB * a.v_row, n - kt * KB, lds0 + (2 + (kt & 1)) * TILE);
  };
  int kbase[NDB][2];
  tr_bases<D>(lane, kbase);
  f32x16 dq[NDB];
#pragma unroll
  for (int i = 0; i < NDB; i++)
#pragma unroll
    for (int r = 0; r < 16; r++) dq[i][r] = 0.f;
  const f32x16 zero = {};
  const float c = a.scale * LOG2E;
  if (nt > 0) issue(0);
  for (int kt = 0; kt < nt; kt++) {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();   // tile kt has landed, and every wave is done with the other buffers
    if (kt + 1 < nt) issue(kt + 1);
    const char* sk = smem + (kt & 1) * TILE;
    const char* sv = smem + (2 + (kt & 1)) * TILE;
    const bool mask = (kt + 1) * KB > all_vis;
#pragma unroll
    for (int kb = 0; kb < KB / 32; kb++) {
      f32x16 s, dp;
#pragma unroll
      for (int x = 0; x < NKS; x++) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Tile::read(sk, 32 * kb + l32, 2 * x + half), qf[x], x == 0 ? zero : s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Tile::read(sv, 32 * kb + l32, 2 * x + half), df[x], x == 0 ? zero : dp, 0, 0, 0);
      }
      if (mask) {
#pragma unroll
        for (int r = 0; r < 16; r++)
          if (kt * KB + 32 * kb + 8 * (r >> 2) + 4 * half + (r & 3) >= vis) s[r] = -INFINITY;
      }
      bf16x8 ds[2];
#pragma unroll
      for (int h = 0; h < 2; h++)
#pragma unroll
        for (int j = 0; j < 8; j++) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[8 * h + j], c, -lse2));
          ds[h][j] = (__bf16)(p * (dp[8 * h + j] - delta));
        }
#pragma unroll
      for (int h = 0; h < 2; h++)
#pragma unroll
        for (int db = 0; db < NDB; db++) {
          const char* p0 = sk + (32 * kb + 16 * h) * RB;
          dq[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(join_tr(read_tr(p0 + kbase[db][0]), read_tr(p0 + kbase[db][1])),
                                                           ds[h], dq[db], 0, 0, 0);
        }
    }
  }
  if (__ballot(vis <= 0) != 0) {   // rows that see no key: nothing of one that is no number
#pragma unroll
    for (int i = 0; i < NDB; i++)
      if (vis <= 0) dq[i] = zero;
  }
  __syncthreads();   // every wave is done with the K buffers
  store_columns<D>(smem + wave * 32 * RB, dq, a.scale, lane, [&](int r, int ch, uint4 v) {
    const int rr = row0 + wave * 32 + r;
    if (rr < rows) {
      const int t = rr / a.G, hd = g * a.G + (rr - t * a.G);
      *(uint4*)((u16*)a.dq + (int64_t)(q0 + t) * a.q_row + (int64_t)hd * a.q_head + 8 * ch) = v;
    }
  });
}

// ---------------------------------------------------------------------------
// dk, dv: 128 keys of one key/value head against 32-query tiles of every head of its group in turn. V stays in LDS and K in
// registers: with both in registers 40 of them spilled at two waves per SIMD (these products alone, joint attention at 512x512:
// 232 us against 197).
// The tiles may be shared out between a.shares workgroups, whose sums meet in the workspace (shares_join).
// ---------------------------------------------------------------------------
// The first of `steps` that share i of n takes.
__device__ __forceinline__ int share_begin(int steps, int i, int n) { return (int)((int64_t)steps * i / n); }
// Where share i keeps dk (without the factor scale) and dv of a key: 2 D floats.
__device__ __forceinline__ float* share_row(const PackedArgs& a, int D, int i, int64_t key_row, int g) {
  return a.share_sums + (((int64_t)i * a.kr.total + key_row) * a.Hkv + g) * 2 * D;
}

template <int D>
__device__ __forceinline__ void dkdv_bf16(const PackedArgs& a, int block, char* smem) {   // [Q0][Q1][dO0][dO1][V], then the rows' statistics
  constexpr int KEYS = 128, QB = 32, NDB = D / 32, NKS = D / 16;
  using Tile = RowTile<D, QB, 4>;
  constexpr int TILE = Tile::BYTES, RB = Tile::RB;
  static_assert(4 * TILE + KEYS * RB + 4 * QB * 4 <= GRAD_LDS<D>, "");
  auto stat = (float4(*)[2][QB / 4])(smem + 4 * TILE + KEYS * RB);   // lse (log2 units) and delta of a tile's rows
  const int g = block % a.Hkv;
  int seq, kt;
  PackedSeq ps;
  if (!find_key_tile<KEYS>(a, block, a.shares, seq, kt, ps)) return;
  const int share = block / a.Hkv % a.shares;
  const int m = ps.m, n = ps.n;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int half = lane >> 5, l32 = lane & 31;
  const int64_t q0 = ps.q0, k0 = ps.k0;
  const int key = kt * KEYS + wave * 32 + l32;
  bf16x8 kf[NKS];
  {
    const int64_t kr = k0 + min(key, n - 1);
    const u16* krow = (const u16*)a.k + kr * a.k_row + (int64_t)g * a.k_head;
#pragma unroll
    for (int s = 0; s < NKS; s++) {
      kf[s] = *(const bf16x8*)(krow + 16 * s + 8 * half);
    }
  }
  // the first query that sees any of the tile's keys; queries from `first` of this lane on see its key
  const int first = a.causal ? key - (n - m) : 0;
  const int t0 = a.causal ? min(max(kt * KEYS - (n - m), 0), m) / QB : 0;
  const int wave_first = a.causal ? kt * KEYS + __builtin_amdgcn_readfirstlane(wave) * 32 + 31 - (n - m) : 0;
  const int per = cdiv(m, QB) - t0;   // tiles of one head
  const int begin = share_begin(per * a.G, share, a.shares), steps = share_begin(per * a.G, share + 1, a.shares) - begin;
  Tile tq, td;
  tq.init(wave, lane, a.q_row);
  td.init(wave, lane, a.o_row);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem;
  {
    RowTile<D, KEYS, 4> tv;
    tv.init(wave, lane, a.v_row);
    tv.load((const u16*)a.v + (k0 + kt * KEYS) * a.v_row + (int64_t)g * a.v_head, n - kt * KEYS, lds0 + 4 * TILE);
  }
  const char* sv = smem + 4 * TILE + wave * 32 * RB;
  int ih = per > 0 ? begin / per : 0, it = t0 + begin - ih * per;   // head and tile of the next loads
  float2 nstat = make_float2(INFINITY, 0.f);
  auto issue = [&](int i) {
    const int64_t head = (int64_t)g * a.G + ih;
    tq.load((const u16*)a.q + (q0 + it * QB) * a.q_row + head * a.q_head, m - it * QB, lds0 + (i & 1) * TILE);
    td.load((const u16*)a.d_o + (q0 + it * QB) * a.o_row + head * a.o_head, m - it * QB, lds0 + (2 + (i & 1)) * TILE);
    if (tid < QB) {
      const int t = it * QB + tid;
      nstat = t < m ? stats_of(a, q0 + t, head) : make_float2(INFINITY, 0.f);   // rows past the end: p = 0
    }
    if (++it == t0 + per) {
      it = t0;
      ih++;
    }
  };
  auto put_stats = [&](int i) {
    if (tid < QB) {
      ((float*)stat[i & 1][0])[tid] = nstat.x;
      ((float*)stat[i & 1][1])[tid] = nstat.y;
    }
  };
  int base[NDB][2];
  tr_bases<D>(lane, base);
  f32x16 dk[NDB], dv[NDB];
#pragma unroll
  for (int i = 0; i < NDB; i++)
#pragma unroll
    for (int r = 0; r < 16; r++) dk[i][r] = dv[i][r] = 0.f;
  const f32x16 zero = {};
  const float c = a.scale * LOG2E;
  const int it0 = it;
  if (steps > 0) {
    issue(0);
    put_stats(0);
  }
  int ct = it0;
  for (int i = 0; i < steps; i++) {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();   // tile i has landed, and every wave is done with the other buffers
    if (i + 1 < steps) issue(i + 1);
    const char* sq = smem + (i & 1) * TILE;
    const char* sd = smem + (2 + (i & 1)) * TILE;
#pragma unroll
    for (int qb = 0; qb < QB / 32; qb++) {
      f32x16 s, dp;
#pragma unroll
      for (int x = 0; x < NKS; x++) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Tile::read(sq, 32 * qb + l32, 2 * x + half), kf[x], x == 0 ? zero : s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Tile::read(sd, 32 * qb + l32, 2 * x + half), Tile::read(sv, l32, 2 * x + half), x == 0 ? zero : dp, 0, 0, 0);
      }
      const int r0 = ct * QB + 32 * qb;
      if (r0 < wave_first) {
#pragma unroll
        for (int r = 0; r < 16; r++)
          if (r0 + 8 * (r >> 2) + 4 * half + (r & 3) < first) s[r] = -INFINITY;
      }
      bf16x8 pf[2], ds[2];
#pragma unroll
      for (int h = 0; h < 2; h++)
#pragma unroll
        for (int j4 = 0; j4 < 2; j4++) {
          const float4 l4 = stat[i & 1][0][8 * qb + 4 * h + 2 * j4 + half], d4 = stat[i & 1][1][8 * qb + 4 * h + 2 * j4 + half];
          const float ls[4] = {l4.x, l4.y, l4.z, l4.w}, de[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
          for (int j = 0; j < 4; j++) {
            const int x = 8 * h + 4 * j4 + j;
            const float p = __builtin_amdgcn_exp2f(fmaf(s[x], c, -ls[j]));
            pf[h][4 * j4 + j] = (__bf16)p;
            ds[h][4 * j4 + j] = (__bf16)(p * (dp[x] - de[j]));
          }
        }
#pragma unroll
      for (int h = 0; h < 2; h++)
#pragma unroll
        for (int db = 0; db < NDB; db++) {
          const int at = (32 * qb + 16 * h) * RB;
          dv[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              join_tr(read_tr(sd + at + base[db][0]), read_tr(sd + at + base[db][1])), pf[h], dv[db], 0, 0, 0);
          dk[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              join_tr(read_tr(sq + at + base[db][0]), read_tr(sq + at + base[db][1])), ds[h], dk[db], 0, 0, 0);
        }
    }
    if (i + 1 < steps) put_stats(i + 1);
    if (++ct == t0 + per) ct = t0;
  }
  if (a.shares > 1) {
    if (key < n) {
      float* pk = share_row(a, D, share, k0 + key, g);
#pragma unroll
      for (int db = 0; db < NDB; db++)
#pragma unroll
        for (int q = 0; q < 4; q++) {
          const int e = 32 * db + 8 * q + 4 * half;
          *(float4*)(pk + e) = make_float4(dk[db][4 * q], dk[db][4 * q + 1], dk[db][4 * q + 2], dk[db][4 * q + 3]);
          *(float4*)(pk + D + e) = make_float4(dv[db][4 * q], dv[db][4 * q + 1], dv[db][4 * q + 2], dv[db][4 * q + 3]);
        }
    }
    return;
  }
  __syncthreads();
  auto rows_to = [&](void* dst, int64_t row_stride, int64_t head_stride) {
    return [=](int r, int ch, uint4 v) {
      const int kk = kt * KEYS + wave * 32 + r;
      if (kk < n) *(uint4*)((u16*)dst + (k0 + kk) * row_stride + (int64_t)g * head_stride + 8 * ch) = v;
    };
  };
  store_columns<D>(smem + wave * 32 * RB, dk, a.scale, lane, rows_to(a.dk, a.k_row, a.k_head));
  store_columns<D>(smem + wave * 32 * RB, dv, 1.f, lane, rows_to(a.dv, a.v_row, a.v_head));
}

template <int D>
__global__ void __launch_bounds__(256, 2) packed_gradients_bf16(PackedArgs a, int key_blocks) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[GRAD_LDS<D>];
  if ((int)blockIdx.x < key_blocks) dkdv_bf16<D>(a, blockIdx.x, smem);
  else dq_bf16<D>(a, blockIdx.x - key_blocks, smem);
#endif
}

// ---------------------------------------------------------------------------
// fp32: 4 waves own 16 rows (or keys) each and share tiles of 16 keys (rows) of both operands. SPLIT, for problems that have too few such
// workgroups to fill the chip: the waves own the same 16 and take every fourth tile, each staging its own, so that
// the chain of tiles is a quarter as long; their sums meet at the end.
// ---------------------------------------------------------------------------
template <int D, bool SPLIT> constexpr int WALK_LDS = (SPLIT ? 4 : 2) * 16 * (D + 4);   // floats of one operand's tiles

template <int D, bool SPLIT>
__device__ __forceinline__ void dq_f32(const PackedArgs& a, int block, float* smem) {
  constexpr int ROWS = SPLIT ? 16 : 64, NKC = D / 16, LANES = SPLIT ? 64 : 256;
  using W = WalkF32<D, LANES>;
  auto sk = (float(*)[W::NROW * W::LD])smem, sv = (float(*)[W::NROW * W::LD])(smem + WALK_LDS<D, SPLIT>);
  const int g = block % a.Hkv;
  int seq, rt;
  PackedSeq sq;
  if (!find_row_tile<ROWS>(a, block, seq, rt, sq)) return;
  const int m = sq.m, n = sq.n, rows = m * a.G;
  if (a.causal) rt = cdiv(rows, ROWS) - 1 - rt;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
  const int row0 = rt * ROWS, mine = row0 + (SPLIT ? 0 : wave * 16) + l16;
  const int64_t q0 = sq.q0, k0 = sq.k0;
  const float* Kg = (const float*)a.k + k0 * a.k_row + (int64_t)g * a.k_head;
  const float* Vg = (const float*)a.v + k0 * a.v_row + (int64_t)g * a.v_head;
  const int row = min(mine, rows - 1);
  const int tok = row / a.G, head = g * a.G + (row - tok * a.G);
  const int vis = a.causal ? min(tok + n - m + 1, n) : n;
  f32x4 qf[NKC], df[NKC];
  {
    const float* qrow = (const float*)a.q + (q0 + tok) * a.q_row + (int64_t)head * a.q_head;
    const float* drow = (const float*)a.d_o + (q0 + tok) * a.o_row + (int64_t)head * a.o_head;
#pragma unroll
    for (int c = 0; c < NKC; c++) {
      qf[c] = *(const f32x4*)(qrow + 16 * c + 4 * g4);
#pragma unroll
      for (int e = 0; e < 4; e++) qf[c][e] *= a.scale;
      df[c] = *(const f32x4*)(drow + 16 * c + 4 * g4);
    }
  }
  const float2 st = stats_of(a, q0 + tok, head);
  const int last_tok = (min(row0 + ROWS, rows) - 1) / a.G;
  const int nvis = a.causal ? min(max(last_tok + n - m + 1, 0), n) : n;
  const int nt = cdiv(nvis, W::NROW), first = SPLIT ? wave : 0, step = SPLIT ? 4 : 1;
  f32x4 dq[NKC];
#pragma unroll
  for (int i = 0; i < NKC; i++) dq[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  W w;
  auto fetch = [&](int kt) {
    w.fetch(Kg + (int64_t)kt * W::NROW * a.k_row, a.k_row, Vg + (int64_t)kt * W::NROW * a.v_row, a.v_row, n - kt * W::NROW);
  };
  auto buf_of = [&](int kt) { return SPLIT ? wave : kt & 1; };
  if (first < nt) {
    fetch(first);
    w.stage(sk[buf_of(first)], sv[buf_of(first)]);
    if (SPLIT) wave_fence();
  }
  for (int kt = first; kt < nt; kt += step) {
    const int buf = buf_of(kt);
    if (!SPLIT) __syncthreads();   // (a wave's own tile needs none)
    if (kt + step < nt) fetch(kt + step);
    f32x4 s = W::dot(sk[buf], qf, l16, g4), dp = W::dot(sv[buf], df, l16, g4);
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const bool hidden = kt * W::NROW + 4 * g4 + r >= vis;
      s[r] = hidden ? 0.f : p_f32(s[r], st.x) * (dp[r] - st.y);
    }
    W::add(dq, sk[buf], s, l16, g4);
    if (SPLIT) wave_fence();
    if (kt + step < nt) w.stage(sk[buf_of(kt + step)], sv[buf_of(kt + step)]);
    if (SPLIT) wave_fence();
  }
  if (SPLIT) {
    join_waves<D>(sk[0], dq, wave, l16, g4);
    if (wave > 0) return;
  }
  if (mine >= rows) return;
  if (vis <= 0)   // a row that sees no key: nothing of one that is no number
#pragma unroll
    for (int i = 0; i < NKC; i++) dq[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float* out = (float*)a.dq + (q0 + tok) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
  for (int i = 0; i < NKC; i++)
    *(float4*)(out + 16 * i + 4 * g4) = make_float4(dq[i][0] * a.scale, dq[i][1] * a.scale, dq[i][2] * a.scale, dq[i][3] * a.scale);
}

template <int D, bool SPLIT>
__device__ __forceinline__ void dkdv_f32(const PackedArgs& a, int block, float* smem) {
  constexpr int KEYS = SPLIT ? 16 : 64, NKC = D / 16, LANES = SPLIT ? 64 : 256;
  using W = WalkF32<D, LANES>;
  auto sq = (float(*)[W::NROW * W::LD])smem, sd = (float(*)[W::NROW * W::LD])(smem + WALK_LDS<D, SPLIT>);
  const int g = block % a.Hkv;
  int seq, kt;
  PackedSeq ps;
  if (!find_key_tile<KEYS>(a, block, a.shares, seq, kt, ps)) return;
  const int share = block / a.Hkv % a.shares;
  const int m = ps.m, n = ps.n;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
  const int64_t q0 = ps.q0, k0 = ps.k0;
  const int key = kt * KEYS + (SPLIT ? 0 : wave * 16) + l16;
  f32x4 kf[NKC], vf[NKC];
  {
    const int64_t kr = k0 + min(key, n - 1);
    const float* krow = (const float*)a.k + kr * a.k_row + (int64_t)g * a.k_head;
    const float* vrow = (const float*)a.v + kr * a.v_row + (int64_t)g * a.v_head;
#pragma unroll
    for (int c = 0; c < NKC; c++) {
      kf[c] = *(const f32x4*)(krow + 16 * c + 4 * g4);
#pragma unroll
      for (int e = 0; e < 4; e++) kf[c][e] *= a.scale;
      vf[c] = *(const f32x4*)(vrow + 16 * c + 4 * g4);
    }
  }
  const int first = a.causal ? key - (n - m) : 0;
  const int t0 = a.causal ? min(max(kt * KEYS - (n - m), 0), m) / W::NROW : 0;
  const int per = cdiv(m, W::NROW) - t0;
  f32x4 dk[NKC], dv[NKC];
#pragma unroll
  for (int i = 0; i < NKC; i++) dk[i] = dv[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  W w;
  float2 st[4], next[4];   // of rows 4 g4 + r
  // step i of all heads' tiles in turn: head i / per, tile t0 + i % per
  auto fetch = [&](int i) {
    const int h = i / per, t = t0 + i - h * per;
    const int64_t head = (int64_t)g * a.G + h, at = q0 + t * W::NROW;
    w.fetch((const float*)a.q + at * a.q_row + head * a.q_head, a.q_row,
            (const float*)a.d_o + at * a.o_row + head * a.o_head, a.o_row, m - t * W::NROW);
#pragma unroll
    for (int r = 0; r < 4; r++) next[r] = stats_of(a, q0 + min(t * W::NROW + 4 * g4 + r, m - 1), head);
  };
  const int begin = share_begin(per * a.G, share, a.shares) + (SPLIT ? wave : 0), end = share_begin(per * a.G, share + 1, a.shares);
  const int step = SPLIT ? 4 : 1;
  auto buf_of = [&](int i) { return SPLIT ? wave : i & 1; };
  if (begin < end) {
    fetch(begin);
    w.stage(sq[buf_of(begin)], sd[buf_of(begin)]);
    if (SPLIT) wave_fence();
  }
  for (int i = begin; i < end; i += step) {
    const int buf = buf_of(i), t = t0 + i % per;
    if (!SPLIT) __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; r++) st[r] = next[r];
    if (i + step < end) fetch(i + step);
    f32x4 s = W::dot(sq[buf], kf, l16, g4), dp = W::dot(sd[buf], vf, l16, g4);
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int tok = t * W::NROW + 4 * g4 + r;
      const bool hidden = tok >= m || tok < first;
      s[r] = hidden ? 0.f : p_f32(s[r], st[r].x);
      dp[r] = hidden ? 0.f : s[r] * (dp[r] - st[r].y);
    }
    W::add(dv, sd[buf], s, l16, g4);
    W::add(dk, sq[buf], dp, l16, g4);
    if (SPLIT) wave_fence();
    if (i + step < end) w.stage(sq[buf_of(i + step)], sd[buf_of(i + step)]);
    if (SPLIT) wave_fence();
  }
  if (SPLIT) {
    join_waves<D>(sq[0], dk, wave, l16, g4);
    join_waves<D>(sq[0], dv, wave, l16, g4);
    if (wave > 0) return;
  }
  if (key >= n) return;
  float* ok = (float*)a.dk + (k0 + key) * a.k_row + (int64_t)g * a.k_head;
  float* ov = (float*)a.dv + (k0 + key) * a.v_row + (int64_t)g * a.v_head;
  float f = a.scale;
  if (a.shares > 1) {
    ok = share_row(a, D, share, k0 + key, g);
    ov = ok + D;
    f = 1.f;
  }
#pragma unroll
  for (int i = 0; i < NKC; i++) {
    *(float4*)(ok + 16 * i + 4 * g4) = make_float4(dk[i][0] * f, dk[i][1] * f, dk[i][2] * f, dk[i][3] * f);
    *(float4*)(ov + 16 * i + 4 * g4) = make_float4(dv[i][0], dv[i][1], dv[i][2], dv[i][3]);
  }
}

template <int D, bool SPLIT>
__global__ void __launch_bounds__(256) packed_gradients_f32(PackedArgs a, int key_blocks) {
  __shared__ __attribute__((aligned(16))) float smem[2 * WALK_LDS<D, SPLIT>];
  if ((int)blockIdx.x < key_blocks) dkdv_f32<D, SPLIT>(a, blockIdx.x, smem);
  else dq_f32<D, SPLIT>(a, blockIdx.x - key_blocks, smem);
}

// dk and dv of a key from its shares, in their order. Workgroup: 64 keys of one key/value head.
template <typename T, int D>
__global__ void __launch_bounds__(256) shares_join(PackedArgs a) {
  constexpr int KEYS = 64, LPR = D / 4;
  const int g = blockIdx.x % a.Hkv;
  int seq, kt;
  PackedSeq ps;
  if (!find_key_tile<KEYS>(a, blockIdx.x, 1, seq, kt, ps)) return;
  const int n = ps.n, e = 4 * (threadIdx.x % LPR);
  const int64_t k0 = ps.k0;
  for (int r = threadIdx.x / LPR; r < KEYS && kt * KEYS + r < n; r += 256 / LPR) {
    const int64_t key = k0 + kt * KEYS + r;
    float k[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < a.shares; i++) {
      const float* p = share_row(a, D, i, key, g) + e;
      const float4 x = *(const float4*)p, y = *(const float4*)(p + D);
      k[0] += x.x; k[1] += x.y; k[2] += x.z; k[3] += x.w;
      v[0] += y.x; v[1] += y.y; v[2] += y.z; v[3] += y.w;
    }
#pragma unroll
    for (int j = 0; j < 4; j++) k[j] *= a.scale;
    store4<T>((T*)a.dk + key * a.k_row + (int64_t)g * a.k_head + e, k);
    store4<T>((T*)a.dv + key * a.v_row + (int64_t)g * a.v_head + e, v);
  }
}

size_t stats_bytes(int H, int total_q) { return ((size_t)total_q * H * 8 + 255) & ~(size_t)255; }

int64_t tiles_of(int nseq, int64_t rows, int64_t most, int tile) {   // of the sequences of a packed tensor, at most
  return std::min<int64_t>(rows / tile + nseq, (int64_t)nseq * ((most + tile - 1) / tile));
}
// Keys and query rows of a workgroup; fp32: 16, whose walk its waves split, where tiles of 64 would be fewer than four workgroups per CU
// (64 dims) or two (128 dims, where the split form's registers leave one workgroup per CU). All gradients, causal, us as tiles of 16 / 64:
//   64 dims     4 x 200 tokens, 4 heads (128 tiles of 64) 20 / 34;  4 x 300, 16 heads (704) 65 / 74;  8 x 300, 12 heads (1080) 96 / 84
//   128 dims    4 x 200 tokens, 4 heads (128) 32 / 55;  4 x 300, 16 heads (704) 157 / 113
int grad_tile(int dtype, int nseq, int H, int Hkv, int d, int total_q, int total_k) {
  if (dtype == DT_BF16) return 128;
  const int64_t rows = (int64_t)total_q * (H / Hkv);
  return (tiles_of(nseq, total_k, total_k, 64) + tiles_of(nseq, rows, rows, 64)) * Hkv < (d == 64 ? 1024 : 512) ? 16 : 64;
}

// Into how many workgroups the rows that a key tile walks are shared out. A share costs a write and a read of its fp32 sums.
//   fewer key tiles than CUs      as many as fill two workgroups per CU, of 512 rows at least (all gradients, us with 256 / 512 / 1024
//                                 at least: 1024 causal tokens of 16 over 4 heads 85 / 73 / 76, 4 x 512 66 / 59 / 74, 1000 of 2 over 1
//                                 50 / 51 / 95)
//   causal, few tiles             two: the tiles' work falls from all rows to none, and the longest ones run alone at the end unless the
//                                 workgroups of dq, or a second round of tiles, are enough to fill the chip meanwhile. All gradients of
//                                 128 dims, us in two shares / one: 256 tiles of 8192 rows 307 / 433; 512 tiles of 4096 rows 404 / 355,
//                                 of 8192 632 / 596, of 16384 1008 / 1047, of 32768 1821 / 1992; 768 of 16384 1518 / 1477
int shares_of(int dtype, int nseq, int H, int Hkv, int d, int total_q, int total_k, int causal) {
  const int64_t units = ((int64_t)total_k / grad_tile(dtype, nseq, H, Hkv, d, total_q, total_k) + nseq) * Hkv, rows = (int64_t)total_q * (H / Hkv) / nseq;
  if (units < 256) return (int)std::max<int64_t>(1, std::min<int64_t>(512 / units, rows / 512));
  return causal && dtype == DT_BF16 && (units < 400 ? rows >= 4096 : units < 600 && rows >= 16384) ? 2 : 1;   // (units count one more tile a sequence)
}

}  // namespace

// what is known of each row; the shares of dk and dv
size_t packed_backward_ws(int dtype, int nseq, int H, int Hkv, int d, int total_q, int total_k, int causal) {
  if (nseq == 0) return 0;
  const int shares = shares_of(dtype, nseq, H, Hkv, d, total_q, total_k, causal);
  return stats_bytes(H, total_q) + (shares > 1 ? (size_t)shares * total_k * Hkv * 2 * d * 4 : 0);
}

// Workgroups of a call's launches.
struct BackwardGroups {
  int tile, shares;
  int64_t stats, keys, rows, joins;   // (those of keys and rows are in one launch)
};
static BackwardGroups groups_of(const PackedArgs& a, int dtype, int d) {
  const int total_q = a.qr.total, total_k = a.kr.total;
  BackwardGroups g{};
  g.tile = grad_tile(dtype, a.nseq, a.H, a.Hkv, d, total_q, total_k);
  g.shares = shares_of(dtype, a.nseq, a.H, a.Hkv, d, total_q, total_k, a.causal);
  g.stats = ((int64_t)total_q * a.H * (d * (dtype == DT_BF16 ? 2 : 4) / 16) + 255) / 256;
  g.keys = total_k > 0 ? tiles_of(a.nseq, total_k, total_k, g.tile) * a.Hkv * g.shares : 0;
  g.rows = tiles_of(a.nseq, (int64_t)total_q * a.G, (int64_t)a.max_q * a.G, g.tile) * a.Hkv;
  g.joins = g.shares > 1 && total_k > 0 ? ((int64_t)total_k / 64 + a.nseq) * a.Hkv : 0;
  return g;
}
int64_t packed_backward_threads(const PackedArgs& a, int dtype, int d) {
  const BackwardGroups g = groups_of(a, dtype, d);
  return 256 * std::max({g.stats, g.keys + g.rows, g.joins});
}

hipError_t packed_attention_stats(PackedArgs a, int dtype, int d, void* ws, hipStream_t s) {
  a.stats = (float2*)ws;
  const int64_t grid = groups_of(a, dtype, d).stats;
  if (grid == 0) return hipSuccess;
  if (dtype == DT_BF16 && d == 128) stats_kernel<u16, 128><<<grid, 256, 0, s>>>(a);
  else if (dtype == DT_BF16) stats_kernel<u16, 64><<<grid, 256, 0, s>>>(a);
  else if (d == 128) stats_kernel<float, 128><<<grid, 256, 0, s>>>(a);
  else stats_kernel<float, 64><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

template <int D>
static void gradients_launch(const PackedArgs& a, int dtype, int tile, int key_blocks, int64_t blocks, int64_t joins, hipStream_t s) {
  if (dtype == DT_BF16) packed_gradients_bf16<D><<<blocks, 256, 0, s>>>(a, key_blocks);
  else if (tile == 16) packed_gradients_f32<D, true><<<blocks, 256, 0, s>>>(a, key_blocks);
  else packed_gradients_f32<D, false><<<blocks, 256, 0, s>>>(a, key_blocks);
  if (joins == 0) return;
  if (dtype == DT_BF16) shares_join<u16, D><<<joins, 256, 0, s>>>(a);
  else shares_join<float, D><<<joins, 256, 0, s>>>(a);
}
hipError_t packed_attention_gradients(PackedArgs a, int dtype, int d, void* ws, hipStream_t s) {
  const BackwardGroups g = groups_of(a, dtype, d);
  a.stats = (float2*)ws;
  a.shares = g.shares;
  a.share_sums = (float*)((char*)ws + stats_bytes(a.H, a.qr.total));
  if (g.keys + g.rows == 0) return hipSuccess;
  if (d == 128) gradients_launch<128>(a, dtype, g.tile, (int)g.keys, g.keys + g.rows, g.joins, s);
  else gradients_launch<64>(a, dtype, g.tile, (int)g.keys, g.keys + g.rows, g.joins, s);
  return hipGetLastError();
}

}  // namespace dit
