// Attention over packed sequences on gfx950: o = softmax(scale q k^T) v per sequence, with grouped heads and an
// optional causal mask (the last query of a sequence sees its last key).
//
// Rows. The G = heads / kv_heads query heads that share a key/value head are rows of one problem: row r of a
// sequence of m queries is query r / G, head r % G of the group, r < m G. Keys and values are then read once per
// tile of rows for the whole group, one new token of G heads is a tile of G rows, and a causal tile of R rows
// spans only R / G diagonal positions.
//
// bf16: flash-style with v_mfma_f32_32x32x16_bf16, 4 waves of 32 rows, 64-key tiles of K and V in two LDS buffers
// each. Scores are computed transposed (S^T = K Q^T), so that a lane owns one row and its probabilities are
// operand B of O^T = V^T P^T as they stand; the exponentials of tile t share one instruction stream with the score
// MFMAs of tile t + 1. Probabilities are rounded to bf16 for the second product, by up to 2^-8 of each, because that is what the
// matrix instruction takes at its full rate; sums and maxima stay fp32. o averages over the keys and its error with it, so the error is
// of the size of o's own rounding: in the 2-norm o is off by 0.0019 to 0.0024 of itself, by 0.0016 to 0.0017 were only o rounded.
// Bound by the matrix instructions and the exponentials between them (8 samples of 1101 to 2560 tokens, 24 heads of 128, no mask:
// 372 to 403 us from card to card, 910 to 980 TFLOP/s, where a large library product runs at 1160 to 1230); few rows, below, by reading the keys once.
#include <algorithm>

#include "attn_common.h"
#include "packed.h"

namespace dit {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float M_FLOOR = -3.4028235e38f;   // running maximum of a row that has seen no key: finite, and no finite score is below it

// Whether a query sees any key: o of one that does not is 0 and its lse -inf, whatever its sum is (one whose scores are all -inf
// has a sum of 0 too).
__device__ __forceinline__ bool sees_keys(const PackedArgs& a, const PackedSeq& s, int tok) {
  return s.n > 0 && (!a.causal || tok + s.n - s.m >= 0);
}

// What a workgroup works on: rows [ROWS rt, ...) of a sequence, key/value head g, part `part` of its keys.
struct PackedTile {
  PackedSeq s;
  int g, rt, part, parts;
  int seq, local;   // which sequence's, and which of its (row tile, part)
  bool any;
};
__device__ __forceinline__ int parts_of(const PackedArgs& a, const PackedSeq& s) {
  return a.part_tiles ? max(cdiv(cdiv(s.n, 64), a.part_tiles), 1) : 1;
}
template <int ROWS> __device__ __forceinline__ int row_tiles_of(const PackedArgs& a, const PackedSeq& s) {
  return (s.m * a.G + ROWS - 1) / ROWS;
}
template <int ROWS>
__device__ __forceinline__ PackedTile packed_tile(const PackedArgs& a) {
  PackedTile t{};
  const int u = blockIdx.x / a.Hkv;
  t.g = blockIdx.x - u * a.Hkv;
  t.any = find_unit(a.nseq, u, [&](int i) { return a.sequence(i); },
                    [&](const PackedSeq& s) { return row_tiles_of<ROWS>(a, s) * parts_of(a, s); }, t.seq, t.local, t.s);
  if (!t.any) return t;
  t.parts = parts_of(a, t.s);
  t.rt = t.local / t.parts;
  t.part = t.local - t.rt * t.parts;
  if (a.causal) t.rt = row_tiles_of<ROWS>(a, t.s) - 1 - t.rt;   // the rows that see most keys first
  return t;
}

// Where partial results are kept: those of one head lie together, in the order of the sequences that have any. -1: there is no place for
// `count` of them from the sequence's local-th on (offsets that are not increasing). All lanes of a wave call it.
template <int ROWS> __device__ __forceinline__ int64_t partial_slot(const PackedArgs& a, int g, int seq, int local, int count) {
  unsigned before = 0;   // (offsets that are not increasing may wrap it: a place all the same)
  for (int base = 0; base < seq; base += 64) {
    const int i = base + (threadIdx.x & 63);
    const PackedSeq s = a.sequence(min(i, seq));
    const int parts = parts_of(a, s);
    before += i < seq && parts > 1 ? row_tiles_of<ROWS>(a, s) * parts : 0;
  }
  const int64_t first = (int64_t)(unsigned)__builtin_amdgcn_readlane(seq ? wave_scan(before) : 0, 63) + local;
  return first + count > a.slots ? -1 : (int64_t)g * a.slots + first;
}

template <int D, bool PARTS>
__global__ void __launch_bounds__(256, 2) packed_fwd_bf16(PackedArgs a) {
  constexpr int ROWS = 128, KB = 64, NDB = D / 32, NKS = D / 16;
  constexpr float TAU = 8.f;           // lazy-rescale threshold (log2 units)
  using Tile = RowTile<D, KB, 4>;
  constexpr int CH = Tile::CH, RB = Tile::RB, TILE = Tile::BYTES;
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[4 * TILE];   // [K0][K1][V0][V1]
  const PackedTile t = packed_tile<ROWS>(a);
  if (!t.any) return;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int half = lane >> 5, l32 = lane & 31;
  const int rows = t.s.m * a.G, row0 = t.rt * ROWS;
  const int q0 = t.s.q0;
  const int64_t k0 = t.s.k0;
  const u16* Kg = (const u16*)a.k + k0 * a.k_row + (int64_t)t.g * a.k_head;
  const u16* Vg = (const u16*)a.v + k0 * a.v_row + (int64_t)t.g * a.v_head;

  // this lane's row and its Q fragments: q[row][16 s + 8 half + 0..7]; vis keys are visible to it
  const int row = min(row0 + wave * 32 + l32, rows - 1);
  const int tok = row / a.G, head = t.g * a.G + (row - tok * a.G);
  const int vis = a.causal ? min(tok + t.s.n - t.s.m + 1, t.s.n) : t.s.n;
  bf16x8 qf[NKS];
  {
    const u16* qrow = (const u16*)a.q + (int64_t)(q0 + tok) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
    for (int s = 0; s < NKS; s++) qf[s] = *(const bf16x8*)(qrow + 16 * s + 8 * half);
  }
  // keys the tile needs: those of its last row; keys every row of this wave sees: those of its first
  const int last_tok = (min(row0 + ROWS, rows) - 1) / a.G;
  const int nvis = a.causal ? min(max(last_tok + t.s.n - t.s.m + 1, 0), t.s.n) : t.s.n;
  const int all_vis = __builtin_amdgcn_readfirstlane(vis);
  int kt0 = 0, nt = cdiv(nvis, KB);
  if (PARTS) {
    kt0 = min(t.part * a.part_tiles, nt);
    nt = min(kt0 + a.part_tiles, nt);
  }

  Tile tk, tv;
  tk.init(wave, lane, a.k_row);
  tv.init(wave, lane, a.v_row);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem;
  auto issue_k = [&](int kt) { tk.load(Kg + (int64_t)kt * KB * a.k_row, t.s.n - kt * KB, lds0 + (kt & 1) * TILE); };
  auto issue_v = [&](int kt) { tv.load(Vg + (int64_t)kt * KB * a.v_row, t.s.n - kt * KB, lds0 + (2 + (kt & 1)) * TILE); };

  // V^T fragment quarters: this lane points at 4 dims of key 4 half + (lane >> 2) % 4 of a step
  const int vkey = 4 * half + ((lane >> 2) & 3);
  int vbase[NDB][2];
#pragma unroll
  for (int db = 0; db < NDB; db++) {
    const int ch = 4 * db + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
#pragma unroll
    for (int e = 0; e < 2; e++)   // (the swizzle has period 16, a step's keys)
      vbase[db][e] = (vkey + 8 * e) * RB + ((ch ^ tile_swizzle<D>(vkey + 8 * e)) << 4) + 8 * (lane & 1);
  }

  f32x16 o[NDB];
#pragma unroll
  for (int i = 0; i < NDB; i++)
#pragma unroll
    for (int r = 0; r < 16; r++) o[i][r] = 0.f;
  const f32x16 zero = {};
  const float c = a.scale * LOG2E;
  // p = exp2(c_row s - m_run) in one operation. The rounding of m_run = c_row max s leaves the same factor for every key of the row, which
  // cancels, as long as it is a number: up to |m_run| = FAR it is within 2^32. Scores past that are at least 2^4 apart in log2
  // units where they differ at all, so any steeper or flatter exponential tells the largest from the others as well: c_row
  // becomes the power of two that brings the maximum to 2^28, where neither product rounds.
  constexpr float FAR = 536870912.f;   // 2^29
  float c_row = c, m_run = M_FLOOR, l_run = 0.f;

  auto scores = [&](int kt, f32x16* sn) {
    const char* sk = smem + (kt & 1) * TILE;
    constexpr int NS = NKS / 4;
#pragma unroll
    for (int g = 0; g < 4; g++) {
      bf16x8 kf[NS][KB / 32];
#pragma unroll
      for (int s = 0; s < NS; s++)
#pragma unroll
        for (int kb = 0; kb < KB / 32; kb++) kf[s][kb] = Tile::read(sk, 32 * kb + l32, 2 * (g * NS + s) + half);
#pragma unroll
      for (int s = 0; s < NS; s++)
#pragma unroll
        for (int kb = 0; kb < KB / 32; kb++) {
          const int sg = g * NS + s;
          sn[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s][kb], qf[sg], sg == 0 ? zero : sn[kb], 0, 0, 0);
        }
    }
  };
  // hidden keys score -inf; returns this lane's max
  auto mask_max = [&](int kt, f32x16* sn) {
    if ((kt + 1) * KB > all_vis) {
#pragma unroll
      for (int kb = 0; kb < KB / 32; kb++)
#pragma unroll
        for (int r = 0; r < 16; r++) {
          const int key = kt * KB + 32 * kb + 8 * (r >> 2) + 4 * half + (r & 3);
          if (key >= vis) sn[kb][r] = -INFINITY;
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < KB / 32; kb++)
#pragma unroll
      for (int r = 0; r < 16; r++) mx = fmaxf(mx, sn[kb][r]);
    return mx;
  };
  auto step = [&](int kt, f32x16* st, float& mx, f32x16* sn, float& mxn, auto next_c) {
    constexpr bool NEXT = decltype(next_c)::value;
    // every wave is done with K buffer kt&1 and V buffer (kt+1)&1; the loads of the buffers read below have landed
    __syncthreads();
    if (kt + 2 < nt) issue_k(kt + 2);
    const char* sv = smem + (2 + (kt & 1)) * TILE;
    mx = pair_max(mx);
    const float mxs = mx * c_row;
    if (__ballot(mxs > m_run + TAU) != 0) {
      float m_new = fmaxf(m_run, mxs), c_new = c_row;
      if (mxs > m_run) {
        c_new = c;
        m_new = mx * c;
        if (fabsf(m_new) > FAR) {
          c_new = __uint_as_float(((127 + 28 + 127) << 23) - (__float_as_uint(mx) & 0x7f800000u));
          m_new = mx * c_new;
        }
      }
      const float alpha = c_new == c_row ? __builtin_amdgcn_exp2f(m_run - m_new) : 0.f;
      m_run = m_new;
      c_row = c_new;
      l_run *= alpha;
#pragma unroll
      for (int i = 0; i < NDB; i++)
#pragma unroll
        for (int r = 0; r < 16; r++) o[i][r] *= alpha;
    }
    float psum = 0.f;
    bf16x8 pf[KB / 32][2];
#pragma unroll
    for (int kb = 0; kb < KB / 32; kb++)
#pragma unroll
      for (int h = 0; h < 2; h++)
#pragma unroll
        for (int j = 0; j < 8; j++) {
          const float p = __builtin_amdgcn_exp2f(fmaf(st[kb][8 * h + j], c_row, -m_run));
          psum += p;
          pf[kb][h][j] = (__bf16)p;
        }
    if constexpr (NEXT) scores(kt + 1, sn);
    l_run += psum;
    if (NEXT) issue_v(kt + 1);
    // keys 16 q + {4 half + 0..3, 8 + 4 half + 0..3}: the order of the score accumulator
#pragma unroll
    for (int q = 0; q < KB / 16; q++) {
      bf16x8 vf[NDB];
#pragma unroll
      for (int db = 0; db < NDB; db++)
        vf[db] = join_tr(read_tr(sv + 16 * q * RB + vbase[db][0]), read_tr(sv + 16 * q * RB + vbase[db][1]));
#pragma unroll
      for (int db = 0; db < NDB; db++)
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[db], pf[q >> 1][q & 1], o[db], 0, 0, 0);
    }
    if constexpr (NEXT) mxn = mask_max(kt + 1, sn);
    __builtin_amdgcn_s_waitcnt(0);
  };

  if (kt0 < nt) {
    issue_k(kt0);
    issue_v(kt0);
    if (kt0 + 1 < nt) issue_k(kt0 + 1);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    f32x16 sa[KB / 32], sb[KB / 32];
    float ma, mb = -INFINITY;
    scores(kt0, sa);
    ma = mask_max(kt0, sa);
    int kt = kt0;
    for (; kt + 2 < nt; kt += 2) {
      step(kt, sa, ma, sb, mb, std::true_type());
      step(kt + 1, sb, mb, sa, ma, std::true_type());
    }
    if (kt + 1 < nt) {
      step(kt, sa, ma, sb, mb, std::true_type());
      step(kt + 1, sb, mb, sa, ma, std::false_type());
    } else {
      step(kt, sa, ma, sb, mb, std::false_type());
    }
  }

  const float l_all = pair_sum(l_run);
  const bool real = row0 + wave * 32 + l32 < rows;
  if (PARTS && t.parts > 1) {
    const int64_t place = partial_slot<ROWS>(a, t.g, t.seq, t.local, 1), slot = place * ROWS + wave * 32 + l32;
    if (place < 0) return;
    // the maximum in units of the scores, and what its rounding changes
    const float m = m_run == M_FLOOR ? M_FLOOR : m_run / c_row;
    const float f = m_run == M_FLOOR ? 1.f : __builtin_amdgcn_exp2f(fmaf(-m, c_row, m_run));
    if (real) {
      if (half == 0) a.part_ml[slot] = make_float2(m, l_all * f);
      float* po = a.part_o + slot * D;
#pragma unroll
      for (int db = 0; db < NDB; db++)
#pragma unroll
        for (int g = 0; g < 4; g++)
          *(float4*)(po + 32 * db + 8 * g + 4 * half) = make_float4(o[db][4 * g] * f, o[db][4 * g + 1] * f, o[db][4 * g + 2] * f, o[db][4 * g + 3] * f);
    }
    return;
  }
  const bool sees = vis > 0;
  if (__ballot(!sees) != 0) {   // nothing of a value that is no number (0 times it is none either)
#pragma unroll
    for (int i = 0; i < NDB; i++)
      if (!sees) o[i] = zero;
  }
  const float inv = sees ? 1.0f / l_all : 0.f, log2_l = __builtin_amdgcn_logf(l_all);
  const float lse = !sees ? -INFINITY : c_row == c ? (m_run + log2_l) * LN2 : m_run * __builtin_amdgcn_rcpf(c_row) * a.scale;
  if (a.lse && real && half == 0) a.lse[(int64_t)(q0 + tok) * a.H + head] = lse;
  // The output leaves through the 32 rows of the K buffers that belong to this wave, so that a store writes whole
  // rows. (Both K buffers were last read before the last step's barrier.)
  {
    char* so = smem + wave * 32 * RB;
#pragma unroll
    for (int db = 0; db < NDB; db++)
#pragma unroll
      for (int g = 0; g < 4; g++) {
        const int ch = 4 * db + g;
        uint2 u;
        u.x = pack_bf16x2(o[db][4 * g] * inv, o[db][4 * g + 1] * inv);
        u.y = pack_bf16x2(o[db][4 * g + 2] * inv, o[db][4 * g + 3] * inv);
        *(uint2*)(so + l32 * RB + ((ch ^ (l32 % CH)) << 4) + 8 * half) = u;
      }
    wave_fence();
    constexpr int RPI = 64 / CH;
#pragma unroll
    for (int i = 0; i < 32 / RPI; i++) {
      const int r = i * RPI + lane / CH, ch = lane % CH;
      const uint4 v = *(const uint4*)(so + r * RB + ((ch ^ (r % CH)) << 4));
      const int rr = row0 + wave * 32 + r;
      if (rr < rows) {
        const int tk_ = rr / a.G, hd = t.g * a.G + (rr - tk_ * a.G);
        *(uint4*)((u16*)a.o + (int64_t)(q0 + tk_) * a.o_row + (int64_t)hd * a.o_head + 8 * ch) = v;
      }
    }
  }
#endif
}

// ---------------------------------------------------------------------------
// fp32 on v_mfma_f32_16x16x4_f32 (fp32 operands, products and sums): 4 waves of 16 rows share K/V tiles of 32 keys (16
// at D = 128), staged through registers one tile ahead; the same transposed orientation, one rescale per tile.
// ---------------------------------------------------------------------------
template <int D>
__global__ void __launch_bounds__(256, 2) packed_fwd_f32(PackedArgs a) {
  constexpr int ROWS = 64, KB = D == 64 ? 32 : 16, NKB = KB / 16, LD = D + 4, NDB = D / 16, NKC = D / 16;
  constexpr int CPT = KB * D / 4 / 256;   // 16-byte chunks of K (and of V) each thread stages per tile
  __shared__ __attribute__((aligned(16))) float sk[2][KB * LD];
  __shared__ __attribute__((aligned(16))) float sv[2][KB * LD];
  const PackedTile t = packed_tile<ROWS>(a);
  if (!t.any) return;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int l16 = lane & 15, g4 = lane >> 4;
  const int rows = t.s.m * a.G, row0 = t.rt * ROWS;
  const int q0 = t.s.q0;
  const int64_t k0 = t.s.k0;
  const float* Kg = (const float*)a.k + k0 * a.k_row + (int64_t)t.g * a.k_head;
  const float* Vg = (const float*)a.v + k0 * a.v_row + (int64_t)t.g * a.v_head;
  const int row = min(row0 + wave * 16 + l16, rows - 1);
  const int tok = row / a.G, head = t.g * a.G + (row - tok * a.G);
  const int vis = a.causal ? min(tok + t.s.n - t.s.m + 1, t.s.n) : t.s.n;
  f32x4 qf[NKC];   // scaled before the products, which may overflow without
  {
    const float* qrow = (const float*)a.q + (int64_t)(q0 + tok) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
    for (int c = 0; c < NKC; c++) {
      qf[c] = *(const f32x4*)(qrow + 16 * c + 4 * g4);
#pragma unroll
      for (int e = 0; e < 4; e++) qf[c][e] *= a.scale;
    }
  }
  const int last_tok = (min(row0 + ROWS, rows) - 1) / a.G;
  const int nvis = a.causal ? min(max(last_tok + t.s.n - t.s.m + 1, 0), t.s.n) : t.s.n;
  const int nt = cdiv(nvis, KB);
  f32x4 rk[CPT], rv[CPT];
  // rows past the end repeat the last key, whose scores are masked there, with a value of zero
  auto fetch = [&](int kt) {
#pragma unroll
    for (int i = 0; i < CPT; i++) {
      const int idx = tid + 256 * i, r = min(kt * KB + idx / (D / 4), t.s.n - 1), c = idx % (D / 4);
      rk[i] = *(const f32x4*)(Kg + r * a.k_row + 4 * c);
      rv[i] = *(const f32x4*)(Vg + r * a.v_row + 4 * c);
    }
  };
  auto stage = [&](int kt) {
    const int buf = kt & 1;
#pragma unroll
    for (int i = 0; i < CPT; i++) {
      const int idx = tid + 256 * i, r = idx / (D / 4), c = idx % (D / 4);
      *(f32x4*)(&sk[buf][r * LD + 4 * c]) = rk[i];
      *(f32x4*)(&sv[buf][r * LD + 4 * c]) = kt * KB + r < t.s.n ? rv[i] : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  f32x4 o[NDB];
#pragma unroll
  for (int i = 0; i < NDB; i++) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = M_FLOOR, l_run = 0.f;
  if (nt > 0) {
    fetch(0);
    stage(0);
  }
  for (int kt = 0; kt < nt; kt++) {
    const int buf = kt & 1;
    __syncthreads();   // tile kt is staged, and every wave is done with the other buffer
    if (kt + 1 < nt) fetch(kt + 1);
    f32x4 s[NKB];
    {
      f32x4 kf[NKB][NKC];
#pragma unroll
      for (int kb = 0; kb < NKB; kb++)
#pragma unroll
        for (int c = 0; c < NKC; c++) kf[kb][c] = *(const f32x4*)(&sk[buf][(16 * kb + l16) * LD + 16 * c + 4 * g4]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kb = 0; kb < NKB; kb++) s[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NKC; c++)
#pragma unroll
        for (int e = 0; e < 4; e++)
#pragma unroll
          for (int kb = 0; kb < NKB; kb++)
            s[kb] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[kb][c][e], qf[c][e], s[kb], 0, 0, 0);
    }
    float vf[NKB][4][NDB];
#pragma unroll
    for (int kb = 0; kb < NKB; kb++)
#pragma unroll
      for (int r = 0; r < 4; r++)
#pragma unroll
        for (int i = 0; i < NDB; i++) vf[kb][r][i] = sv[buf][(16 * kb + 4 * g4 + r) * LD + l16 + 16 * i];
    __builtin_amdgcn_sched_barrier(0);
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < NKB; kb++)
#pragma unroll
      for (int r = 0; r < 4; r++) {
        if (kt * KB + 16 * kb + 4 * g4 + r >= vis) s[kb][r] = -INFINITY;
        mx = fmaxf(mx, s[kb][r]);
      }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_new = fmaxf(m_run, mx);
    const float alpha = __builtin_amdgcn_exp2f((m_run - m_new) * LOG2E);
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int i = 0; i < NDB; i++)
#pragma unroll
      for (int r = 0; r < 4; r++) o[i][r] *= alpha;
    float psum = 0.f;
#pragma unroll
    for (int kb = 0; kb < NKB; kb++)
#pragma unroll
      for (int r = 0; r < 4; r++) {
        s[kb][r] = __builtin_amdgcn_exp2f((s[kb][r] - m_new) * LOG2E);
        psum += s[kb][r];
      }
    l_run += psum;
#pragma unroll
    for (int kb = 0; kb < NKB; kb++)
#pragma unroll
      for (int r = 0; r < 4; r++)
#pragma unroll
        for (int i = 0; i < NDB; i++) o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[kb][r][i], s[kb][r], o[i], 0, 0, 0);
    if (kt + 1 < nt) stage(kt + 1);
  }
  l_run += __shfl_xor(l_run, 16, 64);
  l_run += __shfl_xor(l_run, 32, 64);
  if (row0 + wave * 16 + l16 >= rows) return;
  const bool sees = vis > 0;
  const float inv = sees ? 1.0f / l_run : 0.f;
  if (!sees)   // nothing of a value that is no number
#pragma unroll
    for (int i = 0; i < NDB; i++) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float lse = sees ? m_run + __builtin_amdgcn_logf(l_run) * LN2 : -INFINITY;
  float* orow = (float*)a.o + (int64_t)(q0 + tok) * a.o_row + (int64_t)head * a.o_head;
  float* olse = a.lse ? a.lse + (int64_t)(q0 + tok) * a.H + head : nullptr;
  if (olse && g4 == 0) *olse = lse;
#pragma unroll
  for (int i = 0; i < NDB; i++)   // dims 16 i + 4 g4 + 0..3 of this lane's row
    *(float4*)(orow + 16 * i + 4 * g4) = make_float4(o[i][0] * inv, o[i][1] * inv, o[i][2] * inv, o[i][3] * inv);
}

// ---------------------------------------------------------------------------
// fp32 where tiles of 64 rows would be few: 16 rows per workgroup, whose 4 waves take every fourth 16-key tile, each staging its
// own, with a running maximum and sum of their own; they meet at the end.
// ---------------------------------------------------------------------------
template <int D>
__global__ void __launch_bounds__(256) packed_split_f32(PackedArgs a) {
  constexpr int ROWS = 16, NKC = D / 16;
  using W = WalkF32<D, 64>;
  __shared__ __attribute__((aligned(16))) float sk[4][W::NROW * W::LD], sv[4][W::NROW * W::LD];
  __shared__ float2 ml[4][ROWS];
  const PackedTile t = packed_tile<ROWS>(a);
  if (!t.any) return;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
  const int rows = t.s.m * a.G, row0 = t.rt * ROWS, n = t.s.n;
  const int64_t q0 = t.s.q0, k0 = t.s.k0;
  const float* Kg = (const float*)a.k + k0 * a.k_row + (int64_t)t.g * a.k_head;
  const float* Vg = (const float*)a.v + k0 * a.v_row + (int64_t)t.g * a.v_head;
  const int row = min(row0 + l16, rows - 1);
  const int tok = row / a.G, head = t.g * a.G + (row - tok * a.G);
  const int vis = a.causal ? min(tok + n - t.s.m + 1, n) : n;
  const int last_tok = (min(row0 + ROWS, rows) - 1) / a.G;
  const int nvis = a.causal ? min(max(last_tok + n - t.s.m + 1, 0), n) : n;
  int kt0 = 0, nt = cdiv(nvis, 16);
  if (a.part_tiles) {
    kt0 = min(t.part * a.part_tiles * 4, nt);
    nt = min(kt0 + a.part_tiles * 4, nt);
  }
  f32x4 qf[NKC];   // scaled before the products, which may overflow without
  {
    const float* qrow = (const float*)a.q + (q0 + tok) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
    for (int c = 0; c < NKC; c++) {
      qf[c] = *(const f32x4*)(qrow + 16 * c + 4 * g4);
#pragma unroll
      for (int e = 0; e < 4; e++) qf[c][e] *= a.scale;
    }
  }
  W w;
  auto fetch = [&](int kt) { w.fetch(Kg + (int64_t)kt * 16 * a.k_row, a.k_row, Vg + (int64_t)kt * 16 * a.v_row, a.v_row, n - kt * 16); };
  f32x4 o[NKC];
#pragma unroll
  for (int i = 0; i < NKC; i++) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = M_FLOOR, l_run = 0.f;
  if (kt0 + wave < nt) {
    fetch(kt0 + wave);
    w.stage(sk[wave], sv[wave]);
    wave_fence();
  }
  for (int kt = kt0 + wave; kt < nt; kt += 4) {
    if (kt + 4 < nt) fetch(kt + 4);
    f32x4 s = W::dot(sk[wave], qf, l16, g4);
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 4; r++) {
      if (kt * 16 + 4 * g4 + r >= vis) s[r] = -INFINITY;
      mx = fmaxf(mx, s[r]);
    }
    mx = pair_max(fmaxf(mx, __shfl_xor(mx, 16, 64)));
    const float m_new = fmaxf(m_run, mx), alpha = __builtin_amdgcn_exp2f((m_run - m_new) * LOG2E);
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int i = 0; i < NKC; i++)
#pragma unroll
      for (int r = 0; r < 4; r++) o[i][r] *= alpha;
#pragma unroll
    for (int r = 0; r < 4; r++) {
      s[r] = __builtin_amdgcn_exp2f((s[r] - m_new) * LOG2E);
      l_run += s[r];
    }
    W::add(o, sv[wave], s, l16, g4);
    wave_fence();
    if (kt + 4 < nt) w.stage(sk[wave], sv[wave]);
    wave_fence();
  }
  l_run += __shfl_xor(l_run, 16, 64);
  l_run = pair_sum(l_run);
  if (g4 == 0) ml[wave][l16] = make_float2(m_run, l_run);
  __syncthreads();
  float m = M_FLOOR, l = 0.f;
#pragma unroll
  for (int x = 0; x < 4; x++) m = fmaxf(m, ml[x][l16].x);
#pragma unroll
  for (int x = 0; x < 4; x++) l = fmaf(__builtin_amdgcn_exp2f((ml[x][l16].x - m) * LOG2E), ml[x][l16].y, l);
  const float mine = __builtin_amdgcn_exp2f((m_run - m) * LOG2E);
#pragma unroll
  for (int i = 0; i < NKC; i++) o[i] *= mine;
  join_waves<D>(sk[0], o, wave, l16, g4);
  if (wave > 0) return;
  const bool partial = a.part_tiles && t.parts > 1;
  const int64_t place = partial ? partial_slot<ROWS>(a, t.g, t.seq, t.local, 1) : 0;
  if (row0 + l16 >= rows || place < 0) return;
  const bool sees = vis > 0;
  float inv = sees ? 1.0f / l : 0.f;
  if (!sees)   // nothing of a value that is no number
#pragma unroll
    for (int i = 0; i < NKC; i++) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float* orow = (float*)a.o + (q0 + tok) * a.o_row + (int64_t)head * a.o_head;
  if (partial) {
    const int64_t slot = place * ROWS + l16;
    orow = a.part_o + slot * D;
    inv = 1.f;
    if (g4 == 0) a.part_ml[slot] = make_float2(m, l);
  } else if (a.lse && g4 == 0) {
    a.lse[(q0 + tok) * a.H + head] = sees ? m + __builtin_amdgcn_logf(l) * LN2 : -INFINITY;
  }
#pragma unroll
  for (int i = 0; i < NKC; i++)
    *(float4*)(orow + 16 * i + 4 * g4) = make_float4(o[i][0] * inv, o[i][1] * inv, o[i][2] * inv, o[i][3] * inv);
}

// ---------------------------------------------------------------------------
// bf16, few rows: a new token (or a few) of each sequence against its keys, bound by reading K and V once. Tiles of 16 rows on
// v_mfma_f32_16x16x32_bf16; the four waves of a workgroup do not share rows but keys: wave w takes the 32-key stages w, w + 4, ...
// of the part with a running maximum, sum and output of its own, so no barrier stands in the loop, and they meet at
// the end. K goes to registers (a lane's 16 bytes are operand A as they stand), V straight to LDS for the
// transposing read; both one stage ahead, 16 KB per wave in flight.
// ---------------------------------------------------------------------------
template <int D>
__global__ void __launch_bounds__(256, 2) packed_few_bf16(PackedArgs a) {
  constexpr int NW = 4, ROWS = 16, KB = 32, NKS = D / 32, NDB = D / 16;
  using Tile = RowTile<D, KB, 1>;
  constexpr int RB = Tile::RB, TILE = Tile::BYTES;
  constexpr int MERGE = NW * ROWS * (D + 4) * 4 + NW * ROWS * 8;
  constexpr int LDS = 2 * NW * TILE > MERGE ? 2 * NW * TILE : MERGE;
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[LDS];   // per wave [V0][V1]
  const PackedTile t = packed_tile<ROWS>(a);
  if (!t.any) return;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int l16 = lane & 15, g4 = lane >> 4;
  const int rows = t.s.m * a.G, row0 = t.rt * ROWS;
  const int q0 = t.s.q0;
  const int64_t k0 = t.s.k0;
  const u16* Kg = (const u16*)a.k + k0 * a.k_row + (int64_t)t.g * a.k_head;
  const u16* Vg = (const u16*)a.v + k0 * a.v_row + (int64_t)t.g * a.v_head;
  const int row = min(row0 + l16, rows - 1);
  const int tok = row / a.G, head = t.g * a.G + (row - tok * a.G);
  const int vis = a.causal ? min(tok + t.s.n - t.s.m + 1, t.s.n) : t.s.n;
  const int last_tok = (min(row0 + ROWS, rows) - 1) / a.G;
  const int nvis = a.causal ? min(max(last_tok + t.s.n - t.s.m + 1, 0), t.s.n) : t.s.n;
  const int all_vis = __builtin_amdgcn_readfirstlane(vis);
  int begin = 0, end = nvis;
  if (a.part_tiles) {
    begin = min(t.part * a.part_tiles * 64, nvis);
    end = min(begin + a.part_tiles * 64, nvis);
  }
  bf16x8 qf[NKS];   // q[row][32 s + 8 g4 + 0..7]
  {
    const u16* qrow = (const u16*)a.q + (int64_t)(q0 + tok) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
    for (int s = 0; s < NKS; s++) qf[s] = *(const bf16x8*)(qrow + 32 * s + 8 * g4);
  }
  Tile tv;
  tv.init(0, lane, a.v_row);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem + wave * 2 * TILE;
  const char* sv0 = smem + wave * 2 * TILE;
  auto load_k = [&](int key0, bf16x8 (*kf)[2]) {
#pragma unroll
    for (int kb = 0; kb < 2; kb++) {
      const u16* krow = Kg + (int64_t)min(key0 + 16 * kb + l16, end - 1) * a.k_row + 8 * g4;
#pragma unroll
      for (int s = 0; s < NKS; s++) kf[s][kb] = *(const bf16x8*)(krow + 32 * s);
    }
  };
  auto load_v = [&](int key0, int buf) { tv.load(Vg + (int64_t)key0 * a.v_row, end - key0, lds0 + buf * TILE); };
  int vbase[NDB][2];   // 4 dims of key 4 g4 + (lane >> 2) % 4 (+ 16)
#pragma unroll
  for (int db = 0; db < NDB; db++)
#pragma unroll
    for (int e = 0; e < 2; e++) {
      const int r = 4 * g4 + ((lane >> 2) & 3) + 16 * e, ch = 2 * db + ((lane >> 1) & 1);
      vbase[db][e] = r * RB + ((ch ^ tile_swizzle<D>(r)) << 4) + 8 * (lane & 1);
    }
  f32x4 o[NDB];
#pragma unroll
  for (int i = 0; i < NDB; i++) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float c = a.scale * LOG2E;
  float m_run = M_FLOOR, l_run = 0.f;
  auto step = [&](int key0, int buf, bf16x8 (*kf)[2], bf16x8 (*kn)[2]) {
    // the next stage's loads go out in any case, so that the number in flight is known: past the end they repeat the
    // last key and read no value
    const int next = key0 + NW * KB;
    load_k(next, kn);
    f32x4 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; kb++) {
      s[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < NKS; x++) s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[x][kb], qf[x], s[kb], 0, 0, 0);
    }
    load_v(next, buf ^ 1);
    if (key0 + KB > min(all_vis, end)) {
#pragma unroll
      for (int kb = 0; kb < 2; kb++)
#pragma unroll
        for (int r = 0; r < 4; r++) {
          const int key = key0 + 16 * kb + 4 * g4 + r;
          if (key >= vis || key >= end) s[kb][r] = -INFINITY;
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; kb++)
#pragma unroll
      for (int r = 0; r < 4; r++) mx = fmaxf(mx, s[kb][r]);
    mx = pair_max(fmaxf(mx, __shfl_xor(mx, 16, 64)));
    if (__ballot(mx > m_run) != 0) {
      const float m_new = fmaxf(m_run, mx), alpha = __builtin_amdgcn_exp2f((m_run - m_new) * c);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int i = 0; i < NDB; i++)
#pragma unroll
        for (int r = 0; r < 4; r++) o[i][r] *= alpha;
    }
    bf16x8 pf;   // keys 4 g4 + 0..3, 16 + 4 g4 + 0..3
#pragma unroll
    for (int kb = 0; kb < 2; kb++)
#pragma unroll
      for (int r = 0; r < 4; r++) {
        const float p = __builtin_amdgcn_exp2f((s[kb][r] - m_run) * c);   // (the difference first: exact however large they are)
        l_run += p;
        pf[4 * kb + r] = (__bf16)p;
      }
    wait_loads<2 * NKS + Tile::LOADS>();   // only the next stage's loads are still in flight
    __builtin_amdgcn_sched_barrier(0);
    const char* sv = sv0 + buf * TILE;
#pragma unroll
    for (int db = 0; db < NDB; db++)
      o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(join_tr(read_tr(sv + vbase[db][0]), read_tr(sv + vbase[db][1])), pf, o[db], 0, 0, 0);
    // (the reads are complete before the MFMAs that use them, so the buffer may be loaded again)
    __builtin_amdgcn_sched_barrier(0);
  };
  {
    int key0 = begin + wave * KB;
    bf16x8 ka[NKS][2], kb[NKS][2];
    if (key0 < end) {
      load_k(key0, ka);
      load_v(key0, 0);
    }
    while (key0 < end) {
      step(key0, 0, ka, kb);
      key0 += NW * KB;
      if (key0 >= end) break;
      step(key0, 1, kb, ka);
      key0 += NW * KB;
    }
  }
  wait_loads<0>();   // (loads past the end write their zeros to LDS too)
  l_run += __shfl_xor(l_run, 16, 64);
  l_run = pair_sum(l_run);
  // the waves' results meet: [wave][row][D + 4] outputs, [wave][row] maxima and sums
  __syncthreads();
  float* mo = (float*)smem;
  float2* ml = (float2*)(smem + NW * ROWS * (D + 4) * 4);
#pragma unroll
  for (int db = 0; db < NDB; db++) *(f32x4*)(mo + (wave * ROWS + l16) * (D + 4) + 16 * db + 4 * g4) = o[db];
  if (g4 == 0) ml[wave * ROWS + l16] = make_float2(m_run, l_run);
  __syncthreads();
  constexpr int EPT = 8, LPR = D / EPT;   // elements of a row per thread, threads per row
  const int r = tid / LPR, e0 = (tid % LPR) * EPT, rr = row0 + r;
  const bool partial = a.part_tiles && t.parts > 1;
  const int64_t place = partial ? partial_slot<ROWS>(a, t.g, t.seq, t.local, 1) : 0;
  if (r >= ROWS || rr >= rows || place < 0) return;
  float m = M_FLOOR, l = 0.f, acc[EPT];
#pragma unroll
  for (int w = 0; w < NW; w++) m = fmaxf(m, ml[w * ROWS + r].x);
#pragma unroll
  for (int e = 0; e < EPT; e++) acc[e] = 0.f;
#pragma unroll
  for (int w = 0; w < NW; w++) {
    const float2 x = ml[w * ROWS + r];
    const float f = __builtin_amdgcn_exp2f((x.x - m) * c);
    l = fmaf(f, x.y, l);
#pragma unroll
    for (int e = 0; e < EPT; e += 4) {
      const f32x4 y = *(const f32x4*)(mo + (w * ROWS + r) * (D + 4) + e0 + e);
#pragma unroll
      for (int j = 0; j < 4; j++) acc[e + j] = fmaf(f, y[j], acc[e + j]);
    }
  }
  if (partial) {
    const int64_t slot = place * ROWS + r;
    if (e0 == 0) a.part_ml[slot] = make_float2(m, l);
#pragma unroll
    for (int e = 0; e < EPT; e += 4) store4<float>(a.part_o + slot * D + e0 + e, acc + e);
    return;
  }
  const int tk = rr / a.G, hd = t.g * a.G + (rr - tk * a.G);
  const bool sees = sees_keys(a, t.s, tk);
  const float inv = sees ? 1.0f / l : 0.f;
  const float lse = sees ? fmaf(m, a.scale, __builtin_amdgcn_logf(l) * LN2) : -INFINITY;
#pragma unroll
  for (int e = 0; e < EPT; e++) acc[e] = sees ? acc[e] * inv : 0.f;   // (nothing of a value that is no number)
  if (a.lse && e0 == 0) a.lse[(int64_t)(q0 + tk) * a.H + hd] = lse;
#pragma unroll
  for (int e = 0; e < EPT; e += 4) store4<u16>((u16*)a.o + (int64_t)(q0 + tk) * a.o_row + (int64_t)hd * a.o_head + e0 + e, acc + e);
#endif
}

// Joins the parts of each row, in their order: with w_p = exp(m_p - max m), o = sum w_p o_p / sum w_p l_p. (Not from an lse of each part,
// m_p + log l_p: that loses what l_p says where m_p is large, and a maximum over NaN drops them.) One wave per row, 4 rows per
// workgroup; the parts' rows are loaded eight at a time.
template <typename T, int ROWS>
__global__ void __launch_bounds__(256) packed_join(PackedArgs a, int d) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int quad = blockIdx.x % (ROWS / 4), gu = blockIdx.x / (ROWS / 4);
  const int u = gu / a.Hkv, g = gu - u * a.Hkv;
  int seq, rt;
  PackedSeq sq;
  if (!find_unit(a.nseq, u, [&](int i) { return a.sequence(i); }, [&](const PackedSeq& s) { return row_tiles_of<ROWS>(a, s); }, seq, rt, sq))
    return;
  const int parts = parts_of(a, sq);
  const int rows = sq.m * a.G, q0 = sq.q0, row = rt * ROWS + 4 * quad + wave;
  if (parts <= 1 || row >= rows) return;
  const int place = a.causal ? cdiv(rows, ROWS) - 1 - rt : rt;   // where the tile stands in the order of the units
  const int64_t first = partial_slot<ROWS>(a, g, seq, place * parts, parts);
  if (first < 0) return;
  const int64_t slot = first * ROWS + 4 * quad + wave;   // of part 0; parts are ROWS apart
  const float2* ml = a.part_ml + slot;
  const float* po = a.part_o + slot * d;
  const int tok = row / a.G, head = g * a.G + row - tok * a.G;
  const float scale = sizeof(T) == 2 ? a.scale : 1.f, c = scale * LOG2E;   // (fp32 scores are scaled)
  float top = M_FLOOR;
  for (int p = lane; p < parts; p += 64) top = fmaxf(top, ml[(int64_t)p * ROWS].x);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  const int e = d > 64 ? 2 * lane : lane;
  float total = 0.f, acc0 = 0.f, acc1 = 0.f;
  for (int p0 = 0; p0 < parts; p0 += 64) {
    const int np = min(parts - p0, 64);
    float w = 0.f, l = 0.f;
    if (lane < np) {
      const float2 x = ml[(int64_t)(p0 + lane) * ROWS];
      w = __builtin_amdgcn_exp2f((x.x - top) * c);
      l = x.y;
    }
    for (int p = 0; p < np; p += 8) {
      float2 v[8];
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const float* x = po + (int64_t)(p0 + min(p + j, np - 1)) * ROWS * d + e;
        v[j] = d > 64 ? *(const float2*)x : make_float2(*x, 0.f);
      }
#pragma unroll
      for (int j = 0; j < 8; j++)
        if (p + j < np) {
          const float wj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), p + j));
          total = fmaf(wj, __int_as_float(__builtin_amdgcn_readlane(__float_as_int(l), p + j)), total);
          acc0 = fmaf(wj, v[j].x, acc0);
          acc1 = fmaf(wj, v[j].y, acc1);
        }
    }
  }
  const bool sees = sees_keys(a, sq, tok);
  const float inv = sees ? 1.f / total : 0.f;
  T* orow = (T*)a.o + (int64_t)(q0 + tok) * a.o_row + (int64_t)head * a.o_head + e;
  orow[0] = from_f32<T>(sees ? acc0 * inv : 0.f);   // (nothing of a value that is no number)
  if (d > 64) orow[1] = from_f32<T>(sees ? acc1 * inv : 0.f);
  if (a.lse && lane == 0)
    a.lse[(int64_t)(q0 + tok) * a.H + head] = sees ? fmaf(top, scale, __builtin_amdgcn_logf(total) * LN2) : -INFINITY;
}

// Tiles and parts.
//   rows   16 where no sequence has more than FEW_ROWS (query, head) rows per key/value head; else bf16: 128, fp32: 64, or 16 where
//          tiles of 64 are fewer than two workgroups per CU (4 x 300 tokens, 16 heads of 64: 22 us, as tiles of 64 28)
//   parts  16-row tiles: one CU streams keys at 60 GB/s (128 keys of K and V at head_dim 128 in 1.09 us, after 4.2 us for a call), and
//          the launch that joins parts costs 4 us. So keys are shared out where a sequence may have more than 12 tiles, for about
//          two workgroups per CU (32 tokens, 90 k keys of 8 heads: 80 us; four per CU: 88), in parts of at least 4 tiles (one
//          token, 2048 keys: 10.5 us; 16 tiles: 16.7), or of 12 where the sequences alone fill the chip (32 tokens, 300 keys
//          each: 11.2 us; 4 tiles: 15.5). fp32 tiles take twice as long: parts of 2 at least, from 5 tiles on (700 keys 29 us whole,
//          18 in parts of 4, 14 in parts of 2; sequences that fill the chip as above). Other tiles: only where they alone leave CUs without a workgroup, and
//          128 rows only where a part is WORTH tiles shorter than the average sequence: their results are about 67 MB to write and
//          read however the keys are cut (us whole / shared out: 1024 keys of 16 over 4 heads 23 / 38, 2048 of 8 over 1 38 / 40, of
//          4 over 4 37 / 32, 4096 of 4 over 1 68 / 51, 8192 of 2 over 1 129 / 72). The host knows the average length alone, so a long
//          sequence beside short ones stays whole where it would gain (4096 and 200 keys of 4 over 1: 70 / 56).
PackedPlan packed_plan(int dtype, int nseq, int H, int Hkv, int d, int total_q, int total_k, int max_q, int max_k) {
  constexpr int CUS = 256, FEW_ROWS = 32, MIN_PART = 4, WHOLE = 12, WORTH = 26;
  PackedPlan p{};
  const int G = H / Hkv;
  const bool few = (int64_t)max_q * G <= FEW_ROWS;
  auto tiles_of = [&](int rows) { return std::min<int64_t>((int64_t)total_q * G / rows + nseq, (int64_t)nseq * cdiv((int64_t)max_q * G, rows)); };
  p.rows = few || (dtype == DT_F32 && tiles_of(64) * Hkv < 2 * CUS) ? 16 : dtype == DT_F32 ? 64 : 128;
  const int64_t per_seq = cdiv((int64_t)max_q * G, p.rows);   // no sequence has more row tiles
  p.row_tiles = p.units = (int)tiles_of(p.rows);
  const int64_t groups = (int64_t)p.row_tiles * Hkv;
  if (groups == 0 || (!few && groups >= CUS)) return p;
  const int64_t tiles = cdiv(total_k, 64), work = tiles * groups / nseq;
  const bool split_f32 = dtype == DT_F32 && groups < CUS;
  const int whole = split_f32 ? 4 : WHOLE;
  const int64_t per = std::max<int64_t>(split_f32 ? 2 : groups < CUS ? MIN_PART : WHOLE, (work + 2 * CUS - 1) / (2 * CUS));
  if (p.rows == 128 && tiles / nseq - per < WORTH) return p;
  const int64_t units = per_seq * (tiles / per + nseq);   // a sequence of n tiles has at most n / per + 1 parts
  if (cdiv(max_k, 64) <= std::max<int64_t>(whole, per) || (!few && units * Hkv > 16 * CUS)) return p;
  p.part_tiles = (int)per;
  p.units = (int)units;
  // sequences of more than one part have more than 64 per keys, n keys in fewer than n / (64 per) + 1 parts: fewer than 2 n / (64 per)
  p.slots = (int)std::min(units, per_seq * (total_k / (32 * per)));
  p.ws = (size_t)Hkv * p.slots * p.rows * (d + 2) * 4;
  return p;
}

template <int D>
static void fwd_launch(const PackedArgs& a, int dtype, int rows, int64_t grid, hipStream_t s) {
  if (dtype == DT_F32 && rows == 16) packed_split_f32<D><<<grid, 256, 0, s>>>(a);
  else if (dtype == DT_F32) packed_fwd_f32<D><<<grid, 256, 0, s>>>(a);
  else if (rows == 16) packed_few_bf16<D><<<grid, 256, 0, s>>>(a);
  else if (a.part_tiles) packed_fwd_bf16<D, true><<<grid, 256, 0, s>>>(a);
  else packed_fwd_bf16<D, false><<<grid, 256, 0, s>>>(a);
}

static PackedPlan plan_of(const PackedArgs& a, int dtype, int d) {
  return packed_plan(dtype, a.nseq, a.H, a.Hkv, d, a.qr.total, a.kr.total, a.max_q, a.kr.off ? a.kr.total : a.kr.len);
}
static int64_t join_groups(const PackedArgs& a, const PackedPlan& p) { return p.part_tiles ? (int64_t)p.row_tiles * a.Hkv * (p.rows / 4) : 0; }
int64_t packed_forward_threads(const PackedArgs& a, int dtype, int d) {
  const PackedPlan p = plan_of(a, dtype, d);
  return 256 * std::max((int64_t)p.units * a.Hkv, join_groups(a, p));
}

hipError_t packed_attention_fwd(PackedArgs a, int dtype, int d, void* ws, hipStream_t s) {
  const PackedPlan p = plan_of(a, dtype, d);
  if (p.row_tiles == 0) return hipSuccess;
  a.part_tiles = p.part_tiles;
  a.slots = p.slots;
  a.part_o = (float*)ws;
  a.part_ml = (float2*)(a.part_o + (int64_t)a.Hkv * p.slots * p.rows * d);
  const int64_t grid = (int64_t)p.units * a.Hkv;
  if (d == 128) fwd_launch<128>(a, dtype, p.rows, grid, s);
  else fwd_launch<64>(a, dtype, p.rows, grid, s);
  if (p.part_tiles) {
    const int64_t jg = join_groups(a, p);
    if (p.rows == 16 && dtype == DT_F32) packed_join<float, 16><<<jg, 256, 0, s>>>(a, d);
    else if (p.rows == 16) packed_join<u16, 16><<<jg, 256, 0, s>>>(a, d);
    else packed_join<u16, 128><<<jg, 256, 0, s>>>(a, d);   // (64-row tiles of fp32 fill the chip by themselves)
  }
  return hipGetLastError();
}

}  // namespace dit
