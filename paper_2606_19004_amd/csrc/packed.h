// Packed sequences and the operands of the kernels that work on them (device side), and the entry points
// of k_packed_attn.hip, k_packed_attn_bwd.hip, k_gated_norm.hip and k_policy_loss.hip.
#pragma once
#include "internal.h"

namespace dit {

// Rows of the sequences of a packed tensor: offsets on the device, or equal lengths (off null).
struct RowSpan {
  int begin, count;
};
struct PackedRows {
  const int* off;
  int total, len;   // rows of the tensor; of each sequence where off is null
  // the offsets' two entries as loaded, so that a caller's loads can all go out before the first is looked at
  __device__ __forceinline__ int2 raw(int i) const { return off ? make_int2(off[i], off[i + 1]) : make_int2(i * len, (i + 1) * len); }
  __device__ __forceinline__ RowSpan clamped(int2 r) const {
    const int b = min(max(r.x, 0), total);
    return RowSpan{b, max(min(r.y, total), b) - b};
  }
  __device__ __forceinline__ RowSpan span(int i) const { return clamped(raw(i)); }
};

// A sequence's queries q0 .. q0 + m and keys k0 .. k0 + n.
struct PackedSeq {
  int q0, m, k0, n;
};
struct PackedArgs {
  const void* q; const void* k; const void* v; void* o;
  float* lse;                       // [total_q][H], null: not wanted (forward)
  PackedRows qr, kr;
  const int* k_len;                 // or null
  int nseq, H, Hkv, G, max_q, causal;
  float scale;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
  // long keys shared out in parts of part_tiles 64-key tiles (0: one part), whose results meet in the workspace
  int part_tiles, slots;            // slots: upper bound on (sequence, row tile, part) of the sequences with more than one part, per key/value head
  float* part_o; float2* part_ml;   // [Hkv * slots][row tile][d] sums of p v, [Hkv * slots][row tile] running maximum and sum of p
  // backward
  const void* d_o; void* dq; void* dk; void* dv;
  float2* stats;                    // [H][total_q] (lse, for bf16 in log2 units, rowsum(d_o o))
  int shares; float* share_sums;    // workgroups that share a key tile's rows, and their sums
  __device__ __forceinline__ PackedSeq sequence(int i) const {
    const int2 q = qr.raw(i), k = kr.raw(i);
    const int used = k_len ? k_len[i] : 0x7fffffff;
    const RowSpan qs = qr.clamped(q), ks = kr.clamped(k);
    return PackedSeq{qs.begin, min(qs.count, max_q), ks.begin, min(max(used, 0), ks.count)};
  }
};

// Inclusive sum over the wave: 1, 2, 4 and 8 lanes before within rows of 16 lanes, then the rows before. VALU moves, no LDS.
template <int CTRL, int ROWS> __device__ __forceinline__ unsigned moved_up(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ unsigned wave_scan(unsigned v) {
  v += moved_up<0x111, 0xf>(v);
  v += moved_up<0x112, 0xf>(v);
  v += moved_up<0x114, 0xf>(v);
  v += moved_up<0x118, 0xf>(v);
  v += moved_up<0x142, 0xa>(v);
  v += moved_up<0x143, 0xc>(v);
  return v;
}

// The sequence that unit u belongs to, where a sequence with what = load(i) (a struct of int) has count(what) units, and u's place
// in it. Every wave finds it by itself, 64 sequences at a time: no host-made list of tiles, no empty workgroups where
// lengths are unlike. What is known of the sequence comes from the lane that looked at it, with no further loads.
// BLOCKS: how many times 64 sequences are loaded together (1000 sequences of 64 keys, 8 key/value heads of 128, one new token each: 191 to
// 203 us from card to card; one block at a time, with a sum by LDS permutes, 239. Reading the keys and values once takes 53.)
template <int BLOCKS, typename S, typename L, typename C>
__device__ __forceinline__ bool find_unit_in(int nseq, int u, L&& load, C&& count, int& seq, int& local, S& what) {
  const int lane = threadIdx.x & 63;
  unsigned carry = 0;   // <= u
  for (int base = 0; base < nseq; base += 64 * BLOCKS) {
    S mine[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; b++) mine[b] = load(min(base + 64 * b + lane, nseq - 1));
#pragma unroll
    for (int b = 0; b < BLOCKS; b++) {
      if (base + 64 * b >= nseq) return false;
      // (no count of a tensor within the entry points' limits is larger: tiles of 64 of fewer than 2^30 rows, of 16 only where they are
      // few, chunks of 8 of at most 2^28 rows where there are many; and 64 of these fit)
      const unsigned c = base + 64 * b + lane < nseq ? min(count(mine[b]), 1 << 25) : 0, incl = wave_scan(c);
      const unsigned total = __builtin_amdgcn_readlane(incl, 63);
      if ((unsigned)u < carry + total) {
        const int l = __builtin_ctzll(__ballot(carry + incl > (unsigned)u));
        seq = base + 64 * b + l;
        local = u - (int)(carry + __builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(c, l));
        union {
          S s;
          int w[sizeof(S) / 4];
        } in, out;
        in.s = mine[b];
#pragma unroll
        for (int i = 0; i < (int)(sizeof(S) / 4); i++) out.w[i] = __builtin_amdgcn_readlane(in.w[i], l);
        what = out.s;
        return true;
      }
      carry += total;
    }
  }
  return false;
}
template <typename S, typename L, typename C>
__device__ __forceinline__ bool find_unit(int nseq, int u, L&& load, C&& count, int& seq, int& local, S& what) {
  return nseq <= 64 ? find_unit_in<1>(nseq, u, load, count, seq, local, what) : find_unit_in<4>(nseq, u, load, count, seq, local, what);
}

// How a call runs (host): see packed_plan in k_packed_attn.hip
struct PackedPlan {
  int rows;         // query rows of a workgroup's tile
  int part_tiles;   // 64-key tiles of a part, 0: keys are not shared out
  int row_tiles, units, slots;   // upper bounds per key/value head: row tiles, (row tile, part), those of sequences with more than one part
  size_t ws;        // bytes
};
PackedPlan packed_plan(int dtype, int nseq, int H, int Hkv, int d, int total_q, int total_k, int max_q, int max_k);
// Threads of the largest launch of a call: one takes fewer than 2^32.
int64_t packed_forward_threads(const PackedArgs& a, int dtype, int d);
int64_t packed_backward_threads(const PackedArgs& a, int dtype, int d);
hipError_t packed_attention_fwd(PackedArgs a, int dtype, int d, void* ws, hipStream_t s);
size_t packed_backward_ws(int dtype, int nseq, int H, int Hkv, int d, int total_q, int total_k, int causal);
hipError_t packed_attention_stats(PackedArgs a, int dtype, int d, void* ws, hipStream_t s);
hipError_t packed_attention_gradients(PackedArgs a, int dtype, int d, void* ws, hipStream_t s);

enum NormKind { NORM_NONE = 0, NORM_LAYER = 1, NORM_RMS = 2 };
struct GatedNormArgs {
  const void* x; const void* y; const void* post_w; const void* pre_w;
  const float* gate; const float* scale; const float* shift;
  PackedRows pr;
  int nseq, rows, D, post, pre;
  float eps, alpha;
  int64_t x_row, y_row, h_row, mod_row;
  void* x_out; void* h;
  // backward (x is the forward's x_out)
  const void* dx_out; const void* dh; void* dx; void* dy;
  float* dgate; float* dscale; float* dshift; float* dpost_w; float* dpre_w;
  float* parts;   // [chunks][3][D] column sums of the row chunks
  int chunks;     // upper bound on (sequence, chunk)
};
int64_t gated_norm_forward_threads(const GatedNormArgs& a);    // of the largest launch
int64_t gated_norm_backward_threads(const GatedNormArgs& a);
hipError_t gated_norm_fwd(const GatedNormArgs& a, int dtype, hipStream_t s);
int gated_norm_chunks(int nseq, int rows, int D);   // row chunks of the backward pass, at most
size_t gated_norm_ws(int nseq, int rows, int D);
hipError_t gated_norm_rows_bwd(const GatedNormArgs& a, int dtype, hipStream_t s);
hipError_t gated_norm_columns_bwd(const GatedNormArgs& a, int dtype, hipStream_t s);

struct PolicyLossArgs {
  const float* x; const float* v; const float* xn; const float* v_ref;
  int batch; int64_t n;
  double cx, cv, var, cst;   // mean = cx x + cv v; cst: the constant of logp
  const double* logp_old; const float* adv;
  double logp_scale, clip_low, clip_high, kl_weight;
  double* loss; double* logp; double* ratio; float* dv;
  double* parts;   // [batch][chunks][2] sums of (x_next - mean)^2 and (v - v_ref)^2
  int chunks;
};
int policy_loss_chunks(int batch, int64_t n);
hipError_t policy_loss_sums(const PolicyLossArgs& a, hipStream_t s);
hipError_t policy_loss_finish(const PolicyLossArgs& a, hipStream_t s);

}  // namespace dit
