// Shared by the attention kernels: their arguments, and how the work of a call is dealt out.
#pragma once
#include "sp_common.cuh"

namespace sp {

struct AttnParams {
  const void *q, *k, *v;
  void* o;
  int64_t ldq, ldk, ldv, ldo;
  float* lse;
  const int32_t* cu_q;
  const int32_t* cu_k;
  int32_t Nq, Nk, n_seq, n_heads, n_kv, g, dh, causal;
  float scale_log2;            // scale * log2(e): softmax in base 2
  // Key axis in parts of `part` keys (a multiple of the key tile; 0: not cut).  Part c of row i leaves its normalised
  // result and lse (base 2) at [c][i] of these; a sequence of n_k keys has max(1, ceil(n_k / part)) parts.
  int32_t part, max_parts;
  float* part_o;               // [max_parts, Nq, n_heads * dh]
  float* part_lse;             // [max_parts, Nq, n_heads]
  int32_t* status;
  long long wait_budget;
};

// One piece of work: a tile of a sequence's rows (queries x the heads that share a key head, head fastest), one key / value
// head, one part of the keys.
struct AttnItem {
  int32_t q0, nq, k0, nk;           // first row of the sequence in Q and K, their numbers
  int32_t head, tile, c;            // key / value head, tile of rows, part of keys
};

// Deals the items of a call in a fixed order: 32 sequences at a time; among them, tiles of rows from the last to the first (by number: with the
// causal mask of equal lengths a tile costs what its number says, so that items get lighter), sequences, heads, parts.  (Sequence by sequence:
// 16 documents of up to 2048 tokens kept SMs busy for 0.80 .. 1.13 of the mean, so 0.92 .. 1.10.)  A caller asks for rising item numbers; the 32 sequences at
// hand stay in registers, a lane each.  Every warp keeps a dealer of its own; all lanes of the warp call.
struct AttnDealer {
  int32_t base = 0;            // sequences before this group of 32 are passed
  bool at_hand = false;        // the group's are in the registers below
  int32_t level;               // tile number at hand
  int32_t q0, nq, k0, nk, tiles, parts;
  int64_t passed = 0;          // items of the groups that are passed
  int64_t total, above;        // items of the group, of its higher tiles
  int64_t mine, upto, here;    // items of this tile number: of this lane's sequence, up to it, of all
  static __device__ __forceinline__ int32_t bound(int32_t x, int32_t n) { return x < 0 ? 0 : x > n ? n : x; }
  __device__ __forceinline__ void scan(int heads) {
    const int lane = threadIdx.x & 31;
    mine = tiles > level ? (int64_t)heads * parts : 0;
    upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t t = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += t;
    }
    here = __shfl_sync(0xffffffffu, upto, 31);
  }
  // row_mul: rows per query; rows_per_tile counts those
  __device__ __forceinline__ bool find(const AttnParams& p, int64_t item, int rows_per_tile, int row_mul, int heads,
                                       AttnItem& it) {
    const int lane = threadIdx.x & 31;
    while (true) {
      if (!at_hand) {
        if (base >= p.n_seq) return false;
        const int s = base + lane;
        q0 = nq = k0 = nk = tiles = 0;
        parts = 1;
        if (s < p.n_seq) {
          q0 = bound(p.cu_q[s], p.Nq);
          nq = bound(p.cu_q[s + 1], p.Nq) - q0;
          k0 = bound(p.cu_k[s], p.Nk);
          nk = bound(p.cu_k[s + 1], p.Nk) - k0;
          if (nq < 0) nq = 0;
          if (nk < 0) nk = 0;
          tiles = (int)(((int64_t)nq * row_mul + rows_per_tile - 1) / rows_per_tile);
          if (p.part > 0 && nk > p.part) parts = (nk - 1) / p.part + 1;
        }
        total = (int64_t)tiles * heads * parts;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        level = __reduce_max_sync(0xffffffffu, tiles) - 1;
        above = 0;
        scan(heads);
        at_hand = true;
      }
      if (item < passed + total) {
        int64_t rest = item - passed;
        while (rest >= above + here) {
          // down to the item's tile number, or to the next one that more sequences have
          const int32_t join = __reduce_max_sync(0xffffffffu, tiles <= level ? tiles : 0);
          const int64_t same = level - join + 1, gone = quotient(rest - above, here), skip = gone < same ? gone : same;
          above += skip * here;
          level -= (int32_t)skip;
          if (skip == same) scan(heads);
        }
        rest -= above;
        const int l = __ffs(__ballot_sync(0xffffffffu, rest < upto)) - 1;
        it.q0 = __shfl_sync(0xffffffffu, q0, l);
        it.nq = __shfl_sync(0xffffffffu, nq, l);
        it.k0 = __shfl_sync(0xffffffffu, k0, l);
        it.nk = __shfl_sync(0xffffffffu, nk, l);
        const int of_parts = __shfl_sync(0xffffffffu, parts, l);
        rest -= __shfl_sync(0xffffffffu, upto - mine, l);
        it.tile = level;
        it.head = (int)quotient(rest, of_parts);
        it.c = (int)(rest - (int64_t)it.head * of_parts);
        return true;
      }
      passed += total;
      base += 32;
      at_hand = false;
    }
  }
  static __device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {      // of numbers >= 0 (64-bit divisions are slow)
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
  }
};

// Few rows on average (single tokens): kernels that stream the keys past them.
inline bool attention_few_rows(int64_t Nq, int64_t g, int64_t n_seq) { return Nq * g <= 16 * n_seq; }
sp_status attention_rows(const AttnParams& p, cudaStream_t stream);      // bf16 (sp_attention_rows.cu), layouts as below
bool attention_rows_f32_supported(const AttnParams& p);                     // fp32 (sp_attention_rows_f32.cu): rows that 16-byte copies can take
cudaError_t attention_rows_f32(const AttnParams& p, cudaStream_t stream);
// tcgen05 form (sp_attention_tc.cu): layouts that tensor maps can describe
bool attention_tc_supported(const AttnParams& a);
sp_status attention_tc(const AttnParams& a, cudaStream_t stream);

}  // namespace sp
