// bf16 attention on the tensor cores of sm_100a: S = Q K^T and O += P V as tcgen05.mma with fp32 accumulators in tensor
// memory, operands brought in by TMA, softmax on the CUDA cores in between.
//
// A CTA (one per SM, persistent) works on two tiles of up to 128 rows at a time, "half" 0 and 1, that share every key and value tile:
// while the softmax warps of one half turn its S into P, the tensor core multiplies for the other.  Rows of a tile are queries x the heads
// that share a key head (head fastest), so that grouped heads read K and V once; a 3-D tensor map (channel, head, token) lands them in
// that order.  Per half and key tile of 128:
//   S (128 columns of tensor memory) -> registers, one row per thread; row maximum; P = 2^(c S - c r) in bf16, written back over the
//   first 64 columns of S; O += P V with P read from tensor memory.
// The reference r of a row follows its running maximum only when that has risen by more than 2^8 in P's scale: O is then rescaled in tensor
// memory by the same threads.  P and its sum l stay relative to r, so nothing is approximated by waiting, and l <= 2^8 n holds in fp32.
// Masked values: S is replaced by -infinity.  V is not touched by that: 0 times what stands there would be NaN for an infinity.  So in tiles
// that some row does not see whole, two warps clear the rows of V that no row sees, and set non-finite values in rows that only some see to
// zero; those rows then get them back at the end (rows_with_bad_values).
//
// S and P of a key tile and a half (a job) take one of BUFS buffers of tensor memory in turn: three for heads up to 64 (O is narrow there),
// so that S of a half's next tile is there when its softmax ends, two for wider ones.  A tile of which only half 0 has rows (few queries, the
// end of a sequence) has all of them for itself ("alone").
//
// Warps: 0-3 and 4-7 softmax of half 0 and 1 (lane and warp give the row), 8 finds the items and issues TMA, 9 MMA issue and tensor memory,
// 10-11 edge tiles of V.  Items go to the other warps through shared memory (finding one takes two thousand cycles).
// What bounds it: per half and tile 128 exponentials a row (1024 cycles of the pipe that two warps share) between two products (1024 cycles
// together for heads of 128).  One prompt of 8192, 32 heads of 128 on 8: 488 us after a pause, 531 in a row of calls (power cap); 16 documents of up to
// 2048 tokens, 32 heads of 64 on 8: 167 and 156 us.  (Figures beside the steps below are of the kernel of that time.)
// HALF: operands opened from a cache of 4 bits, fp16 in units of a text's key head and of a row's queries (HalfTops): the same instructions with
// eight times finer roundings, of P as well, whose reference leaves it 2^6 higher so that its small values keep theirs.  A text's head whose
// sizes leave fp16 comes in bf16: the format is an item's.
// Waits for copies, the tensor core and other warps are bounded by a clock budget (SP_ERR_TIMEOUT through status).
#include <cuda_fp16.h>
#include <math.h>
#include <string.h>

#include <type_traits>

#include "sp_attention.cuh"
#include "sp_f32x2.cuh"
#include "sp_tc.cuh"

namespace sp {
namespace {

constexpr int kRows = 128, kKeys = 128;
constexpr int kThreads = 384;
constexpr long long kWaitBudget = 4000000000LL, kDrainBudget = 200000000LL;    // clock cycles: ~2 s, ~0.1 s
// Registers of a thread: 168 at launch (384 threads); the eight softmax warps hold a whole row of S and take what the others leave.
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88;
static_assert(2 * kSoftmaxRegs + kOtherRegs <= 3 * 168, "shares of the registers at launch");
constexpr int kBadSlots = 32;       // items with keys between the edge warps and the epilogue: less than the stages of the ring
constexpr int kItems = 8;           // items handed from the TMA warp to the softmax and edge warps

template <int DH>
struct Cfg {
  static constexpr int CH = DH / 64;                       // 128-byte wide chunks of a row
  static constexpr int CHUNK = 128 * 128;                  // bytes of one: 128 rows of 128 bytes
  static constexpr int TILE = CH * CHUNK;
  static constexpr int STAGES = DH == 128 ? 5 : 8;
  static constexpr int BUFS = DH == 128 ? 2 : 3;           // tiles of S and P in tensor memory
  static constexpr int BARS = 4 * STAGES + 17 + 2 * kItems;
  static constexpr size_t SMEM = (size_t)(2 + STAGES) * TILE + 1024 + 8 * BARS;
  static constexpr uint32_t O_COL = 128 * BUFS, O_COLS = DH;      // tensor memory: BUFS x 128 columns of S, then O of both halves
  static_assert(O_COL + 2 * O_COLS <= 512, "tensor memory");
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int32_t c0, int32_t c1, int32_t c2, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_commit_one(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Shared-memory descriptors (make_smem_desc of sp_tc.cuh) in two words: the upper one is the same for all tiles here, the lower
// one moves with the address in units of 16 bytes, so that an instruction's descriptors cost an addition.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_low(uint32_t addr, uint32_t leading) { return ((addr & 0x3ffffu) >> 4) | ((leading >> 4) << 16); }
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint32_t a_low, uint32_t b_low, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}"
      ::"r"(d), "r"(a_low), "r"(b_low), "r"(idesc), "r"(accumulate), "r"(kDescHigh)
      : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint32_t b_low, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 b, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b_low), "r"(idesc), "r"(accumulate), "r"(kDescHigh)
      : "memory");
}
__device__ __forceinline__ void tc_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
        "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
        "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {       // NaN if one of them is
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// One lane of a converged warp, chosen by the hardware.  Behind this branch the compiler knows that one lane is active and keeps the
// operands of the matrix instructions in uniform registers; behind lane == 0 every issue cost 75 cycles.
__device__ __forceinline__ bool elect_one() {
  uint32_t pred;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(pred));
  return pred != 0;
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {      // without suspending the thread
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// fp16 or (kBf16) bf16 operands, fp32 accumulator, 128 x n; B K-major or (V: keys are K, channels contiguous) MN-major
constexpr uint32_t kBf16 = (1u << 7) | (1u << 10);
__device__ __forceinline__ uint32_t instr_desc(bool b_kmajor, int n) {
  return (1u << 4) | ((b_kmajor ? 0u : 1u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24);
}

struct TcAttnParams {
  AttnParams a;
  int32_t gp, tokens;        // heads in a tile's rows, tokens of a half: gp * tokens <= 128
  int32_t heads;             // items' heads: key heads, or query heads when these are not packed (gp = 1)
  int32_t vec_out;           // rows of O can be stored 16 bytes at a time
};

// What all warps derive from an item.
struct Work {
  int t0;                    // first token of the tile within its sequence
  int kb;                    // first key of the part
  int n[2];                  // key tiles of each half
  bool alone;                // half 1 has no rows
  int sure;                  // keys [0, sure) are seen by every row
  int seen;                  // keys [0, seen) are seen by some row (no later one is in the part either)
  __device__ __forceinline__ int tiles() const { return n[0] > n[1] ? n[0] : n[1]; }
  __device__ __forceinline__ bool edge(int i) const { return kb + (i + 1) * kKeys > sure; }
};
__device__ __forceinline__ int visible(const AttnItem& it, int causal, int token) {
  if (!causal) return it.nk;
  const int64_t v = (int64_t)token + it.nk - it.nq + 1;
  return v < 0 ? 0 : v < it.nk ? (int)v : it.nk;
}
__device__ __forceinline__ Work work_of(const TcAttnParams& p, const AttnItem& it) {
  Work w;
  w.t0 = it.tile * 2 * p.tokens;
  const bool cut = p.a.part > 0 && it.nk > p.a.part;
  w.kb = cut ? it.c * p.a.part : 0;
  const int end = cut && it.nk - w.kb > p.a.part ? w.kb + p.a.part : it.nk;
  w.sure = visible(it, p.a.causal, w.t0);
  w.seen = 0;
  w.alone = w.t0 + p.tokens >= it.nq;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int first = w.t0 + h * p.tokens;
    int last = first + p.tokens - 1;
    if (last > it.nq - 1) last = it.nq - 1;
    int v = first < it.nq ? visible(it, p.a.causal, last) : 0;
    if (v > end) v = end;
    if (v > w.seen) w.seen = v;
    w.n[h] = v > w.kb ? (v - w.kb + kKeys - 1) / kKeys : 0;
  }
  return w;
}

// The k-th item of this CTA.  Items get lighter (of 32 sequences); every other round is dealt backwards, so that no CTA always has the
// heavier ones (one prompt of 8192: busy cycles of the SMs from 0.86 to 1.14 of their mean without).
__device__ __forceinline__ int64_t item_of(int k) {
  return (int64_t)k * gridDim.x + (k & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
}

// What the thread that issues the matrix instructions has to know of an item (it is one lane, and an item is found by a warp: the TMA warp leaves
// this in shared memory before the item's Q): key tiles of each half, 0 and 0 behind the last item, and the first edge tile.
struct Brief {
  int n0, n1, edge;
  uint32_t type;             // of the operands: 0, kBf16
};
constexpr int kBriefs = 8;             // more than the buffers of S: items between the issue of S and of P V

// A walk over the jobs of an item: key tile by key tile, the halves that see the tile.  (Half 1 has the later rows and sees no fewer tiles
// than half 0; a tile of rows without half 1 is half 0 alone.)
struct Cursor {
  Brief w;
  int i, h;                            // key tile, half
  int b = 0;                           // buffer of S and P
  int stage = 0;                       // of the ring: the tile's K, its V is in the next one
  bool open = false;
  __device__ __forceinline__ void start(const Brief& of) {
    w = of;
    i = 0;
    h = w.n0 > 0 ? 0 : 1;
    open = true;
  }
  __device__ __forceinline__ int tiles() const { return w.n0 > w.n1 ? w.n0 : w.n1; }
  __device__ __forceinline__ bool first() const { return h == 0 || w.n0 <= i; }       // of the tile
  __device__ __forceinline__ bool last() const { return h == 1 || w.n1 <= i; }
  __device__ __forceinline__ void advance(int bufs, int stages) {
    b = b + 1 == bufs ? 0 : b + 1;
    if (!last()) {
      h = 1;
      return;
    }
    ++i;
    stage = stage + 2 >= stages ? stage + 2 - stages : stage + 2;
    h = w.n0 > i ? 0 : 1;
    open = i < tiles();
  }
};

constexpr float kHalfLift = 6.f;       // HALF: P and its sums by 2^6

template <int DH, bool HALF>
__global__ void __launch_bounds__(kThreads, 1)
attention_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                    const __grid_constant__ CUtensorMap tmV, const TcAttnParams p) {
  using C = Cfg<DH>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint32_t s_tmem_base;
  __shared__ int s_abort;
  __shared__ Brief s_brief[kBriefs];
  __shared__ AttnItem s_item[kItems];    // tile < 0: no more
  __shared__ HalfUnits s_units[HALF ? kItems : 1];
  __shared__ int s_bad[kBadSlots];       // slot of an item: its number where V had non-finite values behind the mask

  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t q_smem = (raw + 1023u) & ~1023u;
  const uint32_t ring = q_smem + 2 * C::TILE;
  const uint32_t bars = ring + C::STAGES * C::TILE;
  auto full_bar = [&](int s) { return bars + 8u * s; };                         // a K tile, or a V tile seen whole
  auto edge_bar = [&](int s) { return bars + 8u * (C::STAGES + s); };           // a V tile that the edge warps look at first
  auto ready_bar = [&](int s) { return bars + 8u * (2 * C::STAGES + s); };      // they have
  auto empty_bar = [&](int s) { return bars + 8u * (3 * C::STAGES + s); };
  const uint32_t misc = bars + 8u * 4 * C::STAGES;
  const uint32_t q_full = misc, q_empty = misc + 8, drain_bar = misc + 16;
  auto pv_done = [&](int h) { return misc + 24u + 8u * h; };                    // O of half h += P V of a key tile
  // S in buffer b, for half h.  (A wait tells a phase from the next one only: every phase of a barrier is waited for by the same warps.)
  auto s_full = [&](int h, int b) { return misc + 40u + 8u * (3 * h + b); };
  auto p_half = [&](int b) { return misc + 88u + 8u * b; };                     // the first 64 columns of P
  auto p_full = [&](int b) { return misc + 112u + 8u * b; };
  auto item_full = [&](int k) { return misc + 136u + 16u * (k % kItems); };
  auto item_empty = [&](int k) { return misc + 144u + 16u * (k % kItems); };

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort_flag = &s_abort;
  const long long budget = p.a.wait_budget;

  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int s = 0; s < C::STAGES; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(edge_bar(s), 1);
      mbar_init(ready_bar(s), 2);
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    mbar_init(drain_bar, 1);
    for (int k = 0; k < kItems; ++k) {
      mbar_init(item_full(k), 1);
      mbar_init(item_empty(k), 10);
    }
    for (int h = 0; h < 2; ++h) {
      mbar_init(pv_done(h), 1);
      for (int b = 0; b < C::BUFS; ++b) mbar_init(s_full(h, b), 1);
    }
    for (int b = 0; b < C::BUFS; ++b) {
      mbar_init(p_half(b), 4);
      mbar_init(p_full(b), 4);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (threadIdx.x < kBadSlots) s_bad[threadIdx.x] = -1;
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem_base)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem_base;
  kernel_begin();

  AttnItem it;
  int seq = 0;                // number of the item among those of this CTA that have keys
  // the k-th item of this CTA, for the softmax and edge warps; false behind the last one, or when a wait ran out
  auto next_item = [&](int k, bool& ok, long long patience) {
    ok = __all_sync(0xffffffffu, mbar_wait(item_full(k), (uint32_t)(k / kItems) & 1u, abort_flag, patience));
    if (!ok) return false;
    it = s_item[k % kItems];
    return it.tile >= 0;
  };
  auto item_read = [&](int k) {
    __syncwarp();
    if (lane == 0) mbar_arrive(item_empty(k));
  };
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == 8) {
      // ------------------------------------------------------------------------------------------------ TMA
      AttnDealer dealer;
      uint32_t pos = 0;         // tiles loaded so far
      int loaded = 0;           // items with keys so far (their Q was loaded)
      bool ok = true;
      for (int k = 0;; ++k) {
        const bool more = dealer.find(p.a, item_of(k), 2 * p.tokens, 1, p.heads, it);
        if (!more) it.tile = -1;
        const int kvh = p.gp == 1 ? it.head / p.a.g : it.head;
        HalfUnits units = {1.f, 1.f, 0};
        if (HALF && more && lane == 0) units = half_units(p.a.half_tops[(int64_t)it.s * p.a.n_kv + kvh]);
        if (lane == 0) {
          if (k >= kItems) ok = mbar_wait(item_empty(k), (uint32_t)(k / kItems - 1) & 1u, abort_flag, budget);
          s_item[k % kItems] = it;
          if (HALF) s_units[k % kItems] = units;
          if (ok) mbar_arrive(item_full(k));
        }
        ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
        if (!ok || !more) break;
        const Work w = work_of(p, it);
        const int n = w.tiles();
        if (n == 0) continue;
        if (lane == 0) {
          if (loaded > 0) ok = mbar_wait(q_empty, (uint32_t)(loaded - 1) & 1u, abort_flag, budget);
          if (ok) {
            const int halves = w.alone ? 1 : 2;
            s_brief[loaded % kBriefs] = Brief{w.n[0], w.n[1], w.sure > w.kb ? (w.sure - w.kb) / kKeys : 0, HALF && units.half ? 0u : kBf16};
            mbar_expect_tx(q_full, (uint32_t)(halves * C::CH * p.gp * p.tokens * 128));
            for (int h = 0; h < halves; ++h)
  #pragma unroll
              for (int c = 0; c < C::CH; ++c)
                tma_load_3d(q_smem + h * C::TILE + c * C::CHUNK, &tmQ, c * 64, it.head * p.gp, it.q0 + w.t0 + h * p.tokens, q_full);
          }
          for (int i = 0; i < 2 * n && ok; ++i) {
            const int s = (int)(pos % C::STAGES);
            if (!mbar_wait(empty_bar(s), (pos / C::STAGES + 1) & 1u, abort_flag, budget)) { ok = false; break; }
            const bool v = i & 1;
            const uint32_t bar = v && w.edge(i >> 1) ? edge_bar(s) : full_bar(s);
            mbar_expect_tx(bar, C::TILE);
  #pragma unroll
            for (int c = 0; c < C::CH; ++c)
              tma_load_3d(ring + s * C::TILE + c * C::CHUNK, v ? &tmV : &tmK, c * 64, kvh, it.k0 + w.kb + (i >> 1) * kKeys, bar);
            ++pos;
          }
        }
        ++loaded;
        ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
        if (!ok) break;
      }
      if (ok && lane == 0) {      // no more
        if (loaded > 0) ok = mbar_wait(q_empty, (uint32_t)(loaded - 1) & 1u, abort_flag, budget);
        s_brief[loaded % kBriefs] = Brief{0, 0, 0, 0u};
        if (ok) mbar_arrive(q_full);
      }
      if (!ok && lane == 0) report_status(p.a.status, SP_ERR_TIMEOUT, (int32_t)blockIdx.x, 11);
    } else if (warp == 9) {
      // ------------------------------------------------------------------------------------------------ MMA
      // Two cursors over the same jobs (key tile, half): one issues S of a job, the other O += P V.  S of the next jobs is issued as soon
      // as a buffer, its keys and its rows are there, across the items; a buffer is free behind the product that reads its P, since the tensor
      // core takes the instructions of a thread in order.  With two buffers a softmax waits for this thread: S of the next job follows the product
      // at once, before the signals (prompt of 8192: 524 -> 479 us).  With three it does not, and one loop
      // for both halves was better than a warp for each, whose instructions alternate (519 us, 189).
      bool ok = true;
      if (elect_one()) {
        const uint32_t id_s0 = instr_desc(true, kKeys), id_o0 = instr_desc(false, DH);
        uint32_t full_ph = 0, ready_ph = 0, p_ph = 0;    // phases of the barriers of a stage, of a buffer: a bit each
        int items_s = 0, items_v = 0;                    // items that the cursors have been given
        int ahead = 0;                                   // jobs whose S is issued and whose P V is not
        bool end = false, issued = false, keys = false;  // keys: K of the next S has been waited for
        Cursor cs, cv;
        long long t0 = 0;                                // since when nothing could be issued (0: something was)
        auto keys_there = [&] {                          // of the next S
          if (!cs.open) return false;
          if (!cs.first() || keys) return true;
          const int s = cs.stage;
          keys = mbar_test(full_bar(s), (full_ph >> s) & 1u);
          if (keys) full_ph ^= 1u << s;
          return keys;
        };
        auto issue_s = [&] {
          const int s = cs.stage;
          const uint32_t a0 = desc_low(q_smem + cs.h * C::TILE, 16), b0 = desc_low(ring + s * C::TILE, 16);
          const uint32_t d = tmem + 128u * cs.b, id_s = id_s0 | (HALF ? cs.w.type : kBf16);
#pragma unroll
          for (int k = 0; k < DH / 16; ++k) {
            const uint32_t off = (uint32_t)((k / 4) * C::CHUNK + (k % 4) * 32) >> 4;
            tc_mma_ss(d, a0 + off, b0 + off, id_s, k > 0);
          }
          tc_commit_one(s_full(cs.h, cs.b));
          if (cs.last()) {
            tc_commit_one(empty_bar(s));
            if (cs.i + 1 == cs.tiles()) tc_commit_one(q_empty);
          }
          issued = true;
          keys = false;
          ++ahead;
          cs.advance(C::BUFS, C::STAGES);
        };
        while (true) {
          if (!cs.open && !end && mbar_test(q_full, (uint32_t)items_s & 1u)) {
            const Brief w = s_brief[items_s % kBriefs];
            ++items_s;
            end = w.n0 == 0 && w.n1 == 0;
            if (!end) cs.start(w);
          }
          if (ahead < C::BUFS && keys_there()) {
            tc_fence_after();
            issue_s();
            t0 = 0;
            continue;
          }
          if (ahead > 0) {
            if (!cv.open) cv.start(s_brief[items_v++ % kBriefs]);
            if (mbar_test(p_half(cv.b), (p_ph >> cv.b) & 1u)) {
              const int s = cv.stage + 1 == C::STAGES ? 0 : cv.stage + 1;
              if (cv.first()) {
                if (cv.i >= cv.w.edge) {
                  ok = mbar_wait(ready_bar(s), (ready_ph >> s) & 1u, abort_flag, budget);
                  ready_ph ^= 1u << s;
                } else {
                  ok = mbar_wait(full_bar(s), (full_ph >> s) & 1u, abort_flag, budget);
                  full_ph ^= 1u << s;
                }
                if (!ok) break;
              }
              // (P of a half's first key tile also says that its warps have read O of the item before)
              const uint32_t d = tmem + C::O_COL + C::O_COLS * cv.h, a0 = tmem + 128u * cv.b, id_o = id_o0 | (HALF ? cv.w.type : kBf16);
              const uint32_t v0 = desc_low(ring + s * C::TILE, C::CHUNK);
              tc_fence_after();
#pragma unroll
              for (int k = 0; k < kKeys / 32; ++k) tc_mma_ts(d, a0 + 8u * k, v0 + 128u * k, id_o, cv.i > 0 || k > 0);
              const bool more = keys_there();            // (before the wait: S of the next job follows the product at once)
              ok = mbar_wait(p_full(cv.b), (p_ph >> cv.b) & 1u, abort_flag, budget);
              p_ph ^= 1u << cv.b;
              if (!ok) break;
              tc_fence_after();
#pragma unroll
              for (int k = kKeys / 32; k < kKeys / 16; ++k) tc_mma_ts(d, a0 + 8u * k, v0 + 128u * k, id_o, 1u);
              --ahead;
              if (C::BUFS == 2 && more) issue_s();       // (with three: 184 us for the documents)
              tc_commit_one(pv_done(cv.h));
              if (cv.last()) tc_commit_one(empty_bar(s));
              cv.advance(C::BUFS, C::STAGES);
              t0 = 0;
              continue;
            }
          } else if (end) {
            break;
          }
          if (t0 == 0) {
            t0 = clock64();
          } else if (clock64() - t0 > budget) {
            *abort_flag = 1;
          }
          if (*abort_flag) {
            ok = false;
            break;
          }
        }
        if (!ok) report_status(p.a.status, SP_ERR_TIMEOUT, (int32_t)blockIdx.x, 12);
        // (in a complete run the epilogues have seen the last products; this matters when a role gave up)
        if (issued && (!ok || *abort_flag)) {
          tc_commit_one(drain_bar);
          const long long t1 = clock64();
          while (!mbar_try(drain_bar, 0u) && clock64() - t1 < kDrainBudget) {}
        }
      }
      __syncwarp();
    } else {
      // ------------------------------------------------------------------------------------------------ edge tiles of V
      const int tid = threadIdx.x - 320;               // 0 .. 63
      uint32_t pos = 0, edge_ph = 0;
      bool ok = true;
      long long patience = budget;                     // (these warps wait for as long as the others work on an item)
      for (int k = 0; ok && next_item(k, ok, patience); ++k) {
        // a bf16 (fp16) of all-ones exponent: its magnitude plus this reaches the sign bit
        const uint32_t to_sign = HALF && s_units[k % kItems].half ? 0x04000400u : 0x00800080u;
        item_read(k);
        const Work w = work_of(p, it);
        const int n = w.tiles();
        if (n == 0) continue;
        patience = budget + 20000ll * n;
        for (int i = 0; i < n && ok; ++i, pos += 2) {
          if (!w.edge(i)) continue;
          const int s = (int)((pos + 1) % C::STAGES);
          const bool got = mbar_wait(edge_bar(s), (edge_ph >> s) & 1u, abort_flag, patience);
          edge_ph ^= 1u << s;
          ok = __all_sync(0xffffffffu, got);
          if (!ok) break;
          const int k0 = w.kb + i * kKeys;
          uint8_t* tile = smem_raw + (ring - raw) + (size_t)s * C::TILE;
          bool found = false;
          for (int j = tid; j < kKeys; j += 64) {
            if (k0 + j < w.sure) continue;             // seen by every row
            const bool clear = k0 + j >= w.seen;
  #pragma unroll
            for (int c = 0; c < C::CH; ++c)
  #pragma unroll
              for (int x = 0; x < 8; ++x) {
                uint4* at = reinterpret_cast<uint4*>(tile + c * C::CHUNK + j * 128 + ((x + j) & 7) * 16);
                if (clear) {
                  *at = make_uint4(0u, 0u, 0u, 0u);
                } else {
                  const uint4 v = *at;
                  auto mark = [to_sign](uint32_t u) { return ((u & 0x7fff7fffu) + to_sign) & 0x80008000u; };
                  if (mark(v.x) | mark(v.y) | mark(v.z) | mark(v.w)) {
                    auto fix = [&](uint32_t u) {
                      const uint32_t b = mark(u);
                      return u & ~((b & 0x8000u ? 0xffffu : 0u) | (b & 0x80000000u ? 0xffff0000u : 0u));
                    };
                    *at = make_uint4(fix(v.x), fix(v.y), fix(v.z), fix(v.w));
                    found = true;
                  }
                }
              }
          }
          if (found) *reinterpret_cast<volatile int*>(&s_bad[seq % kBadSlots]) = seq;
          fence_async_smem();                          // the tensor core reads what was written here
          __syncwarp();
          if (lane == 0) mbar_arrive(ready_bar(s));
        }
        ++seq;
      }
      if (!ok && lane == 0) report_status(p.a.status, SP_ERR_TIMEOUT, (int32_t)blockIdx.x, 13);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    // ------------------------------------------------------------------------------------------------ softmax and output
    const int h = warp >> 2, q = warp & 3;
    const int row = q * 32 + lane;                   // of the half, and lane of tensor memory
    const uint32_t lanes = (uint32_t)(q * 32) << 16;
    const uint32_t t_o = tmem + C::O_COL + C::O_COLS * h + lanes;
    uint32_t s_ph = 0, pv_ph = 0, jobs = 0;          // (of a buffer: a bit each; jobs of the items before)
    bool ok = true;
    int waits = 0;                                   // key tiles of the item before: half 1 waits for as long as half 0 works on one alone
    for (int k = 0; ok && next_item(k, ok, budget + 20000ll * waits); ++k) {
      int lim, n, n0, kb;                            // (a row of S leaves few registers: the rest is derived again for the output)
      bool alone, busy;
      float c = p.a.scale_log2;                      // of a value of S to base 2
      {
        const Work w = work_of(p, it);
        const int token = w.t0 + h * p.tokens + row / p.gp;
        const bool valid = row < p.gp * p.tokens && token < it.nq;
        lim = valid ? min(visible(it, p.a.causal, token), w.seen) : 0;       // keys [0, lim)
        busy = __any_sync(0xffffffffu, valid);
        n0 = w.n[0];
        n = h ? w.n[1] : n0;
        kb = w.kb;
        alone = w.alone;
        if (HALF) {
          const int head = p.gp == 1 ? it.head : it.head * p.gp + row % p.gp;
          c *= s_units[k % kItems].k * (valid ? p.a.half_q[((int64_t)it.q0 + token) * p.a.n_heads + head] : 1.f);
          if (c < 1.2e-38f) c = 1.2e-38f;            // (0 times the mask's -infinity would be NaN; S is below 2^38)
        }
      }
      const uint64_t c2 = pack2(c, c);
      float r = -INFINITY, l = 0.f;                  // reference (not yet times c) and sum
      for (int i = 0; i < n; ++i) {
        const int b_ = (int)((jobs + (alone ? i : i < n0 ? 2 * i + h : n0 + i)) % C::BUFS);      // the buffer of the job
        const uint32_t t_s = tmem + 128u * b_ + lanes;
        bool got = mbar_wait(s_full(h, b_), (s_ph >> b_) & 1u, abort_flag, budget);
        s_ph ^= 1u << b_;
        ok = __all_sync(0xffffffffu, got);
        if (!ok) break;
        bool o_still = i == 0;                       // the product of the tile before may still add to O
        auto wait_o_still = [&] {
          if (o_still) return;
          got = mbar_wait(pv_done(h), pv_ph, abort_flag, budget);
          pv_ph ^= 1u;
          o_still = true;
          ok = __all_sync(0xffffffffu, got);
        };
        if (busy) {
          tc_fence_after();
          uint32_t x[128];
#pragma unroll
          for (int b = 0; b < 4; ++b) tc_ld32(t_s + 32u * b, x + 32 * b);
          tc_wait_ld();
          const int left = lim - (kb + i * kKeys);   // keys of this tile that the row sees
          if (__any_sync(0xffffffffu, left < kKeys)) {
#pragma unroll
            for (int j = 0; j < kKeys; ++j)
              if (j >= left) x[j] = 0xff800000u;
          }
          float m8[8];
#pragma unroll
          for (int y = 0; y < 8; ++y)
            m8[y] = max_nan(__uint_as_float(x[3 * y]), __uint_as_float(x[3 * y + 1]), __uint_as_float(x[3 * y + 2]));
#pragma unroll
          for (int j = 24; j + 16 <= kKeys; j += 16)
#pragma unroll
            for (int y = 0; y < 8; ++y) m8[y] = max_nan(m8[y], __uint_as_float(x[j + 2 * y]), __uint_as_float(x[j + 2 * y + 1]));
          static_assert((kKeys - 24) % 16 == 8, "the last eight");
#pragma unroll
          for (int y = 0; y < 4; ++y)
            m8[y] = max_nan(m8[y], __uint_as_float(x[kKeys - 8 + 2 * y]), __uint_as_float(x[kKeys - 7 + 2 * y]));
          const float m = max_nan(max_nan(m8[0], m8[1], m8[2]), max_nan(m8[3], m8[4], m8[5]), max_nan(m8[6], m8[7], m8[7]));
          // the reference follows a maximum that has risen by more than 2^8 (from -infinity: by anything), and a NaN
          const bool rise = m != -INFINITY && !((m - r) * c <= 8.f);
          if (__any_sync(0xffffffffu, rise)) {
            const float f = rise ? exp2_fast((r - m) * c) : 1.f;       // r = -infinity: 0
            if (rise) r = m;
            l *= f;
            if (i > 0) {
              wait_o_still();
              if (!ok) break;
              tc_fence_after();
#pragma unroll 1
              for (int b = 0; b < DH / 32; ++b) {
                uint32_t o[32];
                tc_ld32(t_o + 32u * b, o);
                tc_wait_ld();
#pragma unroll
                for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                tc_st32(t_o + 32u * b, o);
              }
            }
          }
          const float shift = r == -INFINITY ? 0.f : HALF ? fmaf(-r, c, kHalfLift) : -r * c;
          const uint64_t shift2 = pack2(shift, shift);
          uint64_t l2[2] = {pack2(l, 0.f), pack2(0.f, 0.f)};
          const auto put_p = [&](auto fp16) {
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            uint32_t w16[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const uint64_t t = fma2(pack2(__uint_as_float(x[32 * b + 2 * j]), __uint_as_float(x[32 * b + 2 * j + 1])), c2, shift2);
              float e0, e1;
              unpack2(t, e0, e1);
              e0 = exp2_fast(e0);
              e1 = exp2_fast(e1);
              l2[j & 1] = add2(l2[j & 1], pack2(e0, e1));
              if constexpr (decltype(fp16)::value) {
                const __half2 e = __floats2half2_rn(e0, e1);
                w16[j] = *reinterpret_cast<const uint32_t*>(&e);
              } else {
                const __nv_bfloat162 e = __floats2bfloat162_rn(e0, e1);
                w16[j] = *reinterpret_cast<const uint32_t*>(&e);
              }
            }
            if (b < 2) tc_st16(t_s + 16u * b, w16);
            if (b == 2) {                            // the tensor core starts on the first half (stored while this quarter was computed)
              tc_wait_st();
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(p_half(b_));
            }
            if (b >= 2) tc_st16(t_s + 16u * b, w16);
          }
          };
          if (HALF && s_units[k % kItems].half) put_p(std::integral_constant<bool, HALF>());
          else put_p(std::false_type());
          float l0, l1;
          unpack2(add2(l2[0], l2[1]), l0, l1);
          l = l0 + l1;
          tc_wait_st();
          tc_fence_before();
        }
        if (!busy && lane == 0) mbar_arrive(p_half(b_));
        wait_o_still();      // at the latest here, so that no phase of the barrier is passed over
        if (!ok) break;
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(b_));
      }
      if (!ok) break;
      // ---- output of the item
      it = s_item[k % kItems];
      const Work w = work_of(p, it);
      const int token = w.t0 + h * p.tokens + row / p.gp;
      const bool valid = row < p.gp * p.tokens && token < it.nq;
      const int64_t out_row = (int64_t)it.q0 + token;
      const int head = p.gp == 1 ? it.head : it.head * p.gp + row % p.gp;
      const bool cut = p.a.part > 0 && it.nk > p.a.part;
      // no key seen: no reference r.  With one, 2^(c (x - r)) of the row's largest logit is 1 or more, unless c r is beyond fp32: then the row is NaN.
      const bool none = r == -INFINITY;
      const bool half = HALF && s_units[k % kItems].half;
      const float unit = HALF ? s_units[k % kItems].v : 1.f;
      const float inv = l == 0.f ? NAN : unit / l;
      const float lse2 = none ? -INFINITY : l == 0.f ? NAN : fmaf(r, c, log2f(l) - (HALF ? kHalfLift : 0.f));
      __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.a.o) + out_row * p.a.ldo + (int64_t)head * p.a.dh;
      float* part = cut ? p.a.part_o + ((int64_t)it.c * p.a.Nq + out_row) * ((int64_t)p.a.n_heads * p.a.dh) + (int64_t)head * p.a.dh
                        : nullptr;
      bool bad = false;
      if (n > 0) {
        const bool got = mbar_wait(pv_done(h), pv_ph, abort_flag, budget);
        pv_ph ^= 1u;
        ok = __all_sync(0xffffffffu, got);
        if (!ok) break;
        tc_fence_after();
        bad = *reinterpret_cast<volatile int*>(&s_bad[seq % kBadSlots]) == seq;
      }
      if (busy) {
#pragma unroll 1
        for (int b = 0; b < DH / 32; ++b) {
          uint32_t o[32];
          __syncwarp();                              // (lanes without a row skipped the rest of the round before)
          if (n > 0) {
            tc_ld32(t_o + 32u * b, o);
            tc_wait_ld();
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = 0u;
          }
          if (!valid || 32 * b >= p.a.dh) continue;
          float f[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) f[j] = none ? 0.f : __uint_as_float(o[j]) * inv;
          if (bad) {
            // values of V that the edge warps set to zero, for the rows that do see them
            const int kvh = p.gp == 1 ? it.head / p.a.g : it.head;
            const __nv_bfloat16* V = reinterpret_cast<const __nv_bfloat16*>(p.a.v) + (int64_t)kvh * p.a.dh + 32 * b;
            for (int key = max(w.sure, w.kb); key < lim; ++key)
#pragma unroll 1
              for (int j = 0; j < 32 && 32 * b + j < p.a.dh; ++j) {
                const float v = half ? __half2float(reinterpret_cast<const __half*>(V)[((int64_t)it.k0 + key) * p.a.ldv + j])
                                     : __bfloat162float(V[((int64_t)it.k0 + key) * p.a.ldv + j]);
                if (!(fabsf(v) < INFINITY)) {
#pragma unroll
                  for (int y = 0; y < 32; ++y)
                    if (y == j) f[y] += v;
                }
              }
          }
          if (cut) {
#pragma unroll
            for (int j = 0; j < 32; j += 4)
              if (32 * b + j < p.a.dh) *reinterpret_cast<float4*>(part + 32 * b + j) = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
          } else if (p.vec_out) {
#pragma unroll
            for (int j = 0; j < 32; j += 8)
              if (32 * b + j < p.a.dh) {
                uint32_t u[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                  const __nv_bfloat162 e = __floats2bfloat162_rn(f[j + 2 * y], f[j + 2 * y + 1]);
                  u[y] = *reinterpret_cast<const uint32_t*>(&e);
                }
                *reinterpret_cast<uint4*>(out + 32 * b + j) = make_uint4(u[0], u[1], u[2], u[3]);
              }
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (32 * b + j < p.a.dh) out[32 * b + j] = __float2bfloat16_rn(f[j]);
          }
        }
        if (valid) {
          if (cut) p.a.part_lse[((int64_t)it.c * p.a.Nq + out_row) * p.a.n_heads + head] = lse2;
          else if (p.a.lse) p.a.lse[out_row * p.a.n_heads + head] = lse2 == -INFINITY ? lse2 : lse2 * 0.6931471805599453f;
        }
      }
      tc_fence_before();                             // (the next P of this half says that O has been read)
      jobs = (jobs + w.n[0] + w.n[1]) % C::BUFS;
      waits = w.tiles();
      if (waits > 0) ++seq;
      item_read(k);
    }
    if (!ok && lane == 0) report_status(p.a.status, SP_ERR_TIMEOUT, (int32_t)blockIdx.x, 14);
  }
  tc_fence_before();
  __syncthreads();
  if (s_abort) {              // a role gave up: copies that another one had in flight land before shared memory is released
    const long long t0 = clock64();
    while (clock64() - t0 < kDrainBudget) {}
  }
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

template <int DH, bool HALF>
sp_status launch_tc(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const TcAttnParams& p, int64_t work,
                    cudaStream_t stream) {
  static PerDeviceOnce attr_once;
  const auto kernel = attention_tc_kernel<DH, HALF>;
  if (attr_once.run([&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg<DH>::SMEM);
      }) != cudaSuccess)
    return SP_ERR_CUDA;
  const dim3 grid((unsigned)(work < sm_count() ? work : sm_count()));
  return launch(kernel, grid, dim3(kThreads), Cfg<DH>::SMEM, stream, tmQ, tmK, tmV, p) == cudaSuccess ? SP_OK : SP_ERR_CUDA;
}

}  // namespace

bool attention_tc_supported(const AttnParams& a) {
  const auto fits = [](const void* ptr, int64_t ld) { return ld % 8 == 0 && (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; };
  return a.dh % 8 == 0 && a.dh <= 128 && a.Nk > 0 && fits(a.q, a.ldq) && fits(a.k, a.ldk) && fits(a.v, a.ldv);
}

sp_status attention_tc(const AttnParams& a, cudaStream_t stream) {
  TcAttnParams p;
  p.a = a;
  p.a.wait_budget = wait_budget_cycles() > 0 ? wait_budget_cycles() : kWaitBudget;
  // Heads that share a key head fill the rows of a tile together.  Groups of more than half a tile would leave too many rows
  // empty: their heads go one by one.
  p.gp = a.g <= kRows / 2 ? a.g : 1;
  p.tokens = kRows / p.gp;
  p.heads = p.gp == 1 ? a.n_heads : a.n_kv;
  p.vec_out = a.ldo % 8 == 0 && (reinterpret_cast<uintptr_t>(a.o) & 15u) == 0;
  CUtensorMap tmQ, tmK, tmV;
  if (!make_map3(&tmQ, a.q, a.dh, a.n_heads, a.Nq, a.dh, a.ldq, 64, p.gp, p.tokens) ||
      !make_map3(&tmK, a.k, a.dh, a.n_kv, a.Nk, a.dh, a.ldk, 64, 1, kKeys) ||
      !make_map3(&tmV, a.v, a.dh, a.n_kv, a.Nk, a.dh, a.ldv, 64, 1, kKeys))
    return SP_ERR_CUDA;
  const int64_t tiles = min((int64_t)a.Nq / (2 * p.tokens) + a.n_seq, (int64_t)a.Nq);
  const int64_t work = tiles * p.heads * (a.part > 0 ? a.max_parts : 1);
  if (a.half_tops) return a.dh <= 64 ? launch_tc<64, true>(tmQ, tmK, tmV, p, work, stream) : launch_tc<128, true>(tmQ, tmK, tmV, p, work, stream);
  return a.dh <= 64 ? launch_tc<64, false>(tmQ, tmK, tmV, p, work, stream) : launch_tc<128, false>(tmQ, tmK, tmV, p, work, stream);
}

}  // namespace sp
