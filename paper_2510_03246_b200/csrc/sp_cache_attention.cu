// Attention over a paged cache.
//
//   O_i = sum_j p_ij V_j, p = softmax(scale Q K^T), keys and values in pages; in 4 bits K_j = s_j n_j + z_j by groups of 64 channels, so that
//   <Q_i, K_j> = sum_g s_jg sum_c q_ic n_jc + z_jg sum_c q_ic and O_ic = sum_j (p_ij s_jg) n_jc + sum_j p_ij z_jg: the matrix instructions
//   contract the numbers themselves, and scales and offsets go to logits and probabilities.
//
// Few rows (queries x the heads that share a key head) stream the cache past them; what bounds that is reading it once, and in 4 bits as
// much the instructions that open the numbers.  Each of eight warps brings its own blocks of 16 keys in by 16-byte asynchronous copies, a ring of
// stages ahead, so that no warp waits for another before the end of a piece.  Products are m16n8k16 of bf16, turned so that keys and channels
// fill them: S^T = K Q^T and O^T += V^T P^T.  The order in which an instruction contracts channels is free, and so is the channel that a row of
// V^T stands for.  In 4 bits a lane therefore takes whole words of eight numbers as they lie: for K the two words 2 t4, 2 t4 + 1 of a group, for V
// word g4 of four keys.
//   K: the byte of a number n is n / 512 as e4m3 (the values below the first power of two and above it lie equally close), so that a mask opens
//   four of them for m16n8k32 of e4m3, a faster instruction too.  Queries are two e4m3 parts, eight bits of what a power of two per row takes to
//   128 .. 255, the second 2^5 times as large, with sums of its own; what is lost lies 2^-22 and more below a row's largest value.  (In one unit it was 2^-17, and
//   lse off by 2e-6 of its size.)
//   V: number n becomes the fp16 64 + n by a shift and one logical operation, two at a time; a second instruction with a constant takes 72 away
//   again, so that n - 8 is left.  Probabilities times scales are fp16 as well, in units of a power of two that follows the scales: with bf16
//   their roundings left 2.4e-3 of the result's norm (16 tokens after 2048 .. 31013 keys), with fp16 1.7e-3, the result's own.
// fp32 queries are three bf16 parts that add up to them, as are the probabilities' products with the scales; numbers are bf16 for both products, and
// sums of 16 keys are added up outside the matrix unit.
//
// More rows of bf16 open the pages into rows of the workspace and take sp_attention: a tile of 128 rows reads opened keys at the tensor cores' rate, where this
// form would open them again for every 16 rows.  4 bits are opened into fp16 in units of a text's key head (bf16 queries in those of a row): rounded to bf16,
// results were 4.2e-3 from the formula (512 queries after 16384 keys, 32 heads of 128 on 8), and as two bf16 parts each 2.3e-3, in 312 us instead of
// 192; in fp16 they are 1.7e-3 from it.  (Rounded values of equal scales are all off by the same, which no sum over keys takes away.)
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <math.h>

#include <type_traits>

#include "sp_attention.cuh"
#include "sp_cache.cuh"
#include "sp_f32x2.cuh"

namespace sp {
namespace {

constexpr int kBlock = 16;
constexpr int kPlanSeqs = 128;             // sequences of a launch
constexpr int kLead = 64;                  // what a tile and head costs beside its blocks of keys, in those
constexpr int kLeastShare = 16;            // of the line of work to a thread block, at least
constexpr int kMostCtas = 2 * 148;         // thread blocks of a launch, at most
constexpr int kPlanThreads = 256;
constexpr float kNoWeight = -3.402823466e38f;      // lse of a piece whose keys are seen and have none
constexpr uint32_t kNoPage = 0xffffffffu;

struct PagedParams {
  CacheView c;
  const void* q;
  void* o;
  int64_t ldq, ldo;
  float* lse;
  const int32_t* cu_q;
  int32_t Nq, n_heads, g, causal;
  int32_t s0, n_here;                      // sequences of this launch
  float scale_log2;
  int64_t* plan;                           // [n_here + 1] where each sequence's work starts, then the thread blocks that share it
  float* part_o;                           // [2 kMostCtas, row, dh]
  float* part_lse;                         // [2 kMostCtas, row] in base 2
  int32_t* status;
};

template <int DH, bool FOUR>
struct Ring {
  static constexpr int PIECES = DH / 8;                                     // 16-byte pieces of a key's row, bf16
  static constexpr int PITCH = FOUR ? DH / 2 : (PIECES | 1) * 16;           // bytes from a key to the next (bf16: an odd number of pieces,
                                                                            // so that eight rows' pieces lie in different banks)
  static constexpr int TILE = kBlock * PITCH;                               // K or V of a stage
  static constexpr int G = DH / kCacheGroup;
  static constexpr int SCALES = FOUR ? kBlock * G * 4 : 0;
  static constexpr int STAGE = 2 * TILE + 2 * SCALES;
  static constexpr int STAGES = FOUR ? (DH == 128 ? 5 : 8) : 3;
  static constexpr int BYTES = STAGES * STAGE;                              // of a warp
};
template <int DH, bool FOUR, int ROWS, int PARTS>
struct PagedCfg {
  using R = Ring<DH, FOUR>;
  static constexpr int PITCH = DH + 4;                                      // floats of a row of a warp's O
  static constexpr int JOIN = ROWS * (PITCH + 2) * 4;                       // a warp's results, in its own ring
  static constexpr int WARP = (R::BYTES > JOIN ? R::BYTES : JOIN) / 128 * 128 + 128;
  // Warps of a block and blocks of an SM: twice 8 (128 registers of a thread), for 16 rows of wide heads in 4 bits once 12 (168), once 8 where
  // the ring, or three parts of wide queries, need an SM for themselves.
  static constexpr bool ALONE = 8 * WARP > 113 * 1024 || (PARTS > 1 && DH > 64);
  static constexpr bool TWELVE = !ALONE && FOUR && DH == 128 && ROWS > 8;
  static constexpr int W = TWELVE ? 12 : 8, CTAS = ALONE || TWELVE ? 1 : 2, THREADS = 32 * W;
  static constexpr size_t SMEM = (size_t)W * WARP;
};

__device__ __forceinline__ uint32_t shared_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_half(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_e4m3(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_turned(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t turned8x8(uint32_t a) {       // 8 x 8 values of two bytes: row g4, columns 2 t4 and 2 t4 + 1
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
  uint32_t r;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r) : "r"(addr) : "memory");
  return r;
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
  uint2 r;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(addr) : "memory");
  return r;
}
// The fp16 pair (64 + n_i, 64 + n_{i + 4}) of a word of eight numbers: the mantissa's last bit of 64 .. 127 is 1 / 16, so that a number stands in
// bits 4 .. 7, where number 1 stands already.
template <int I>
__device__ __forceinline__ uint32_t opened(uint32_t w) {
  const uint32_t at = I == 0 ? w * 16u : w >> (I == 0 ? 0 : 4 * I - 4);
  return (at & 0x00f000f0u) | 0x54005400u;
}
// The same as bf16 and n - 8, for fp32: sums of larger numbers would round by more.
__device__ __forceinline__ uint32_t opened_centred(uint32_t w, int i) {
  const uint32_t at = i == 0 ? w << 3 : w >> (4 * i - 3), v = (at & 0x00780078u) | 0x41804180u;
  const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), __floats2bfloat162_rn(24.f, 24.f));
  return *reinterpret_cast<const uint32_t*>(&d);
}
template <int I>
__device__ __forceinline__ uint32_t opened_centred(uint32_t w) { return opened_centred(w, I); }
// four values as e4m3, the first in the lowest byte
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3) |
         (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3) << 16;
}
// kLeftUnits (a - packed): of a value below 2^8 at most 2^3 is left, so that 2^5 of it stay below 448
constexpr float kLeftUnits = 32.f;
__device__ __forceinline__ uint32_t left_of_e4m3(const float (&a)[4], uint32_t packed) {
  const __half2 lo = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(packed & 0xffffu), __NV_E4M3));
  const __half2 hi = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(packed >> 16), __NV_E4M3));
  return pack_e4m3(kLeftUnits * (a[0] - __low2float(lo)), kLeftUnits * (a[1] - __high2float(lo)), kLeftUnits * (a[2] - __low2float(hi)),
                   kLeftUnits * (a[3] - __high2float(hi)));
}
__device__ __forceinline__ float low(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float high(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 e = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&e);
}
// PARTS bf16 pairs that add up to (lo, hi): one is the values rounded, three are exact
template <int PARTS>
__device__ __forceinline__ void split(float lo, float hi, uint32_t (&r)[PARTS]) {
#pragma unroll
  for (int i = 0; i < PARTS; ++i) {
    r[i] = pack_bf16(lo, hi);
    if (i + 1 < PARTS) {
      lo -= low(r[i]);
      hi -= high(r[i]);
    }
  }
}
// Two parts of numbers that are not negative, both above 0 where the number is: times an infinite value they are infinite, not NaN.  (Less its last
// bit a number is cut to bf16; the rest is rounded: 2^-15 of the number.)
__device__ __forceinline__ void split_above_zero(float lo, float hi, uint32_t (&r)[2]) {
  constexpr float kBelow = 0x1.fffffep-1f;
  r[0] = __byte_perm(__float_as_uint(lo * kBelow), __float_as_uint(hi * kBelow), 0x7632);
  r[1] = pack_bf16(lo - low(r[0]), hi - high(r[0]));
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 e = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&e);
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// A value that all lanes of a warp have, as the compiler can know it: loops and addresses then need no lane's registers, and branches no
// meeting points.
__device__ __forceinline__ int32_t uniform(int32_t x) { return __shfl_sync(0xffffffffu, x, 0); }

// What a sequence brings: its rows of queries and its keys.
struct Seq {
  int32_t q0, nq, nk;
};
__device__ __forceinline__ Seq seq_at(const PagedParams& p, int32_t s) {
  Seq r;
  r.q0 = bounded(p.cu_q[s], p.Nq);
  r.nq = max(0, bounded(p.cu_q[s + 1], p.Nq) - r.q0);
  r.nk = r.nq > 0 ? max(0, p.c.lens[s]) : 0;
  return r;
}
template <int ROWS>
__device__ __forceinline__ int32_t tiles_of(const PagedParams& p, const Seq& s) {
  return (int32_t)(((int64_t)s.nq * p.g + ROWS - 1) / ROWS);
}
// blocks of keys of a tile (one at least: a tile without keys has rows to write)
__device__ __forceinline__ int32_t blocks_of(int32_t nk) { return nk > 0 ? (nk - 1) / kBlock + 1 : 1; }
__device__ __forceinline__ int32_t visible(int32_t nk, int64_t shift, int64_t token) {
  return (int32_t)max((int64_t)0, min((int64_t)nk, token + shift + 1));
}

// The work of a launch is a line of blocks: sequence by sequence, of each its tiles of rows, of each the key heads, of each kLead that stand for
// its queries and its output (some microseconds; without them 12 texts of 700 .. 11447 keys kept SMs busy for half of the time: 76 us, with 32 52, with
// 64 46), and the blocks of keys.  `ctas` thread blocks share it in equal pieces: the b-th has [b total / ctas, (b + 1) total / ctas).  A tile and head
// that lies in several thread blocks' pieces is joined from what they leave: the one that goes on in it from a predecessor at 2 b, the one that begins it at 2 b + 1.
__device__ __forceinline__ int64_t first_of(int64_t b, int64_t total, int64_t ctas) { return b * total / ctas; }
__device__ __forceinline__ int64_t cta_of(int64_t x, int64_t total, int64_t ctas) { return ((x + 1) * ctas - 1) / total; }

// sum over the block's threads, and what stands before this one's
template <int WARPS>
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* s_word, int64_t& before) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t upto = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t t = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += t;
  }
  __syncthreads();
  if (lane == 31) s_word[warp] = upto;
  __syncthreads();
  int64_t sum = 0, below = 0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    if (w < warp) below += s_word[w];
    sum += s_word[w];
  }
  before = below + upto - v;
  return sum;
}

template <typename T, int DH, bool FOUR, int ROWS>
__global__ void __launch_bounds__((PagedCfg<DH, FOUR, ROWS, sizeof(T) == 4 ? 3 : 1>::THREADS), (PagedCfg<DH, FOUR, ROWS, sizeof(T) == 4 ? 3 : 1>::CTAS))
paged_rows_kernel(const PagedParams p) {
  kernel_begin();
  using C = PagedCfg<DH, FOUR, ROWS, sizeof(T) == 4 ? 3 : 1>;
  using R = typename C::R;
  constexpr int H = ROWS / 8, PARTS = sizeof(T) == 4 ? 3 : 1, G = FOUR ? R::G : 1, K16 = DH / 16, W = C::W;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int64_t s_first[kPlanSeqs + 1];
  __shared__ Seq s_seq[kPlanSeqs];
  __shared__ int64_t s_word[W];
  __shared__ int s_bad;
  const int lane = threadIdx.x & 31, warp = uniform((int)threadIdx.x >> 5), g4 = lane >> 2, t4 = lane & 3;
  const int n_kv = p.c.n_kv, dh = FOUR ? DH : p.c.dh;

  // The plan, the same in every block: where the work of each sequence starts.
  {
    const int per = (p.n_here + C::THREADS - 1) / C::THREADS;    // consecutive sequences of a thread
    const int i0 = (int)threadIdx.x * per, i1 = min(i0 + per, p.n_here);
    int64_t mine = 0, before;
    for (int i = i0; i < i1; ++i) {
      const Seq s = seq_at(p, p.s0 + i);
      s_seq[i] = s;
      s_first[i] = (int64_t)tiles_of<ROWS>(p, s) * n_kv * (kLead + blocks_of(s.nk));
      mine += s_first[i];
    }
    const int64_t all = block_scan<W>(mine, s_word, before);
    for (int i = i0; i < i1; ++i) {
      const int64_t n = s_first[i];
      s_first[i] = before;
      before += n;
    }
    if (threadIdx.x == 0) s_first[p.n_here] = all;
    __syncthreads();
  }
  const int64_t total = s_first[p.n_here];
  const int64_t ctas = max((int64_t)1, min((int64_t)gridDim.x, total / kLeastShare));
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i <= p.n_here; i += C::THREADS) p.plan[i] = s_first[i];
    if (threadIdx.x == 0) p.plan[p.n_here + 1] = ctas;
  }
  if (blockIdx.x >= ctas) return;
  int64_t at = first_of(blockIdx.x, total, ctas);
  const int64_t end = first_of((int64_t)blockIdx.x + 1, total, ctas);

  // Where a lane's piece of 16 bytes goes, and where its words stand, in a stage (4 bits; see fetch).  Eight keys further, in rows of 32 bytes,
  // the line's number has changed by two.
  constexpr uint32_t kFlip = DH == 64 ? 0x40u : 0u;
  const uint32_t piece_to = (16u * lane) ^ ((4u * lane) & 0x60u);
  const uint32_t k_row = (uint32_t)(g4 * (DH / 2) + 8 * t4), k_at = k_row ^ ((k_row >> 2) & 0x60u);
  uint32_t v_at[2][G];
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int gr = 0; gr < G; ++gr) {
      const uint32_t byte = (uint32_t)((2 * t4 + x) * (DH / 2) + 32 * gr + 4 * g4);
      v_at[x][gr] = byte ^ ((byte >> 2) & 0x60u);
    }
  uint8_t* mine = smem + warp * C::WARP;
  const uint32_t ring = shared_at(mine);
  float* s_o = reinterpret_cast<float*>(mine);                   // [row][PITCH], after a piece's last block
  while (at < end) {
    // the last sequence whose work starts at or before `at`
    int lo = 0, hi = p.n_here;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (s_first[mid] <= at) lo = mid;
      else hi = mid;
    }
    const int32_t sq = p.s0 + lo;
    const Seq it = s_seq[lo];
    const uint32_t all_blocks = (uint32_t)blocks_of(it.nk), of_tile = kLead + all_blocks;
    const int64_t from_seq = at - s_first[lo], unit_ = from_seq / of_tile;
    const uint32_t from = (uint32_t)(from_seq - unit_ * of_tile);                    // of the tile and head
    const uint32_t to = (uint32_t)min((int64_t)of_tile, from + end - at);
    at += to - from;
    if (to <= kLead) continue;                                                       // (no block of keys: the next thread block begins)
    const uint32_t block0 = from > kLead ? from - kLead : 0u, piece = to - kLead - block0;
    const uint32_t tile = (uint32_t)(unit_ / n_kv);
    const int32_t head = (int32_t)(unit_ - (int64_t)tile * n_kv);
    const bool cut = piece < all_blocks;
    const int32_t slot_of = 2 * (int32_t)blockIdx.x + (block0 == 0 ? 1 : 0);
    const uint32_t g = (uint32_t)p.g, r0 = tile * ROWS;
    const int rows = (int)min((uint32_t)ROWS, (uint32_t)it.nq * g - r0);
    const int64_t shift = p.causal ? (int64_t)it.nk - it.nq : (int64_t)it.nk;        // query i sees keys j <= i + shift
    const int32_t sure = uniform(visible(it.nk, shift, r0 / g));                     // keys that every row sees
    const int32_t kb = uniform((int32_t)block0 * kBlock);
    int32_t seen = visible(it.nk, shift, (r0 + rows - 1) / g);                       // keys that some row sees
    if (seen - kb > (int32_t)piece * kBlock) seen = kb + (int32_t)piece * kBlock;
    seen = uniform(seen);
    const int32_t blocks = seen > kb ? (seen - kb + kBlock - 1) / kBlock : 0;
    const int32_t own = blocks > warp ? (blocks - warp - 1) / W + 1 : 0;             // this warp's: warp, warp + W, ...

    // ---- copies, on their way before the queries are read: block i of this warp starts at key kb + 16 (warp + W i).  Where 32 of them stand is looked
    // up at a time, a lane each, in units of 128 bytes (kNoPage: there is none) and of 64 for the scales.
    uint32_t places = kNoPage, scale_places = 0u;
    uint32_t missing = 0u;                                       // a bit per block fetched, the last one lowest: it has no page
    uint32_t into = ring + R::BYTES - R::STAGE;                  // the stage that was filled last
    const int row_bytes = FOUR ? DH / 2 : 2 * dh;
    const uint8_t *k_from = p.c.k + 16 * lane, *v_from = p.c.v + 16 * lane;
    const uint8_t* s_from = FOUR ? (lane < 16 ? p.c.ks : p.c.vs) + 16 * (lane & 15) : nullptr;
    const uint32_t s_to = 2 * R::TILE + (lane < 16 ? 0 : R::SCALES) + 16 * (lane & 15);
    const bool has_scale = (lane & 15) < 4 * G;
    const auto fetch = [&](int32_t i) {
      missing <<= 1;
      if (i < own) {
        if ((i & 31) == 0) {
          const int32_t at_ = i + lane, key = kb + kBlock * (warp + W * at_), entry = key / p.c.page_len;
          const int32_t page = at_ < own ? page_of(p.c, sq, entry) : -1;
          const int64_t token = (int64_t)head * p.c.page_len + (key - entry * p.c.page_len);
          places = page < 0 ? kNoPage : (uint32_t)((page * p.c.step + token * row_bytes) >> 7);
          if (FOUR) scale_places = (uint32_t)((page * p.c.scale_step + token * (4 * G)) >> 6);
        }
        const uint32_t place = __shfl_sync(0xffffffffu, places, i & 31);
        into = into + R::STAGE == ring + R::BYTES ? ring : into + R::STAGE;
        if (place == kNoPage) {                                  // (what stands in the stage only meets probabilities that are NaN)
          missing |= 1u;
          copies_end();
          return;
        }
        const uint8_t *k = k_from + (uint64_t)place * 128u, *v = v_from + (uint64_t)place * 128u;
        if constexpr (FOUR) {
#pragma unroll
          for (int e = 0; e < DH / 2; e += 32) {                 // pieces of the block's 16 rows
            // 32-byte quarters of a 128-byte line change places with the line's number: the four keys of a half warp's read of K, and the
            // four pairs of keys of a read of V, lie in different banks
            copy16(into + 16 * e + piece_to, k + 16 * e);
            copy16(into + R::TILE + 16 * e + piece_to, v + 16 * e);
          }
          const uint32_t scale_place = __shfl_sync(0xffffffffu, scale_places, i & 31);
          if (has_scale) copy16(into + s_to, s_from + (uint64_t)scale_place * 64u);
        } else if (dh == DH) {
#pragma unroll
          for (int e = 0; e < kBlock * R::PIECES; e += 32) {
            const int row = e / R::PIECES + lane / R::PIECES;    // (a power of two, at most 32)
            const uint32_t to = into + row * R::PITCH + 16 * (lane % R::PIECES);
            copy16(to, k + 16 * e);
            copy16(to + R::TILE, v + 16 * e);
          }
        } else {
          const int per = dh / 8;
#pragma unroll 1
          for (int e = lane; e < kBlock * per; e += 32) {
            const int row = e / per;
            const uint32_t to = into + row * R::PITCH + 16 * (e - row * per);
            copy16(to, k + 16 * (e - lane));
            copy16(to + R::TILE, v + 16 * (e - lane));
          }
        }
      }
      copies_end();
    };
#pragma unroll
    for (int i = 0; i < R::STAGES - 1; ++i) fetch(i);

    // ---- queries
    uint32_t q[H][PARTS][K16][2];
    float qsum[H][G][2], to_log2[H][2];                          // rows 8 h + 2 t4 + x: 4 bits: sums over a group; logits to base 2
    int32_t lim[H][2];                                           // keys [0, lim) of those rows
    const T* Q = reinterpret_cast<const T*>(p.q);
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const bool valid = 8 * h + g4 < rows;
      const uint32_t rr = valid ? r0 + 8 * h + g4 : r0, token = rr / g;
      const T* src = Q + (it.q0 + (int64_t)token) * p.ldq + ((int64_t)head * g + (rr - token * g)) * dh;
      if constexpr (FOUR) {
        float v[G][2][8], sum[G], top = 0.f;
        bool odd = false;
#pragma unroll
        for (int gr = 0; gr < G; ++gr) {
          sum[gr] = 0.f;
#pragma unroll
          for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float u = valid ? load1(src + 64 * gr + 8 * (2 * t4 + w) + i) : 0.f;
              v[gr][w][i] = u;
              sum[gr] += u;
              top = fmaxf(top, fabsf(u));
              odd |= !(fabsf(u) < INFINITY);
            }
#pragma unroll
          for (int w = 1; w < 4; w <<= 1) sum[gr] += __shfl_xor_sync(0xffffffffu, sum[gr], w);
        }
        float unit = 1.f;                                        // of this row's e4m3 values
        if constexpr (PARTS == 1) {
#pragma unroll
          for (int w = 1; w < 4; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
          // 2^(e - 7) of the exponent e of the largest value; NaN where there is one, or an infinity: every logit is then
          unit = __uint_as_float(max(__float_as_uint(top) >> 23, 20u) - 7u << 23);
          if (__ballot_sync(0xffffffffu, odd) >> (lane & 28) & 15u) unit = NAN;
          const float inv = 1.f / unit;
#pragma unroll
          for (int gr = 0; gr < G; ++gr)
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
              for (int x = 0; x < 2; ++x) {                      // numbers x, x + 2, x + 4, x + 6 of a word stand side by side
                float a[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] = v[gr][w][x + 2 * i] * inv;
                const uint32_t hi = pack_e4m3(a[0], a[1], a[2], a[3]);
                q[h][0][4 * gr + 2 * w][x] = hi;
                q[h][0][4 * gr + 2 * w + 1][x] = left_of_e4m3(a, hi);
              }
        } else {
#pragma unroll
          for (int gr = 0; gr < G; ++gr)
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
              for (int i = 0; i < 4; ++i) {                      // numbers (i, i + 4) of a word stand side by side
                uint32_t r[PARTS];
                split<PARTS>(v[gr][w][i], v[gr][w][i + 4], r);
#pragma unroll
                for (int u = 0; u < PARTS; ++u) q[h][u][4 * gr + 2 * w + i / 2][i & 1] = r[u];
              }
        }
        // what a lane needs of its rows 2 t4 + x: logits come in units of a row
        const float of_sum = PARTS == 1 ? 512.f * unit : 1.f;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const float u = __shfl_sync(0xffffffffu, of_sum, (2 * t4 + x) * 4);
          const float f = u * p.scale_log2;
          to_log2[h][x] = f < 1.2e-38f ? 1.2e-38f : f;           // (0 times the mask's -infinity would be NaN)
#pragma unroll
          for (int gr = 0; gr < G; ++gr) qsum[h][gr][x] = __shfl_sync(0xffffffffu, sum[gr], (2 * t4 + x) * 4) / u;
        }
      } else {
#pragma unroll
        for (int j = 0; j < K16; ++j)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int d = 16 * j + 8 * x + 2 * t4;
            const bool there = valid && d < dh;
            uint32_t r[PARTS];
            split<PARTS>(there ? load1(src + d) : 0.f, there ? load1(src + d + 1) : 0.f, r);
#pragma unroll
            for (int u = 0; u < PARTS; ++u) q[h][u][j][x] = r[u];
          }
        to_log2[h][0] = to_log2[h][1] = p.scale_log2;
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {                              // (rows that are none: any values, kept to themselves)
        const int row = 8 * h + 2 * t4 + x;
        lim[h][x] = row < rows ? min(visible(it.nk, shift, (r0 + row) / g), seen) : seen;
      }
    }
    // 4 bits, bf16: probabilities are taken 2^kLift higher, and O holds them in units of 1 / per_vunit, half of a power of two that no scale has passed
    // yet.  (fp16: at most 2^(8 + kLift) 4, and small ones keep ten bits down to 2^-20 of the reference.)  A scale below 2^-20 of the unit
    // would lose its own: from such a block on, probabilities times scales are three bf16 parts, as for fp32, in units that no longer move.  So a
    // scale of any size, at a key that few rows see or that has no weight, takes nothing from the others.
    constexpr uint32_t kWide = 0x7f807f80u;                      // as vhigh: such a block has been met
    // vhigh: twice the unit, vlow: less one, 2^-20 of it, as bits of bf16, in both halves of a word: two scales are compared at once.
    constexpr bool HALF = FOUR && PARTS == 1;
    constexpr float kLift = HALF ? 5.f : 0.f, kWideUnit = 16777216.f;      // (2^24: no finite scale times a lifted probability leaves fp32)
    constexpr float kOffsetPer = HALF ? 1.f / kWideUnit : 1.f;   // sums of offsets, and what warps join, are in such units for the same reason
    // O: 4 bits: channels 64 (j / 4) + 8 g4 + j % 4 (| + 4) of rows 2 t4 + (x & 1); bf16: channels 16 j + g4 (| + 8)
    float o[K16][H][4], offset[H][G][2], per_vunit = 0.f, r[H][2], ref[H][2], most[H][2], l[H][2];
#pragma unroll
    for (int h = 0; h < H; ++h) {
#pragma unroll
      for (int j = 0; j < K16; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[j][h][x] = 0.f;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        r[h][x] = most[h][x] = -INFINITY;                        // reference of the rows' exponents, the logit up to which it stays
        ref[h][x] = l[h][x] = 0.f;                               // r, 0 while there is none; this lane's part of the rows' sums
#pragma unroll
        for (int gr = 0; gr < G; ++gr) offset[h][gr][x] = 0.f;
      }
    }
    uint32_t vhigh = 0u, vlow = 0u;
    bool found = false;                                          // bf16: non-finite values behind some row's mask

    // The values of a block for probabilities s (HALF, scales of any size): O stands in local memory meanwhile and everything goes step by step, so that
    // a path that is seldom taken costs the others no registers.
    const auto add_wide = [&](int32_t kt, uint32_t stage, const float (&s)[H][4]) {
      float held[H * K16 * 4], held_offset[H * G * 2];
#pragma unroll
      for (int h = 0; h < H; ++h) {
#pragma unroll
        for (int j = 0; j < K16; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x) held[(h * K16 + j) * 4 + x] = o[j][h][x];
#pragma unroll
        for (int gr = 0; gr < G; ++gr)
#pragma unroll
          for (int x = 0; x < 2; ++x) held_offset[(h * G + gr) * 2 + x] = offset[h][gr][x];
      }
#pragma unroll 1
      for (int gr = 0; gr < G; ++gr) {
        uint32_t w[4];                                           // as in add_values
        for (int x = 0; x < 4; ++x) {
          const uint32_t byte = (uint32_t)((2 * t4 + (x & 1)) * (DH / 2) + 32 * gr + 4 * g4);
          w[x] = lds32(stage + R::TILE + ((byte ^ ((byte >> 2) & 0x60u)) ^ (kFlip * (x >> 1))) + 8 * (x >> 1) * (DH / 2));
        }
        const uint32_t m[4] = {__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x5410),
                               __byte_perm(w[2], w[3], 0x7632)};
#pragma unroll
        for (int h = 0; h < H; ++h) {
          uint32_t pb[3][2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const uint32_t pair = lds32(stage + 2 * R::TILE + R::SCALES + ((g4 + 8 * y) * G + gr) * 4);
            const float scale = low(pair), zero = fmaf(8.f * kOffsetPer, scale, kOffsetPer * high(pair));
            float ps[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const bool sees = kt + 8 * y + g4 < lim[h][x];
              ps[x] = sees ? s[h][2 * y + x] * (scale * per_vunit) : 0.f;
              if (sees) held_offset[(h * G + gr) * 2 + x] = fmaf(s[h][2 * y + x], zero, held_offset[(h * G + gr) * 2 + x]);
            }
            uint32_t u[3];
            split<3>(ps[0], ps[1], u);
#pragma unroll
            for (int x = 0; x < 3; ++x) pb[x][y] = turned8x8(u[x]);
          }
#pragma unroll 1
          for (int j = 0; j < 4; ++j) {
            uint32_t a[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) a[x] = opened_centred(m[x], j);
            float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 2; x >= 0; --x) mma(t, a[0], a[1], a[2], a[3], pb[x][0], pb[x][1]);
            for (int x = 0; x < 4; ++x) held[(h * K16 + 4 * gr + j) * 4 + x] += t[x];
          }
        }
      }
#pragma unroll
      for (int h = 0; h < H; ++h) {
#pragma unroll
        for (int j = 0; j < K16; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[j][h][x] = held[(h * K16 + j) * 4 + x];
#pragma unroll
        for (int gr = 0; gr < G; ++gr)
#pragma unroll
          for (int x = 0; x < 2; ++x) offset[h][gr][x] = held_offset[(h * G + gr) * 2 + x];
      }
    };
    uint32_t stage = ring + R::BYTES - R::STAGE;
    for (int32_t i = 0; i < own; ++i) {
      const int32_t kt = kb + kBlock * (warp + W * i);
      fetch(i + R::STAGES - 1);
      copies_wait<R::STAGES - 1>();
      __syncwarp();
      stage = stage + R::STAGE == ring + R::BYTES ? ring : stage + R::STAGE;
      const bool edge = kt + kBlock > sure;
      float s[H][4];                                             // keys kt + g4 | + 8, rows 2 t4, 2 t4 + 1
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int x = 0; x < 4; ++x) s[h][x] = 0.f;
      if constexpr (FOUR) {
        uint32_t pair[2][G];
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int gr = 0; gr < G; ++gr) pair[y][gr] = lds32(stage + 2 * R::TILE + ((g4 + 8 * y) * G + gr) * 4);
#pragma unroll
        for (int gr = 0; gr < G; ++gr) {
          float a[H][4], left[H][4];                             // (left: e4m3 queries' second part)
#pragma unroll
          for (int h = 0; h < H; ++h)
#pragma unroll
            for (int x = 0; x < 4; ++x) a[h][x] = left[h][x] = 0.f;
          uint2 w[2];                                            // keys g4, g4 + 8
#pragma unroll
          for (int y = 0; y < 2; ++y) w[y] = lds64(stage + (k_at ^ (32u * gr + kFlip * y)) + 8 * y * (DH / 2));
          if constexpr (PARTS == 1) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const uint32_t w0 = u == 0 ? w[0].x : w[0].y, w1 = u == 0 ? w[1].x : w[1].y;
              const uint32_t a0 = w0 & 0x0f0f0f0fu, a1 = w1 & 0x0f0f0f0fu, a2 = (w0 >> 4) & 0x0f0f0f0fu, a3 = (w1 >> 4) & 0x0f0f0f0fu;
#pragma unroll
              for (int h = 0; h < H; ++h) {
                mma_e4m3(a[h], a0, a1, a2, a3, q[h][0][4 * gr + 2 * u][0], q[h][0][4 * gr + 2 * u][1]);
                mma_e4m3(left[h], a0, a1, a2, a3, q[h][0][4 * gr + 2 * u + 1][0], q[h][0][4 * gr + 2 * u + 1][1]);
              }
            }
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
              for (int x = 0; x < 4; ++x) a[h][x] = fmaf(left[h][x], 1.f / kLeftUnits, a[h][x]);
          } else {
            const uint32_t n[4][4] = {
                {opened_centred<0>(w[0].x), opened_centred<0>(w[1].x), opened_centred<1>(w[0].x), opened_centred<1>(w[1].x)},
                {opened_centred<2>(w[0].x), opened_centred<2>(w[1].x), opened_centred<3>(w[0].x), opened_centred<3>(w[1].x)},
                {opened_centred<0>(w[0].y), opened_centred<0>(w[1].y), opened_centred<1>(w[0].y), opened_centred<1>(w[1].y)},
                {opened_centred<2>(w[0].y), opened_centred<2>(w[1].y), opened_centred<3>(w[0].y), opened_centred<3>(w[1].y)}};
#pragma unroll
            for (int x = PARTS - 1; x >= 0; --x)                 // (small parts first: their sums round less)
#pragma unroll
              for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int h = 0; h < H; ++h) mma(a[h], n[u][0], n[u][1], n[u][2], n[u][3], q[h][x][4 * gr + u][0], q[h][x][4 * gr + u][1]);
          }
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float scale = low(pair[y][gr]), zero = PARTS == 1 ? high(pair[y][gr]) : fmaf(8.f, scale, high(pair[y][gr]));
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
              for (int x = 0; x < 2; ++x)
                s[h][2 * y + x] = fmaf(zero, qsum[h][gr][x], fmaf(scale, a[h][2 * y + x], s[h][2 * y + x]));
          }
        }
      } else {
        const uint32_t row = stage + (uint32_t)((lane & 7) + 8 * ((lane >> 3) & 1)) * R::PITCH + 16u * (lane >> 4);
#pragma unroll
        for (int j = 0; j < K16; ++j) {
          if (16 * j >= dh) break;
          uint32_t a[4];                                         // matrices (keys 0-7 | 8-15) x (channels 0-7 | 8-15), keys first
          ldsm(a, row + 32u * j);
#pragma unroll
          for (int h = 0; h < H; ++h)
#pragma unroll
            for (int x = PARTS - 1; x >= 0; --x) mma(s[h], a[0], a[1], a[2], a[3], q[h][x][j][0], q[h][x][j][1]);
        }
      }
      // a block of a page that is none: NaN to every row that sees it
      if ((missing >> (R::STAGES - 1)) & 1u) {
        if (lane == 0) report_status(p.status, SP_ERR_SHAPE, sq, kt / p.c.page_len);
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int x = 0; x < 4; ++x) s[h][x] = NAN;
      }
      if (edge) {
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (kt + 8 * (x >> 1) + g4 >= lim[h][x & 1]) s[h][x] = -INFINITY;
        __syncwarp();                                            // (keeps this a branch)
      }
      bool rise = false;
      uint32_t pair_v[2][G];                                     // 4 bits: scales of V of keys g4 | + 8
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          rise |= !(s[h][x] <= most[h][x & 1]);
        }
      if constexpr (HALF) {
        uint32_t top = vhigh, least = vlow, mask = 0x7fff7fffu;
        if (edge) mask = (kt + g4 < seen ? 0x7fffu : 0u) | (kt + 8 + g4 < seen ? 0x7fff0000u : 0u);      // (not of slots that hold nothing)
#pragma unroll
        for (int gr = 0; gr < G; ++gr) {
#pragma unroll
          for (int y = 0; y < 2; ++y) pair_v[y][gr] = lds32(stage + 2 * R::TILE + R::SCALES + ((g4 + 8 * y) * G + gr) * 4);
          const uint32_t both = __byte_perm(pair_v[0][gr], pair_v[1][gr], 0x5410) & mask;
          top = __vmaxu2(top, both);
          least = __vminu2(least, both - 0x00010001u);           // (a scale of 0 counts as none; beside one, the upper may count a bit too low)
        }
        rise |= top != vhigh || least != vlow;
      }
      bool wide = false;
      if (__any_sync(0xffffffffu, rise)) {                       // seldom: the references follow the maxima of this block
        if constexpr (HALF) {
          float top = 0.f, least = INFINITY;
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int gr = 0; gr < G; ++gr) {
              const float u = fabsf(low(pair_v[y][gr]));
              if (u < INFINITY && kt + 8 * y + g4 < seen) {
                top = fmaxf(top, u);
                least = fminf(least, u > 0.f ? u : INFINITY);
              }
            }
#pragma unroll
          for (int w = 1; w < 32; w <<= 1) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
            least = fminf(least, __shfl_xor_sync(0xffffffffu, least, w));
          }
          const float twice = low(vhigh);
          if (vhigh != kWide && (top > twice || (least < INFINITY && least < 0x1p-21f * twice))) {
            float now = top > twice ? __uint_as_float(min(max(__float_as_uint(top) >> 23, 20u), 240u) << 23) : 0.5f * twice;
            vhigh = (__float_as_uint(2.f * now) >> 16) * 0x00010001u;
            vlow = ((__float_as_uint(0x1p-20f * now) >> 16) - 1u) * 0x00010001u;
            // (what O holds would leave fp32 by a large step; scales beyond the largest unit would leave fp16)
            if (least < 0x1p-20f * now || now * per_vunit > 0x1p40f || top >= 0x1p114f) {
              now = kWideUnit;
              vhigh = kWide;
              vlow = 0xffffffffu;                                // (every block but one of zeros comes here)
            }
            const float f = per_vunit > 0.f ? (1.f / per_vunit) / now : 0.f;
            per_vunit = 1.f / now;
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
              for (int j = 0; j < K16; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x) o[j][h][x] *= f;
          }
          // (a vote, and within this branch: with a branch of its own on vhigh 16 tokens after 2048 .. 31013 keys took 130 us, not 121)
          wide = __any_sync(0xffffffffu, vhigh == kWide);
        }
#pragma unroll
        for (int h = 0; h < H; ++h) {
          float f[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float m = fmaxf(s[h][x], s[h][2 + x]) * to_log2[h][x];
            // (beyond fp32: NaN, too)
            const bool nan = s[h][x] != s[h][x] || s[h][2 + x] != s[h][2 + x] || m == INFINITY;
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
            if (__ballot_sync(0xffffffffu, nan) & (0x11111111u << t4)) m = NAN;      // (the lanes of these rows)
            const bool up = m != -INFINITY && !(m - r[h][x] <= 0.f);
            f[x] = up ? exp2_fast(r[h][x] - m) : 1.f;            // r = -infinity: 0
            if (up) {
              r[h][x] = m;
              ref[h][x] = m - kLift;
              most[h][x] = (m + 8.f) / to_log2[h][x];
            }
            l[h][x] *= f[x];
#pragma unroll
            for (int gr = 0; gr < G; ++gr) offset[h][gr][x] *= f[x];
          }
#pragma unroll
          for (int j = 0; j < K16; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[j][h][x] *= f[x & 1];
        }
      }
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          s[h][x] = exp2_fast(fmaf(s[h][x], to_log2[h][x & 1], -ref[h][x & 1]));      // now probabilities, to the reference
          l[h][x & 1] += s[h][x];
        }
      const uint32_t vtile = stage + R::TILE;
      if constexpr (FOUR) {
        if constexpr (!HALF) {
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int gr = 0; gr < G; ++gr) pair_v[y][gr] = lds32(stage + 2 * R::TILE + R::SCALES + ((g4 + 8 * y) * G + gr) * 4);
        }
        // (0 times a scale, and what comes of it, is 0 unless it is beyond what the keys that are seen have; read again here, so that this stays behind
        // the branch)
        bool odd_scales = false;
        if (edge) {
          for (int y = 0; y < 2; ++y)
            for (int gr = 0; gr < G; ++gr) {
              const uint32_t w = lds32(stage + 2 * R::TILE + R::SCALES + ((g4 + 8 * y) * G + gr) * 4);
              odd_scales |= !(fabsf(low(w)) <= (HALF ? low(vhigh) : 1e37f)) || !(fabsf(high(w)) < 1e38f);
            }
          odd_scales = __any_sync(0xffffffffu, odd_scales);
        }
        const auto add_values = [&](auto strict) {
#pragma unroll
        for (int gr = 0; gr < G; ++gr) {
          uint32_t pb[H][PARTS][2];                              // (P s)^T: keys 2 t4, + 1 | 2 t4 + 8, + 9 of row 8 h + g4
#pragma unroll
          for (int h = 0; h < H; ++h)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              // (p s)^T goes into the product with n - 8, the rest into offset, so that a rounding of p s weighs a number's distance from the
              // middle alone (16 tokens after 2048 .. 31013 keys: 4.7e-3 from the formula with n as it is).
              const float scale = low(pair_v[y][gr]), zero = fmaf(8.f * kOffsetPer, scale, kOffsetPer * high(pair_v[y][gr]));
              float ps[2], pz[2];
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                ps[x] = s[h][2 * y + x] * (HALF ? scale * per_vunit : scale);
                pz[x] = zero;
              }
              if constexpr (decltype(strict)::value) {                                      // whatever stands in a slot that the row does not see
#pragma unroll
                for (int x = 0; x < 2; ++x)
                  if (kt + 8 * y + g4 >= lim[h][x]) ps[x] = pz[x] = 0.f;
              }
#pragma unroll
              for (int x = 0; x < 2; ++x) offset[h][gr][x] = fmaf(s[h][2 * y + x], pz[x], offset[h][gr][x]);
              uint32_t u[PARTS];
              if constexpr (HALF) u[0] = pack_half(ps[0], ps[1]);
              else split<PARTS>(ps[0], ps[1], u);
#pragma unroll
              for (int x = 0; x < PARTS; ++x) pb[h][x][y] = turned8x8(u[x]);
            }
          uint32_t w[4];                                         // word g4 of keys 2 t4, + 1, + 8, + 9
#pragma unroll
          for (int x = 0; x < 4; ++x) w[x] = lds32(vtile + (v_at[x & 1][gr] ^ (kFlip * (x >> 1))) + 8 * (x >> 1) * (DH / 2));
          // numbers 0 .. 3 and 4 .. 7 of two keys side by side
          const uint32_t m0 = __byte_perm(w[0], w[1], 0x5410), m1 = __byte_perm(w[0], w[1], 0x7632);
          const uint32_t m2 = __byte_perm(w[2], w[3], 0x5410), m3 = __byte_perm(w[2], w[3], 0x7632);
          uint32_t a[4][4];
          if constexpr (PARTS == 1) {
            a[0][0] = opened<0>(m0); a[0][1] = opened<0>(m1); a[0][2] = opened<0>(m2); a[0][3] = opened<0>(m3);
            a[1][0] = opened<1>(m0); a[1][1] = opened<1>(m1); a[1][2] = opened<1>(m2); a[1][3] = opened<1>(m3);
            a[2][0] = opened<2>(m0); a[2][1] = opened<2>(m1); a[2][2] = opened<2>(m2); a[2][3] = opened<2>(m3);
            a[3][0] = opened<3>(m0); a[3][1] = opened<3>(m1); a[3][2] = opened<3>(m2); a[3][3] = opened<3>(m3);
          } else {
            a[0][0] = opened_centred<0>(m0); a[0][1] = opened_centred<0>(m1); a[0][2] = opened_centred<0>(m2); a[0][3] = opened_centred<0>(m3);
            a[1][0] = opened_centred<1>(m0); a[1][1] = opened_centred<1>(m1); a[1][2] = opened_centred<1>(m2); a[1][3] = opened_centred<1>(m3);
            a[2][0] = opened_centred<2>(m0); a[2][1] = opened_centred<2>(m1); a[2][2] = opened_centred<2>(m2); a[2][3] = opened_centred<2>(m3);
            a[3][0] = opened_centred<3>(m0); a[3][1] = opened_centred<3>(m1); a[3][2] = opened_centred<3>(m2); a[3][3] = opened_centred<3>(m3);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int h = 0; h < H; ++h) {
              if constexpr (PARTS == 1) {
                // (the 72 go block by block: at the end they would be hundreds of times what is left)
                mma_half(o[4 * gr + j][h], 0xd480d480u, 0xd480d480u, 0xd480d480u, 0xd480d480u, pb[h][0][0], pb[h][0][1]);
                mma_half(o[4 * gr + j][h], a[j][0], a[j][1], a[j][2], a[j][3], pb[h][0][0], pb[h][0][1]);
              } else {
                float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = PARTS - 1; x >= 0; --x) mma(t, a[j][0], a[j][1], a[j][2], a[j][3], pb[h][x][0], pb[h][x][1]);
#pragma unroll
                for (int x = 0; x < 4; ++x) o[4 * gr + j][h][x] += t[x];
              }
            }
        }
        };
        if (odd_scales || wide) {
          if (wide) add_wide(kt, stage, s);
          else add_values(std::true_type());
        } else {
          add_values(std::false_type());
        }
      } else {
        // Probabilities as two bf16 parts (16 bits).  Rounded to one they left 2.2e-3 of the result's norm (one token after 777 keys, 12 heads of 64), now
        // 1.7e-3, the result's own rounding; 50 drafted tokens after 700 .. 11447 keys take 52 us for 49.
        constexpr int VPARTS = PARTS == 1 ? 2 : PARTS;
        uint32_t pb[H][VPARTS][2];
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            uint32_t u[VPARTS];
            if constexpr (PARTS == 1) split_above_zero(s[h][2 * y], s[h][2 * y + 1], u);
            else split<VPARTS>(s[h][2 * y], s[h][2 * y + 1], u);
#pragma unroll
            for (int x = 0; x < VPARTS; ++x) pb[h][x][y] = turned8x8(u[x]);
          }
        const uint32_t row = vtile + (uint32_t)((lane & 7) + 8 * (lane >> 4)) * R::PITCH + 16u * ((lane >> 3) & 1);
#pragma unroll
        for (int j = 0; j < K16; ++j) {
          if (16 * j >= dh) break;
          uint32_t a[4];                                         // channels first: keys 2 t4, + 1 (a[0], a[1]) | 2 t4 + 8, + 9
          ldsm_turned(a, row + 32u * j);
          if (edge) {
            // Keys that no row sees are cleared.  At one that only some see, a non-finite value is set to zero (0 times it would
            // be NaN for the others) and given back at the end to the rows that see it; seen by every row, it goes its way.
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int key = kt + 2 * t4 + 8 * (x >> 1);
              uint32_t clear = (key >= seen ? 0xffffu : 0u) | (key + 1 >= seen ? 0xffff0000u : 0u);
              const uint32_t b = ((a[x] & 0x7fff7fffu) + 0x00800080u) & 0x80008000u & ~clear;      // all-ones exponents
              const uint32_t odd = (b & 0x8000u && key >= sure ? 0xffffu : 0u) | (b & 0x80000000u && key + 1 >= sure ? 0xffff0000u : 0u);
              found |= odd != 0u;
              a[x] &= ~(clear | odd);
            }
          }
#pragma unroll
          for (int h = 0; h < H; ++h) {
            if constexpr (PARTS == 1) {
#pragma unroll
              for (int x = VPARTS - 1; x >= 0; --x) mma(o[j][h], a[0], a[1], a[2], a[3], pb[h][x][0], pb[h][x][1]);
            } else {
              float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int x = PARTS - 1; x >= 0; --x) mma(t, a[0], a[1], a[2], a[3], pb[h][x][0], pb[h][x][1]);
#pragma unroll
              for (int x = 0; x < 4; ++x) o[j][h][x] += t[x];
            }
          }
        }
      }
      __syncwarp();                                              // the stage is read: the next copies may take it
    }
    copies_wait<0>();
    __syncwarp();                                                // (every lane's copies: the ring now holds results)
    // ---- the warps join
    if (threadIdx.x == 0) s_bad = 0;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      if constexpr (FOUR) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int gr = 0; gr < G; ++gr) {
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) offset[h][gr][x] += __shfl_xor_sync(0xffffffffu, offset[h][gr][x], w);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float f = !HALF ? 1.f : per_vunit > 0.f ? kOffsetPer / per_vunit : 0.f;
              o[4 * gr + j][h][x] = fmaf(o[4 * gr + j][h][x], f, offset[h][gr][x]);
              o[4 * gr + j][h][2 + x] = fmaf(o[4 * gr + j][h][2 + x], f, offset[h][gr][x]);
            }
          }
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int row = 8 * h + 2 * t4 + x;
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) l[h][x] += __shfl_xor_sync(0xffffffffu, l[h][x], w);
        float* dst = s_o + row * C::PITCH;
#pragma unroll
        for (int j = 0; j < K16; ++j) {
          const int d = FOUR ? 64 * (j / 4) + 8 * g4 + j % 4 : 16 * j + g4;
          dst[d] = o[j][h][x];
          dst[d + (FOUR ? 4 : 8)] = o[j][h][2 + x];
        }
        if (g4 == 0) {
          s_o[ROWS * C::PITCH + row] = r[h][x];
          s_o[ROWS * (C::PITCH + 1) + row] = l[h][x];
        }
      }
    }
    __syncthreads();
    if (found) s_bad = 1;
    if (!FOUR) __syncthreads();
    const bool bad = !FOUR && s_bad != 0;
    const uint32_t quads = (uint32_t)dh / 4;                     // a thread has four channels of a row
    for (uint32_t e = threadIdx.x; e < rows * quads; e += C::THREADS) {
      const uint32_t row = e / quads, d = 4 * (e - row * quads), rr = r0 + row, token = rr / g;
      const int64_t out_row = it.q0 + (int64_t)token;
      const int64_t out_head = (int64_t)head * g + (rr - token * g);
      const auto of = [&](int w) { return reinterpret_cast<const float*>(smem + w * C::WARP); };
      float top = -INFINITY;                                     // (a NaN of one warp's comes in through its sum)
#pragma unroll
      for (int w = 0; w < W; ++w) top = fmaxf(top, of(w)[ROWS * C::PITCH + row]);
      const float base = top == -INFINITY ? 0.f : top;
      float sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = exp2_fast(of(w)[ROWS * C::PITCH + row] - base);      // a warp without keys: 0, and its l and O are 0
        sum = fmaf(of(w)[ROWS * (C::PITCH + 1) + row], f, sum);
        const float4 v = *reinterpret_cast<const float4*>(of(w) + row * C::PITCH + d);
        acc[0] = fmaf(v.x, f, acc[0]);
        acc[1] = fmaf(v.y, f, acc[1]);
        acc[2] = fmaf(v.z, f, acc[2]);
        acc[3] = fmaf(v.w, f, acc[3]);
      }
      // (keys seen, and all logits beyond fp32 below: nothing can be told, unless other pieces of the row's keys have weight)
      const bool lost = sum == 0.f && visible(it.nk, shift, token) > kb;
      const float inv = sum == 0.f ? (lost && !cut ? NAN : 0.f) : 1.f / kOffsetPer / sum;
#pragma unroll
      for (int x = 0; x < 4; ++x) acc[x] *= inv;
      if (bad) {
        const int32_t last = min(visible(it.nk, shift, token), seen);
        for (int32_t key = max(sure, kb); key < last; ++key) {
          const int32_t page = page_of(p.c, sq, key / p.c.page_len);
          if (page < 0) continue;
          const __nv_bfloat16* V = reinterpret_cast<const __nv_bfloat16*>(p.c.v + page * p.c.step) +
                                   ((int64_t)head * p.c.page_len + key % p.c.page_len) * dh;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float u = __bfloat162float(V[d + x]);
            if (!(fabsf(u) < INFINITY)) acc[x] += u;
          }
        }
      }
      if (cut) {
        *reinterpret_cast<float4*>(p.part_o + ((int64_t)slot_of * ROWS + row) * dh + d) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      } else {
        T* out = reinterpret_cast<T*>(p.o) + out_row * p.ldo + out_head * dh + d;
#pragma unroll
        for (int x = 0; x < 4; ++x) store1(out + x, acc[x]);
      }
      if (d == 0) {
        const float lse2 = sum == 0.f ? (!lost ? -INFINITY : cut ? kNoWeight : NAN) : base + (log2f(sum) - kLift);
        if (cut) p.part_lse[slot_of * ROWS + row] = lse2;
        else if (p.lse) p.lse[out_row * p.n_heads + out_head] = lse2 == -INFINITY ? lse2 : lse2 * 0.6931471805599453f;
      }
    }
    __syncthreads();                                             // s_bad and the warps' results are read
  }
}

// O_i = sum_c w_c O_ic / sum_c w_c with w_c = 2^(lse_ic - max) over the pieces of a tile and head: one warp per row and head.
template <typename T, int ROWS>
__global__ void __launch_bounds__(256) paged_join_kernel(const PagedParams p) {
  kernel_begin();
  const int lane = threadIdx.x & 31;
  const int64_t idx = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (idx >= (int64_t)p.Nq * p.n_heads) return;
  const int32_t row = (int32_t)(idx / p.n_heads), h = (int32_t)(idx % p.n_heads);
  const int32_t sq = sequence_of(p.cu_q, p.c.n_seq, p.Nq, row);
  if (sq < p.s0 || sq >= p.s0 + p.n_here) return;
  const Seq it = seq_at(p, sq);
  const int64_t total = p.plan[p.n_here], ctas = p.plan[p.n_here + 1];
  const int32_t of_tile = blocks_of(it.nk);
  const uint32_t rr = (uint32_t)(row - it.q0) * p.g + h % p.g;
  const int64_t first = p.plan[sq - p.s0] + ((int64_t)(rr / ROWS) * p.c.n_kv + h / p.g) * (kLead + of_tile) + kLead;
  const int64_t b0 = cta_of(first, total, ctas), b1 = cta_of(first + of_tile - 1, total, ctas);
  if (b0 == b1 || b0 < 0 || b1 >= kMostCtas) return;      // (whole; outside only where cu_q decreases)
  const int parts = (int)(b1 - b0) + 1, dh = p.c.dh;
  // (the first piece stands at 2 b0 + 1, the others at 2 b)
  const auto slot = [&](int c) { return 2 * (b0 + c) + (c == 0 ? 1 : 0); };
  float mx = -INFINITY;
  bool bad = false;                   // (fmaxf passes over a NaN)
  for (int c = lane; c < parts; c += 32) {
    const float lc = p.part_lse[slot(c) * ROWS + rr % ROWS];
    mx = fmaxf(mx, lc);
    bad |= lc != lc;
  }
#pragma unroll
  for (int w = 16; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
  const float ref = mx == -INFINITY ? 0.f : mx;
  bad = __any_sync(0xffffffffu, bad) || mx == kNoWeight;
  const int d = 4 * lane;             // a lane has channels 4 lane .. (dh is a multiple of 16)
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float total_w = 0.f;
  for (int c0 = 0; c0 < parts; c0 += 32) {
    const float wl = c0 + lane < parts ? exp2f(p.part_lse[slot(c0 + lane) * ROWS + rr % ROWS] - ref) : 0.f;
    const int m = min(32, parts - c0);
#pragma unroll 8
    for (int c = 0; c < m; ++c) {
      const float w = __shfl_sync(0xffffffffu, wl, c);
      total_w += w;
      if (d < dh) {
        const float4 v = *reinterpret_cast<const float4*>(p.part_o + (slot(c0 + c) * ROWS + rr % ROWS) * dh + d);
        acc.x = fmaf(w, v.x, acc.x);
        acc.y = fmaf(w, v.y, acc.y);
        acc.z = fmaf(w, v.z, acc.z);
        acc.w = fmaf(w, v.w, acc.w);
      }
    }
  }
  const float inv = total_w == 0.f ? 0.f : 1.f / total_w;
  if (d < dh) {
    T* out = reinterpret_cast<T*>(p.o) + (int64_t)row * p.ldo + (int64_t)h * dh + d;
    store1(out, bad ? NAN : acc.x * inv);
    store1(out + 1, bad ? NAN : acc.y * inv);
    store1(out + 2, bad ? NAN : acc.z * inv);
    store1(out + 3, bad ? NAN : acc.w * inv);
  }
  if (lane == 0 && p.lse)
    p.lse[(int64_t)row * p.n_heads + h] = bad ? NAN : total_w == 0.f ? -INFINITY : (ref + log2f(total_w)) * 0.6931471805599453f;
}

// Rows of a tile.  (Tiles of 24 or 32 read the cache once for the five drafted tokens of four heads of 64, and took as long: 46 us for 12 texts of
// 700 .. 11447 keys, 8 heads, 16 bits.)
inline int tile_rows(int64_t Nq, int64_t g, int64_t n_seq) { return Nq * g <= 8 * n_seq ? 8 : 16; }
// Whether the cache streams past tiles of 16 rows: up to a number of rows per sequence, on average, that is the larger the fewer sequences and key
// heads there are, since the other form's tiles of 128 rows then leave more of the device idle (less of it where a single sequence is cut to
// fit).  This / the other form in 4 bits and in 16, heads of 128, us.  A single sequence, by key heads: 1 head 16384 keys 160 rows 34 / 56 and 33 / 49; 4 heads
// 8192 keys 128 rows 38 / 40 and 37 / 33, 160 rows 43 / 43 and 42 / 35; 8 heads 2048 keys 64 rows 24 / 29 and 23 / 22, 32768 keys 48 rows 73 / 92 and
// 91 / 86, 64 rows 90 / 90 and 92 / 84, 80 rows 107 / 92 and 122 / 86; 32 heads 8192 keys 48 rows 76 / 95 and 87 / 91, 64 rows 95 / 92 and 99 / 89;
// 40 heads 4096 keys 48 rows 58 / 72 and 62 / 64, 64 rows 71 / 69 and 74 / 62.  Several, by sequences x heads: 12: 12 x 4096 keys 128 rows 51 / 61 and
// 49 / 47; 16: 2 x 4096 keys 80 rows 45 / 50 and 44 / 43, 96 rows 51 / 50 and 49 / 41; 32: 4 x 4096 keys 80 rows 72 / 83 and 70 / 73, 96 rows 83 / 80
// and 80 / 71; 48: 6 x 4096 keys 80 rows 99 / 102 and 99 / 87; 64: 8 x 2048 keys 48 rows 57 / 78 and 55 / 68, 64 rows 70 / 75 and 66 / 67; 96: 12 x 4096
// keys 48 rows 115 / 147 and 117 / 134, 64 rows 149 / 138 and 148 / 127; 512: 64 x 1024 keys 32 rows 161 / 175 and 169 / 157, 48 rows 234 / 187 and
// 254 / 166.  In fp32 this form is always faster, since only it takes the tensor cores: 64 x 1024 keys 16 rows 104 / 541, 256 rows 1378 / 2663; 1 x 16384
// keys 256 rows 235 / 989.
inline bool paged_few_rows(int32_t dtype, int64_t Nq, int64_t g, int64_t n_seq, int64_t n_kv) {
  if (dtype == SP_F32) return true;
  const int64_t streams = n_seq * n_kv;
  const int64_t most = n_seq == 1 ? (streams <= 4 ? 128 : streams <= 12 ? 64 : 48) : streams <= 12 ? 128 : streams <= 48 ? 80 : streams <= 128 ? 48 : 32;
  return Nq * g <= most * n_seq;
}

struct RowsPlan {
  int rows;
  size_t plan_bytes, o_bytes, lse_bytes;
  size_t bytes() const { return plan_bytes + o_bytes + lse_bytes; }
};
RowsPlan rows_plan(int64_t Nq, int64_t n_seq, int64_t g, int64_t dh) {
  RowsPlan r;
  r.rows = tile_rows(Nq, g, n_seq);
  r.plan_bytes = align_up((kPlanSeqs + 2) * sizeof(int64_t), 256);
  r.o_bytes = align_up((size_t)2 * kMostCtas * r.rows * dh * 4, 256);
  r.lse_bytes = align_up((size_t)2 * kMostCtas * r.rows * 4, 256);
  return r;
}

template <typename T, int DH, bool FOUR, int ROWS>
cudaError_t launch_rows(const PagedParams& p, cudaStream_t stream) {
  using C = PagedCfg<DH, FOUR, ROWS, sizeof(T) == 4 ? 3 : 1>;
  static PerDeviceOnce attr_once;
  const auto kernel = paged_rows_kernel<T, DH, FOUR, ROWS>;
  cudaError_t e = attr_once.run([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM); });
  if (e != cudaSuccess) return e;
  // as many blocks as can be resident and may have work
  const int64_t seqs = p.n_here < p.Nq ? p.n_here : p.Nq, keys = (int64_t)p.c.max_pages * p.c.page_len;
  const int64_t tiles = ((int64_t)p.Nq * p.g / ROWS + seqs) * p.c.n_kv, work = ceil_div(tiles * (kLead + 1 + ceil_div(keys, (int64_t)kBlock)), (int64_t)kLeastShare);
  int64_t ctas = (int64_t)sm_count() * C::CTAS;
  if (ctas > kMostCtas) ctas = kMostCtas;
  if (ctas > work) ctas = work;
  count_launch();
  e = launch(kernel, dim3((unsigned)ctas), dim3(C::THREADS), C::SMEM, stream, p);
  if (e != cudaSuccess || ctas < 2) return e;
  count_launch();
  const OverlapScope overlap(true);       // its blocks start while the pieces end
  return launch(paged_join_kernel<T, ROWS>, dim3((unsigned)ceil_div((int64_t)p.Nq * p.n_heads, (int64_t)8)), dim3(256), 0, stream, p);
}
template <typename T, int DH, bool FOUR>
cudaError_t launch_rows(const PagedParams& p, int rows, cudaStream_t stream) {
  return rows == 8 ? launch_rows<T, DH, FOUR, 8>(p, stream) : launch_rows<T, DH, FOUR, 16>(p, stream);
}
template <typename T>
cudaError_t launch_rows(const PagedParams& p, bool four, int rows, cudaStream_t stream) {
  if (p.c.dh <= 64) return four ? launch_rows<T, 64, true>(p, rows, stream) : launch_rows<T, 64, false>(p, rows, stream);
  return four ? launch_rows<T, 128, true>(p, rows, stream) : launch_rows<T, 128, false>(p, rows, stream);
}

// cu_k of the opened keys: the lengths added up; a sequence that does not fit into max_keys (or has more tokens than its table) gets as many
// rows as queries at most, of which every query sees one that it would see, and no number of tokens in `whole`, which makes those NaN.
__global__ void __launch_bounds__(kPlanThreads) open_plan_kernel(const CacheView c, const int32_t* cu_q, int32_t Nq, int32_t max_keys, int32_t* cu_k,
                                                             int32_t* whole, HalfTops* tops, int32_t* status) {
  kernel_begin();
  if (tops)
    for (int64_t i = threadIdx.x; i < (int64_t)c.n_seq * c.n_kv; i += kPlanThreads) tops[i] = HalfTops{0u, kNoLow, 0u, kNoLow};
  __shared__ int64_t s_word[kPlanThreads / 32];
  int64_t at = 0, used = 0;               // rows given to the sequences before, and their keys
  for (int32_t s0 = 0; s0 < c.n_seq; s0 += kPlanThreads) {
    const int32_t s = s0 + threadIdx.x;
    int64_t n = 0, before;
    const int32_t nq = s < c.n_seq ? bounded(cu_q[s + 1], Nq) - bounded(cu_q[s], Nq) : 0;
    if (nq > 0) n = max(0, c.lens[s]);
    const int64_t keys = block_scan<kPlanThreads / 32>(n, s_word, before);
    // (what fits is decided by the sum up to here, whether those before fitted or not: the same answer in any order)
    const bool fits = n == 0 || (used + before + n <= max_keys && n <= (int64_t)c.max_pages * c.page_len);
    if (!fits) {
      report_status(status, SP_ERR_SHAPE, s, -1);
      n = min(n, (int64_t)nq);
    }
    const int64_t rows = block_scan<kPlanThreads / 32>(n, s_word, before);
    if (s < c.n_seq) {
      cu_k[s] = (int32_t)(at + before);
      whole[s] = fits ? (int32_t)n : -1;
    }
    at += rows;
    used += keys;
  }
  if (threadIdx.x == 0) cu_k[c.n_seq] = (int32_t)at;
}

struct OpenPlan {
  int64_t rows;
  size_t cu_bytes, tops_bytes, k_bytes, q_bytes, unit_bytes, attention;
  size_t bytes() const { return cu_bytes + tops_bytes + 2 * k_bytes + q_bytes + unit_bytes + attention; }
};
// (room for what 4 bits need whatever the cache is: the workspace depends on the sizes that its call is given)
OpenPlan open_plan(int64_t Nq, int64_t n_seq, int32_t n_heads, int32_t n_kv, int32_t dh, int64_t max_keys) {
  OpenPlan r;
  r.rows = max_keys + Nq;
  const bool four = dh % kCacheGroup == 0;
  r.cu_bytes = align_up((size_t)(2 * n_seq + 1) * 4, 256);       // and the lengths behind the offsets
  r.tops_bytes = four ? align_up((size_t)n_seq * n_kv * sizeof(HalfTops), 256) : 0;
  r.k_bytes = align_up((size_t)r.rows * n_kv * dh * 2, 256);
  r.q_bytes = four ? align_up((size_t)Nq * n_heads * dh * 2, 256) : 0;
  r.unit_bytes = four ? align_up((size_t)Nq * n_heads * 4, 256) : 0;
  r.attention = attention_workspace(Nq, r.rows, (int32_t)n_seq, n_heads, n_kv, dh, SP_BF16, max_keys);
  return r;
}
// max_keys as the caller gave it, or all that the table can hold
int64_t keys_at_most(int64_t max_keys, int64_t n_seq, int64_t max_pages, int64_t page_len) {
  const int64_t all = n_seq * max_pages * page_len;
  return max_keys > 0 && max_keys < all ? max_keys : all;
}

}  // namespace
}  // namespace sp

extern "C" {

size_t sp_cache_attention_bytes(int64_t Nq, int32_t n_seq, int32_t n_heads, int32_t n_kv_heads, int32_t d_head, int32_t dtype,
                                int32_t max_pages, int32_t page_len, int64_t max_keys) {
  using namespace sp;
  if (Nq < 1 || Nq > (1 << 30) || n_seq < 1 || n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads != 0 || d_head < 1 || d_head > 128 ||
      max_pages < 0 || page_len < 1 || (int64_t)max_pages * page_len > (1 << 30))
    return 0;
  const int64_t g = n_heads / n_kv_heads;
  if (Nq * g > 0x7fffffff) return 0;
  if (paged_few_rows(dtype, Nq, g, n_seq, n_kv_heads)) return rows_plan(Nq, n_seq, g, d_head).bytes();
  const int64_t keys = keys_at_most(max_keys, n_seq, max_pages, page_len);
  if (keys + Nq > (1 << 30)) return 0;
  return open_plan(Nq, n_seq, n_heads, n_kv_heads, d_head, keys).bytes();
}

sp_status sp_cache_attention(const sp_kv_cache* cache, const sp_mat* Q, const int32_t* cu_q, int32_t n_heads, int32_t causal, double scale,
                             int64_t max_keys, const sp_mat* O, float* lse, int32_t* status_dev, void* ws, size_t ws_bytes, void* stream) {
  using namespace sp;
  if (!Q || !O) return SP_ERR_INVALID_ARG;
  const sp_status ok = check_cache(cache, true);
  if (ok != SP_OK) return ok;
  const int32_t dt = Q->dtype, n_seq = cache->n_seq, n_kv = cache->n_kv_heads, dh = cache->d_head;
  if ((dt != SP_F32 && dt != SP_BF16) || O->dtype != dt) return SP_ERR_DTYPE;
  if (n_heads < 1 || n_heads > (1 << 20) || n_heads % n_kv != 0 || max_keys < 0) return SP_ERR_SHAPE;
  const int64_t Nq = Q->rows, cols = (int64_t)n_heads * dh;
  if (Nq < 0 || Nq > (1 << 30) || Q->cols != cols || O->rows != Nq || O->cols != cols) return SP_ERR_SHAPE;
  if (Nq > 1 && (Q->ld < cols || O->ld < cols)) return SP_ERR_SHAPE;
  if (Nq * n_heads > ((int64_t)1 << 33)) return SP_ERR_SHAPE;
  if (!(scale >= 1e-30) || !(scale <= 1e30)) return SP_ERR_INVALID_ARG;
  if (Nq == 0 || n_seq == 0) return SP_OK;
  if (!Q->ptr || !O->ptr || !cu_q) return SP_ERR_INVALID_ARG;
  const int64_t g = n_heads / n_kv;
  const size_t need = sp_cache_attention_bytes(Nq, n_seq, n_heads, n_kv, dh, dt, cache->max_pages, cache->page_len, max_keys);
  if (need == 0) return SP_ERR_SHAPE;                            // (too many rows, or more keys than can be opened: max_keys tells how many there are)
  if (!ws || ws_bytes < need) return SP_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(ws) & 255u) return SP_ERR_ALIGNMENT;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  uint8_t* at = reinterpret_cast<uint8_t*>(ws);
  if (paged_few_rows(dt, Nq, g, n_seq, n_kv)) {
    ProfScope prof(PK_GEMM_TC, 0.0, 0.0, s);
    const RowsPlan plan = rows_plan(Nq, n_seq, g, dh);
    PagedParams p = {};
    p.c = cache_view(cache);
    p.q = Q->ptr; p.o = O->ptr;
    p.ldq = Nq > 1 ? Q->ld : cols; p.ldo = Nq > 1 ? O->ld : cols;
    p.lse = lse;
    p.cu_q = cu_q;
    p.Nq = (int32_t)Nq; p.n_heads = n_heads; p.g = (int32_t)g; p.causal = causal != 0;
    p.scale_log2 = (float)(scale * 1.4426950408889634);
    p.plan = reinterpret_cast<int64_t*>(at);
    p.part_o = reinterpret_cast<float*>(at + plan.plan_bytes);
    p.part_lse = reinterpret_cast<float*>(at + plan.plan_bytes + plan.o_bytes);
    p.status = status_dev;
    for (p.s0 = 0; p.s0 < n_seq; p.s0 += kPlanSeqs) {
      p.n_here = n_seq - p.s0 < kPlanSeqs ? n_seq - p.s0 : kPlanSeqs;
      const bool four = cache->kind == SP_CACHE_4BIT;
      const cudaError_t e = dt == SP_F32 ? launch_rows<float>(p, four, plan.rows, s) : launch_rows<__nv_bfloat16>(p, four, plan.rows, s);
      if (e != cudaSuccess) return SP_ERR_CUDA;
    }
    return SP_OK;
  }
  const int64_t keys = keys_at_most(max_keys, n_seq, cache->max_pages, cache->page_len);
  const OpenPlan plan = open_plan(Nq, n_seq, n_heads, n_kv, dh, keys);
  int32_t *cu_k = reinterpret_cast<int32_t*>(at), *whole = cu_k + n_seq + 1;
  uint8_t *K = at + plan.cu_bytes + plan.tops_bytes, *V = K + plan.k_bytes, *Qh = V + plan.k_bytes, *units = Qh + plan.q_bytes;
  uint8_t* rest = units + plan.unit_bytes;
  const int64_t kv = (int64_t)n_kv * dh;
  const bool half = cache->kind == SP_CACHE_4BIT;
  HalfTops* tops = half ? reinterpret_cast<HalfTops*>(at + plan.cu_bytes) : nullptr;
  float* q_unit = half ? reinterpret_cast<float*>(units) : nullptr;
  {
    ProfScope prof(PK_ELEMENTWISE, 0.0, 0.0, s);                   // (the products have a scope of their own)
    count_launch();
    if (launch(open_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, cache_view(cache), cu_q, (int32_t)Nq, (int32_t)keys, cu_k, whole, tops, status_dev) !=
        cudaSuccess)
      return SP_ERR_CUDA;
    if (half && (cache_tops(cache, cu_k, whole, plan.rows, tops, s) != cudaSuccess ||
                 queries_to_half(cache, Q, cu_q, Qh, q_unit, tops, s) != cudaSuccess))
      return SP_ERR_CUDA;
    if (cache_open(cache, cu_k, whole, plan.rows, K, V, tops, status_dev, s) != cudaSuccess) return SP_ERR_CUDA;
  }
  sp_attention_args a = {};
  a.Q = half ? sp_mat{Qh, dt, 0, Nq, cols, cols} : *Q;
  a.O = *O;
  a.K = sp_mat{K, dt, 0, plan.rows, kv, kv};
  a.V = sp_mat{V, dt, 0, plan.rows, kv, kv};
  a.cu_q = cu_q; a.cu_k = cu_k;
  a.lse = lse;
  a.n_seq = n_seq; a.n_heads = n_heads; a.n_kv_heads = n_kv; a.causal = causal;
  a.scale = scale;
  return attention_forward(&a, tops, q_unit, keys, status_dev, rest, plan.attention, s);
}

}  // extern "C"
