// bf16 attention of few rows against long caches: single new tokens, with the heads that share a key head as rows.
//
// What bounds it is reading K and V once.  One warp brings them in by TMA, 64 keys a stage, through a ring that holds up to 192 KB of an SM in
// flight and runs on from item to item; eight warps multiply, 16 keys of a stage each, four to a stage.  The 128 rows of the
// tcgen05 form (sp_attention_tc.cu) would be nearly empty here (and its softmax, a row per thread, idle: 16 tokens after 2048 .. 31013 keys
// took 262 us), so the products are m16n8k16 instructions, turned so that keys and channels fill them: S^T = K Q^T and O^T += V^T P^T.
// K and V^T come by ldmatrix, P^T is S^T's layout turned within a warp (movmatrix).  (K and V straight into registers, without shared memory:
// 235 us, the loads of a block and their addresses hold the registers that more loads in flight would need.)
// Each warp has its own reference r (it follows only when the maximum has risen by more than 2^8 in P's scale) and sum l per row; the warps join
// in shared memory at the end of an item.
#include <math.h>

#include "sp_attention.cuh"
#include "sp_f32x2.cuh"
#include "sp_tc.cuh"

namespace sp {
namespace {

constexpr int kWarps = 8, kGroup = 4, kBlock = 16, kStage = kGroup * kBlock;      // multiplying warps, of a stage; keys
constexpr int kThreads = (kWarps + 1) * 32;
constexpr long long kWaitBudget = 4000000000LL, kDrainBudget = 200000000LL;       // clock cycles: ~2 s, ~0.1 s

template <int DH, int ROWS>
struct RowsCfg {
  static constexpr int CH = DH / 64;                       // 128-byte wide chunks of a key's row
  static constexpr int CHUNK = kStage * 128;
  static constexpr int TILE = CH * CHUNK;                  // K or V of a stage
  // Even: the groups of warps take the stages of an item in turn, and a wait tells a phase of a barrier from the one after it, not
  // from the one after that.  With an even number a group meets every phase of its stages within an item (between items all meet).
  static constexpr int STAGES = DH == 128 ? (ROWS == 16 ? 4 : 6) : 8;
  static_assert(STAGES % (kWarps / kGroup) == 0, "stages of a group");
  static constexpr int PITCH = DH + 4;                     // floats of a row of a warp's O
  static constexpr int JOIN = kWarps * ROWS * (PITCH + 2) * 4;
  static constexpr size_t SMEM = (size_t)STAGES * 2 * TILE + JOIN + 16 * STAGES + 1024;
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
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_turned(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t turned(uint32_t a) {       // 8 x 8 values of two bytes: row g4, columns 2 t4 and 2 t4 + 1
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 e = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&e);
}
// the multiplying warps meet; whether one of them brought `v`, the same answer in all
__device__ __forceinline__ bool group_any(bool v) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"(v ? 1u : 0u), "n"(kWarps * 32) : "memory");
  return r != 0;
}
__device__ __forceinline__ void group_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory"); }

// What all warps derive from an item: keys [kb, seen) are seen by some row, [.., sure) by every row.
struct Span {
  int kb, seen, sure;
  int64_t shift;
};
__device__ __forceinline__ int visible(const AttnItem& it, int64_t shift, int64_t token) {
  return (int)max((int64_t)0, min((int64_t)it.nk, token + shift + 1));
}
__device__ __forceinline__ Span span_of(const AttnParams& p, const AttnItem& it, int64_t r0, int rows) {
  Span s;
  s.shift = p.causal ? (int64_t)it.nk - it.nq : (int64_t)it.nk;
  s.sure = visible(it, s.shift, r0 / p.g);
  s.seen = visible(it, s.shift, (r0 + rows - 1) / p.g);
  const bool cut = p.part > 0 && it.nk > p.part;
  s.kb = cut ? it.c * p.part : 0;
  if (cut && s.seen - s.kb > p.part) s.seen = s.kb + p.part;
  return s;
}

template <int DH, int ROWS>
__global__ void __launch_bounds__(kThreads, 1)
attention_rows_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const AttnParams p) {
  using C = RowsCfg<DH, ROWS>;
  constexpr int H = ROWS / 8;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int s_abort, s_bad;
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t ring = (raw + 1023u) & ~1023u, bars = ring + C::STAGES * 2 * C::TILE;
  float* s_o = reinterpret_cast<float*>(smem_raw + (bars - raw) + 16 * C::STAGES);      // [warp][row][PITCH]
  float* s_r = s_o + kWarps * ROWS * C::PITCH;                                            // [warp][row]
  float* s_l = s_r + kWarps * ROWS;
  auto full_bar = [&](int s) { return bars + 16u * s; };
  auto empty_bar = [&](int s) { return bars + 16u * s + 8u; };
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  volatile int* abort_flag = &s_abort;
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int s = 0; s < C::STAGES; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), kGroup);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  __syncthreads();
  kernel_begin();

  AttnDealer dealer;
  AttnItem it;
  uint32_t pos = 0;                  // stages of the items before
  bool ok = true;
  for (int64_t item = blockIdx.x; ok && dealer.find(p, item, ROWS, p.g, p.n_kv, it); item += gridDim.x) {
    const int64_t r0 = (int64_t)it.tile * ROWS;
    const int rows = (int)min((int64_t)ROWS, (int64_t)it.nq * p.g - r0);
    const Span sp_ = span_of(p, it, r0, rows);
    const int kb = sp_.kb, seen = sp_.seen, sure = sp_.sure;
    const int n = seen > kb ? (seen - kb + kStage - 1) / kStage : 0;
    if (warp == kWarps) {
      // ---------------------------------------------------------------------------------------------- TMA
      if (lane == 0) {
        for (int i = 0; i < n; ++i) {
          const uint32_t x = pos + i;
          const int s = (int)(x % C::STAGES);
          if (!mbar_wait(empty_bar(s), (x / C::STAGES + 1) & 1u, abort_flag, p.wait_budget)) { ok = false; break; }
          mbar_expect_tx(full_bar(s), 2 * C::TILE);
#pragma unroll
          for (int c = 0; c < C::CH; ++c) {
            tma_load_3d(ring + s * 2 * C::TILE + c * C::CHUNK, &tmK, c * 64, it.head, it.k0 + kb + i * kStage, full_bar(s));
            tma_load_3d(ring + s * 2 * C::TILE + C::TILE + c * C::CHUNK, &tmV, c * 64, it.head, it.k0 + kb + i * kStage, full_bar(s));
          }
        }
      }
      ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
      pos += n;
      continue;
    }
    // ------------------------------------------------------------------------------------------------ products
    const int g4 = lane >> 2, t4 = lane & 3;
    uint32_t q[H][DH / 16][2];
    int lim[H][2];                                             // keys [0, lim) of rows 8 h + 2 t4 + x
    const __nv_bfloat16* Q = reinterpret_cast<const __nv_bfloat16*>(p.q);
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int64_t rr = r0 + 8 * h + g4;
      const bool valid = 8 * h + g4 < rows;
      const __nv_bfloat16* src = Q + (it.q0 + (valid ? rr / p.g : 0)) * p.ldq + (it.head * (int64_t)p.g + rr % p.g) * p.dh;
#pragma unroll
      for (int j = 0; j < DH / 16; ++j)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int d = 16 * j + 8 * x + 2 * t4;
          q[h][j][x] = valid && d < p.dh ? *reinterpret_cast<const uint32_t*>(src + d) : 0u;
        }
#pragma unroll
      for (int x = 0; x < 2; ++x) {                            // (rows that are none: any values, kept to themselves)
        const int row = 8 * h + 2 * t4 + x;
        lim[h][x] = row < rows ? min(visible(it, sp_.shift, (r0 + row) / p.g), seen) : seen;
      }
    }
    float o[DH / 16][H][4];                                    // channels 16 j + g4 (| + 8), rows as lim
#pragma unroll
    for (int j = 0; j < DH / 16; ++j)
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[j][h][x] = 0.f;
    float r[H][2], l[H][2];                                    // reference of the rows; this lane's part of their sums
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int x = 0; x < 2; ++x) r[h][x] = -INFINITY, l[h][x] = 0.f;
    bool found = false;                                        // non-finite values of V behind some row's mask

    // ldmatrix: lane l gives the address of row l % 8 of matrix l / 8.  K: matrices (keys 0-7 | 8-15) x (channels 0-7 | 8-15) of a 16 x 16
    // piece, keys first; V: channels first, turned.  16-byte piece u of key row i sits at piece u ^ (i & 7) (128-byte swizzle).
    const int kw = (warp % kGroup) * kBlock;                   // this warp's keys of a stage
    const int i8 = lane & 7, mt = lane >> 3;
    const uint32_t k_row = (uint32_t)(kw + (mt & 1) * 8 + i8) * 128u, v_row = (uint32_t)(kw + (mt >> 1) * 8 + i8) * 128u;
    for (int i = warp / kGroup; i < n; i += kWarps / kGroup) {
      const uint32_t x_ = pos + i;
      const int s_ = (int)(x_ % C::STAGES);
      const bool got = mbar_wait(full_bar(s_), (x_ / C::STAGES) & 1u, abort_flag, p.wait_budget);
      ok = __all_sync(0xffffffffu, got);
      if (!ok) break;
      const int kt = kb + i * kStage + kw;
      if (kt < seen) {
        const uint32_t kbase = ring + s_ * 2 * C::TILE, vbase = kbase + C::TILE;
        float s[H][4];                                         // keys g4 | g4 + 8 of the block, rows 2 t4, 2 t4 + 1
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int x = 0; x < 4; ++x) s[h][x] = 0.f;
#pragma unroll
        for (int j = 0; j < DH / 16; ++j) {
          uint32_t a[4];
          const int u = 2 * (j % 4) + (mt >> 1);
          ldsm(a, kbase + (j / 4) * C::CHUNK + k_row + (uint32_t)((u ^ i8) << 4));
#pragma unroll
          for (int h = 0; h < H; ++h) mma_16x8x16(s[h], a, q[h][j][0], q[h][j][1]);
        }
        bool rise = false;
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            float& u = s[h][x];
            if (kt + 8 * (x >> 1) + g4 >= lim[h][x & 1]) u = -INFINITY;
            u *= p.scale_log2;
            rise |= u != -INFINITY && !(u - r[h][x & 1] <= 8.f);
          }
        if (__any_sync(0xffffffffu, rise)) {                   // seldom: the references follow the maxima of this block
#pragma unroll
          for (int h = 0; h < H; ++h) {
            float f[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float m = fmaxf(s[h][x], s[h][2 + x]);
              const bool nan = s[h][x] != s[h][x] || s[h][2 + x] != s[h][2 + x];
#pragma unroll
              for (int w = 4; w < 32; w <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
              if (__ballot_sync(0xffffffffu, nan) & (0x11111111u << t4)) m = NAN;      // (the lanes of these rows)
              const bool up = m != -INFINITY && !(m - r[h][x] <= 0.f);
              f[x] = up ? exp2_fast(r[h][x] - m) : 1.f;        // r = -infinity: 0
              if (up) r[h][x] = m;
              l[h][x] *= f[x];
            }
#pragma unroll
            for (int j = 0; j < DH / 16; ++j)
#pragma unroll
              for (int x = 0; x < 4; ++x) o[j][h][x] *= f[x & 1];
          }
        }
        uint32_t pb[H][2];                                     // P^T: keys 2 t4, + 1 | 2 t4 + 8, + 9 of row 8 h + g4
#pragma unroll
        for (int h = 0; h < H; ++h) {
          float e[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float ref = r[h][x & 1];
            e[x] = exp2_fast(s[h][x] - (ref == -INFINITY ? 0.f : ref));
            l[h][x & 1] += e[x];
          }
          pb[h][0] = turned(pack_bf16(e[0], e[1]));
          pb[h][1] = turned(pack_bf16(e[2], e[3]));
        }
        const bool edge = kt + kBlock > sure;
#pragma unroll
        for (int j = 0; j < DH / 16; ++j) {
          uint32_t a[4];                                       // keys 2 t4, + 1 (a[0], a[1]) | 2 t4 + 8, + 9
          const int u = 2 * (j % 4) + (mt & 1);
          ldsm_turned(a, vbase + (j / 4) * C::CHUNK + v_row + (uint32_t)((u ^ i8) << 4));
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
          for (int h = 0; h < H; ++h) mma_16x8x16(o[j][h], a, pb[h][0], pb[h][1]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty_bar(s_));
    }
    pos += n;
    // ---- the warps join
    if (threadIdx.x == 0) s_bad = 0;
    if (group_any(!ok)) { ok = false; break; }                 // a wait ran out; all leave before the next meeting
    if (found) s_bad = 1;
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int row = 8 * h + 2 * t4 + x;
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) l[h][x] += __shfl_xor_sync(0xffffffffu, l[h][x], w);
        if (g4 == 0) {
          s_r[warp * ROWS + row] = r[h][x];
          s_l[warp * ROWS + row] = l[h][x];
        }
        float* dst = s_o + (warp * ROWS + row) * C::PITCH + g4;
#pragma unroll
        for (int j = 0; j < DH / 16; ++j) {
          dst[16 * j] = o[j][h][x];
          dst[16 * j + 8] = o[j][h][2 + x];
        }
      }
    group_sync();
    const bool bad = s_bad != 0, cut = p.part > 0 && it.nk > p.part;
    for (int e = threadIdx.x; e < rows * DH; e += kWarps * 32) {
      const int row = e / DH, d = e % DH;
      const int64_t rr = r0 + row, token = rr / p.g, out_row = it.q0 + token;
      const int head = it.head * p.g + (int)(rr % p.g);
      float ref = -INFINITY;                                   // (a NaN of one warp's comes in through its sum)
#pragma unroll
      for (int w = 0; w < kWarps; ++w) ref = fmaxf(ref, s_r[w * ROWS + row]);
      const float base = ref == -INFINITY ? 0.f : ref;
      float total = 0.f, acc = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = exp2f(s_r[w * ROWS + row] - base);     // a warp without keys: 0, and its l and O are 0
        total = fmaf(s_l[w * ROWS + row], f, total);
        acc = fmaf(s_o[(w * ROWS + row) * C::PITCH + d], f, acc);
      }
      acc = total == 0.f ? 0.f : acc / total;
      if (d < p.dh) {
        if (bad) {
          const __nv_bfloat16* V = reinterpret_cast<const __nv_bfloat16*>(p.v) + (int64_t)it.k0 * p.ldv + it.head * (int64_t)p.dh;
          const int last = min(visible(it, sp_.shift, token), seen);
          for (int key = max(sure, kb); key < last; ++key) {
            const float u = __bfloat162float(V[key * p.ldv + d]);
            if (!(fabsf(u) < INFINITY)) acc += u;
          }
        }
        if (cut) p.part_o[((int64_t)it.c * p.Nq + out_row) * ((int64_t)p.n_heads * p.dh) + (int64_t)head * p.dh + d] = acc;
        else reinterpret_cast<__nv_bfloat16*>(p.o)[out_row * p.ldo + (int64_t)head * p.dh + d] = __float2bfloat16_rn(acc);
      }
      if (d == 0) {
        const float lse2 = total == 0.f ? -INFINITY : base + log2f(total);
        if (cut) p.part_lse[((int64_t)it.c * p.Nq + out_row) * p.n_heads + head] = lse2;
        else if (p.lse) p.lse[out_row * p.n_heads + head] = lse2 == -INFINITY ? lse2 : lse2 * 0.6931471805599453f;
      }
    }
    group_sync();                                              // s_bad and the warps' results are read
  }
  if (!ok && lane == 0) report_status(p.status, SP_ERR_TIMEOUT, (int32_t)blockIdx.x, 21);
  __syncthreads();
  if (s_abort) {              // a role gave up: copies in flight land before shared memory is released
    const long long t0 = clock64();
    while (clock64() - t0 < kDrainBudget) {}
  }
}

template <int DH, int ROWS>
sp_status launch_rows(const CUtensorMap& tmK, const CUtensorMap& tmV, const AttnParams& p, cudaStream_t stream) {
  using C = RowsCfg<DH, ROWS>;
  static PerDeviceOnce attr_once;
  const auto kernel = attention_rows_kernel<DH, ROWS>;
  if (attr_once.run([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM); }) != cudaSuccess)
    return SP_ERR_CUDA;
  const int64_t rows = (int64_t)p.Nq * p.g;
  const int64_t tiles = min(rows / ROWS + p.n_seq, (int64_t)p.Nq * ceil_div((int64_t)p.g, (int64_t)ROWS));
  const int64_t work = tiles * p.n_kv * (p.part > 0 ? p.max_parts : 1);
  const dim3 grid((unsigned)(work < sm_count() ? work : sm_count()));
  return launch(kernel, grid, dim3(kThreads), C::SMEM, stream, tmK, tmV, p) == cudaSuccess ? SP_OK : SP_ERR_CUDA;
}

}  // namespace

sp_status attention_rows(const AttnParams& a, cudaStream_t stream) {
  AttnParams p = a;
  p.wait_budget = wait_budget_cycles() > 0 ? wait_budget_cycles() : kWaitBudget;
  CUtensorMap tmK, tmV;
  if (!make_map3(&tmK, p.k, p.dh, p.n_kv, p.Nk, p.dh, p.ldk, 64, 1, kStage) ||
      !make_map3(&tmV, p.v, p.dh, p.n_kv, p.Nk, p.dh, p.ldv, 64, 1, kStage))
    return SP_ERR_CUDA;
  // eight rows where the sequences have no more on average
  const bool eight = (int64_t)p.Nq * p.g <= (int64_t)8 * p.n_seq;
  if (p.dh <= 64) return eight ? launch_rows<64, 8>(tmK, tmV, p, stream) : launch_rows<64, 16>(tmK, tmV, p, stream);
  return eight ? launch_rows<128, 8>(tmK, tmV, p, stream) : launch_rows<128, 16>(tmK, tmV, p, stream);
}

}  // namespace sp
