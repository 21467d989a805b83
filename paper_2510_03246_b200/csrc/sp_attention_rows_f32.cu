// fp32 attention of few rows against long caches (single new tokens): bound by reading K and V once, like the bf16 form
// (sp_attention_rows.cu), but with the products on the CUDA cores, since no matrix instruction keeps 24 bits.
//
// A block takes 64 keys at a time through a ring of asynchronous copies.  S: four lanes share a key, each with every fourth 16-byte piece of its
// row, for all rows of the tile.  A warp per row turns S into P with the running maximum and sum.  O: a thread has four channels and a share of the
// keys, for all rows; the shares meet at the end of an item.  Per key and channel one 16-byte read serves as many multiply-adds as there are
// rows, so up to eight rows the SM has work for less than the time the keys take to arrive.  16 tokens after 4096 keys, 32 heads of 128 on 8:
// 857 us with tiles of 16 rows x 64 keys (sp_attention.cu), 180 us here.
#include <math.h>

#include "sp_attention.cuh"
#include "sp_f32x2.cuh"

namespace sp {
namespace {

constexpr int kKeys = 64, kThreads = 256;

template <int DH, int ROWS>
struct F32Cfg {
  static constexpr int STAGES = DH == 128 ? 3 : 5;
  static constexpr int PK = DH + 16;                       // floats of a row of K: two rows side by side touch all banks once
  static constexpr int STAGE = kKeys * (PK + DH);          // K, then V
  static constexpr int GROUPS = kThreads / (DH / 4);       // shares of the keys in O += P V
  static constexpr int PP = ROWS + 4;                      // floats of a key's row of S and P
  static constexpr int REST = ROWS * DH + kKeys * PP + 3 * ROWS;
  static constexpr size_t SMEM = ((size_t)STAGES * STAGE + REST) * sizeof(float);
  static_assert(GROUPS * ROWS * DH <= STAGES * STAGE, "the shares of O meet in the ring");
};

__device__ __forceinline__ void copy_async(float* dst, const float* src, bool in) {
  const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int DH, int ROWS>
__global__ void __launch_bounds__(kThreads, 1) attention_rows_f32_kernel(const AttnParams p) {
  kernel_begin();
  using C = F32Cfg<DH, ROWS>;
  constexpr int RW = (ROWS + 7) / 8;                       // rows of a warp in the softmax
  extern __shared__ __align__(16) float sm[];
  float* s_q = sm + C::STAGES * C::STAGE;                  // [ROWS][DH], times the scale
  float* s_p = s_q + ROWS * DH;                            // [key][PP]
  float* s_f = s_p + kKeys * C::PP;                        // what O is scaled by in this step
  float* s_m = s_f + ROWS;
  float* s_l = s_m + ROWS;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int key4 = tid >> 2, q4 = tid & 3;                 // S: key of the stage, which pieces of its row
  const int c4 = tid % (DH / 4) * 4, kg = tid / (DH / 4);  // O: first channel, share of the keys
  const float* Q = reinterpret_cast<const float*>(p.q);
  AttnDealer dealer;
  AttnItem it;
  for (int64_t item = blockIdx.x; dealer.find(p, item, ROWS, p.g, p.n_kv, it); item += gridDim.x) {
    const int64_t r0 = (int64_t)it.tile * ROWS;
    const int rows = (int)min((int64_t)ROWS, (int64_t)it.nq * p.g - r0);
    const int64_t shift = p.causal ? (int64_t)it.nk - it.nq : (int64_t)it.nk;
    auto visible = [&](int64_t token) { return (int)max((int64_t)0, min((int64_t)it.nk, token + shift + 1)); };
    const int sure = visible(r0 / p.g);
    int seen = visible((r0 + rows - 1) / p.g);
    const bool cut = p.part > 0 && it.nk > p.part;
    const int kb = cut ? it.c * p.part : 0;
    if (cut && seen - kb > p.part) seen = kb + p.part;
    const int n = seen > kb ? (seen - kb + kKeys - 1) / kKeys : 0;
    const float* K = reinterpret_cast<const float*>(p.k) + (int64_t)it.k0 * p.ldk + it.head * (int64_t)p.dh;
    const float* V = reinterpret_cast<const float*>(p.v) + (int64_t)it.k0 * p.ldv + it.head * (int64_t)p.dh;
    auto fetch = [&](int i) {
      if (i < n) {
        float* kd = sm + (i % C::STAGES) * C::STAGE;
        float* vd = kd + kKeys * C::PK;
#pragma unroll
        for (int e = tid; e < kKeys * (DH / 4); e += kThreads) {
          const int j = e / (DH / 4), d = e % (DH / 4) * 4, key = kb + i * kKeys + j;
          const bool in = key < seen && d < p.dh;
          // (where nothing is read the address still has to be one of 16 bytes: K's first)
          copy_async(kd + j * C::PK + d, in ? K + (int64_t)key * p.ldk + d : reinterpret_cast<const float*>(p.k), in);
          copy_async(vd + j * DH + d, in ? V + (int64_t)key * p.ldv + d : reinterpret_cast<const float*>(p.k), in);
        }
      }
      commit_copies();
    };
    __syncthreads();                                       // (the item before has left the ring)
    for (int i = 0; i < C::STAGES - 1; ++i) fetch(i);
    for (int e = tid; e < ROWS * DH; e += kThreads) {
      const int r = e / DH, d = e % DH;
      const int64_t rr = r0 + r;
      s_q[e] = r < rows && d < p.dh
                   ? Q[(it.q0 + rr / p.g) * p.ldq + (it.head * (int64_t)p.g + rr % p.g) * p.dh + d] * p.scale_log2 : 0.f;
    }
    float o[ROWS][4];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
      for (int x = 0; x < 4; ++x) o[r][x] = 0.f;
    float m[RW], l[RW];                                    // of this warp's rows, the same in all lanes
    int lim[RW];
#pragma unroll
    for (int y = 0; y < RW; ++y) {
      m[y] = -INFINITY;
      l[y] = 0.f;
      const int row = warp + 8 * y;
      lim[y] = row < rows ? min(visible((r0 + row) / p.g), seen) : 0;
    }
    for (int i = 0; i < n; ++i) {
      wait_copies<C::STAGES - 2>();
      __syncthreads();                                     // stage i is there, and stage i - 1 has been read
      fetch(i + C::STAGES - 1);
      const float* ks = sm + (i % C::STAGES) * C::STAGE;
      const float* vs = ks + kKeys * C::PK;
      const int kt = kb + i * kKeys;
      {
        uint64_t a[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) a[r] = 0ull;
#pragma unroll 4
        for (int j = 0; j < DH / 16; ++j) {
          const int d = 4 * (q4 + 4 * j);
          const ulonglong2 kf = *reinterpret_cast<const ulonglong2*>(ks + key4 * C::PK + d);
#pragma unroll
          for (int r = 0; r < ROWS; ++r) {
            const ulonglong2 qf = *reinterpret_cast<const ulonglong2*>(s_q + r * DH + d);
            a[r] = fma2(qf.y, kf.y, fma2(qf.x, kf.x, a[r]));
          }
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          float x, y;
          unpack2(a[r], x, y);
          x += y;
          x += __shfl_xor_sync(0xffffffffu, x, 1);
          x += __shfl_xor_sync(0xffffffffu, x, 2);
          if (q4 == r % 4) s_p[key4 * C::PP + r] = x;
        }
      }
      __syncthreads();
#pragma unroll
      for (int y = 0; y < RW; ++y) {
        const int row = warp + 8 * y;
        if (row < ROWS) {
          float s0 = s_p[lane * C::PP + row], s1 = s_p[(lane + 32) * C::PP + row];
          if (kt + lane >= lim[y]) s0 = -INFINITY;
          if (kt + lane + 32 >= lim[y]) s1 = -INFINITY;
          float mx = fmaxf(s0, s1);                        // (a NaN is passed over here and stays one in the exponential)
#pragma unroll
          for (int w = 16; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
          const float mn = fmaxf(m[y], mx), ref = mn == -INFINITY ? 0.f : mn, f = exp2_fast(m[y] - ref);
          s0 = exp2_fast(s0 - ref);
          s1 = exp2_fast(s1 - ref);
          float sum = s0 + s1;
#pragma unroll
          for (int w = 16; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
          l[y] = fmaf(l[y], f, sum);
          m[y] = mn;
          s_p[lane * C::PP + row] = s0;
          s_p[(lane + 32) * C::PP + row] = s1;
          if (lane == 0) s_f[row] = f;
        }
      }
      __syncthreads();
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const float f = s_f[r];
#pragma unroll
        for (int x = 0; x < 4; ++x) o[r][x] *= f;
      }
      constexpr int SHARE = kKeys / C::GROUPS;
      if (kt + kKeys <= sure) {
#pragma unroll
        for (int j = 0; j < SHARE; ++j) {
          const int key = kg * SHARE + j;
          const float4 vf = *reinterpret_cast<const float4*>(vs + key * DH + c4);
#pragma unroll
          for (int r = 0; r < ROWS; r += 4) {
            const float4 pf = *reinterpret_cast<const float4*>(s_p + key * C::PP + r);
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const float pv = y == 0 ? pf.x : y == 1 ? pf.y : y == 2 ? pf.z : pf.w;
              o[r + y][0] = fmaf(pv, vf.x, o[r + y][0]);
              o[r + y][1] = fmaf(pv, vf.y, o[r + y][1]);
              o[r + y][2] = fmaf(pv, vf.z, o[r + y][2]);
              o[r + y][3] = fmaf(pv, vf.w, o[r + y][3]);
            }
          }
        }
      } else {
        // a key that the mask hides from a row is not touched: 0 times a NaN in V is no 0
        for (int j = 0; j < SHARE; ++j) {
          const int key = kg * SHARE + j;
          const float4 vf = *reinterpret_cast<const float4*>(vs + key * DH + c4);
#pragma unroll
          for (int r = 0; r < ROWS; ++r) {
            if (r >= rows || kt + key >= min(visible((r0 + r) / p.g), seen)) continue;
            const float pv = s_p[key * C::PP + r];
            o[r][0] = fmaf(pv, vf.x, o[r][0]);
            o[r][1] = fmaf(pv, vf.y, o[r][1]);
            o[r][2] = fmaf(pv, vf.z, o[r][2]);
            o[r][3] = fmaf(pv, vf.w, o[r][3]);
          }
        }
      }
    }
    // the shares meet
    wait_copies<0>();
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROWS; ++r) *reinterpret_cast<float4*>(sm + (kg * ROWS + r) * DH + c4) = make_float4(o[r][0], o[r][1], o[r][2], o[r][3]);
#pragma unroll
    for (int y = 0; y < RW; ++y)
      if (lane == 0 && warp + 8 * y < ROWS) {
        s_m[warp + 8 * y] = m[y];
        s_l[warp + 8 * y] = l[y];
      }
    __syncthreads();
    for (int e = tid; e < rows * DH; e += kThreads) {
      const int r = e / DH, d = e % DH;
      if (d >= p.dh) continue;
      const int64_t rr = r0 + r, row = it.q0 + rr / p.g;
      const int h = it.head * p.g + (int)(rr % p.g);
      float acc = 0.f;
#pragma unroll
      for (int g = 0; g < C::GROUPS; ++g) acc += sm[(g * ROWS + r) * DH + d];
      const float sum = s_l[r], v = sum == 0.f ? 0.f : acc / sum;      // (no visible key: 0)
      if (cut) p.part_o[((int64_t)it.c * p.Nq + row) * ((int64_t)p.n_heads * p.dh) + (int64_t)h * p.dh + d] = v;
      else reinterpret_cast<float*>(p.o)[row * p.ldo + (int64_t)h * p.dh + d] = v;
      if (d == 0) {
        const float lse2 = sum == 0.f ? -INFINITY : s_m[r] + log2f(sum);
        if (cut) p.part_lse[((int64_t)it.c * p.Nq + row) * p.n_heads + h] = lse2;
        else if (p.lse) p.lse[row * p.n_heads + h] = lse2 == -INFINITY ? lse2 : lse2 * 0.6931471805599453f;
      }
    }
  }
}

template <int DH, int ROWS>
cudaError_t launch_rows_f32(const AttnParams& p, cudaStream_t stream) {
  using C = F32Cfg<DH, ROWS>;
  static PerDeviceOnce attr_once;
  const auto kernel = attention_rows_f32_kernel<DH, ROWS>;
  const cudaError_t e = attr_once.run([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM); });
  if (e != cudaSuccess) return e;
  const int64_t rows = (int64_t)p.Nq * p.g;
  const int64_t tiles = min(rows / ROWS + p.n_seq, (int64_t)p.Nq * ceil_div((int64_t)p.g, (int64_t)ROWS));
  const int64_t work = tiles * p.n_kv * (p.part > 0 ? p.max_parts : 1);
  return launch(kernel, dim3((unsigned)(work < sm_count() ? work : sm_count())), dim3(kThreads), C::SMEM, stream, p);
}

}  // namespace

bool attention_rows_f32_supported(const AttnParams& p) {
  const auto fits = [](const void* ptr, int64_t ld) { return ld % 4 == 0 && (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; };
  return p.dh % 4 == 0 && p.Nk > 0 && fits(p.k, p.ldk) && fits(p.v, p.ldv) && (reinterpret_cast<uintptr_t>(p.q) & 3u) == 0;
}

cudaError_t attention_rows_f32(const AttnParams& p, cudaStream_t stream) {
  const int64_t rows = (int64_t)p.Nq * p.g;               // as many rows as the sequences have on average
  if (p.dh <= 64)
    return rows <= 4 * (int64_t)p.n_seq ? launch_rows_f32<64, 4>(p, stream) : rows <= 8 * (int64_t)p.n_seq ? launch_rows_f32<64, 8>(p, stream)
                                                                            : launch_rows_f32<64, 16>(p, stream);
  return rows <= 4 * (int64_t)p.n_seq ? launch_rows_f32<128, 4>(p, stream) : rows <= 8 * (int64_t)p.n_seq ? launch_rows_f32<128, 8>(p, stream)
                                                                           : launch_rows_f32<128, 16>(p, stream);
}

}  // namespace sp
