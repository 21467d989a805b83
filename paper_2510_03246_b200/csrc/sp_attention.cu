// Attention forward over packed sequences: entry points, the CUDA-core kernel, and the join of a key axis that was cut into
// parts.
//
// O_i = sum_j p_ij V_j with p = softmax(scale Q K^T): one pass over the keys, tile by tile, with the running maximum r and
// sum l of a row: when r rises to r', l and the row of O are scaled by 2^(r - r').  Logits are held in base 2.
#include <math.h>

#include "sp_attention.cuh"
#include "sp_f32x2.cuh"

namespace sp {
namespace {

constexpr int kBN = 64;                // keys per tile
constexpr int kSimtThreads = 256;

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// A tile of BM rows (queries x the heads that share a key head) against tiles of 64 keys.  256 threads as 16 x 16: a thread
// has BM / 16 rows x 4 keys (tx, tx + 16, ...) of the logits and BM / 16 rows x DH / 16 columns of O.  Operands lie in shared memory as fp32
// in rows of a pitch 4 beyond a multiple of 32, so that both products read 16-byte pieces along their inner index, eight lanes on
// eight rows without a bank twice.  What bounds it is those reads beside the multiply-adds: with 128 rows twelve for 128 (the logits' sums over
// even and over odd channels side by side, two to an instruction), with 64 eight for 64.
template <typename T, int DH, int BM>
struct SimtTile {
  static constexpr int P = DH + 4, PP = kBN + 4;
  static constexpr int kQ = BM * P, kK = kBN * P, kV = kBN * P, kP = BM * PP;
  static constexpr size_t SMEM = (size_t)(kQ + kK + kV + kP) * sizeof(float);
};
// rows [0, n) of a [.., dh] head into shared memory, zero beyond n and dh; row(i): where row i starts
template <typename T, int DH, int ROWS, typename F>
__device__ __forceinline__ void load_rows(float* dst, int n, int dh, bool vec, float scale, F&& row) {
  constexpr int P = DH + 4;
  for (int e = threadIdx.x; e < ROWS * (DH / 4); e += kSimtThreads) {
    const int i = e / (DH / 4), d = e % (DH / 4) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < n && d < dh) {
      const T* src = row(i) + d;
      if (sizeof(T) == 4 && vec) {
        v = *reinterpret_cast<const float4*>(src);
      } else {
        v.x = load1(src);
        if (d + 1 < dh) v.y = load1(src + 1);
        if (d + 2 < dh) v.z = load1(src + 2);
        if (d + 3 < dh) v.w = load1(src + 3);
      }
      v.x *= scale; v.y *= scale; v.z *= scale; v.w *= scale;
    }
    *reinterpret_cast<float4*>(dst + i * P + d) = v;
  }
}

template <typename T, int DH, int BM>
__global__ void __launch_bounds__(kSimtThreads) attention_simt_kernel(const AttnParams p) {
  kernel_begin();
  using L = SimtTile<T, DH, BM>;
  constexpr int TM = BM / 16, TD = DH / 16;
  extern __shared__ __align__(16) float sm[];
  float* sq = sm;
  float* sk = sq + L::kQ;
  float* sv = sk + L::kK;
  float* sp_ = sv + L::kV;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const T* Q = reinterpret_cast<const T*>(p.q);
  const T* K = reinterpret_cast<const T*>(p.k);
  const T* V = reinterpret_cast<const T*>(p.v);
  const auto aligned = [&](const void* ptr, int64_t ld) {
    return p.dh % 4 == 0 && ld % 4 == 0 && (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0;
  };
  const bool vq = aligned(Q, p.ldq), vk = aligned(K, p.ldk), vv = aligned(V, p.ldv);
  AttnDealer dealer;
  AttnItem it;
  for (int64_t item = blockIdx.x; dealer.find(p, item, BM, p.g, p.n_kv, it); item += gridDim.x) {
    const int rows = (int)min((int64_t)BM, (int64_t)it.nq * p.g - (int64_t)it.tile * BM);
    const int64_t r0 = (int64_t)it.tile * BM;
    const int64_t shift = p.causal ? (int64_t)it.nk - it.nq : (int64_t)it.nk;       // query i sees keys j <= i + shift
    const int last_q = (int)((r0 + rows - 1) / p.g);
    const int seen = (int)max((int64_t)0, min((int64_t)it.nk, last_q + shift + 1));
    const bool cut = p.part > 0 && it.nk > p.part;
    const int kb = cut ? it.c * p.part : 0;
    const int ke = cut && seen - kb > p.part ? kb + p.part : seen;
    __syncthreads();
    load_rows<T, DH, BM>(sq, rows, p.dh, vq, p.scale_log2, [&](int i) {
      const int64_t rr = r0 + i;
      return Q + (it.q0 + rr / p.g) * p.ldq + (it.head * p.g + rr % p.g) * (int64_t)p.dh;
    });
    float o[TM][TD], m[TM], l[TM];
    int lim[TM];                      // keys [0, lim) are visible to the row
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
      const int64_t qi = (r0 + ty * TM + i) / p.g;
      lim[i] = (int)max((int64_t)0, min((int64_t)it.nk, qi + shift + 1));
#pragma unroll
      for (int j = 0; j < TD; ++j) o[i][j] = 0.f;
    }
    for (int kt = kb; kt < ke; kt += kBN) {
      __syncthreads();                // the tile before has been read
      load_rows<T, DH, kBN>(sk, ke - kt, p.dh, vk, 1.f, [&](int j) {
        return K + ((int64_t)it.k0 + kt + j) * p.ldk + it.head * (int64_t)p.dh;
      });
      load_rows<T, DH, kBN>(sv, ke - kt, p.dh, vv, 1.f, [&](int j) {
        return V + ((int64_t)it.k0 + kt + j) * p.ldv + it.head * (int64_t)p.dh;
      });
      __syncthreads();
      float s[TM][4];
      {
        uint64_t s2[TM][4];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) s2[i][j] = 0ull;
#pragma unroll 4
        for (int d = 0; d < DH; d += 4) {
          ulonglong2 kf[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) kf[j] = *reinterpret_cast<const ulonglong2*>(sk + (tx + 16 * j) * L::P + d);
#pragma unroll
          for (int i = 0; i < TM; ++i) {
            const ulonglong2 qf = *reinterpret_cast<const ulonglong2*>(sq + (ty * TM + i) * L::P + d);
#pragma unroll
            for (int j = 0; j < 4; ++j) s2[i][j] = fma2(qf.y, kf[j].y, fma2(qf.x, kf[j].x, s2[i][j]));
          }
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float a, b;
            unpack2(s2[i][j], a, b);
            s[i][j] = a + b;
          }
      }
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (kt + tx + 16 * j >= lim[i] || tx + 16 * j >= ke - kt) s[i][j] = -INFINITY;
          mx = fmaxf(mx, s[i][j]);    // (a NaN is passed over here and stays one in the exponential)
        }
#pragma unroll
        for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
        const float mn = fmaxf(m[i], mx), ref = mn == -INFINITY ? 0.f : mn;
        const float f = exp2_fast(m[i] - ref);
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[i][j] = exp2_fast(s[i][j] - ref);
          sum += s[i][j];
        }
#pragma unroll
        for (int w = 8; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        l[i] = fmaf(l[i], f, sum);
        m[i] = mn;
#pragma unroll
        for (int j = 0; j < TD; ++j) o[i][j] *= f;
#pragma unroll
        for (int j = 0; j < 4; ++j) sp_[(ty * TM + i) * L::PP + tx + 16 * j] = s[i][j];
      }
      __syncwarp();                   // a warp's rows of P are its own: two values of ty
      // In a tile that the mask cuts, a key beyond a row's limit is not touched at all: 0 times a NaN in V is no 0.
      if (kt + kBN <= lim[0]) {          // (rows rise with i and see no fewer keys)
#pragma unroll 2
        for (int j = 0; j < kBN; j += 4) {
          float4 pf[TM];
#pragma unroll
          for (int i = 0; i < TM; ++i) pf[i] = *reinterpret_cast<const float4*>(sp_ + (ty * TM + i) * L::PP + j);
#pragma unroll
          for (int c = 0; c < TD; c += 4)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const float4 vf = *reinterpret_cast<const float4*>(sv + (j + y) * L::P + (c / 4) * 64 + tx * 4);
#pragma unroll
              for (int i = 0; i < TM; ++i) {
                const float pv = y == 0 ? pf[i].x : y == 1 ? pf[i].y : y == 2 ? pf[i].z : pf[i].w;
                o[i][c] = fmaf(pv, vf.x, o[i][c]);
                o[i][c + 1] = fmaf(pv, vf.y, o[i][c + 1]);
                o[i][c + 2] = fmaf(pv, vf.z, o[i][c + 2]);
                o[i][c + 3] = fmaf(pv, vf.w, o[i][c + 3]);
              }
            }
        }
      } else {
        const int jend = min(kBN, ke - kt);
        for (int j = 0; j < jend; ++j) {
          float pv[TM];
#pragma unroll
          for (int i = 0; i < TM; ++i) pv[i] = sp_[(ty * TM + i) * L::PP + j];
#pragma unroll
          for (int c = 0; c < TD; c += 4) {
            const float4 vf = *reinterpret_cast<const float4*>(sv + j * L::P + (c / 4) * 64 + tx * 4);
#pragma unroll
            for (int i = 0; i < TM; ++i)
              if (kt + j < lim[i]) {
                o[i][c] = fmaf(pv[i], vf.x, o[i][c]);
                o[i][c + 1] = fmaf(pv[i], vf.y, o[i][c + 1]);
                o[i][c + 2] = fmaf(pv[i], vf.z, o[i][c + 2]);
                o[i][c + 3] = fmaf(pv[i], vf.w, o[i][c + 3]);
              }
          }
        }
      }
      __syncwarp();
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      if (ty * TM + i >= rows) continue;
      const int64_t rr = r0 + ty * TM + i, row = it.q0 + rr / p.g;
      const int h = it.head * p.g + (int)(rr % p.g);
      // a row without a visible key: l = 0
      const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
      const float lse2 = l[i] == 0.f ? -INFINITY : m[i] + log2f(l[i]);
      float* po = cut ? p.part_o + ((int64_t)it.c * p.Nq + row) * ((int64_t)p.n_heads * p.dh) + (int64_t)h * p.dh : nullptr;
      T* out = reinterpret_cast<T*>(p.o) + row * p.ldo + (int64_t)h * p.dh;
#pragma unroll
      for (int c = 0; c < TD; ++c) {
        const int d = (c / 4) * 64 + tx * 4 + c % 4;
        if (d >= p.dh) continue;
        if (cut) po[d] = o[i][c] * inv;
        else store1(out + d, o[i][c] * inv);
      }
      if (tx == 0) {
        if (cut) p.part_lse[((int64_t)it.c * p.Nq + row) * p.n_heads + h] = lse2;
        else if (p.lse) p.lse[row * p.n_heads + h] = lse2 == -INFINITY ? lse2 : lse2 * 0.6931471805599453f;
      }
    }
  }
}

// O_i = sum_c w_c O_ic / sum_c w_c with w_c = 2^(lse_ic - max): one warp per row and head.  Rows of sequences that are not
// cut have their result already.
template <typename T>
__global__ void __launch_bounds__(256) attention_join_kernel(const AttnParams p) {
  kernel_begin();
  const int64_t idx = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (idx >= (int64_t)p.Nq * p.n_heads) return;
  const int32_t row = (int32_t)(idx / p.n_heads), h = (int32_t)(idx % p.n_heads);
  if (row < AttnDealer::bound(p.cu_q[0], p.Nq) || row >= AttnDealer::bound(p.cu_q[p.n_seq], p.Nq)) return;
  int lo = 0, hi = p.n_seq;           // the last sequence that starts at or before the row
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (AttnDealer::bound(p.cu_q[mid], p.Nq) <= row) lo = mid;
    else hi = mid;
  }
  const int nk = AttnDealer::bound(p.cu_k[lo + 1], p.Nk) - AttnDealer::bound(p.cu_k[lo], p.Nk);
  if (nk <= p.part) return;
  const int parts = (nk - 1) / p.part + 1;
  const float* lses = p.part_lse + (int64_t)row * p.n_heads + h;
  const int64_t lse_step = (int64_t)p.Nq * p.n_heads, o_step = lse_step * p.dh;
  float mx = -INFINITY;
  bool bad = false;                   // (fmaxf passes over a NaN)
  for (int c = lane; c < parts; c += 32) {
    const float lc = lses[c * lse_step];
    mx = fmaxf(mx, lc);
    bad |= lc != lc;
  }
#pragma unroll
  for (int w = 16; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
  const float ref = mx == -INFINITY ? 0.f : mx;
  bad = __any_sync(0xffffffffu, bad);
  // a lane has channels 4 lane ..; what a part without a visible key left (lse -infinity) is zeros
  const int d = 4 * lane;
  float acc[4] = {0.f, 0.f, 0.f, 0.f}, total = 0.f;
  const float* po = p.part_o + ((int64_t)row * p.n_heads + h) * p.dh + d;
  for (int c0 = 0; c0 < parts; c0 += 32) {
    const float wl = c0 + lane < parts ? exp2f(lses[(c0 + lane) * lse_step] - ref) : 0.f;
    const int m = min(32, parts - c0);
#pragma unroll 8
    for (int c = 0; c < m; ++c) {
      const float w = __shfl_sync(0xffffffffu, wl, c);
      total += w;
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (d + x < p.dh) acc[x] = fmaf(w, po[(c0 + c) * o_step + x], acc[x]);
    }
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
  T* out = reinterpret_cast<T*>(p.o) + (int64_t)row * p.ldo + (int64_t)h * p.dh + d;
#pragma unroll
  for (int x = 0; x < 4; ++x)
    if (d + x < p.dh) store1(out + x, bad ? NAN : acc[x] * inv);
  if (lane == 0 && p.lse)
    p.lse[(int64_t)row * p.n_heads + h] = bad ? NAN : total == 0.f ? -INFINITY : (ref + log2f(total)) * 0.6931471805599453f;
}

template <typename T, int DH, int BM>
cudaError_t launch_simt(const AttnParams& p, cudaStream_t stream) {
  using L = SimtTile<T, DH, BM>;
  static PerDeviceOnce attr_once;
  const auto kernel = attention_simt_kernel<T, DH, BM>;
  const cudaError_t e = attr_once.run(
      [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)L::SMEM); });
  if (e != cudaSuccess) return e;
  // as many blocks as can be resident and have work
  const int64_t rows = (int64_t)p.Nq * p.g;
  const int64_t tiles = min(rows / BM + p.n_seq, (int64_t)p.Nq * ceil_div((int64_t)p.g, (int64_t)BM));
  const int64_t work = tiles * p.n_kv * (p.part > 0 ? p.max_parts : 1);
  const int64_t resident = (int64_t)sm_count() * (L::SMEM > 113 * 1024 ? 1 : L::SMEM > 75 * 1024 ? 2 : 3);
  const dim3 grid((unsigned)(work < resident ? work : resident));
  return launch(kernel, grid, dim3(kSimtThreads), L::SMEM, stream, p);
}

template <typename T>
cudaError_t launch_simt(const AttnParams& p, cudaStream_t stream) {
  // 16 rows where the sequences have no more on average (single tokens): a tile's products are the bound there.  128 rows where heads
  // are wider than 64 and that leaves tiles enough for the SMs (4 x 2048, 64 / 128 rows: heads of 128 6.1 / 4.6 ms, of 64 1.2 / 1.3 ms).
  const int64_t rows = (int64_t)p.Nq * p.g;
  const int bm = attention_few_rows(p.Nq, p.g, p.n_seq) ? 16 : p.dh > 64 && rows / 128 * p.n_kv >= 4 * (int64_t)sm_count() ? 128 : 64;
  if (p.dh <= 64) return bm == 16 ? launch_simt<T, 64, 16>(p, stream) : launch_simt<T, 64, 64>(p, stream);
  return bm == 16 ? launch_simt<T, 128, 16>(p, stream) : bm == 64 ? launch_simt<T, 128, 64>(p, stream) : launch_simt<T, 128, 128>(p, stream);
}

struct Cut {
  int32_t part = 0, max_parts = 1;
  size_t bytes = 0;
};
// Whether and how the key axis is cut.  Without a cut there are about Nq g / 128 tiles of rows, at least one for every sequence
// that has queries, times the key heads; fewer than the SMs (148) leave SMs idle.  Parts are then as long as gives four for every SM
// (so that sequences of different lengths even out), at least 256 keys.  With few rows an SM reads 1024 keys of a bf16 head (512 in fp32) in 5 us, about what a second
// launch and the results' way through memory cost: shorter parts do not pay, and beyond 4096 keys for an SM it gets eight.
// Least keys of a part halved / as here / doubled, us with cold caches: bf16, 1 token after 16384 keys, 32 heads of 128 on 8: 39 / 33 / 31, 4 after 8192
// 51 / 45 / 43, 16 after 4096 74 / 72 / 70; fp32, 4 after 2048 39 / 33 / 47; tiles, 128 after 8064 (8 heads of 128) 59 / 41 / 31, 300 after 700 (4 of
// 64) 23 / 23 / 25.  Four / eight parts for an SM: 16 after 16384 191 / 195, 16 after 2048 .. 31013 equal.
// Sequences that are no longer than a part on average are not cut; one of average length falls into equal parts.
Cut plan_cut(int64_t Nq, int64_t Nk, int32_t n_seq, int32_t n_heads, int32_t n_kv, int32_t dh, int32_t dtype) {
  Cut cut;
  if (Nq < 1 || Nk < 1 || n_seq < 1) return cut;
  const int64_t g = n_heads / n_kv, sms = 148;
  const int64_t seqs = n_seq < Nq ? n_seq : Nq;
  const int64_t tiles = (Nq * g / 128 > seqs ? Nq * g / 128 : seqs) * n_kv;
  const int64_t per_tile = ceil_div(Nk, seqs);                 // keys of a tile, on average
  const bool few = attention_few_rows(Nq, g, n_seq);
  const int64_t per_sm = few && tiles * per_tile > sms * 4096 ? 8 : 4;
  if (tiles >= sms * per_sm / 2) return cut;
  int64_t part = (int64_t)align_up((size_t)ceil_div(tiles * per_tile, sms * per_sm), 128);
  const int64_t least = !few ? 256 : dtype == SP_F32 ? 512 : 1024;
  if (part < least) part = least;
  if (part >= per_tile) return cut;                             // (a longer sequence among many short ones is not worth it)
  part = (int64_t)align_up((size_t)ceil_div(per_tile, ceil_div(per_tile, part)), 128);
  const int64_t parts = ceil_div(Nk, part);
  const int64_t elems = parts * Nq * n_heads;
  if (elems * (dh + 1) * 4 > (int64_t)1 << 30) return cut;
  cut.part = (int32_t)part;
  cut.max_parts = (int32_t)parts;
  cut.bytes = align_up((size_t)(elems * dh * 4), 256) + (size_t)(elems * 4);
  return cut;
}

}  // namespace
}  // namespace sp

extern "C" {

size_t sp_attention_workspace_bytes(int64_t Nq, int64_t Nk, int32_t n_seq, int32_t n_heads, int32_t n_kv_heads,
                                    int32_t d_head, int32_t dtype) {
  if (Nq < 0 || Nk < 0 || Nq > (1 << 30) || Nk > (1 << 30)) return 0;
  if (n_seq < 0 || n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads != 0 || d_head < 1 || d_head > 128) return 0;
  return sp::plan_cut(Nq, Nk, n_seq, n_heads, n_kv_heads, d_head, dtype).bytes;
}

sp_status sp_attention(const sp_attention_args* a, int32_t* status_dev, void* ws, size_t ws_bytes, void* stream) {
  using namespace sp;
  if (!a) return SP_ERR_INVALID_ARG;
  const int32_t dt = a->Q.dtype;
  if (dt != SP_F32 && dt != SP_BF16) return SP_ERR_DTYPE;
  if (a->K.dtype != dt || a->V.dtype != dt || a->O.dtype != dt) return SP_ERR_DTYPE;
  if (a->n_heads < 1 || a->n_kv_heads < 1 || a->n_heads % a->n_kv_heads != 0 || a->n_seq < 0) return SP_ERR_SHAPE;
  const int64_t Nq = a->Q.rows, Nk = a->K.rows;
  if (Nq < 0 || Nk < 0 || Nq > (1 << 30) || Nk > (1 << 30)) return SP_ERR_SHAPE;
  if (a->Q.cols < 1 || a->Q.cols % a->n_heads != 0 || a->Q.cols > (1 << 30)) return SP_ERR_SHAPE;
  const int64_t dh = a->Q.cols / a->n_heads;
  if (dh > 128) return SP_ERR_UNSUPPORTED;
  if (a->O.rows != Nq || a->O.cols != a->Q.cols || a->V.rows != Nk || a->K.cols != dh * a->n_kv_heads ||
      a->V.cols != a->K.cols)
    return SP_ERR_SHAPE;
  if ((Nq > 1 && (a->Q.ld < a->Q.cols || a->O.ld < a->O.cols)) || (Nk > 1 && (a->K.ld < a->K.cols || a->V.ld < a->V.cols)))
    return SP_ERR_SHAPE;
  if (Nq * a->n_heads > ((int64_t)1 << 33)) return SP_ERR_SHAPE;       // (blocks of the join)
  if (!(a->scale >= 1e-30) || !(a->scale <= 1e30)) return SP_ERR_INVALID_ARG;
  if (Nq == 0 || a->n_seq == 0) return SP_OK;
  if (!a->Q.ptr || !a->O.ptr || !a->cu_q || !a->cu_k || (Nk > 0 && (!a->K.ptr || !a->V.ptr))) return SP_ERR_INVALID_ARG;
  const Cut cut = plan_cut(Nq, Nk, a->n_seq, a->n_heads, a->n_kv_heads, (int32_t)dh, dt);
  if (cut.part > 0) {
    if (!ws || ws_bytes < cut.bytes) return SP_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(ws) & 255u) return SP_ERR_ALIGNMENT;
  }
  AttnParams p = {};
  p.q = a->Q.ptr; p.k = a->K.ptr; p.v = a->V.ptr; p.o = a->O.ptr;
  // (a single row has no pitch: whatever stands there is not used)
  p.ldq = Nq > 1 ? a->Q.ld : a->Q.cols; p.ldk = Nk > 1 ? a->K.ld : a->K.cols;
  p.ldv = Nk > 1 ? a->V.ld : a->V.cols; p.ldo = Nq > 1 ? a->O.ld : a->O.cols;
  p.lse = a->lse;
  p.cu_q = a->cu_q; p.cu_k = a->cu_k;
  p.Nq = (int32_t)Nq; p.Nk = (int32_t)Nk;
  p.n_seq = a->n_seq; p.n_heads = a->n_heads; p.n_kv = a->n_kv_heads; p.g = a->n_heads / a->n_kv_heads;
  p.dh = (int32_t)dh; p.causal = a->causal != 0;
  p.scale_log2 = (float)(a->scale * 1.4426950408889634);
  p.part = cut.part; p.max_parts = cut.max_parts;
  if (cut.part > 0) {
    p.part_o = reinterpret_cast<float*>(ws);
    p.part_lse = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(ws) +
                                          align_up((size_t)cut.max_parts * Nq * a->n_heads * dh * 4, 256));
  }
  p.status = status_dev;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const bool tc = dt == SP_BF16 && attention_tc_supported(p);
  ProfScope prof(tc ? PK_GEMM_TC : PK_GEMM_SIMT, 0.0, 0.0, s);
  count_launch();
  if (tc && attention_few_rows(Nq, p.g, a->n_seq)) {
    const sp_status st = attention_rows(p, s);
    if (st != SP_OK) return st;
  } else if (tc) {
    const sp_status st = attention_tc(p, s);
    if (st != SP_OK) return st;
  } else if (dt == SP_F32 && attention_few_rows(Nq, p.g, a->n_seq) && attention_rows_f32_supported(p)) {
    if (attention_rows_f32(p, s) != cudaSuccess) return SP_ERR_CUDA;
  } else if ((dt == SP_F32 ? launch_simt<float>(p, s) : launch_simt<__nv_bfloat16>(p, s)) != cudaSuccess) return SP_ERR_CUDA;
  if (cut.part > 0) {
    count_launch();
    const OverlapScope overlap(true);       // its blocks start while the parts end
    const dim3 grid((unsigned)ceil_div(Nq * a->n_heads, (int64_t)8));
    const cudaError_t e = dt == SP_F32 ? launch(attention_join_kernel<float>, grid, dim3(256), 0, s, p)
                                       : launch(attention_join_kernel<__nv_bfloat16>, grid, dim3(256), 0, s, p);
    if (e != cudaSuccess) return SP_ERR_CUDA;
  }
  return SP_OK;
}

}  // extern "C"
