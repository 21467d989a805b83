// Root-mean-square norm of the residual stream, and its gradient.
//
//   h = x + r,  y_j = w_j h_j rstd,  rstd = (sum_j h_j^2 / d + eps)^-1/2;   8 bits: scale = max_j |y_j| / 448, y8_j = e4m3(y_j / scale)
//   dh_j = rstd (w_j dy_j - h_j rstd^2 s / d) + the stream's own gradient,  s = sum_j w_j dy_j h_j;   dw_j = sum_t dy_tj h_tj rstd_t
//
// Both are bound by memory: every value is read once and stays in registers, eight to a chunk, up to four chunks per thread, while its
// row's sums are formed, so that nothing is read a second time (a row of 4096 is 128 threads' 32 values each).  Wider or unaligned rows
// take the looping kernels at the end, which read the row again for each pass (from L2).
#include <cuda_fp8.h>
#include <math.h>

#include "sp_common.cuh"

namespace sp {
namespace {

constexpr float kE4m3Max = 448.f;
constexpr float kLeastMax = 1e-30f;      // of a row's largest value: a row of zeros has a scale that can be divided by

__device__ __forceinline__ float get(const float* p) { return *p; }
__device__ __forceinline__ float get(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(__nv_fp8_storage_t* p, float v) { *p = __nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }

// eight values as they lie in memory (loaded together, turned into fp32 when they are used)
template <typename T> struct Raw8;
template <> struct Raw8<float> { float4 a, b; };
template <> struct Raw8<__nv_bfloat16> { uint4 a; };
__device__ __forceinline__ void fetch(Raw8<float>& r, const float* p) {
  r.a = *reinterpret_cast<const float4*>(p);
  r.b = *reinterpret_cast<const float4*>(p + 4);
}
__device__ __forceinline__ void fetch(Raw8<__nv_bfloat16>& r, const __nv_bfloat16* p) { r.a = *reinterpret_cast<const uint4*>(p); }
// the last chunk of a row whose width is no multiple of eight: nothing behind the row's last value is read, zeros stand for it
__device__ __forceinline__ void fetch_some(Raw8<float>& r, const float* p, int n) {
  r.a = make_float4(p[0], n > 1 ? p[1] : 0.f, n > 2 ? p[2] : 0.f, n > 3 ? p[3] : 0.f);
  r.b = make_float4(n > 4 ? p[4] : 0.f, n > 5 ? p[5] : 0.f, n > 6 ? p[6] : 0.f, 0.f);
}
__device__ __forceinline__ void fetch_some(Raw8<__nv_bfloat16>& r, const __nv_bfloat16* p, int n) {
  const uint16_t* u = reinterpret_cast<const uint16_t*>(p);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (2 * i < n ? (uint32_t)u[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)u[2 * i + 1] << 16 : 0u);
  r.a = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void open8(const Raw8<float>& r, float (&v)[8]) {
  v[0] = r.a.x; v[1] = r.a.y; v[2] = r.a.z; v[3] = r.a.w;
  v[4] = r.b.x; v[5] = r.b.y; v[6] = r.b.z; v[7] = r.b.w;
}
__device__ __forceinline__ void open8(const Raw8<__nv_bfloat16>& r, float (&v)[8]) {
  const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 e = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&e);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(__nv_fp8_storage_t* p, const float (&v)[8]) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    w[i] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[4 * i], v[4 * i + 1]), __NV_SATFINITE, __NV_E4M3) |
           (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[4 * i + 2], v[4 * i + 3]), __NV_SATFINITE, __NV_E4M3) << 16;
  *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
}
template <typename T>
__device__ __forceinline__ void store_some(T* p, const float (&v)[8], int n) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) put(p + i, v[i]);
}
// eight weights from column j on (ones without a weight; any alignment: they come from L1 or L2)
__device__ __forceinline__ void weights8(const float* w, int64_t j, int n, bool vec, float (&v)[8]) {
  if (w == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 1.f;
  } else if (vec && n == 8) {
    Raw8<float> r;
    fetch(r, w + j);
    open8(r, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? w[j + i] : 0.f;
  }
}

struct Sum {
  static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};
struct Max {
  static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); }
};
// over the TPR threads of a row (a warp, or the whole block), in a fixed order; s: a word per warp
template <typename Op, int TPR>
__device__ __forceinline__ float row_reduce(float v, float* s) {
#pragma unroll
  for (int w = 16; w > 0; w >>= 1) v = Op::of(v, __shfl_xor_sync(0xffffffffu, v, w));
  if (TPR > 32) {
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = s[0];
#pragma unroll
    for (int w = 1; w < TPR / 32; ++w) v = Op::of(v, s[w]);
  }
  return v;
}

struct NormParams {
  const void *x, *r;
  void *h, *y;
  const float* w;
  float *scale, *rstd;
  int64_t ldx, ldr, ldh, ldy, T;
  int32_t d, w_vec;
  float eps;
};

constexpr int kChunks = 4;
// TPR threads for a row, kChunks chunks of eight values each; blocks of one row, or of four warps and rows
template <typename TX, typename TR, typename TY, bool RES, int TPR>
__global__ void __launch_bounds__(TPR == 32 ? 128 : TPR) norm_kernel(const NormParams p) {
  kernel_begin();
  __shared__ float s_a[32], s_b[32];
  constexpr bool kEight = sizeof(TY) == 1;
  const int t = TPR == 32 ? threadIdx.x & 31 : threadIdx.x;
  const int64_t row = TPR == 32 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : (int64_t)blockIdx.x;
  if (row >= p.T) return;             // (a whole warp; blocks of one row are all there)
  const TX* x = reinterpret_cast<const TX*>(p.x) + row * p.ldx;
  const TR* r = reinterpret_cast<const TR*>(p.r) + (RES ? row * p.ldr : 0);
  float v[kChunks][8];
  {
    Raw8<TX> a[kChunks];
    Raw8<TR> b[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int j = (c * TPR + t) * 8;
      a[c] = Raw8<TX>();
      b[c] = Raw8<TR>();
      if (j + 8 <= p.d) {
        fetch(a[c], x + j);
        if (RES) fetch(b[c], r + j);
      } else if (j < p.d) {
        fetch_some(a[c], x + j, p.d - j);
        if (RES) fetch_some(b[c], r + j, p.d - j);
      }
    }
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      open8(a[c], v[c]);
      if (RES) {
        float u[8];
        open8(b[c], u);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] += u[i];
      }
    }
  }
  float ss = 0.f;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    float part = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) part = fmaf(v[c][i], v[c][i], part);
    ss += part;
  }
  ss = row_reduce<Sum, TPR>(ss, s_a);
  const float rstd = 1.f / sqrtf(ss / (float)p.d + p.eps);
  if (t == 0 && p.rstd) p.rstd[row] = rstd;
  float top = 0.f;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int j = (c * TPR + t) * 8, n = p.d - j < 8 ? p.d - j : 8;
    if (n <= 0) continue;
    if (p.h) {
      TR* h = reinterpret_cast<TR*>(p.h) + row * p.ldh + j;
      if (n == 8) store8(h, v[c]);
      else store_some(h, v[c], n);
    }
    float w[8];
    weights8(p.w, j, n, p.w_vec != 0, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[c][i] = v[c][i] * rstd * w[i];
      if (kEight) top = fmaxf(top, fabsf(v[c][i]));
    }
  }
  float inv = 1.f;
  if (kEight) {
    top = fmaxf(row_reduce<Max, TPR>(top, s_b), kLeastMax);
    inv = kE4m3Max / top;
    if (t == 0) p.scale[row] = top / kE4m3Max;
  }
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int j = (c * TPR + t) * 8, n = p.d - j < 8 ? p.d - j : 8;
    if (n <= 0) continue;
    if (kEight) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] *= inv;
    }
    TY* y = reinterpret_cast<TY*>(p.y) + row * p.ldy + j;
    if (n == 8) store8(y, v[c]);
    else store_some(y, v[c], n);
  }
}

// Any width and alignment: a block per row, the row read again for each pass.  What is written stands where this thread has read.
template <typename TX, typename TR, typename TY, bool RES>
__global__ void __launch_bounds__(512) norm_loop_kernel(const NormParams p) {
  kernel_begin();
  __shared__ float s_a[32], s_b[32];
  constexpr bool kEight = sizeof(TY) == 1;
  const int64_t row = blockIdx.x;
  const TX* x = reinterpret_cast<const TX*>(p.x) + row * p.ldx;
  const TR* r = reinterpret_cast<const TR*>(p.r) + (RES ? row * p.ldr : 0);
  const auto sum = [&](int j) { return RES ? get(x + j) + get(r + j) : get(x + j); };
  float ss = 0.f;
  for (int j = threadIdx.x; j < p.d; j += 512) {
    const float h = sum(j);
    ss = fmaf(h, h, ss);
  }
  ss = row_reduce<Sum, 512>(ss, s_a);
  const float rstd = 1.f / sqrtf(ss / (float)p.d + p.eps);
  if (threadIdx.x == 0 && p.rstd) p.rstd[row] = rstd;
  float inv = 1.f;
  if (kEight) {
    float top = 0.f;
    for (int j = threadIdx.x; j < p.d; j += 512) top = fmaxf(top, fabsf(sum(j) * rstd * (p.w ? p.w[j] : 1.f)));
    top = fmaxf(row_reduce<Max, 512>(top, s_b), kLeastMax);
    inv = kE4m3Max / top;
    if (threadIdx.x == 0) p.scale[row] = top / kE4m3Max;
  }
  for (int j = threadIdx.x; j < p.d; j += 512) {
    const float h = sum(j);
    float y = h * rstd * (p.w ? p.w[j] : 1.f);
    if (kEight) y *= inv;
    if (p.h) put(reinterpret_cast<TR*>(p.h) + row * p.ldh + j, h);
    put(reinterpret_cast<TY*>(p.y) + row * p.ldy + j, y);
  }
}

template <typename TX, typename TR, typename TY, bool RES>
cudaError_t launch_norm(const NormParams& p, bool vec, cudaStream_t s) {
  const int64_t chunks = ceil_div((int64_t)p.d, (int64_t)8);
  const unsigned T = (unsigned)p.T;
  if (!vec || chunks > 1024 * kChunks) return launch(norm_loop_kernel<TX, TR, TY, RES>, dim3(T), dim3(512), 0, s, p);
  if (chunks <= 32 * kChunks) return launch(norm_kernel<TX, TR, TY, RES, 32>, dim3((T + 3) / 4), dim3(128), 0, s, p);
  if (chunks <= 128 * kChunks) return launch(norm_kernel<TX, TR, TY, RES, 128>, dim3(T), dim3(128), 0, s, p);
  if (chunks <= 256 * kChunks) return launch(norm_kernel<TX, TR, TY, RES, 256>, dim3(T), dim3(256), 0, s, p);
  return launch(norm_kernel<TX, TR, TY, RES, 1024>, dim3(T), dim3(1024), 0, s, p);
}
template <typename TX, typename TR, typename TY>
cudaError_t launch_norm(const NormParams& p, bool vec, cudaStream_t s) {
  return p.r ? launch_norm<TX, TR, TY, true>(p, vec, s) : launch_norm<TX, TR, TY, false>(p, vec, s);
}
template <typename TX, typename TR>
cudaError_t launch_norm(const NormParams& p, bool eight, bool vec, cudaStream_t s) {
  return eight ? launch_norm<TX, TR, __nv_fp8_storage_t>(p, vec, s) : launch_norm<TX, TR, TX>(p, vec, s);
}

// ------------------------------------------------------------------------------------------------------- gradient
struct GradParams {
  const void *dy, *h, *dh;
  void* dx;
  const float *w, *rstd;
  float* part;                 // [blocks, d] sums of a block's rows, or null
  int64_t lddy, ldh, lddh, lddx, T;
  int32_t d, w_vec;
  float eps;
};

__device__ __forceinline__ void copy16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// a chunk from its 16-byte pieces, `step` bytes apart
__device__ __forceinline__ void collect(Raw8<__nv_bfloat16>& r, const uint8_t* at, int) { r.a = *reinterpret_cast<const uint4*>(at); }
__device__ __forceinline__ void collect(Raw8<float>& r, const uint8_t* at, int step) {
  r.a = *reinterpret_cast<const float4*>(at);
  r.b = *reinterpret_cast<const float4*>(at + step);
}
// Rows in the ring: four of bf16 (24 KB each for 4096 columns; two blocks of an SM), two of wider types; one where a row has 1024 threads, two of bf16.
template <typename TY, typename TH, int TPR>
struct GradRing {
  static constexpr int CHUNK = (int)(sizeof(TY) + 2 * sizeof(TH)) / 2;      // pieces of a chunk of eight values of dy, h and the stream's gradient
  static constexpr int PIECES = 2 * CHUNK;
  static constexpr int STAGES = TPR == 1024 ? (CHUNK == 3 ? 2 : 1) : CHUNK == 3 && TPR <= 256 ? 4 : 2;
  static constexpr int THREADS = TPR < 256 ? 256 : TPR;
  static constexpr size_t SMEM = (size_t)STAGES * PIECES * THREADS * 16;
  static_assert(SMEM <= 200 * 1024, "shared memory of a block");
};
// Blocks walk over rows, a grid apart; a thread keeps the weight's gradient of its columns in registers from row to row.
constexpr int kGradChunks = 2;
template <typename TY, typename TH, int TPR>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR, TPR <= 256 && sizeof(TY) + sizeof(TH) == 4 ? 2 : 1) norm_grad_kernel(const GradParams p) {
  kernel_begin();
  constexpr int kRows = TPR < 256 ? 256 / TPR : 1, kWarps = TPR / 32;      // rows of a block at a time, warps of a row
  __shared__ float s_red[2][kRows][kWarps][2];
  __shared__ float s_dw[kRows > 1 ? TPR * kGradChunks * 8 : 1];
  const int t = threadIdx.x % TPR, g = threadIdx.x / TPR, lane = threadIdx.x & 31, warp = t / 32;
  float dw[kGradChunks][8];
#pragma unroll
  for (int c = 0; c < kGradChunks; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[c][i] = 0.f;
  // Whole chunks come through a ring of rows in shared memory, by copies that the thread itself waits for: each has its own places there.
  extern __shared__ __align__(16) uint8_t smem[];
  using R = GradRing<TY, TH, TPR>;
  uint8_t* mine = smem + threadIdx.x * 16;
  constexpr int kStep = R::THREADS * 16;                         // bytes from a piece of the thread's to its next
  const auto piece = [&](int stage, int k) { return mine + (stage * R::PIECES + k) * kStep; };
  const auto bring = [&](int stage, int64_t row) {
    if (row < p.T) {
      const TY* dy = reinterpret_cast<const TY*>(p.dy) + row * p.lddy;
      const TH* h = reinterpret_cast<const TH*>(p.h) + row * p.ldh;
      const TH* dh = reinterpret_cast<const TH*>(p.dh) + row * p.lddh;
#pragma unroll
      for (int c = 0; c < kGradChunks; ++c) {
        const int j = (c * TPR + t) * 8;
        if (j + 8 > p.d) continue;
        int k = c * R::CHUNK;
#pragma unroll
        for (int i = 0; i < (int)sizeof(TY) / 2; ++i) copy16(piece(stage, k++), dy + j + 4 * i);
#pragma unroll
        for (int i = 0; i < (int)sizeof(TH) / 2; ++i) copy16(piece(stage, k++), h + j + 4 * i);
        if (p.dh) {
#pragma unroll
          for (int i = 0; i < (int)sizeof(TH) / 2; ++i) copy16(piece(stage, k++), dh + j + 4 * i);
        }
      }
    }
    copies_end();
  };
  const int64_t stride = (int64_t)gridDim.x * kRows;
  // (weights stay in registers, and the next row's rstd is on its way: beside the ring little of L1 is left, and waits for L2 in every row
  // were what bounded this: 8192 x 4096 77 us with them)
  float w[kGradChunks][8];
#pragma unroll
  for (int c = 0; c < kGradChunks; ++c) {
    const int j = (c * TPR + t) * 8, n = p.d - j < 8 ? p.d - j : 8;
    if (n > 0) weights8(p.w, j, n, p.w_vec != 0, w[c]);
  }
  const auto rstd_of = [&](int64_t row) { return p.rstd && row < p.T ? p.rstd[row] : 0.f; };
  float next_rstd;
  {
    int64_t row = (int64_t)blockIdx.x * kRows + g;
    next_rstd = rstd_of(row);
    for (int k = 0; k < R::STAGES - 1; ++k, row += stride) bring(k, row);
  }
  int flip = 0, stage = 0;
  // (all rows of a block go round together: they meet at the sums)
  for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < p.T; row0 += stride, flip ^= 1) {
    const int64_t row = row0 + g;
    const bool live = row < p.T;
    bring(stage == 0 ? R::STAGES - 1 : stage - 1, row + (R::STAGES - 1) * stride);
    copies_wait<R::STAGES - 1>();
    Raw8<TY> a[kGradChunks];
    Raw8<TH> b[kGradChunks], e[kGradChunks];
#pragma unroll
    for (int c = 0; c < kGradChunks; ++c) {
      const int j = (c * TPR + t) * 8;
      a[c] = Raw8<TY>();
      b[c] = e[c] = Raw8<TH>();
      if (live && j + 8 <= p.d) {
        const int k = c * R::CHUNK;
        collect(a[c], piece(stage, k), kStep);
        collect(b[c], piece(stage, k + sizeof(TY) / 2), kStep);
        if (p.dh) collect(e[c], piece(stage, k + sizeof(TY) / 2 + sizeof(TH) / 2), kStep);
      } else if (live && j < p.d) {
        fetch_some(a[c], reinterpret_cast<const TY*>(p.dy) + row * p.lddy + j, p.d - j);
        fetch_some(b[c], reinterpret_cast<const TH*>(p.h) + row * p.ldh + j, p.d - j);
        if (p.dh) fetch_some(e[c], reinterpret_cast<const TH*>(p.dh) + row * p.lddh + j, p.d - j);
      }
    }
    stage = stage + 1 == R::STAGES ? 0 : stage + 1;
    const float given = next_rstd;
    next_rstd = rstd_of(row + stride);
    float s = 0.f, ss = 0.f;
#pragma unroll
    for (int c = 0; c < kGradChunks; ++c) {
      const int j = (c * TPR + t) * 8, n = p.d - j < 8 ? p.d - j : 8;
      if (n <= 0) continue;
      float u[8], x[8];
      open8(a[c], u);
      open8(b[c], x);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s = fmaf(u[i] * w[c][i], x[i], s);
        if (!p.rstd) ss = fmaf(x[i], x[i], ss);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      if (!p.rstd) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    }
    if (kWarps > 1) {
      // (two sets in turn: the one of the row before may still be read)
      if (lane == 0) {
        s_red[flip][g][warp][0] = s;
        s_red[flip][g][warp][1] = ss;
      }
      __syncthreads();
      s = ss = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        s += s_red[flip][g][w][0];
        ss += s_red[flip][g][w][1];
      }
    }
    const float rstd = p.rstd ? given : 1.f / sqrtf(ss / (float)p.d + p.eps);
    const float f = s / (float)p.d * rstd * rstd;
    TH* dx = reinterpret_cast<TH*>(p.dx) + row * p.lddx;
#pragma unroll
    for (int c = 0; c < kGradChunks; ++c) {
      const int j = (c * TPR + t) * 8, n = p.d - j < 8 ? p.d - j : 8;
      if (!live || n <= 0) continue;
      float u[8], x[8], o[8];
      open8(a[c], u);
      open8(b[c], x);
      open8(e[c], o);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        dw[c][i] = fmaf(u[i], x[i] * rstd, dw[c][i]);
        const float v = rstd * fmaf(-x[i], f, u[i] * w[c][i]);
        o[i] = p.dh ? v + o[i] : v;
      }
      if (n == 8) store8(dx + j, o);
      else store_some(dx + j, o, n);
    }
  }
  if (!p.part) return;
  // the rows that a block had side by side add up in shared memory, always in the same order
  if (kRows > 1) {
    for (int k = 1; k < kRows; ++k) {
      __syncthreads();
      if (g == k) {
#pragma unroll
        for (int c = 0; c < kGradChunks; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) s_dw[(c * 8 + i) * TPR + t] = dw[c][i];
      }
      __syncthreads();
      if (g == 0) {
#pragma unroll
        for (int c = 0; c < kGradChunks; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) dw[c][i] += s_dw[(c * 8 + i) * TPR + t];
      }
    }
    if (g != 0) return;
  }
  float* part = p.part + (int64_t)blockIdx.x * p.d;
#pragma unroll
  for (int c = 0; c < kGradChunks; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = (c * TPR + t) * 8 + i;
      if (j < p.d) part[j] = dw[c][i];
    }
}

// Any width and alignment; the weight's gradient adds up in the block's own row of `part`.
template <typename TY, typename TH>
__global__ void __launch_bounds__(512) norm_grad_loop_kernel(const GradParams p) {
  kernel_begin();
  __shared__ float s_a[32], s_b[32];
  for (int64_t row = blockIdx.x; row < p.T; row += gridDim.x) {
    const TY* dy = reinterpret_cast<const TY*>(p.dy) + row * p.lddy;
    const TH* h = reinterpret_cast<const TH*>(p.h) + row * p.ldh;
    const TH* dh = reinterpret_cast<const TH*>(p.dh) + row * p.lddh;
    TH* dx = reinterpret_cast<TH*>(p.dx) + row * p.lddx;
    float* part = p.part + (int64_t)blockIdx.x * p.d;
    float s = 0.f, ss = 0.f;
    for (int j = threadIdx.x; j < p.d; j += 512) {
      const float x = get(h + j);
      s = fmaf(get(dy + j) * (p.w ? p.w[j] : 1.f), x, s);
      ss = fmaf(x, x, ss);
    }
    __syncthreads();                  // the row before has read its sums
    s = row_reduce<Sum, 512>(s, s_a);
    ss = row_reduce<Sum, 512>(ss, s_b);
    const float rstd = p.rstd ? p.rstd[row] : 1.f / sqrtf(ss / (float)p.d + p.eps);
    const float f = s / (float)p.d * rstd * rstd;
    for (int j = threadIdx.x; j < p.d; j += 512) {
      const float u = get(dy + j), x = get(h + j);
      const float v = rstd * fmaf(-x, f, u * (p.w ? p.w[j] : 1.f));
      const float o = p.dh ? v + get(dh + j) : v;
      if (p.part) part[j] = row == blockIdx.x ? u * (x * rstd) : fmaf(u, x * rstd, part[j]);
      put(dx + j, o);
    }
  }
}

// dw_j: the blocks' sums, in 64 bits and always in the same order.  32 columns x 8 rows at a time per block.
__global__ void __launch_bounds__(256) norm_grad_join_kernel(const float* part, int32_t blocks, int32_t d, float* dw) {
  kernel_begin();
  __shared__ double s[8][33];
  const int j = blockIdx.x * 32 + (threadIdx.x & 31), g = threadIdx.x >> 5;
  double a = 0.0;
  if (j < d) {
#pragma unroll 4
    for (int b = g; b < blocks; b += 8) a += (double)part[(int64_t)b * d + j];
  }
  s[g][threadIdx.x & 31] = a;
  __syncthreads();
  if (g == 0 && j < d) {
    for (int k = 1; k < 8; ++k) a += s[k][threadIdx.x & 31];
    dw[j] = (float)a;
  }
}

// threads of a row; 0: the looping kernel
inline int grad_threads(int64_t d) {
  const int64_t chunks = ceil_div(d, (int64_t)8);
  for (int t : {32, 64, 128, 256, 512, 1024})
    if (chunks <= (int64_t)t * kGradChunks) return t;
  return 0;
}
// Blocks of the gradient: one wave, as many as are resident on 148 SMs (so that the workspace depends on the sizes alone).  loop: of the looping
// kernel, whose blocks have a row at a time: never fewer than of the other.
inline int64_t grad_blocks(int64_t T, int64_t d, bool loop) {
  const int tpr = grad_threads(d);
  const int threads = tpr == 0 ? 512 : tpr < 256 ? 256 : tpr, rows = !loop && tpr > 0 && tpr < 256 ? 256 / tpr : 1;
  const int64_t most = 148 * (threads > 256 ? 1 : 2), want = ceil_div(T, (int64_t)rows);
  return want < most ? (want > 0 ? want : 1) : most;
}

template <typename TY, typename TH, int TPR>
cudaError_t launch_grad(const GradParams& p, dim3 grid, cudaStream_t s) {
  using R = GradRing<TY, TH, TPR>;
  static PerDeviceOnce attr_once;
  const auto kernel = norm_grad_kernel<TY, TH, TPR>;
  const cudaError_t e = attr_once.run([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)R::SMEM); });
  return e == cudaSuccess ? launch(kernel, grid, dim3(R::THREADS), R::SMEM, s, p) : e;
}
template <typename TY, typename TH>
cudaError_t launch_grad(const GradParams& p, bool vec, cudaStream_t s) {
  const dim3 grid((unsigned)grad_blocks(p.T, p.d, !vec));
  switch (vec ? grad_threads(p.d) : 0) {
    case 32: return launch_grad<TY, TH, 32>(p, grid, s);
    case 64: return launch_grad<TY, TH, 64>(p, grid, s);
    case 128: return launch_grad<TY, TH, 128>(p, grid, s);
    case 256: return launch_grad<TY, TH, 256>(p, grid, s);
    case 512: return launch_grad<TY, TH, 512>(p, grid, s);
    case 1024: return launch_grad<TY, TH, 1024>(p, grid, s);
    default: return launch(norm_grad_loop_kernel<TY, TH>, grid, dim3(512), 0, s, p);
  }
}

bool act_dtype(int32_t dt) { return dt == SP_BF16 || dt == SP_F32; }
// eight values of every row start on `bytes`
bool aligned8(const void* ptr, int32_t dtype, int64_t ld, int64_t rows) {
  const int64_t es = (int64_t)dtype_size(dtype), want = es == 1 ? 8 : 16;
  return reinterpret_cast<uintptr_t>(ptr) % want == 0 && (rows < 2 || ld * es % want == 0);
}
sp_status check_rows(const sp_mat* m, int64_t T, int64_t d) {
  if (m->rows != T || m->cols != d || (T > 1 && m->ld < d)) return SP_ERR_SHAPE;
  return SP_OK;
}

}  // namespace
}  // namespace sp

extern "C" {

sp_status sp_rms_norm(const sp_mat* X, const sp_mat* R, const float* weight, double eps, const sp_mat* H, const sp_mat* Y,
                      float* scale, float* rstd, void* stream) {
  using namespace sp;
  if (!X || !Y) return SP_ERR_INVALID_ARG;
  if (!act_dtype(X->dtype) || (R && !act_dtype(R->dtype)) || (H && !act_dtype(H->dtype))) return SP_ERR_DTYPE;
  if (Y->dtype != X->dtype && Y->dtype != SP_E4M3) return SP_ERR_DTYPE;
  if (R && H && R->dtype != H->dtype) return SP_ERR_DTYPE;
  const bool eight = Y->dtype == SP_E4M3;
  if (eight != (scale != nullptr)) return SP_ERR_INVALID_ARG;
  if (!(eps >= 0.0) || !(eps <= 1e30)) return SP_ERR_INVALID_ARG;
  const int64_t T = X->rows, d = X->cols;
  if (T < 0 || d < 1 || T > 0x7fffffff || d > (1 << 30) || (T > 1 && X->ld < d)) return SP_ERR_SHAPE;
  for (const sp_mat* m : {R, H, Y})
    if (m && check_rows(m, T, d) != SP_OK) return SP_ERR_SHAPE;
  if (T == 0) return SP_OK;
  if (!X->ptr || !Y->ptr || (R && !R->ptr) || (H && !H->ptr)) return SP_ERR_INVALID_ARG;
  // (an output in an input's place needs its pitch and type; two outputs in one place are a mistake)
  for (const sp_mat* out : {H, Y})
    for (const sp_mat* in : {X, R})
      if (out && in && out->ptr == in->ptr && (out->dtype != in->dtype || (T > 1 && out->ld != in->ld))) return SP_ERR_INVALID_ARG;
  if (H && H->ptr == Y->ptr) return SP_ERR_INVALID_ARG;
  NormParams p = {};
  p.x = X->ptr; p.r = R ? R->ptr : nullptr; p.h = H ? H->ptr : nullptr; p.y = Y->ptr;
  p.ldx = X->ld; p.ldr = R ? R->ld : 0; p.ldh = H ? H->ld : 0; p.ldy = Y->ld;
  p.w = weight; p.scale = scale; p.rstd = rstd;
  p.T = T; p.d = (int32_t)d; p.eps = (float)eps;
  p.w_vec = (reinterpret_cast<uintptr_t>(weight) & 15u) == 0;
  bool vec = true;
  for (const sp_mat* m : {X, R, H, Y}) vec = vec && (!m || aligned8(m->ptr, m->dtype, m->ld, T));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  count_launch();
  ProfScope prof(PK_ELEMENTWISE, 0.0, 0.0, s);
  const int32_t stream_dtype = R ? R->dtype : H ? H->dtype : X->dtype;
  cudaError_t e;
  if (X->dtype == SP_F32)
    e = stream_dtype == SP_F32 ? launch_norm<float, float>(p, eight, vec, s) : launch_norm<float, __nv_bfloat16>(p, eight, vec, s);
  else
    e = stream_dtype == SP_F32 ? launch_norm<__nv_bfloat16, float>(p, eight, vec, s)
                               : launch_norm<__nv_bfloat16, __nv_bfloat16>(p, eight, vec, s);
  return e == cudaSuccess ? SP_OK : SP_ERR_CUDA;
}

size_t sp_rms_norm_grad_bytes(int64_t T, int64_t d) {
  if (T < 1 || d < 1 || T > 0x7fffffff || d > (1 << 30)) return 0;
  return (size_t)sp::grad_blocks(T, d, true) * (size_t)d * sizeof(float);
}

sp_status sp_rms_norm_grad(const sp_mat* dY, const sp_mat* H, const float* weight, const float* rstd, double eps, const sp_mat* dH,
                           const sp_mat* dX, float* dweight, void* ws, size_t ws_bytes, void* stream) {
  using namespace sp;
  if (!dY || !H || !dX) return SP_ERR_INVALID_ARG;
  if (!act_dtype(dY->dtype) || !act_dtype(H->dtype) || dX->dtype != H->dtype || (dH && dH->dtype != H->dtype)) return SP_ERR_DTYPE;
  if (!(eps >= 0.0) || !(eps <= 1e30)) return SP_ERR_INVALID_ARG;
  const int64_t T = dY->rows, d = dY->cols;
  if (T < 0 || d < 1 || T > 0x7fffffff || d > (1 << 30) || (T > 1 && dY->ld < d)) return SP_ERR_SHAPE;
  for (const sp_mat* m : {H, dH, dX})
    if (m && check_rows(m, T, d) != SP_OK) return SP_ERR_SHAPE;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (T == 0) return dweight && cudaMemsetAsync(dweight, 0, (size_t)d * 4, s) != cudaSuccess ? SP_ERR_CUDA : SP_OK;
  if (!dY->ptr || !H->ptr || !dX->ptr || (dH && !dH->ptr)) return SP_ERR_INVALID_ARG;
  for (const sp_mat* in : {dY, H, dH})
    if (in && dX->ptr == in->ptr && (dX->dtype != in->dtype || (T > 1 && dX->ld != in->ld))) return SP_ERR_INVALID_ARG;
  if (dweight) {
    if (!ws || ws_bytes < sp_rms_norm_grad_bytes(T, d)) return SP_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(ws) & 255u) return SP_ERR_ALIGNMENT;
  }
  GradParams p = {};
  p.dy = dY->ptr; p.h = H->ptr; p.dh = dH ? dH->ptr : nullptr; p.dx = dX->ptr;
  p.lddy = dY->ld; p.ldh = H->ld; p.lddh = dH ? dH->ld : 0; p.lddx = dX->ld;
  p.w = weight; p.rstd = rstd; p.part = dweight ? reinterpret_cast<float*>(ws) : nullptr;
  p.T = T; p.d = (int32_t)d; p.eps = (float)eps;
  p.w_vec = (reinterpret_cast<uintptr_t>(weight) & 15u) == 0;
  bool vec = true;
  for (const sp_mat* m : {dY, H, dH, dX}) vec = vec && (!m || aligned8(m->ptr, m->dtype, m->ld, T));
  ProfScope prof(PK_ELEMENTWISE, 0.0, 0.0, s);
  count_launch();
  cudaError_t e;
  if (dY->dtype == SP_F32)
    e = H->dtype == SP_F32 ? launch_grad<float, float>(p, vec, s) : launch_grad<float, __nv_bfloat16>(p, vec, s);
  else
    e = H->dtype == SP_F32 ? launch_grad<__nv_bfloat16, float>(p, vec, s) : launch_grad<__nv_bfloat16, __nv_bfloat16>(p, vec, s);
  if (e == cudaSuccess && dweight) {
    count_launch();
    const OverlapScope overlap(true);      // its blocks start while the rows' end
    e = launch(norm_grad_join_kernel, dim3((unsigned)ceil_div(d, (int64_t)32)), dim3(256), 0, s, (const float*)p.part,
               (int32_t)grad_blocks(T, d, !vec), p.d, dweight);
  }
  return e == cudaSuccess ? SP_OK : SP_ERR_CUDA;
}

}  // extern "C"
