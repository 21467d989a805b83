// sp_linear for few rows, up to some hundred: Y = act(X W^T + bias) (+|*) other, bound by reading W once.
//
// A 128-row tile of the tensor-core product would be nearly empty, and a call has few of them: its time is that of a few SMs reading W
// (16 x 768 -> 1536 took 32 us from cold caches).  Here a block takes 16 outputs and all of K, its eight warps every eighth piece of 32
// values: W goes from memory into the operand registers of the matrix instruction (m16n8k16, outputs x rows of X) without shared
// memory, 16 bytes of an output's row per lane.  Which values of K an instruction contracts is free as long as X has them in the same
// order, so X is read the same way (from L2 but for the first time).  The warps' sums meet in shared memory, always in the same order.
// Pieces that lie whole within K are loaded without a condition: behind one the loads of a warp followed one another (fp32, one row,
// 4096 -> 16384: 172 us, 61 without; bf16, 16 rows: 39 and 35).
#include <type_traits>

#include "sp_common.cuh"

namespace sp {
namespace {

constexpr int kWarps = 8, kOut = 16, kPiece = 32;

__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 8 values of a row from k on, zero from K on.  A piece that K cuts is read value by value: what stands behind the last value of a matrix may not be
// the caller's.
__device__ __forceinline__ uint4 row_piece(const __nv_bfloat16* row, int64_t k, int64_t K, bool stream) {
  if (k + 8 <= K) {
    const uint4* at = reinterpret_cast<const uint4*>(row + k);
    return stream ? __ldcs(at) : *at;
  }
  uint32_t w[4] = {0u, 0u, 0u, 0u};
  const uint16_t* bits = reinterpret_cast<const uint16_t*>(row);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (k + i < K) w[i / 2] |= (uint32_t)bits[k + i] << (16 * (i & 1));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

struct FewParams {
  const __nv_bfloat16 *x, *w;
  int64_t ldx, ldw, ldo, ldy, T, K, N;
  LinearEpi epi;
  const void* other;
  void* y;
  int32_t y_f32;
};

// NT: groups of eight rows of X
template <int NT>
__global__ void __launch_bounds__(kWarps * 32, NT > 1 ? 2 : 3) linear_few_kernel(const FewParams p) {
  kernel_begin();
  constexpr int kUnroll = NT > 2 ? 2 : 4;
  __shared__ float s_acc[kWarps][NT * 8][kOut + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g4 = lane >> 2, t4 = lane & 3;
  const int64_t o0 = (int64_t)blockIdx.x * kOut, t0 = (int64_t)blockIdx.y * (NT * 8);
  // (rows behind the last one: any values, not stored)
  const __nv_bfloat16* w0 = p.w + min(o0 + g4, p.N - 1) * p.ldw;
  const __nv_bfloat16* w1 = p.w + min(o0 + g4 + 8, p.N - 1) * p.ldw;
  const __nv_bfloat16* xr[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) xr[n] = p.x + min(t0 + 8 * n + g4, p.T - 1) * p.ldx;
  float acc[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[n][i] = 0.f;
  constexpr int64_t kAll = (int64_t)kWarps * kPiece;
  const auto pieces = [&](int64_t k0, auto count, auto&& piece) {      // `count` pieces of this warp from k0 on
    constexpr int C = decltype(count)::value;
    uint4 a[C][2], b[C][NT];
#pragma unroll
    for (int u = 0; u < C; ++u) {
      const int64_t k = k0 + u * kAll + 8 * t4;
      a[u][0] = piece(w0, k, true);
      a[u][1] = piece(w1, k, true);
#pragma unroll
      for (int n = 0; n < NT; ++n) b[u][n] = piece(xr[n], k, false);
    }
#pragma unroll
    for (int u = 0; u < C; ++u)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        mma_16x8x16(acc[n], a[u][0].x, a[u][1].x, a[u][0].y, a[u][1].y, b[u][n].x, b[u][n].y);
        mma_16x8x16(acc[n], a[u][0].z, a[u][1].z, a[u][0].w, a[u][1].w, b[u][n].z, b[u][n].w);
      }
  };
  int64_t k0 = (int64_t)warp * kPiece;
  for (; k0 + (kUnroll - 1) * kAll + kPiece <= p.K; k0 += kUnroll * kAll)      // whole pieces: no condition between the loads
    pieces(k0, std::integral_constant<int, kUnroll>(), [](const __nv_bfloat16* row, int64_t k, bool stream) {
      const uint4* at = reinterpret_cast<const uint4*>(row + k);
      return stream ? __ldcs(at) : *at;
    });
  for (; k0 < p.K; k0 += kAll)
    pieces(k0, std::integral_constant<int, 1>(), [&](const __nv_bfloat16* row, int64_t k, bool stream) { return row_piece(row, k, p.K, stream); });
  // a lane holds outputs g4 (| + 8) of rows 8 n + 2 t4 and + 1
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) s_acc[warp][8 * n + 2 * t4 + (i & 1)][g4 + 8 * (i >> 1)] = acc[n][i];
  __syncthreads();
  for (int e = threadIdx.x; e < NT * 8 * kOut; e += kWarps * 32) {
    const int64_t row = t0 + e / kOut, j = o0 + e % kOut;
    if (row >= p.T || j >= p.N) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += s_acc[w][e / kOut][e % kOut];
    v = linear_act(p.epi.bias ? v + p.epi.bias[j] : v, p.epi.act);
    if (p.y_f32) {
      if (p.other) v = linear_combine(v, reinterpret_cast<const float*>(p.other)[row * p.ldo + j], p.epi.combine);
      reinterpret_cast<float*>(p.y)[row * p.ldy + j] = v;
    } else {
      if (p.other) v = linear_combine(v, __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p.other)[row * p.ldo + j]), p.epi.combine);
      reinterpret_cast<__nv_bfloat16*>(p.y)[row * p.ldy + j] = __float2bfloat16_rn(v);
    }
  }
}

// The same in fp32 with sums in fp64: m16n8k8 of the fp64 matrix instruction, four values of a row per lane and load.  Up to eight rows the
// reading of W bounds it (4.4 TB/s), beyond them the instruction (256 rows, 4096 -> 16384: 32 TFLOP/s).  Rows of X beyond 8 NT are other blocks'.
struct FewF32Params {
  const float *x, *w;
  int64_t ldx, ldw, ldo, ldy, T, K, N;
  LinearEpi epi;
  const float* other;
  float* y;
};
__device__ __forceinline__ void dmma_16x8x8(double (&d)[4], double a0, double a1, double a2, double a3, double b0, double b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k8.row.col.f64.f64.f64.f64 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+d"(d[0]), "+d"(d[1]), "+d"(d[2]), "+d"(d[3])
      : "d"(a0), "d"(a1), "d"(a2), "d"(a3), "d"(b0), "d"(b1));
}
// the same for 4 values of fp32; VEC: rows start on 16 bytes
template <bool VEC>
__device__ __forceinline__ float4 row_piece(const float* row, int64_t k, int64_t K, bool stream) {
  if (VEC && k + 4 <= K) {
    const float4* at = reinterpret_cast<const float4*>(row + k);
    return stream ? __ldcs(at) : *at;
  }
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (k < K) v.x = row[k];
  if (k + 1 < K) v.y = row[k + 1];
  if (k + 2 < K) v.z = row[k + 2];
  if (k + 3 < K) v.w = row[k + 3];
  return v;
}

template <int NT, bool VEC>
__global__ void __launch_bounds__(kWarps * 32, 2) linear_few_f32_kernel(const FewF32Params p) {
  kernel_begin();
  constexpr int kUnroll = NT > 2 ? 2 : 4, kStep = 16;
  __shared__ double s_acc[kWarps][NT * 8][kOut + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g4 = lane >> 2, t4 = lane & 3;
  const int64_t o0 = (int64_t)blockIdx.x * kOut, t0 = (int64_t)blockIdx.y * (NT * 8);
  const float* w0 = p.w + min(o0 + g4, p.N - 1) * p.ldw;
  const float* w1 = p.w + min(o0 + g4 + 8, p.N - 1) * p.ldw;
  const float* xr[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) xr[n] = p.x + min(t0 + 8 * n + g4, p.T - 1) * p.ldx;
  double acc[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[n][i] = 0.0;
  constexpr int64_t kAll = (int64_t)kWarps * kStep;
  const auto pieces = [&](int64_t k0, auto count, auto&& piece) {      // `count` pieces of this warp from k0 on
    constexpr int C = decltype(count)::value;
    float4 a[C][2], b[C][NT];
#pragma unroll
    for (int u = 0; u < C; ++u) {
      const int64_t k = k0 + u * kAll + 4 * t4;
      a[u][0] = piece(w0, k, true);
      a[u][1] = piece(w1, k, true);
#pragma unroll
      for (int n = 0; n < NT; ++n) b[u][n] = piece(xr[n], k, false);
    }
#pragma unroll
    for (int u = 0; u < C; ++u)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        dmma_16x8x8(acc[n], a[u][0].x, a[u][1].x, a[u][0].y, a[u][1].y, b[u][n].x, b[u][n].y);
        dmma_16x8x8(acc[n], a[u][0].z, a[u][1].z, a[u][0].w, a[u][1].w, b[u][n].z, b[u][n].w);
      }
  };
  int64_t k0 = (int64_t)warp * kStep;
  if (VEC)                             // whole pieces: no condition between the loads
    for (; k0 + (kUnroll - 1) * kAll + kStep <= p.K; k0 += kUnroll * kAll)
      pieces(k0, std::integral_constant<int, kUnroll>(), [](const float* row, int64_t k, bool stream) {
        const float4* at = reinterpret_cast<const float4*>(row + k);
        return stream ? __ldcs(at) : *at;
      });
  for (; k0 < p.K; k0 += kAll)
    pieces(k0, std::integral_constant<int, 1>(), [&](const float* row, int64_t k, bool stream) { return row_piece<VEC>(row, k, p.K, stream); });
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) s_acc[warp][8 * n + 2 * t4 + (i & 1)][g4 + 8 * (i >> 1)] = acc[n][i];
  __syncthreads();
  for (int e = threadIdx.x; e < NT * 8 * kOut; e += kWarps * 32) {
    const int64_t row = t0 + e / kOut, j = o0 + e % kOut;
    if (row >= p.T || j >= p.N) continue;
    double v = 0.0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += s_acc[w][e / kOut][e % kOut];
    if (p.epi.bias) v += (double)p.epi.bias[j];
    v = linear_act(v, p.epi.act);
    if (p.other) v = linear_combine(v, (double)p.other[row * p.ldo + j], p.epi.combine);
    p.y[row * p.ldy + j] = (float)v;
  }
}
template <int NT>
cudaError_t launch_few_f32(const FewF32Params& p, bool vec, cudaStream_t stream) {
  const dim3 grid((unsigned)ceil_div(p.N, (int64_t)kOut), (unsigned)ceil_div(p.T, (int64_t)(8 * NT)));
  return vec ? launch(linear_few_f32_kernel<NT, true>, grid, dim3(kWarps * 32), 0, stream, p)
             : launch(linear_few_f32_kernel<NT, false>, grid, dim3(kWarps * 32), 0, stream, p);
}

}  // namespace

cudaError_t linear_few_f32(int64_t M, int64_t N, int64_t K, Operand A, Operand W, const LinearEpi& epi, Operand other, OutOperand C,
                           cudaStream_t stream) {
  FewF32Params p;
  p.x = reinterpret_cast<const float*>(A.ptr);
  p.w = reinterpret_cast<const float*>(W.ptr);
  p.ldx = A.s0; p.ldw = W.s0; p.ldo = other.s0; p.ldy = C.ld;
  p.T = M; p.K = K; p.N = N;
  p.epi = epi;
  p.other = reinterpret_cast<const float*>(other.ptr);
  p.y = reinterpret_cast<float*>(C.ptr);
  count_launch();
  ProfScope prof(PK_GEMM_SIMT, 2.0 * (double)M * (double)N * (double)K, 0.0, stream);
  const auto whole = [](const void* ptr, int64_t ld, int64_t rows) {      // rows start on 16 bytes
    return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0 && (rows == 1 || ld % 4 == 0);
  };
  const bool vec = whole(p.x, p.ldx, M) && whole(p.w, p.ldw, N);
  return M <= 8 ? launch_few_f32<1>(p, vec, stream) : M <= 16 ? launch_few_f32<2>(p, vec, stream) : launch_few_f32<4>(p, vec, stream);
}

cudaError_t linear_few(int64_t M, int64_t N, int64_t K, TcOperand A, TcOperand W, const LinearEpi& epi, Operand other, OutOperand C,
                       cudaStream_t stream) {
  FewParams p;
  p.x = reinterpret_cast<const __nv_bfloat16*>(A.ptr);
  p.w = reinterpret_cast<const __nv_bfloat16*>(W.ptr);
  p.ldx = A.ld; p.ldw = W.ld; p.ldo = other.s0; p.ldy = C.ld;
  p.T = M; p.K = K; p.N = N;
  p.epi = epi;
  p.other = other.ptr;
  p.y = C.ptr;
  p.y_f32 = C.dtype == SP_F32 ? 1 : 0;
  count_launch();
  ProfScope prof(PK_GEMM_SIMT, 2.0 * (double)M * (double)N * (double)K, 0.0, stream);
  const dim3 grid((unsigned)ceil_div(N, (int64_t)kOut), (unsigned)ceil_div(M, (int64_t)32));
  return M <= 8 ? launch(linear_few_kernel<1>, grid, dim3(kWarps * 32), 0, stream, p)
       : M <= 16 ? launch(linear_few_kernel<2>, grid, dim3(kWarps * 32), 0, stream, p)
                : launch(linear_few_kernel<4>, grid, dim3(kWarps * 32), 0, stream, p);
}

}  // namespace sp
