// sp_linear_e4m3: Y = act(x_scale_t w_scale_o sum_k X8 W8 + bias) (+|*) other.
//
// Many rows take the tensor-core product of sp_gemm_tc.cu in its 8-bit form; few rows stream W past them here, bound by reading W once.
// A block takes 16 outputs and all of K, its eight warps every eighth piece of 64 values: W goes from memory into the operand registers of the
// matrix instruction (m16n8k32, outputs x rows of X) without shared memory, 16 bytes of an output's row per lane.  Which values of K an
// instruction contracts is free as long as X has them in the same order.  The warps' sums meet in shared memory, always in the same order.
#include <type_traits>

#include "sp_common.cuh"

namespace sp {
namespace {

constexpr int kWarps = 8, kOut = 16, kPiece = 64;

__device__ __forceinline__ void mma_16x8x32(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 16 values of a row from k on, zero from K on: nothing behind the last value of a row is read
__device__ __forceinline__ uint4 some_of(const uint8_t* row, int64_t k, int64_t K) {
  if (k + 16 <= K) return *reinterpret_cast<const uint4*>(row + k);
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (k + i < K) w[i / 4] |= (uint32_t)row[k + i] << (8 * (i & 3));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

struct FewParams {
  const uint8_t *x, *w;
  int64_t ldx, ldw, ldo, ldy, T, K, N;
  LinearEpi epi;
  const void* other;
  void* y;
  int32_t y_f32;
};

// NT: groups of eight rows of X.  CTAS: blocks that an SM holds.  Two groups have four pieces of a warp in flight in two blocks, or two pieces in three:
// faster where there are more blocks than fit at once by two.  Two / three blocks, us, 16 rows: 4096 -> 6144 9.0 / 7.8, 4096 -> 32000 30.3 / 29.5,
// 8192 -> 2048 8.1 / 10.2, 4096 -> 1024 4.8 / 5.9.
template <int NT, int CTAS>
__global__ void __launch_bounds__(kWarps * 32, CTAS) linear_e4m3_few_kernel(const FewParams p) {
  kernel_begin();
  constexpr int kUnroll = NT > 2 || (NT == 2 && CTAS > 2) ? 2 : 4;
  __shared__ float s_acc[kWarps][NT * 8][kOut + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g4 = lane >> 2, t4 = lane & 3;
  const int64_t o0 = (int64_t)blockIdx.x * kOut, t0 = (int64_t)blockIdx.y * (NT * 8);
  // (rows behind the last one: any values, not stored)
  const uint8_t* w0 = p.w + min(o0 + g4, p.N - 1) * p.ldw;
  const uint8_t* w1 = p.w + min(o0 + g4 + 8, p.N - 1) * p.ldw;
  const uint8_t* xr[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) xr[n] = p.x + min(t0 + 8 * n + g4, p.T - 1) * p.ldx;
  float acc[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[n][i] = 0.f;
  constexpr int64_t kAll = (int64_t)kWarps * kPiece;
  const auto pieces = [&](int64_t k0, auto count, auto whole) {      // `count` pieces of this warp from k0 on
    constexpr int C = decltype(count)::value;
    constexpr bool WHOLE = decltype(whole)::value;                   // they lie within K: no condition between the loads
    uint4 a[C][2], b[C][NT];
#pragma unroll
    for (int u = 0; u < C; ++u) {
      const int64_t k = k0 + u * kAll + 16 * t4;
      if (WHOLE) {
        a[u][0] = __ldcs(reinterpret_cast<const uint4*>(w0 + k));
        a[u][1] = __ldcs(reinterpret_cast<const uint4*>(w1 + k));
#pragma unroll
        for (int n = 0; n < NT; ++n) b[u][n] = *reinterpret_cast<const uint4*>(xr[n] + k);
      } else {
        a[u][0] = some_of(w0, k, p.K);
        a[u][1] = some_of(w1, k, p.K);
#pragma unroll
        for (int n = 0; n < NT; ++n) b[u][n] = some_of(xr[n], k, p.K);
      }
    }
#pragma unroll
    for (int u = 0; u < C; ++u)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        mma_16x8x32(acc[n], a[u][0].x, a[u][1].x, a[u][0].y, a[u][1].y, b[u][n].x, b[u][n].y);
        mma_16x8x32(acc[n], a[u][0].z, a[u][1].z, a[u][0].w, a[u][1].w, b[u][n].z, b[u][n].w);
      }
  };
  int64_t k0 = (int64_t)warp * kPiece;
  for (; k0 + (kUnroll - 1) * kAll + kPiece <= p.K; k0 += kUnroll * kAll) pieces(k0, std::integral_constant<int, kUnroll>(), std::true_type());
  for (; k0 < p.K; k0 += kAll) pieces(k0, std::integral_constant<int, 1>(), std::false_type());
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
    v = v * p.epi.x_scale[row] * p.epi.w_scale[j];
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

}  // namespace
}  // namespace sp

extern "C" sp_status sp_linear_e4m3(const sp_mat* X, const float* x_scale, const sp_mat* W, const float* w_scale, const float* bias,
                                    int32_t act, const sp_mat* other, int32_t combine, const sp_mat* Y, int32_t* status_dev,
                                    void* stream) {
  using namespace sp;
  if (!X || !W || !Y) return SP_ERR_INVALID_ARG;
  if (act < SP_LINEAR_NONE || act > SP_LINEAR_GELU) return SP_ERR_INVALID_ARG;
  if (combine != SP_COMBINE_ADD && combine != SP_COMBINE_MUL) return SP_ERR_INVALID_ARG;
  if (X->dtype != SP_E4M3 || W->dtype != SP_E4M3) return SP_ERR_DTYPE;
  if (Y->dtype != SP_BF16 && Y->dtype != SP_F32) return SP_ERR_DTYPE;
  if (other && other->dtype != Y->dtype) return SP_ERR_DTYPE;
  const int64_t T = X->rows, K = X->cols, N = W->rows;
  if (T < 0 || N < 0 || K < 1 || W->cols != K || Y->rows != T || Y->cols != N) return SP_ERR_SHAPE;
  if (other && (other->rows != T || other->cols != N)) return SP_ERR_SHAPE;
  if (T > (1 << 30) || N > (1 << 30) || K > (1 << 30) || ceil_div(T, (int64_t)128) * ceil_div(N, (int64_t)128) > 0x7fffffff)
    return SP_ERR_SHAPE;
  if ((T > 1 && (X->ld < K || Y->ld < N || (other && other->ld < N))) || (N > 1 && W->ld < K)) return SP_ERR_SHAPE;
  if (T == 0 || N == 0) return SP_OK;
  if (!X->ptr || !W->ptr || !Y->ptr || !x_scale || !w_scale || (other && !other->ptr)) return SP_ERR_INVALID_ARG;
  if (other && other->ptr == Y->ptr && T > 1 && other->ld != Y->ld) return SP_ERR_INVALID_ARG;
  // (a single row has no pitch: whatever stands there is not used)
  const int64_t whole = (K + 15) / 16 * 16, ldx = T > 1 ? X->ld : whole, ldw = N > 1 ? W->ld : whole;
  if (ldx % 16 != 0 || ldw % 16 != 0 || (reinterpret_cast<uintptr_t>(X->ptr) & 15u) || (reinterpret_cast<uintptr_t>(W->ptr) & 15u))
    return SP_ERR_ALIGNMENT;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  LinearEpi epi;
  epi.bias = bias;
  epi.x_scale = x_scale;
  epi.w_scale = w_scale;
  epi.act = act;
  epi.combine = combine;
  const Operand o = other ? Operand{other->ptr, other->dtype, other->ld, 1} : Operand{nullptr, Y->dtype, 0, 1};
  if (!linear_few_rows_e4m3(T, N))
    return gemm_tc(T, N, K, 1.f, TcOperand{X->ptr, ldx, true}, TcOperand{W->ptr, ldw, true}, other ? 1.f : 0.f, o,
                   OutOperand{Y->ptr, Y->dtype, Y->ld}, false, status_dev, s, nullptr, -1.0, 0, nullptr, &epi);
  FewParams p;
  p.x = reinterpret_cast<const uint8_t*>(X->ptr);
  p.w = reinterpret_cast<const uint8_t*>(W->ptr);
  p.ldx = ldx; p.ldw = ldw; p.ldo = o.s0; p.ldy = Y->ld;
  p.T = T; p.K = K; p.N = N;
  p.epi = epi;
  p.other = o.ptr;
  p.y = Y->ptr;
  p.y_f32 = Y->dtype == SP_F32 ? 1 : 0;
  count_launch();
  ProfScope prof(PK_GEMM_SIMT, 2.0 * (double)T * (double)N * (double)K, 0.0, s);
  const dim3 grid((unsigned)ceil_div(N, (int64_t)kOut), (unsigned)ceil_div(T, (int64_t)32));
  const auto kernel = T <= 8 ? linear_e4m3_few_kernel<1, 3>
                      : T > 16 ? linear_e4m3_few_kernel<4, 2>
                      : (int64_t)grid.x > 2 * (int64_t)sm_count() ? linear_e4m3_few_kernel<2, 3> : linear_e4m3_few_kernel<2, 2>;
  const cudaError_t e = launch(kernel, grid, dim3(kWarps * 32), 0, s, p);
  return e == cudaSuccess ? SP_OK : SP_ERR_CUDA;
}
