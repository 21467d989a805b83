// sp_linear for up to 32 rows in bf16: Y = act(X W^T + bias) (+|*) other, bound by reading W once.
//
// A 128-row tile of the tensor-core product would be nearly empty, and a call has few of them: its time is that of a few SMs reading W
// (16 x 768 -> 1536 took 32 us from cold caches).  Here a block takes 16 outputs and all of K, its eight warps every eighth piece of 32
// values: W goes from memory into the operand registers of the matrix instruction (m16n8k16, outputs x rows of X) without shared
// memory, 16 bytes of an output's row per lane.  Which values of K an instruction contracts is free as long as X has them in the same
// order, so X is read the same way (from L2 but for the first time).  The warps' sums meet in shared memory, always in the same order.
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
// 8 values of a row from k on, zero from K on (what stands there, to align the rows, is no part of the product)
__device__ __forceinline__ uint4 row_piece(const __nv_bfloat16* row, int64_t k, int64_t K, bool stream) {
  if (k >= K) return make_uint4(0u, 0u, 0u, 0u);
  const uint4* at = reinterpret_cast<const uint4*>(row + k);
  uint4 v = stream ? __ldcs(at) : *at;
  if (k + 8 > K) {
    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] &= (k + 2 * i < K ? 0xffffu : 0u) | (k + 2 * i + 1 < K ? 0xffff0000u : 0u);
  }
  return v;
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
  const int64_t o0 = (int64_t)blockIdx.x * kOut;
  // (rows behind the last one: any values, not stored)
  const __nv_bfloat16* w0 = p.w + min(o0 + g4, p.N - 1) * p.ldw;
  const __nv_bfloat16* w1 = p.w + min(o0 + g4 + 8, p.N - 1) * p.ldw;
  const __nv_bfloat16* xr[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) xr[n] = p.x + min((int64_t)(8 * n + g4), p.T - 1) * p.ldx;
  float acc[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[n][i] = 0.f;
  for (int64_t k0 = (int64_t)warp * kPiece; k0 < p.K; k0 += (int64_t)kWarps * kPiece * kUnroll) {
    uint4 a[kUnroll][2], b[kUnroll][NT];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t k = k0 + (int64_t)u * kWarps * kPiece + 8 * t4;
      a[u][0] = row_piece(w0, k, p.K, true);
      a[u][1] = row_piece(w1, k, p.K, true);
#pragma unroll
      for (int n = 0; n < NT; ++n) b[u][n] = row_piece(xr[n], k, p.K, false);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        mma_16x8x16(acc[n], a[u][0].x, a[u][1].x, a[u][0].y, a[u][1].y, b[u][n].x, b[u][n].y);
        mma_16x8x16(acc[n], a[u][0].z, a[u][1].z, a[u][0].w, a[u][1].w, b[u][n].z, b[u][n].w);
      }
  }
  // a lane holds outputs g4 (| + 8) of rows 8 n + 2 t4 and + 1
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) s_acc[warp][8 * n + 2 * t4 + (i & 1)][g4 + 8 * (i >> 1)] = acc[n][i];
  __syncthreads();
  for (int e = threadIdx.x; e < NT * 8 * kOut; e += kWarps * 32) {
    const int row = e / kOut, out = e % kOut;
    const int64_t j = o0 + out;
    if (row >= p.T || j >= p.N) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += s_acc[w][row][out];
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
  const dim3 grid((unsigned)ceil_div(N, (int64_t)kOut));
  return M <= 8 ? launch(linear_few_kernel<1>, grid, dim3(kWarps * 32), 0, stream, p)
       : M <= 16 ? launch(linear_few_kernel<2>, grid, dim3(kWarps * 32), 0, stream, p)
                : launch(linear_few_kernel<4>, grid, dim3(kWarps * 32), 0, stream, p);
}

}  // namespace sp
