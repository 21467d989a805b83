// Appending to a paged cache with the rotation of positions on the way, and reading it back.
//
// Token i of the n that a call brings to sequence s stands at p = lens[s] - n + i and goes to slot p % page_len of page table[s][p / page_len].
// Rotation: channels (a, b) of a pair with frequency f become (a cos - b sin, b cos + a sin), angle p f.  The angle is taken in 64 bits and
// in whole turns away first: at p = 10^5 an angle in 32 bits would be off by 10^-2.
// 4 bits: of every 64 channels of a head, zero = bf16(least), scale = bf16((largest - zero) / 15), n = (x - zero) / scale rounded to the
// nearest of 0 .. 15.  A value next to the border of two steps, a rotated one too, falls on the side on which the formula in 64 bits has it.
//
// Both kernels are bound by memory (append: 16384 x (32 + 2 x 8) heads of 128: 200 MB in, 150 MB out); a thread has eight channels at a time,
// 16 bytes of bf16, four bytes of a page in 4 bits; the eight lanes of a group find its bounds by shuffles.
#include <cuda_fp16.h>
#include <math.h>

#include <type_traits>

#include "sp_attention.cuh"
#include "sp_cache.cuh"

namespace sp {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kMaxTurned = 128;

// Quotients by numbers that the host knows: n / d = (n m) >> s with m = ceil(2^s / d), exact for n below 2^20 and d below 2^20 (s = 40).
struct Divisor {
  uint64_t m;
  uint32_t d;
};
inline Divisor divisor(int64_t d) { return Divisor{((uint64_t(1) << 40) + (uint64_t)d - 1) / (uint64_t)d, (uint32_t)d}; }
__device__ __forceinline__ uint32_t quotient(uint32_t n, const Divisor& d) { return (uint32_t)((n * d.m) >> 40); }

struct AppendParams {
  CacheView c;
  Divisor q_row, q_head, k_row, k_head;    // chunks of a row (queries: pairs of chunks), of a head
  const void *q, *k, *v;
  void *q_out, *k_out;
  int64_t ldq, ldk, ldv, ldqo, ldko;
  const int32_t* cu;
  const int32_t* positions;
  const float* inv_freq;
  int32_t rows, n_heads, turned, neighbours;
  int32_t per_block;                       // rows of a block
  int32_t q_vec, k_vec, v_vec;             // rows start on 16 bytes
  int32_t* status;
};

// Eight values from p on, in fp32.  VEC: rows start on 16 bytes in every matrix of the call; else `vec` tells of this one.
template <bool VEC>
__device__ __forceinline__ void load8(const __nv_bfloat16* p, bool vec, float (&x)[8]) {
  if (VEC || vec) {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __bfloat162float(p[i]);
  }
}
template <bool VEC>
__device__ __forceinline__ void load8(const float* p, bool vec, float (&x)[8]) {
  if (VEC || vec) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[i];
  }
}
template <bool VEC>
__device__ __forceinline__ void put8(__nv_bfloat16* p, bool vec, const float (&x)[8]) {
  if (VEC || vec) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 e = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&e);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __float2bfloat16_rn(x[i]);
  }
}
template <bool VEC>
__device__ __forceinline__ void put8(float* p, bool vec, const float (&x)[8]) {
  if (VEC || vec) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = x[i];
  }
}

// A pair (a, b) turned: three roundings each, so that the values are those of the formula's steps in fp32.
__device__ __forceinline__ float turned_low(float a, float b, float2 cs) { return __fsub_rn(__fmul_rn(a, cs.x), __fmul_rn(b, cs.y)); }
__device__ __forceinline__ float turned_high(float a, float b, float2 cs) { return __fadd_rn(__fmul_rn(b, cs.x), __fmul_rn(a, cs.y)); }

// The eight lanes of a group hold eight channels each: their 4-bit numbers packed, and the group's scale and offset.  f: the values in fp32, at most `off`
// from the exact ones (OFF; else they are those), which exact() makes in 64 bits.  fp32 decides where it can: something that its error could round
// elsewhere takes the formula in 64 bits, one warp in a hundred.  (10584 rows of 32, 8 and 8 heads of 128: 74 us, all in 64 bits 85.)
template <bool OFF, typename E>
__device__ __forceinline__ uint32_t four_bits(const float (&f)[8], float off, const E& exact, uint32_t& pair) {
  float lo = f[0], hi = f[0], none = 0.f;  // none: NaN with a NaN or an infinity
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, f[i]);
    hi = fmaxf(hi, f[i]);
    none = fmaf(f[i], 0.f, none);
  }
#pragma unroll
  for (int w = 1; w < 8; w <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, w));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, w));
    if (OFF) off = fmaxf(off, __shfl_xor_sync(0xffffffffu, off, w));
  }
  const bool odd = ((__ballot_sync(0xffffffffu, none != none) >> (threadIdx.x & 24)) & 0xffu) != 0u;
  float zero = __bfloat162float(__float2bfloat16_rn(lo));            // (rounding keeps the order: the least value's)
  bool unsure = OFF && __bfloat162float(__float2bfloat16_rn(lo - off)) != __bfloat162float(__float2bfloat16_rn(lo + off));
  // hi - zero, its product with 1 / 15 and that constant are rounded: 3 x 2^-24 of the quotient
  const float fifteenth = (hi - zero) * (1.f / 15.f), about = fabsf(fifteenth) * 0x1p-22f + (OFF ? off : 0.f);
  float scale = __bfloat162float(__float2bfloat16_rn(fifteenth));
  unsure |= __bfloat162float(__float2bfloat16_rn(fifteenth - about)) != __bfloat162float(__float2bfloat16_rn(fifteenth + about));
  unsure |= fabsf(fifteenth) < 1e-30f && hi != zero;                 // its reciprocal, or a product with it, may leave the range of fp32
  const float inv = scale > 0.f ? __fdividef(1.f, scale) * (1.f / 15.f) : 0.f;
  // in steps: the difference, the reciprocal, the constant and two products are rounded, 16 x 6 x 2^-24 together
  const float near = OFF ? fmaf(16.f * off, inv, 1e-5f) : 1e-5f;
  constexpr float kRound = 12582912.f;     // 1.5 2^23: added, what is left behind the point is rounded away
  float edge = 0.f, sum[2] = {8388608.f, 8388608.f};                 // (2^23: the sums of four numbers times 16^i stand in its last bits)
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = __saturatef((f[i] - zero) * inv), n = fmaf(t, 15.f, kRound) - kRound;
    edge = fmaxf(edge, fabsf(fmaf(t, 15.f, -n)));
    sum[i / 4] = fmaf(n, (float)(1 << (4 * (i & 3))), sum[i / 4]);
  }
  uint32_t packed = __byte_perm(__float_as_uint(sum[0]), __float_as_uint(sum[1]), 0x5410);
  const bool border = edge > 0.5f - near;
  if (OFF) {
    unsure |= border;
  } else if (__any_sync(0xffffffffu, border)) {
    // Values of few bits often lie between two steps exactly.  Their difference from there has the sign of d - (n + 1/2) scale, whose product has 13
    // bits, with what d = f - zero leaves; a rest that 64 bits would lose is left to them.
    packed = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float d = f[i] - zero, back = d - f[i], left = (f[i] - (d - back)) - (zero + back);
      const float below = floorf(__saturatef(d * inv) * 15.f), at = fmaf(-(below + 0.5f), scale, d), side = at + left;
      const int n = (int)below;
      packed |= (uint32_t)(side > 0.f || (side == 0.f && (n & 1)) ? n + 1 : n) << (4 * i);
      unsure |= at == 0.f && left != 0.f && fabsf(left) < d * 0x1p-50f;
    }
  }
  if (__any_sync(0xffffffffu, unsure && !odd)) {
    double x[8];
    exact(x);
    double top = x[0];
    lo = (float)x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      lo = fminf(lo, (float)x[i]);
      top = x[i] > top ? x[i] : top;
    }
#pragma unroll
    for (int w = 1; w < 8; w <<= 1) {
      lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, w));
      const double other = __shfl_xor_sync(0xffffffffu, top, w);
      top = other > top ? other : top;
    }
    zero = __bfloat162float(__float2bfloat16_rn(lo));
    scale = __bfloat162float(__float2bfloat16_rn((float)((top - (double)zero) / 15.0)));
    packed = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double n = rint((x[i] - (double)zero) / (double)scale);
      packed |= (uint32_t)fmin(fmax(n, 0.0), 15.0) << (4 * i);
    }
  }
  // (with a NaN or an infinity the offset reads back as NaN whatever the numbers are)
  pair = odd ? 0x7fc07fc0u : (__float_as_uint(scale) >> 16) | (__float_as_uint(zero) & 0xffff0000u);
  return odd || !(scale > 0.f) ? 0u : packed;
}

// A block has `per_block` consecutive rows: first their places and angles, a warp to a row, then all their chunks of channels in one walk, several of
// a thread's in flight.  (One row at a time spends most of a block's life on the way to its first chunk: the sequence, its length, its page, the
// angles, one after the other; 10584 rows of 48 heads of 128 took 145 us.)
constexpr int kMaxRows = 4;
// Angle f of a row: the k-th angles of consecutive chunks side by side, since the lanes of a warp read those.
__device__ __forceinline__ int placed(int f) { return (f & 7) * (kMaxTurned / 16) + (f >> 3); }
template <typename T, bool FOUR, bool VEC>
__global__ void __launch_bounds__(kAppendThreads, 4) cache_append_kernel(const AppendParams p) {
  kernel_begin();
  __shared__ float2 s_turn[kMaxRows][kMaxTurned / 2];                       // cos, sin of a row's angles
  __shared__ double2 s_exact[FOUR ? kMaxRows : 1][kMaxTurned / 2];          // the same in 64 bits, for keys that go to 4 bits
  __shared__ int32_t s_page[kMaxRows], s_slot[kMaxRows];                    // -2: a row of no sequence
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t row0 = blockIdx.x * p.per_block, rows = min(p.per_block, p.rows - row0);
  const int half = p.turned / 2, dh = p.c.dh;
  if (warp < rows) {
    const int32_t row = row0 + warp, s = sequence_of(p.cu, p.c.n_seq, p.rows, row);
    int32_t page = -2, slot = 0;
    if (s >= 0) {
      const int32_t i = row - bounded(p.cu[s], p.rows), n = bounded(p.cu[s + 1], p.rows) - (row - i);
      const int32_t place = p.c.lens ? p.c.lens[s] - n + i : i;
      page = -1;
      if (p.c.k) {
        const int32_t entry = place >= 0 ? place / p.c.page_len : -1;
        page = page_of(p.c, s, entry);
        slot = place - entry * p.c.page_len;
        if (page < 0 && lane == 0) report_status(p.status, SP_ERR_SHAPE, s, row);
      }
      const double position = half > 0 ? (double)(p.positions ? p.positions[row] : place) : 0.0;
      for (int f = lane; f < half; f += 32) {
        const double turns = position * (double)p.inv_freq[f] * 0.15915494309189533577;      // angle / 2 pi
        double sn, cs;
        sincospi(2.0 * (turns - rint(turns)), &sn, &cs);
        if (FOUR) s_exact[warp][placed(f)] = make_double2(cs, sn);
        s_turn[warp][placed(f)] = make_float2((float)cs, (float)sn);
      }
    }
    if (lane == 0) {
      s_page[warp] = page;
      s_slot[warp] = slot;
    }
  }
  __syncthreads();
  const int per_head = dh / 8, half8 = half / 8, turned8 = p.turned / 8;
  // queries: a thread has both chunks of a pair, so that a row may be turned in its place; two units of a thread in flight
  if (p.q) {
    const int apart = p.neighbours ? 0 : half8;                  // pairs of chunks: chunk and chunk + apart
    const uint32_t all = (uint32_t)rows * p.q_row.d;
    const bool vec = p.q_vec != 0;
    for (uint32_t e0 = threadIdx.x; e0 < all; e0 += 2 * kAppendThreads) {
      float a[2][8], b[2][8];
      uint32_t r[2], head[2];
      int chunk[2];
      bool live[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const uint32_t e = e0 + y * kAppendThreads;
        r[y] = quotient(e, p.q_row);
        live[y] = e < all && s_page[r[y]] != -2;
        const uint32_t x_ = e - r[y] * p.q_row.d;
        head[y] = quotient(x_, p.q_head);
        const int u = (int)(x_ - head[y] * p.q_head.d);
        chunk[y] = u < apart || apart == 0 ? u : u + apart;
        if (!live[y]) continue;
        const T* src = reinterpret_cast<const T*>(p.q) + (row0 + r[y]) * p.ldq + head[y] * dh + 8 * chunk[y];
        load8<VEC>(src, vec, a[y]);
        if (apart > 0 && chunk[y] < turned8) load8<VEC>(src + half, vec, b[y]);
      }
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        if (!live[y]) continue;
        T* dst = reinterpret_cast<T*>(p.q_out) + (row0 + r[y]) * p.ldqo + head[y] * dh + 8 * chunk[y];
        if (chunk[y] >= turned8) {
          put8<VEC>(dst, vec, a[y]);
        } else if (apart > 0) {
          float x[8], z[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float2 cs = s_turn[r[y]][placed(8 * chunk[y] + k)];
            x[k] = turned_low(a[y][k], b[y][k], cs);
            z[k] = turned_high(a[y][k], b[y][k], cs);
          }
          put8<VEC>(dst, vec, x);
          put8<VEC>(dst + half, vec, z);
        } else {
          float x[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 cs = s_turn[r[y]][placed(4 * chunk[y] + k)];
            x[2 * k] = turned_low(a[y][2 * k], a[y][2 * k + 1], cs);
            x[2 * k + 1] = turned_high(a[y][2 * k], a[y][2 * k + 1], cs);
          }
          put8<VEC>(dst, vec, x);
        }
      }
    }
  }
  // keys and values: eight channels as they stand side by side in the cache, a key's partners read beside them
  const int chunks = p.c.n_kv * per_head;
  const uint32_t all = (uint32_t)rows * p.k_row.d;               // (whole warps to a row: groups of eight lanes stay together)
  for (uint32_t e = threadIdx.x; e < all; e += kAppendThreads) {
    const uint32_t r = quotient(e, p.k_row);                     // (the same in a warp)
    const int x_ = (int)(e - r * p.k_row.d), page = s_page[r];
    if (page == -2) continue;
    const bool live = x_ < chunks;
    const int head = live ? (int)quotient((uint32_t)x_, p.k_head) : 0, chunk = live ? x_ - head * per_head : 0;
    const bool turns = chunk < turned8, second = !p.neighbours && chunk >= half8;      // the pair's other value stands `half` before, or behind
    const int64_t column = head * dh + 8 * chunk;
    const T* src = reinterpret_cast<const T*>(p.k) + (row0 + r) * p.ldk + column;
    float a[8], b[8], v[8];
    load8<VEC>(src, p.k_vec != 0, a);
    if (turns && !p.neighbours) load8<VEC>(second ? src - half : src + half, p.k_vec != 0, b);
    if (p.c.k) load8<VEC>(reinterpret_cast<const T*>(p.v) + (row0 + r) * p.ldv + column, p.v_vec != 0, v);
    // x = a cos + b sin, b with the sign that it has in the pair
    float x[8];
    const float sign = second ? 1.f : -1.f;
    if (!turns) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[k] = a[k];
        b[k] = 0.f;
      }
    } else if (p.neighbours) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float2 cs = s_turn[r][placed(4 * chunk + k / 2)];
        b[k] = k & 1 ? a[k - 1] : -a[k + 1];
        x[k] = __fadd_rn(__fmul_rn(a[k], cs.x), __fmul_rn(b[k], cs.y));
      }
    } else {
      const float2* turn = s_turn[r] + placed(8 * (second ? chunk - half8 : chunk));
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float2 cs = turn[placed(k)];
        x[k] = fmaf(__fmul_rn(b[k], cs.y), sign, __fmul_rn(a[k], cs.x));      // (a product with 1 or -1 is exact: the sum is rounded, as above)
      }
    }
    if (p.k_out && live) put8<VEC>(reinterpret_cast<T*>(p.k_out) + (row0 + r) * p.ldko + column, p.k_vec != 0, x);
    if (!p.c.k) continue;
    const int64_t at = (int64_t)head * p.c.page_len + s_slot[r];      // (head, token) of the page
    if constexpr (FOUR) {
      // a turned value's cosine, sine, products and sum are rounded: 3 x 2^-24 of |a| + |b|
      float off = 0.f;
      if (turns) {
#pragma unroll
        for (int k = 0; k < 8; ++k) off = fmaxf(off, fabsf(a[k]) + fabsf(b[k]));
        off *= 0x1p-22f;
      }
      uint32_t pair_k, pair_v;
      const uint32_t packed_k = four_bits<true>(x, off, [&](double (&y)[8]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          y[k] = (double)a[k];
          if (!turns) continue;
          const double2 cs = s_exact[r][placed(p.neighbours ? 4 * chunk + k / 2 : 8 * (second ? chunk - half8 : chunk) + k)];
          y[k] = fma((double)a[k], cs.x, (double)b[k] * (p.neighbours || second ? cs.y : -cs.y));
        }
      }, pair_k);
      const uint32_t packed_v = four_bits<false>(v, 0.f, [&](double (&y)[8]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = (double)v[k];
      }, pair_v);
      if (page >= 0 && live) {
        const int64_t to = page * p.c.step + at * (dh / 2) + 4 * chunk;
        *reinterpret_cast<uint32_t*>(p.c.k + to) = packed_k;
        *reinterpret_cast<uint32_t*>(p.c.v + to) = packed_v;
        if (chunk % 8 == 0) {
          const int64_t pair_to = page * p.c.scale_step + (at * (dh / kCacheGroup) + chunk / 8) * 4;
          *reinterpret_cast<uint32_t*>(p.c.ks + pair_to) = pair_k;
          *reinterpret_cast<uint32_t*>(p.c.vs + pair_to) = pair_v;
        }
      }
    } else if (page >= 0 && live) {
      const int64_t to = page * p.c.step + (at * dh + 8 * chunk) * 2;
      put8<true>(reinterpret_cast<__nv_bfloat16*>(p.c.k + to), true, x);
      put8<true>(reinterpret_cast<__nv_bfloat16*>(p.c.v + to), true, v);
    }
  }
}

struct ReadParams {
  CacheView c;
  const int32_t* cu;
  void *k, *v;
  int64_t ldk, ldv;
  const int32_t* whole;                    // null: any last tokens
  int32_t rows, k_vec, v_vec;
  Divisor head;                            // chunks of a head
  const HalfTops* tops;
  int32_t* status;
};
// The eight values of a word of numbers, one rounding each: scale n + zero.  A number is put in the place of a mantissa's bits of 2^23, 2^19 ..,
// which are taken away again: conversions of integers have a sixteenth of the rate of that.
__device__ __forceinline__ void open8(uint32_t w, uint32_t pair, float (&x)[8]) {
  const float scale = __uint_as_float(pair << 16), zero = __uint_as_float(pair & 0xffff0000u);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint32_t from = k < 4 ? w : w >> 16;
    const int at = 4 * (k & 3);
    x[k] = fmaf(__uint_as_float((from & (15u << at)) | ((150u - at) << 23)) - (float)(1 << (23 - at)), scale, zero);
  }
}
// The same in fp16, in units of 1 / f: scales and offsets fit into it but for what lies 2^-28 below the largest of the text's head.
__device__ __forceinline__ void open8_half(__half* p, uint32_t w, uint32_t pair, float f) {
  const __half2 scale = __float2half2_rn(__uint_as_float(pair << 16) * f), zero = __float2half2_rn(__uint_as_float(pair & 0xffff0000u) * f);
  __half2 x[4];                            // channels i and i + 4
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = ((w >> (4 * i)) & 0x000f000fu) | 0x64006400u;             // 1024 + n
    x[i] = __hfma2(__hsub2(*reinterpret_cast<const __half2*>(&m), __half2half2(__ushort_as_half(0x6400u))), scale, zero);
  }
  const __half2 y[4] = {__lows2half2(x[0], x[1]), __lows2half2(x[2], x[3]), __highs2half2(x[0], x[1]), __highs2half2(x[2], x[3])};
  *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(y);
}

constexpr uint32_t kNan2 = 0x7fff7fffu;   // two of fp16, or of bf16

// a warp per row: eight channels of keys and of values at a time in every lane (more warps at once are worth more than two chunks of a lane in
// flight: 17k rows of 8 heads of 128 to fp16 20 us, unrolled 23).  T of fp16: contiguous rows in the units that tops give, or of bf16.
template <typename T, bool FOUR>
__global__ void __launch_bounds__(256) cache_read_kernel(const ReadParams p) {
  kernel_begin();
  const int lane = threadIdx.x & 31;
  const int32_t row = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= p.rows) return;
  const int32_t s = sequence_of(p.cu, p.c.n_seq, p.rows, row);
  if (s < 0) return;
  const int32_t i = row - bounded(p.cu[s], p.rows), n = bounded(p.cu[s + 1], p.rows) - (row - i);
  const int32_t length = p.c.lens[s], place = length - n + i;
  const int32_t entry = place >= 0 ? place / p.c.page_len : -1;
  const int32_t page = p.whole && n != p.whole[s] ? -1 : page_of(p.c, s, entry);
  const int32_t slot = place - entry * p.c.page_len;
  if (page < 0 && lane == 0) report_status(p.status, SP_ERR_SHAPE, s, entry);
  constexpr bool HALF = std::is_same<T, __half>::value;
  const int dh = p.c.dh, chunks = p.c.n_kv * (dh / 8);
  T *k_row = reinterpret_cast<T*>(p.k) + row * p.ldk, *v_row = reinterpret_cast<T*>(p.v) + row * p.ldv;
#pragma unroll 1
  for (int e = lane; e < chunks; e += 32) {
    const int head = (int)quotient((uint32_t)e, p.head), chunk = e - head * (int)p.head.d;       // (heads are whole chunks: they go to 8 e)
    const int64_t at = (int64_t)head * p.c.page_len + slot;
    float x[8], y[8];
    if (page < 0) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = y[k] = NAN;       // (fp16: below)
    } else if constexpr (FOUR) {
      const int64_t from = page * p.c.step + at * (dh / 2) + 4 * chunk, g = page * p.c.scale_step + (at * (dh / kCacheGroup) + chunk / 8) * 4;
      const uint32_t a = *reinterpret_cast<const uint32_t*>(p.c.k + from), b = *reinterpret_cast<const uint32_t*>(p.c.v + from);
      const uint32_t sa = *reinterpret_cast<const uint32_t*>(p.c.ks + g), sb = *reinterpret_cast<const uint32_t*>(p.c.vs + g);
      if constexpr (HALF) {
        const HalfTops t = p.tops[(int64_t)s * p.c.n_kv + head];
        if (half_holds(t)) {
          open8_half(k_row + 8 * e, a, sa, power_of_two(-half_exponent(t.k_top)));
          open8_half(v_row + 8 * e, b, sb, power_of_two(-half_exponent(t.v_top)));
          continue;
        }
      }
      open8(a, sa, x);
      open8(b, sb, y);
    } else {
      const int64_t from = page * p.c.step + (at * dh + 8 * chunk) * 2;
      load8<true>(reinterpret_cast<const __nv_bfloat16*>(p.c.k + from), true, x);
      load8<true>(reinterpret_cast<const __nv_bfloat16*>(p.c.v + from), true, y);
    }
    if constexpr (HALF) {
      if (page < 0) {
        *reinterpret_cast<uint4*>(k_row + 8 * e) = *reinterpret_cast<uint4*>(v_row + 8 * e) = make_uint4(kNan2, kNan2, kNan2, kNan2);
      } else {
        put8<true>(reinterpret_cast<__nv_bfloat16*>(k_row) + 8 * e, true, x);
        put8<true>(reinterpret_cast<__nv_bfloat16*>(v_row) + 8 * e, true, y);
      }
    } else {
      put8<false>(k_row + 8 * e, p.k_vec != 0, x);
      put8<false>(v_row + 8 * e, p.v_vec != 0, y);
    }
  }
}

// Least and largest bound 15 |scale| + |zero| of the keys and of the values of every text and key head, among the rows that cache_open opens.  A block
// takes one key head of consecutive rows, 256 at a time, a row to a thread, since a head's scales of the rows of a page stand side by side; with a row
// to a warp every 8 bytes come in a sector of their own.  A warp leaves its bounds where a text ends, and what a block has of one text at its end
// meets in shared memory: an atomic of each warp queues at a few words, one of each thread all the more.  (Maxima and minima are the same in any order.)
struct TopsParams {
  CacheView c;
  const int32_t *cu, *whole;
  int32_t rows, per_strip;
  HalfTops* tops;
};
__global__ void __launch_bounds__(256) cache_tops_kernel(const TopsParams p) {
  kernel_begin();
  __shared__ int s_seq;
  __shared__ HalfTops s_tops[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t head = (int32_t)(blockIdx.x % (uint32_t)p.c.n_kv);
  const int64_t begin = (int64_t)(blockIdx.x / (uint32_t)p.c.n_kv) * p.per_strip, end = min(begin + p.per_strip, (int64_t)p.rows);
  const int per_head = p.c.dh / kCacheGroup;
  const HalfTops none = {0u, kNoLow, 0u, kNoLow};
  HalfTops mine = none;
  int32_t seq = -1;                        // the text that `mine` is of
  const auto leave = [&](int32_t s, const HalfTops& t) {
    HalfTops* to = p.tops + (int64_t)s * p.c.n_kv + head;
    if (t.k_top != 0u) atomicMax(&to->k_top, t.k_top);
    if (t.k_low != kNoLow) atomicMin(&to->k_low, t.k_low);
    if (t.v_top != 0u) atomicMax(&to->v_top, t.v_top);
    if (t.v_low != kNoLow) atomicMin(&to->v_low, t.v_low);
  };
  // bounds of the lanes that have this lane's text; whether this lane speaks for them
  const auto meet = [&] {
    const uint32_t peers = __match_any_sync(0xffffffffu, seq);
    mine.k_top = __reduce_max_sync(peers, mine.k_top);
    mine.k_low = __reduce_min_sync(peers, mine.k_low);
    mine.v_top = __reduce_max_sync(peers, mine.v_top);
    mine.v_low = __reduce_min_sync(peers, mine.v_low);
    return seq >= 0 && lane == __ffs(peers) - 1;
  };
  const auto take = [](uint32_t& top, uint32_t& low, uint32_t pair) {
    const float scale = fabsf(__uint_as_float(pair << 16)), zero = fabsf(__uint_as_float(pair & 0xffff0000u));
    if (!(scale < INFINITY) || !(zero < INFINITY)) return;                // (a NaN either)
    const uint32_t bits = __float_as_uint(fminf(fmaf(15.f, scale, zero), 3.402823466e38f));
    top = max(top, bits);
    if (bits != 0u) low = min(low, bits);
  };
  for (int64_t row0 = begin; row0 < end; row0 += 256) {
    const int64_t row = row0 + threadIdx.x;
    int32_t s = -1, place = 0, entry = 0, page = -1;
    if (row < end) {
      s = sequence_near(p.cu, p.c.n_seq, p.rows, row);                    // (cu[0] is 0)
      const int32_t first = bounded(p.cu[s], p.rows), n = bounded(p.cu[s + 1], p.rows) - first;
      place = (int32_t)row - first;
      entry = place / p.c.page_len;
      if (place < n && n == p.whole[s]) page = page_of(p.c, s, entry);
    }
    if (__any_sync(0xffffffffu, page >= 0 && seq >= 0 && s != seq)) {
      if (meet()) leave(seq, mine);
      mine = none;
      seq = -1;
    }
    if (page < 0) continue;
    seq = s;
    const int64_t at = page * p.c.scale_step + ((int64_t)head * p.c.page_len + place - entry * p.c.page_len) * per_head * 4;
#pragma unroll 2
    for (int g = 0; g < per_head; ++g) {
      take(mine.k_top, mine.k_low, *reinterpret_cast<const uint32_t*>(p.c.ks + at + 4 * g));
      take(mine.v_top, mine.v_low, *reinterpret_cast<const uint32_t*>(p.c.vs + at + 4 * g));
    }
  }
  __syncwarp();
  const bool first = meet();
  if (threadIdx.x == 0) s_seq = -1;
  __syncthreads();
  if (seq >= 0) atomicMax(&s_seq, seq);
  if (lane == 0) s_tops[warp] = none;
  __syncthreads();
  const int32_t text = s_seq;
  if (!__syncthreads_and(seq < 0 || seq == text)) {
    if (first) leave(seq, mine);
    return;
  }
  if (first) s_tops[warp] = mine;
  __syncthreads();
  if (threadIdx.x != 0 || text < 0) return;
  HalfTops all = none;
  for (int w = 0; w < 8; ++w) {
    all.k_top = max(all.k_top, s_tops[w].k_top);
    all.k_low = min(all.k_low, s_tops[w].k_low);
    all.v_top = max(all.v_top, s_tops[w].v_top);
    all.v_low = min(all.v_low, s_tops[w].v_low);
  }
  leave(text, all);
}
struct QueriesParams {
  const __nv_bfloat16* q;
  const int32_t* cu_q;
  const HalfTops* tops;
  __half* out;
  float* unit;
  int64_t ldq, rows;
  int32_t n_heads, n_kv, dh, n_seq, vec;
};
// eight channels to a thread, the 8 or 16 threads of a head side by side in a warp
__global__ void __launch_bounds__(256) queries_to_half_kernel(const QueriesParams p) {
  kernel_begin();
  const int32_t per_head = p.dh / 8, per_row = p.n_heads * per_head;
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = min(e / per_row, p.rows - 1);              // (lanes behind the end stay for the shuffles)
  const int32_t j = (int32_t)(e % per_row), head = j / per_head;
  float x[8], top = 0.f;
  load8<false>(p.q + row * p.ldq + 8 * j, p.vec != 0, x);
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (fabsf(x[k]) < INFINITY) top = fmaxf(top, fabsf(x[k]));
  for (int w = 1; w < per_head; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
  if (e >= p.rows * per_row) return;
  const int32_t s = sequence_near(p.cu_q, p.n_seq, (int32_t)p.rows, row);
  const bool half = half_holds(p.tops[(int64_t)s * p.n_kv + head / (p.n_heads / p.n_kv)]);
  const int unit = half ? half_exponent(__float_as_uint(top)) : 0;
  if (j % per_head == 0) p.unit[row * p.n_heads + head] = power_of_two(unit);
  __half* to = p.out + row * ((int64_t)p.n_heads * p.dh) + 8 * j;
  if (!half) {
    put8<true>(reinterpret_cast<__nv_bfloat16*>(to), true, x);
    return;
  }
  const float f = power_of_two(-unit);
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 y = __floats2half2_rn(x[2 * i] * f, x[2 * i + 1] * f);
    u[i] = *reinterpret_cast<const uint32_t*>(&y);
  }
  *reinterpret_cast<uint4*>(to) = make_uint4(u[0], u[1], u[2], u[3]);
}

bool rows_of_16(const void* ptr, int64_t ld, int32_t dtype, int64_t rows) {
  return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0 && (rows < 2 || ld * (int64_t)dtype_size(dtype) % 16 == 0);
}
bool step_fits(int64_t step, int64_t page_bytes, int64_t unit, int32_t n_pages) {
  return n_pages < 2 || (step % unit == 0 && step >= page_bytes && step <= (int64_t)0xfffffffe * unit / n_pages);
}

}  // namespace

sp_status check_cache(const sp_kv_cache* c, bool pages) {
  if (!c) return SP_ERR_INVALID_ARG;
  if (c->kind != SP_CACHE_BF16 && c->kind != SP_CACHE_4BIT) return SP_ERR_INVALID_ARG;
  if (c->n_kv_heads < 1 || c->n_kv_heads > (1 << 12) || c->d_head < 1 || c->n_seq < 0) return SP_ERR_SHAPE;
  if (c->d_head > 128 || c->d_head % (c->kind == SP_CACHE_4BIT ? kCacheGroup : 16) != 0) return SP_ERR_UNSUPPORTED;
  if (!c->k) return pages ? SP_ERR_INVALID_ARG : SP_OK;
  const bool four = c->kind == SP_CACHE_4BIT;
  if (!c->v || (four && (!c->k_scale || !c->v_scale))) return SP_ERR_INVALID_ARG;
  if (c->n_seq > 0 && (!c->table || !c->lens)) return SP_ERR_INVALID_ARG;
  if (c->n_pages < 1 || c->page_len < 16 || c->page_len > 65536 || c->page_len % 16 != 0 || c->max_pages < 0 ||
      (int64_t)c->max_pages * c->page_len > (1 << 30) || (c->n_seq > 1 && c->table_ld < c->max_pages))
    return SP_ERR_SHAPE;
  const int64_t tokens = (int64_t)c->n_kv_heads * c->page_len, bytes = tokens * (four ? c->d_head / 2 : 2 * c->d_head);
  // (a place in a page is named by 32 bits in units of 128 bytes, of 64 among the scales)
  if (!step_fits(c->step, bytes, 128, c->n_pages) ||
      (four && !step_fits(c->scale_step, tokens * (c->d_head / kCacheGroup) * 4, 64, c->n_pages)))
    return SP_ERR_SHAPE;
  for (const void* ptr : {c->k, c->v, four ? c->k_scale : nullptr, four ? c->v_scale : nullptr})
    if (reinterpret_cast<uintptr_t>(ptr) & 15u) return SP_ERR_ALIGNMENT;
  return SP_OK;
}

CacheView cache_view(const sp_kv_cache* c) {
  CacheView w = {};
  w.k = reinterpret_cast<uint8_t*>(c->k); w.v = reinterpret_cast<uint8_t*>(c->v);
  w.ks = reinterpret_cast<uint8_t*>(c->k_scale); w.vs = reinterpret_cast<uint8_t*>(c->v_scale);
  w.step = c->step; w.scale_step = c->scale_step;
  w.table = c->table; w.lens = c->lens; w.table_ld = c->table_ld;
  w.n_pages = c->n_pages; w.page_len = c->page_len; w.max_pages = c->max_pages;
  w.n_kv = c->n_kv_heads; w.dh = c->d_head; w.n_seq = c->n_seq;
  return w;
}

namespace {
cudaError_t read_rows(const sp_kv_cache* c, const int32_t* cu, const int32_t* whole, int64_t rows, void* K, void* V, int64_t ldk, int64_t ldv,
                      int32_t dtype, const HalfTops* tops, int32_t* status, cudaStream_t stream) {
  ReadParams p = {};
  p.c = cache_view(c);
  p.cu = cu;
  p.k = K; p.v = V; p.ldk = ldk; p.ldv = ldv;
  p.rows = (int32_t)rows;
  p.whole = whole;
  p.head = divisor(c->d_head / 8);
  p.k_vec = rows_of_16(K, ldk, dtype, rows); p.v_vec = rows_of_16(V, ldv, dtype, rows);
  p.tops = tops;
  p.status = status;
  count_launch();
  const dim3 grid((unsigned)ceil_div(rows, (int64_t)8));
  const bool four = c->kind == SP_CACHE_4BIT;
  if (tops) return launch(cache_read_kernel<__half, true>, grid, dim3(256), 0, stream, p);
  if (dtype == SP_F32)
    return four ? launch(cache_read_kernel<float, true>, grid, dim3(256), 0, stream, p)
                : launch(cache_read_kernel<float, false>, grid, dim3(256), 0, stream, p);
  return four ? launch(cache_read_kernel<__nv_bfloat16, true>, grid, dim3(256), 0, stream, p)
              : launch(cache_read_kernel<__nv_bfloat16, false>, grid, dim3(256), 0, stream, p);
}
}  // namespace

cudaError_t cache_read(const sp_kv_cache* c, const int32_t* cu, int64_t rows, void* K, void* V, int64_t ldk, int64_t ldv, int32_t dtype,
                       int32_t* status, cudaStream_t stream) {
  return read_rows(c, cu, nullptr, rows, K, V, ldk, ldv, dtype, nullptr, status, stream);
}
cudaError_t cache_open(const sp_kv_cache* c, const int32_t* cu, const int32_t* whole, int64_t rows, void* K, void* V, const HalfTops* tops,
                       int32_t* status, cudaStream_t stream) {
  const int64_t ld = (int64_t)c->n_kv_heads * c->d_head;
  return read_rows(c, cu, whole, rows, K, V, ld, ld, SP_BF16, tops, status, stream);
}
cudaError_t cache_tops(const sp_kv_cache* c, const int32_t* cu, const int32_t* whole, int64_t rows, HalfTops* tops, cudaStream_t stream) {
  TopsParams p = {};
  p.c = cache_view(c);
  p.cu = cu; p.whole = whole;
  p.rows = (int32_t)rows;
  p.tops = tops;
  const int64_t most = ceil_div(4 * (int64_t)sm_count(), (int64_t)c->n_kv_heads);
  p.per_strip = (int32_t)align_up((size_t)ceil_div(rows, most), 256);
  count_launch();
  return launch(cache_tops_kernel, dim3((unsigned)(ceil_div(rows, (int64_t)p.per_strip) * c->n_kv_heads)), dim3(256), 0, stream, p);
}
cudaError_t queries_to_half(const sp_kv_cache* c, const sp_mat* Q, const int32_t* cu_q, void* Q_half, float* q_unit, const HalfTops* tops,
                            cudaStream_t stream) {
  QueriesParams p = {};
  p.q = reinterpret_cast<const __nv_bfloat16*>(Q->ptr);
  p.cu_q = cu_q;
  p.tops = tops;
  p.out = reinterpret_cast<__half*>(Q_half);
  p.unit = q_unit;
  p.ldq = Q->ld; p.rows = Q->rows;
  p.n_heads = (int32_t)(Q->cols / c->d_head); p.n_kv = c->n_kv_heads; p.dh = c->d_head; p.n_seq = c->n_seq;
  p.vec = rows_of_16(Q->ptr, Q->ld, SP_BF16, Q->rows);
  count_launch();
  return launch(queries_to_half_kernel, dim3((unsigned)ceil_div(Q->rows * (Q->cols / 8), (int64_t)256)), dim3(256), 0, stream, p);
}

}  // namespace sp

extern "C" {

sp_status sp_cache_append(const sp_kv_cache* cache, const sp_cache_append_args* a, int32_t* status_dev, void* stream) {
  using namespace sp;
  if (!a) return SP_ERR_INVALID_ARG;
  const sp_status ok = check_cache(cache, false);
  if (ok != SP_OK) return ok;
  const int32_t dt = a->K.dtype;
  if (dt != SP_F32 && dt != SP_BF16) return SP_ERR_DTYPE;
  const bool pages = cache->k != nullptr;
  const int64_t N = a->K.rows, kv = (int64_t)cache->n_kv_heads * cache->d_head;
  if (N < 0 || N > (1 << 30) || a->K.cols != kv || (N > 1 && a->K.ld < kv)) return SP_ERR_SHAPE;
  if (pages) {
    if (a->V.dtype != dt) return SP_ERR_DTYPE;
    if (a->V.rows != N || a->V.cols != kv || (N > 1 && a->V.ld < kv)) return SP_ERR_SHAPE;
  }
  const bool queries = a->Q.ptr != nullptr || a->Q_out.ptr != nullptr, keys = a->K_out.ptr != nullptr;
  if (queries) {
    if (!a->Q.ptr || !a->Q_out.ptr) return SP_ERR_INVALID_ARG;
    if (a->Q.dtype != dt || a->Q_out.dtype != dt) return SP_ERR_DTYPE;
    const int64_t q = (int64_t)a->n_heads * cache->d_head;
    if (a->n_heads < 1 || a->n_heads > (1 << 12)) return SP_ERR_SHAPE;
    for (const sp_mat* m : {&a->Q, &a->Q_out})
      if (m->rows != N || m->cols != q || (N > 1 && m->ld < q)) return SP_ERR_SHAPE;
    if (a->Q.ptr == a->Q_out.ptr && N > 1 && a->Q.ld != a->Q_out.ld) return SP_ERR_INVALID_ARG;
  }
  if (keys) {
    if (a->K_out.dtype != dt) return SP_ERR_DTYPE;
    if (a->K_out.rows != N || a->K_out.cols != kv || (N > 1 && a->K_out.ld < kv)) return SP_ERR_SHAPE;
    if (a->K_out.ptr == a->K.ptr) return SP_ERR_INVALID_ARG;      // (a key's partner may be read after it is written)
  }
  if (a->turned < 0 || a->turned > cache->d_head || a->turned % 16 != 0) return SP_ERR_SHAPE;
  if (a->turned > 0 && !a->inv_freq) return SP_ERR_INVALID_ARG;
  if (N == 0 || cache->n_seq == 0) return SP_OK;
  if (!a->K.ptr || !a->cu || (pages && !a->V.ptr)) return SP_ERR_INVALID_ARG;
  AppendParams p = {};
  p.c = cache_view(cache);
  p.q = a->Q.ptr; p.k = a->K.ptr; p.v = a->V.ptr; p.q_out = a->Q_out.ptr; p.k_out = a->K_out.ptr;
  p.ldq = a->Q.ld; p.ldk = a->K.ld; p.ldv = a->V.ld; p.ldqo = a->Q_out.ld; p.ldko = a->K_out.ld;
  p.cu = a->cu; p.positions = a->positions; p.inv_freq = a->inv_freq;
  p.rows = (int32_t)N; p.n_heads = a->n_heads; p.turned = a->turned; p.neighbours = a->neighbours != 0;
  p.q_vec = queries && rows_of_16(a->Q.ptr, a->Q.ld, dt, N) && rows_of_16(a->Q_out.ptr, a->Q_out.ld, dt, N);
  p.k_vec = rows_of_16(a->K.ptr, a->K.ld, dt, N) && (!keys || rows_of_16(a->K_out.ptr, a->K_out.ld, dt, N));
  p.v_vec = pages && rows_of_16(a->V.ptr, a->V.ld, dt, N);
  p.status = status_dev;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  count_launch();
  ProfScope prof(PK_ELEMENTWISE, 0.0, 0.0, s);
  // as many rows to a block as leave four blocks for every SM
  const int64_t most = N / (4 * (int64_t)sm_count());
  p.per_block = most < 1 ? 1 : most < kMaxRows ? (int32_t)most : kMaxRows;
  const int64_t per_head = cache->d_head / 8, units = per_head - (p.neighbours ? 0 : p.turned / 16);
  p.q_head = divisor(units); p.q_row = divisor(queries ? units * a->n_heads : 1);
  p.k_head = divisor(per_head); p.k_row = divisor((int64_t)align_up((size_t)(per_head * cache->n_kv_heads), 32));
  const dim3 grid((unsigned)ceil_div(N, (int64_t)p.per_block));
  const bool four = pages && cache->kind == SP_CACHE_4BIT;
  const bool vec = (!queries || p.q_vec) && p.k_vec && (!pages || p.v_vec);
  const auto run = [&](auto t) {
    using T = decltype(t);
    const dim3 block(kAppendThreads);
    if (vec) return four ? launch(cache_append_kernel<T, true, true>, grid, block, 0, s, p) : launch(cache_append_kernel<T, false, true>, grid, block, 0, s, p);
    return four ? launch(cache_append_kernel<T, true, false>, grid, block, 0, s, p) : launch(cache_append_kernel<T, false, false>, grid, block, 0, s, p);
  };
  const cudaError_t e = dt == SP_F32 ? run(float()) : run(__nv_bfloat16());
  return e == cudaSuccess ? SP_OK : SP_ERR_CUDA;
}

sp_status sp_cache_read(const sp_kv_cache* cache, const int32_t* cu, const sp_mat* K, const sp_mat* V, int32_t* status_dev,
                        void* stream) {
  using namespace sp;
  if (!K || !V) return SP_ERR_INVALID_ARG;
  const sp_status ok = check_cache(cache, true);
  if (ok != SP_OK) return ok;
  if ((K->dtype != SP_F32 && K->dtype != SP_BF16) || V->dtype != K->dtype) return SP_ERR_DTYPE;
  const int64_t N = K->rows, kv = (int64_t)cache->n_kv_heads * cache->d_head;
  for (const sp_mat* m : {K, V})
    if (m->rows != N || m->cols != kv || (N > 1 && m->ld < kv)) return SP_ERR_SHAPE;
  if (N < 0 || N > (1 << 30)) return SP_ERR_SHAPE;
  if (N == 0 || cache->n_seq == 0) return SP_OK;
  if (!cu || !K->ptr || !V->ptr || K->ptr == V->ptr) return SP_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  ProfScope prof(PK_ELEMENTWISE, 0.0, 0.0, s);
  return cache_read(cache, cu, N, K->ptr, V->ptr, K->ld, V->ld, K->dtype, status_dev, s) == cudaSuccess ? SP_OK : SP_ERR_CUDA;
}

}  // extern "C"
