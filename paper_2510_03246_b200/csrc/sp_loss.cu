// Log probabilities of given tokens with entropy and best alternatives, and their gradient with respect to the logits.
//
// With c = log2(e) scale and any reference r:  t_v = c (x_v - r), s = sum_v 2^t_v, w = sum_v t_v 2^t_v give
//   lse = scale r + ln2 log2 s,   log p_v = ln2 (t_v - log2 s),   entropy = ln2 (log2 s - w / s),
// and (r, s, w) of two parts of a row join by shifting both to the larger r.  So one pass over the logits suffices: every
// thread keeps its own (r, s, w) with r near its running maximum, and they are joined at the end.  All of it is held in fp32.  (The
// difference before the product: a row of nothing but the type's lowest value has finite t, while c x_v would not be.)
//
// The n best logits need no list during that pass, only every thread's largest value.  The n-th largest of those of a row is a floor that at
// least n logits reach, and few more do; they stand in the vectors of the (about n) threads whose largest value reaches it.  These
// vectors are looked at again afterwards, a warp at a time and out of L2, and what reaches the floor is gathered in shared memory, where each
// one's place is the number of larger ones.  (Sorted lists in every warp, joined by one: 285 us for 8192 rows of 50257 with eight alternatives;
// insertions follow one another.)  Where more are gathered than there is room for (many equal logits), such lists do serve.
#include <math.h>

#include "sp_common.cuh"
#include "sp_f32x2.cuh"

namespace sp {
namespace {

constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kLossThreads = 256;
constexpr int kMaxCluster = 8;
constexpr int kWideRoom = 512, kNarrowRoom = 256;      // keys gathered for a row of many warps, of one
static_assert(kNarrowRoom >= SP_MAX_ALTS && kWideRoom >= kLossThreads / 32 * SP_MAX_ALTS && kWideRoom >= kMaxCluster * SP_MAX_ALTS, "lists");

// 16 bytes of a row as floats
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& q, float (&x)[4]) {
    x[0] = __uint_as_float(q.x); x[1] = __uint_as_float(q.y); x[2] = __uint_as_float(q.z); x[3] = __uint_as_float(q.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
  // largest value of n vectors, NaN passed over; of nothing but NaN: NaN, which is not to be taken for the number -infinity
  template <int n>
  static __device__ __forceinline__ float largest(const uint4 (&q)[n]) {
    float m = __uint_as_float(q[0].x);
#pragma unroll
    for (int i = 0; i < n; ++i) {
      float x[4];
      unpack(q[i], x);
      m = fmaxf(m, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])));
    }
    return m;
  }
  static __device__ __forceinline__ float one(float v) { return v; }
  static __device__ __forceinline__ float to(float v) { return v; }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& q, float (&x)[8]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  template <int n>
  static __device__ __forceinline__ float largest(const uint4 (&q)[n]) {
    __nv_bfloat162 m = *reinterpret_cast<const __nv_bfloat162*>(&q[0].x);
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&q[i]);
      m = __hmax2(m, __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
    }
    return fmaxf(__low2float(m), __high2float(m));
  }
  static __device__ __forceinline__ float one(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 to(float v) { return __float2bfloat16_rn(v); }
};

// (r, s, w) of a part of a row; r = -infinity: nothing but -infinity so far
struct Part {
  float r, s, w;
};
__device__ __forceinline__ Part join(const Part& a, const Part& b, float c) {
  const float r = fmaxf(a.r, b.r);
  if (r == -INFINITY) return Part{r, a.s + b.s, a.w + b.w};     // (zeros, or the NaN of a NaN logit)
  // a part with r = -infinity holds zeros: its shift is taken as zero (0 * infinity), and no shift is more than 2^t can tell from 0
  const float da = a.r == -INFINITY ? 0.f : fmaxf((a.r - r) * c, -10000.f), db = b.r == -INFINITY ? 0.f : fmaxf((b.r - r) * c, -10000.f);
  const float fa = exp2_fast(da), fb = exp2_fast(db);
  return Part{r, a.s * fa + b.s * fb, (a.w + da * a.s) * fa + (b.w + db * b.s) * fb};
}

// Keys of the selection: larger value first, then the lower index; NaN below everything, zeros equal.
__device__ __forceinline__ uint32_t order_bits(float x) {
  if (x != x) return 0u;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t k) {
  if (k == 0u) return __uint_as_float(0x7fffffffu);
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ unsigned long long make_key(float x, uint32_t index) {
  return ((unsigned long long)order_bits(x) << 32) | (uint32_t)~index;
}

// The n best keys a warp has seen, one per lane in falling order (0: none yet).  floor_key: keys up to it are of no use, since
// n larger ones are known (to this warp or another one of the row).
struct WarpBest {
  unsigned long long key;
  // every lane calls; keys of the lanes in `offer` are inserted
  __device__ __noinline__ void insert(bool offer, unsigned long long k, int n, unsigned long long& floor_key, int lane) {
    uint32_t m = __ballot_sync(0xffffffffu, offer && k > floor_key);
    while (m) {
      const unsigned long long c = __shfl_sync(0xffffffffu, k, __ffs(m) - 1);
      m &= m - 1;
      if (c <= floor_key) continue;                       // the same in every lane
      const int at = __popc(__ballot_sync(0xffffffffu, key > c));
      const unsigned long long up = __shfl_up_sync(0xffffffffu, key, 1);
      if (lane == at) key = c;
      else if (lane > at) key = up;
      const unsigned long long last = __shfl_sync(0xffffffffu, key, n - 1);
      if (last > floor_key) floor_key = last;
    }
  }
};

struct LogprobParams {
  const void* x;
  int64_t ld, T;
  int32_t V, n_alts;
  float scale;
  const int64_t* targets;
  float* logp;
  float* lse;
  float* entropy;
  int32_t* alt_ids;
  float* alt_logp;
  int32_t* status;
};

// A row belongs to WARPS warps (one: eight rows a block) of each of the CTAs of a cluster (gridDim.x = rows x cluster).
constexpr int loss_threads(int warps) { return warps == 1 ? kLossThreads : warps * 32; }
template <typename T, int WARPS, bool ENT, bool ALTS>
__global__ void __launch_bounds__(loss_threads(WARPS), WARPS == 1 ? 4 : 8) token_logprobs_kernel(const LogprobParams p, int cluster) {
  kernel_begin();
  constexpr int kThreads = loss_threads(WARPS), kWarps = kThreads / 32, N = Vec<T>::N, U = 4;     // U vectors in flight per thread
  constexpr int kRoom = WARPS == 1 ? kNarrowRoom : kWideRoom, kRowsHere = WARPS == 1 ? kWarps : 1;
  __shared__ Part s_part[kWarps];
  __shared__ unsigned long long s_keys[ALTS ? kRowsHere : 1][ALTS ? kRoom : 1];
  __shared__ int s_count[kRowsHere], s_hots[kRowsHere];
  __shared__ uint32_t s_floor[kRowsHere];
  __shared__ __align__(16) uint32_t s_top[ALTS ? kThreads : 4];      // largest values of the threads
  __shared__ uint8_t s_hot[ALTS ? kThreads : 1];                      // threads of the row whose vectors are looked at again
  __shared__ Part s_all[kMaxCluster];
  __shared__ unsigned long long s_all_best[ALTS ? kMaxCluster * SP_MAX_ALTS : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rank = WARPS == 1 ? 0 : (int)(blockIdx.x % cluster);
  const int64_t row = WARPS == 1 ? (int64_t)blockIdx.x * kWarps + warp : (int64_t)(blockIdx.x / cluster);
  const bool live = row < p.T;
  const int wl = WARPS == 1 ? 0 : warp;                // warp within the row
  // (the other CTAs of a cluster write into the first one's shared memory: all have started once they meet)
  if (WARPS > 1 && cluster > 1) {
    if (ALTS)
      for (int i = threadIdx.x; i < kMaxCluster * SP_MAX_ALTS; i += kThreads) s_all_best[i] = 0ull;
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  }
  const int tid = WARPS == 1 ? lane : (int)threadIdx.x;      // thread within the row
  unsigned long long* keys = s_keys[WARPS == 1 && ALTS ? warp : 0];
  const int rh = WARPS == 1 ? warp : 0;                      // row within the block
  int* count = &s_count[rh];
  auto row_sync = [&] {
    if (WARPS > 1) __syncthreads();
    else __syncwarp();
  };
  const float c = p.scale * kLog2E;
  Part a{-INFINITY, 0.f, 0.f};
  float rc = 0.f;                                      // a.r, or 0 while that is -infinity
  float top = -INFINITY;                               // largest value of this thread's vectors
  bool any = false;                                    // it has had one that is a number

  // The reference follows a maximum that has risen by more than 2^4 (from -infinity: by anything), so that rescaling is rare.  (Not
  // much more: log2 s and w / s, the difference of which is the entropy, grow by as much.)
  auto raise = [&](float m) {
    if ((m - a.r) * c > 4.f) {
      const float d = fmaxf((a.r - m) * c, -10000.f), f = exp2_fast(d);      // a.r = -infinity: f = 0, and s = w = 0
      if (ENT) a.w = f * fmaf(d, a.s, a.w);
      a.s *= f;
      a.r = m;
      rc = m;
    }
  };
  auto take_one = [&](float v) {
    const float t = (v - rc) * c, e = exp2_fast(t);
    a.s += e;
    // (a logit of -infinity: e = 0, and 0 times a finite number is added)
    if (ENT) a.w = fmaf(e, fmaxf(t, -10000.f), a.w);
  };
  const uint64_t c2 = pack2(c, c);
  // Vectors into (r, s, w), two values at a time.  A logit of -infinity adds 0 times infinity to w: seen afterwards (as is a NaN), and
  // the vectors are then taken value by value.
  auto take = [&](const auto& q) {
    constexpr int n = sizeof(q) / sizeof(uint4);
    const float hi = Vec<T>::largest(q);
    raise(hi);
    if (ALTS) {
      any |= hi == hi;
      top = fmaxf(top, hi);
    }
    const uint64_t r2 = pack2(-rc, -rc);
    uint64_t s2 = pack2(a.s, 0.f), w2 = pack2(a.w, 0.f);
#pragma unroll
    for (int u = 0; u < n; ++u) {
      float x[N];
      Vec<T>::unpack(q[u], x);
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        const uint64_t t = mul2(add2(pack2(x[i], x[i + 1]), r2), c2);
        float e0, e1;
        unpack2(t, e0, e1);
        const uint64_t e = pack2(exp2_fast(e0), exp2_fast(e1));
        s2 = add2(s2, e);
        if (ENT) w2 = fma2(e, t, w2);
      }
    }
    float u, v, y, z;
    unpack2(s2, u, v);
    unpack2(w2, y, z);
    if (ENT && y + z != y + z) {
#pragma unroll
      for (int k = 0; k < n; ++k) {
        float x[N];
        Vec<T>::unpack(q[k], x);
#pragma unroll
        for (int i = 0; i < N; ++i) take_one(x[i]);
      }
      return;
    }
    a.s = u + v;
    if (ENT) a.w = y + z;
  };

  if (live) {
    const T* xr = reinterpret_cast<const T*>(p.x) + row * p.ld;
    // whole vectors of the row, which start on 16 bytes, and the values before and behind them; this CTA's vectors: [v0, v1)
    const int head = (int)(((16u - (uint32_t)(reinterpret_cast<uintptr_t>(xr) & 15u)) & 15u) / sizeof(T));
    const int first = head < p.V ? head : p.V;
    const int nvec = (p.V - first) / N;
    const int per = (nvec + cluster - 1) / cluster;
    const int v0 = min(rank * per, nvec), v1 = min(v0 + per, nvec);
    const uint4* xv = reinterpret_cast<const uint4*>(xr + first);
    const int tail0 = first + nvec * N;
    auto scalar = [&](int i, bool in) {                // one value per lane (loose ends)
      const float v = in ? Vec<T>::one(xr[i]) : -INFINITY;
      if (in) {
        raise(v);
        take_one(v);
      }
      return v;
    };
    float lead = 0.f, rear = 0.f;
    const bool has_lead = wl == 0 && rank == 0, has_rear = wl == WARPS - 1 && rank == cluster - 1;
    if (has_lead) lead = scalar(lane, lane < first);
    constexpr int STEP = WARPS * 32;
    int v = v0 + wl * 32 + lane;
    for (; v + (U - 1) * STEP < v1; v += STEP * U) {
      uint4 q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) q[u] = ALTS ? __ldcg(xv + v + u * STEP) : __ldcs(xv + v + u * STEP);      // (some are read again: from L2)
      take(q);
    }
    uint4 last[U - 1];                                 // what is left, in flight together
#pragma unroll
    for (int u = 0; u < U - 1; ++u)
      if (v + u * STEP < v1) last[u] = ALTS ? __ldcg(xv + v + u * STEP) : __ldcs(xv + v + u * STEP);
#pragma unroll
    for (int u = 0; u < U - 1; ++u)
      if (v + u * STEP < v1) {
        const uint4 q[1] = {last[u]};
        take(q);
      }
    if (has_rear) rear = scalar(tail0 + lane, tail0 + lane < p.V);
    if (ALTS) {
      constexpr int kRowThreads = WARPS * 32;
      const uint32_t mine = any ? order_bits(top) : 0u;        // 0: nothing that is a number
      s_top[threadIdx.x] = mine;
      if (tid == 0) {
        *count = 0;
        s_hots[rh] = 0;
        s_floor[rh] = 0xffffffffu;
      }
      row_sync();
      int larger = 0;
      const uint4* tops = reinterpret_cast<const uint4*>(s_top + rh * kRowThreads);
#pragma unroll 8
      for (int i = 0; i < kRowThreads / 4; ++i) {
        const uint4 t = tops[i];
        larger += (t.x > mine) + (t.y > mine) + (t.z > mine) + (t.w > mine);
      }
      if (larger < p.n_alts) {                                 // ties at the floor all count
        s_hot[rh * kRowThreads + atomicAdd(&s_hots[rh], 1)] = (uint8_t)tid;
        atomicMin(&s_floor[rh], mine);
      }
      row_sync();
      const uint32_t kth = s_floor[rh];
      const float floor_value = kth == 0u ? NAN : order_value(kth);      // (nothing is less than a NaN: all go on to their keys)
      auto gather = [&](bool in, float v, uint32_t index) {
        if (in && !(v < floor_value)) {
          const int at = atomicAdd(count, 1);
          if (at < kRoom) keys[at] = make_key(v, index);
        }
      };
      // f(in, value, index) for every value that may reach the floor, all lanes at once
      auto for_hot = [&](auto&& f) {
        if (has_lead) f(lane < first, lead, (uint32_t)lane);
        if (has_rear) f(tail0 + lane < p.V, rear, (uint32_t)(tail0 + lane));
        const int hots = s_hots[rh];
        for (int h = wl; h < hots; h += WARPS) {       // the vectors of one thread, a lane each
          for (int v = v0 + s_hot[rh * kRowThreads + h]; v < v1; v += STEP * 64) {
            uint4 q[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const int at = v + STEP * (lane + 32 * y);
              q[y] = at < v1 ? __ldcg(xv + at) : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              if (v + STEP * 32 * y >= v1) continue;   // the same in all lanes
              const int at = v + STEP * (lane + 32 * y);
              float x[N];
              Vec<T>::unpack(q[y], x);
#pragma unroll
              for (int i = 0; i < N; ++i) f(at < v1, x[i], (uint32_t)(first + at * N + i));
            }
          }
        }
      };
      for_hot(gather);
      row_sync();
      if (*count > kRoom) {                            // the same in all threads of the row
        WarpBest best{0ull};
        unsigned long long floor_key = kth == 0u ? 0ull : ((unsigned long long)kth << 32) - 1ull;
        for_hot([&](bool in, float v, uint32_t index) {
          if (__any_sync(0xffffffffu, in && !(v < floor_value))) best.insert(in, make_key(v, index), p.n_alts, floor_key, lane);
        });
        row_sync();
        if (lane < p.n_alts) keys[wl * p.n_alts + lane] = best.key;
        if (tid == 0) *count = WARPS * p.n_alts;
        row_sync();
      }
    }
  }

  // join the lanes, then the warps of the row, then the CTAs of the cluster
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Part b{__shfl_xor_sync(0xffffffffu, a.r, o), __shfl_xor_sync(0xffffffffu, a.s, o),
                 __shfl_xor_sync(0xffffffffu, a.w, o)};
    a = lane & o ? join(b, a, c) : join(a, b, c);            // the same order in both lanes
  }
  // every warp joins the parts of the row's warps
  auto join_parts = [&](const Part* parts, int n) {
    Part b = lane < n ? parts[lane] : Part{-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
      const Part d{__shfl_xor_sync(0xffffffffu, b.r, o), __shfl_xor_sync(0xffffffffu, b.s, o),
                   __shfl_xor_sync(0xffffffffu, b.w, o)};
      b = lane & o ? join(d, b, c) : join(b, d, c);
    }
    return Part{__shfl_sync(0xffffffffu, b.r, 0), __shfl_sync(0xffffffffu, b.s, 0), __shfl_sync(0xffffffffu, b.w, 0)};
  };
  // f(place, key) for the n best of m keys (0: none); no two are equal
  auto for_best = [&](const unsigned long long* k, int m, auto&& f) {
    for (int i = tid; i < m; i += WARPS * 32) {
      const unsigned long long mine = k[i];
      int place = 0;
#pragma unroll 4
      for (int j = 0; j < m; ++j) place += k[j] > mine;
      if (mine != 0ull && place < p.n_alts) f(place, mine);
    }
  };
  static_assert(kWarps <= 8 && kMaxCluster <= 8, "three rounds join the parts");
  const unsigned long long* found = keys;
  int n_found = ALTS && live ? *count : 0;
  if (WARPS > 1) {
    if (lane == 0) s_part[warp] = a;
    __syncthreads();
    a = join_parts(s_part, kWarps);
    if (cluster > 1) {
      asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
      if (threadIdx.x == 0) {
        uint32_t dst = (uint32_t)__cvta_generic_to_shared(&s_all[rank]);
        asm volatile("mapa.shared::cluster.u32 %0, %0, 0;" : "+r"(dst));
        asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0+4], %2;\n\t"
                     "st.shared::cluster.f32 [%0+8], %3;" ::"r"(dst), "f"(a.r), "f"(a.s), "f"(a.w) : "memory");
      }
      if (ALTS)
        for_best(found, n_found, [&](int place, unsigned long long key) {
          uint32_t dst = (uint32_t)__cvta_generic_to_shared(&s_all_best[rank * SP_MAX_ALTS + place]);
          asm volatile("mapa.shared::cluster.u32 %0, %0, 0;" : "+r"(dst));
          asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(dst), "l"(key) : "memory");
        });
      asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
      if (rank != 0) return;
      a = join_parts(s_all, cluster);
      found = s_all_best;
      n_found = cluster * SP_MAX_ALTS;
    }
  }
  if (!live) return;
  // (all -infinity: s = 0, unless a NaN made it NaN)
  const bool none = a.r == -INFINITY && a.s == 0.f;
  const float r = a.r == -INFINITY ? 0.f : a.r;
  const float l2 = none ? -INFINITY : log2f(a.s);
  // (a logit of +infinity makes r infinite and s NaN)
  auto logp_of = [&](float x) { return none ? -INFINITY : kLn2 * ((x - r) * c - l2); };
  if (tid == 0) {
    if (p.lse) p.lse[row] = none ? -INFINITY : fmaf(p.scale, r, kLn2 * l2);
    if (ENT && p.entropy) p.entropy[row] = none ? 0.f : kLn2 * (l2 - a.w / a.s);
    if (p.logp && p.targets) {
      const int64_t t = p.targets[row];
      float v = 0.f;
      if (t >= p.V) {
        v = NAN;
        report_status(p.status, SP_ERR_SHAPE, (int32_t)row, 0);
      } else if (t >= 0) {
        v = logp_of(Vec<T>::one(reinterpret_cast<const T*>(p.x)[row * p.ld + t]));
      }
      p.logp[row] = v;
    }
  }
  if (ALTS)
    for_best(found, n_found, [&](int place, unsigned long long key) {
      const int64_t o = row * p.n_alts + place;
      if (p.alt_ids) p.alt_ids[o] = (int32_t)~(uint32_t)key;
      if (p.alt_logp) p.alt_logp[o] = logp_of(order_value((uint32_t)(key >> 32)));
    });
}

struct GradParams {
  const void* x;
  void* d;
  int64_t ld_x, ld_d, T;
  int32_t V, chunks;
  float scale;
  const int64_t* targets;
  const float* lse;
  const float* entropy;
  const float* g_logp;
  const float* g_entropy;
};
constexpr int kGradVecs = 4;       // vectors of 16 bytes per thread

// p = e^(scale x - lse) is off by a factor that lse's own rounding gives, 2^-24 |lse|.  Where a row's logits lie far from zero that is all of p: in
// a row of nothing but the type's lowest value log V is lost beside it in lse, so that p = 1, and with a scale above 1 lse overflows.  From kFarLse on
// (2^-14 there, a 64th of the rounding to bf16) one block of the row takes its largest logit r and the sum s of 2^(c (x - r)) again, c = log2(e) scale, and has
// log2 p = c (x - r) - log2 s, the difference before the product.  The row's other blocks leave at once, since the result may be written over the
// logits.  Two more reads, value by value, and one block for a row, so not for all rows: 4096 x 128256 in bf16 takes 305 us
// without far rows, 448 with one in 64, 1519 with nothing else; 100 x 50257 in fp32 12, 43, 54.
constexpr float kFarLse = 1024.f;
struct FarRow {
  float r, l2;                     // largest logit, log2 s; none: nothing but -infinity
  bool none;
};
template <typename T>
__device__ __noinline__ FarRow far_row(const T* xr, int V, float c) {
  __shared__ float s_r[kLossThreads / 32], s_s[kLossThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float r = -INFINITY, s = 0.f;
#pragma unroll 8
  for (int i = threadIdx.x; i < V; i += kLossThreads) r = fmaxf(r, Vec<T>::one(xr[i]));      // (NaN passed over: it comes in through the sum)
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) r = fmaxf(r, __shfl_xor_sync(0xffffffffu, r, o));
  if (lane == 0) s_r[warp] = r;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kLossThreads / 32; ++w) r = fmaxf(r, s_r[w]);
  const float ref = r == -INFINITY ? 0.f : r;
#pragma unroll 8
  for (int i = threadIdx.x; i < V; i += kLossThreads) s += exp2_fast((Vec<T>::one(xr[i]) - ref) * c);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) s_s[warp] = s;
  __syncthreads();                 // (the whole row has been read, too)
  s = 0.f;
#pragma unroll
  for (int w = 0; w < kLossThreads / 32; ++w) s += s_s[w];
  return FarRow{ref, s == 0.f ? 0.f : log2f(s), s == 0.f};
}

// d_v = p_v (A + B u_v) + (v == target) scale g,  u = scale x - lse = log p,  A = -scale (g + h H), B = -scale h.
// One read and one write of the row: 8 elementary operations per value, bound by DRAM.
template <typename T>
__global__ void __launch_bounds__(kLossThreads) token_logprobs_grad_kernel(const GradParams p) {
  kernel_begin();
  constexpr int N = Vec<T>::N;
  const int64_t row = blockIdx.x / p.chunks;
  const int chunk = (int)(blockIdx.x % p.chunks);
  const T* xr = reinterpret_cast<const T*>(p.x) + row * p.ld_x;
  T* dr = reinterpret_cast<T*>(p.d) + row * p.ld_d;
  const int64_t target64 = p.targets ? p.targets[row] : -1;
  const int target = target64 >= 0 && target64 < p.V ? (int)target64 : -1;
  const float lse = p.lse[row];
  const float g = target >= 0 && p.g_logp ? p.g_logp[row] : 0.f;
  float A = -p.scale * g, B = 0.f;
  if (p.g_entropy) {
    const float h = p.g_entropy[row];
    A = -p.scale * fmaf(h, p.entropy[row], g);
    B = -p.scale * h;
  }
  const float add = p.scale * g;
  if (!(fabsf(lse) < kFarLse)) {                         // (infinite or NaN, too)
    if (chunk != 0) return;
    const float c = p.scale * kLog2E;
    const FarRow f = far_row(xr, p.V, c);
#pragma unroll 8
    for (int i = threadIdx.x; i < p.V; i += kLossThreads) {
      const float t = fmaf(Vec<T>::one(xr[i]) - f.r, c, -f.l2);
      const float d = exp2_fast(t) * fmaf(B, fmaxf(t * kLn2, -10000.f), A) + (i == target ? add : 0.f);
      dr[i] = Vec<T>::to(f.none ? 0.f : d);
    }
    return;
  }
  auto one = [&](float x) {
    const float u = fmaf(x, p.scale, -lse);
    return exp2_fast(u * kLog2E) * fmaf(B, fmaxf(u, -10000.f), A);
  };
  const uint32_t phase = (uint32_t)(reinterpret_cast<uintptr_t>(xr) & 15u);
  const bool same = phase == (uint32_t)(reinterpret_cast<uintptr_t>(dr) & 15u);
  const int head = same ? (int)(((16u - phase) & 15u) / sizeof(T)) : p.V;     // rows of two phases go value by value
  const int first = head < p.V ? head : p.V;
  constexpr int kPer = kLossThreads * kGradVecs;
  if (same) {
    const int nvec = (p.V - first) / N;
    uint4 q[kGradVecs];
#pragma unroll
    for (int i = 0; i < kGradVecs; ++i) {
      const int v = chunk * kPer + i * kLossThreads + (int)threadIdx.x;
      if (v < nvec) q[i] = __ldcs(reinterpret_cast<const uint4*>(xr + first) + v);
    }
#pragma unroll
    for (int i = 0; i < kGradVecs; ++i) {
      const int v = chunk * kPer + i * kLossThreads + (int)threadIdx.x;
      if (v < nvec) {
        float x[N];
        Vec<T>::unpack(q[i], x);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          x[j] = one(x[j]);
          if (first + v * N + j == target) x[j] += add;
        }
        __stcs(reinterpret_cast<uint4*>(dr + first) + v, Vec<T>::pack(x));
      }
    }
    if (chunk == 0) {
      const int loose = first + (p.V - first) % N;       // before the first and behind the last vector
      for (int i = threadIdx.x; i < loose; i += kLossThreads) {
        const int at = i < first ? i : first + nvec * N + (i - first);
        dr[at] = Vec<T>::to(one(Vec<T>::one(xr[at])) + (at == target ? add : 0.f));
      }
    }
  } else {
    const int lo = chunk * kPer * N;
    for (int i = lo + (int)threadIdx.x; i < p.V && i < lo + kPer * N; i += kLossThreads)
      dr[i] = Vec<T>::to(one(Vec<T>::one(xr[i])) + (i == target ? add : 0.f));
  }
}

template <typename T, int WARPS>
cudaError_t launch_logprobs(const LogprobParams& p, int cluster, cudaStream_t stream) {
  const bool ent = p.entropy != nullptr, alts = p.n_alts > 0;
  const auto kernel = ent ? (alts ? token_logprobs_kernel<T, WARPS, true, true> : token_logprobs_kernel<T, WARPS, true, false>)
                          : (alts ? token_logprobs_kernel<T, WARPS, false, true> : token_logprobs_kernel<T, WARPS, false, false>);
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)cluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  const int64_t blocks = WARPS == 1 ? ceil_div(p.T, (int64_t)kLossThreads / 32) : p.T * cluster;
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(loss_threads(WARPS));
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = cluster > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, p, cluster);
}

bool scale_fits(double v) { return v >= 1e-30 && v <= 1e30; }

}  // namespace
}  // namespace sp

extern "C" {

sp_status sp_token_logprobs(const sp_mat* logits, const int64_t* targets, double scale, int32_t n_alts, float* logp,
                            float* lse, float* entropy, int32_t* alt_ids, float* alt_logp, int32_t* status_dev,
                            void* stream) {
  using namespace sp;
  if (!logits) return SP_ERR_INVALID_ARG;
  if (logits->dtype != SP_F32 && logits->dtype != SP_BF16) return SP_ERR_DTYPE;
  const int64_t T = logits->rows, V = logits->cols;
  if (T < 0 || V < 0 || V > (1 << 30) || (T > 1 && logits->ld < V)) return SP_ERR_SHAPE;
  if (n_alts < 0 || n_alts > SP_MAX_ALTS || n_alts > V) return SP_ERR_SHAPE;
  if (!scale_fits(scale)) return SP_ERR_INVALID_ARG;
  if (n_alts > 0 ? !alt_ids && !alt_logp : alt_ids != nullptr || alt_logp != nullptr) return SP_ERR_INVALID_ARG;
  if (logp && !targets) return SP_ERR_INVALID_ARG;
  if (!logp && !lse && !entropy && n_alts == 0) return SP_ERR_INVALID_ARG;
  if (T == 0) return SP_OK;
  if (V < 1 || T * kMaxCluster > 0x7fffffff) return SP_ERR_SHAPE;
  if (!logits->ptr) return SP_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const LogprobParams p{logits->ptr, logits->ld, T, (int32_t)V, n_alts, (float)scale, targets, logp, lse, entropy,
                        alt_ids, alt_logp, status_dev};
  // Short rows: a warp each.  Long ones: a block of four warps, so that the rows of an SM are many and at different places (8192 x 50257, warps
  // per row 8 / 4: 182 / 161 us, with eight alternatives 245 / 229), or a cluster of blocks while there are too few rows to fill the SMs.
  // Border of the short rows at 2048 / here, us: 4096 x 2500 25 / 14, 8192 x 3000 in fp32 43 / 29; here / at 8192: 4096 x 6000 29 / 23, with five
  // alternatives 43 / 29 (this border could lie higher).  Two / four / eight blocks for an SM: 100 x 50257 in fp32 21 / 17 / 16, 64 x 32000 with five
  // alternatives 16 / 25 / 25, 300 x 32000 equal.  Least values of a block 1024 / 2048 / 4096: equal within 2 us but 64 x 32000 with five (25, 25, 16).
  const bool narrow = V <= 4096;
  int cluster = 1;
  while (!narrow && cluster < kMaxCluster && T * cluster * 2 <= (int64_t)sm_count() * 4 && V / (cluster * 2) >= 2048) cluster *= 2;
  count_launch();
  ProfScope prof(PK_SCORES, 0.0, (double)T * V * dtype_size(logits->dtype), s);
  const auto run = [&](auto type) {
    using E = decltype(type);
    return narrow ? launch_logprobs<E, 1>(p, 1, s) : launch_logprobs<E, 4>(p, cluster, s);
  };
  const cudaError_t e = logits->dtype == SP_F32 ? run(float()) : run(__nv_bfloat16());
  return e == cudaSuccess ? SP_OK : SP_ERR_CUDA;
}

sp_status sp_token_logprobs_grad(const sp_mat* logits, const int64_t* targets, double scale, const float* lse,
                                 const float* entropy, const float* g_logp, const float* g_entropy,
                                 const sp_mat* dlogits, void* stream) {
  using namespace sp;
  if (!logits || !dlogits) return SP_ERR_INVALID_ARG;
  if ((logits->dtype != SP_F32 && logits->dtype != SP_BF16) || dlogits->dtype != logits->dtype) return SP_ERR_DTYPE;
  const int64_t T = logits->rows, V = logits->cols;
  if (T < 0 || V < 0 || V > (1 << 30) || (T > 1 && (logits->ld < V || dlogits->ld < V))) return SP_ERR_SHAPE;
  if (dlogits->rows != T || dlogits->cols != V) return SP_ERR_SHAPE;
  if (!scale_fits(scale) || (!g_logp && !g_entropy)) return SP_ERR_INVALID_ARG;
  if (T == 0) return SP_OK;
  const int n = 16 / (int)dtype_size(logits->dtype);
  const int64_t chunks = ceil_div(ceil_div(V, (int64_t)n), (int64_t)kLossThreads * kGradVecs);
  if (V < 1 || T > 0x7fffffff || T * chunks > 0x7fffffff) return SP_ERR_SHAPE;
  if (!logits->ptr || !dlogits->ptr || !lse || (g_logp && !targets) || (g_entropy && !entropy)) return SP_ERR_INVALID_ARG;
  // the same values at another pitch would be overwritten before they are read
  if (logits->ptr == dlogits->ptr && T > 1 && logits->ld != dlogits->ld) return SP_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const GradParams p{logits->ptr, dlogits->ptr, logits->ld, dlogits->ld, T, (int32_t)V, (int32_t)chunks, (float)scale,
                     targets, lse, entropy, g_logp, g_entropy};
  count_launch();
  ProfScope prof(PK_ELEMENTWISE, 0.0, 2.0 * T * V * dtype_size(logits->dtype), s);
  const dim3 grid((unsigned)(T * chunks));
  const cudaError_t e = logits->dtype == SP_F32
                            ? launch(token_logprobs_grad_kernel<float>, grid, dim3(kLossThreads), 0, s, p)
                            : launch(token_logprobs_grad_kernel<__nv_bfloat16>, grid, dim3(kLossThreads), 0, s, p);
  return e == cudaSuccess ? SP_OK : SP_ERR_CUDA;
}

}  // extern "C"
