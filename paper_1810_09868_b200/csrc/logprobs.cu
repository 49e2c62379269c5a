// Log probabilities of given classes, log-sum-exp, entropy and the top alternatives of rows of logits, and their
// gradient.  For a row z of n logits
//   lse = log sum_j exp(z_j),   log p_j = z_j - lse,   H = -sum_j p_j log p_j,
//   d(sum_i g_i log p[id_i] + w H) / dz_j = sum_i g_i [j = id_i] - p_j (sum_i g_i + w (log p_j + H)).
//
// Both directions are bound by reading the logits (and writing the gradient) once.  The forward kernel makes one
// pass: every thread keeps a reference `ref` (a value near the largest it has seen), S = sum exp(z - ref) and
// U = sum exp(z - ref) (z - ref), in fp32, and at the end H = log S - U / S, lse = ref + log S.  Issue slots are what it
// has to save (bf16 at the memory's rate leaves 11 instructions a logit): exponents and sums go two at a time
// (f32x2), the reference is looked at once per 16 logits.
//
// The top alternatives cost that pass one maximum per thread.  A value that at least top_k of the threads' maxima
// reach (found by bisection) is reached by top_k logits; only the threads whose maximum reaches it, about top_k, read
// their logits again and sort those that do, as 64-bit keys (value, then lower index).  Keeping a sorted list during
// the pass instead took twice the time for the best 8 of 50021.
//
// A short row (up to 1024 classes) belongs to one warp, a longer one to one block, or, where there are fewer rows than the
// GPU has room for, to a cluster of up to eight blocks that join through distributed shared memory: one launch, no
// scratch, and an order of summation that depends on the sizes alone.
//
// Measured (B200, device time): 2048 rows of 50021 fp32 with the best 8 in 80 us, 5.1 TB/s (0.80 of a copy's rate; without a
// top list 66 us, 0.97); 4096 rows of 32003 bf16 forward in 54 us and the gradient in 83 us (4.9 and 6.3 TB/s); one row of
// 131072 bf16 with the best 20 in 8.2 us, of 1000 fp32 with the best 5 in 3.4 us, all latency.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "../../include/vgg19_b200.h"
#include "common.cuh"

namespace cg = cooperative_groups;

namespace vgg {
namespace {

static __device__ int g_logprobs_error[1];  // kDevBadLabel once an id outside [0, classes) was met

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// A reference moves only when a value exceeds it by this much (natural units): exp(z - ref) then stays below e^4, and
// the moves stay rare after the first vectors.
constexpr float kRefMargin = 4.f;
constexpr float kFloor = -200.f;  // exp2 of anything lower is 0 in fp32; keeps 0 * (-inf) out of U
constexpr int kMaxTop = VGG19_LOGPROBS_MAX_TOP, kMaxIds = VGG19_LOGPROBS_MAX_IDS;

__device__ __forceinline__ float max_nan(float a, float b) {  // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float fast_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// values ordered as unsigned integers; -0 counts as 0
__device__ __forceinline__ unsigned ordered(float v) {
  const int b = __float_as_int(v + 0.f);
  return b < 0 ? ~(unsigned)b : (unsigned)b | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned o) { return __int_as_float((int)(o & 0x80000000u ? o & 0x7fffffffu : ~o)); }
constexpr unsigned kLowest = 0x00800000u;  // ordered(lowest finite value)
__device__ __forceinline__ unsigned long long make_key(float v, unsigned index) {
  return ((unsigned long long)ordered(v) << 32) | (0xffffffffu - index);
}
__device__ __forceinline__ float key_value(unsigned long long k) { return value_of((unsigned)(k >> 32)); }
__device__ __forceinline__ unsigned key_index(unsigned long long k) { return 0xffffffffu - (unsigned)k; }

// 16 bytes of logits as floats
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  __device__ static void unpack(const uint4& w, float* x) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
  }
  __device__ static uint4 pack(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
  static constexpr unsigned kMinusInf = 0xff800000u;
};
template <> struct Vec<bf16> {
  static constexpr int N = 8;
  __device__ static void unpack(const uint4& w, float* x) {
    const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  __device__ static uint4 pack(const float* x) {
    unsigned u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      u[i] = *reinterpret_cast<const unsigned*>(&b);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
  static constexpr unsigned kMinusInf = 0xff80ff80u;
};

// A row as [head | whole 16-byte vectors | tail]: rows of an odd number of classes start anywhere.
template <typename T> struct RowSplit {
  int head, nvec, tail;
  __device__ RowSplit(const T* row, int n) {
    constexpr int V = Vec<T>::N;
    head = (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(T);
    if (head > n) head = n;
    nvec = (n - head) / V;
    tail = n - head - nvec * V;
  }
};

struct Sums {  // of a set of logits: reference, sum of exp, sum of exp times its exponent in base 2
  float ref, S, U;
};
// A thread's sums over the logits it has seen, and the largest of them.
struct Scan {
  float ref = -INFINITY, r = 0.f, top = -INFINITY;  // r: ref, but 0 while that is -inf, when every exponent is -inf anyway
  f32x2 S = 0, U = 0;                               // (the bits of two zeros)

  template <int N> __device__ __forceinline__ void add(const float (&x)[N]) {
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) mx = fmaxf(mx, x[e]);
    top = fmaxf(top, mx);
    if (mx > ref + kRefMargin) {
      if (ref != -INFINITY) {
        const float d = (ref - mx) * kLog2e, f = fast_exp2(d);
        const f32x2 dd = pack2(d, d), ff = pack2(f, f);
        U = f > 0.f ? mul2(fma2(dd, S, U), ff) : mul2(U, ff);
        S = mul2(S, ff);
      }
      ref = r = mx;
    }
    const f32x2 minus = pack2(-r, -r), log2e = pack2(kLog2e, kLog2e);
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      float a, b;
      unpack2(mul2(add2(pack2(x[e], e + 1 < N ? x[e + 1] : -INFINITY), minus), log2e), a, b);
      a = max_nan(a, kFloor);
      b = max_nan(b, kFloor);
      const f32x2 p = pack2(fast_exp2(a), fast_exp2(b));
      S = add2(S, p);
      U = fma2(p, pack2(a, b), U);
    }
  }
};

// The sums of a warp's lanes (lanes without any have ref = -inf, S = U = 0), in every lane.
__device__ __forceinline__ Sums lanes_join(Sums a) {
  float m = a.ref;
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float d = a.ref == m ? 0.f : (a.ref - m) * kLog2e, f = fast_exp2(d);
  float S = a.S * f, U = f > 0.f ? (a.U + d * a.S) * f : a.U * 0.f;  // a vanished part would bring -inf * 0
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    S += __shfl_xor_sync(0xffffffffu, S, o);
    U += __shfl_xor_sync(0xffffffffu, U, o);
  }
  return Sums{m, S, U};
}

// A warp's best keys, sorted over its lanes, largest first; 0 for none.
struct Best {
  unsigned long long key = 0;
  // The elements of the lanes' x that are at least thr.  Where there are many, as in a row of equals, they have to be better than
  // the last place wanted first (512 rows of 50021 equals, the best 5: 738 us without that, 70 with it).
  template <int N, typename Index> __device__ __forceinline__ void add(const float (&x)[N], float thr, int top_k, Index index) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      unsigned hits = __ballot_sync(0xffffffffu, x[e] >= thr);
      if (!hits) continue;
      const unsigned long long mine = make_key(x[e], index(e));
      if (__popc(hits) > 4) {  // (of the whole warp)
        const unsigned long long last = __shfl_sync(0xffffffffu, key, top_k - 1);
        hits = __ballot_sync(0xffffffffu, x[e] >= thr && mine > last);
      }
      while (hits) {
        const unsigned long long c = __shfl_sync(0xffffffffu, mine, __ffs(hits) - 1), up = __shfl_up_sync(0xffffffffu, key, 1);
        hits &= hits - 1;
        if (c > key) key = lane > 0 && c > up ? up : c;
      }
    }
  }
};

__device__ __forceinline__ float lane_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The best top_k of `n` keys in shared memory (distinct, 0 = none), sorted, by counting for each how many are larger.
__device__ __forceinline__ void rank_keys(const unsigned long long* keys, int n, int top_k, unsigned long long* out) {
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const unsigned long long k = keys[i];
    if (!k) continue;
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += keys[j] > k;
    if (rank < top_k) out[rank] = k;
  }
}

struct FwdArgs {
  const void* logits;
  const int32_t* ids;
  float *logprob, *lse, *entropy, *top_logprob;
  int32_t* top_id;
  long ld;
  int classes, n_ids, top_k;
};

constexpr int kMaxCluster = 8;

template <typename T, int NT, int UNROLL>
__global__ void __launch_bounds__(NT) logprobs_kernel(const FwdArgs a) {
  constexpr int V = Vec<T>::N, W = NT / 32, GROUP = 16 / V;  // vectors a look at the reference
  static_assert(UNROLL % GROUP == 0 && W <= 32 && kMaxCluster <= 32, "whole groups; a warp joins all parts");
  __shared__ Sums part[W];
  __shared__ unsigned low[W], high[W];
  __shared__ unsigned long long keys[W * kMaxTop], best[kMaxTop];
  __shared__ int n_keys;
  __shared__ Sums cpart[kMaxCluster];                             // of the cluster's blocks, in its first
  __shared__ unsigned long long ckeys[kMaxCluster * kMaxTop];
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  if (C > 1) cluster.barrier_arrive();  // waited for before the first write into the first block's shared memory
  const long row = blockIdx.x / C;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  const RowSplit<T> sp(z, a.classes);
  const uint4* body = reinterpret_cast<const uint4*>(z + sp.head);
  const int v0 = (int)((long)sp.nvec * rank / C), v1 = (int)((long)sp.nvec * (rank + 1) / C);
  if (tid == 0) n_keys = 0;

  // thread t has the vectors v0 + t, v0 + t + NT, ...
  Scan w;
  const uint4 none = make_uint4(Vec<T>::kMinusInf, Vec<T>::kMinusInf, Vec<T>::kMinusInf, Vec<T>::kMinusInf);
  for (int base = v0 + tid; base < v1; base += NT * UNROLL) {
    uint4 r[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) r[u] = base + u * NT < v1 ? __ldg(body + base + u * NT) : none;
#pragma unroll
    for (int u = 0; u < UNROLL; u += GROUP) {
      float x[16];
#pragma unroll
      for (int g = 0; g < GROUP; ++g) Vec<T>::unpack(r[u + g], x + g * V);
      w.add(x);
    }
  }
  const float top = w.top;
  // the logits before and behind the vectors: one a lane of the first warp
  int at = -1;
  float edge[1] = {-INFINITY};
  if (rank == 0 && warp == 0 && sp.head + sp.tail > 0) {
    const int t = lane - 8;  // lanes 0..7 the head, 8..15 the tail
    at = lane < sp.head ? lane : t >= 0 && t < sp.tail ? sp.head + sp.nvec * V + t : -1;
    if (at >= 0) edge[0] = to_f32(z[at]);
    w.add(edge);
  }
  {
    Sums s{w.ref, 0.f, 0.f};
    float b;
    unpack2(w.S, s.S, b); s.S += b;
    unpack2(w.U, s.U, b); s.U += b;
    s = lanes_join(s);
    if (lane == 0) part[warp] = s;
  }

  if (a.top_k) {
    // a bound that at least top_k of the threads' maxima reach, and few more
    const unsigned mine = ordered(top);
    const unsigned mn = __reduce_min_sync(0xffffffffu, mine), mx = __reduce_max_sync(0xffffffffu, mine);
    if (lane == 0) { low[warp] = mn; high[warp] = mx; }
    const int finite = __syncthreads_count(mine >= kLowest);
    unsigned lo = kLowest;
    if (finite > a.top_k) {
      unsigned hi = 0, least = 0xffffffffu;
      for (int i = 0; i < W; ++i) { hi = max(hi, high[i]); least = min(least, low[i]); }
      if (least > lo) lo = least;
      // invariant: top_k maxima reach lo; fewer reach hi + 1
      while (lo < hi) {
        const unsigned mid = lo + (hi - lo + 1) / 2;
        const int n = __syncthreads_count(mine >= mid);
        if (n >= a.top_k) lo = mid; else hi = mid - 1;
        if (n >= a.top_k && n <= a.top_k + a.top_k / 4) break;
      }
    }
    const float thr = value_of(lo);
    Best b;
    unsigned hot = __ballot_sync(0xffffffffu, mine >= lo);
    // The lanes share the vectors of each thread whose maximum reaches the bound, one thread after another, or, where a thread
    // has few, several at once: `share` lanes to a thread's.  (700 rows of 1467, the best 31: 13.5 -> 9.5 us; with many vectors
    // a thread the first loop is the faster one, 61 against 67 us for 2048 rows of 50021.)
    const int each = (v1 - v0 + NT - 1) / NT;
    if (each > 16) {
      while (hot) {
        const int t = warp * 32 + __ffs(hot) - 1;
        hot &= hot - 1;
        for (int v = v0 + t; v < v1; v += 32 * NT) {
          const int u = v + lane * NT;
          float x[V];
          Vec<T>::unpack(u < v1 ? __ldg(body + u) : none, x);
          const int first = sp.head + u * V;
          b.add(x, thr, a.top_k, [first](int e) { return (unsigned)(first + e); });
        }
      }
    } else {
      const int share = each > 8 ? 16 : each > 4 ? 8 : 4;
      while (hot) {
        unsigned m = hot;  // without the threads of the lanes before these
        for (int j = 0; j < 32 / share; ++j) {
          if (j < lane / share) m &= m - 1;
          hot &= hot - 1;
        }
        const int k = lane % share, u = v0 + warp * 32 + __ffs(m) - 1 + k * NT;  // (m may be 0)
        float x[V];
        Vec<T>::unpack(m && k < each && u < v1 ? __ldg(body + u) : none, x);
        const int first = sp.head + u * V;
        b.add(x, thr, a.top_k, [first](int e) { return (unsigned)(first + e); });
      }
    }
    if (rank == 0 && warp == 0) b.add(edge, thr, a.top_k, [at](int) { return (unsigned)at; });
    const bool have = lane < a.top_k && b.key != 0;
    const unsigned m = __ballot_sync(0xffffffffu, have);
    int to = 0;
    if (lane == 0 && m) to = atomicAdd(&n_keys, __popc(m));  // (their order does not matter)
    to = __shfl_sync(0xffffffffu, to, 0);
    if (have) keys[to + lane] = b.key;
    if (tid < a.top_k) best[tid] = 0;
    __syncthreads();
    rank_keys(keys, n_keys, a.top_k, best);
  }
  __syncthreads();
  if (warp != 0 && C == 1) return;
  Sums all = lanes_join(lane < W ? part[lane] : Sums{-INFINITY, 0.f, 0.f});
  if (C > 1) {
    cluster.barrier_wait();
    if (tid == 0) cluster.map_shared_rank(cpart, 0)[rank] = all;
    if (tid < a.top_k) cluster.map_shared_rank(ckeys, 0)[rank * a.top_k + tid] = best[tid];
    cluster.sync();
    if (rank != 0) return;
    all = lanes_join(lane < C ? cpart[lane] : Sums{-INFINITY, 0.f, 0.f});
    if (a.top_k) {
      if (tid < a.top_k) best[tid] = 0;
      __syncthreads();
      rank_keys(ckeys, C * a.top_k, a.top_k, best);
      __syncthreads();
    }
    if (warp != 0) return;
  }

  // (z - ref) - log S, not z - lse: lse is rounded to its own magnitude
  const bool bad = !(all.S == all.S) || all.ref == INFINITY, empty = !bad && all.ref == -INFINITY;
  const float nan = __int_as_float(0x7fc00000);
  const float logS = logf(all.S);
  if (lane == 0) {
    if (a.lse) a.lse[row] = bad ? nan : empty ? -INFINITY : all.ref + logS;
    if (a.entropy) a.entropy[row] = bad ? nan : empty ? 0.f : fmaxf(logS - kLn2 * (all.U / all.S), 0.f);
  }
  for (int i = lane; i < a.n_ids; i += 32) {
    const int id = a.ids[row * a.n_ids + i];
    float v = 0.f;
    if (id != VGG19_NO_CLASS) {
      if ((unsigned)id < (unsigned)a.classes) {
        v = bad ? nan : empty ? -INFINITY : (to_f32(z[id]) - all.ref) - logS;
      } else {  // never used as an index
        v = nan;
        atomicCAS(g_logprobs_error, 0, (int)kDevBadLabel);
      }
    }
    a.logprob[row * a.n_ids + i] = v;
  }
  if (lane < a.top_k) {
    const unsigned long long k = bad ? 0 : best[lane];
    a.top_id[row * a.top_k + lane] = k ? (int32_t)key_index(k) : VGG19_NO_CLASS;
    a.top_logprob[row * a.top_k + lane] = bad ? nan : k ? (key_value(k) - all.ref) - logS : -INFINITY;
  }
}

struct BwdArgs {
  const void* logits;
  void* d_logits;
  const int32_t* ids;
  const float *lse, *entropy, *d_logprob, *d_entropy;
  long ld, d_ld;
  int classes, n_ids, chunks;
};

// One block takes `chunk` vectors of one row.  Every warp finds the ids that fall into the chunk (usually none or one) by
// itself, lane by lane, and hands them round with shuffles, in their order: a class named twice gets both shares in the
// same order every time, every element is rounded and written once, no warp waits for another, and d_logits may be logits.
constexpr int kBwdThreads = 256, kBwdUnroll = 4;

template <typename T, bool MANY>  // MANY: more than 32 ids
__global__ void __launch_bounds__(kBwdThreads) logprobs_backward_kernel(const BwdArgs a) {
  constexpr int V = Vec<T>::N, IDS = kMaxIds / 32;
  const long row = blockIdx.x / a.chunks;
  const int chunk = (int)(blockIdx.x - row * a.chunks), tid = threadIdx.x, lane = tid & 31;
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  T* dz = static_cast<T*>(a.d_logits) + row * a.d_ld;
  const RowSplit<T> sp(z, a.classes);
  const bool same = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0;
  const uint4* body = reinterpret_cast<const uint4*>(z + sp.head);
  const int v0 = chunk * (kBwdThreads * kBwdUnroll);

  uint4 r[kBwdUnroll];
#pragma unroll
  for (int u = 0; u < kBwdUnroll; ++u) {
    const int v = v0 + u * kBwdThreads + tid;
    if (v < sp.nvec) r[u] = __ldcs(body + v);
  }
  // the elements this block writes: its vectors, and in the first block the head and the tail
  const int lo = sp.head + min(v0, sp.nvec) * V, hi = sp.head + min(v0 + kBwdThreads * kBwdUnroll, sp.nvec) * V;
  auto load_id = [&](int i, float& g, bool& mine) {
    const int id = i + lane < a.n_ids ? a.ids[row * a.n_ids + i + lane] : VGG19_NO_CLASS;
    const bool in = (unsigned)id < (unsigned)a.classes;
    if (!in && id != VGG19_NO_CLASS) atomicCAS(g_logprobs_error, 0, (int)kDevBadLabel);
    g = in ? a.d_logprob[row * a.n_ids + i + lane] : 0.f;
    mine = in && ((id >= lo && id < hi) || (chunk == 0 && (id < sp.head || id >= sp.head + sp.nvec * V)));
    return id;
  };
  // the first 32 ids stay in registers; which further ones are this block's, as a mask per 32
  float g0, sum;
  bool mine0;
  const int id0 = load_id(0, g0, mine0);
  const unsigned hits0 = __ballot_sync(0xffffffffu, mine0);
  sum = lane_sum(g0);
  unsigned more[IDS] = {};
  bool any_more = false;
  if (MANY) {
#pragma unroll
    for (int k = 1; k < IDS; ++k)
      if (k * 32 < a.n_ids) {
        float g;
        bool mine;
        load_id(k * 32, g, mine);
        more[k] = __ballot_sync(0xffffffffu, mine);
        any_more |= more[k] != 0;
        sum += lane_sum(g);
      }
  }
  const float lse = a.lse[row], w = a.d_entropy ? a.d_entropy[row] : 0.f;
  const float c = sum + (a.d_entropy ? w * a.entropy[row] : 0.f);
  const bool empty = lse == -INFINITY;  // a row with no class left has no gradient
  // f(id, g) for this block's ids, in order, called by whole warps
  auto each_hit = [&](auto f) {
    for (unsigned m = hits0; m; m &= m - 1) {
      const int l = __ffs(m) - 1;
      f(__shfl_sync(0xffffffffu, id0, l), __shfl_sync(0xffffffffu, g0, l));
    }
    if (MANY && any_more) {
#pragma unroll
      for (int k = 1; k < IDS; ++k)
        for (unsigned m = more[k]; m; m &= m - 1) {
          const long at = row * a.n_ids + k * 32 + __ffs(m) - 1;
          f(a.ids[at], a.d_logprob[at]);
        }
    }
  };
  const f32x2 minus = pack2(-lse, -lse), log2e = pack2(kLog2e, kLog2e), w2 = pack2(-w, -w), c2 = pack2(-c, -c);
#pragma unroll
  for (int u = 0; u < kBwdUnroll; ++u) {
    const int v = v0 + u * kBwdThreads + tid;
    if (v - lane >= sp.nvec) break;  // whole warps
    float x[V] = {};
    if (v < sp.nvec) Vec<T>::unpack(r[u], x);
    const int first = sp.head + v * V;
#pragma unroll
    for (int e = 0; e < V; e += 2) {
      float p, q;
      unpack2(add2(pack2(x[e], x[e + 1]), minus), p, q);
      const f32x2 lp = pack2(max_nan(p, kFloor), max_nan(q, kFloor));
      unpack2(mul2(lp, log2e), p, q);
      unpack2(mul2(pack2(fast_exp2(p), fast_exp2(q)), fma2(w2, lp, c2)), x[e], x[e + 1]);
    }
    if (empty) {
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = 0.f;
    } else {
      each_hit([&](int id, float g) {
        const int d = id - first;
        if ((unsigned)d < (unsigned)V) {
#pragma unroll
          for (int e = 0; e < V; ++e) x[e] += e == d ? g : 0.f;
        }
      });
    }
    if (v < sp.nvec) {
      if (same) {
        __stcs(reinterpret_cast<uint4*>(dz + first), Vec<T>::pack(x));
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) dz[first + e] = from_f32<T>(x[e]);
      }
    }
  }
  if (chunk == 0 && tid < 32 && sp.head + sp.tail > 0) {  // (at most 14 of them)
    const int at = lane < sp.head ? lane : lane < sp.head + sp.tail ? sp.nvec * V + lane : -1;
    float d = 0.f;
    if (at >= 0 && !empty) {
      const float lp = max_nan(to_f32(z[at]) - lse, kFloor);
      d = fast_exp2(lp * kLog2e) * fmaf(-w, lp, -c);
    }
    each_hit([&](int id, float g) { d += id == at && !empty ? g : 0.f; });
    if (at >= 0) dz[at] = from_f32<T>(d);
  }
}

// ---- short rows ------------------------------------------------------------------------------------------------
// A warp per row, its logits in registers (element e of a lane is class lane + 32 e): no thread waits for another warp, and
// no pass is repeated for the top list, which is taken one class after another from the lanes' best.
// Measured against the blocks above (B200): 2048 rows of 250, bf16, the best 32: 9.4 against 60 us, none: 2.5 against 6.3, gradient 2.8
// against 5.6; one row of 1000, fp32, the best 5: 3.6 against 4.2, the best 32: 10 against 6.4; 100 rows' gradient at 1000: 3.4
// against 2.0, 2048 rows': 4.0 against 5.6.
constexpr int kShortWarps = 4;
bool short_forward_wins(int classes, int top_k) { return classes <= 512 || (classes <= 1024 && top_k <= 8); }
bool short_backward_wins(int classes, long rows) { return classes <= 256 || (classes <= 1024 && rows >= 512); }

template <typename T, int P>
__global__ void __launch_bounds__(32 * kShortWarps) short_rows_kernel(const FwdArgs a, long rows) {
  const int lane = threadIdx.x & 31, n = a.classes;
  const long row = (long)blockIdx.x * kShortWarps + threadIdx.x / 32;
  if (row >= rows) return;
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  float x[P];
#pragma unroll
  for (int e = 0; e < P; ++e) x[e] = lane + 32 * e < n ? to_f32(z[lane + 32 * e]) : -INFINITY;
  float ref = x[0];
#pragma unroll
  for (int e = 1; e < P; ++e) ref = fmaxf(ref, x[e]);
#pragma unroll
  for (int o = 16; o; o >>= 1) ref = fmaxf(ref, __shfl_xor_sync(0xffffffffu, ref, o));  // (passes over NaN: S will be one)
  const float r = ref == -INFINITY ? 0.f : ref;
  float S = 0.f, U = 0.f;
#pragma unroll
  for (int e = 0; e < P; ++e) {
    const float d = max_nan((x[e] - r) * kLog2e, kFloor), p = fast_exp2(d);
    S += p;
    U = fmaf(p, d, U);
  }
  S = lane_sum(S);
  U = lane_sum(U);
  const bool bad = !(S == S) || ref == INFINITY, empty = !bad && ref == -INFINITY;
  const float nan = __int_as_float(0x7fc00000), logS = logf(S);
  if (lane == 0) {
    if (a.lse) a.lse[row] = bad ? nan : empty ? -INFINITY : ref + logS;
    if (a.entropy) a.entropy[row] = bad ? nan : empty ? 0.f : fmaxf(logS - kLn2 * (U / S), 0.f);
  }
  for (int i = lane; i < a.n_ids; i += 32) {
    const int id = a.ids[row * a.n_ids + i];
    float v = 0.f;
    if (id != VGG19_NO_CLASS) {
      if ((unsigned)id < (unsigned)n) {
        v = bad ? nan : empty ? -INFINITY : (to_f32(z[id]) - ref) - logS;
      } else {  // never used as an index
        v = nan;
        atomicCAS(g_logprobs_error, 0, (int)kDevBadLabel);
      }
    }
    a.logprob[row * a.n_ids + i] = v;
  }
  if (!a.top_k) return;
  unsigned left[P], mine = 0;  // what the lane has not given yet, and the largest of it (the first among equals)
  int at = 0;
#pragma unroll
  for (int e = 0; e < P; ++e) left[e] = ordered(x[e]);
  auto look = [&] {
    mine = left[0];
    at = 0;
#pragma unroll
    for (int e = 1; e < P; ++e)
      if (left[e] > mine) { mine = left[e]; at = e; }
  };
  look();
  unsigned value = 0;
  int id = VGG19_NO_CLASS;  // of place `lane` in the list
  for (int k = 0; k < a.top_k && !bad; ++k) {
    const unsigned most = __reduce_max_sync(0xffffffffu, mine);
    if (most < kLowest) break;  // excluded classes only
    const unsigned index = mine == most ? lane + 32 * at : 0xffffffffu, first = __reduce_min_sync(0xffffffffu, index);
    if (lane == k) { value = most; id = (int)first; }
    if (index == first) {
#pragma unroll
      for (int e = 0; e < P; ++e)
        if (e == at) left[e] = 0;
      look();
    }
  }
  if (lane < a.top_k) {
    a.top_id[row * a.top_k + lane] = id;
    a.top_logprob[row * a.top_k + lane] = bad ? nan : id != VGG19_NO_CLASS ? (value_of(value) - ref) - logS : -INFINITY;
  }
}

template <typename T, int P>
__global__ void __launch_bounds__(32 * kShortWarps) short_rows_backward_kernel(const BwdArgs a, long rows) {
  const int lane = threadIdx.x & 31, n = a.classes;
  const long row = (long)blockIdx.x * kShortWarps + threadIdx.x / 32;
  if (row >= rows) return;
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  T* dz = static_cast<T*>(a.d_logits) + row * a.d_ld;
  float x[P], given[P];
#pragma unroll
  for (int e = 0; e < P; ++e) {
    x[e] = lane + 32 * e < n ? to_f32(z[lane + 32 * e]) : 0.f;
    given[e] = 0.f;
  }
  float sum = 0.f;
  for (int i = 0; i < a.n_ids; i += 32) {  // in their order
    const int id = i + lane < a.n_ids ? a.ids[row * a.n_ids + i + lane] : VGG19_NO_CLASS;
    const bool in = (unsigned)id < (unsigned)n;
    if (!in && id != VGG19_NO_CLASS) atomicCAS(g_logprobs_error, 0, (int)kDevBadLabel);
    const float g = in ? a.d_logprob[row * a.n_ids + i + lane] : 0.f;
    sum += lane_sum(g);
    for (unsigned m = __ballot_sync(0xffffffffu, in); m; m &= m - 1) {
      const int l = __ffs(m) - 1, d = __shfl_sync(0xffffffffu, id, l) - lane;
      const float v = __shfl_sync(0xffffffffu, g, l);
#pragma unroll
      for (int e = 0; e < P; ++e) given[e] += d == 32 * e ? v : 0.f;
    }
  }
  const float lse = a.lse[row], w = a.d_entropy ? a.d_entropy[row] : 0.f;
  const float c = sum + (a.d_entropy ? w * a.entropy[row] : 0.f);
  const bool empty = lse == -INFINITY;  // a row with no class left has no gradient
#pragma unroll
  for (int e = 0; e < P; ++e)
    if (lane + 32 * e < n) {
      const float lp = max_nan(x[e] - lse, kFloor);
      dz[lane + 32 * e] = from_f32<T>(empty ? 0.f : fmaf(fast_exp2(lp * kLog2e), fmaf(-w, lp, -c), given[e]));
    }
}

// How many blocks share a row: enough to give every SM two blocks while each still has a few thousand classes.
int cluster_size(long rows, int classes) {
  int c = 1;
  while (c < kMaxCluster && rows * c * 2 <= 296 && classes / (c * 2) >= 2048) c *= 2;
  return c;
}

template <typename T, int NT, int UNROLL> cudaError_t launch_forward(const FwdArgs& a, long rows, int C, cudaStream_t st) {
  if (C == 1) {
    logprobs_kernel<T, NT, UNROLL><<<(unsigned)rows, NT, 0, st>>>(a);
    return cudaGetLastError();
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(rows * C));
  cfg.blockDim = dim3(NT);
  cfg.stream = st;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = (unsigned)C;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, logprobs_kernel<T, NT, UNROLL>, a);
}

template <typename T, int P> cudaError_t short_forward(const FwdArgs& a, long rows, cudaStream_t st) {
  short_rows_kernel<T, P><<<(unsigned)((rows + kShortWarps - 1) / kShortWarps), 32 * kShortWarps, 0, st>>>(a, rows);
  return cudaGetLastError();
}
template <typename T, int P> cudaError_t short_backward(const BwdArgs& a, long rows, cudaStream_t st) {
  short_rows_backward_kernel<T, P><<<(unsigned)((rows + kShortWarps - 1) / kShortWarps), 32 * kShortWarps, 0, st>>>(a, rows);
  return cudaGetLastError();
}

template <typename T> cudaError_t forward(const FwdArgs& a, long rows, cudaStream_t st) {
  if (short_forward_wins(a.classes, a.top_k)) {
    if (a.classes <= 64) return short_forward<T, 2>(a, rows, st);
    if (a.classes <= 256) return short_forward<T, 8>(a, rows, st);
    if (a.classes <= 512) return short_forward<T, 16>(a, rows, st);
    return short_forward<T, 32>(a, rows, st);
  }
  const int C = cluster_size(rows, a.classes), per = a.classes / C;
  if (per <= 2048) return launch_forward<T, 128, 4>(a, rows, C, st);
  return launch_forward<T, 256, 4>(a, rows, C, st);
}

template <typename T> cudaError_t backward(const BwdArgs& a, long rows, cudaStream_t st) {
  if (short_backward_wins(a.classes, rows)) {
    if (a.classes <= 64) return short_backward<T, 2>(a, rows, st);
    if (a.classes <= 256) return short_backward<T, 8>(a, rows, st);
    if (a.classes <= 512) return short_backward<T, 16>(a, rows, st);
    return short_backward<T, 32>(a, rows, st);
  }
  const unsigned blocks = (unsigned)(rows * a.chunks);
  if (a.n_ids > 32) logprobs_backward_kernel<T, true><<<blocks, kBwdThreads, 0, st>>>(a);
  else logprobs_backward_kernel<T, false><<<blocks, kBwdThreads, 0, st>>>(a);
  return cudaGetLastError();
}

int common_checks(const void* logits, int32_t dtype, int64_t rows, int32_t classes, int64_t ld, const int32_t* ids,
                  int32_t n_ids) {
  if (dtype != VGG19_FP32 && dtype != VGG19_BF16)
    return note_error(VGG19_ERR_ARG, "dtype %d is neither VGG19_FP32 nor VGG19_BF16", dtype);
  if (rows < 0 || rows > (1 << 26) || classes < 1 || classes > (1 << 30))
    return note_error(VGG19_ERR_SHAPE, "%lld rows of %d classes: rows in [0, 2^26], classes in [1, 2^30]", (long long)rows, classes);
  if (ld < classes) return note_error(VGG19_ERR_SHAPE, "row stride %lld below %d classes", (long long)ld, classes);
  if (n_ids < 0 || n_ids > kMaxIds) return note_error(VGG19_ERR_ARG, "%d ids a row: at most %d", n_ids, kMaxIds);
  if (rows == 0) return VGG19_OK;
  if (!logits || (n_ids && !ids)) return note_error(VGG19_ERR_ARG, "logits, and ids where n_ids > 0, must not be null");
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == VGG19_FP32 ? 4 : 2))
    return note_error(VGG19_ERR_ARG, "logits are not aligned to their type");
  return VGG19_OK;
}
// whether all of these (null among them) are addresses of 32-bit values
template <typename... P> bool words(P... p) { return ((reinterpret_cast<uintptr_t>(p) % 4 == 0) && ...); }

}  // namespace

cudaError_t logprobs_error_words(ErrorWords* words) { return cudaGetSymbolAddress(reinterpret_cast<void**>(&words->at[kErrorId]), g_logprobs_error); }

}  // namespace vgg

extern "C" int vgg19_logprobs(const void* logits, int32_t dtype, int64_t rows, int32_t classes, int64_t ld,
                              const int32_t* ids, int32_t n_ids, int32_t top_k, float* logprob, float* lse,
                              float* entropy, int32_t* top_id, float* top_logprob, void* stream) {
  using namespace vgg;
  const int rc = common_checks(logits, dtype, rows, classes, ld, ids, n_ids);
  if (rc != VGG19_OK) return rc;
  if (top_k < 0 || top_k > kMaxTop) return note_error(VGG19_ERR_ARG, "top_k %d outside [0, %d]", top_k, kMaxTop);
  if (rows == 0) return VGG19_OK;
  if ((n_ids && !logprob) || (top_k && (!top_id || !top_logprob)))
    return note_error(VGG19_ERR_ARG, "null output for %d ids or the top %d", n_ids, top_k);
  if (!words(ids, logprob, lse, entropy, top_id, top_logprob)) return note_error(VGG19_ERR_ARG, "ids or an output is not aligned to 4 bytes");
  const long elt = dtype == VGG19_FP32 ? 4 : 2, given = 4L * rows * n_ids, top = 4L * rows * top_k, each = 4L * rows;
  const Span all[] = {{logprob, given}, {lse, each}, {entropy, each}, {top_id, top}, {top_logprob, top}, {ids, given}};
  bool meet = spans_meet(all, 5);
  for (int i = 0; i < 5; ++i) meet = meet || rows_meet(logits, rows, classes * elt, ld * elt, all[i].p, all[i].bytes > 0, all[i].bytes, 0);
  if (meet) return note_error(VGG19_ERR_ARG, "an output overlaps logits, ids or another output");
  const FwdArgs a{logits, ids, logprob, lse, entropy, top_logprob, top_id, (long)ld, classes, n_ids, top_k};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == VGG19_BF16 ? forward<bf16>(a, rows, st) : forward<float>(a, rows, st);
  return e == cudaSuccess ? VGG19_OK : note_error(VGG19_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}

extern "C" int vgg19_logprobs_backward(const void* logits, int32_t dtype, int64_t rows, int32_t classes, int64_t ld,
                                       const int32_t* ids, int32_t n_ids, const float* lse, const float* entropy,
                                       const float* d_logprob, const float* d_entropy, void* d_logits, int64_t d_ld,
                                       void* stream) {
  using namespace vgg;
  const int rc = common_checks(logits, dtype, rows, classes, ld, ids, n_ids);
  if (rc != VGG19_OK) return rc;
  if (d_ld < classes) return note_error(VGG19_ERR_SHAPE, "row stride %lld below %d classes", (long long)d_ld, classes);
  if (rows == 0) return VGG19_OK;
  if (!lse || !d_logits || (n_ids && !d_logprob) || (d_entropy && !entropy))
    return note_error(VGG19_ERR_ARG, "null lse or d_logits, ids without d_logprob, or d_entropy without entropy");
  if (reinterpret_cast<uintptr_t>(d_logits) % (dtype == VGG19_FP32 ? 4 : 2))
    return note_error(VGG19_ERR_ARG, "d_logits is not aligned to its type");
  if (!words(ids, lse, entropy, d_logprob, d_entropy)) return note_error(VGG19_ERR_ARG, "ids or an fp32 input is not aligned to 4 bytes");
  const long elt = dtype == VGG19_FP32 ? 4 : 2;
  if (!(d_logits == logits && (d_ld == ld || rows == 1)) && rows_meet(logits, rows, classes * elt, ld * elt, d_logits, rows, classes * elt, d_ld * elt))
    return note_error(VGG19_ERR_ARG, "d_logits overlaps logits without being the same rows");
  const int per = kBwdThreads * kBwdUnroll * (dtype == VGG19_BF16 ? 8 : 4);
  const int64_t chunks = (classes + per - 1) / per;
  if (rows * chunks > 0x7fffffffLL) return note_error(VGG19_ERR_SHAPE, "%lld rows of %d classes are too many", (long long)rows, classes);
  const Span read[] = {{ids, 4L * rows * n_ids}, {d_logprob, 4L * rows * n_ids}, {lse, 4L * rows}, {entropy, 4L * rows}, {d_entropy, 4L * rows}};
  for (const Span& s : read)
    if (rows_meet(d_logits, rows, classes * elt, d_ld * elt, s.p, s.bytes > 0, s.bytes, 0))
      return note_error(VGG19_ERR_ARG, "d_logits overlaps another input than logits");
  const BwdArgs a{logits, d_logits, ids, lse, entropy, d_logprob, d_entropy, (long)ld, (long)d_ld, classes, n_ids, (int)chunks};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == VGG19_BF16 ? backward<bf16>(a, rows, st) : backward<float>(a, rows, st);
  return e == cudaSuccess ? VGG19_OK : note_error(VGG19_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}
