// Log probabilities of given classes, log-sum-exp, entropy and the top alternatives of rows of logits, and their
// gradient.  For a row z of n logits
//   lse = log sum_j exp(z_j),   log p_j = z_j - lse,   H = -sum_j p_j log p_j,
//   d(sum_i g_i log p[id_i] + w H) / dz_j = sum_i g_i [j = id_i] - p_j (sum_i g_i + w (log p_j + H)).
//
// Both directions are bound by reading the logits (and writing the gradient) once.  The forward kernel makes one
// pass: every warp keeps a reference `ref` (a value near the largest it has seen), S = sum exp(z - ref) and
// U = sum exp(z - ref) (z - ref), in fp32, and at the end H = log S - U / S, lse = ref + log S.  The top
// alternatives ride on the same pass: a warp holds its best `top_k` as 64-bit keys (value, then lower index), sorted
// over its lanes, and looks closer only at vectors whose maximum reaches the smallest of them.
//
// A row belongs to one block, or, where there are fewer rows than the GPU has room for, to a cluster of up to
// eight blocks that join through distributed shared memory: one launch, no scratch, and an order of summation that
// depends on the sizes alone.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "../../include/vgg19_b200.h"
#include "common.cuh"

namespace cg = cooperative_groups;

namespace vgg {
namespace {

static __device__ int g_logprobs_error;  // kDevBadLabel once an id outside [0, classes) was met

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// A warp's reference moves only when a value exceeds it by this much (natural units): exp(z - ref) then stays below
// e^4, and the moves, each a branch of the whole warp, stay rare after the first vectors.
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

// values ordered as unsigned integers; -0 counts as 0
__device__ __forceinline__ unsigned long long make_key(float v, unsigned index) {
  const int b = __float_as_int(v + 0.f);
  const unsigned o = b < 0 ? ~(unsigned)b : (unsigned)b | 0x80000000u;
  return ((unsigned long long)o << 32) | (0xffffffffu - index);
}
__device__ __forceinline__ float key_value(unsigned long long k) {
  const unsigned o = (unsigned)(k >> 32);
  return __int_as_float((int)(o & 0x80000000u ? o & 0x7fffffffu : ~o));
}
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
// b folded into a; either may be empty (ref = -inf, S = 0, or NaN when a NaN was met)
__device__ __forceinline__ Sums join(Sums a, Sums b) {
  const float m = fmaxf(a.ref, b.ref);
  const float da = a.ref == m ? 0.f : (a.ref - m) * kLog2e, db = b.ref == m ? 0.f : (b.ref - m) * kLog2e;
  const float fa = fast_exp2(da), fb = fast_exp2(db);
  Sums r;
  r.ref = m;
  r.S = a.S * fa + b.S * fb;
  // an empty or vanished part (factor 0) would bring -inf * 0
  r.U = (fa > 0.f ? (a.U + da * a.S) * fa : a.U * 0.f) + (fb > 0.f ? (b.U + db * b.S) * fb : b.U * 0.f);
  return r;
}

// A warp's state over the logits it has seen.
struct WarpScan {
  float ref, S, U;         // ref is the same in all lanes, S and U are a lane's share
  unsigned long long key;  // lane i: the i-th best so far, 0 for none
  float thr;               // a logit below this cannot enter the best top_k
  int top_k;

  __device__ WarpScan(int k) : ref(-INFINITY), S(0.f), U(0.f), key(0), thr(k > 0 ? -3.402823466e38f : INFINITY), top_k(k) {}

  __device__ __forceinline__ void insert(unsigned long long c) {
    const unsigned long long up = __shfl_up_sync(0xffffffffu, key, 1);
    const int lane = threadIdx.x & 31;
    if (c > key) key = lane > 0 && c > up ? up : c;
  }

  // the vector's N logits; index(e) is the class of element e of this lane
  template <int N, typename Index> __device__ __forceinline__ void add(const float (&x)[N], Index index) {
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) mx = fmaxf(mx, x[e]);
    if (__any_sync(0xffffffffu, mx > ref + kRefMargin || mx >= thr)) slow(x, mx, index);
    const float r = ref == -INFINITY ? 0.f : ref;  // nothing but -inf so far: every exponent is -inf
    float s0 = 0.f, s1 = 0.f, u0 = 0.f, u1 = 0.f;
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      const float t0 = max_nan((x[e] - r) * kLog2e, kFloor);
      const float e0 = fast_exp2(t0);
      s0 += e0; u0 = fmaf(e0, t0, u0);
      if (e + 1 < N) {
        const float t1 = max_nan((x[e + 1] - r) * kLog2e, kFloor);
        const float e1 = fast_exp2(t1);
        s1 += e1; u1 = fmaf(e1, t1, u1);
      }
    }
    S += s0 + s1;
    U += u0 + u1;
  }

  template <int N, typename Index> __device__ __forceinline__ void slow(const float (&x)[N], float mx, Index index) {
    const unsigned full = 0xffffffffu;
    float wm = mx;
#pragma unroll
    for (int o = 16; o; o >>= 1) wm = fmaxf(wm, __shfl_xor_sync(full, wm, o));
    if (wm > ref + kRefMargin) {
      if (ref != -INFINITY) {
        const float d = (ref - wm) * kLog2e, f = fast_exp2(d);
        U = f > 0.f ? (U + d * S) * f : 0.f * U;
        S *= f;
      }
      ref = wm;
    }
    if (top_k == 0 || !__any_sync(full, mx >= thr)) return;
    const int lane = threadIdx.x & 31;
    if (__shfl_sync(full, key, top_k - 1) == 0) {
      // not full yet: the top_k-th largest of the lanes' maxima is a bound that top_k logits reach
      int rank = 0;
      for (int j = 0; j < 32; ++j) {
        const float v = __shfl_sync(full, mx, j);
        rank += v > mx || (v == mx && j < lane);
      }
      const unsigned at = __ballot_sync(full, rank == top_k - 1);
      const float bound = at ? __shfl_sync(full, mx, __ffs(at) - 1) : -INFINITY;  // (a NaN lane takes no rank)
      if (bound > thr) thr = bound;
    }
#pragma unroll 1
    for (int e = 0; e < N; ++e) {
      float v = x[0];
#pragma unroll
      for (int k = 1; k < N; ++k)
        if (k == e) v = x[k];
      unsigned hits = __ballot_sync(full, v >= thr);
      if (!hits) continue;
      const unsigned long long mine = v >= thr ? make_key(v, index(e)) : 0;
      while (hits) {
        const int src = __ffs(hits) - 1;
        hits &= hits - 1;
        insert(__shfl_sync(full, mine, src));
      }
      const unsigned long long last = __shfl_sync(full, key, top_k - 1);
      if (last) thr = fmaxf(thr, key_value(last));
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
  constexpr int V = Vec<T>::N, W = NT / 32;
  __shared__ Sums part[W];
  __shared__ unsigned long long keys[W * kMaxTop];
  __shared__ Sums cpart[kMaxCluster];                             // of the cluster's blocks, in its first
  __shared__ unsigned long long ckeys[kMaxCluster * kMaxTop], best[kMaxTop];
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  if (C > 1) cluster.barrier_arrive();  // waited for before the first write into the first block's shared memory
  const long row = blockIdx.x / C;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  const RowSplit<T> sp(z, a.classes);
  const uint4* body = reinterpret_cast<const uint4*>(z + sp.head);
  const int v0 = (int)((long)sp.nvec * rank / C), v1 = (int)((long)sp.nvec * (rank + 1) / C);

  WarpScan w(a.top_k);
  const uint4 none = make_uint4(Vec<T>::kMinusInf, Vec<T>::kMinusInf, Vec<T>::kMinusInf, Vec<T>::kMinusInf);
  for (int base = v0 + warp * 32; base < v1; base += NT * UNROLL) {  // (a warp leaves the loop as one)
    uint4 r[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int v = base + u * NT + lane;
      r[u] = v < v1 ? __ldcs(body + v) : none;
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      float x[V];
      Vec<T>::unpack(r[u], x);
      const int first = sp.head + (base + u * NT + lane) * V;
      w.add(x, [first](int e) { return (unsigned)(first + e); });
    }
  }
  if (rank == 0 && warp == 0 && sp.head + sp.tail > 0) {
    const int t = lane - 8;  // lanes 0..7 the head, 8..15 the tail
    const int at = lane < sp.head ? lane : t >= 0 && t < sp.tail ? sp.head + sp.nvec * V + t : -1;
    float x[1] = {at >= 0 ? to_f32(z[at]) : -INFINITY};
    w.add(x, [at](int) { return (unsigned)at; });
  }

  const float S = lane_sum(w.S), U = lane_sum(w.U);
  if (lane == 0) part[warp] = Sums{w.ref, S, U};
  if (lane < a.top_k) keys[warp * a.top_k + lane] = w.key;
  if (tid < a.top_k) best[tid] = 0;
  __syncthreads();
  Sums all = part[0];
  for (int i = 1; i < W; ++i) all = join(all, part[i]);
  if (a.top_k) {
    rank_keys(keys, W * a.top_k, a.top_k, best);
    __syncthreads();
  }
  if (C > 1) {
    cluster.barrier_wait();
    if (tid == 0) cluster.map_shared_rank(cpart, 0)[rank] = all;
    if (tid < a.top_k) cluster.map_shared_rank(ckeys, 0)[rank * a.top_k + tid] = best[tid];
    cluster.sync();
    if (rank != 0) return;
    all = cpart[0];
    for (int i = 1; i < C; ++i) all = join(all, cpart[i]);
    if (a.top_k) {
      if (tid < a.top_k) best[tid] = 0;
      __syncthreads();
      rank_keys(ckeys, C * a.top_k, a.top_k, best);
      __syncthreads();
    }
  }

  // (z - ref) - log S, not z - lse: lse is rounded to its own magnitude
  const bool bad = !(all.S == all.S) || all.ref == INFINITY, empty = !bad && all.ref == -INFINITY;
  const float nan = __int_as_float(0x7fc00000);
  const float logS = logf(all.S);
  if (tid == 0) {
    if (a.lse) a.lse[row] = bad ? nan : empty ? -INFINITY : all.ref + logS;
    if (a.entropy) a.entropy[row] = bad ? nan : empty ? 0.f : fmaxf(logS - kLn2 * (all.U / all.S), 0.f);
  }
  for (int i = tid; i < a.n_ids; i += NT) {
    const int id = a.ids[row * a.n_ids + i];
    float v = 0.f;
    if (id != VGG19_NO_CLASS) {
      if ((unsigned)id < (unsigned)a.classes) {
        v = bad ? nan : empty ? -INFINITY : (to_f32(z[id]) - all.ref) - logS;
      } else {  // never used as an index
        v = nan;
        atomicCAS(&g_logprobs_error, 0, (int)kDevBadLabel);
      }
    }
    a.logprob[row * a.n_ids + i] = v;
  }
  if (tid < a.top_k) {
    const unsigned long long k = bad ? 0 : best[tid];
    a.top_id[row * a.top_k + tid] = k ? (int32_t)key_index(k) : VGG19_NO_CLASS;
    a.top_logprob[row * a.top_k + tid] = bad ? nan : k ? (key_value(k) - all.ref) - logS : -INFINITY;
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

// One block takes `chunk` vectors of one row.  The ids that fall into its chunk (usually none or one) are listed in
// shared memory first, in their order, so that a class named twice gets both shares in the same order every time and
// every element is rounded and written once; d_logits may be logits.
constexpr int kBwdThreads = 256, kBwdUnroll = 8;

template <typename T>
__global__ void __launch_bounds__(kBwdThreads) logprobs_backward_kernel(const BwdArgs a) {
  constexpr int V = Vec<T>::N;
  __shared__ int hit_at[kMaxIds];
  __shared__ float hit_g[kMaxIds];
  __shared__ float s_sum;
  __shared__ int s_hits;
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
  if (tid < 32) {
    float sum = 0.f;
    int hits = 0;
    for (int i = 0; i < a.n_ids; i += 32) {
      const int id = i + lane < a.n_ids ? a.ids[row * a.n_ids + i + lane] : VGG19_NO_CLASS;
      const bool in = (unsigned)id < (unsigned)a.classes;
      if (!in && id != VGG19_NO_CLASS) atomicCAS(&g_logprobs_error, 0, (int)kDevBadLabel);
      const float g = in ? a.d_logprob[row * a.n_ids + i + lane] : 0.f;
      sum += lane_sum(g);
      const bool mine = in && ((id >= lo && id < hi) || (chunk == 0 && (id < sp.head || id >= sp.head + sp.nvec * V)));
      const unsigned m = __ballot_sync(0xffffffffu, mine);
      if (mine) {
        const int at = hits + __popc(m & ((1u << lane) - 1));
        hit_at[at] = id;
        hit_g[at] = g;
      }
      hits += __popc(m);
    }
    if (lane == 0) { s_sum = sum; s_hits = hits; }
  }
  __syncthreads();
  const float lse = a.lse[row], w = a.d_entropy ? a.d_entropy[row] : 0.f;
  const float c = s_sum + (a.d_entropy ? w * a.entropy[row] : 0.f);
  const int hits = s_hits;
  const bool empty = lse == -INFINITY;  // a row with no class left has no gradient
  auto grad = [&](float x) {
    const float lp = max_nan(x - lse, kFloor);
    return -fast_exp2(lp * kLog2e) * fmaf(w, lp, c);
  };
#pragma unroll
  for (int u = 0; u < kBwdUnroll; ++u) {
    const int v = v0 + u * kBwdThreads + tid;
    if (v >= sp.nvec) break;
    float x[V];
    Vec<T>::unpack(r[u], x);
    const int first = sp.head + v * V;
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = empty ? 0.f : grad(x[e]);
    for (int h = 0; h < hits; ++h) {
      const int d = hit_at[h] - first;
      if ((unsigned)d < (unsigned)V && !empty) {
        const float g = hit_g[h];
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] += e == d ? g : 0.f;
      }
    }
    if (same) {
      __stcs(reinterpret_cast<uint4*>(dz + first), Vec<T>::pack(x));
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) dz[first + e] = from_f32<T>(x[e]);
    }
  }
  if (chunk == 0 && tid < sp.head + sp.tail) {
    const int at = tid < sp.head ? tid : sp.nvec * V + tid;
    float d = empty ? 0.f : grad(to_f32(z[at]));
    for (int h = 0; h < hits; ++h)
      if (hit_at[h] == at && !empty) d += hit_g[h];
    dz[at] = from_f32<T>(d);
  }
}

// How many blocks share a row: enough to give every SM two blocks while each still has a few thousand classes.
int cluster_size(long rows, int classes) {
  int c = 1;
  while (c < kMaxCluster && rows * c * 2 <= 296 && classes / (c * 2) >= 2048) c *= 2;
  return c;
}

template <typename T, int NT, int UNROLL> cudaError_t launch_forward(const FwdArgs& a, long rows, int C, cudaStream_t st) {
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

template <typename T> cudaError_t forward(const FwdArgs& a, long rows, cudaStream_t st) {
  const int C = cluster_size(rows, a.classes), per = a.classes / C;
  if (per <= 2048) return launch_forward<T, 128, 2>(a, rows, C, st);
  return launch_forward<T, 256, 4>(a, rows, C, st);
}

template <typename T> cudaError_t backward(const BwdArgs& a, long rows, cudaStream_t st) {
  logprobs_backward_kernel<T><<<(unsigned)(rows * a.chunks), kBwdThreads, 0, st>>>(a);
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

}  // namespace

cudaError_t logprobs_take_error(int* code) {
  cudaError_t e = cudaMemcpyFromSymbol(code, g_logprobs_error, sizeof(int));
  if (e == cudaSuccess && *code) {
    const int zero = 0;
    e = cudaMemcpyToSymbol(g_logprobs_error, &zero, sizeof(int));
  }
  return e;
}

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
  const int per = kBwdThreads * kBwdUnroll * (dtype == VGG19_BF16 ? 8 : 4);
  const int64_t chunks = (classes + per - 1) / per;
  if (rows * chunks > 0x7fffffffLL) return note_error(VGG19_ERR_SHAPE, "%lld rows of %d classes are too many", (long long)rows, classes);
  const BwdArgs a{logits, d_logits, ids, lse, entropy, d_logprob, d_entropy, (long)ld, (long)d_ld, classes, n_ids, (int)chunks};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == VGG19_BF16 ? backward<bf16>(a, rows, st) : backward<float>(a, rows, st);
  return e == cudaSuccess ? VGG19_OK : note_error(VGG19_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}
