// The last dense layer with its loss for up to eight rows of fp32, the loss alone for up to 24, on the CUDA cores (formulas in linear_loss.cu).  So few rows are
// bound by reading w, and writing dw; the tensor cores would have it written down as three bf16 planes first, half as much again as w itself, and
// read again from there.  (bf16 weights need no planes: there the tiles are as fast or faster.)  Forward, w is read once: a warp takes a few
// classes, its lanes along the inputs, with the rows of x in shared memory.  Backward it is read twice: for z, which becomes dz [classes][rows],
// and by threads that keep four inputs each, of x and of dx, and go through a range of the classes, writing dw.  All sums are fp32 FMAs.
//
// Measured (B200, device time; the planes' way behind): 4096 inputs against 50021 classes, one row 142 us and 416 us for the gradients (781 and 1396),
// eight rows 221 and 624 (778 and 1303); against 1000 classes, one row 13 and 19 (21 and 41), eight 23 and 34 (20 and 41).  One row reads w at 5.8 TB/s (0.9 of a
// copy's rate); eight rows read x twice from shared memory for every value of w, with one block of sixteen warps an SM (eight warps: 321 us).  More rows are
// groups of eight, each with a share of the SMs, that read w beside one another, mostly from L2: 9 to 16 rows 382 us (775), 17 to 24 537 (782).
// (Gradients of groups: dx and dw of sixteen rows want 180 registers a thread and are bound by their loads, 1230 us for all where the planes take 1310, but 124
// against 106 for 16 rows of 1024 against 16000 classes and 440 against 400 for 512 against 131072: left to the planes.)
#include <cuda_runtime.h>

#include "../../include/vgg19_b200.h"
#include "linear_loss.cuh"

namespace vgg {
namespace {

static __device__ int g_few_label_error[1];  // kDevBadLabel once a label outside [0, classes) was met

constexpr int kV = 4;  // values of a slot: 16 bytes

// What another launch may have written is read by ordinary loads: kernels are set up while the ones before them run (an update's that writes w, the
// one that writes dz), and the read-only path is for memory that nobody writes as long as its reader lives.  __ldcg, from L2, for what is read
// once; load_again, through L1, for dz, which all of a block's warps read (from L2 one row against 50021 classes of 4096 takes 464 us for all gradients, this
// way 411).  Both stay behind the wait for the launch before, but stores do not hold them up, as they would a plain dereference.
__device__ __forceinline__ float load_again(const float* p) {
  float v;
  asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ float4 load_again(const float4* p) {
  float4 v;
  asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p));
  return v;
}
constexpr int kMostWarps = 16;

// Slot q of a row: V values, those from q V on where rows are aligned; else of every 32 V values, q % 32 and every 32nd behind it, so that lanes
// run along the row either way.
struct Slots {
  int in;
  bool aligned;
  __device__ __forceinline__ int at(int q, int j) const { return aligned ? q * kV + j : (q / 32 * kV + j) * 32 + q % 32; }
};
// The values of a slot; beyond the row there are zeros.  whole: whether the row's 16 bytes can be read at once, where slots are that.
__device__ __forceinline__ float4 load_slot(const float* row, int q, const Slots& s, bool whole = true) {
  if (s.aligned && whole && (q + 1) * kV <= s.in) return __ldcg(reinterpret_cast<const float4*>(row) + q);
  float v[kV];
#pragma unroll
  for (int j = 0; j < kV; ++j) {
    const int k = s.at(q, j);
    v[j] = k < s.in ? __ldcg(row + k) : 0.f;
  }
  return make_float4(v[0], v[1], v[2], v[3]);
}

// The rows of x in shared memory, slot by slot.
template <int RM>
__device__ __forceinline__ void stage_rows(float* xs, const float* x, long ldx, int rows, const Slots& s, int warps_slots, bool whole) {
  const int slots = warps_slots * 32;
#pragma unroll
  for (int r = 0; r < RM; ++r)
#pragma unroll 4
    for (int q = threadIdx.x; q < slots; q += blockDim.x)
      reinterpret_cast<float4*>(xs)[r * slots + q] = r < rows ? load_slot(x + r * ldx, q, s, whole) : make_float4(0.f, 0.f, 0.f, 0.f);
}

// acc[b * RM + r]: the lane's share of row r times class b of those at `w`, of which there are `left`.
template <int RM, int B>
__device__ __forceinline__ void share_of_products(float (&acc)[B * RM], const float* w, long ldw, int left, const float* xs, const Slots& s, int warps_slots) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < B * RM; ++i) acc[i] = 0.f;
#pragma unroll 2
  for (int c = 0; c < warps_slots; ++c) {
    const int q = c * 32 + lane;
    float4 v[B];
#pragma unroll
    for (int b = 0; b < B; ++b) v[b] = load_slot(w + min(b, left - 1) * ldw, q, s);
#pragma unroll
    for (int r = 0; r < RM; ++r) {
      const float4 x = reinterpret_cast<const float4*>(xs)[r * warps_slots * 32 + q];
#pragma unroll
      for (int b = 0; b < B; ++b) {
        float& t = acc[b * RM + r];
        t = fmaf(v[b].w, x.w, fmaf(v[b].z, x.z, fmaf(v[b].y, x.y, fmaf(v[b].x, x.x, t))));
      }
    }
  }
}
// The sums of N values over the warp's lanes: lane l gets number l % N's, in an order that is always the same.
template <int N> __device__ __forceinline__ float sum_over_lanes(float (&v)[N]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int w = N / 2; w; w >>= 1) {
    const bool upper = lane & w;
#pragma unroll
    for (int j = 0; j < w; ++j) {
      const float give = upper ? v[j] : v[j + w], keep = upper ? v[j + w] : v[j];
      v[j] = keep + __shfl_xor_sync(0xffffffffu, give, w);
    }
  }
#pragma unroll
  for (int w = N; w < 32; w *= 2) v[0] += __shfl_xor_sync(0xffffffffu, v[0], w);
  return v[0];
}

struct Layer {
  const float *x, *w;
  long ldx, ldw;
  const float* bias;
  const int32_t* labels;
  int rows, in, classes, warps_slots;  // warps_slots: a lane's slots of a row
  int aligned, x_aligned;              // whether 16 bytes of w (2: and of dw), of x can be taken at once
  // forward
  float2* part;
  float* label_z;
  // backward
  FewGradients g;
};

template <int RM, int B> __global__ void __launch_bounds__(32 * kMostWarps) few_loss_kernel(const __grid_constant__ Layer a) {
  extern __shared__ float xs[];
  __shared__ float2 got[kMostWarps][RM];
  behind_previous();
  const Slots s{a.in, a.aligned != 0};
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x / 32;
  const int row0 = blockIdx.y * RM, rows = min(RM, a.rows - row0);
  stage_rows<RM>(xs, a.x + row0 * a.ldx, a.ldx, rows, s, a.warps_slots, a.x_aligned != 0);
  __syncthreads();
  constexpr int N = B * RM;
  const int r = lane % N % RM, b = lane % N / RM;
  const int label = r < rows ? a.labels[row0 + r] : VGG19_NO_CLASS;
  float2 most = make_float2(-INFINITY, 0.f);
  for (int n0 = (blockIdx.x * warps + warp) * B; n0 < a.classes; n0 += gridDim.x * warps * B) {
    float acc[N];
    share_of_products<RM, B>(acc, a.w + n0 * a.ldw, a.ldw, a.classes - n0, xs, s, a.warps_slots);
    const float sum = sum_over_lanes<N>(acc);
    const int n = n0 + b;
    if (lane < N && n < a.classes) {
      const float z = sum + (a.bias ? __ldcg(a.bias + n) : 0.f);
      if (n == label) a.label_z[row0 + r] = z;
      most = join(most, z != z ? make_float2(-INFINITY, z) : make_float2(z, z == -INFINITY ? 0.f : 1.f));
    }
  }
#pragma unroll
  for (int w = N / 2; w >= RM; w /= 2) {  // the lanes of one row
    const float2 o = make_float2(__shfl_down_sync(0xffffffffu, most.x, w), __shfl_down_sync(0xffffffffu, most.y, w));
    if (lane < w) most = join(most, o);
  }
  if (lane < RM) got[warp][lane] = most;
  __syncthreads();
  if (threadIdx.x >= rows) return;
  most = got[0][threadIdx.x];
  for (int k = 1; k < warps; ++k) most = join(most, got[k][threadIdx.x]);
  a.part[(long)blockIdx.x * a.rows + row0 + threadIdx.x] = most;
}

// dz [classes][RM] from z, and db.
template <int RM, int B> __global__ void __launch_bounds__(32 * kMostWarps) few_logit_gradient_kernel(const __grid_constant__ Layer a) {
  extern __shared__ float xs[];
  behind_previous();
  const Slots s{a.in, a.aligned != 0};
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x / 32;
  stage_rows<RM>(xs, a.x, a.ldx, a.rows, s, a.warps_slots, a.x_aligned != 0);
  __syncthreads();
  constexpr int N = B * RM;
  const int r = lane % N % RM, b = lane % N / RM;
  int label = VGG19_NO_CLASS;
  float lse = 0.f, d_loss = 0.f;
  if (r < a.rows) {
    label = a.labels[r];
    lse = a.g.lse[r];
    const bool real = (unsigned)label < (unsigned)a.classes;
    if (!real && label != VGG19_NO_CLASS && blockIdx.x == 0) atomicCAS(g_few_label_error, 0, (int)kDevBadLabel);
    d_loss = real && lse != -INFINITY ? a.g.d_loss[r] : 0.f;
  }
  for (int n0 = (blockIdx.x * warps + warp) * B; n0 < a.classes; n0 += gridDim.x * warps * B) {
    float acc[N];
    share_of_products<RM, B>(acc, a.w + n0 * a.ldw, a.ldw, a.classes - n0, xs, s, a.warps_slots);
    const float sum = sum_over_lanes<N>(acc);
    const int n = n0 + b;
    float d = 0.f;
    if (n < a.classes && d_loss != 0.f) {  // (a row that counts for nothing may hold anything; a NaN is not 0)
      const float p = fast_exp2((sum + (a.bias ? __ldcg(a.bias + n) : 0.f) - lse) * kLossLog2e);
      d = d_loss * (n == label ? p - 1.f : p);
    }
    if (lane < N && n < a.classes) a.g.dz[(long)n * RM + r] = d;
    if (a.g.db) {  // over the rows, which are neighbouring lanes
#pragma unroll
      for (int k = RM / 2; k; k /= 2) d += __shfl_xor_sync(0xffffffffu, d, k);
      if (lane < N && r == 0 && n < a.classes) a.g.db[n] = d;
    }
  }
}

// dw of a range of the classes, and its part of dx: a thread has one slot of every row.
constexpr int kProductThreads = 128;
template <int RM> __global__ void __launch_bounds__(kProductThreads) few_products_kernel(const __grid_constant__ Layer a, int range) {
  constexpr int UNROLL = RM == 8 ? 4 : 8;  // classes whose weights are requested at once
  behind_previous();
  const Slots s{a.in, a.aligned != 0};
  const int q = blockIdx.x * kProductThreads + threadIdx.x;
  if (q >= a.warps_slots * 32) return;
  const bool whole = a.aligned == 2 && (q + 1) * kV <= a.in;
  float x[RM][kV], dx[RM][kV];
#pragma unroll
  for (int r = 0; r < RM; ++r)
#pragma unroll
    for (int j = 0; j < kV; ++j) {
      const int k = s.at(q, j);
      x[r][j] = r < a.rows && k < a.in ? a.x[r * a.ldx + k] : 0.f;
      dx[r][j] = 0.f;
    }
  const int first = blockIdx.y * range, end = min(first + range, a.classes);
  for (int n0 = first; n0 < end; n0 += UNROLL) {
    float4 w[UNROLL];
    if (a.g.dx_part) {
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) w[u] = load_slot(a.w + min(n0 + u, end - 1) * a.ldw, q, s);
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int n = n0 + u;
      if (n >= end) break;
      float e[RM];
#pragma unroll
      for (int r = 0; r < RM; r += RM < 4 ? 1 : 4) {
        const float* at = a.g.dz + (long)n * RM + r;
        if (RM < 4) {
          e[r] = load_again(at);
        } else {
          const float4 v = load_again(reinterpret_cast<const float4*>(at));
          e[r] = v.x; e[(r + 1) % RM] = v.y; e[(r + 2) % RM] = v.z; e[(r + 3) % RM] = v.w;
        }
      }
      if (a.g.dx_part) {
#pragma unroll
        for (int r = 0; r < RM; ++r) {
          dx[r][0] = fmaf(e[r], w[u].x, dx[r][0]); dx[r][1] = fmaf(e[r], w[u].y, dx[r][1]);
          dx[r][2] = fmaf(e[r], w[u].z, dx[r][2]); dx[r][3] = fmaf(e[r], w[u].w, dx[r][3]);
        }
      }
      if (a.g.dw) {
        float v[kV];
#pragma unroll
        for (int j = 0; j < kV; ++j) {
          v[j] = e[0] * x[0][j];
#pragma unroll
          for (int r = 1; r < RM; ++r) v[j] = fmaf(e[r], x[r][j], v[j]);
        }
        float* out = a.g.dw + n * a.g.dw_ld;
        if (whole) {
          reinterpret_cast<float4*>(out)[q] = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
          for (int j = 0; j < kV; ++j) {
            const int k = s.at(q, j);
            if (k < a.in) out[k] = v[j];
          }
        }
      }
    }
  }
  if (!a.g.dx_part) return;
#pragma unroll
  for (int r = 0; r < RM; ++r)
#pragma unroll
    for (int j = 0; j < kV; ++j) {
      const int k = s.at(q, j);
      if (r < a.rows && k < a.in) a.g.dx_part[((long)blockIdx.y * a.rows + r) * a.g.dx_ld + k] = dx[r][j];
    }
}

// Rows of a group, rounded up to what there are kernels for, and groups.
int group_up(const vgg19_linear_loss& a) { return few_rows_up((int)a.rows); }
int groups(const vgg19_linear_loss& a) { return (int)(a.rows + 7) / 8; }
// Classes that a warp takes at once: eight (four of eight rows: 32 sums), or two where more would leave SMs without a warp.
constexpr int many(int rm) { return rm == 8 ? 4 : 8; }
int classes_at_once(const vgg19_linear_loss& a, int sms) {
  const int b = many(group_up(a));
  return a.classes < sms / groups(a) * 8 * b ? 2 : b;
}
// Warps of a block: every SM has one before a block has several, unless the rows that a block keeps are many bytes; where an SM has room for one
// block's rows alone, that has sixteen.
constexpr int kMostKept = 32768;  // values (rounded up to 128 a row, which divides it for any number of rows)
int kept_values(const vgg19_linear_loss& a) { return group_up(a) * a.in; }
int warps_of(const vgg19_linear_loss& a, int sms) {
  const int b = classes_at_once(a, sms);
  sms /= groups(a);
  int warps = 8;
  if (kept_values(a) > 12288) return (a.classes + 8 * b - 1) / (8 * b) > sms ? kMostWarps : warps;
  if (kept_values(a) > 2048) return warps;
  while (warps > 1 && (a.classes + b * warps - 1) / (b * warps) < sms) warps /= 2;
  return warps;
}

Layer layer_of(const vgg19_linear_loss& a) {
  Layer l{};
  l.x = static_cast<const float*>(a.x); l.w = static_cast<const float*>(a.w); l.ldx = a.ldx; l.ldw = a.ldw; l.bias = a.bias; l.labels = a.labels;
  l.rows = (int)a.rows; l.in = a.in; l.classes = a.classes;
  l.aligned = reinterpret_cast<uintptr_t>(a.w) % 16 == 0 && (a.classes == 1 || a.ldw % 4 == 0);
  l.x_aligned = reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && (a.rows == 1 || a.ldx % 4 == 0);
  l.warps_slots = (a.in + 32 * kV - 1) / (32 * kV);
  return l;
}

template <typename K> cudaError_t launch_logits(K kernel, const Layer& l, int rm, int blocks, int warps, cudaStream_t st) {
  const dim3 grid((unsigned)blocks, (unsigned)((l.rows + rm - 1) / rm));
  const int smem = rm * l.warps_slots * 32 * kV * 4;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostKept * 4);  // (the same for all: calls may be made from several threads)
  return e == cudaSuccess ? launch_behind(kernel, grid, 32 * warps, smem, st, l) : e;
}
template <int RM> cudaError_t loss_of(const Layer& l, int b, int blocks, int warps, cudaStream_t st) {
  return b == 2 ? launch_logits(few_loss_kernel<RM, 2>, l, RM, blocks, warps, st) : launch_logits(few_loss_kernel<RM, many(RM)>, l, RM, blocks, warps, st);
}
template <int RM> cudaError_t gradients_of(const Layer& l, int b, int blocks, int warps, int ranges, cudaStream_t st) {
  const cudaError_t e = b == 2 ? launch_logits(few_logit_gradient_kernel<RM, 2>, l, RM, blocks, warps, st)
                               : launch_logits(few_logit_gradient_kernel<RM, many(RM)>, l, RM, blocks, warps, st);
  if (e != cudaSuccess || (!l.g.dx_part && !l.g.dw)) return e;
  const dim3 grid((unsigned)((l.warps_slots * 32 + kProductThreads - 1) / kProductThreads), (unsigned)ranges);
  return launch_behind(few_products_kernel<RM>, grid, kProductThreads, 0, st, l, (l.classes + ranges - 1) / ranges);
}

}  // namespace

cudaError_t few_rows_error_words(ErrorWords* words) { return cudaGetSymbolAddress(reinterpret_cast<void**>(&words->at[kErrorFewLabel]), g_few_label_error); }

bool few_rows(const vgg19_linear_loss& a, bool backward) {
  if (a.dtype != VGG19_FP32 || a.rows > (backward ? 8 : 24) || a.in > kMostKept / group_up(a)) return false;
  // Groups of eight: where a block's classes are worth the rows of x that it keeps (against 1000 classes of 4096 they take 23 us, the planes 20; of 2048 14.7
  // and 16), and w's rows are worth reading for every group (64 inputs against 131072: 61 and 41 us; three groups of 300 against 100003: 129 and 118).
  return a.rows <= 8 || (a.in >= (a.rows <= 16 ? 256 : 512) && a.classes >= a.in / 3);
}

int few_rows_blocks(const vgg19_linear_loss& a, int sms) {
  const int per = classes_at_once(a, sms) * warps_of(a, sms), batches = (a.classes + per - 1) / per;
  const int most = (kept_values(a) > 24576 ? 1 : 2) * (sms / groups(a));  // (one block's rows are all that an SM has room for, or two blocks' are not)
  return batches < most ? batches : most;
}

// Ranges of classes: enough blocks for every SM to have sixteen warps, of at least eight classes each.
int few_rows_ranges(const vgg19_linear_loss& a, int sms) {
  const int columns = ((a.in + 32 * kV - 1) / (32 * kV) * 32 + kProductThreads - 1) / kProductThreads;
  int ranges = (4 * sms + columns - 1) / columns;
  if (ranges > (a.classes + 7) / 8) ranges = (a.classes + 7) / 8;
  const int range = (a.classes + ranges - 1) / ranges;
  return (a.classes + range - 1) / range;  // none is empty
}

cudaError_t few_rows_loss(const vgg19_linear_loss& a, float2* part, float* label_z, int sms, cudaStream_t st) {
  Layer l = layer_of(a);
  l.part = part; l.label_z = label_z;
  const int b = classes_at_once(a, sms), blocks = few_rows_blocks(a, sms), warps = warps_of(a, sms);
  switch (group_up(a)) {
    case 1: return loss_of<1>(l, b, blocks, warps, st);
    case 2: return loss_of<2>(l, b, blocks, warps, st);
    case 4: return loss_of<4>(l, b, blocks, warps, st);
    default: return loss_of<8>(l, b, blocks, warps, st);
  }
}

cudaError_t few_rows_gradients(const vgg19_linear_loss& a, const FewGradients& g, int sms, cudaStream_t st) {
  Layer l = layer_of(a);
  l.g = g;
  if (l.aligned && reinterpret_cast<uintptr_t>(g.dw) % 16 == 0 && (a.classes == 1 || g.dw_ld % 4 == 0)) l.aligned = 2;  // dw too
  const int b = classes_at_once(a, sms), blocks = few_rows_blocks(a, sms), warps = warps_of(a, sms), ranges = few_rows_ranges(a, sms);
  switch (few_rows_up(l.rows)) {
    case 1: return gradients_of<1>(l, b, blocks, warps, ranges, st);
    case 2: return gradients_of<2>(l, b, blocks, warps, ranges, st);
    case 4: return gradients_of<4>(l, b, blocks, warps, ranges, st);
    default: return gradients_of<8>(l, b, blocks, warps, ranges, st);
  }
}

}  // namespace vgg
