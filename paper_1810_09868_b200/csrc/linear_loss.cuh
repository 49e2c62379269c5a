// What the two halves of the last layer with its loss share: linear_loss.cu (tiles on the tensor cores, and the entry points) and
// linear_loss_few.cu (a few rows on the CUDA cores).
#pragma once

#include "common.cuh"

namespace vgg {

constexpr float kLossLog2e = 1.4426950408889634f;

// A launch's kernel may be set up while the one before it in the stream ends; what it reads is there from here on.
__device__ __forceinline__ void behind_previous() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}
__device__ __forceinline__ float fast_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Statistics of some logits, (m, s): the largest and the sum of exp(z - m); of none: (-inf, 0).  A NaN stays in s.
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  if (m == -INFINITY) return make_float2(m, a.y + b.y);
  return make_float2(m, a.y * fast_exp2((a.x - m) * kLossLog2e) + b.y * fast_exp2((b.x - m) * kLossLog2e));
}

// A launch whose set-up overlaps the one before it in the stream (the kernels wait for that one themselves).
template <typename... A>
cudaError_t launch_clusters(void (*kernel)(A...), unsigned cluster, dim3 blocks, int threads, int smem, cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = blocks;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2] = {};
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
template <typename... A>
cudaError_t launch_behind(void (*kernel)(A...), dim3 blocks, int threads, int smem, cudaStream_t st, const A&... args) {
  return launch_clusters(kernel, 1, blocks, threads, smem, st, args...);
}

// ---- a few rows of fp32 (linear_loss_few.cu) ------------------------------------------------------------------------------
constexpr int few_rows_up(int rows) { return rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : 8; }
// Whether a layer is taken this way, for its loss or (backward) its gradients; the blocks of which each leaves statistics of its own, and the ranges of classes that dx is added up from.
bool few_rows(const vgg19_linear_loss& a, bool backward);
int few_rows_blocks(const vgg19_linear_loss& a, int sms);
int few_rows_ranges(const vgg19_linear_loss& a, int sms);
// (largest, sum) of a block's logits at part[block * rows + r]; z at the label.
cudaError_t few_rows_loss(const vgg19_linear_loss& a, float2* part, float* label_z, int sms, cudaStream_t st);
// dz: scratch, [classes][few_rows_up(rows)]; dx_part: [ranges][rows][dx_ld], or null; dw, db or null.
struct FewGradients {
  const float *lse, *d_loss;
  float* dz;
  float* dx_part;
  long dx_ld;
  float* dw;
  long dw_ld;
  float* db;
};
cudaError_t few_rows_gradients(const vgg19_linear_loss& a, const FewGradients& g, int sms, cudaStream_t st);

}  // namespace vgg
