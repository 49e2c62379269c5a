// Shared declarations of the VGG19 device library: status codes, small
// device helpers, and the host-side launch functions each .cu file exports
// to the pass scheduler in vgg19_api.cu.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/vgg19_b200.h"

namespace vgg {

typedef __nv_bfloat16 bf16;

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_f32<bf16>(float v) { return __float2bfloat16_rn(v); }

// Device-side error word (one per network).  A kernel whose bounded wait ran
// out stores a nonzero code here and returns; the host reads it at
// vgg19_sync_status().
enum DeviceError : int {
  kDevOk = 0,
  kDevTimeoutTmaFull = 1,   // consumer waited too long for a TMA stage
  kDevTimeoutStageFree = 2, // producer waited too long for a free stage
  kDevTimeoutAccum = 3,     // epilogue waited too long for the accumulator
  kDevTimeoutTmemFree = 4,  // MMA issuer waited too long for a drained accumulator
  kDevTimeoutTest = 5,      // the self-test kernel's wait on a barrier nobody arrives on
  kDevBadLabel = 64,        // a label outside [0, classes): not a timeout, reported as a bad argument
  kDevSplitRange = 65,      // fp32 configuration on tensor cores: an activation beyond fp16's range
};

// A wait gives up after this long (far above any tile's duration, profiler
// replays included), records a DeviceError code and lets the CTA drain.
constexpr long long kWaitLimitCycles = 4000ll * 1000ll * 1000ll;  // about two seconds of SM clock

// How the waits of an operator's kernels end when what they wait for does not come, and where that is recorded: in a network's error word for
// its own calls, in the operator's for calls without a handle (null).  A copy's barrier expects `signals` signals and gets one: two, and
// the waits are certain to run out, for the self-test.
struct Waits {
  int* error = nullptr;
  long long limit_cycles = kWaitLimitCycles;
  int signals = 1;
};

// Sets the text vgg19_last_error(NULL) gives and returns `code`: for entry points without a handle.
int note_error(int code, const char* fmt, ...);

// Whether `n` rows of `bytes` each, `pitch` bytes apart, meet m rows of other_bytes, other_pitch apart (pitches at least the rows).
// Rows of one pitch may lie between one another; otherwise what counts is the range, save that a single row may lie between.
inline bool rows_meet(const void* a, long n, long bytes, long pitch, const void* b, long m, long other_bytes, long other_pitch) {
  if (!a || !b || n < 1 || m < 1) return false;
  if (m == 1) other_pitch = pitch;
  if (n == 1) pitch = other_pitch;
  const long x = (long)reinterpret_cast<uintptr_t>(a), y = (long)reinterpret_cast<uintptr_t>(b);
  if (x + (n - 1) * pitch + bytes <= y || y + (m - 1) * other_pitch + other_bytes <= x) return false;
  if (pitch != other_pitch || pitch < 1) return true;
  const long d = ((y - x) % pitch + pitch) % pitch;  // where b's rows start between a's
  return d < bytes || d + other_bytes > pitch;
}

// Bytes from p on; none where p is null.
struct Span {
  const void* p;
  long bytes;
};
// Whether one of the first `written` of them meets any other.
template <int M> inline bool spans_meet(const Span (&all)[M], int written) {
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < M; ++j)
      if (rows_meet(all[i].p, all[i].bytes > 0, all[i].bytes, 0, all[j].p, all[j].bytes > 0, all[j].bytes, 0)) return true;
  return false;
}

// Waits for the stream; *code becomes the device error word's value and the word 0, in one exchange on the device: what a kernel on another
// stream records meanwhile is either taken or left for the next status.  word[1] is the exchange's own.  One host thread at a time.
cudaError_t take_error(int* word, int* code, cudaStream_t st);
// The same for the words of calls without a handle (logprobs.cu, q4_dense.cu, muon.cu), on the current device.
cudaError_t logprobs_take_error(int* code, cudaStream_t st);
cudaError_t q4_take_error(int* code, cudaStream_t st);
cudaError_t muon_take_error(int* code, cudaStream_t st);

// vgg19_muon_update with the waits of its kernels (muon.cu).
int muon_update(const vgg19_muon_tensor* tensors, int32_t count, float lr, float momentum, float decay, int32_t steps, int32_t nesterov,
                void* workspace, size_t bytes, const Waits& products, const Waits& small_steps, void* stream);

// m <- mu m + g, w <- w - lr (g + mu m or m), w16 the rounded copy (or null), for each vector (muon.cu).
struct MuonVector {
  const float* grad;
  float *momentum, *w;
  bf16* w16;
  int n;
};
cudaError_t muon_vector_update(const MuonVector* v, int count, float lr, float mu, bool nesterov, cudaStream_t st);

// Dense layers over 4-bit weights (q4_dense.cu; layout and formulas in the public header).  T: type of w, x and y.
size_t q4_code_bytes(int out, int in);
size_t q4_scale_bytes(int out, int in, int group);
template <typename T>
cudaError_t q4_pack(const T* w, long ld, int out, int in, int group, void* codes, void* scales, cudaStream_t st);
template <typename T>
cudaError_t q4_linear(const T* x, long ldx, long rows, int in, const void* codes, const void* scales, int out, int group,
                      const float* bias, bool relu, T* y, float* y_f32, const Waits& waits, cudaStream_t st);

// ---- CUDA-core kernels (simt_kernels.cu) ---------------------------------
// T is the storage type of activations and weights (float or bf16); every
// sum is accumulated in fp32.

struct ConvShape {
  int N, H, W, Cin, Cout;
};

// out = [relu](conv3x3(in, wt) + bias) [* (mask > 0)], NHWC, wt [Cout][3][3][Cin].
template <typename T>
cudaError_t simt_conv3x3(const T* in, const T* wt, const float* bias, const T* mask, T* out,
                         ConvShape s, bool relu, cudaStream_t st);

// dW[k][r][s][c] = sum_p dz[p][k] x[p+(r-1,s-1)][c]; db[k] = sum_p dz[p][k].
// partial: fp32 scratch of simt_wgrad_scratch_elems() elements.
size_t simt_wgrad_scratch_elems(ConvShape s);
template <typename T>
cudaError_t simt_conv3x3_wgrad(const T* x, const T* dz, float* dW, float* db, float* partial,
                               ConvShape s, cudaStream_t st);

// db[c] = sum_p dz[p][c]; partial: fp32 scratch of at least 1024 * C elements.
template <typename T>
cudaError_t simt_bias_grad(const T* dz, float* db, float* partial, long P, int C, cudaStream_t st);
// db[o] = sum_m dY[m][o]
template <typename T>
cudaError_t simt_dense_db(const T* dY, float* db, int M, int Out, cudaStream_t st);

// y = max over 2x2 windows (stride 2) of x, NHWC.  code (or null), one byte per element of y: where the
// window's maximum sits, 0..3 in the order (0,0), (0,1), (1,0), (1,1), the first one on ties; 4 when the
// maximum is not positive (the ReLU that produced x passes no gradient to this window).
template <typename T>
cudaError_t simt_maxpool_fwd(const T* x, T* y, int N, int H, int W, int C, cudaStream_t st, uint8_t* code = nullptr);

// Pool scatter from the stored codes: dy[n][2i + a][2j + b][c] = dp[n][i][j][c] where code = 2a + b,
// 0 elsewhere (and everywhere for code 4): select-and-scatter fused with the ReLU mask below it,
// without reading the activation again.  H, W are the full-resolution sizes.
template <typename T>
cudaError_t simt_pool_scatter(const uint8_t* code, const T* dp, T* dy, int N, int H, int W, int C, cudaStream_t st);

// dy[pos] = dp[window] where pos is the window's first maximum of y and
// y[pos] > 0, else 0 (pool scatter fused with the ReLU mask of the layer that
// produced y).
template <typename T>
cudaError_t simt_maxpool_bwd_relu(const T* y, const T* dp, T* dy, int N, int H, int W, int C,
                                  cudaStream_t st);

// C[m][n] = epilogue(sum_k A[m][k] * B[n][k]); A [M][K] and B [N][K] row-major.
// Epilogue: + bias[n], ReLU, * (mask[m][n] > 0); written as T (out_t) and/or fp32 (out_f).
template <typename T>
cudaError_t simt_dense_nt(const T* A, const T* B, const float* bias, const T* mask, T* out_t,
                          float* out_f, int M, int N, int K, bool relu, cudaStream_t st);

// dX[m][i] = (sum_o dY[m][o] * W[o][i]) * (mask[m][i] > 0)      (W [Out][In] row-major)
template <typename T>
cudaError_t simt_dense_dx(const T* dY, const T* W, const T* mask, T* dX, int M, int In, int Out,
                          cudaStream_t st);

// dW[o][i] = sum_m dY[m][o] * X[m][i];  db[o] = sum_m dY[m][o]   (fp32 out)
template <typename T>
cudaError_t simt_dense_dw(const T* dY, const T* X, float* dW, float* db, int M, int In, int Out,
                          cudaStream_t st);

// Row-wise softmax of fp32 logits (probs may be null), and for the backward
// pass the per-row loss and dlogits = (p - onehot(label)) / rows, stored as T.
// A label outside [0, classes) is never dereferenced: the row's loss becomes NaN and kDevBadLabel is
// recorded in dev_error (when given).
template <typename T>
cudaError_t softmax_xent(const float* logits, const int32_t* labels, float* probs, T* dlogits,
                         float* row_loss, float* loss, int rows, int classes, cudaStream_t st,
                         int* dev_error = nullptr);

// fp32 -> T copy (weights), and the dgrad filter: wt_t[c][r][s][k] = w[k][2-r][2-s][c].
template <typename T>
cudaError_t convert_f32(const float* src, T* dst, size_t n, cudaStream_t st);
// Where the filters of layers 2..16 sit: in the flat fp32 parameter buffer (w_off) and in the three
// bf16 copy buffers (copy_off, the same in each); first[l] = number of 32 x 32 tiles (per tap, of the
// [Cout][Cin] matrix) before layer l, total = all tiles.  Cin and Cout are multiples of 32.
struct FilterCopyTable {
  int layers;
  long total;
  long first[16];
  long w_off[16];
  long copy_off[16];
  int Cin[16], Cout[16];
};
// Rebuilds, from the fp32 master, the rotated filters of the input gradients ([Cin][3][3][Cout], rotated
// by 180 degrees), the tap-major filters [9][Cout][Cin] and the rotated tap-major filters [9][Cin][Cout]
// of every layer in the table, all bf16, in one launch.
cudaError_t refresh_filter_copies(const float* params, bf16* dgrad_w, bf16* tap_fwd, bf16* tap_bwd,
                                  const FilterCopyTable& tab, cudaStream_t st);

// params -= lr * grads (fp32 master, in place); params_t (the storage-type copy, or null when T is
// float and the master is the copy) receives the rounded result in the same pass.  With lr_dev the
// rate is read from that device scalar instead of `lr` (a recorded graph keeps working when it changes).
template <typename T>
cudaError_t sgd_update(float* params, const float* grads, T* params_t, float lr, size_t n, cudaStream_t st,
                       const float* lr_dev = nullptr);
cudaError_t set_scalar(float* dst, float v, cudaStream_t st);
template <typename T>
cudaError_t make_dgrad_filter(const float* w, T* wt_t, int Cin, int Cout, cudaStream_t st);

// fp32 tensors as pairs of fp16 terms (split_kernels.cu): a row of C values as [hi | lo], hi = fp16(v),
// lo = fp16(v - hi), the same bytes as the fp32 row (the 16-bit words are passed as `half16`).  split_rows /
// merge_rows convert between the forms (dst may be src); C must divide 4096; a value beyond fp16's range sets
// kDevSplitRange in *dev_error.  maxpool_split pools [N][H][W][2C]; with rows_per_image the output is one row
// [all hi | all lo] per image, the form a dense layer reads.  split_weights turns rows of K weights, scaled
// by kSplitWeightScale, into rows [hi | lo | hi] of 3K.
typedef unsigned short half16;
// Weights are split after scaling by this power of two (exact), so that the lo terms of weights around 1e-2
// stay above fp16's smallest normal number; the kernels that multiply by them scale their sums back.
constexpr float kSplitWeightScale = 64.f;
bool split_rows_supported(int C);
cudaError_t split_rows(const float* src, half16* dst, long rows, int C, int* dev_error, cudaStream_t st);
cudaError_t merge_rows(const half16* src, float* dst, long rows, int C, cudaStream_t st);
cudaError_t maxpool_split(const half16* x, half16* y, int N, int H, int W, int C, bool rows_per_image, cudaStream_t st);
cudaError_t split_weights(const float* w, half16* out, long rows, int K, cudaStream_t st);

}  // namespace vgg
