// Dropout from a counter-based generator: y = x * keep / (1 - q), keep_e = [u_e >= t], q = t / 65536, where u_e are 16 bits of Philox 4x32
// with ten rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): a block
// of four words from the counter (e / 8, step) under the seed as key.  The mask is never stored: the gradient computes it again.
//
// Reading x and writing y is what it cannot do without.  Ten rounds are 20 products of 32 x 32 -> 64 bits and 20 three-way exclusive ors
// (the keys of the rounds are the same for all and come as constants); one value a word would make 10 instructions a
// value of that, beside 5 for the value itself, which is what bf16 at the memory's rate leaves; 16 bits a value make it 5, and
// rates in steps of 2^-16.
//
// Measured (B200): 4096 x 25088 bf16 in 69.6 us, 5.9 TB/s, where a copy of it takes 65.8 and the kernel without the generator 63.9; 1001 rows of
// 4099 fp32, 4112 apart, which no block of the generator is aligned with, in 10.1 us (5.0 by the bytes).
#include <cuda_runtime.h>

#include <cmath>

#include "../../include/vgg19_b200.h"
#include "common.cuh"

namespace vgg {
namespace {

struct Args {
  const void* x;
  void* y;
  long ldx, ldy, rows, cols, count;  // count: rows * cols
  const unsigned long long* step_counter;
  unsigned long long step, first;
  uint32_t limit;  // t << 16; a value stays where its 16 bits, moved up, are at least this
  int none;        // t == 65536: nothing stays
  float scale;
  uint32_t key[20];  // of the ten rounds, two words each
};

__device__ __forceinline__ uint4 philox(const Args& a, unsigned long long block, unsigned long long step) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)step, c3 = (uint32_t)(step >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long p = (unsigned long long)0xD2511F53u * c0, q = (unsigned long long)0xCD9E8D57u * c2;
    c0 = (uint32_t)(q >> 32) ^ c1 ^ a.key[2 * r];
    c1 = (uint32_t)q;
    c2 = (uint32_t)(p >> 32) ^ c3 ^ a.key[2 * r + 1];
    c3 = (uint32_t)p;
  }
  return a.none ? make_uint4(0, 0, 0, 0) : make_uint4(c0, c1, c2, c3);
}
// Of a word of the block: whether its two values stay.  (Where none does, the words are 0 and the limit is not.)
__device__ __forceinline__ bool low_stays(const Args& a, uint32_t w) { return (w << 16) >= a.limit; }
__device__ __forceinline__ bool high_stays(const Args& a, uint32_t w) { return w >= a.limit; }
__device__ __forceinline__ unsigned long long step_of(const Args& a) { return a.step + (a.step_counter ? *a.step_counter : 0ull); }

// (x may be y: no __restrict__, and every value is read before it is written, by the thread that writes it)
template <typename T> struct Eight;
template <> struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = reinterpret_cast<const float4*>(p)[0]; b = reinterpret_cast<const float4*>(p)[1]; }
  __device__ __forceinline__ void apply(const Args& d, const uint4& u) {
    a.x = low_stays(d, u.x) ? a.x * d.scale : 0.f; a.y = high_stays(d, u.x) ? a.y * d.scale : 0.f;
    a.z = low_stays(d, u.y) ? a.z * d.scale : 0.f; a.w = high_stays(d, u.y) ? a.w * d.scale : 0.f;
    b.x = low_stays(d, u.z) ? b.x * d.scale : 0.f; b.y = high_stays(d, u.z) ? b.y * d.scale : 0.f;
    b.z = low_stays(d, u.w) ? b.z * d.scale : 0.f; b.w = high_stays(d, u.w) ? b.w * d.scale : 0.f;
  }
  __device__ __forceinline__ void store(float* p) const { reinterpret_cast<float4*>(p)[0] = a; reinterpret_cast<float4*>(p)[1] = b; }
};
template <> struct Eight<bf16> {
  uint4 v;
  __device__ __forceinline__ void load(const bf16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void apply(const Args& d, const uint4& u) {
    const uint32_t r[4] = {u.x, u.y, u.z, u.w};
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float lo = low_stays(d, r[j]) ? __uint_as_float(w[j] << 16) * d.scale : 0.f, hi = high_stays(d, r[j]) ? __uint_as_float(w[j] & 0xffff0000u) * d.scale : 0.f;
      const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
      w[j] = *reinterpret_cast<const uint32_t*>(&h);
    }
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void store(bf16* p) const { *reinterpret_cast<uint4*>(p) = v; }
};

constexpr int kThreads = 256;

// Blocks of eight values that lie together and aligned: whole vectors.  One "row" where rows follow one another without gaps;
// the last block of all may then be short.
template <typename T, int UNROLL>
__global__ void __launch_bounds__(kThreads) dropout_vector_kernel(const __grid_constant__ Args a, long blocks, unsigned blocks_a_row) {
  const unsigned long long step = step_of(a);
  const long q0 = (long)blockIdx.x * (kThreads * UNROLL) + threadIdx.x;
  Eight<T> v[UNROLL];
  long ax[UNROLL], ay[UNROLL];
  const long whole = blocks_a_row ? blocks : a.count / 8;
#pragma unroll
  for (int i = 0; i < UNROLL; ++i) {
    const long q = q0 + i * kThreads;
    if (blocks_a_row) {
      const long r = (unsigned long)q < 0x100000000ul ? (unsigned)q / blocks_a_row : q / blocks_a_row, c = q - r * blocks_a_row;
      ax[i] = r * a.ldx + 8 * c;
      ay[i] = r * a.ldy + 8 * c;
    } else {
      ax[i] = ay[i] = 8 * q;
    }
    if (q < whole) v[i].load(static_cast<const T*>(a.x) + ax[i]);
  }
#pragma unroll
  for (int i = 0; i < UNROLL; ++i) {
    const long q = q0 + i * kThreads;
    if (q >= blocks) break;
    const uint4 u = philox(a, a.first / 8 + q, step);
    if (q < whole) {
      v[i].apply(a, u);
      v[i].store(static_cast<T*>(a.y) + ay[i]);
    } else {
      const T* x = static_cast<const T*>(a.x) + ax[i];
      T* y = static_cast<T*>(a.y) + ay[i];
      const uint32_t r[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < a.count - 8 * q) y[j] = from_f32<T>((j & 1 ? high_stays(a, r[j / 2]) : low_stays(a, r[j / 2])) ? to_f32(x[j]) * a.scale : 0.f);
    }
  }
}

// Any rows, strides and beginnings: a warp takes 256 values, 32 blocks of the generator, one a lane, and its accesses run
// along the rows.  I: a type that counts all that the rows span.
template <typename T, typename I>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const __grid_constant__ Args a, long groups) {
  const unsigned long long step = step_of(a);
  const int lane = threadIdx.x & 31;
  const long warps = (long)gridDim.x * (kThreads / 32);
  const int lead = (int)(a.first % 256);
  const I cols = (I)a.cols, count = (I)a.count, ldx = (I)a.ldx, ldy = (I)a.ldy;
  for (long g = (long)blockIdx.x * (kThreads / 32) + threadIdx.x / 32; g < groups; g += warps) {
    const I e0 = (I)(g * 256 - lead + lane);  // the lane's first value; before 0 and from count on there is none
    T v[8];
    I ay[8];
    I r = 0, c = e0;  // (of a value before 0: it will be in the first row, or be divided anew)
    if (e0 >= cols) {
      r = e0 / cols;
      c = e0 - r * cols;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const I e = e0 + 32 * i;
      ay[i] = -1;
      if (e >= 0 && e < count) {
        v[i] = static_cast<const T*>(a.x)[r * ldx + c];
        ay[i] = r * ldy + c;
      }
      c += 32;
      if (c >= cols) {
        if (cols >= 32) {
          c -= cols;
          ++r;
        } else {
          const I more = c / cols;
          c -= more * cols;
          r += more;
        }
      }
    }
    const uint4 u = philox(a, (a.first / 256 + g) * 32 + lane, step);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint32_t mine = 0;  // bit j: whether value j of the lane's block stays
#pragma unroll
    for (int j = 0; j < 4; ++j) mine |= (low_stays(a, w[j]) ? 1u << (2 * j) : 0u) | (high_stays(a, w[j]) ? 2u << (2 * j) : 0u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t m = __shfl_sync(0xffffffffu, mine, 4 * i + lane / 8);
      if (ay[i] >= 0) static_cast<T*>(a.y)[ay[i]] = from_f32<T>(m >> (lane % 8) & 1 ? to_f32(v[i]) * a.scale : 0.f);
    }
  }
}

template <typename T> cudaError_t launch(const Args& a, cudaStream_t st) {
  auto aligned = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
  const bool dense = (a.ldx == a.cols && a.ldy == a.cols) || a.rows == 1;
  const bool even = a.cols % 8 == 0 && a.ldx * sizeof(T) % 16 == 0 && a.ldy * sizeof(T) % 16 == 0;
  if (aligned(a.x) && aligned(a.y) && a.first % 8 == 0 && (dense || even)) {
    constexpr int UNROLL = sizeof(T) == 2 ? 4 : 2;
    const long blocks = (a.count + 7) / 8;
    const long per = kThreads * UNROLL;
    dropout_vector_kernel<T, UNROLL><<<(unsigned)((blocks + per - 1) / per), kThreads, 0, st>>>(a, blocks, dense ? 0u : (unsigned)(a.cols / 8));
  } else {
    const long groups = (a.count + (long)(a.first % 256) + 255) / 256, blocks = (groups + kThreads / 32 - 1) / (kThreads / 32);
    const unsigned grid = (unsigned)(blocks < 148 * 64 ? blocks : 148 * 64);
    if (a.rows * (a.ldx > a.ldy ? a.ldx : a.ldy) < (1L << 31) - 1024) dropout_kernel<T, int><<<grid, kThreads, 0, st>>>(a, groups);
    else dropout_kernel<T, long><<<grid, kThreads, 0, st>>>(a, groups);
  }
  return cudaGetLastError();
}

__global__ void count_up_kernel(unsigned long long* counter, unsigned long long by) { *counter += by; }

}  // namespace

cudaError_t count_up(unsigned long long* counter, unsigned long long by, cudaStream_t st) {
  count_up_kernel<<<1, 1, 0, st>>>(counter, by);
  return cudaGetLastError();
}

cudaError_t dropout(const void* x, bool half, long rows, long cols, long ldx, float rate, unsigned long long seed, unsigned long long step,
                    const unsigned long long* step_counter, unsigned long long first, void* y, long ldy, cudaStream_t st) {
  Args a{};
  a.x = x; a.y = y; a.ldx = ldx; a.ldy = ldy; a.rows = rows; a.cols = cols; a.count = rows * cols;
  a.step_counter = step_counter; a.step = step; a.first = first;
  const uint32_t t = (uint32_t)std::floor((double)rate * 65536.0 + 0.5);
  a.none = t >= 65536;
  a.limit = a.none ? 0xffffffffu : t << 16;
  a.scale = a.none ? 0.f : (float)(65536.0 / (65536.0 - t));
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
  for (int r = 0; r < 10; ++r) {
    a.key[2 * r] = k0;
    a.key[2 * r + 1] = k1;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return half ? launch<bf16>(a, st) : launch<float>(a, st);
}

namespace {
int checked(const void* x, int32_t dtype, int64_t rows, int32_t cols, int64_t ldx, float rate, uint64_t seed, uint64_t step,
            const uint64_t* step_counter, uint64_t first, void* y, int64_t ldy, void* stream) {
  if (dtype != VGG19_FP32 && dtype != VGG19_BF16) return note_error(VGG19_ERR_ARG, "dtype %d is neither VGG19_FP32 nor VGG19_BF16", dtype);
  if (rows < 0 || cols < 1 || rows > (1LL << 40) / cols)
    return note_error(VGG19_ERR_SHAPE, "%lld rows of %d values: at most 2^40 values", (long long)rows, cols);
  if (ldx < cols || ldy < cols || ldx >= (1LL << 40) || ldy >= (1LL << 40))
    return note_error(VGG19_ERR_SHAPE, "row strides %lld and %lld for %d values", (long long)ldx, (long long)ldy, cols);
  if (first >= 1ull << 62) return note_error(VGG19_ERR_ARG, "the first value's number is not below 2^62");
  if (!(rate >= 0.f && rate <= 1.f)) return note_error(VGG19_ERR_ARG, "rate %g outside [0, 1]", (double)rate);
  if (rows == 0) return VGG19_OK;
  if (!x || !y) return note_error(VGG19_ERR_ARG, "null input or output");
  const long elt = dtype == VGG19_FP32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(x) % elt || reinterpret_cast<uintptr_t>(y) % elt || reinterpret_cast<uintptr_t>(step_counter) % 8)
    return note_error(VGG19_ERR_ARG, "a pointer is not aligned to its type");
  if (!(x == y && (ldx == ldy || rows == 1)) && rows_meet(x, rows, cols * elt, ldx * elt, y, rows, cols * elt, ldy * elt))
    return note_error(VGG19_ERR_ARG, "the output overlaps the input without being the same rows");
  if (rows_meet(y, rows, cols * elt, ldy * elt, step_counter, step_counter != nullptr, 8, 0)) return note_error(VGG19_ERR_ARG, "the output overlaps the step counter");
  const cudaError_t e = dropout(x, dtype == VGG19_BF16, rows, cols, ldx, rate, seed, step, reinterpret_cast<const unsigned long long*>(step_counter), first, y, ldy,
                                static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? VGG19_OK : note_error(VGG19_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}
}  // namespace

}  // namespace vgg

extern "C" int vgg19_dropout(const void* x, int32_t dtype, int64_t rows, int32_t cols, int64_t ldx, float rate, uint64_t seed, uint64_t step,
                             const uint64_t* step_counter, uint64_t first, void* y, int64_t ldy, void* stream) {
  return vgg::checked(x, dtype, rows, cols, ldx, rate, seed, step, step_counter, first, y, ldy, stream);
}

extern "C" int vgg19_dropout_backward(const void* dy, int32_t dtype, int64_t rows, int32_t cols, int64_t lddy, float rate, uint64_t seed, uint64_t step,
                                      const uint64_t* step_counter, uint64_t first, void* dx, int64_t lddx, void* stream) {
  return vgg::checked(dy, dtype, rows, cols, lddy, rate, seed, step, step_counter, first, dx, lddx, stream);
}
