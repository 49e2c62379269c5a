// Dense layers over 4-bit weights with group scales, for a few rows at a time:
//   y[b][o] = act(sum_g s[o][g] * sum_{k in g} x[b][k] * (code[o][k] - 8) + bias[o]).
//
// For few rows the layer is bound by reading its weights, and 4 bits are a quarter of the bf16 copy's bytes.  What
// stands against that rate is unpacking: 64 codes per lane and KB.  So the products run on the tensor cores
// (mma.sync m16n8k16, bf16 operands, fp32 sums): a code becomes an exact bf16 value in 1.4 instructions, 16 rows of
// weights meet up to 8 rows of x per instruction, and the scale is applied once per group, in fp32, to the sum over
// the group (exact products, so nothing but the sums is rounded).  tcgen05 would need the codes unpacked into shared
// memory first, a round trip that costs more than the products.  fp32 activations travel as three bf16 terms that
// add up to them exactly, three products per product.
//
// Layout (made by q4_pack, documented in the header): blocks of 16 rows x 128 weights, 1 KB each, in which lane
// (g, t) of a warp finds with two 16-byte loads what its fragments need: row g (and g + 8), and in each of the four
// 32-weight groups the eight weights 8 t .. 8 t + 7.  All 16 weights of one instruction's K then lie in one group.
//
// A block owns RW tiles of 16 output rows over a share of K, one a warp or one for two warps that take turns.  Every warp
// has its own ring of bulk copies (four or eight blocks on their way, no registers held, no other warp waited for); the
// block's share of x is staged in shared memory meanwhile, once for all its rows.  The shares of a cluster join through
// distributed shared memory, in a fixed order: one launch, no scratch.
//
// Measured (B200, device time): 25088 -> 4096 in groups of 128 or 64, one row, bf16: 18.4 to 18.8 us, 2.8 TB/s.  No pipe is full there: issue slots 51 %,
// the integer pipe 45 % (76 instructions a KB to unpack), DRAM 29 %, 13 warps an SM (256 blocks on 148 SMs); the same copies without the products take
// 12 us, and a few of the 18 are x on its way and the cluster's meeting.  One row of fp32: 23.8 us; two of bf16 20.7; sixteen, groups of 64: 32 us, and as
// much again for every further sixteen; 4096 -> 4096, sixteen rows, groups of 32: 8.3 us, 2.4 of them until x is staged, 2.3 products, 2.2 joining;
// 6344 -> 11710, ten rows of fp32: 36 us, where the tensor cores (three terms, two tiles of rows: 48 products a KB at 8 cycles) are busy a third of the time.
// Packing 25088 x 4096 takes 249 us from fp32 or bf16 (by bytes 72 and 40): a warp's 128 weights in scalar loads and two-byte stores.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "../../include/vgg19_b200.h"
#include "tc_common.cuh"

namespace cg = cooperative_groups;

namespace vgg {
namespace {

using namespace tc;

static __device__ int g_q4_error[2];  // a DeviceError code once a bounded wait of a call without a handle ran out

constexpr int kTileRows = 16, kBlockK = 128, kBlockBytes = kTileRows * kBlockK / 2;
constexpr int kMaxRows = 16;                 // rows of x per launch
constexpr int kMaxKSplit = 8;

// Two codes, four nibbles apart, become a pair of bf16 values (code - 8) / 16: 0x4100 | code is 8 + code / 16.  (Sixteenths,
// so that no product is larger than its activation; the factor comes back with the last sum.)
__device__ __forceinline__ uint32_t codes_to_bf16x2(uint32_t w, uint32_t mask, uint32_t magic, uint32_t offset) {
  uint32_t v;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(v) : "r"(w), "r"(mask), "r"(magic));  // (w & mask) | magic
  asm("sub.bf16x2 %0, %0, %1;" : "+r"(v) : "r"(offset));
  return v;
}

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

struct Q4Args {
  const void* x;
  const uint4* codes;
  const uint16_t* scales;
  const float* bias;
  void* y;
  float* y_f32;
  long ldx;
  int in, out, rows, blocks, ksplit, stage_blocks, relu;
  Waits waits;
};

// The terms of eight consecutive activations, each a 16-byte row of bf16 in the order 0 4 1 5 2 6 3 7 (the order in
// which codes_to_bf16x2 yields them).  fp32: truncated to 8 bits three times, the rest exact each time.
template <typename T> struct Terms;
template <> struct Terms<bf16> {
  static constexpr int N = 1;
  __device__ static void split(const bf16* v, uint32_t (&out)[1][4]) {
    const uint16_t* h = reinterpret_cast<const uint16_t*>(v);
#pragma unroll
    for (int i = 0; i < 4; ++i) out[0][i] = (uint32_t)h[i] | (uint32_t)h[i + 4] << 16;
  }
};
template <> struct Terms<float> {
  static constexpr int N = 3;
  __device__ static void split(const float* v, uint32_t (&out)[3][4]) {
    uint32_t t[3][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = __float_as_uint(v[i]);
      const bool finite = (b & 0x7f800000u) != 0x7f800000u;
      const bool nan = (b & 0x7fffffffu) > 0x7f800000u;
      t[0][i] = nan ? 0x7fc0u : b >> 16;
      const float r1 = finite ? v[i] - __uint_as_float(b & 0xffff0000u) : 0.f;
      const uint32_t b1 = __float_as_uint(r1);
      t[1][i] = b1 >> 16;
      t[2][i] = __float_as_uint(r1 - __uint_as_float(b1 & 0xffff0000u)) >> 16;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) out[k][i] = t[k][i] | t[k][i + 4] << 16;
  }
};

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

// (volatile: stays where it is in the order of requests)
__device__ __forceinline__ uint4 load_now(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

constexpr int kRing = 2;  // copies on their way
template <int PER, int SLOT> __host__ __device__ constexpr int slot_bytes() { return SLOT * (kBlockBytes + kTileRows * PER * 2); }

// Resident blocks that registers are kept for, which is also how many the plan counts on (counting on three where there is room for two
// took 30.4 us for one row of fp32, 13196 -> 7140, where 20.8 are enough; 33.5 against 24.1 for thirteen of bf16, 4268 -> 14582).
template <typename T, int NT, int WARPS> constexpr int kResident = NT == 2 || Terms<T>::N == 3 ? 2 : 24 / WARPS;

// NT: tiles of eight rows of x.  GROUP: 32, 64 or 128 weights a scale.  RW x KW warps: row tiles, warps to a tile.  SLOT: blocks a copy.
template <typename T, int GROUP, int NT, int RW, int KW, int SLOT>
__global__ void __launch_bounds__(32 * RW * KW, kResident<T, NT, RW * KW>) q4_linear_kernel(const Q4Args a) {
  constexpr int TERMS = Terms<T>::N, PER = kBlockK / GROUP, USTEP = GROUP / 32, kThreads = 32 * RW * KW, STEP = KW * SLOT;
  extern __shared__ __align__(128) unsigned char smem[];  // the rings, then x
  __shared__ float part[KW][RW][NT * 8][kTileRows];
  __shared__ float inbox[RW * NT * 8 * kTileRows + kMaxKSplit];
  __shared__ __align__(8) unsigned long long bars[RW * KW][kRing];
  __shared__ int abort_flag, ran_out;  // (where that is recorded takes registers that the products want: found out once it happens)
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int ks = a.ksplit, rank = ks > 1 ? (int)cluster.block_rank() : 0;
  const int first_tile = blockIdx.x / ks * RW, tile = min(first_tile + warp % RW, (a.out - 1) / kTileRows);  // (a tile too many repeats the last)
  const int b0 = (int)((long)a.blocks * rank / ks), b1 = (int)((long)a.blocks * (rank + 1) / ks);
  const unsigned char* codes = reinterpret_cast<const unsigned char*>(a.codes) + (long)tile * a.blocks * kBlockBytes;
  const unsigned char* scales = reinterpret_cast<const unsigned char*>(a.scales) + (long)tile * a.blocks * (kTileRows * PER * 2);
  const unsigned char* ring = smem + warp * kRing * slot_bytes<PER, SLOT>();
  const uint32_t ring_u32 = smem_u32(ring), bar_u32 = smem_u32(&bars[warp][0]);
  unsigned char* staged = smem + RW * KW * kRing * slot_bytes<PER, SLOT>();
  const int stride = a.stage_blocks * kBlockK * 2 + 64;  // bytes of a staged row: rows 64 bytes apart modulo 128
  const int term_bytes = a.rows * stride;

  const int first = b0 + warp / RW * SLOT;  // this warp's blocks: a slot's, then those STEP further
  auto request = [&](int slot, int b) {  // lane 0: a slot's blocks of this warp's tile, from b
    const int n = min(SLOT, b1 - b);
    const uint32_t bar = bar_u32 + 8 * slot, dst = ring_u32 + slot * slot_bytes<PER, SLOT>();
    mbar_expect_tx(bar, n * (kBlockBytes + kTileRows * PER * 2));
    bulk_copy(dst, codes + (long)b * kBlockBytes, n * kBlockBytes, bar);
    bulk_copy(dst + SLOT * kBlockBytes, scales + (long)b * (kTileRows * PER * 2), n * (kTileRows * PER * 2), bar);
  };
  if (ks > 1) cluster.barrier_arrive();  // waited for before the first write into another block's shared memory
  if (tid == 0) abort_flag = ran_out = 0;

  float acc[NT][4] = {};
  int xrow[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) xrow[n] = min(n * 8 + g, a.rows - 1) * stride + t * 16;  // columns past the last row are not used

  // in registers, where an instruction can take all three
  uint32_t mask = 0x000f000fu, magic = 0x41004100u, offset = 0x41084108u;
  asm volatile("" : "+r"(mask), "+r"(magic), "+r"(offset));
  // one block of weights in the ring by the staged x of the same K
  auto multiply = [&](const unsigned char* wb, const unsigned char* sb, const unsigned char* xb) {
    const uint4 l4 = *reinterpret_cast<const uint4*>(wb + lane * 16), h4 = *reinterpret_cast<const uint4*>(wb + 512 + lane * 16);
    const uint32_t lo[4] = {l4.x, l4.y, l4.z, l4.w}, hi[4] = {h4.x, h4.y, h4.z, h4.w};
    const uint16_t *sl = reinterpret_cast<const uint16_t*>(sb) + g * PER, *sh = sl + 8 * PER;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      float d[NT][4] = {}, e[NT][4] = {};  // (two chains of products)
#pragma unroll
      for (int q = 0; q < USTEP; ++q) {
        const int v = p * USTEP + q;
        uint32_t al[4], ah[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          al[i] = codes_to_bf16x2(lo[v] >> (4 * i), mask, magic, offset);
          ah[i] = codes_to_bf16x2(hi[v] >> (4 * i), mask, magic, offset);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int m = TERMS - 1; m >= 0; --m) {  // the small terms first
            const uint4 xv = *reinterpret_cast<const uint4*>(xb + m * term_bytes + xrow[n] + v * 64);
            mma(d[n], al[0], ah[0], al[1], ah[1], xv.x, xv.y);
            mma(e[n], al[2], ah[2], al[3], ah[3], xv.z, xv.w);
          }
      }
      const float s0 = __uint_as_float((uint32_t)sl[p] << 16), s1 = __uint_as_float((uint32_t)sh[p] << 16);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        acc[n][0] = fmaf(d[n][0] + e[n][0], s0, acc[n][0]);
        acc[n][1] = fmaf(d[n][1] + e[n][1], s0, acc[n][1]);
        acc[n][2] = fmaf(d[n][2] + e[n][2], s1, acc[n][2]);
        acc[n][3] = fmaf(d[n][3] + e[n][3], s1, acc[n][3]);
      }
    }
  };

  int slot = 0;
  uint32_t phase = 0;
  bool ok = true;  // of this warp; one that gave up still meets the others
  for (int c0 = b0; c0 < b1; c0 += a.stage_blocks) {
    const int c1 = min(c0 + a.stage_blocks, b1);
    if (c0 != b0) __syncthreads();
    const int items = (c1 - c0) * (kBlockK / 8) * a.rows, n8 = (c1 - c0) * (kBlockK / 8);
    constexpr int BATCH = TERMS == 1 ? 4 : 2;  // rounds of requests before the first is used
    for (int i0 = tid; i0 < items || (c0 == b0 && i0 == tid); i0 += BATCH * kThreads) {
      T v[BATCH][8];
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const int i = i0 + u * kThreads;
        if (i < items) {
          const int row = a.rows == 1 ? 0 : i / n8, k = c0 * kBlockK + (i - row * n8) * 8;
          const T* src = static_cast<const T*>(a.x) + row * a.ldx + k;
          if (k + 8 <= a.in && (reinterpret_cast<uintptr_t>(src) & 15) == 0) {
#pragma unroll
            for (int j = 0; j < (int)(8 * sizeof(T) / 16); ++j) reinterpret_cast<uint4*>(v[u])[j] = load_now(reinterpret_cast<const uint4*>(src) + j);
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[u][j] = k + j < a.in ? src[j] : from_f32<T>(0.f);
          }
        }
      }
      // The weights are asked for behind the first of x, not before: x is little and everything waits for it (asked for
      // after them it came 2.5 us later).
      if (c0 == b0 && i0 == tid && lane == 0) {
        for (int s = 0; s < kRing; ++s) mbar_init(bar_u32 + 8 * s, a.waits.signals);
        mbar_fence_init();
        for (int s = 0; s < kRing; ++s)
          if (first + s * STEP < b1) request(s, first + s * STEP);
      }
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const int i = i0 + u * kThreads;
        if (i < items) {
          const int row = a.rows == 1 ? 0 : i / n8, k8 = i - row * n8;
          uint32_t o[TERMS][4];
          Terms<T>::split(v[u], o);
#pragma unroll
          for (int q = 0; q < TERMS; ++q)
            *reinterpret_cast<uint4*>(staged + q * term_bytes + row * stride + k8 * 16) = make_uint4(o[q][0], o[q][1], o[q][2], o[q][3]);
        }
      }
    }
    __syncthreads();
    for (int b = c0 + warp / RW * SLOT; b < c1; b += STEP) {  // (a part of x is a multiple of STEP, but for the last)
      if (!ok) break;
      ok = __all_sync(0xffffffffu, mbar_wait(bar_u32 + 8 * slot, phase, &abort_flag, &ran_out, kDevTimeoutTmaFull, a.waits.limit_cycles));
      if (!ok) {
        __syncwarp();  // (the lane that ran out has written its code)
        if (lane == 0 && ran_out) atomicCAS(a.waits.error ? a.waits.error : g_q4_error, 0, ran_out);
        // let what is on its way land before shared memory goes away
        if (lane == 0) {
          const unsigned long long t0 = global_timer_ns();
          for (int i = 0; i < kRing && b + i * STEP < b1; ++i) {
            while (!mbar_try_wait(bar_u32 + 8 * slot, phase) && global_timer_ns() - t0 < 100000000ull) {}
            if (++slot == kRing) { slot = 0; phase ^= 1; }
          }
        }
        break;
      }
      const unsigned char* w = ring + slot * slot_bytes<PER, SLOT>();
      const unsigned char *sc = w + SLOT * kBlockBytes, *xb = staged + (b - c0) * (kBlockK * 2);
#pragma unroll
      for (int u = 0; u < SLOT; ++u)
        if (b + u < c1) multiply(w + u * kBlockBytes, sc + u * (kTileRows * PER * 2), xb + u * (kBlockK * 2));
      __syncwarp();
      if (lane == 0 && b + kRing * STEP < b1) request(slot, b + kRing * STEP);
      if (++slot == kRing) { slot = 0; phase ^= 1; }
    }
  }

  // accumulator: rows g, g + 8 of the tile by columns 2 t, 2 t + 1 of the rows of x
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    part[warp / RW][warp % RW][n * 8 + 2 * t][g] = acc[n][0];
    part[warp / RW][warp % RW][n * 8 + 2 * t + 1][g] = acc[n][1];
    part[warp / RW][warp % RW][n * 8 + 2 * t][g + 8] = acc[n][2];
    part[warp / RW][warp % RW][n * 8 + 2 * t + 1][g + 8] = acc[n][3];
  }
  __syncthreads();
  // Results, a row of x at a time.  Every block of the cluster finishes a share of them: it gets the others' parts by their
  // writing them into its shared memory, so that one meeting of the cluster is enough.
  const int results = RW * a.rows * kTileRows, per = (results + ks - 1) / ks;
  auto sum_of = [&](int i) {
    const int o = i % kTileRows, r = i / kTileRows % RW, n = i / kTileRows / RW;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < KW; ++k) v += part[k][r][n][o];
    return v;
  };
  if (ks > 1) {
    cluster.barrier_wait();  // every block has started
    for (int i = tid; i < results; i += kThreads) cluster.map_shared_rank(inbox, i / per)[rank * per + i % per] = sum_of(i);
    cluster.sync();
  }
  for (int i = rank * per + tid; i < min(results, (rank + 1) * per); i += kThreads) {
    const int o = i % kTileRows, r = i / kTileRows % RW, n = i / kTileRows / RW, col = (first_tile + r) * kTileRows + o;
    if (col >= a.out) continue;
    float v = 0.f;
    if (ks > 1)
      for (int c = 0; c < ks; ++c) v += inbox[c * per + i - rank * per];
    else
      v = sum_of(i);
    v *= 16.f;
    if (a.bias) v += a.bias[col];
    if (a.relu) v = v < 0.f ? 0.f : v;  // a NaN stays
    if (a.y) static_cast<T*>(a.y)[(long)n * a.out + col] = from_f32<T>(v);
    if (a.y_f32) a.y_f32[(long)n * a.out + col] = v;
  }
}

// One warp per row and block of 128 weights, four consecutive weights per lane.
template <typename T>
__global__ void __launch_bounds__(256) q4_pack_kernel(const T* w, long ld, int out, int in, int blocks, int group, uint8_t* codes, bf16* scales) {
  const long item = (long)blockIdx.x * 8 + threadIdx.x / 32;
  const int lane = threadIdx.x & 31;
  const long total = (long)((out + kTileRows - 1) / kTileRows) * kTileRows * blocks;
  if (item >= total) return;
  const int b = (int)(item % blocks);
  const long row = item / blocks;
  const int k = b * kBlockK + lane * 4;
  float v[4] = {};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (row < out && k + j < in) v[j] = to_f32(w[row * ld + k + j]);
  float m = 0.f;
  bool nan = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) { m = fmaxf(m, fabsf(v[j])); nan |= v[j] != v[j]; }
  if (nan) m = INFINITY;  // a group with a NaN or an infinity gets an infinite scale: its row's results become NaN
  for (int o = 1; o < group / 4; o *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const bf16 sb = __float2bfloat16_rn(m / 7.f);
  const float s = __bfloat162float(sb);
  uint32_t c = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float q = s > 0.f && s < INFINITY ? rintf(v[j] / s) : 0.f;
    q = fminf(fmaxf(q, -8.f), 7.f);
    c |= (uint32_t)((int)q + 8) << (4 * j);
  }
  const int u = lane / 8, t = lane % 8 / 2;
  const long block = (row / kTileRows) * blocks + b;
  uint8_t* dst = codes + block * kBlockBytes + (row % kTileRows) * 64 + (4 * t + u) * 4 + (lane & 1) * 2;
  *reinterpret_cast<uint16_t*>(dst) = (uint16_t)c;
  if (lane % (group / 4) == 0) scales[(block * kTileRows + row % kTileRows) * (kBlockK / group) + lane / (group / 4)] = sb;
}

// A launch's shape, and an estimate of its time.
struct Plan {
  int ksplit, stage_blocks;
  size_t smem;
  double cost;
};

template <typename T, int GROUP, int NT, int RW, int KW, int SLOT> struct Shape {
  static constexpr int PER = kBlockK / GROUP, kRings = RW * KW * kRing * slot_bytes<PER, SLOT>(), STEP = KW * SLOT;
  static constexpr int kStatic = RW * (KW + 1) * NT * 8 * kTileRows * 4 + 512, kStage = SLOT == 4 ? 48 << 10 : 40 << 10;  // of x in shared memory at a time
  static_assert((KW == 1 ? kMaxRows * 3 : 2) * STEP * kBlockK * 2 <= kStage, "a step's part of x fits");

  // How many blocks share K.  A block of weights keeps a warp about twenty times as long as it keeps the SM's issue slots,
  // so an SM wants that many warps, and more only bring start-ups (three blocks' worth): the least estimated time wins.
  static Plan plan(const Q4Args& a) {
    const int groups = ((a.out + kTileRows - 1) / kTileRows + RW - 1) / RW, block_bytes = a.rows * Terms<T>::N * kBlockK * 2;
    Plan best{};
    for (int ks = 1; ks <= kMaxKSplit && ks <= a.blocks; ++ks) {
      const int share = (a.blocks + ks - 1) / ks, most = kStage / block_bytes / STEP * STEP, want = (share + STEP - 1) / STEP * STEP;
      const int stage = want < most ? want : most;
      const size_t smem = kRings + a.rows * Terms<T>::N * (stage * kBlockK * 2 + 64);
      const long n = (long)groups * ks, per = (share + KW - 1) / KW;
      long resident = (220 << 10) / (smem + kStatic + 1024);
      if (resident > kResident<T, NT, RW * KW>) resident = kResident<T, NT, RW * KW>;
      const long sms = ks > 2 ? 141 : 148, each = (n + sms - 1) / sms;  // (a cluster stays within a part of the GPU, and some of a part's SMs stay empty)
      const long rounds = (each + resident - 1) / resident, warps = (each < resident ? each : resident) * RW * KW;
      const double cost = rounds * (per + 3) * (warps > 20 ? warps : 20) * (SLOT == 4 ? 1.0 : 1.1);
      if (best.ksplit == 0 || cost < best.cost) best = Plan{ks, stage, smem, cost};
    }
    return best;
  }

  static cudaError_t launch(Q4Args a, const Plan& p, cudaStream_t st) {
    const int groups = ((a.out + kTileRows - 1) / kTileRows + RW - 1) / RW;
    a.ksplit = p.ksplit;
    a.stage_blocks = p.stage_blocks;
    auto kernel = q4_linear_kernel<T, GROUP, NT, RW, KW, SLOT>;
    if (p.smem + kStatic > (48 << 10)) {
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRings + kStage + kMaxRows * 3 * 64);
      if (e != cudaSuccess) return e;
    }
    if (a.ksplit == 1) {
      kernel<<<(unsigned)groups, 32 * RW * KW, p.smem, st>>>(a);
      return cudaGetLastError();
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(groups * a.ksplit));
    cfg.blockDim = dim3(32 * RW * KW);
    cfg.dynamicSmemBytes = p.smem;
    cfg.stream = st;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = (unsigned)a.ksplit;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a);
  }
};

// Copies of four blocks, whose products fill one another's gaps, or of two, a tenth slower, which leave shared memory for a
// second block per SM where x takes much of it: 4096 -> 4096 at sixteen rows takes 8.2 against 8.4 us, 6344 -> 11710 at
// ten rows of fp32 69 against 36.
template <typename T, int GROUP, int NT, int RW> cudaError_t launch_rows(const Q4Args& a, cudaStream_t st) {
  using Long = Shape<T, GROUP, NT, RW, 1, 4>;
  using Short = Shape<T, GROUP, NT, RW, 1, 2>;
  const Plan l = Long::plan(a), s = Short::plan(a);
  return l.cost <= s.cost ? Long::launch(a, l, st) : Short::launch(a, s, st);
}

// One or two rows of bf16 take blocks of four row tiles, two warps to a tile; the products of an fp32 row are three times as many, and with them blocks of eight
// win at the larger of a network's layers: 25088 -> 4096 takes 23.7 us against 28.5, 4096 -> 4096 6.9 against 7.1, 4096 -> 1000 5.1 against
// 5.4 (though 11710 -> 6344 25.4 against 23.0, 16000 -> 300 10.1 against 7.1).
template <typename T, int GROUP> cudaError_t launch_group(const Q4Args& a, cudaStream_t st) {
  if (a.rows > 8) return launch_rows<T, GROUP, 2, 8>(a, st);
  if constexpr (Terms<T>::N == 1) {
    using Few = Shape<T, GROUP, 1, 4, 2, 4>;
    if (a.rows <= 2) return Few::launch(a, Few::plan(a), st);
  }
  return launch_rows<T, GROUP, 1, 8>(a, st);
}

template <typename T> cudaError_t launch_type(const Q4Args& a, int group, cudaStream_t st) {
  return group == 32 ? launch_group<T, 32>(a, st) : group == 64 ? launch_group<T, 64>(a, st) : launch_group<T, 128>(a, st);
}

int shape_checks(int32_t out, int32_t in, int32_t group) {
  if (out < 1 || in < 1 || out > (1 << 24) || in > (1 << 24))
    return note_error(VGG19_ERR_SHAPE, "%d x %d weights: both sizes in [1, 2^24]", out, in);
  if (group != 32 && group != 64 && group != 128) return note_error(VGG19_ERR_ARG, "group %d is none of 32, 64, 128", group);
  return VGG19_OK;
}

}  // namespace

size_t q4_code_bytes(int out, int in) {
  return (size_t)((out + kTileRows - 1) / kTileRows) * ((in + kBlockK - 1) / kBlockK) * kBlockBytes;
}
size_t q4_scale_bytes(int out, int in, int group) {
  return (size_t)((out + kTileRows - 1) / kTileRows) * ((in + kBlockK - 1) / kBlockK) * kTileRows * (kBlockK / group) * 2;
}

template <typename T>
cudaError_t q4_pack(const T* w, long ld, int out, int in, int group, void* codes, void* scales, cudaStream_t st) {
  const int blocks = (in + kBlockK - 1) / kBlockK;
  const long items = (long)((out + kTileRows - 1) / kTileRows) * kTileRows * blocks;
  q4_pack_kernel<T><<<(unsigned)((items + 7) / 8), 256, 0, st>>>(w, ld, out, in, blocks, group, static_cast<uint8_t*>(codes),
                                                                static_cast<bf16*>(scales));
  return cudaGetLastError();
}

template <typename T>
cudaError_t q4_linear(const T* x, long ldx, long rows, int in, const void* codes, const void* scales, int out, int group,
                      const float* bias, bool relu, T* y, float* y_f32, const Waits& waits, cudaStream_t st) {
  for (long r = 0; r < rows; r += kMaxRows) {
    Q4Args a{};
    a.x = x + r * ldx;
    a.codes = static_cast<const uint4*>(codes);
    a.scales = static_cast<const uint16_t*>(scales);
    a.bias = bias;
    a.y = y ? y + r * out : nullptr;
    a.y_f32 = y_f32 ? y_f32 + r * out : nullptr;
    a.ldx = ldx; a.in = in; a.out = out; a.relu = relu;
    a.rows = (int)(rows - r < kMaxRows ? rows - r : kMaxRows);
    a.blocks = (in + kBlockK - 1) / kBlockK;
    a.waits = waits;
    const cudaError_t e = launch_type<T>(a, group, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t q4_take_error(int* code, cudaStream_t st) {
  void* word = nullptr;
  const cudaError_t e = cudaGetSymbolAddress(&word, g_q4_error);
  return e == cudaSuccess ? take_error(static_cast<int*>(word), code, st) : e;
}

#define INSTANTIATE(T)                                                                                                    \
  template cudaError_t q4_pack<T>(const T*, long, int, int, int, void*, void*, cudaStream_t);                             \
  template cudaError_t q4_linear<T>(const T*, long, long, int, const void*, const void*, int, int, const float*, bool, T*, \
                                    float*, const Waits&, cudaStream_t);
INSTANTIATE(float)
INSTANTIATE(bf16)

}  // namespace vgg

extern "C" {

size_t vgg19_q4_code_bytes(int32_t out, int32_t in) {
  return vgg::shape_checks(out, in, 32) == VGG19_OK ? vgg::q4_code_bytes(out, in) : 0;
}
size_t vgg19_q4_scale_bytes(int32_t out, int32_t in, int32_t group) {
  return vgg::shape_checks(out, in, group) == VGG19_OK ? vgg::q4_scale_bytes(out, in, group) : 0;
}

int vgg19_q4_pack(const void* w, int32_t dtype, int32_t out, int32_t in, int64_t ld, int32_t group, void* codes,
                  void* scales, void* stream) {
  using namespace vgg;
  const int rc = shape_checks(out, in, group);
  if (rc != VGG19_OK) return rc;
  if (dtype != VGG19_FP32 && dtype != VGG19_BF16)
    return note_error(VGG19_ERR_ARG, "dtype %d is neither VGG19_FP32 nor VGG19_BF16", dtype);
  if (!w || !codes || !scales) return note_error(VGG19_ERR_ARG, "weights, codes and scales must not be null");
  if (ld < in) return note_error(VGG19_ERR_SHAPE, "row stride %lld below %d", (long long)ld, in);
  if (reinterpret_cast<uintptr_t>(w) % (dtype == VGG19_FP32 ? 4 : 2) || reinterpret_cast<uintptr_t>(codes) % 16 ||
      reinterpret_cast<uintptr_t>(scales) % 16)
    return note_error(VGG19_ERR_ARG, "weights are aligned to their type, codes and scales to 16 bytes");
  if (((long)((out + kTileRows - 1) / kTileRows) * kTileRows * ((in + kBlockK - 1) / kBlockK) + 7) / 8 > 0x7fffffffL)
    return note_error(VGG19_ERR_SHAPE, "%d x %d weights are too many for one call", out, in);
  const long elt = dtype == VGG19_FP32 ? 4 : 2;
  const Span packed[] = {{codes, (long)q4_code_bytes(out, in)}, {scales, (long)q4_scale_bytes(out, in, group)}};
  if (spans_meet(packed, 1) || rows_meet(w, out, elt * in, elt * ld, codes, 1, packed[0].bytes, 0) ||
      rows_meet(w, out, elt * in, elt * ld, scales, 1, packed[1].bytes, 0))
    return note_error(VGG19_ERR_ARG, "codes and scales overlap the weights or one another");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == VGG19_BF16 ? q4_pack(static_cast<const bf16*>(w), ld, out, in, group, codes, scales, st)
                                            : q4_pack(static_cast<const float*>(w), ld, out, in, group, codes, scales, st);
  return e == cudaSuccess ? VGG19_OK : note_error(VGG19_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}

int vgg19_q4_linear(const void* x, int32_t dtype, int64_t rows, int32_t in, int64_t ldx, const void* codes,
                    const void* scales, int32_t out, int32_t group, const float* bias, int32_t relu, void* y,
                    float* y_f32, void* stream) {
  using namespace vgg;
  const int rc = shape_checks(out, in, group);
  if (rc != VGG19_OK) return rc;
  if (dtype != VGG19_FP32 && dtype != VGG19_BF16)
    return note_error(VGG19_ERR_ARG, "dtype %d is neither VGG19_FP32 nor VGG19_BF16", dtype);
  if (rows < 0 || rows > (1 << 20)) return note_error(VGG19_ERR_SHAPE, "%lld rows outside [0, 2^20]", (long long)rows);
  if (ldx < in) return note_error(VGG19_ERR_SHAPE, "row stride %lld below %d", (long long)ldx, in);
  if (rows == 0) return VGG19_OK;
  if (!x || !codes || !scales || (!y && !y_f32))
    return note_error(VGG19_ERR_ARG, "x, codes, scales and one of the outputs must not be null");
  const uintptr_t elt = dtype == VGG19_FP32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(x) % elt || reinterpret_cast<uintptr_t>(y) % elt || reinterpret_cast<uintptr_t>(y_f32) % 4 ||
      reinterpret_cast<uintptr_t>(bias) % 4 || reinterpret_cast<uintptr_t>(codes) % 16 || reinterpret_cast<uintptr_t>(scales) % 16)
    return note_error(VGG19_ERR_ARG, "x, bias and outputs are aligned to their types, codes and scales to 16 bytes");
  const long x_bytes = (long)elt * in, x_pitch = (long)elt * ldx, y_bytes = (long)elt * out * rows, f_bytes = 4L * out * rows;
  const Span all[] = {{y, y_bytes}, {y_f32, f_bytes}, {codes, (long)q4_code_bytes(out, in)}, {scales, (long)q4_scale_bytes(out, in, group)}, {bias, 4L * out}};
  if (rows_meet(x, rows, x_bytes, x_pitch, y, 1, y_bytes, 0) || rows_meet(x, rows, x_bytes, x_pitch, y_f32, 1, f_bytes, 0) || spans_meet(all, 2))
    return note_error(VGG19_ERR_ARG, "an output overlaps x, the weights, the bias or the other output");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e =
      dtype == VGG19_BF16
          ? q4_linear(static_cast<const bf16*>(x), ldx, rows, in, codes, scales, out, group, bias, relu != 0, static_cast<bf16*>(y), y_f32, Waits{}, st)
          : q4_linear(static_cast<const float*>(x), ldx, rows, in, codes, scales, out, group, bias, relu != 0, static_cast<float*>(y), y_f32, Waits{}, st);
  return e == cudaSuccess ? VGG19_OK : note_error(VGG19_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}

}  // extern "C"
