// The last dense layer and the softmax cross entropy of its rows in one, without keeping the logits.  For rows x of `in`
// values, weights w [classes][in], bias b and one label a row
//   z = x w^T + b,   lse_r = log sum_n exp z_rn,   loss_r = lse_r - z_r,label,
//   dz_rn = d_loss_r (exp(z_rn - lse_r) - [n = label_r]),   dx = dz w,   dw = dz^T x,   db = sum_r dz.
//
// Forward: the products z by tiles, whose epilogue keeps of each row and 128 classes the largest z and the sum of
// exp(z - largest), and z at the label; a second kernel joins them.  Backward: z again, tile by tile, with dz as the
// epilogue's result, for as many classes at a time ("a piece") as the workspace has room for; then dw of the piece and
// the piece's share of dx, both in one launch.  That is 8 rows classes in operations in all, where a kept matrix of logits
// would take 6 and 4 bytes a logit and pass over it.
#include <cuda_runtime.h>

#include <atomic>

#include "../../include/vgg19_b200.h"
#include "tc_common.cuh"

namespace vgg {
namespace {

using namespace tc;

static __device__ int g_loss_error[2];   // a DeviceError code once a bounded wait of a call without a handle ran out
static __device__ int g_label_error[2];  // kDevBadLabel once a label outside [0, classes) was met

// ---- sizes -----------------------------------------------------------------------------------------------------
constexpr int BM = 128, BN = 256, BK = 64;   // rows per CTA (a pair has 256), columns per pair, K per stage
constexpr int kBoxBytes = 64 * BK * 2;       // what one copy brings: 64 x 64 values
constexpr int kPlaneBytes = 2 * kBoxBytes;   // one operand's share of a CTA in a stage
// P planes: bf16 values are one plane, fp32 values three (each the bf16 rounding of what the ones before leave: 24 bits).
template <int P> constexpr int kStageBytes = 2 * P * kPlaneBytes;
template <int P> constexpr int kStages = P == 1 ? 6 : 2;
template <int P> constexpr int kBuffers = P == 1 ? 2 : 1;  // accumulators: with three planes one, and one for the small products
constexpr int kRingBytes = 6 * kStageBytes<1>;
static_assert(kRingBytes == 2 * kStageBytes<3>, "the same shared memory");
constexpr int kEpilogueWarps = 8, kThreads = 128 + 32 * kEpilogueWarps;  // a warpgroup for producer and issuer, two of epilogue warps
// Registers per thread after the split: 168 at launch, 3 x 168 = 40 + 2 x 232.
constexpr int kFewRegisters = 40, kManyRegisters = 232;
constexpr int kPieceBytes = 4096;            // an epilogue warp's own 32 rows of 128 bytes
constexpr int kBiasBytes = 128;              // its 32 biases
constexpr int kSmemBytes = kRingBytes + kEpilogueWarps * (kPieceBytes + kBiasBytes) + 1024 + 256;

constexpr float kLog2e = 1.4426950408889634f;

enum Epilogue { kStatistics, kLogitGradient, kProduct };

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
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2)
               : "memory");
}
__device__ __forceinline__ void tma_add_3d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2) {
  asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2)
               : "memory");
}
__device__ __noinline__ void report(const Waits& waits, int code) { atomicCAS(waits.error ? waits.error : g_loss_error, 0, code); }

// ---- one product -------------------------------------------------------------------------------------------------
// D[i][j] = sum_k A(i, k) B(j, k), m x n, in tiles of 256 x 256.  An operand lies K-major (a row per i or j) or, with _mn, with a row per k.
enum Store { kCopied, kAdded, kByThreads };  // results leave by copies, by copies that add in fp32, by the threads' own stores
struct __align__(64) Job {
  CUtensorMap a, b, c;
  int m, n, k_blocks, tiles_m, tiles_n;
  int splits, per_split;  // the sum cut into that many parts, of that many K blocks; part s is plane s of the result
  int chain;              // K blocks that the tensor cores add up before the sums go to the epilogue's registers
  int a_mn, b_mn;
  int store, f32;         // f32: the result is fp32, else bf16
  void* out;              // for kByThreads: one plane, row stride ld
  long ld;
  // the column sums of dz, by the tiles of the first column: of row i the `parts` rows of db_part
  const float* db_part;
  float* db;
  int parts;
};
// What the epilogues of z need: everything about rows is by row, about classes by class of the piece.
struct Rows {
  const float* bias;       // of the piece, or null
  const int32_t* labels;
  int first_class, classes, all_classes;  // the piece and the whole
  // kStatistics: (largest, sum) at part[p * rows + r], p two a tile from first_part on; z at the label
  float2* part;
  float* label_z;
  int first_part;
  // kLogitGradient
  const float *lse, *d_loss;
  float* db_part;          // [rows / 32][classes of a piece], or null
};
struct Launch {
  Waits waits;
  int count, first_tile[3];
  Job job[2];
  Rows rows;
};

struct Tile {
  int i, j, split, k0, k1;
};
// Sixteen rows of tiles at a time, which share their columns' operand: both then stay in L2 while they are needed.
__device__ __forceinline__ Tile find_tile(const Job& p, int t) {
  constexpr int GROUP = 16;
  Tile r{};
  const int all = p.tiles_m * p.tiles_n;
  r.split = t / all;
  t -= r.split * all;
  const int first = t / (GROUP * p.tiles_n) * GROUP, height = min(GROUP, p.tiles_m - first);
  t -= first * p.tiles_n;
  r.j = t / height;
  r.i = first + t - r.j * height;
  r.k0 = r.split * p.per_split;
  r.k1 = min(r.k0 + p.per_split, p.k_blocks);
  return r;
}

__device__ __forceinline__ int piece_at(int row, int chunk) { return row * 8 + (chunk ^ (row & 7)); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// a pair of values as bf16; v keeps what that leaves of them
__device__ __forceinline__ uint32_t take2(float& a, float& b) {
  const uint32_t w = pack2(a, b);
  a -= __uint_as_float(w << 16);
  b -= __uint_as_float(w & 0xffff0000u);
  return w;
}
// Sums of 32 columns over the warp's 32 rows (a row per lane): lane j gets column j's, in an order that is always the same.
__device__ __forceinline__ float column_sums(float (&v)[32], int lane) {
#pragma unroll
  for (int w = 16; w; w >>= 1) {
    const bool upper = lane & w;
#pragma unroll
    for (int j = 0; j < w; ++j) {
      const float give = upper ? v[j] : v[j + w], keep = upper ? v[j + w] : v[j];
      v[j] = keep + __shfl_xor_sync(0xffffffffu, give, w);
    }
  }
  return v[0];
}

template <int P, int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) loss_product_kernel(const __grid_constant__ Launch L) {
  constexpr int STAGES = kStages<P>, STAGE_BYTES = kStageBytes<P>, BUFFERS = kBuffers<P>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t pieces = smem_base + kRingBytes, biases = pieces + kEpilogueWarps * kPieceBytes, bars = biases + kEpilogueWarps * kBiasBytes;
  auto full_bar = [&](int s) { return bars + 8u * s; };                                // used in the even CTA
  auto empty_bar = [&](int s) { return bars + 8u * (STAGES + s); };                   // both CTAs
  auto acc_full_bar = [&](int b) { return bars + 8u * (2 * STAGES + b); };            // both CTAs
  auto acc_empty_bar = [&](int b) { return bars + 8u * (2 * STAGES + BUFFERS + b); }; // used in the even CTA
  const uint32_t drain_bar = bars + 8u * (2 * STAGES + 2 * BUFFERS);
  __shared__ uint32_t tmem_base_slot;
  __shared__ int abort_flag, ran_out;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1, total = L.first_tile[L.count];

  if (threadIdx.x == 0) {
    abort_flag = ran_out = 0;
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), L.waits.signals); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < BUFFERS; ++b) { mbar_init(acc_full_bar(b), 1); mbar_init(acc_empty_bar(b), 2 * kEpilogueWarps); }
    mbar_init(drain_bar, 1);
    mbar_fence_init();
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(&tmem_base_slot), 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // the peer's barriers are initialised before anything signals them
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_slot;
  behind_previous();

  if (warp < 4) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegisters));
  if (warp == 0) {
    // ------------------------------ TMA producer ------------------------------
    if (lane == 0) {
      uint32_t fills[STAGES];
#pragma unroll
      for (int s = 0; s < STAGES; ++s) fills[s] = 0;
      int stage = 0, ji = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int w = pair; w < total && ok; w += n_pairs) {
        while (w >= L.first_tile[ji + 1]) ++ji;
        const Job& p = L.job[ji];
        const Tile tile = find_tile(p, w - L.first_tile[ji]);
        const int row = (2 * tile.i + (int)rank) * BM, col = tile.j * BN + (int)rank * (BN / 2), a_mn = p.a_mn, b_mn = p.b_mn;
        for (int kb = tile.k0; kb < tile.k1; ++kb) {
          if (!mbar_wait(empty_bar(stage), phase ^ 1, &abort_flag, &ran_out, kDevTimeoutStageFree, L.waits.limit_cycles)) { ok = false; break; }
          const uint32_t sa = smem_base + stage * STAGE_BYTES, sb = sa + P * kPlaneBytes;
          const uint32_t full = map_to_cta(full_bar(stage), 0);
          // the even CTA announces the bytes of both CTAs' copies; what lies outside a matrix arrives as zeros
          if (leader) mbar_expect_tx(full_bar(stage), 2 * STAGE_BYTES);
#pragma unroll
          for (int h = 0; h < P; ++h)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              const int r = row + 64 * q, c = col + 64 * q, k = kb * BK;
              tma_load_3d_pair(sa + h * kPlaneBytes + q * kBoxBytes, &p.a, full, a_mn ? r : k, a_mn ? k : r, h);
              tma_load_3d_pair(sb + h * kPlaneBytes + q * kBoxBytes, &p.b, full, b_mn ? c : k, b_mn ? k : c, h);
            }
#pragma unroll
          for (int s = 0; s < STAGES; ++s) fills[s] += s == stage;
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
      }
      if (!ok) {
        // let every copy in flight land before the CTA may exit
        if (leader) {
#pragma unroll
          for (int s = 0; s < STAGES; ++s)
            if (fills[s]) {
              const unsigned long long t0 = global_timer_ns();
              while (!mbar_try_wait(full_bar(s), (fills[s] - 1) & 1) && global_timer_ns() - t0 < 100000000ull) {}
            }
        } else {
          const unsigned long long t0 = global_timer_ns();
          while (global_timer_ns() - t0 < 1000000ull) {}
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------- MMA issuer (even CTA only) -------------------------
    if (lane == 0 && leader) {
      int stage = 0, ji = 0;
      uint32_t phase = 0, count = 0;
      bool ok = true;
      for (int w = pair; w < total && ok; w += n_pairs) {
        while (w >= L.first_tile[ji + 1]) ++ji;
        const Job& p = L.job[ji];
        const Tile tile = find_tile(p, w - L.first_tile[ji]);
        // K-major: 16 k = 32 bytes of the swizzled row.  A row per k: two boxes of 64 columns, 16 k = 16 rows.
        const uint32_t idesc = umma_idesc_bf16(2 * BM, BN, p.a_mn, p.b_mn);
        const uint32_t a_step = p.a_mn ? 2048 : 32, a_lbo = p.a_mn ? kBoxBytes : 16, b_step = p.b_mn ? 2048 : 32, b_lbo = p.b_mn ? kBoxBytes : 16;
        for (int kb0 = tile.k0, kb1; kb0 < tile.k1 && ok; kb0 = kb1, ++count) {
          kb1 = p.chain < tile.k1 - kb0 ? kb0 + p.chain : tile.k1;
          const int buf = count % BUFFERS;
          if (!mbar_wait(acc_empty_bar(buf), ((count / BUFFERS) & 1) ^ 1, &abort_flag, &ran_out, kDevTimeoutTmemFree, L.waits.limit_cycles)) { ok = false; break; }
          tc_fence_after();
          const uint32_t d = tmem_base + (uint32_t)(buf * BN);
          for (int kb = kb0; kb < kb1; ++kb) {
            if (!mbar_wait(full_bar(stage), phase, &abort_flag, &ran_out, kDevTimeoutTmaFull, L.waits.limit_cycles)) { ok = false; break; }
            tc_fence_after();
            const uint32_t sa = smem_base + stage * STAGE_BYTES, sb = sa + P * kPlaneBytes;
            uint64_t a[P], b[P];
#pragma unroll
            for (int h = 0; h < P; ++h) {
              a[h] = smem_desc_sw128(sa + h * kPlaneBytes, a_lbo);
              b[h] = smem_desc_sw128(sb + h * kPlaneBytes, b_lbo);
            }
#pragma unroll
            for (int k = 0; k < BK / 16; ++k) {
              const uint32_t more = kb != kb0 || k ? 1u : 0u;
              umma_bf16_pair(d, desc_advance(a[0], k * a_step), desc_advance(b[0], k * b_step), idesc, more);
              if (P == 3) {
                // the products of the lesser planes, at most 2^-8 of the first, have a sum of their own: the tensor core truncates
                // its sums, relative to their size, so the chain that matters has a sixth of the instructions
                auto small = [&](int u, int v, uint32_t m) {
                  umma_bf16_pair(tmem_base + BN, desc_advance(a[u], k * a_step), desc_advance(b[v], k * b_step), idesc, m);
                };
                small(0, P - 1, more);
                small(P - 1, 0, 1u);
                small(1 % P, 1 % P, 1u);
                small(0, 1 % P, 1u);
                small(1 % P, 0, 1u);
              }
            }
            umma_commit_pair(empty_bar(stage), 3);  // frees the stage in both CTAs
            if (++stage == STAGES) { stage = 0; phase ^= 1; }
          }
          if (ok) umma_commit_pair(acc_full_bar(buf), 3);
        }
      }
      if (!ok) {
        umma_commit_pair(drain_bar, 1);
        const unsigned long long t0 = global_timer_ns();
        while (!mbar_try_wait(drain_bar, 0) && global_timer_ns() - t0 < 100000000ull) {}
      }
    }
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegisters));
    // -------------------------------- epilogue --------------------------------
    const int group = (warp - 4) >> 2, quarter = warp & 3;  // half of the columns; the lane quarter this warp may read
    const uint32_t piece_addr = pieces + (warp - 4) * kPieceBytes;
    uint4* piece = reinterpret_cast<uint4*>(smem_raw + (piece_addr - smem_u32(smem_raw)));
    float* bias_s = reinterpret_cast<float*>(smem_raw + (biases + (warp - 4) * kBiasBytes - smem_u32(smem_raw)));
    int ji = 0;
    uint32_t count = 0;
    bool ok = true;
    for (int w = pair; w < total && ok; w += n_pairs) {
      while (w >= L.first_tile[ji + 1]) ++ji;
      const Job& p = L.job[ji];
      const Tile tile = find_tile(p, w - L.first_tile[ji]);
      const int i0 = (2 * tile.i + (int)rank) * BM + quarter * 32, j0 = tile.j * BN + group * 128;  // the warp's first row and column
      const int rows = p.m - i0, cols = p.n - j0;                                                 // what there is from there on
      const int row = i0 + lane;
      // what a row needs, requested while the products run
      float lse = 0.f, d_loss = 0.f, next_bias = 0.f;
      int label = VGG19_NO_CLASS;
      // columns beyond the classes get the bias of an excluded class
      auto bias_of = [&](int c) { return c < cols ? L.rows.bias ? __ldg(L.rows.bias + j0 + c) : 0.f : -INFINITY; };
      if (EPI != kProduct) {
        if (lane < rows) {
          label = L.rows.labels[row];
          if (EPI == kLogitGradient) { lse = L.rows.lse[row]; d_loss = L.rows.d_loss[row]; }
        }
        const bool real = (unsigned)label < (unsigned)L.rows.all_classes;
        if (EPI == kLogitGradient) {
          if (!real && label != VGG19_NO_CLASS && j0 == 0) atomicCAS(g_label_error, 0, (int)kDevBadLabel);
          // no label, or no class left: no gradient
          if (!real || lse == -INFINITY) d_loss = 0.f;
          label = d_loss != 0.f || d_loss != d_loss ? label - L.rows.first_class : -1;
        } else {
          label = real ? label - L.rows.first_class : -1;
        }
        next_bias = bias_of(lane);
      }
      if (EPI == kProduct && p.db && tile.j == 0 && group == 0 && tile.split == 0 && lane < rows) {
        float s = 0.f;
#pragma unroll 8
        for (int q = 0; q < p.parts; ++q) s += p.db_part[(long)q * p.m + row];
        p.db[row] = s;
      }
      float v[128];  // the tile's sums of this row and half
      for (long kb0 = tile.k0; kb0 < tile.k1; kb0 += p.chain, ++count) {
        const int buf = count % BUFFERS;
        if (!__all_sync(0xffffffffu, mbar_wait(acc_full_bar(buf), (count / BUFFERS) & 1, &abort_flag, &ran_out, kDevTimeoutAccum, L.waits.limit_cycles))) { ok = false; break; }
        tc_fence_after();
        const uint32_t src = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * BN + group * 128);
        const bool more = kb0 != tile.k0;
#pragma unroll
        for (int c = 0; c < 128; c += 32) {
          uint32_t t[32];
          tmem_ld_32x32(src + c, t);
          if (P == 3) {
            uint32_t u[32];
            tmem_ld_32x32(src + BN + c, u);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) t[j] = __float_as_uint(__uint_as_float(t[j]) + __uint_as_float(u[j]));
          } else {
            tmem_ld_wait();
          }
#pragma unroll
          for (int j = 0; j < 32; ++j) v[c + j] = (more ? v[c + j] : 0.f) + __uint_as_float(t[j]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(map_to_cta(acc_empty_bar(buf), 0));
      }
      if (!ok) break;
      auto add_bias = [&](int c) {
        bias_s[lane] = next_bias;
        __syncwarp();
        if (c + 32 < 128) next_bias = bias_of(c + 32 + lane);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const float4 b = reinterpret_cast<const float4*>(bias_s)[q];
          v[c + 4 * q] += b.x; v[c + 4 * q + 1] += b.y; v[c + 4 * q + 2] += b.z; v[c + 4 * q + 3] += b.w;
        }
        __syncwarp();
      };

      if (EPI == kStatistics) {
        float most = -INFINITY, sum = 0.f;
#pragma unroll
        for (int c = 0; c < 128; c += 32) {
          add_bias(c);
#pragma unroll
          for (int j = 0; j < 32; ++j) most = fmaxf(most, v[c + j]);
          const int at = label - j0 - c;  // the label's column among these
          if (__any_sync(0xffffffffu, (unsigned)at < 32u)) {
            float z = 0.f;
#pragma unroll
            for (int j = 0; j < 32; ++j) z = at == j ? v[c + j] : z;
            if ((unsigned)at < 32u && at < cols - c) L.rows.label_z[row] = z;
          }
        }
        const float ref = most == -INFINITY ? 0.f : most;
#pragma unroll
        for (int c = 0; c < 128; c += 32) {
          float part = 0.f;
#pragma unroll
          for (int j = 0; j < 32; ++j) part += fast_exp2((v[c + j] - ref) * kLog2e);
          sum += part;
        }
        if (lane < rows && cols > 0) L.rows.part[(long)(L.rows.first_part + 2 * tile.j + group) * p.m + row] = make_float2(most, sum);
      } else if (EPI == kLogitGradient) {
        const float ref = lse == -INFINITY ? 0.f : lse;
#pragma unroll
        for (int c0 = 0; c0 < 128; c0 += 64) {
#pragma unroll
          for (int c = c0; c < c0 + 64; c += 32) {
            add_bias(c);
            const int at = label - j0 - c;
#pragma unroll
            for (int j = 0; j < 32; ++j) v[c + j] = fast_exp2((v[c + j] - ref) * kLog2e);
            if (__any_sync(0xffffffffu, (unsigned)at < 32u)) {
#pragma unroll
              for (int j = 0; j < 32; ++j) v[c + j] = at == j ? v[c + j] - 1.f : v[c + j];
            }
#pragma unroll
            for (int j = 0; j < 32; ++j) v[c + j] = d_loss == 0.f ? 0.f : d_loss * v[c + j];  // (a row that counts for nothing may hold anything)
            if (L.rows.db_part) {
              float t[32];
#pragma unroll
              for (int j = 0; j < 32; ++j) t[j] = v[c + j];
              const float s = column_sums(t, lane);
              if (c + lane < cols && rows > 0) L.rows.db_part[(long)(i0 / 32) * p.n + j0 + c + lane] = s;
            }
          }
#pragma unroll
          for (int h = 0; h < P; ++h) {
            if (lane == 0) tma_store_wait_read<0>();
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              float* e = v + c0 + 8 * k;
              piece[piece_at(lane, k)] = P == 1 ? make_uint4(pack2(e[0], e[1]), pack2(e[2], e[3]), pack2(e[4], e[5]), pack2(e[6], e[7]))
                                                : make_uint4(take2(e[0], e[1]), take2(e[2], e[3]), take2(e[4], e[5]), take2(e[6], e[7]));
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0 && rows > 0 && c0 < cols) {
              tma_store_3d(&p.c, piece_addr, j0 + c0, i0, h);
              tma_store_commit();
            }
          }
        }
      } else {
        const bool f32 = p.f32 != 0;
#pragma unroll
        for (int c0 = 0; c0 < 128; c0 += 32) {
          const int half = f32 ? 0 : (c0 >> 5) & 1;  // bf16: two of these fill a piece
          if (!half) {
            if (lane == 0) tma_store_wait_read<0>();
            __syncwarp();
          }
          if (f32) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
              piece[piece_at(lane, k)] = make_uint4(__float_as_uint(v[c0 + 4 * k]), __float_as_uint(v[c0 + 4 * k + 1]), __float_as_uint(v[c0 + 4 * k + 2]),
                                                    __float_as_uint(v[c0 + 4 * k + 3]));
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float* e = v + c0 + 8 * k;
              piece[piece_at(lane, 4 * half + k)] = make_uint4(pack2(e[0], e[1]), pack2(e[2], e[3]), pack2(e[4], e[5]), pack2(e[6], e[7]));
            }
            if (!half) continue;
          }
          const int from = f32 ? c0 : c0 - 32, wide = f32 ? 32 : 64;  // the piece's columns
          if (p.store == kByThreads) {
            __syncwarp();
            const int n = min(32, rows);
            for (int r = 0; r < n; ++r)
              for (int c = lane; c < wide; c += 32) {
                if (from + c >= cols) continue;
                const long at = (long)(i0 + r) * p.ld + j0 + from + c;
                if (f32) static_cast<float*>(p.out)[at] = reinterpret_cast<const float*>(piece + piece_at(r, c / 4))[c % 4];
                else static_cast<bf16*>(p.out)[at] = reinterpret_cast<const bf16*>(piece + piece_at(r, c / 8))[c % 8];
              }
            __syncwarp();
            continue;
          }
          fence_async_smem();
          __syncwarp();
          if (lane == 0 && rows > 0 && from < cols) {
            if (p.store == kAdded) tma_add_3d(&p.c, piece_addr, j0 + from, i0, tile.split);
            else tma_store_3d(&p.c, piece_addr, j0 + from, i0, tile.split);
            tma_store_commit();
          }
        }
      }
    }
    if (EPI != kStatistics && lane == 0) tma_store_wait_all();
  }

  // Neither CTA may release tensor memory or exit while the other can still signal its barriers, read its shared
  // memory or write its accumulator.
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (threadIdx.x == 0 && ran_out) report(L.waits, ran_out);
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, 512);
  }
}

// ---- the rows' parts joined ------------------------------------------------------------------------------------------
struct Join {
  const float2* part;
  const float* label_z;
  const int32_t* labels;
  float *loss, *lse;
  int parts, rows, classes;
};
constexpr int kJoinGroups = 8;

// (m, s) with the largest z so far and the sum of exp(z - m); nothing so far: (-inf, 0).  A NaN stays in s.
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  if (m == -INFINITY) return make_float2(m, a.y + b.y);
  return make_float2(m, a.y * fast_exp2((a.x - m) * kLog2e) + b.y * fast_exp2((b.x - m) * kLog2e));
}

__global__ void __launch_bounds__(32 * kJoinGroups) join_rows_kernel(const __grid_constant__ Join a) {
  __shared__ float2 got[kJoinGroups][32];
  behind_previous();
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, row = blockIdx.x * 32 + lane;
  float2 v = make_float2(-INFINITY, 0.f);
  if (row < a.rows)
    for (int p = group; p < a.parts; p += kJoinGroups) v = join(v, a.part[(long)p * a.rows + row]);
  got[group][lane] = v;
  __syncthreads();
  if (group || row >= a.rows) return;
#pragma unroll
  for (int g = 1; g < kJoinGroups; ++g) v = join(v, got[g][lane]);
  const float log_sum = logf(v.y), lse = v.x + log_sum;
  if (a.lse) a.lse[row] = lse;
  const int label = a.labels[row];
  float loss = 0.f;
  if ((unsigned)label < (unsigned)a.classes) {
    // (the largest z less the label's is exact where they are near each other, so a loss near 0 is not a difference of two roundings)
    loss = lse == -INFINITY ? INFINITY : v.x - a.label_z[row] + log_sum;
  } else if (label != VGG19_NO_CLASS) {
    loss = __int_as_float(0x7fc00000);
    atomicCAS(g_label_error, 0, (int)kDevBadLabel);
  }
  if (a.loss) a.loss[row] = loss;
}

// ---- rows as planes of bf16 ------------------------------------------------------------------------------------------
// dst[h][r][k], row stride ld (a multiple of 8): the value itself, or an fp32 value's three terms.
template <typename T, int P>
__global__ void __launch_bounds__(256) planes_kernel(const T* __restrict__ src, long src_ld, bf16* dst, long rows, int in, long ld) {
  behind_previous();
  const int chunks = (int)(ld / 8);
  const long all = rows * chunks;
  for (long t = (long)blockIdx.x * blockDim.x + threadIdx.x; t < all; t += (long)gridDim.x * blockDim.x) {
    const long r = t / chunks;
    const int k = (int)(t - r * chunks) * 8;
    const T* at = src + r * src_ld + k;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = k + e < in ? to_f32(at[e]) : 0.f;
#pragma unroll
    for (int h = 0; h < P; ++h) {
      uint4 q;
      q.x = take2(v[0], v[1]); q.y = take2(v[2], v[3]); q.z = take2(v[4], v[5]); q.w = take2(v[6], v[7]);
      *reinterpret_cast<uint4*>(dst + (h * rows + r) * ld + k) = q;
    }
  }
}

// ---- dx from its parts -----------------------------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256) sum_parts_kernel(const float* __restrict__ part, int parts, long rows, int in, long ld, T* out, long out_ld) {
  behind_previous();
  const int chunks = (int)(ld / 4);
  const long all = rows * chunks;
  for (long t = (long)blockIdx.x * blockDim.x + threadIdx.x; t < all; t += (long)gridDim.x * blockDim.x) {
    const long r = t / chunks;
    const int k = (int)(t - r * chunks) * 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
      const float4 v = *reinterpret_cast<const float4*>(part + (p * rows + r) * ld + k);
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (k + e < in) out[r * out_ld + k + e] = from_f32<T>(v[e]);
  }
}

// db of a piece where no product of dw does it on the way
__global__ void __launch_bounds__(256) sum_columns_kernel(const float* part, int parts, int n, float* db) {
  behind_previous();
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= n) return;
  float s = 0.f;
#pragma unroll 8
  for (int q = 0; q < parts; ++q) s += part[(long)q * n + c];
  db[c] = s;
}

// ---- host side -------------------------------------------------------------------------------------------------------
constexpr long up(long v, long a) { return (v + a - 1) / a * a; }

// [planes][rows][cols] of bf16 or fp32, rows ld and planes rows * ld apart, in boxes of box_rows rows of 128 bytes
bool planes_map(CUtensorMap* map, const void* base, bool f32, long planes, long rows, long cols, long ld, uint32_t box_rows) {
  const TensorMapApi& api = tensor_map_api();
  if (!api.ok) return false;
  const long elt = f32 ? 4 : 2;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  cuuint64_t strides[2] = {(cuuint64_t)(ld * elt), (cuuint64_t)(rows * ld * elt)};
  cuuint32_t box[3] = {(cuuint32_t)(128 / elt), box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return api.encode_tiled(map, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides,
                          box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Whether rows can be read by copies where they lie.
bool copyable(const void* p, long rows, long ld, long elt) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows == 1 || (ld * elt % 16 == 0 && ld * elt < (1L << 40)));
}
// And whether they can be written: a copy writes whole 16 bytes, zeros behind the end of a row.
bool writable(const void* p, long rows, long cols, long ld, long elt) { return copyable(p, rows, ld, elt) && cols * elt % 16 == 0; }

// How a call is cut up, and where its parts lie in the workspace.
struct Plan {
  int planes;             // 1 or 3
  bool take_x, take_w;    // whether they are laid out anew (as planes, or to be read by copies at all)
  long ld;                // row stride of what is
  long piece;             // classes at a time
  int pieces;
  int dx_splits;          // parts of dx's sum within a piece
  bool dx_parts;          // whether dx is added up in fp32 outside the products
  long dx_ld;
  size_t x, w, part, label_z, dz, db_part, dx, total;
};

int pairs_of_device() {
  int dev = 0, sms = 148;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms / 2;
}

// The tensor core truncates its fp32 sums, an error that grows with the chain: 1.8e-6 of the loss over 4096 values in one chain.  The
// sums of shorter ones are added in registers, rounded to nearest.  Gradients in bf16 need none of that.
constexpr int chain_blocks(int planes, int epilogue) { return planes == 3 ? 8 : epilogue == kProduct ? 1 << 30 : 16; }

constexpr long kPieceBytesMost = 256L << 20;  // of dz, or of the planes of w

Plan make_plan(const vgg19_linear_loss& a, bool backward, int pairs) {
  Plan p{};
  const bool f32 = a.dtype == VGG19_FP32;
  p.planes = f32 ? 3 : 1;
  p.take_x = f32 || !copyable(a.x, a.rows, a.ldx, 2);
  p.take_w = f32 || !copyable(a.w, a.classes, a.ldw, 2);
  p.ld = up(a.in, 8);
  const long all = up(a.classes, BN);
  p.piece = all;
  auto most = [&](long bytes_a_class) {
    const long fit = kPieceBytesMost / bytes_a_class / BN * BN, least = 4096;
    if (p.piece > (fit > least ? fit : least)) p.piece = fit > least ? fit : least;
  };
  if (p.take_w) most(2 * p.planes * p.ld);
  if (backward) most(2 * p.planes * a.rows);
  p.pieces = (int)((all + p.piece - 1) / p.piece);
  p.piece = up((all + p.pieces - 1) / p.pieces, BN);  // pieces of about one size
  p.pieces = (int)((all + p.piece - 1) / p.piece);
  size_t at = 0;
  auto take = [&at](size_t bytes) { const size_t o = at; at += (bytes + 255) / 256 * 256; return o; };
  if (p.take_x) p.x = take((size_t)p.planes * a.rows * p.ld * 2);
  if (p.take_w) p.w = take((size_t)p.planes * (p.piece < a.classes ? p.piece : a.classes) * p.ld * 2);
  if (!backward) {
    p.part = take((size_t)p.pieces * (p.piece / 128) * a.rows * sizeof(float2));
    p.label_z = take((size_t)a.rows * 4);
  } else {
    p.dz = take((size_t)p.planes * a.rows * p.piece * 2);
    p.db_part = take((size_t)(up(a.rows, 32) / 32) * p.piece * 4);
    // dx has rows x in tiles; where they leave pairs idle, its sum is cut into parts
    const long tiles = (up(a.rows, 2 * BM) / (2 * BM)) * (up(a.in, BN) / BN);
    const long blocks = (p.piece < a.classes ? p.piece : (long)a.classes + BK - 1) / BK;
    long want = pairs / tiles;
    if (want > blocks / 16) want = blocks / 16;  // parts of at least sixteen blocks: each is written, and read again
    p.dx_splits = (int)(want < 1 ? 1 : want > 64 ? 64 : want);
    p.dx_parts = p.pieces > 1 || p.dx_splits > 1;
    p.dx_ld = up(a.in, 4);
    if (p.dx_parts) p.dx = take((size_t)p.dx_splits * a.rows * p.dx_ld * 4);
  }
  p.total = at < 256 ? 256 : at;
  return p;
}

template <typename... A>
cudaError_t launch_behind(void (*kernel)(A...), unsigned blocks, int threads, int smem, cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int P, int EPI> cudaError_t launch_products(Launch& L, int pairs, cudaStream_t st) {
  int tiles = 0;
  for (int i = 0; i < L.count; ++i) {
    Job& p = L.job[i];
    p.tiles_m = (p.m + 2 * BM - 1) / (2 * BM);
    p.tiles_n = (p.n + BN - 1) / BN;
    if (p.splits < 1) p.splits = 1;
    p.per_split = (p.k_blocks + p.splits - 1) / p.splits;
    p.chain = chain_blocks(P, EPI);
    p.splits = (p.k_blocks + p.per_split - 1) / p.per_split;  // none is empty
    L.first_tile[i] = tiles;
    tiles += p.splits * p.tiles_m * p.tiles_n;
  }
  L.first_tile[L.count] = tiles;
  const cudaError_t e = cudaFuncSetAttribute(loss_product_kernel<P, EPI>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
  if (e != cudaSuccess) return e;
  return launch_behind(loss_product_kernel<P, EPI>, (unsigned)(2 * (tiles < pairs ? tiles : pairs)), kThreads, kSmemBytes, st, L);
}

// The operands of one call in the form that the products read: x once, w piece by piece.
template <int P> struct Operands {
  const vgg19_linear_loss& a;
  const Plan& p;
  char* ws;
  cudaStream_t st;
  CUtensorMap x, w;

  cudaError_t lay_out(const void* src, long src_ld, long rows, size_t at) {
    bf16* dst = reinterpret_cast<bf16*>(ws + at);
    const long chunks = rows * (p.ld / 8);
    const unsigned blocks = (unsigned)(chunks / 256 + 1 < 148 * 16 ? chunks / 256 + 1 : 148 * 16);
    if (P == 3) return launch_behind(planes_kernel<float, 3>, blocks, 256, 0, st, static_cast<const float*>(src), src_ld, dst, rows, (int)a.in, p.ld);
    return launch_behind(planes_kernel<bf16, 1>, blocks, 256, 0, st, static_cast<const bf16*>(src), src_ld, dst, rows, (int)a.in, p.ld);
  }
  cudaError_t rows() {
    if (!p.take_x) return planes_map(&x, a.x, false, 1, a.rows, a.in, a.rows == 1 ? p.ld : a.ldx, 64) ? cudaSuccess : cudaErrorInvalidValue;
    const cudaError_t e = lay_out(a.x, a.ldx, a.rows, p.x);
    if (e != cudaSuccess) return e;
    return planes_map(&x, ws + p.x, false, P, a.rows, a.in, p.ld, 64) ? cudaSuccess : cudaErrorInvalidValue;
  }
  cudaError_t weights(long first, long n) {
    const long elt = P == 3 ? 4 : 2;
    const char* src = static_cast<const char*>(a.w) + first * a.ldw * elt;
    if (!p.take_w) return planes_map(&w, src, false, 1, n, a.in, a.classes == 1 ? p.ld : a.ldw, 64) ? cudaSuccess : cudaErrorInvalidValue;
    const cudaError_t e = lay_out(src, a.ldw, n, p.w);
    if (e != cudaSuccess) return e;
    return planes_map(&w, ws + p.w, false, P, n, a.in, p.ld, 64) ? cudaSuccess : cudaErrorInvalidValue;
  }
};

// The products z of one piece.
template <int P> Launch logits(const Operands<P>& o, long first, long n, const Waits& waits) {
  Launch L{};
  L.waits = waits;
  L.count = 1;
  Job& j = L.job[0];
  j.a = o.x; j.b = o.w; j.c = o.w;
  j.m = (int)o.a.rows; j.n = (int)n; j.k_blocks = (o.a.in + BK - 1) / BK;
  Rows& r = L.rows;
  r.bias = o.a.bias ? o.a.bias + first : nullptr;
  r.labels = o.a.labels;
  r.first_class = (int)first; r.classes = (int)n; r.all_classes = o.a.classes;
  return L;
}

template <int P>
cudaError_t forward(const vgg19_linear_loss& a, float* loss, float* lse, char* ws, const Plan& p, int pairs, const Waits& waits, cudaStream_t st) {
  Operands<P> o{a, p, ws, st, {}, {}};
  cudaError_t e = o.rows();
  int part = 0;
  for (int i = 0; i < p.pieces && e == cudaSuccess; ++i) {
    const long first = i * p.piece, n = a.classes - first < p.piece ? a.classes - first : p.piece;
    e = o.weights(first, n);
    if (e != cudaSuccess) break;
    Launch L = logits<P>(o, first, n, waits);
    L.rows.part = reinterpret_cast<float2*>(ws + p.part);
    L.rows.label_z = reinterpret_cast<float*>(ws + p.label_z);
    L.rows.first_part = part;
    part += (int)((n + 127) / 128);
    e = launch_products<P, kStatistics>(L, pairs, st);
  }
  if (e != cudaSuccess) return e;
  const Join j{reinterpret_cast<const float2*>(ws + p.part), reinterpret_cast<const float*>(ws + p.label_z), a.labels, loss, lse, part, (int)a.rows, a.classes};
  return launch_behind(join_rows_kernel, (unsigned)((a.rows + 31) / 32), 32 * kJoinGroups, 0, st, j);
}

struct Gradients {
  const float *lse, *d_loss;
  void* dx;
  long dx_ld;
  void* dw;
  int dw_f32;
  long dw_ld;
  float* db;
};

template <int P>
cudaError_t backward(const vgg19_linear_loss& a, const Gradients& g, char* ws, const Plan& p, int pairs, const Waits& waits, cudaStream_t st) {
  Operands<P> o{a, p, ws, st, {}, {}};
  cudaError_t e = o.rows();
  float* dx_part = reinterpret_cast<float*>(ws + p.dx);
  float* db_part = reinterpret_cast<float*>(ws + p.db_part);
  int slots = 0;
  for (int i = 0; i < p.pieces && e == cudaSuccess; ++i) {
    const long first = i * p.piece, n = a.classes - first < p.piece ? a.classes - first : p.piece;
    e = o.weights(first, n);
    if (e != cudaSuccess) break;
    const long dz_ld = up(n, 8);
    CUtensorMap dz, dz_out;
    if (!planes_map(&dz, ws + p.dz, false, P, a.rows, n, dz_ld, 64) || !planes_map(&dz_out, ws + p.dz, false, P, a.rows, n, dz_ld, 32))
      return cudaErrorInvalidValue;
    Launch L = logits<P>(o, first, n, waits);
    L.job[0].c = dz_out;
    L.rows.lse = g.lse; L.rows.d_loss = g.d_loss;
    L.rows.db_part = g.db ? db_part : nullptr;
    e = launch_products<P, kLogitGradient>(L, pairs, st);
    if (e != cudaSuccess) break;

    Launch M{};
    M.waits = waits;
    const bool f32 = P == 3;
    if (g.dw) {  // dw of the piece: [n][in] = dz^T x
      Job& j = M.job[M.count++];
      const bool out32 = f32 || g.dw_f32;
      const long elt = out32 ? 4 : 2;
      j.a = dz; j.a_mn = 1; j.b = o.x; j.b_mn = 1;
      j.m = (int)n; j.n = a.in; j.k_blocks = (int)((a.rows + BK - 1) / BK);
      j.f32 = out32;
      j.out = static_cast<char*>(g.dw) + first * g.dw_ld * elt; j.ld = g.dw_ld;
      j.store = writable(j.out, n, a.in, g.dw_ld, elt) ? kCopied : kByThreads;
      j.c = j.a;
      if (j.store == kCopied && !planes_map(&j.c, j.out, out32, 1, n, a.in, n == 1 ? up(a.in, 8) : g.dw_ld, 32)) return cudaErrorInvalidValue;
      j.db_part = db_part; j.db = g.db ? g.db + first : nullptr;
      j.parts = (int)((a.rows + 31) / 32);
    }
    if (g.dx) {  // dx, or the piece's share of it: [rows][in] = dz w
      Job& j = M.job[M.count++];
      j.a = dz; j.b = o.w; j.b_mn = 1;
      j.m = (int)a.rows; j.n = a.in; j.k_blocks = (int)((n + BK - 1) / BK);
      j.c = j.a;
      if (p.dx_parts) {
        j.f32 = 1;
        j.splits = slots && slots < p.dx_splits ? slots : p.dx_splits;  // later pieces add to the parts that the first one wrote
        j.store = i ? kAdded : kCopied;
        if (!planes_map(&j.c, dx_part, true, p.dx_splits, a.rows, a.in, p.dx_ld, 32)) return cudaErrorInvalidValue;
        if (!i) {
          const int per = (j.k_blocks + j.splits - 1) / j.splits;
          slots = (j.k_blocks + per - 1) / per;
        }
      } else {
        const long elt = f32 ? 4 : 2;
        j.f32 = f32;
        j.out = g.dx; j.ld = g.dx_ld;
        j.store = writable(g.dx, a.rows, a.in, g.dx_ld, elt) ? kCopied : kByThreads;
        if (j.store == kCopied && !planes_map(&j.c, g.dx, f32, 1, a.rows, a.in, a.rows == 1 ? up(a.in, 8) : g.dx_ld, 32)) return cudaErrorInvalidValue;
      }
    }
    if (M.count) e = launch_products<P, kProduct>(M, pairs, st);
    if (!g.dw && g.db && e == cudaSuccess)
      e = launch_behind(sum_columns_kernel, (unsigned)((n + 255) / 256), 256, 0, st, static_cast<const float*>(db_part), (int)((a.rows + 31) / 32), (int)n, g.db + first);
  }
  if (e != cudaSuccess || !g.dx || !p.dx_parts) return e;
  const long chunks = a.rows * (p.dx_ld / 4);
  const unsigned blocks = (unsigned)(chunks / 256 + 1 < 148 * 16 ? chunks / 256 + 1 : 148 * 16);
  if (P == 3)
    return launch_behind(sum_parts_kernel<float>, blocks, 256, 0, st, static_cast<const float*>(dx_part), slots, (long)a.rows, (int)a.in, p.dx_ld, static_cast<float*>(g.dx), g.dx_ld);
  return launch_behind(sum_parts_kernel<bf16>, blocks, 256, 0, st, static_cast<const float*>(dx_part), slots, (long)a.rows, (int)a.in, p.dx_ld, static_cast<bf16*>(g.dx), g.dx_ld);
}

int check(const vgg19_linear_loss* a) {
  if (!a) return note_error(VGG19_ERR_ARG, "no description of the layer");
  if (a->dtype != VGG19_FP32 && a->dtype != VGG19_BF16)
    return note_error(VGG19_ERR_ARG, "dtype %d is neither VGG19_FP32 nor VGG19_BF16", a->dtype);
  if (a->rows < 0 || a->rows > (1 << 22) || a->in < 1 || a->in > (1 << 20) || a->classes < 1 || a->classes > (1 << 24))
    return note_error(VGG19_ERR_SHAPE, "%lld rows of %d values, %d classes: rows in [0, 2^22], values in [1, 2^20], classes in [1, 2^24]",
                      (long long)a->rows, a->in, a->classes);
  if (a->ldx < a->in || a->ldw < a->in || a->ldx >= (1LL << 36) || a->ldw >= (1LL << 36))
    return note_error(VGG19_ERR_SHAPE, "row strides %lld and %lld for %d values", (long long)a->ldx, (long long)a->ldw, a->in);
  return VGG19_OK;
}
int check_pointers(const vgg19_linear_loss& a, const void* workspace) {
  const uintptr_t elt = a.dtype == VGG19_FP32 ? 4 : 2;
  if (!a.x || !a.w || !a.labels) return note_error(VGG19_ERR_ARG, "x, w and labels must not be null");
  if (reinterpret_cast<uintptr_t>(a.x) % elt || reinterpret_cast<uintptr_t>(a.w) % elt) return note_error(VGG19_ERR_ARG, "x or w is not aligned to its type");
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256) return note_error(VGG19_ERR_WORKSPACE, "the workspace is null or not 256-byte aligned");
  return VGG19_OK;
}
// whether all of these (null among them) are addresses of 32-bit values
template <typename... Q> bool words(Q... q) { return ((reinterpret_cast<uintptr_t>(q) % 4 == 0) && ...); }

// Rows of a matrix, or a vector as one row.
struct Block {
  const void* p;
  long rows, bytes, pitch;
};
bool meet(const Block& a, const Block& b) { return rows_meet(a.p, a.rows, a.bytes, a.pitch, b.p, b.rows, b.bytes, b.pitch); }
// Whether one of the first `written` meets any other.
template <int N> bool blocks_meet(const Block (&all)[N], int written) {
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < N; ++j)
      if (meet(all[i], all[j])) return true;
  return false;
}

}  // namespace

cudaError_t loss_take_error(int* code, int* label, cudaStream_t st) {
  void *word = nullptr, *label_word = nullptr;
  cudaError_t e = cudaGetSymbolAddress(&word, g_loss_error);
  if (e == cudaSuccess) e = cudaGetSymbolAddress(&label_word, g_label_error);
  if (e == cudaSuccess) e = take_error(static_cast<int*>(word), code, st);
  return e == cudaSuccess ? take_error(static_cast<int*>(label_word), label, st) : e;
}

int linear_loss(const vgg19_linear_loss* layer, float* loss, float* lse, void* workspace, size_t bytes, const Waits& waits, void* stream) {
  const int rc = check(layer);
  if (rc != VGG19_OK || layer->rows == 0) return rc;
  const vgg19_linear_loss& a = *layer;
  const int bad = check_pointers(a, workspace);
  if (bad != VGG19_OK) return bad;
  if (!words(a.bias, a.labels, loss, lse)) return note_error(VGG19_ERR_ARG, "bias, labels, loss or lse is not aligned to 4 bytes");
  const int pairs = pairs_of_device();
  const Plan p = make_plan(a, false, pairs);
  if (bytes < p.total) return note_error(VGG19_ERR_WORKSPACE, "workspace has %zu bytes, this call needs %zu", bytes, p.total);
  const long elt = a.dtype == VGG19_FP32 ? 4 : 2, each = 4L * a.rows;
  const Block all[] = {{loss, 1, each, 0}, {lse, 1, each, 0}, {workspace, 1, (long)p.total, 0}, {a.labels, 1, each, 0}, {a.bias, 1, 4L * a.classes, 0},
                       {a.x, a.rows, a.in * elt, a.ldx * elt}, {a.w, a.classes, a.in * elt, a.ldw * elt}};
  if (blocks_meet(all, 3)) return note_error(VGG19_ERR_ARG, "an output or the workspace overlaps an input or another output");
  if (!loss && !lse) return VGG19_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  const cudaError_t e = p.planes == 3 ? forward<3>(a, loss, lse, ws, p, pairs, waits, st) : forward<1>(a, loss, lse, ws, p, pairs, waits, st);
  return e == cudaSuccess ? VGG19_OK : note_error(VGG19_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}

}  // namespace vgg

extern "C" size_t vgg19_linear_cross_entropy_bytes(const vgg19_linear_loss* layer, int32_t backward) {
  using namespace vgg;
  if (check(layer) != VGG19_OK) return 0;
  return make_plan(*layer, backward != 0, pairs_of_device()).total;
}

extern "C" int vgg19_linear_cross_entropy(const vgg19_linear_loss* layer, float* loss, float* lse, void* workspace, size_t bytes, void* stream) {
  return vgg::linear_loss(layer, loss, lse, workspace, bytes, vgg::Waits{}, stream);
}

extern "C" int vgg19_linear_cross_entropy_backward(const vgg19_linear_loss* layer, const float* lse, const float* d_loss, void* dx, int64_t lddx,
                                                   void* dw, int32_t dw_dtype, int64_t lddw, float* db, void* workspace, size_t bytes, void* stream) {
  using namespace vgg;
  const int rc = check(layer);
  if (rc != VGG19_OK) return rc;
  const vgg19_linear_loss& a = *layer;
  if ((dx && (lddx < a.in || lddx >= (1LL << 36))) || (dw && (lddw < a.in || lddw >= (1LL << 36))))
    return note_error(VGG19_ERR_SHAPE, "row strides %lld of dx and %lld of dw for %d values", (long long)lddx, (long long)lddw, a.in);
  if (dw && dw_dtype != VGG19_FP32 && dw_dtype != a.dtype) return note_error(VGG19_ERR_ARG, "dw is neither fp32 nor of the type of w");
  const long elt = a.dtype == VGG19_FP32 ? 4 : 2, dw_elt = dw_dtype == VGG19_FP32 ? 4 : 2, each = 4L * a.rows;
  if ((dx && reinterpret_cast<uintptr_t>(dx) % elt) || (dw && reinterpret_cast<uintptr_t>(dw) % dw_elt)) return note_error(VGG19_ERR_ARG, "dx or dw is not aligned to its type");
  if (!words(a.bias, a.labels, lse, d_loss, db)) return note_error(VGG19_ERR_ARG, "bias, labels, lse, d_loss or db is not aligned to 4 bytes");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a.rows == 0) {  // sums over no rows
    cudaError_t e = cudaSuccess;
    if (dw) e = cudaMemset2DAsync(dw, lddw * dw_elt, 0, a.in * dw_elt, a.classes, st);
    if (db && e == cudaSuccess) e = cudaMemsetAsync(db, 0, 4L * a.classes, st);
    return e == cudaSuccess ? VGG19_OK : note_error(VGG19_ERR_CUDA, "clearing the gradients failed: %s", cudaGetErrorString(e));
  }
  const int bad = check_pointers(a, workspace);
  if (bad != VGG19_OK) return bad;
  if (!lse || !d_loss) return note_error(VGG19_ERR_ARG, "lse and d_loss must not be null");
  const int pairs = pairs_of_device();
  const Plan p = make_plan(a, true, pairs);
  if (bytes < p.total) return note_error(VGG19_ERR_WORKSPACE, "workspace has %zu bytes, this call needs %zu", bytes, p.total);
  const Block all[] = {{dx, a.rows, a.in * elt, lddx * elt}, {dw, a.classes, a.in * dw_elt, lddw * dw_elt}, {db, 1, 4L * a.classes, 0}, {workspace, 1, (long)p.total, 0},
                       {a.labels, 1, each, 0}, {a.bias, 1, 4L * a.classes, 0}, {lse, 1, each, 0}, {d_loss, 1, each, 0},
                       {a.x, a.rows, a.in * elt, a.ldx * elt}, {a.w, a.classes, a.in * elt, a.ldw * elt}};
  if (blocks_meet(all, 4)) return note_error(VGG19_ERR_ARG, "an output or the workspace overlaps an input or another output");
  if (!dx && !dw && !db) return VGG19_OK;
  const Gradients g{lse, d_loss, dx, (long)lddx, dw, dw_dtype == VGG19_FP32, (long)lddw, db};
  char* ws = static_cast<char*>(workspace);
  const Waits waits{};
  const cudaError_t e = p.planes == 3 ? backward<3>(a, g, ws, p, pairs, waits, st) : backward<1>(a, g, ws, p, pairs, waits, st);
  return e == cudaSuccess ? VGG19_OK : note_error(VGG19_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}
