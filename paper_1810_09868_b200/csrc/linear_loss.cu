// The last dense layer and the softmax cross entropy of its rows in one, without keeping the logits.  For rows x of `in`
// values, weights w [classes][in], bias b and one label a row
//   z = x w^T + b,   lse_r = log sum_n exp z_rn,   loss_r = lse_r - z_r,label,
//   dz_rn = d_loss_r (exp(z_rn - lse_r) - [n = label_r]),   dx = dz w,   dw = dz^T x,   db = sum_r dz.
//
// Forward: the products z by tiles, whose epilogue keeps of each row and half a tile's classes the largest z and the sum of
// exp(z - largest), and z at the label; a second kernel joins them.  Backward: z again, tile by tile, with dz as the
// epilogue's result, for as many classes at a time ("a piece") as the workspace has room for; then dw of the piece and
// the piece's share of dx, both in one launch, the longer tiles first.  That is 8 rows in classes operations in all, where a kept matrix
// of logits would take 6, and 4 bytes a logit to write and read twice.  Sums over parts, rows and pieces are added in an order that the sizes alone
// decide: no atomics, the same bits every time.
//
// The product kernel: persistent, tcgen05 with fp32 sums in tensor memory, operands by TMA, row-major or by columns as the product asks for,
// 256 x 256 tiles by pairs of CTAs, or 128 rows by one (kShapes), two accumulators, so that eight epilogue warps work behind the next tile's
// products.  A pair loads 64 KB a K block of 64 (a CTA's own 128 rows, half of the columns), 0.32 us of loads alone and 0.33 us of
// products alone where all SMs are busy, 0.39 us together (2048 x 4096 against 50021 classes): 1.5 PFLOP/s until the power cap lowers the clock.
//
// Few tiles (a batch of 100 against 1000 classes has four) leave most SMs idle: then z's sum over the inputs is cut into parts that small
// kernels add up (fp32, in L2), which is 31 -> 11 us forward there; dx's sum over the classes likewise.  What is cut, and how tiles are, is
// decided by measured times of tiles (plan_logits, plan_gradients).
//
// fp32: a value is three bf16 planes (24 bits), a product six products of planes, those down to 2^-16 of the first; the five lesser ones
// have an accumulator of their own.  A few rows go another way (linear_loss_few.cu).
//
// Precision.  The tensor core truncates its fp32 sums, so a chain ends after 16 K blocks (8 with three planes; 64 or 512 in gradients of bf16 values) and the
// epilogue adds the chains in registers: the loss of rows of 4096 is 3e-7 from 64 bits, 1.9e-6 with one chain.  dz is fp32 until it is rounded to bf16 for the
// products (three planes in fp32); db is summed before that.  (An operand of a bf16 product has to be bf16; a second one for what the rounding leaves would
// double the products of dx and dw.  dx and dw are 2.3e-3 from 64 bits, of which the rounding of the result alone is 1.7e-3.)
//
// Measured (B200, device time): 4096 rows of 4096 against 131072 bf16 classes, loss 3.2 ms and gradients 10.5 ms, 1.28 PFLOP/s, 0.95 of the measured
// sustained rate; 2048 rows of 4096 against 50021, loss 0.57 ms, 1.47 PFLOP/s; 100 rows of 4096 against 50021, loss 83 us (4.9 TB/s of
// weights) and gradients 250 us (reading w twice at that rate, and writing dw as fast as a plain fill of its 410 MB, 107 us); 100
// against 1000, loss 10.8 and gradients 21 us, chains of latencies of two and three launches.
#include <cuda_runtime.h>

#include "../../include/vgg19_b200.h"
#include "linear_loss.cuh"
#include "tc_common.cuh"

namespace vgg {
namespace {

using namespace tc;

static __device__ int g_loss_error[1];   // a DeviceError code once a bounded wait of a call without a handle ran out
static __device__ int g_label_error[1];  // kDevBadLabel once a label outside [0, classes) was met

// ---- sizes -----------------------------------------------------------------------------------------------------
constexpr int BM = 128, BN = 256, BK = 64;   // rows of a CTA (a pair has 256), columns of a tile (at most: 256, 192 or 128), K per stage
constexpr int kBoxBytes = 64 * BK * 2;       // what one copy brings: 64 x 64 values
// P planes: bf16 values are one plane, fp32 values three (each the bf16 rounding of what the ones before leave: 24 bits).
// PAIR: two CTAs work on a tile of 256 rows, each with its 128 and half of the columns' operand in shared memory; else one on 128 rows, for
// what has no more: a pair would multiply nothing by 128 of its rows.  With three planes such a tile has 128 columns at most.
template <bool PAIR> constexpr int kTileRows = PAIR ? 2 * BM : BM;
constexpr int kPlaneBytes = 2 * kBoxBytes;   // 128 rows
template <int P, bool PAIR> constexpr int kOtherBoxes = PAIR || P == 3 ? 2 : 4;  // of the columns' operand, a plane
template <int P, bool PAIR> constexpr int kStageBytes = P * (kPlaneBytes + kOtherBoxes<P, PAIR> * kBoxBytes);
constexpr int kRingBytes = 192 * 1024;
template <int P, bool PAIR> constexpr int kStages = kRingBytes / kStageBytes<P, PAIR>;
static_assert(kStages<1, true> == 6 && kStages<1, false> == 4 && kStages<3, true> == 2 && kStages<3, false> == 2, "whole stages");
template <int P> constexpr int kBuffers = P == 1 ? 2 : 1;  // accumulators: with three planes one, and one for the small products
constexpr int kEpilogueWarps = 8, kThreads = 128 + 32 * kEpilogueWarps;  // a warpgroup for producer and issuer, two of epilogue warps
// Registers per thread after the split: 168 at launch, 3 x 168 = 40 + 2 x 232.
constexpr int kFewRegisters = 40, kManyRegisters = 232;
constexpr int kPieceBytes = 4096;            // an epilogue warp's own 32 rows of 128 bytes
constexpr int kBiasBytes = 128;              // its 32 biases
constexpr int kSmemBytes = kRingBytes + kEpilogueWarps * (kPieceBytes + kBiasBytes) + 1024 + 256;

// What a tile's sums become: the statistics of its rows, dz, the product itself, or parts of z's sum (kept in fp32, added up in chains).
// kLongProduct: a product whose sums are too long for one chain.
enum Epilogue { kStatistics, kLogitGradient, kProduct, kSums, kLongProduct };

// What one CTA, or a pair, does.
template <bool PAIR> __device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
  if (PAIR) tma_load_3d_pair(dst, map, bar, c0, c1, c2); else tma_load_3d(dst, map, bar, c0, c1, c2);
}
template <bool PAIR> __device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t more) {
  if (PAIR) umma_bf16_pair(d, a, b, idesc, more); else umma_bf16(d, a, b, idesc, more);
}
template <bool PAIR> __device__ __forceinline__ void signal_when_done(uint32_t bar, uint16_t ctas) {
  if (PAIR) umma_commit_pair(bar, ctas); else umma_commit(bar);
}
__device__ __noinline__ void report(const Waits& waits, int code) { atomicCAS(waits.error ? waits.error : g_loss_error, 0, code); }

// ---- one product -------------------------------------------------------------------------------------------------
// D[i][j] = sum_k A(i, k) B(j, k), m x n, in tiles.  An operand lies K-major (a row per i or j) or, with _mn, with a row per k.
// Results leave 16 bytes a lane, into rows that have room for whole 16 bytes or not, are added to fp32 that is there, or leave one value a
// lane (rows of any alignment).
enum Store { kWhole, kPadded, kAdded, kSingle };
struct __align__(64) Job {
  CUtensorMap a, b;
  int m, n, k_blocks, tiles_m, tiles_n;
  int bn;                 // columns of a tile
  int group;              // rows of tiles that are worked on together
  int splits, per_split;  // the sum cut into that many parts, of that many K blocks; part s is plane s of the result
  int chain;              // K blocks that the tensor cores add up before the sums go to the epilogue's registers
  int longest;            // how many those may be, in a product of bf16 values
  int a_mn, b_mn;
  int store, f32;         // f32: the result is fp32, else bf16
  void* out;              // row stride ld, planes m * ld apart
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
// A worker's tile of a round: every other round from the other end, so that who has a long one in the first has none in a last round that is
// not full.
__device__ __forceinline__ int turn(int round, int worker, int workers) { return round * workers + (round & 1 ? workers - 1 - worker : worker); }
// A few rows of tiles at a time, which share their columns' operand: both operands then stay in L2 while they are needed.
__device__ __forceinline__ Tile find_tile(const Job& p, int t) {
  Tile r{};
  const int all = p.tiles_m * p.tiles_n;
  r.split = t / all;
  t -= r.split * all;
  const int first = t / (p.group * p.tiles_n) * p.group, height = min(p.group, p.tiles_m - first);
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

// What a piece holds of a tile that ends within it, or whose rows are not aligned, or are added to: `rows` and `cols` from `out` on.
__device__ __noinline__ void put_some(const uint4* piece, char* out, long ld, int rows, int cols, int elt, int store) {
  const int lane = threadIdx.x & 31, n = 16 / elt;
  if (store == kSingle) {
    const int last = min(rows, 32), wide = min(cols, 8 * n);
    for (int r = 0; r < last; ++r, out += ld * elt)
      for (int c = lane; c < wide; c += 32) {
        if (elt == 4) reinterpret_cast<float*>(out)[c] = reinterpret_cast<const float*>(piece + piece_at(r, c / 4))[c % 4];
        else reinterpret_cast<unsigned short*>(out)[c] = reinterpret_cast<const unsigned short*>(piece + piece_at(r, c / 8))[c % 8];
      }
    return;
  }
  const int r0 = lane / 8, k0 = lane % 8, left = cols - k0 * n;
  out += r0 * ld * elt + 16 * k0;
  if (left <= 0) return;
  for (int r = r0; r < min(rows, 32); r += 4, out += 4 * ld * elt) {
    const uint4 w = piece[piece_at(r, k0)];
    if (store == kAdded) {  // (fp32, and rows have room for whole fours)
      const float4 old = *reinterpret_cast<const float4*>(out);
      *reinterpret_cast<float4*>(out) = make_float4(__uint_as_float(w.x) + old.x, __uint_as_float(w.y) + old.y, __uint_as_float(w.z) + old.z, __uint_as_float(w.w) + old.w);
    } else if (left >= n || store == kPadded) {
      *reinterpret_cast<uint4*>(out) = w;
    } else {
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
      for (int e = 0; e < left; ++e) {
        const uint32_t one = e < 2 * (4 / elt) ? (e < 4 / elt ? u[0] : u[1]) : (e < 3 * (4 / elt) ? u[2] : u[3]);
        if (elt == 4) reinterpret_cast<uint32_t*>(out)[e] = one;
        else reinterpret_cast<unsigned short*>(out)[e] = (unsigned short)(one >> (16 * (e & 1)));
      }
    }
  }
}

template <int P, int EPI, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1) loss_product_kernel(const __grid_constant__ Launch L) {
  constexpr int STAGES = kStages<P, PAIR>, STAGE_BYTES = kStageBytes<P, PAIR>, BUFFERS = kBuffers<P>, OTHER = kOtherBoxes<P, PAIR>;
  constexpr bool PRODUCT = EPI == kProduct || EPI == kLongProduct;
  constexpr bool CHAINED = EPI != kSums && (P == 3 || EPI != kProduct);  // whether a tile's sums may come in several chains
  constexpr bool DIRECT = !CHAINED || EPI == kLongProduct;              // whether one chain may go to memory as it is
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
  const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
  const bool leader = rank == 0;
  const int worker = PAIR ? blockIdx.x >> 1 : blockIdx.x, workers = PAIR ? gridDim.x >> 1 : gridDim.x, total = L.first_tile[L.count];

  if (threadIdx.x == 32) {
    tma_prefetch_desc(&L.job[0].a);
    tma_prefetch_desc(&L.job[0].b);
  }
  if (threadIdx.x == 0) {
    abort_flag = ran_out = 0;
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), L.waits.signals); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < BUFFERS; ++b) { mbar_init(acc_full_bar(b), 1); mbar_init(acc_empty_bar(b), (PAIR ? 2 : 1) * kEpilogueWarps); }
    mbar_init(drain_bar, 1);
    mbar_fence_init();
  }
  if (warp == 1) {
    if (PAIR) {
      tmem_alloc_pair(smem_u32(&tmem_base_slot), 512);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(smem_u32(&tmem_base_slot), 512);
      tmem_relinquish();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();  // the peer's barriers are initialised before anything signals them
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
      for (int round = 0, w; ok && (w = turn(round, worker, workers)) < total; ++round) {
        while (w >= L.first_tile[ji + 1]) ++ji;
        const Job& p = L.job[ji];
        const Tile tile = find_tile(p, w - L.first_tile[ji]);
        const int row = tile.i * kTileRows<PAIR> + (int)rank * BM, bn = p.bn, col = tile.j * bn + (int)rank * (bn / 2), a_mn = p.a_mn, b_mn = p.b_mn;
        const int boxes = PAIR ? (bn + 127) / 128 : bn / 64;  // of B, a plane
        for (int kb = tile.k0; kb < tile.k1; ++kb) {
          if (!mbar_wait(empty_bar(stage), phase ^ 1, &abort_flag, &ran_out, kDevTimeoutStageFree, L.waits.limit_cycles)) { ok = false; break; }
          const uint32_t sa = smem_base + stage * STAGE_BYTES, sb = sa + P * kPlaneBytes;
          const uint32_t full = PAIR ? map_to_cta(full_bar(stage), 0) : full_bar(stage);
          // the even CTA announces the bytes of both CTAs' copies; what lies outside a matrix arrives as zeros
          if (leader) mbar_expect_tx(full_bar(stage), (PAIR ? 2 : 1) * P * (kPlaneBytes + boxes * kBoxBytes));
#pragma unroll
          for (int h = 0; h < P; ++h)
#pragma unroll
            for (int q = 0; q < OTHER; ++q) {
              const int r = row + 64 * q, c = col + 64 * q, k = kb * BK;
              if (q < 2) load_box<PAIR>(sa + h * kPlaneBytes + q * kBoxBytes, &p.a, full, a_mn ? r : k, a_mn ? k : r, h);
              if (q < boxes) load_box<PAIR>(sb + (h * OTHER + q) * kBoxBytes, &p.b, full, b_mn ? c : k, b_mn ? k : c, h);
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
      for (int round = 0, w; ok && (w = turn(round, worker, workers)) < total; ++round) {
        while (w >= L.first_tile[ji + 1]) ++ji;
        const Job& p = L.job[ji];
        const Tile tile = find_tile(p, w - L.first_tile[ji]);
        // K-major: 16 k = 32 bytes of the swizzled row.  A row per k: two boxes of 64 columns, 16 k = 16 rows.
        const uint32_t idesc = umma_idesc_bf16(kTileRows<PAIR>, p.bn, p.a_mn, p.b_mn);
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
              b[h] = smem_desc_sw128(sb + h * OTHER * kBoxBytes, b_lbo);
            }
#pragma unroll
            for (int k = 0; k < BK / 16; ++k) {
              const uint32_t more = kb != kb0 || k ? 1u : 0u;
              multiply<PAIR>(d, desc_advance(a[0], k * a_step), desc_advance(b[0], k * b_step), idesc, more);
              if (P == 3) {
                // the products of the lesser planes, at most 2^-8 of the first, have a sum of their own: the tensor core truncates
                // its sums, relative to their size, so the chain that matters has a sixth of the instructions
                auto small = [&](int u, int v, uint32_t m) {
                  multiply<PAIR>(tmem_base + BN, desc_advance(a[u], k * a_step), desc_advance(b[v], k * b_step), idesc, m);
                };
                small(0, P - 1, more);
                small(P - 1, 0, 1u);
                small(1 % P, 1 % P, 1u);
                small(0, 1 % P, 1u);
                small(1 % P, 0, 1u);
              }
            }
            signal_when_done<PAIR>(empty_bar(stage), 3);  // frees the stage in both CTAs
            if (++stage == STAGES) { stage = 0; phase ^= 1; }
          }
          if (ok) signal_when_done<PAIR>(acc_full_bar(buf), 3);
        }
      }
      if (!ok) {
        signal_when_done<PAIR>(drain_bar, 1);
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
    // What a tile of z needs of its rows and columns: requested while the tile before is worked on.
    constexpr bool LOGITS = EPI == kStatistics || EPI == kLogitGradient;
    struct {
      int i, j, label;
      float lse, d_loss, bias[4];
    } next;
    auto request = [&](int w) {
      if (w >= total) return;
      const Job& p = L.job[0];
      const Tile tile = find_tile(p, w);
      const int half = p.bn / 2, row = tile.i * kTileRows<PAIR> + (int)rank * BM + quarter * 32 + lane, j0 = tile.j * p.bn + group * half, cols = min(p.n - j0, half);
      next.i = tile.i; next.j = tile.j;
      next.label = VGG19_NO_CLASS;
      next.lse = next.d_loss = 0.f;
      if (row < p.m) {
        next.label = L.rows.labels[row];
        if (EPI == kLogitGradient) { next.lse = L.rows.lse[row]; next.d_loss = L.rows.d_loss[row]; }
      }
      // columns beyond the classes get the bias of an excluded class
#pragma unroll
      for (int k = 0; k < 4; ++k) next.bias[k] = 32 * k + lane < cols ? L.rows.bias ? L.rows.bias[j0 + 32 * k + lane] : 0.f : -INFINITY;
    };
    if (LOGITS) request(turn(0, worker, workers));
    for (int round = 0, w; ok && (w = turn(round, worker, workers)) < total; ++round) {
      if (!LOGITS) while (w >= L.first_tile[ji + 1]) ++ji;
      const Job& p = L.job[ji];
      Tile tile{};
      if (LOGITS) { tile.i = next.i; tile.j = next.j; tile.k1 = p.k_blocks; }
      else tile = find_tile(p, w - L.first_tile[ji]);
      const int half = p.bn / 2;
      const int i0 = tile.i * kTileRows<PAIR> + (int)rank * BM + quarter * 32, j0 = tile.j * p.bn + group * half;  // the warp's first row and column
      const int rows = p.m - i0, cols = min(p.n - j0, half);                                         // what there is from there on
      const int row = i0 + lane;
      if (PRODUCT && p.db && tile.j == 0 && group == 0 && tile.split == 0 && lane < rows) {
        float s[8] = {};  // (as sum_columns_kernel adds them)
        for (int q = 0; q < p.parts; q += 8) {
#pragma unroll
          for (int k = 0; k < 8; ++k) s[k] += q + k < p.parts ? p.db_part[(long)(q + k) * p.m + row] : 0.f;
        }
#pragma unroll
        for (int k = 1; k < 8; ++k) s[0] += s[k];
        p.db[row] = s[0];
      }
      // The piece, `from` on of the half's columns, to memory: lanes along the rows, four whole 128-byte lines at a time.
      const int elt = EPI == kSums || (PRODUCT && p.f32) ? 4 : 2;
      const bool whole = rows >= 32 && cols == half && (EPI == kLogitGradient || p.store <= kPadded);
      char* const out = EPI == kStatistics ? nullptr : static_cast<char*>(p.out) + (((long)(EPI == kLogitGradient ? 0 : tile.split) * p.m + i0) * p.ld + j0) * elt;
      auto put_piece = [&](int from, int plane) {
        __syncwarp();
        char* at = out + (plane * p.m * p.ld + from) * elt;
        if (whole && from + 128 / elt <= half) {
          const int r0 = lane / 8, k0 = lane % 8;
          uint4 w[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) w[q] = piece[piece_at(q * 4 + r0, k0)];
          const long step = 4 * p.ld * elt;
          at += r0 * p.ld * elt + 16 * k0;
#pragma unroll
          for (int q = 0; q < 8; ++q, at += step) *reinterpret_cast<uint4*>(at) = w[q];
        } else {
          put_some(piece, at, p.ld, rows, cols - from, elt, EPI == kLogitGradient ? (int)kPadded : p.store);
        }
        __syncwarp();
      };
      auto sums_are_there = [&] {
        const int buf = count % BUFFERS;
        return __all_sync(0xffffffffu, mbar_wait(acc_full_bar(buf), (count / BUFFERS) & 1, &abort_flag, &ran_out, kDevTimeoutAccum, L.waits.limit_cycles)) != 0;
      };
      auto sums_are_read = [&] {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR) mbar_arrive_cluster(map_to_cta(acc_empty_bar(count % BUFFERS), 0)); else mbar_arrive(acc_empty_bar(count % BUFFERS));
        }
        ++count;
      };
      auto sums_at = [&] { return tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)((count % BUFFERS) * BN + group * half); };

      const bool direct = !CHAINED || (DIRECT && tile.k1 - tile.k0 <= p.chain);
      if (DIRECT && direct) {
        // one chain, and nothing to compute: 128 bytes of a row at a time, in little code (a call of few tiles runs it once, from memory)
        if (!sums_are_there()) { ok = false; break; }
        tc_fence_after();
        const uint32_t src = sums_at();
        const int most = min(half, (cols + 31) / 32 * 32);  // columns that anything is done with
        if (rows > 0) {
          if (elt == 4) {
#pragma unroll 1
            for (int c0 = 0; c0 < most; c0 += 32) {
              uint32_t t[32];
              tmem_ld_32x32(src + c0, t);
              if (P == 3) {
                uint32_t u[32];
                tmem_ld_32x32(src + BN + c0, u);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 32; ++j) t[j] = __float_as_uint(__uint_as_float(t[j]) + __uint_as_float(u[j]));
              } else {
                tmem_ld_wait();
              }
#pragma unroll
              for (int k = 0; k < 8; ++k) piece[piece_at(lane, k)] = make_uint4(t[4 * k], t[4 * k + 1], t[4 * k + 2], t[4 * k + 3]);
              put_piece(c0, 0);
            }
          } else {
#pragma unroll 1
            for (int c0 = 0; c0 < most; c0 += 64) {
              uint32_t t[2][32];
              tmem_ld_32x32(src + c0, t[0]);
              tmem_ld_32x32(src + c0 + 32, t[1]);
              tmem_ld_wait();
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const uint32_t* e = t[k / 4] + k % 4 * 8;
                auto two = [&](int j) { return pack2(__uint_as_float(e[j]), __uint_as_float(e[j + 1])); };
                piece[piece_at(lane, k)] = make_uint4(two(0), two(2), two(4), two(6));
              }
              put_piece(c0, 0);
            }
          }
        }
        sums_are_read();
      }
      if constexpr (CHAINED) if (!DIRECT || !direct) {
        float v[128];  // the tile's sums of this row and half
        for (long kb0 = tile.k0; kb0 < tile.k1; kb0 += p.chain) {
          if (!sums_are_there()) { ok = false; break; }
          tc_fence_after();
          const uint32_t src = sums_at();
          if (kb0 == tile.k0) {
            uint32_t t[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld_32x32(src + 32 * c, t[c]);  // (of a narrow tile the second two mean nothing)
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 128; ++j) v[j] = __uint_as_float(t[j / 32][j % 32]);
          }
          if (P == 3 || kb0 != tile.k0) {
            for (int plane = kb0 == tile.k0; plane < (P == 3 ? 2 : 1); ++plane) {
#pragma unroll
              for (int c = 0; c < 128; c += 32) {
                uint32_t t[32];
                tmem_ld_32x32(src + plane * BN + c, t);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 32; ++j) v[c + j] += __uint_as_float(t[j]);
              }
            }
          }
          sums_are_read();
        }
        if (!ok) break;
        float lse = 0.f, d_loss = 0.f, bias[4];
        int label = VGG19_NO_CLASS;
        if (LOGITS) {
          label = next.label; lse = next.lse; d_loss = next.d_loss;
#pragma unroll
          for (int k = 0; k < 4; ++k) bias[k] = next.bias[k];
          request(turn(round + 1, worker, workers));
          const bool real = (unsigned)label < (unsigned)L.rows.all_classes;
          if (EPI == kLogitGradient) {
            if (!real && label != VGG19_NO_CLASS && j0 == 0) atomicCAS(g_label_error, 0, (int)kDevBadLabel);
            // no label, or no class left: no gradient
            if (!real || lse == -INFINITY) d_loss = 0.f;
            label = d_loss != 0.f || d_loss != d_loss ? label - L.rows.first_class : -1;
          } else {
            label = real ? label - L.rows.first_class : -1;
          }
        }
        auto add_bias = [&](int c) {
          bias_s[lane] = bias[c / 32];
          __syncwarp();
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const float4 b = reinterpret_cast<const float4*>(bias_s)[q];
            v[c + 4 * q] += b.x; v[c + 4 * q + 1] += b.y; v[c + 4 * q + 2] += b.z; v[c + 4 * q + 3] += b.w;
          }
          __syncwarp();
        };

        if (EPI == kStatistics) {
          float four[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, sum = 0.f;
#pragma unroll
          for (int c = 0; c < 128; c += 32) {
            if (c >= half) break;
            add_bias(c);
#pragma unroll
            for (int j = 0; j < 32; ++j) four[j % 4] = fmaxf(four[j % 4], v[c + j]);
            const int at = label - j0 - c;  // the label's column among these
            if (__any_sync(0xffffffffu, (unsigned)at < 32u)) {
              float z = 0.f;
#pragma unroll
              for (int j = 0; j < 32; ++j) z = at == j ? v[c + j] : z;
              if ((unsigned)at < 32u && at < cols - c) L.rows.label_z[row] = z;
            }
          }
          const float most = fmaxf(fmaxf(four[0], four[1]), fmaxf(four[2], four[3])), ref = most == -INFINITY ? 0.f : most;
#pragma unroll
          for (int c = 0; c < 128; c += 32) {
            if (c >= half) break;
            float part[4] = {};
#pragma unroll
            for (int j = 0; j < 32; ++j) part[j % 4] += fast_exp2((v[c + j] - ref) * kLossLog2e);
            sum += part[0] + part[1] + (part[2] + part[3]);
          }
          if (cols < half && sum != sum) {
            // an infinity among x times the zeros beyond the classes is no number, whatever is added to it: the sum again without them (the
            // largest has not taken it)
            sum = 0.f;
#pragma unroll
            for (int j = 0; j < 128; ++j)
              if (j < cols) sum += fast_exp2((v[j] - ref) * kLossLog2e);
          }
          if (lane < rows && cols > 0) L.rows.part[(long)(L.rows.first_part + 2 * tile.j + group) * p.m + row] = make_float2(most, sum);
        } else if (EPI == kLogitGradient) {
          const float ref = lse == -INFINITY ? 0.f : lse;
#pragma unroll
          for (int c0 = 0; c0 < 128; c0 += 64) {
            if (c0 >= half) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int c = c0 + 32 * h;
              add_bias(c);
              const int at = label - j0 - c;
#pragma unroll
              for (int j = 0; j < 32; ++j) v[c + j] = fast_exp2((v[c + j] - ref) * kLossLog2e);
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
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const int e = c0 + 8 * k;
                uint4 w;
                if (P == 1) {
                  w = make_uint4(pack2(v[e], v[e + 1]), pack2(v[e + 2], v[e + 3]), pack2(v[e + 4], v[e + 5]), pack2(v[e + 6], v[e + 7]));
                } else {
                  w.x = take2(v[e], v[e + 1]); w.y = take2(v[e + 2], v[e + 3]);
                  w.z = take2(v[e + 4], v[e + 5]); w.w = take2(v[e + 6], v[e + 7]);
                }
                piece[piece_at(lane, k)] = w;
              }
              put_piece(c0, h);
            }
          }
        } else if (P == 1 && elt == 2) {
#pragma unroll
          for (int c0 = 0; c0 < 128; c0 += 64) {
            if (c0 >= min(cols, half)) break;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const int e = c0 + 8 * k;
              piece[piece_at(lane, k)] = make_uint4(pack2(v[e], v[e + 1]), pack2(v[e + 2], v[e + 3]), pack2(v[e + 4], v[e + 5]), pack2(v[e + 6], v[e + 7]));
            }
            put_piece(c0, 0);
          }
        } else {
#pragma unroll
          for (int c0 = 0; c0 < 128; c0 += 32) {  // (of three planes always)
            if (c0 >= cols) break;
#pragma unroll
            for (int k = 0; k < 8; ++k)
              piece[piece_at(lane, k)] = make_uint4(__float_as_uint(v[c0 + 4 * k]), __float_as_uint(v[c0 + 4 * k + 1]), __float_as_uint(v[c0 + 4 * k + 2]),
                                                    __float_as_uint(v[c0 + 4 * k + 3]));
            put_piece(c0, 0);
          }
        }
      }
    }
  }

  // Neither CTA may release tensor memory or exit while the other can still signal its barriers, read its shared
  // memory or write its accumulator.
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();
  if (threadIdx.x == 0 && ran_out) report(L.waits, ran_out);
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    if (PAIR) tmem_dealloc_pair(tmem_base, 512); else tmem_dealloc(tmem_base, 512);
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
constexpr int kJoinRows = 4, kJoinGroups = 64;  // rows of a block (whole sectors), and threads of each

// What a row answers with.
__device__ __forceinline__ void finish_row(float2 v, int label, int classes, float label_z, float* loss, float* lse) {
  const float log_sum = logf(v.y), sum = v.x + log_sum;
  if (lse) *lse = sum;
  float l = 0.f;
  if ((unsigned)label < (unsigned)classes) {
    // (the largest z less the label's is exact where they are near each other, so a loss near 0 is not a difference of two roundings)
    l = sum == -INFINITY ? INFINITY : v.x - label_z + log_sum;
  } else if (label != VGG19_NO_CLASS) {
    l = __int_as_float(0x7fc00000);
    atomicCAS(g_label_error, 0, (int)kDevBadLabel);
  }
  if (loss) *loss = l;
}

__global__ void __launch_bounds__(kJoinRows * kJoinGroups) join_rows_kernel(const __grid_constant__ Join a) {
  __shared__ float2 got[kJoinGroups][kJoinRows];
  behind_previous();
  const int r = threadIdx.x % kJoinRows, group = threadIdx.x / kJoinRows, row = blockIdx.x * kJoinRows + r;
  float2 v = make_float2(-INFINITY, 0.f);
  if (row < a.rows) {
#pragma unroll 4
    for (int p = group; p < a.parts; p += kJoinGroups) v = join(v, a.part[(long)p * a.rows + row]);
  }
  got[group][r] = v;
#pragma unroll
  for (int n = kJoinGroups / 2; n; n /= 2) {
    __syncthreads();
    if (group < n) got[group][r] = v = join(v, got[group + n][r]);
  }
  if (group || row >= a.rows) return;
  finish_row(v, a.labels[row], a.classes, a.label_z[row], a.loss ? a.loss + row : nullptr, a.lse ? a.lse + row : nullptr);
}

// ---- few tiles: z in parts of its sum -----------------------------------------------------------------------------------
// Where z has too few tiles for the pairs, its sum over the inputs is cut among them and the parts, [parts][rows][ld] in fp32, are
// added here: a small matrix, that stays in L2.
struct Parts {
  const float* z;
  int parts, rows, classes;
  long ld;
  const float* bias;
  const int32_t* labels;
  // forward
  float *loss, *lse_out;
  // backward
  const float *lse, *d_loss;
  bf16* dz;
  long dz_ld;
  float* db_part;  // [rows / kPartRows][classes], or null
};
__device__ __forceinline__ float4 sum_of_parts(const Parts& a, int row, int c) {
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  const float* at = a.z + (long)row * a.ld + c;
  for (int p = 0; p < a.parts; p += 8) {  // eight requests at once, the last ones too
    float4 v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k, at += a.rows * a.ld) v[k] = p + k < a.parts ? __ldcg(reinterpret_cast<const float4*>(at)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < 8; ++k) { s.x += v[k].x; s.y += v[k].y; s.z += v[k].z; s.w += v[k].w; }
  }
  const float none = -INFINITY;  // beyond the classes
  auto bias = [&](int k) { return c + k < a.classes ? a.bias ? a.bias[c + k] : 0.f : none; };
  s.x = c < a.classes ? s.x + bias(0) : none;
  s.y = c + 1 < a.classes ? s.y + bias(1) : none;
  s.z = c + 2 < a.classes ? s.z + bias(2) : none;
  s.w = c + 3 < a.classes ? s.w + bias(3) : none;
  return s;
}

constexpr int kRowThreads = 256;
constexpr unsigned kFirstLanes = (1u << kRowThreads / 32) - 1;  // a lane for each of the warps
// loss and log-sum-exp of a row a block
__global__ void __launch_bounds__(kRowThreads) loss_of_parts_kernel(const __grid_constant__ Parts a) {
  __shared__ float2 got[kRowThreads / 32];
  __shared__ float label_z;
  behind_previous();
  const int row = blockIdx.x, label = a.labels[row];
  float2 v = make_float2(-INFINITY, 0.f);
  for (int c = 4 * threadIdx.x; c < a.classes; c += 4 * kRowThreads) {
    const float4 z = sum_of_parts(a, row, c);
    if ((unsigned)(label - c) < 4u && label < a.classes) label_z = label - c == 0 ? z.x : label - c == 1 ? z.y : label - c == 2 ? z.z : z.w;
    const float m = fmaxf(fmaxf(z.x, z.y), fmaxf(z.z, z.w)), ref = m == -INFINITY ? 0.f : m;
    v = join(v, make_float2(m, (fast_exp2((z.x - ref) * kLossLog2e) + fast_exp2((z.y - ref) * kLossLog2e)) + (fast_exp2((z.z - ref) * kLossLog2e) + fast_exp2((z.w - ref) * kLossLog2e))));
  }
#pragma unroll
  for (int n = 16; n; n /= 2) v = join(v, make_float2(__shfl_down_sync(0xffffffffu, v.x, n), __shfl_down_sync(0xffffffffu, v.y, n)));
  if (threadIdx.x % 32 == 0) got[threadIdx.x / 32] = v;
  __syncthreads();
  if (threadIdx.x >= kRowThreads / 32) return;
  v = got[threadIdx.x];
#pragma unroll
  for (int n = kRowThreads / 64; n; n /= 2) v = join(v, make_float2(__shfl_down_sync(kFirstLanes, v.x, n), __shfl_down_sync(kFirstLanes, v.y, n)));
  if (threadIdx.x) return;
  finish_row(v, label, a.classes, label_z, a.loss ? a.loss + row : nullptr, a.lse_out ? a.lse_out + row : nullptr);
}

constexpr int kPartRows = 8;  // rows of a block
// dz, P planes, of kPartRows rows and 128 classes a block, and their sums over the rows
template <int P> __global__ void __launch_bounds__(32 * kPartRows) gradient_of_parts_kernel(const __grid_constant__ Parts a) {
  __shared__ float4 sums[kPartRows][32];
  behind_previous();
  const int r = threadIdx.x / 32, row = blockIdx.y * kPartRows + r, c = blockIdx.x * 128 + threadIdx.x % 32 * 4;
  float g[4] = {0.f, 0.f, 0.f, 0.f};
  if (row < a.rows && c < a.classes) {
    const float4 z = sum_of_parts(a, row, c);
    const int label = a.labels[row];
    const bool real = (unsigned)label < (unsigned)a.classes;
    const float lse = a.lse[row], d_loss = real && lse != -INFINITY ? a.d_loss[row] : 0.f;
    if (!real && label != VGG19_NO_CLASS && c == 0) atomicCAS(g_label_error, 0, (int)kDevBadLabel);
    const float v[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float e = fast_exp2((v[k] - lse) * kLossLog2e);
      g[k] = d_loss == 0.f ? 0.f : d_loss * (label - c == k ? e - 1.f : e);
    }
  }
  if (a.db_part) {
    sums[r][threadIdx.x % 32] = make_float4(g[0], g[1], g[2], g[3]);
    __syncthreads();
    if (threadIdx.x < 128) {
      const float* at = reinterpret_cast<const float*>(sums) + threadIdx.x;
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < kPartRows; ++k) s += at[128 * k];
      const int mine = blockIdx.x * 128 + threadIdx.x;
      if (mine < a.classes) a.db_part[(long)blockIdx.y * a.classes + mine] = s;
    }
  }
  if (row >= a.rows || c >= a.classes) return;
#pragma unroll
  for (int h = 0; h < P; ++h) {  // (rows have room for whole eights)
    uint2 w;
    w.x = take2(g[0], g[1]);
    w.y = take2(g[2], g[3]);
    *reinterpret_cast<uint2*>(a.dz + ((long)h * a.rows + row) * a.dz_ld + c) = w;
  }
}

// ---- rows as planes of bf16 ------------------------------------------------------------------------------------------
// dst[h][r][k], row stride ld (a multiple of 8): the value itself, or an fp32 value's three terms.  Two matrices of as many columns at once.
struct Layout {
  const void* src[2];
  bf16* dst[2];
  long src_ld[2], rows[2];  // (no rows: nothing)
  int in;
  long ld;
};
template <typename T, int P>
__global__ void __launch_bounds__(256) planes_kernel(const __grid_constant__ Layout a) {
  behind_previous();
  const int chunks = (int)(a.ld / 8);
  const long all = (a.rows[0] + a.rows[1]) * chunks;
  for (long t = (long)blockIdx.x * blockDim.x + threadIdx.x; t < all; t += (long)gridDim.x * blockDim.x) {
    const long row = (unsigned long)t < 0x100000000ul ? (unsigned)t / (unsigned)chunks : t / chunks;
    const int k = (int)(t - row * chunks) * 8;
    const bool second = row >= a.rows[0];
    const long r = second ? row - a.rows[0] : row, rows = second ? a.rows[1] : a.rows[0];
    const T* at = static_cast<const T*>(second ? a.src[1] : a.src[0]) + r * (second ? a.src_ld[1] : a.src_ld[0]) + k;
    bf16* dst = second ? a.dst[1] : a.dst[0];
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = k + e < a.in ? to_f32(at[e]) : 0.f;
#pragma unroll
    for (int h = 0; h < P; ++h) {
      uint4 q;
      q.x = take2(v[0], v[1]); q.y = take2(v[2], v[3]); q.z = take2(v[4], v[5]); q.w = take2(v[6], v[7]);
      *reinterpret_cast<uint4*>(dst + (h * rows + r) * a.ld + k) = q;
    }
  }
}

// ---- dx from its parts -----------------------------------------------------------------------------------------------
// GROUPS: threads that share a sum of many parts, for few values.
template <typename T, int GROUPS>
__global__ void __launch_bounds__(256) sum_parts_kernel(const float* part, int parts, long rows, int in, long ld, T* out, long out_ld) {
  constexpr int WIDE = 256 / GROUPS;
  __shared__ float4 got[GROUPS][WIDE];
  behind_previous();
  const int chunks = (int)(ld / 4), lane = threadIdx.x % WIDE, group = threadIdx.x / WIDE;
  const long all = rows * chunks;
  for (long t0 = (long)blockIdx.x * WIDE; t0 < all; t0 += (long)gridDim.x * WIDE) {
    const long t = t0 + lane, r = t / chunks;
    const int k = (int)(t - r * chunks) * 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (t < all)
      for (int p = group; p < parts; p += 8 * GROUPS) {  // eight requests at once, the last ones too
        float4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          v[i] = p + i * GROUPS < parts ? *reinterpret_cast<const float4*>(part + ((p + i * GROUPS) * rows + r) * ld + k) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 8; ++i) { s.x += v[i].x; s.y += v[i].y; s.z += v[i].z; s.w += v[i].w; }
      }
    if (GROUPS > 1) {
      got[group][lane] = s;
      __syncthreads();
      if (group == 0) {
#pragma unroll
        for (int g = 1; g < GROUPS; ++g) { s.x += got[g][lane].x; s.y += got[g][lane].y; s.z += got[g][lane].z; s.w += got[g][lane].w; }
      }
      __syncthreads();
    }
    const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (group == 0 && t < all && k + e < in) out[r * out_ld + k + e] = from_f32<T>(v[e]);
  }
}

// db of a piece where no product of dw does it on the way
__global__ void __launch_bounds__(256) sum_columns_kernel(const float* part, int parts, int n, float* db) {
  __shared__ float got[8][32];
  behind_previous();
  const int lane = threadIdx.x % 32, group = threadIdx.x / 32, c = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < n) {
#pragma unroll 8
    for (int q = group; q < parts; q += 8) s += part[(long)q * n + c];
  }
  got[group][lane] = s;
  __syncthreads();
  if (group || c >= n) return;
#pragma unroll
  for (int g = 1; g < 8; ++g) s += got[g][lane];
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
// How tiles are cut: by pairs or by single CTAs, and their columns.
struct Shape {
  bool pair;
  int bn;
};
// How a call is cut up, and where its parts lie in the workspace.
struct Plan {
  int few;                // not 0: few rows of fp32, on the CUDA cores, with so many parts; of what follows there are then part, label_z, dz and dx alone
  int planes;             // 1 or 3
  bool take_x, take_w;    // whether they are laid out anew (as planes, or to be read by copies at all)
  long ld;                // row stride of what is
  long piece;             // classes at a time
  int pieces;
  Shape z_shape;          // z's tiles, and parts of its sum where there are few of them
  int z_splits;
  int db_rows;            // rows whose dz a part of db has summed
  Shape dx_shape, dw_shape;  // (pairs both, or none)
  int dx_splits;          // parts of dx's sum within a piece
  bool dx_parts;          // whether dx is added up in fp32 outside the products
  int dw_splits;          // the same of dw's, with all classes in one piece
  long dx_ld;
  size_t x, w, z, part, label_z, dz, db_part, dx, dw, total;
};

int pairs_of_device() {
  int dev = 0, sms = 148;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms / 2;
}

// The tensor core truncates its fp32 sums, an error that grows with the chain: 1.8e-6 of the loss over 4096 values in one chain.  The
// sums of shorter ones are added in registers, rounded to nearest.
// (Parts of z's sum are no longer than a chain.)
constexpr int kOneChain = 1 << 30;
constexpr int chain_blocks(int planes, int epilogue) { return epilogue == kSums || (epilogue == kProduct && planes == 1) ? kOneChain : planes == 3 ? 8 : 16; }
// Gradients of bf16 values, whose dz is rounded to bf16 anyway, take longer ones.  An instruction adds 16 products and loses less than a step of
// the sum so far, 2^-23 of it, always towards zero: 64 K blocks, 256 instructions, less than 3.1e-5 of a sum of one sign, 512 less than
// 2.5e-4, a sixteenth of the half step 2^-8 that the result is rounded by.  (One chain over 1.2 million rows was 5.2e-3 off.  The shorter ones cost nothing up
// to these lengths, and 1 to 6 % of all gradients beyond.)
constexpr int kLongestF32 = 64, kLongestBf16 = 512;

constexpr long kPieceBytesMost = 256L << 20;  // of dz, or of the planes of w

constexpr Shape kShapes[] = {{true, 256}, {true, 192}, {true, 128}, {false, 256}, {false, 192}, {false, 128}};
bool possible(Shape s, int planes) { return s.pair || planes == 1 || s.bn == 128; }
long tiles_of(long m, long n, Shape s) { const long rows = s.pair ? 2 * BM : BM; return up(m, rows) / rows * (up(n, s.bn) / s.bn); }
long workers_of(Shape s, int pairs) { return s.pair ? pairs : 2 * pairs; }
// What the plan goes by, in microseconds of a worker (measured): a K block of a tile (six products with three planes, and a single CTA loads half
// as much again as one of a pair), and a tile's epilogue, which hides behind the next tile's products if those take longer: with `stored` it is
// what a worker has of the memory's rate.
double tile_time(Shape s, long blocks, int planes, bool stored) {
  const double products = blocks * (0.27 + 0.0007 * s.bn) * (s.pair ? 1.0 : 1.05) * (planes == 3 ? 6 : 1);
  const double epilogue = stored ? (s.bn == BN ? 2.2 : 1.3) : 0.005 * s.bn;
  return products > epilogue ? products : epilogue;
}
constexpr double kMeeting = 0.7;  // what a pair's beginning and end take beyond a single CTA's
// What parts of a sum cost beyond the products: another kernel, and each value written and read.
double parts_time(double values, int parts) { return parts > 1 ? 2.5 + 8.0 * values * parts / 6e6 : 0; }

constexpr double kOtherSum = 4;  // and what they cost dw besides, whose parts are added up behind dx's

// z's tiles and into how many parts its sum is cut: what takes the least time.
void plan_logits(long m, long n, long blocks, int planes, int pairs, bool parts, Shape* shape, int* splits) {
  double least = -1;
  for (const Shape& b : kShapes) {
    if (!possible(b, planes)) continue;
    const long tiles = tiles_of(m, n, b), workers = workers_of(b, pairs);
    for (int s = 1; s == 1 || (parts && s * tiles <= workers && s <= blocks); ++s) {
      const long per = (blocks + s - 1) / s;
      if (s > 1 && per > chain_blocks(planes, kStatistics)) continue;
      const double t = (s * tiles + workers - 1) / workers * tile_time(b, per, planes, s > 1) + parts_time((double)m * n, s) + (b.pair ? kMeeting : 0);
      if (least < 0 || t < least) { least = t; *shape = b; *splits = (int)((blocks + per - 1) / per); }
    }
  }
}
// The same for dx [rows][in] over the classes of a piece and dw [classes][in] over the rows, which share a launch.  dw's sum is cut too where its tiles are
// few and many rows long (`parts`: may be), into a power of two parts of at least four K blocks each.  Measured (all gradients, bf16 and
// fp32; whole sums behind): 4037 rows of 35 values against 48 classes 23 and 31 us (36 and 96), 16384 of 256 against 257 56 and 106 us (89 and 342), 8192 of 1024
// against 1000 81 and 271 us (104 and 440); 4096 of 4096 against 10 53 and 179 us (50 and 206).
void plan_gradients(long rows, long in, long classes, int planes, int pairs, bool parts, Plan* p) {
  const long class_blocks = (classes + BK - 1) / BK, row_blocks = (rows + BK - 1) / BK;
  double least = -1;
  for (const Shape& b : kShapes)
    for (const Shape& c : kShapes) {
      if (b.pair != c.pair || b.bn == 192 || c.bn == 192 || !possible(b, planes) || !possible(c, planes)) continue;
      const long workers = workers_of(b, pairs), dx_tiles = tiles_of(rows, in, b), dw_tiles = tiles_of(classes, in, c);
      for (int t = 1; t == 1 || (parts && t <= 64 && 4 * t <= row_blocks && t * dw_tiles <= workers); t *= 2) {
        const double w = tile_time(c, (row_blocks + t - 1) / t, planes, true), w_sum = t > 1 ? kOtherSum + parts_time((double)classes * in, t) : 0;
        for (int s = 1; s <= 64 && s <= class_blocks && (s == 1 || s * dx_tiles <= workers); ++s) {
          const double x = tile_time(b, (class_blocks + s - 1) / s, planes, true);
          const double all = (s * dx_tiles * x + t * dw_tiles * w) / workers + (x < w ? x : w) / 2;
          const double longest = x > w ? x : w;
          const double time = (all > longest ? all : longest) + 0.1 * longest + parts_time((double)rows * in, s) + w_sum + (b.pair ? kMeeting : 0);  // (the shorter the longest, the evener the end)
          if (least < 0 || time < least) { least = time; p->dx_shape = b; p->dx_splits = s; p->dw_shape = c; p->dw_splits = t; }
        }
      }
    }
}

// in_pairs: for the self-test, whether z's tiles are pairs', or null.
Plan make_plan(const vgg19_linear_loss& a, bool backward, int pairs, const bool* in_pairs = nullptr) {
  Plan p{};
  const bool f32 = a.dtype == VGG19_FP32;
  size_t at = 0;
  auto take = [&at](size_t bytes) { const size_t o = at; at += (bytes + 255) / 256 * 256; return o; };
  if (!in_pairs && few_rows(a, backward)) {
    p.few = backward ? few_rows_ranges(a, 2 * pairs) : few_rows_blocks(a, 2 * pairs);
    p.dx_ld = up(a.in, 4);
    if (backward) {
      p.dz = take((size_t)a.classes * few_rows_up((int)a.rows) * 4);
      p.dx = take((size_t)p.few * a.rows * p.dx_ld * 4);
    } else {
      p.part = take((size_t)p.few * a.rows * sizeof(float2));
      p.label_z = take((size_t)a.rows * 4);
    }
    p.total = at < 256 ? 256 : at;
    return p;
  }
  p.planes = f32 ? 3 : 1;
  p.take_x = f32 || !copyable(a.x, a.rows, a.ldx, 2);
  p.take_w = f32 || !copyable(a.w, a.classes, a.ldw, 2);
  p.ld = up(a.in, 8);
  const long all = up(a.classes, BN);
  p.piece = all;
  auto most = [&](long bytes_a_class) {
    // at least 4096 classes, since dx is read and written again for every piece, unless those are over a gigabyte
    const long fit = kPieceBytesMost / bytes_a_class / BN * BN, few = (1L << 30) / bytes_a_class / BN * BN, least = few >= 4096 ? 4096 : few > BN ? few : BN;
    if (p.piece > (fit > least ? fit : least)) p.piece = fit > least ? fit : least;
  };
  if (p.take_w) most(2 * p.planes * p.ld);
  if (backward) most(2 * p.planes * a.rows);
  p.pieces = (int)((all + p.piece - 1) / p.piece);
  p.piece = up((all + p.pieces - 1) / p.pieces, BN);  // pieces of about one size
  p.pieces = (int)((all + p.piece - 1) / p.piece);
  if (p.take_x) p.x = take((size_t)p.planes * a.rows * p.ld * 2);
  if (p.take_w) p.w = take((size_t)p.planes * (p.piece < a.classes ? p.piece : a.classes) * p.ld * 2);
  const long blocks = (a.in + BK - 1) / BK, piece_classes = p.piece < a.classes ? p.piece : a.classes;
  plan_logits(a.rows, piece_classes, blocks, p.planes, pairs, p.pieces == 1, &p.z_shape, &p.z_splits);
  if (in_pairs) {
    p.z_shape = Shape{*in_pairs, 128};
    p.z_splits = 1;
  }
  if (p.z_splits > 1) p.z = take((size_t)p.z_splits * a.rows * up(a.classes, 4) * 4);
  p.db_rows = p.z_splits > 1 ? kPartRows : 32;
  if (!backward) {
    if (p.z_splits == 1) p.part = take((size_t)p.pieces * up(p.piece, p.z_shape.bn / 2) / (p.z_shape.bn / 2) * a.rows * sizeof(float2));
    if (p.z_splits == 1) p.label_z = take((size_t)a.rows * 4);
  } else {
    p.dz = take((size_t)p.planes * a.rows * p.piece * 2);
    p.db_part = take((size_t)(up(a.rows, p.db_rows) / p.db_rows) * p.piece * 4);
    plan_gradients(a.rows, a.in, piece_classes, p.planes, pairs, p.pieces == 1, &p);
    p.dx_parts = p.pieces > 1 || p.dx_splits > 1;
    p.dx_ld = up(a.in, 4);
    if (p.dx_parts) p.dx = take((size_t)p.dx_splits * a.rows * p.dx_ld * 4);
    if (p.dw_splits > 1) p.dw = take((size_t)p.dw_splits * a.classes * p.dx_ld * 4);
  }
  p.total = at < 256 ? 256 : at;
  return p;
}

template <int P, int EPI, bool PAIR> cudaError_t launch_tiles(const Launch& L, int pairs, cudaStream_t st) {
  const cudaError_t e = cudaFuncSetAttribute(loss_product_kernel<P, EPI, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
  if (e != cudaSuccess) return e;
  const int tiles = L.first_tile[L.count], workers = PAIR ? pairs : 2 * pairs;
  return launch_clusters(loss_product_kernel<P, EPI, PAIR>, PAIR ? 2 : 1, dim3((unsigned)((tiles < workers ? tiles : workers) * (PAIR ? 2 : 1))), kThreads, kSmemBytes, st, L);
}
template <int P, int EPI> cudaError_t launch_products(Launch& L, bool pair, int pairs, cudaStream_t st) {
  int tiles = 0;
  bool is_long = false;
  for (int i = 0; i < L.count; ++i) {
    Job& p = L.job[i];
    const int rows = pair ? kTileRows<true> : kTileRows<false>;
    p.tiles_m = (p.m + rows - 1) / rows;
    p.tiles_n = (p.n + p.bn - 1) / p.bn;
    if (p.splits < 1) p.splits = 1;
    if (!p.group) p.group = 16;
    p.per_split = (p.k_blocks + p.splits - 1) / p.splits;
    p.splits = (p.k_blocks + p.per_split - 1) / p.per_split;  // none is empty
    p.chain = chain_blocks(P, EPI);
    if (P == 1 && EPI == kProduct && p.per_split > p.longest) is_long = true;
    L.first_tile[i] = tiles;
    tiles += p.splits * p.tiles_m * p.tiles_n;
  }
  L.first_tile[L.count] = tiles;
  if constexpr (P == 1 && EPI == kProduct) {
    if (is_long) {
      for (int i = 0; i < L.count; ++i) L.job[i].chain = L.job[i].longest;
      return pair ? launch_tiles<P, kLongProduct, true>(L, pairs, st) : launch_tiles<P, kLongProduct, false>(L, pairs, st);
    }
  }
  return pair ? launch_tiles<P, EPI, true>(L, pairs, st) : launch_tiles<P, EPI, false>(L, pairs, st);
}

// The operands of one call in the form that the products read: x once, w piece by piece.
template <int P> struct Operands {
  const vgg19_linear_loss& a;
  const Plan& p;
  char* ws;
  cudaStream_t st;
  CUtensorMap x, w;

  // The maps of x (with the first piece) and of the piece of w; what copies cannot read where it lies is laid out first.
  cudaError_t prepare(long first, long n) {
    const long elt = P == 3 ? 4 : 2;
    const char* src = static_cast<const char*>(a.w) + first * a.ldw * elt;
    Layout l{};
    l.in = a.in; l.ld = p.ld;
    if (p.take_x && first == 0) {
      l.src[0] = a.x; l.src_ld[0] = a.ldx; l.rows[0] = a.rows;
      l.dst[0] = reinterpret_cast<bf16*>(ws + p.x);
    }
    if (p.take_w) {
      l.src[1] = src; l.src_ld[1] = a.ldw; l.rows[1] = n;
      l.dst[1] = reinterpret_cast<bf16*>(ws + p.w);
    }
    const long chunks = (l.rows[0] + l.rows[1]) * (p.ld / 8);
    if (chunks) {
      const unsigned blocks = (unsigned)(chunks / 256 + 1 < 148 * 16 ? chunks / 256 + 1 : 148 * 16);
      const cudaError_t e = P == 3 ? launch_behind(planes_kernel<float, 3>, blocks, 256, 0, st, l) : launch_behind(planes_kernel<bf16, 1>, blocks, 256, 0, st, l);
      if (e != cudaSuccess) return e;
    }
    const bool maps = (first > 0 || (p.take_x ? planes_map(&x, ws + p.x, false, P, a.rows, a.in, p.ld, 64) : planes_map(&x, a.x, false, 1, a.rows, a.in, a.rows == 1 ? p.ld : a.ldx, 64))) &&
                      (p.take_w ? planes_map(&w, ws + p.w, false, P, n, a.in, p.ld, 64) : planes_map(&w, src, false, 1, n, a.in, a.classes == 1 ? p.ld : a.ldw, 64));
    return maps ? cudaSuccess : cudaErrorInvalidValue;
  }
};

// The products z of one piece.
template <int P> Launch logits(const Operands<P>& o, const Plan& p, long first, long n, const Waits& waits) {
  Launch L{};
  L.waits = waits;
  L.count = 1;
  Job& j = L.job[0];
  j.a = o.x; j.b = o.w;
  j.m = (int)o.a.rows; j.n = (int)n; j.k_blocks = (o.a.in + BK - 1) / BK; j.bn = p.z_shape.bn;
  Rows& r = L.rows;
  r.bias = o.a.bias ? o.a.bias + first : nullptr;
  r.labels = o.a.labels;
  r.first_class = (int)first; r.classes = (int)n; r.all_classes = o.a.classes;
  return L;
}

cudaError_t join_parts(const vgg19_linear_loss& a, float* loss, float* lse, char* ws, const Plan& p, int parts, cudaStream_t st);

// z in parts of its sum.
template <int P> cudaError_t logits_in_parts(const Operands<P>& o, const Plan& p, int pairs, const Waits& waits, Parts& parts, cudaStream_t st) {
  Launch L = logits<P>(o, p, 0, o.a.classes, waits);
  Job& j = L.job[0];
  j.splits = p.z_splits;
  j.store = kPadded;
  j.out = o.ws + p.z; j.ld = up(o.a.classes, 4);
  parts = Parts{};
  parts.z = reinterpret_cast<const float*>(o.ws + p.z); parts.ld = j.ld;
  parts.parts = p.z_splits; parts.rows = (int)o.a.rows; parts.classes = o.a.classes;
  parts.bias = o.a.bias; parts.labels = o.a.labels;
  return launch_products<P, kSums>(L, p.z_shape.pair, pairs, st);
}

template <int P>
cudaError_t forward(const vgg19_linear_loss& a, float* loss, float* lse, char* ws, const Plan& p, int pairs, const Waits& waits, cudaStream_t st) {
  Operands<P> o{a, p, ws, st, {}, {}};
  cudaError_t e = cudaSuccess;
  if (p.z_splits > 1) {
    e = o.prepare(0, a.classes);
    Parts parts;
    if (e == cudaSuccess) e = logits_in_parts<P>(o, p, pairs, waits, parts, st);
    parts.loss = loss; parts.lse_out = lse;
    return e == cudaSuccess ? launch_behind(loss_of_parts_kernel, (unsigned)a.rows, kRowThreads, 0, st, parts) : e;
  }
  int part = 0;
  for (int i = 0; i < p.pieces && e == cudaSuccess; ++i) {
    const long first = i * p.piece, n = a.classes - first < p.piece ? a.classes - first : p.piece;
    e = o.prepare(first, n);
    if (e != cudaSuccess) break;
    Launch L = logits<P>(o, p, first, n, waits);
    L.rows.part = reinterpret_cast<float2*>(ws + p.part);
    L.rows.label_z = reinterpret_cast<float*>(ws + p.label_z);
    L.rows.first_part = part;
    part += (int)((n + p.z_shape.bn / 2 - 1) / (p.z_shape.bn / 2));
    e = launch_products<P, kStatistics>(L, p.z_shape.pair, pairs, st);
  }
  if (e != cudaSuccess) return e;
  return join_parts(a, loss, lse, ws, p, part, st);
}

cudaError_t join_parts(const vgg19_linear_loss& a, float* loss, float* lse, char* ws, const Plan& p, int parts, cudaStream_t st) {
  const Join j{reinterpret_cast<const float2*>(ws + p.part), reinterpret_cast<const float*>(ws + p.label_z), a.labels, loss, lse, parts, (int)a.rows, a.classes};
  return launch_behind(join_rows_kernel, (unsigned)((a.rows + kJoinRows - 1) / kJoinRows), kJoinRows * kJoinGroups, 0, st, j);
}
cudaError_t forward_few(const vgg19_linear_loss& a, float* loss, float* lse, char* ws, const Plan& p, int pairs, cudaStream_t st) {
  const cudaError_t e = few_rows_loss(a, reinterpret_cast<float2*>(ws + p.part), reinterpret_cast<float*>(ws + p.label_z), 2 * pairs, st);
  return e == cudaSuccess ? join_parts(a, loss, lse, ws, p, p.few, st) : e;
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

// dx or dw from the parts of its sum.
template <typename T>
cudaError_t sum_parts(const char* part, int parts, long rows, const vgg19_linear_loss& a, const Plan& p, void* out, long out_ld, cudaStream_t st) {
  const bool many = parts > 16;
  const long threads = rows * (p.dx_ld / 4) * (many ? 8 : 1), blocks = (threads + 255) / 256;
  return launch_behind(many ? sum_parts_kernel<T, 8> : sum_parts_kernel<T, 1>, (unsigned)(blocks < 148 * 16 ? blocks : 148 * 16), 256, 0, st,
                       reinterpret_cast<const float*>(part), parts, rows, (int)a.in, p.dx_ld, static_cast<T*>(out), out_ld);
}
cudaError_t sum_dx(const vgg19_linear_loss& a, const Gradients& g, char* ws, const Plan& p, int parts, cudaStream_t st) {
  return a.dtype == VGG19_FP32 ? sum_parts<float>(ws + p.dx, parts, a.rows, a, p, g.dx, g.dx_ld, st) : sum_parts<bf16>(ws + p.dx, parts, a.rows, a, p, g.dx, g.dx_ld, st);
}

template <int P>
cudaError_t backward(const vgg19_linear_loss& a, const Gradients& g, char* ws, const Plan& p, int pairs, const Waits& waits, cudaStream_t st) {
  Operands<P> o{a, p, ws, st, {}, {}};
  cudaError_t e = cudaSuccess;
  float* dx_part = reinterpret_cast<float*>(ws + p.dx);
  float* db_part = reinterpret_cast<float*>(ws + p.db_part);
  int slots = 0;
  for (int i = 0; i < p.pieces && e == cudaSuccess; ++i) {
    const long first = i * p.piece, n = a.classes - first < p.piece ? a.classes - first : p.piece;
    e = o.prepare(first, n);
    if (e != cudaSuccess) break;
    const long dz_ld = up(n, 8);
    CUtensorMap dz;
    if (!planes_map(&dz, ws + p.dz, false, P, a.rows, n, dz_ld, 64)) return cudaErrorInvalidValue;
    if (p.z_splits > 1) {
      Parts parts;
      e = logits_in_parts<P>(o, p, pairs, waits, parts, st);
      if (e != cudaSuccess) break;
      parts.lse = g.lse; parts.d_loss = g.d_loss;
      parts.dz = reinterpret_cast<bf16*>(ws + p.dz); parts.dz_ld = dz_ld;
      parts.db_part = g.db ? db_part : nullptr;
      e = launch_behind(gradient_of_parts_kernel<P>, dim3((unsigned)((n + 127) / 128), (unsigned)((a.rows + kPartRows - 1) / kPartRows)), 32 * kPartRows, 0, st, parts);
    } else {
      Launch L = logits<P>(o, p, first, n, waits);
      L.job[0].out = ws + p.dz; L.job[0].ld = dz_ld;
      L.rows.lse = g.lse; L.rows.d_loss = g.d_loss;
      L.rows.db_part = g.db ? db_part : nullptr;
      e = launch_products<P, kLogitGradient>(L, p.z_shape.pair, pairs, st);
    }
    if (e != cudaSuccess) break;

    Launch M{};
    M.waits = waits;
    const bool f32 = P == 3;
    bool with_db = false;  // whether dw's tiles add up db on the way
    if (g.dx) {  // dx, or the piece's share of it: [rows][in] = dz w.  Its tiles, over all classes, take longer than dw's: they come first
      Job& j = M.job[M.count++];
      j.a = dz; j.b = o.w; j.b_mn = 1;
      j.longest = kLongestBf16;
      j.m = (int)a.rows; j.n = a.in; j.k_blocks = (int)((n + BK - 1) / BK); j.bn = p.dx_shape.bn;
      if (p.dx_parts) {
        j.f32 = 1;
        j.out = dx_part; j.ld = p.dx_ld;
        j.splits = slots && slots < p.dx_splits ? slots : p.dx_splits;  // later pieces add to the parts that the first one wrote
        j.store = i ? kAdded : kWhole;  // (rows have room for whole fours)
        if (!i) {
          const int per = (j.k_blocks + j.splits - 1) / j.splits;
          slots = (j.k_blocks + per - 1) / per;
        }
      } else {
        j.f32 = f32;
        j.out = g.dx; j.ld = g.dx_ld;
        j.store = copyable(g.dx, a.rows, g.dx_ld, f32 ? 4 : 2) ? kWhole : kSingle;
      }
    }
    if (g.dw) {  // dw of the piece: [n][in] = dz^T x
      Job& j = M.job[M.count++];
      j.a = dz; j.a_mn = 1; j.b = o.x; j.b_mn = 1;
      j.longest = g.dw_f32 ? kLongestF32 : kLongestBf16;
      j.group = 4;  // whole rows of dw at a time (sixteen: 2 % slower)
      j.m = (int)n; j.n = a.in; j.k_blocks = (int)((a.rows + BK - 1) / BK); j.bn = p.dw_shape.bn;
      if (p.dw_splits > 1) {
        j.splits = p.dw_splits;
        j.f32 = 1;
        j.out = ws + p.dw; j.ld = p.dx_ld;
        j.store = kWhole;
      } else {
        j.f32 = f32 || g.dw_f32;
        const long elt = j.f32 ? 4 : 2;
        j.out = static_cast<char*>(g.dw) + first * g.dw_ld * elt; j.ld = g.dw_ld;
        j.store = copyable(j.out, n, g.dw_ld, elt) ? kWhole : kSingle;
      }
      // (A sum in chains wants its epilogue all along, which then does not add up db besides: 300000 rows of 1000 against 4000, dw in fp32,
      // 11.6 ms, 13.4 if it does.)
      const int dw_splits = p.dw_splits > 1 ? p.dw_splits : 1;
      with_db = P == 3 || (j.k_blocks + dw_splits - 1) / dw_splits <= j.longest;
      j.db_part = db_part; j.db = g.db && with_db ? g.db + first : nullptr;
      j.parts = (int)((a.rows + p.db_rows - 1) / p.db_rows);
    }
    if (M.count) e = launch_products<P, kProduct>(M, p.dx_shape.pair, pairs, st);
    if (!with_db && g.db && e == cudaSuccess)
      e = launch_behind(sum_columns_kernel, (unsigned)((n + 31) / 32), 256, 0, st, static_cast<const float*>(db_part), (int)((a.rows + p.db_rows - 1) / p.db_rows), (int)n, g.db + first);
  }
  if (e == cudaSuccess && g.dx && p.dx_parts) e = sum_dx(a, g, ws, p, slots, st);
  if (e == cudaSuccess && g.dw && p.dw_splits > 1) {
    const int blocks = (int)((a.rows + BK - 1) / BK), per = (blocks + p.dw_splits - 1) / p.dw_splits, parts = (blocks + per - 1) / per;
    e = P == 3 || g.dw_f32 ? sum_parts<float>(ws + p.dw, parts, a.classes, a, p, g.dw, g.dw_ld, st) : sum_parts<bf16>(ws + p.dw, parts, a.classes, a, p, g.dw, g.dw_ld, st);
  }
  return e;
}

cudaError_t backward_few(const vgg19_linear_loss& a, const Gradients& g, char* ws, const Plan& p, int pairs, cudaStream_t st) {
  const FewGradients f{g.lse, g.d_loss, reinterpret_cast<float*>(ws + p.dz), g.dx ? reinterpret_cast<float*>(ws + p.dx) : nullptr, p.dx_ld,
                       static_cast<float*>(g.dw), g.dw_ld, g.db};
  const cudaError_t e = few_rows_gradients(a, f, 2 * pairs, st);
  return e == cudaSuccess && g.dx ? sum_dx(a, g, ws, p, p.few, st) : e;
}

int check(const vgg19_linear_loss* a) {
  if (!a) return note_error(VGG19_ERR_ARG, "no description of the layer");
  if (a->dtype != VGG19_FP32 && a->dtype != VGG19_BF16)
    return note_error(VGG19_ERR_ARG, "dtype %d is neither VGG19_FP32 nor VGG19_BF16", a->dtype);
  if (a->rows < 0 || a->rows > (1 << 22) || a->in < 1 || a->in > (1 << 20) || a->classes < 1 || a->classes > (1 << 24))
    return note_error(VGG19_ERR_SHAPE, "%lld rows of %d values, %d classes: rows in [0, 2^22], values in [1, 2^20], classes in [1, 2^24]",
                      (long long)a->rows, a->in, a->classes);
  if (a->rows * a->classes > (1LL << 44)) return note_error(VGG19_ERR_SHAPE, "%lld rows against %d classes: at most 2^44 logits", (long long)a->rows, a->classes);
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

cudaError_t loss_error_words(ErrorWords* words) {
  const cudaError_t e = cudaGetSymbolAddress(reinterpret_cast<void**>(&words->at[kErrorLoss]), g_loss_error);
  return e == cudaSuccess ? cudaGetSymbolAddress(reinterpret_cast<void**>(&words->at[kErrorLabel]), g_label_error) : e;
}

int linear_loss(const vgg19_linear_loss* layer, float* loss, float* lse, void* workspace, size_t bytes, const Waits& waits, const bool* in_pairs, void* stream) {
  const int rc = check(layer);
  if (rc != VGG19_OK || layer->rows == 0) return rc;
  const vgg19_linear_loss& a = *layer;
  const int bad = check_pointers(a, workspace);
  if (bad != VGG19_OK) return bad;
  if (!words(a.bias, a.labels, loss, lse)) return note_error(VGG19_ERR_ARG, "bias, labels, loss or lse is not aligned to 4 bytes");
  const int pairs = pairs_of_device();
  const Plan p = make_plan(a, false, pairs, in_pairs);
  if (bytes < p.total) return note_error(VGG19_ERR_WORKSPACE, "workspace has %zu bytes, this call needs %zu", bytes, p.total);
  const long elt = a.dtype == VGG19_FP32 ? 4 : 2, each = 4L * a.rows;
  const Block all[] = {{loss, 1, each, 0}, {lse, 1, each, 0}, {workspace, 1, (long)p.total, 0}, {a.labels, 1, each, 0}, {a.bias, 1, 4L * a.classes, 0},
                       {a.x, a.rows, a.in * elt, a.ldx * elt}, {a.w, a.classes, a.in * elt, a.ldw * elt}};
  if (blocks_meet(all, 3)) return note_error(VGG19_ERR_ARG, "an output or the workspace overlaps an input or another output");
  if (!loss && !lse) return VGG19_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  const cudaError_t e = p.few ? forward_few(a, loss, lse, ws, p, pairs, st) : p.planes == 3 ? forward<3>(a, loss, lse, ws, p, pairs, waits, st) : forward<1>(a, loss, lse, ws, p, pairs, waits, st);
  return e == cudaSuccess ? VGG19_OK : note_error(VGG19_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}

}  // namespace vgg

extern "C" size_t vgg19_linear_cross_entropy_bytes(const vgg19_linear_loss* layer, int32_t backward) {
  using namespace vgg;
  if (check(layer) != VGG19_OK) return 0;
  if (layer->rows == 0) return 256;  // (nothing is cut up, and nothing used)
  // (a step has one workspace for both calls; the loss of many classes, whose gradients come in pieces, takes more than those)
  const int pairs = pairs_of_device();
  const size_t loss = make_plan(*layer, false, pairs).total;
  if (!backward) return loss;
  const size_t gradients = make_plan(*layer, true, pairs).total;
  return gradients > loss ? gradients : loss;
}

extern "C" int vgg19_linear_cross_entropy(const vgg19_linear_loss* layer, float* loss, float* lse, void* workspace, size_t bytes, void* stream) {
  return vgg::linear_loss(layer, loss, lse, workspace, bytes, vgg::Waits{}, nullptr, stream);
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
  const cudaError_t e = p.few ? backward_few(a, g, ws, p, pairs, st) : p.planes == 3 ? backward<3>(a, g, ws, p, pairs, waits, st) : backward<1>(a, g, ws, p, pairs, waits, st);
  return e == cudaSuccess ? VGG19_OK : note_error(VGG19_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}
