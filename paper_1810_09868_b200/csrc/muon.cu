// The orthogonalised update of weight matrices:
//   M <- mu M + G,   U = G + mu M (Nesterov) or M,   X_0 = U / |U|_F   (transposed where U has more rows than columns)
//   X <- p(X X^T) X,  p(A) = a I + b A + c A^2,       `steps` times (Newton-Schulz towards the orthogonal factor of U)
//   W <- (1 - lr decay) W - lr sqrt(max(1, rows / cols)) X.
//
// Every p(A_k) is a polynomial of A_0 = X_0 X_0^T, so the products commute and the iteration can run on m x m symmetric
// matrices: Q <- p(A) Q, A <- p(A) A p(A), and X = Q X_0 once at the end.  With r = n / m columns per row a step then
// costs four symmetric products (half a product each) instead of 3 r + 1.  A alone forgets singular values below the square
// root of its precision, which the iteration amplifies up to 3.4 times a step: so after every two steps, at first three, X is formed
// and A taken from it anew (five steps: 6 r + 14 such halves against 15 r + 5).  Measured against 64 bits, five steps: 4e-6 to 7e-6
// relative on gradients of low rank with noise, where plain fp32 products give 6e-6 to 3.9e-5 (without the restart 3e-5 to 1.8e-4),
// and 4e-6 to 7e-6 on Gaussian ones, where plain fp32 gives 1.6e-6 (70 x 200) to 4.8e-6 (4096 x 4096): there 22 bits are fewer than 24.
// Ten steps: 9e-6 to 1.9e-5 on Gaussian matrices, fp32 2.5e-6 to 1.3e-5.  The iteration does not settle: a singular value near 0.868 has its error multiplied
// by 1.6 a step, in any arithmetic.
//
// Precision.  A matrix is kept as two fp16 planes hi + lo of its values times a power of two (22 bits; the scales below
// keep every entry inside fp16's range), a product is hi hi + hi lo + lo hi in fp32, on tcgen05.  The tensor core's fp32
// accumulation truncates (about half a unit of the sum so far per instruction), so a chain ends after one to four stages
// of 64 and the epilogue warps add the chains in registers.
//
// Identities stay out of the products: with p(A) = a I + R and Q = q0 I + S the epilogues add a and q0 times their matrix in
// fp32, and what the tensor core truncates is relative to the smaller rest (9e-6 -> 5e-6).
//
// The product kernel: CTA pairs (cta_group::2), 256 x 256 tiles, persistent.  A stage holds hi and lo of both operands
// (64 KB per CTA) and feeds three products, so what a CTA loads per product is two thirds of what one pair of
// planes at a time would take; the plain pair kernels of this library are bound by exactly that rate.  All tensors of a call and
// all products that do not depend on one another share a launch.  Symmetric results are computed on and above the
// diagonal and stored twice.  The last product's epilogue updates the weights: X itself is never stored.
//
// Measured (B200, five steps): the dense layers of a 224 x 224 network (4096 x 25088, 4096 x 4096, 1000 x 4096) in 12.8 ms, of which
// 0.43 ms momentum, norm and X_0 at 6.9 TB/s; 14.7 TFLOP of fp16 products at 1.19 PFLOP/s, 0.86 of the measured sustained rate
// under the power cap that bounds them (the tensor pipe of a 4096 x 8192 Gram product is active 79 % of the time, at 1.58 GHz).  The sixteen filters in 0.66 ms: launches of 15 to 25 us, each a chain of latencies (3 us
// from one launch to the next, 5 us for the addends beside the stages on an SM's 64 bytes a cycle from L2, 0.8 us a stage, 4 us of stores).
#include <cuda_fp16.h>

#include <algorithm>
#include <vector>

#include "../../include/vgg19_b200.h"
#include "tc_common.cuh"

namespace vgg {
namespace {

using namespace tc;

static __device__ int g_muon_error[2];  // a DeviceError code once a bounded wait of a call without a handle ran out

// ---- sizes -----------------------------------------------------------------------------------------------------
constexpr int BM = 128, BK = 64;                 // rows per CTA (a pair has 256), K per stage
constexpr int kPlaneBytes = 128 * BK * 2;        // 128 rows (or K-rows) of one plane in a stage
constexpr int kOperandBytes = 2 * kPlaneBytes;   // hi and lo
// Columns per pair: 256, or 128 where that still leaves pairs idle: then a tile's loads, products, addends and stores are
// what a launch takes, and half of each is 10 us where a whole is 16.
template <int BN> constexpr int kOtherBytes = BN * BK * 2;  // hi and lo of a CTA's half of the columns
template <int BN> constexpr int kStageBytes = kOperandBytes + kOtherBytes<BN>;
template <int BN> constexpr int kStages = BN == 256 ? 3 : 4;
constexpr int kRingBytes = 3 * kStageBytes<256>;
static_assert(kRingBytes == 4 * kStageBytes<128>, "the same shared memory");

// Stages (12 MMAs each) of an accumulation chain.  The error of a chain grows with its length, the hand-over of a chain to
// the epilogue warps costs the tensor cores a few hundred cycles.  At 2048 and 4096 rows a chain of 4 is within 1.7 times
// plain fp32 (which itself sums longer there) and 8 % faster than single stages; below, single stages are what it takes.
// The last product, whose epilogue is the longest and whose error nothing amplifies, takes two.
template <bool FINAL> __device__ __forceinline__ int chain_stages(int k_stages) { return k_stages >= 32 ? 4 : FINAL ? 2 : 1; }
constexpr int kThreads = 384;                    // a warpgroup for producer and issuer, two of epilogue warps
// Registers per thread after the split: 168 at launch, 3 x 168 = 40 + 2 x 232.
constexpr int kFewRegisters = 40, kManyRegisters = 232;
constexpr int kPieceBytes = 4096;                // an epilogue warp's own 32 rows of 128 bytes
constexpr int kSmemBytes = kRingBytes + 8 * kPieceBytes + 1024 + 256;
constexpr int kMaxTensors = 20, kMaxProblems = 2 * kMaxTensors;

// The quintic's coefficients, and the scales of what is stored.  |X| <= 1.21 after any step, so |A| <= 1.47 and (by the
// polynomial's range on [0, 1.47]) |p| <= 3.45, |p A| <= 1.3, and Q of two and three steps is below 11.9 and 41.
constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kScaleX = 4096.f, kScaleA = 16384.f, kScaleP = 8192.f, kScaleQ2 = 4096.f, kScaleQ3 = 1024.f;
// Steps between two Gram matrices: two, and three at first where their number is odd.  At first the singular values are small and Q is close to
// its q0 I; later they are around one, Q = q0 I + S is too, and S is what cancels q0 = a^k: 12 after two steps, 41 after three, and that many
// times the rounding.  (Eight steps of Gaussian matrices as 3 + 3 + 2: 3e-5 to 1.1e-4 from 64 bits, plain fp32 products 2e-6 to 1e-5.)
__host__ __device__ constexpr int steps_of_group(int done, int steps) { return steps == 1 ? 1 : done == 0 && steps % 2 ? 3 : 2; }
// R = b A + c A A from A: the product's factor and the addend's, as Problem has them; the scale of S after step k.
__host__ __device__ constexpr float poly_alpha() { return kC * kScaleP / (kScaleA * kScaleA); }
__host__ __device__ constexpr float poly_c1() { return kB * kScaleP / kScaleA / poly_alpha(); }
__host__ __device__ constexpr float rest_scale(int k) { return k == 0 ? kScaleP : k == 1 ? kScaleQ2 : kScaleQ3; }

// What a kernel did before this overlapped the launch before it in the stream; what follows reads that one's results.  (Its
// own successor may be set up from here on.)
__device__ __forceinline__ void behind_previous() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Once per block, of a wait that ran out.
__device__ __noinline__ void report(const Waits& waits, int code) { atomicCAS(waits.error ? waits.error : g_muon_error, 0, code); }

// ---- one product ---------------------------------------------------------------------------------------------
// D[i][j] = alpha * (c1 add1[i][j] + c2 add2[i][j] + sum_k A[i][k] B[j][k]) (or B[k][j]: b_mn), m x n.
struct __align__(64) Problem {
  CUtensorMap a, b;
  int m, n, k_stages, tiles_m, tiles_n;
  int sym;         // tiles on and above the diagonal only; what lies above it is stored twice (or mirrored by gram_finish_kernel)
  int square;      // for the host: 1 always so, 2 so with square tiles, else all tiles
  int splits, per_split;  // K is cut into that many parts, of that many stages
  int b_mn;
  float alpha;
  // result as planes [2][m][ld], or ...
  half16* out;
  long plane, ld;
  // the sums starting from c1 * (hi + lo of add1) + c2 * (hi + lo of add2), planes of the same strides, where not null;
  const half16 *add1, *add2;
  float c1, c2;
  // ... or, with K cut, the bare sums in fp32, [splits][m][ld], for gram_finish_kernel;
  float* partial;
  // ... or the update of w (and its bf16 copy): w <- keep * w + that, at [i][j], or at [j][i] where transposed
  float* w;
  bf16* w16;
  long w_ld;
  int transposed, w_vec;
  float keep;
};
template <int N> struct Launch {
  Waits waits;
  int count;
  int first_tile[N + 1];  // apart from the problems: finding a tile's problem touches two lines of constant memory
  Problem p[N];
};

struct Tile {
  int i, j, split, k0, k1;  // in tiles; the part of K and its stages
};
// Of a symmetric result, the tiles that reach the diagonal or lie above it: in row i of tiles those from column (256 / BN) i on.
// (Halves there too: 1500 x 1500 689 -> 541 us.)
template <int BN> __device__ __forceinline__ Tile find_tile(const Problem& p, int t) {
  constexpr int WIDE = 2 * BM / BN;  // tiles of columns to a tile of rows
  Tile r{};
  if (p.splits > 1) { r.split = t % p.splits; t /= p.splits; }
  if (p.sym) {
    int left = p.tiles_n;
    while (t >= left) { t -= left; left -= WIDE; ++r.i; }
    r.j = WIDE * r.i + t;
  } else {
    r.j = t / p.tiles_m;  // row tiles fastest: they share the wide operand's columns
    r.i = t - r.j * p.tiles_m;
  }
  r.k0 = r.split * p.per_split;
  r.k1 = min(r.k0 + p.per_split, p.k_stages);
  return r;
}

__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_half2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }

// v as fp16 terms hi + lo
__device__ __forceinline__ void split8(const float (&v)[8], uint32_t (&hi)[4], uint32_t (&lo)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    hi[e] = pack_half2(v[2 * e], v[2 * e + 1]);
    const float2 f = unpack_half2(hi[e]);
    lo[e] = pack_half2(v[2 * e] - f.x, v[2 * e + 1] - f.y);
  }
}

// An epilogue thread holds a row of the tile; in memory a row is contiguous.  So tiles pass through 4 KB of shared memory
// per warp, 32 rows of 128 bytes with their 16-byte chunks swizzled, and every access to global memory covers four whole
// 128-byte lines (one thread per row took 3 to 4 us per tile and matrix, eight sectors where one would do).
__device__ __forceinline__ int piece_at(int row, int chunk) { return row * 8 + (chunk ^ (row & 7)); }

// sum (+)= c (hi + lo) of CW columns of planes; m points at the warp's first row and column.  What this costs is the latency
// of its requests: while the sums are still to be set (FIRST) there are registers for both planes of 64 columns at once.
template <bool FIRST, int CW>
__device__ __forceinline__ void add_planes(float (&sum)[CW], const half16* m, long plane, int ld, int rows, int cols, float c, uint4* piece, int lane) {
  const int r0 = lane / 8, k0 = lane % 8;
  m += (long)r0 * ld + k0 * 8;
  auto request = [&](uint4 (&v)[8], int h, int c0) {
    const half16* at = m + h * plane + c0;
#pragma unroll
    for (int q = 0; q < 8; ++q, at += 4 * ld)
      v[q] = q * 4 + r0 < rows && c0 + k0 * 8 < cols ? *reinterpret_cast<const uint4*>(at) : make_uint4(0, 0, 0, 0);
  };
  auto add = [&](const uint4 (&v)[8], int h, int c0) {
#pragma unroll
    for (int q = 0; q < 8; ++q) piece[piece_at(q * 4 + r0, k0)] = v[q];
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint4 x = piece[piece_at(lane, k)];
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = unpack_half2(w[e]);
        float &s0 = sum[c0 + 8 * k + 2 * e], &s1 = sum[c0 + 8 * k + 2 * e + 1];
        s0 = fmaf(c, f.x, FIRST && h == 0 ? 0.f : s0);
        s1 = fmaf(c, f.y, FIRST && h == 0 ? 0.f : s1);
      }
    }
    __syncwarp();
  };
#pragma unroll
  for (int c0 = 0; c0 < CW; c0 += 64) {
    uint4 hi[8];
    request(hi, 0, c0);
    if (FIRST) {
      uint4 lo[8];
      request(lo, 1, c0);
      add(hi, 0, c0);
      add(lo, 1, c0);
    } else {
      add(hi, 0, c0);
      request(hi, 1, c0);
      add(hi, 1, c0);
    }
  }
}
__device__ __forceinline__ void put(float* w, bf16* w16, long at, float v) {
  w[at] = v;
  if (w16) w16[at] = __float2bfloat16_rn(v);
}

// FINAL: every problem updates its w; else none does.
template <int N, bool FINAL, int BN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
split_product_pair_kernel(const __grid_constant__ Launch<N> L) {
  constexpr int STAGES = kStages<BN>, STAGE_BYTES = kStageBytes<BN>, CW = BN / 2;  // CW: columns of an epilogue group, a thread's sums
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t pieces = smem_base + kRingBytes, bars = pieces + 8 * kPieceBytes;
  auto full_bar = [&](int s) { return bars + 8u * s; };                   // used in the even CTA
  auto empty_bar = [&](int s) { return bars + 8u * (STAGES + s); };      // both CTAs
  auto acc_full_bar = [&](int b) { return bars + 8u * (2 * STAGES + b); };       // both CTAs
  auto acc_empty_bar = [&](int b) { return bars + 8u * (2 * STAGES + 2 + b); };  // used in the even CTA
  const uint32_t drain_bar = bars + 8u * (2 * STAGES + 4);
  __shared__ uint32_t tmem_base_slot;
  __shared__ int abort_flag, ran_out;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1, total = L.first_tile[L.count];

  if (threadIdx.x == 0) {
    abort_flag = ran_out = 0;
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), L.waits.signals); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(acc_full_bar(b), 1); mbar_init(acc_empty_bar(b), 16); }  // the epilogue warps of both CTAs
    mbar_init(drain_bar, 1);
    mbar_fence_init();
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(&tmem_base_slot), 2 * BN);
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
      int stage = 0, pi = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int w = pair; w < total && ok; w += n_pairs) {
        while (w >= L.first_tile[pi + 1]) ++pi;
        const Problem& p = L.p[pi];
        const Tile tile = find_tile<BN>(p, w - L.first_tile[pi]);
        const int row = (2 * tile.i + (int)rank) * BM, col = tile.j * BN + (int)rank * (BN / 2), mn = p.b_mn;
        for (int kb = tile.k0; kb < tile.k1; ++kb) {
          if (!mbar_wait(empty_bar(stage), phase ^ 1, &abort_flag, &ran_out, kDevTimeoutStageFree, L.waits.limit_cycles)) { ok = false; break; }
          const uint32_t sa = smem_base + stage * STAGE_BYTES, sb = sa + kOperandBytes;
          const uint32_t full = map_to_cta(full_bar(stage), 0);
          // the even CTA announces the bytes of both CTAs' copies; what lies outside a matrix arrives as zeros
          if (leader) mbar_expect_tx(full_bar(stage), 2 * STAGE_BYTES);
          tma_load_3d_pair(sa, &p.a, full, kb * BK, row, 0);
          if (mn) {
            tma_load_3d_pair(sb, &p.b, full, col, kb * BK, 0);
            if (BN == 256) tma_load_3d_pair(sb + kPlaneBytes, &p.b, full, col + 64, kb * BK, 0);
          } else {
            tma_load_3d_pair(sb, &p.b, full, kb * BK, col, 0);
          }
#pragma unroll
          for (int s = 0; s < STAGES; ++s) fills[s] += s == stage;
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
      }
      if (!ok) {
        // let every copy in flight land before the CTA may exit (see the pair convolution)
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
      int stage = 0, pi = 0;
      uint32_t phase = 0, chunk = 0;
      bool ok = true;
      for (int w = pair; w < total && ok; w += n_pairs) {
        while (w >= L.first_tile[pi + 1]) ++pi;
        const Problem& p = L.p[pi];
        const bool mn = p.b_mn != 0;
        const Tile tile = find_tile<BN>(p, w - L.first_tile[pi]);
        const int k_stages = tile.k1 - tile.k0, chain = chain_stages<FINAL>(k_stages);
        const uint32_t idesc = umma_idesc_f16(2 * BM, BN, 0, mn);
        // K-major: lo behind all rows of hi, 16 k = 32 bytes of the swizzled row.  MN-major: two groups of 64 columns, each
        // 64 k-rows of hi then of lo; 16 k = 16 rows.
        const uint32_t b_lo = mn ? kPlaneBytes / 2 : kOtherBytes<BN> / 2, b_step = mn ? 2048 : 32, b_lbo = mn ? kPlaneBytes : 16;
        for (int kb0 = 0, kb1; kb0 < k_stages && ok; kb0 = kb1, ++chunk) {
          kb1 = min(kb0 + chain, k_stages);
          const int buf = chunk & 1;
          if (!mbar_wait(acc_empty_bar(buf), ((chunk >> 1) & 1) ^ 1, &abort_flag, &ran_out, kDevTimeoutTmemFree, L.waits.limit_cycles)) { ok = false; break; }
          tc_fence_after();
          const uint32_t d = tmem_base + (uint32_t)(buf * BN);
          for (int kb = kb0; kb < kb1; ++kb) {
            if (!mbar_wait(full_bar(stage), phase, &abort_flag, &ran_out, kDevTimeoutTmaFull, L.waits.limit_cycles)) { ok = false; break; }
            tc_fence_after();
            const uint32_t sa = smem_base + stage * STAGE_BYTES, sb = sa + kOperandBytes;
            const uint64_t ah = smem_desc_sw128(sa, 16), al = smem_desc_sw128(sa + kPlaneBytes, 16);
            const uint64_t bh = smem_desc_sw128(sb, b_lbo), bl = smem_desc_sw128(sb + b_lo, b_lbo);
            // the small products first: what the tensor core truncates is relative to the sum so far
            umma_bf16_pair(d, al, bh, idesc, kb != kb0 ? 1u : 0u);
            umma_bf16_pair_acc(d, ah, bl, idesc);
#pragma unroll
            for (int k = 1; k < BK / 16; ++k) {
              umma_bf16_pair_acc(d, desc_advance(al, k * 32), desc_advance(bh, k * b_step), idesc);
              umma_bf16_pair_acc(d, desc_advance(ah, k * 32), desc_advance(bl, k * b_step), idesc);
            }
#pragma unroll
            for (int k = 0; k < BK / 16; ++k)
              umma_bf16_pair_acc(d, desc_advance(ah, k * 32), desc_advance(bh, k * b_step), idesc);
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
    uint4* piece = reinterpret_cast<uint4*>(smem_raw + (pieces - smem_u32(smem_raw)) + (warp - 4) * kPieceBytes);
    int pi = 0;
    uint32_t chunk = 0;
    bool ok = true;
    for (int w = pair; w < total && ok; w += n_pairs) {
      while (w >= L.first_tile[pi + 1]) ++pi;
      const Problem& p = L.p[pi];
      const Tile tile = find_tile<BN>(p, w - L.first_tile[pi]);
      const int i0 = (2 * tile.i + (int)rank) * BM + quarter * 32, j0 = tile.j * BN + group * CW;  // the warp's first row and column
      const int rows = p.m - i0, cols = p.n - j0;                                           // what there is from there on
      const int k_stages = tile.k1 - tile.k0, chain = chain_stages<FINAL>(k_stages);
      // the sums start from what is added to the product: its loads pass while the first chain runs
      float sum[CW];
      if (FINAL && rows > 0) {  // the weights of the warp's rows come from far: have them nearer by the time they are updated
#pragma unroll
        for (int c = 0; c < CW; c += 32) {
          if (p.transposed) {  // a row of w per column, 32 elements of each
            if (c + lane < cols) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.w + (j0 + c + lane) * p.w_ld + i0));
          } else if (p.w_vec && lane < rows && c < cols) {
            asm volatile("prefetch.global.L2 [%0];" ::"l"(p.w + (i0 + lane) * p.w_ld + j0 + c));
          }
        }
      }
      if (p.add1 && rows > 0 && cols > 0) {
        add_planes<true, CW>(sum, p.add1 + i0 * p.ld + j0, p.plane, (int)p.ld, rows, cols, p.c1, piece, lane);
        if (!FINAL && p.add2) add_planes<false, CW>(sum, p.add2 + i0 * p.ld + j0, p.plane, (int)p.ld, rows, cols, p.c2, piece, lane);
      } else {
#pragma unroll
        for (int j = 0; j < CW; ++j) sum[j] = 0.f;
      }
      for (int kb0 = 0; kb0 < k_stages; kb0 += chain, ++chunk) {
        const int buf = chunk & 1;
        if (!__all_sync(0xffffffffu, mbar_wait(acc_full_bar(buf), (chunk >> 1) & 1, &abort_flag, &ran_out, kDevTimeoutAccum, L.waits.limit_cycles))) { ok = false; break; }
        tc_fence_after();
        const uint32_t src = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * BN + group * CW);
#pragma unroll
        for (int c = 0; c < CW; c += 32) {
          uint32_t v[32];
          tmem_ld_32x32(src + c, v);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 32; ++j) sum[c + j] += __uint_as_float(v[j]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(map_to_cta(acc_empty_bar(buf), 0));
      }
      if (!ok) break;

      if (rows <= 0 || cols <= 0) continue;
      const float alpha = p.alpha;
      const long ld = p.ld;
      const int r0 = lane / 8, k0 = lane % 8;  // what this lane moves between memory and a piece: rows r0, r0 + 4, ..., chunk k0
      if (!FINAL && p.partial) {
        float* out = p.partial + ((long)tile.split * p.m + i0) * ld + j0;
#pragma unroll
        for (int c0 = 0; c0 < CW; c0 += 32) {
          if (c0 >= cols) break;
#pragma unroll
          for (int k = 0; k < 8; ++k)
            piece[piece_at(lane, k)] = make_uint4(__float_as_uint(sum[c0 + 4 * k]), __float_as_uint(sum[c0 + 4 * k + 1]),
                                                  __float_as_uint(sum[c0 + 4 * k + 2]), __float_as_uint(sum[c0 + 4 * k + 3]));
          __syncwarp();
#pragma unroll
          for (int q = 0; q < 8; ++q)  // (a row has room for whole eights)
            if (q * 4 + r0 < rows && c0 + k0 * 4 < cols)
              *reinterpret_cast<uint4*>(out + (q * 4 + r0) * ld + c0 + k0 * 4) = piece[piece_at(q * 4 + r0, k0)];
          __syncwarp();
        }
      } else if (!FINAL) {
        half16* out = p.out + i0 * ld + j0;
#pragma unroll
        for (int c0 = 0; c0 < CW; c0 += 64) {
          if (c0 >= cols) break;
          uint32_t hi[8][4], lo[8][4];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = alpha * sum[c0 + 8 * k + e];
            split8(v, hi[k], lo[k]);
          }
          if (p.sym && tile.j / (2 * BM / BN) != tile.i && lane < rows) {  // the mirror image, lanes along a row
            half16* at = p.out + (j0 + c0) * ld + i0 + lane;
#pragma unroll
            for (int j = 0; j < 64; ++j)
              if (c0 + j < cols) {
                at[j * ld] = (half16)(hi[j / 8][j % 8 / 2] >> (16 * (j & 1)));
                at[p.plane + j * ld] = (half16)(lo[j / 8][j % 8 / 2] >> (16 * (j & 1)));
              }
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
              piece[piece_at(lane, k)] = h ? make_uint4(lo[k][0], lo[k][1], lo[k][2], lo[k][3]) : make_uint4(hi[k][0], hi[k][1], hi[k][2], hi[k][3]);
            __syncwarp();
#pragma unroll
            for (int q = 0; q < 8; ++q)
              if (q * 4 + r0 < rows && c0 + k0 * 8 < cols)
                *reinterpret_cast<uint4*>(out + h * p.plane + (q * 4 + r0) * ld + c0 + k0 * 8) = piece[piece_at(q * 4 + r0, k0)];
            __syncwarp();
          }
        }
      } else if (p.transposed) {  // lanes along a row of w
        if (lane < rows) {
          const long at = j0 * p.w_ld + i0 + lane, w_ld = p.w_ld;
          const float keep = p.keep;
#pragma unroll
          for (int c0 = 0; c0 < CW; c0 += 16) {
            float old[16];
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (c0 + j < cols) old[j] = p.w[at + (c0 + j) * w_ld];
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (c0 + j < cols) put(p.w, p.w16, at + (c0 + j) * w_ld, fmaf(keep, old[j], alpha * sum[c0 + j]));
          }
        }
      } else {
        const float keep = p.keep;
        const long w_ld = p.w_ld;
        float* w = p.w + i0 * w_ld + j0;
        bf16* w16 = p.w16 ? p.w16 + i0 * w_ld + j0 : nullptr;
#pragma unroll
        for (int c0 = 0; c0 < CW; c0 += 32) {
          if (c0 >= cols) break;
          {
            float4 old[8];
            if (p.w_vec) {
#pragma unroll
              for (int q = 0; q < 8; ++q)
                if (q * 4 + r0 < rows && c0 + k0 * 4 < cols) old[q] = *reinterpret_cast<const float4*>(w + (q * 4 + r0) * w_ld + c0 + k0 * 4);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
              piece[piece_at(lane, k)] = make_uint4(__float_as_uint(alpha * sum[c0 + 4 * k]), __float_as_uint(alpha * sum[c0 + 4 * k + 1]),
                                                    __float_as_uint(alpha * sum[c0 + 4 * k + 2]), __float_as_uint(alpha * sum[c0 + 4 * k + 3]));
            __syncwarp();
            if (p.w_vec) {
#pragma unroll
              for (int q = 0; q < 8; ++q) {
                const int r = q * 4 + r0;
                if (r >= rows || c0 + k0 * 4 >= cols) break;
                const uint4 d = piece[piece_at(r, k0)];
                float4 v;
                v.x = fmaf(keep, old[q].x, __uint_as_float(d.x));
                v.y = fmaf(keep, old[q].y, __uint_as_float(d.y));
                v.z = fmaf(keep, old[q].z, __uint_as_float(d.z));
                v.w = fmaf(keep, old[q].w, __uint_as_float(d.w));
                *reinterpret_cast<float4*>(w + r * w_ld + c0 + k0 * 4) = v;
                if (w16) {
                  const __nv_bfloat162 b[2] = {__floats2bfloat162_rn(v.x, v.y), __floats2bfloat162_rn(v.z, v.w)};
                  *reinterpret_cast<uint2*>(w16 + r * w_ld + c0 + k0 * 4) = *reinterpret_cast<const uint2*>(b);
                }
              }
            } else if (c0 + lane < cols) {
#pragma unroll 1
              for (int q = 0; q < 32; q += 8) {
                float one[8];
#pragma unroll
                for (int r = 0; r < 8; ++r)
                  if (q + r < rows) one[r] = w[(q + r) * w_ld + c0 + lane];
#pragma unroll
                for (int r = 0; r < 8; ++r)
                  if (q + r < rows)
                    put(w, w16, (q + r) * w_ld + c0 + lane,
                        fmaf(keep, one[r], reinterpret_cast<const float*>(piece + piece_at(q + r, lane / 4))[lane % 4]));
              }
            }
            __syncwarp();
          }
        }
      }
    }
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
    tmem_dealloc_pair(tmem_base, 2 * BN);
  }
}

// ---- a Gram matrix from the parts of its sums -----------------------------------------------------------------
// 32 x 32 elements on and above the diagonal per block: the parts added in their order, split, stored, and stored mirrored.
struct GramFinish {
  int count;
  float alpha;
  struct {
    const float* partial;
    half16* out;
    long plane, ld;
    int m, splits, first_block;
  } t[kMaxTensors];
};
__global__ void __launch_bounds__(256) gram_finish_kernel(const __grid_constant__ GramFinish a) {
  behind_previous();
  int k = 0;
  while (k + 1 < a.count && (int)blockIdx.x >= a.t[k + 1].first_block) ++k;
  const auto& t = a.t[k];
  int left = (t.m + 31) / 32, bi = 0, bj = blockIdx.x - t.first_block;
  while (bj >= left) { bj -= left; --left; ++bi; }
  bj += bi;
  __shared__ float tile[32][33];
  const int x = threadIdx.x % 32, y = threadIdx.x / 32;
  const long ld = t.ld, part = (long)t.m * ld;
  auto store = [&](int i, int j, float v) {
    const __half h = __float2half_rn(v), l = __float2half_rn(v - __half2float(h));
    t.out[i * ld + j] = __half_as_ushort(h);
    t.out[t.plane + i * ld + j] = __half_as_ushort(l);
  };
  const int j = bj * 32 + x;
  float v[4][8];  // everything this thread adds, requested at once
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int i = bi * 32 + y + 8 * r;
      v[r][p] = p < t.splits && i < t.m && j < t.m ? t.partial[p * part + i * ld + j] : 0.f;
    }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int i = bi * 32 + y + 8 * r;
    float s = v[r][0];
#pragma unroll
    for (int p = 1; p < 8; ++p) s += v[r][p];
    s *= a.alpha;
    tile[y + 8 * r][x] = s;
    if (i < t.m && j < t.m) store(i, j, s);
  }
  if (bi == bj) return;
  __syncthreads();
#pragma unroll
  for (int r = y; r < 32; r += 8) {
    const int i = bj * 32 + r, c = bi * 32 + x;
    if (i < t.m && c < t.m) store(i, c, tile[x][r]);
  }
}

// ---- all steps of small matrices in one block --------------------------------------------------------------------
// Where every matrix of a call has at most 128 rows, a launch per product is nearly all latency (11 us for 2 us of work).
// Then one block per tensor keeps A, R and S in shared memory, 64 KB each as K-major operand tiles, and takes the steps
// between two Gram matrices in one launch.  The products, their chains and the order of every addition are the product
// kernel's: the results are the same, bit for bit.
constexpr int kSmall = 128, kSmallThreads = 256, kSmallBytes = 4 * kPlaneBytes;  // a matrix: [64 columns][hi, lo][128 rows][128 bytes]
constexpr int kSmallSmem = 3 * kSmallBytes + 1024 + 64;
struct SmallTensor {
  CUtensorMap gram, rest;  // A, and where S goes
  int k_stages, pad[15];
};
struct SmallLaunch {
  Waits waits;
  int group, pad[9];
  SmallTensor t[kMaxTensors];
};

__global__ void __launch_bounds__(kSmallThreads, 1) small_steps_kernel(const __grid_constant__ SmallLaunch L) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t A = base, R = base + kSmallBytes, S = R + kSmallBytes, load_bar = S + kSmallBytes, done_bar = load_bar + 8;
  __shared__ uint32_t tmem_base_slot;
  __shared__ int abort_flag, ran_out;
  const SmallTensor& t = L.t[blockIdx.x];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, k_stages = t.k_stages;
  if (tid == 0) {
    abort_flag = ran_out = 0;
    mbar_init(load_bar, L.waits.signals);
    mbar_init(done_bar, 1);
    mbar_fence_init();
  }
  if (warp == 0) {
    tmem_alloc(smem_u32(&tmem_base_slot), 256);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_slot;
  behind_previous();

  if (tid == 0) {
    mbar_expect_tx(load_bar, k_stages * kOperandBytes);
    for (int kb = 0; kb < k_stages; ++kb) tma_load_3d(A + kb * kOperandBytes, &t.gram, load_bar, kb * BK, 0, 0);
  }
  bool ok = __syncthreads_and(mbar_wait(load_bar, 0, &abort_flag, &ran_out, kDevTimeoutTmaFull, L.waits.limit_cycles));
  tc_fence_after();

  // thread: row `row` and 64 columns of every result
  const int row = (warp & 3) * 32 + lane, group = warp >> 2;
  uint8_t* generic = smem_raw + (base - smem_u32(smem_raw)) + group * kOperandBytes + row * 128;
  auto at = [&](uint32_t m, int plane, int chunk) { return reinterpret_cast<uint4*>(generic + (m - base) + plane * kPlaneBytes + ((chunk ^ (row & 7)) << 4)); };
  uint32_t phase = 0;
  // D = alpha * (c1 add1 + c2 add2 + x y)
  auto product = [&](uint32_t x, uint32_t y, uint32_t d, float alpha, uint32_t add1, float c1, uint32_t add2, float c2) {
    if (!ok) return;
    if (tid == 0) {
      constexpr uint32_t idesc = umma_idesc_f16(128, 128, 0, 0);
      for (int kb = 0; kb < k_stages; ++kb) {
        const uint32_t sx = x + kb * kOperandBytes, sy = y + kb * kOperandBytes, acc = tmem_base + kb * 128;
        const uint64_t xh = smem_desc_sw128(sx, 16), xl = smem_desc_sw128(sx + kPlaneBytes, 16);
        const uint64_t yh = smem_desc_sw128(sy, 16), yl = smem_desc_sw128(sy + kPlaneBytes, 16);
        umma_bf16(acc, xl, yh, idesc, 0u);
        umma_bf16_acc(acc, xh, yl, idesc);
#pragma unroll
        for (int k = 1; k < BK / 16; ++k) {
          umma_bf16_acc(acc, desc_advance(xl, k * 32), desc_advance(yh, k * 32), idesc);
          umma_bf16_acc(acc, desc_advance(xh, k * 32), desc_advance(yl, k * 32), idesc);
        }
#pragma unroll
        for (int k = 0; k < BK / 16; ++k) umma_bf16_acc(acc, desc_advance(xh, k * 32), desc_advance(yh, k * 32), idesc);
      }
      umma_commit(done_bar);
    }
    float sum[64];
#pragma unroll
    for (int j = 0; j < 64; ++j) sum[j] = 0.f;
    if (group < k_stages) {
      auto add = [&](uint32_t m, float c) {
#pragma unroll
        for (int plane = 0; plane < 2; ++plane)
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const uint4 h = *at(m, plane, k);
            const uint32_t w[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 f = unpack_half2(w[e]);
              sum[8 * k + 2 * e] = fmaf(c, f.x, sum[8 * k + 2 * e]);
              sum[8 * k + 2 * e + 1] = fmaf(c, f.y, sum[8 * k + 2 * e + 1]);
            }
          }
      };
      add(add1, c1);
      if (add2) add(add2, c2);
    }
    ok = __syncthreads_and(mbar_wait(done_bar, phase, &abort_flag, &ran_out, kDevTimeoutAccum, L.waits.limit_cycles));
    phase ^= 1;
    if (!ok) return;
    tc_fence_after();
    if (group < k_stages) {
      for (int kb = 0; kb < k_stages; ++kb) {
#pragma unroll
        for (int c = 0; c < 64; c += 16) {
          uint32_t v[16];
          tmem_ld_32x16(tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(kb * 128 + group * 64 + c), v);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 16; ++j) sum[c + j] += __uint_as_float(v[j]);
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = alpha * sum[8 * k + e];
        uint32_t hi[4], lo[4];
        split8(v, hi, lo);
        *at(d, 0, k) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *at(d, 1, k) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      }
    }
    tc_fence_before();
    fence_async_smem();  // the tensor core and the copy engine read what was written here
    __syncthreads();
    tc_fence_after();
  };

  float q0 = kA, sq = kScaleP;
  for (int k = 0; k < L.group; ++k) {
    const uint32_t poly = k == 0 ? S : R;
    product(A, A, poly, poly_alpha(), A, poly_c1(), 0, 0.f);
    if (k > 0) {
      const float sn = rest_scale(k);
      const float alpha = sn / (kScaleP * sq);
      product(R, S, S, alpha, S, kA * sn / sq / alpha, R, q0 * sn / kScaleP / alpha);
      q0 *= kA;
      sq = sn;
    }
    if (k + 1 < L.group)
      for (int twice = 0; twice < 2; ++twice) product(poly, A, A, 1.f / kScaleP, A, kA / (1.f / kScaleP), 0, 0.f);
  }
  if (tid == 0 && ok) {
    for (int kb = 0; kb < k_stages; ++kb)
      asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(&t.rest),
                   "r"(S + kb * kOperandBytes), "r"(kb * BK), "r"(0), "r"(0) : "memory");
    tma_store_commit();
    tma_store_wait_all();
  }
  if (tid == 0 && !ok) {
    // gave up: copies and products in flight get a while to end before shared and tensor memory go away
    const unsigned long long t0 = global_timer_ns();
    while (!mbar_try_wait(load_bar, 0) && global_timer_ns() - t0 < 100000000ull) {}
    while (!mbar_try_wait(done_bar, phase ^ 1) && global_timer_ns() - t0 < 100000000ull) {}
  }
  tc_fence_before();
  __syncthreads();
  if (tid == 0 && ran_out) report(L.waits, ran_out);
  if (warp == 0) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem_base, 256);
  }
}

// ---- momentum, norm, X_0 ----------------------------------------------------------------------------------------
struct Element {
  const float* grad;
  float* momentum;
  half16* x;       // planes of X_0 [2][m][ld]
  long rows, cols, ld, plane;
  long first_norm, first_split;  // first block of each kernel
  int transposed, vec;
};
struct Elements {
  int count, nesterov;
  float mu;
  long norm_blocks;
  double* partial;  // a sum of squares per block of the first kernel
  double* inverse;  // 1 / |U|_F per tensor
  Element t[kMaxTensors];
};
constexpr int kNormThreads = 256, kNormChunk = 8192;

__device__ __forceinline__ float direction(float g, float m, float mu, int nesterov) { return nesterov ? fmaf(mu, m, g) : m; }

// M <- mu M + G; the block's sum of squares of U, in 64 bits: neither tiny nor huge gradients leave the range.
__global__ void __launch_bounds__(kNormThreads) momentum_norm_kernel(const __grid_constant__ Elements a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  int t = 0;
  while (t + 1 < a.count && blockIdx.x >= a.t[t + 1].first_norm) ++t;
  const Element& e = a.t[t];
  const long n = e.rows * e.cols, begin = (blockIdx.x - e.first_norm) * kNormChunk;
  const long end = begin + kNormChunk < n ? begin + kNormChunk : n;
  double s = 0.0;
  if (e.vec) {
    for (long i = begin + threadIdx.x * 4; i < end; i += kNormThreads * 4) {
      const float4 g = __ldcs(reinterpret_cast<const float4*>(e.grad + i));
      float4 m = *reinterpret_cast<const float4*>(e.momentum + i);
      m.x = fmaf(a.mu, m.x, g.x); m.y = fmaf(a.mu, m.y, g.y); m.z = fmaf(a.mu, m.z, g.z); m.w = fmaf(a.mu, m.w, g.w);
      *reinterpret_cast<float4*>(e.momentum + i) = m;
      const double u0 = direction(g.x, m.x, a.mu, a.nesterov), u1 = direction(g.y, m.y, a.mu, a.nesterov);
      const double u2 = direction(g.z, m.z, a.mu, a.nesterov), u3 = direction(g.w, m.w, a.mu, a.nesterov);
      s += (u0 * u0 + u1 * u1) + (u2 * u2 + u3 * u3);
    }
  } else {
    for (long i = begin + threadIdx.x; i < end; i += kNormThreads) {
      const float g = e.grad[i], m = fmaf(a.mu, e.momentum[i], g);
      e.momentum[i] = m;
      const double u = direction(g, m, a.mu, a.nesterov);
      s += u * u;
    }
  }
  __shared__ double part[kNormThreads / 32];
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kNormThreads / 32; ++i) s += part[i];
    a.partial[blockIdx.x] = s;
  }
}

// One block per tensor adds its blocks' sums, always in the same order.
__global__ void __launch_bounds__(1024) inverse_norm_kernel(const __grid_constant__ Elements a) {
  behind_previous();
  const int t = blockIdx.x;
  const long begin = a.t[t].first_norm, end = t + 1 < a.count ? a.t[t + 1].first_norm : a.norm_blocks;
  double s = 0.0;
  for (long i = begin + threadIdx.x; i < end; i += 1024) s += a.partial[i];
  __shared__ double part[32];
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 32; ++i) s += part[i];
    // no direction in a zero gradient; a NaN or an infinity anywhere makes the tensor's update NaN
    a.inverse[t] = s == 0.0 ? 0.0 : isinf(s) ? (double)NAN : 1.0 / sqrt(s);
  }
}

// X_0 = U / |U|_F as planes, transposed where the matrix has more rows than columns.
constexpr int kSplitThreads = 256;
__global__ void __launch_bounds__(kSplitThreads) split_kernel(const __grid_constant__ Elements a) {
  behind_previous();
  int t = 0;
  while (t + 1 < a.count && blockIdx.x >= a.t[t + 1].first_split) ++t;
  const Element& e = a.t[t];
  const long block = blockIdx.x - e.first_split;
  const double f = a.inverse[t] * kScaleX;
  auto value = [&](long i) { return (float)(f * direction(e.grad[i], e.momentum[i], a.mu, a.nesterov)); };
  if (!e.transposed) {
    const long per_row = e.ld / 8, item = block * kSplitThreads + threadIdx.x;
    const long r = item / per_row, c = (item - r * per_row) * 8;
    if (r >= e.rows) return;
    const long i = r * e.cols + c;
    float v[8];
    if (e.vec && c + 8 <= e.cols && e.cols % 4 == 0) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 g = __ldcs(reinterpret_cast<const float4*>(e.grad + i) + h), m = __ldcs(reinterpret_cast<const float4*>(e.momentum + i) + h);
        v[4 * h] = (float)(f * direction(g.x, m.x, a.mu, a.nesterov));
        v[4 * h + 1] = (float)(f * direction(g.y, m.y, a.mu, a.nesterov));
        v[4 * h + 2] = (float)(f * direction(g.z, m.z, a.mu, a.nesterov));
        v[4 * h + 3] = (float)(f * direction(g.w, m.w, a.mu, a.nesterov));
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = c + k < e.cols ? value(i + k) : 0.f;
    }
    uint32_t hi[4], lo[4];
    split8(v, hi, lo);
    half16* dst = e.x + r * e.ld + c;
    *reinterpret_cast<uint4*>(dst) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(dst + e.plane) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  } else {
    __shared__ float tile[32][33];
    const long across = (e.cols + 31) / 32, r0 = block / across * 32, c0 = block % across * 32;
    const int x = threadIdx.x % 32, y = threadIdx.x / 32;
    for (int k = y; k < 32; k += 8)
      if (r0 + k < e.rows && c0 + x < e.cols) tile[k][x] = value((r0 + k) * e.cols + c0 + x);
    __syncthreads();
    for (int k = y; k < 32; k += 8)
      if (c0 + k < e.cols && r0 + x < e.rows) {
        const float v = tile[x][k];
        const __half h = __float2half_rn(v), l = __float2half_rn(v - __half2float(h));
        half16* dst = e.x + (c0 + k) * e.ld + r0 + x;
        dst[0] = __half_as_ushort(h);
        dst[e.plane] = __half_as_ushort(l);
      }
  }
}

// Biases: momentum, and a plain step along U.
struct Vectors {
  int count, nesterov;
  float mu, lr;
  struct { const float* grad; float *momentum, *w; bf16* w16; int n; } t[32];
};
__global__ void vector_update_kernel(const __grid_constant__ Vectors a) {
  const auto& v = a.t[blockIdx.x];
  for (int i = threadIdx.x; i < v.n; i += blockDim.x) {
    const float g = v.grad[i], m = fmaf(a.mu, v.momentum[i], g);
    v.momentum[i] = m;
    const float w = fmaf(-a.lr, direction(g, m, a.mu, a.nesterov), v.w[i]);
    v.w[i] = w;
    if (v.w16) v.w16[i] = __float2bfloat16_rn(w);
  }
}

// ---- host ------------------------------------------------------------------------------------------------------
size_t up(size_t v, size_t a) { return (v + a - 1) / a * a; }

struct Shape {
  long m, n, ldn, ldm;  // of X: rows <= columns; row strides of X and of the m x m matrices
  bool transposed;
  explicit Shape(const vgg19_muon_tensor& t)
      : m(t.rows < t.cols ? t.rows : t.cols), n(t.rows < t.cols ? t.cols : t.rows), ldn((long)up(n, 8)), ldm((long)up(m, 8)),
        transposed(t.rows > t.cols) {}
  size_t x_bytes() const { return up((size_t)2 * m * ldn * 2, 256); }
  size_t a_bytes() const { return up((size_t)2 * m * ldm * 2, 256); }
  // A Gram matrix of at most 1024 rows has few tiles and may have a long K, which is then cut into parts of about 16 stages
  // (one 512 x 4608 filter's takes 85 us uncut); a larger one into as many as leave every pair of SMs a tile, which is two up to
  // 1408 rows (1200 x 8000 673 us, uncut 748; 1408 x 8000 738, uncut 811) and none beyond.  By the
  // tensor alone, so that no result depends on what else is updated.
  int gram_stages() const { return (int)((n + BK - 1) / BK); }
  int gram_splits() const {
    const long i = (m + 2 * BM - 1) / (2 * BM), j = (m + BM - 1) / BM, halves = i * j - i * (i - 1);  // tiles of 128 columns from the diagonal on
    const long most = m <= 1024 ? 8 : 74 / halves, parts = (gram_stages() + 15) / 16;
    return (int)(most < 2 || parts < 2 ? 1 : parts < most ? parts : most);
  }
  size_t partial_bytes() const { return gram_splits() > 1 ? up((size_t)gram_splits() * m * ldm * 4, 256) : 0; }
  long norm_blocks() const { return (m * n + kNormChunk - 1) / kNormChunk; }
  long split_blocks() const {
    return transposed ? ((n + 31) / 32) * ((m + 31) / 32) : (m * (ldn / 8) + kSplitThreads - 1) / kSplitThreads;
  }
};

enum Matrix { kX0, kX1, kGramA, kPoly, kQa, kQb, kPA, kMatrices };

// The planes of one tensor in the workspace and their tensor maps.
struct Planes {
  half16* at[kMatrices];
  float* partial;
  CUtensorMap k_major[kMatrices], box64[kMatrices];  // boxes of 128 and of 64 rows
};

bool plane_map(CUtensorMap* map, const half16* base, long rows, long cols, long ld, uint32_t box_rows) {
  const TensorMapApi& api = tensor_map_api();
  if (!api.ok) return false;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, 2};
  cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)rows * ld * 2};
  cuuint32_t box[3] = {BK, box_rows, 2};
  cuuint32_t estr[3] = {1, 1, 1};
  return api.encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<half16*>(base), dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

size_t tensor_bytes(const Shape& s) { return 2 * s.x_bytes() + 5 * s.a_bytes() + s.partial_bytes(); }

size_t batch_bytes(const vgg19_muon_tensor* t, int count) {
  size_t b = up(kMaxTensors * sizeof(double), 256);
  long blocks = 0;
  for (int i = 0; i < count; ++i) {
    const Shape s(t[i]);
    b += tensor_bytes(s);
    blocks += s.norm_blocks();
  }
  return b + up(blocks * sizeof(double), 256);
}

// A launch whose set-up overlaps the one before it in the stream (the kernel waits for that one itself).
template <typename P> cudaError_t launch_behind(void (*kernel)(P), unsigned blocks, int threads, int smem, const P& params, cudaStream_t st) {
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
  return cudaLaunchKernelEx(&cfg, kernel, params);
}

// The launch's tiles of 256 x bn.
template <int N> int count_tiles(Launch<N>& L, int bn) {
  int tiles = 0;
  const int wide = 2 * BM / bn;
  for (int i = 0; i < L.count; ++i) {
    Problem& p = L.p[i];
    if (p.splits < 1) { p.splits = 1; p.per_split = p.k_stages; }
    p.tiles_m = (p.m + 2 * BM - 1) / (2 * BM);
    p.tiles_n = (p.n + bn - 1) / bn;
    p.sym = p.square == 1 || (p.square == 2 && bn == 2 * BM);
    L.first_tile[i] = tiles;
    tiles += p.splits * (p.tiles_m * p.tiles_n - (p.sym ? wide * (p.tiles_m * (p.tiles_m - 1) / 2) : 0));
  }
  L.first_tile[L.count] = tiles;
  return tiles;
}

// The longest that a pair is busy with 256 x bn tiles: with each its stages, and about seven more for what comes before and
// after them; a half takes about 5/8 of a whole.  (The sums are the same, bit for bit.)  Measured: the sixteen filters
// 674 -> 657 us against counting tiles alone, with the largest tensors first in both.
template <int N> long busiest(Launch<N>& L, int bn, int pairs) {
  constexpr int kMost = 128;
  const int tiles = count_tiles(L, bn);
  if (pairs > kMost || (bn == 128 && tiles > 16 * pairs)) return 1L << 60;
  if (tiles > 16 * pairs) return 0;
  long load[kMost] = {}, most = 0;
  for (int i = 0; i < L.count; ++i)
    for (int t = L.first_tile[i]; t < L.first_tile[i + 1]; ++t) {
      long& l = load[t % pairs];
      l += (7 + L.p[i].per_split) * (bn == 128 ? 5 : 8);
      if (l > most) most = l;
    }
  return most;
}

template <bool FINAL, int BN, int N> cudaError_t launch_tiles(const Launch<N>& L, int pairs, cudaStream_t st) {
  const cudaError_t e = cudaFuncSetAttribute(split_product_pair_kernel<N, FINAL, BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
  if (e != cudaSuccess) return e;
  const int tiles = L.first_tile[L.count];
  return launch_behind(split_product_pair_kernel<N, FINAL, BN>, (unsigned)(2 * (tiles < pairs ? tiles : pairs)), kThreads, kSmemBytes, L, st);
}

// narrow[i]: the map of problem i's second operand in boxes of 64 rows, or null where p.b is that (or it is read by columns).
template <bool FINAL, int N> cudaError_t launch_products(Launch<N>& L, const CUtensorMap* const* narrow, cudaStream_t st) {
  int dev = 0, sms = 148;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  const int pairs = sms / 2;
  if (busiest(L, 128, pairs) < busiest(L, 256, pairs)) {
    count_tiles(L, 128);
    for (int i = 0; i < L.count; ++i)
      if (narrow[i]) L.p[i].b = *narrow[i];
    return launch_tiles<FINAL, 128>(L, pairs, st);
  }
  count_tiles(L, 256);
  return launch_tiles<FINAL, 256>(L, pairs, st);
}

cudaError_t launch_small(const SmallLaunch& L, int count, cudaStream_t st) {
  cudaError_t e = cudaFuncSetAttribute(small_steps_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallSmem);
  if (e != cudaSuccess) return e;
  return launch_behind(small_steps_kernel, (unsigned)count, kSmallThreads, kSmallSmem, L, st);
}

struct Options {
  float lr, mu, decay;
  int steps, nesterov;
  Waits products, small_steps;  // of either kernel
};

// The whole update of up to kMaxTensors tensors; N is the largest number of products per launch.
template <int N>
cudaError_t update_batch(const vgg19_muon_tensor* given, const int count, const Options& o, char* ws, cudaStream_t st) {
  // the largest first: their tiles are the longest, and what is left over at the end of a launch should be short
  vgg19_muon_tensor tensors[kMaxTensors];
  for (int i = 0; i < count; ++i) {
    int at = i;
    for (; at > 0 && Shape(tensors[at - 1]).m < Shape(given[i]).m; --at) tensors[at] = tensors[at - 1];
    tensors[at] = given[i];
  }
  static thread_local Planes planes[kMaxTensors];
  Elements el{};
  el.count = count; el.nesterov = o.nesterov; el.mu = o.mu;
  el.inverse = reinterpret_cast<double*>(ws);
  ws += up(kMaxTensors * sizeof(double), 256);
  long norm_blocks = 0, split_blocks = 0;
  for (int i = 0; i < count; ++i) {
    const vgg19_muon_tensor& t = tensors[i];
    const Shape s(t);
    Planes& q = planes[i];
    for (int k = 0; k < kMatrices; ++k) {
      const bool x = k <= kX1;
      q.at[k] = reinterpret_cast<half16*>(ws);
      ws += x ? s.x_bytes() : s.a_bytes();
      if (!plane_map(&q.k_major[k], q.at[k], s.m, x ? s.n : s.m, x ? s.ldn : s.ldm, 128)) return cudaErrorInvalidValue;
      if (!plane_map(&q.box64[k], q.at[k], s.m, x ? s.n : s.m, x ? s.ldn : s.ldm, 64)) return cudaErrorInvalidValue;
    }
    q.partial = reinterpret_cast<float*>(ws);
    ws += s.partial_bytes();
    Element& e = el.t[i];
    e.grad = t.grad; e.momentum = t.momentum; e.x = q.at[kX0];
    e.rows = t.rows; e.cols = t.cols; e.ld = s.ldn; e.plane = s.m * s.ldn;
    e.transposed = s.transposed;
    // (a chunk of the first kernel starts on a multiple of four elements, and so do the last whole fours of a tensor)
    e.vec = reinterpret_cast<uintptr_t>(t.grad) % 16 == 0 && reinterpret_cast<uintptr_t>(t.momentum) % 16 == 0 && t.rows * t.cols % 4 == 0;
    e.first_norm = norm_blocks; e.first_split = split_blocks;
    norm_blocks += s.norm_blocks();
    split_blocks += s.split_blocks();
  }
  el.norm_blocks = norm_blocks;
  el.partial = reinterpret_cast<double*>(ws);
  momentum_norm_kernel<<<(unsigned)norm_blocks, kNormThreads, 0, st>>>(el);
  cudaError_t err = cudaGetLastError();
  if (err == cudaSuccess) err = launch_behind(inverse_norm_kernel, (unsigned)count, 1024, 0, el, st);
  if (err == cudaSuccess) err = launch_behind(split_kernel, (unsigned)split_blocks, kSplitThreads, 0, el, st);
  if (err != cudaSuccess) return err;

  static thread_local Launch<N> L;
  const CUtensorMap* narrow[N];
  // D = scale_d * (A / scale_a) (B / scale_b), all m x m symmetric
  auto symmetric = [&](int i, Matrix a, float sa, Matrix b, float sb, Matrix d, float sd) -> Problem& {
    const Shape s(tensors[i]);
    Problem& p = L.p[L.count++];
    p = Problem{};
    p.a = planes[i].k_major[a]; p.b = planes[i].k_major[b];
    narrow[L.count - 1] = &planes[i].box64[b];
    p.m = p.n = (int)s.m;
    p.k_stages = (int)((s.m + BK - 1) / BK);
    p.square = s.m > 1024;  // (where all tiles are taken, halves of them can fill idle pairs, and none is stored twice)
    p.alpha = sd / (sa * sb);
    p.out = planes[i].at[d]; p.ld = s.ldm; p.plane = s.m * s.ldm;
    return p;
  };
  auto run = [&] {
    if (err == cudaSuccess) err = L.p[0].w ? launch_products<true>(L, narrow, st) : launch_products<false>(L, narrow, st);
    L.count = 0;
  };
  bool small = true;
  for (int i = 0; i < count; ++i) small = small && Shape(tensors[i]).m <= kSmall;
  L.count = 0;
  L.waits = o.products;
  int x = kX0;
  for (int done = 0; done < o.steps;) {
    const int group = steps_of_group(done, o.steps);
    GramFinish finish{};
    int finish_blocks = 0;
    for (int i = 0; i < count; ++i) {
      Problem& p = symmetric(i, (Matrix)x, kScaleX, (Matrix)x, kScaleX, kGramA, kScaleA);
      const Shape s(tensors[i]);
      p.k_stages = s.gram_stages();
      if (s.gram_splits() > 1) {
        p.splits = s.gram_splits();
        p.per_split = (p.k_stages + p.splits - 1) / p.splits;
        p.partial = planes[i].partial;
        auto& t = finish.t[finish.count++];
        t.partial = p.partial; t.out = p.out; t.plane = p.plane; t.ld = p.ld;
        t.m = p.m; t.splits = p.splits; t.first_block = finish_blocks;
        finish.alpha = p.alpha;
        if (!p.square) p.square = 2;
        const int b = (p.m + 31) / 32;
        finish_blocks += b * (b + 1) / 2;
      }
    }
    run();
    if (finish.count && err == cudaSuccess) {
      err = launch_behind(gram_finish_kernel, (unsigned)finish_blocks, 256, 0, finish, st);
    }
    // p(A) = a I + R with R = b A + c A A; Q = q0 I + S.  The identity's share is added in the epilogues, in fp32: what
    // the tensor core truncates is then relative to the smaller rest.
    Matrix q = kQa;  // S
    float sq = kScaleP, q0 = kA;
    if (small) {
      static thread_local SmallLaunch sl;
      sl.waits = o.small_steps;
      sl.group = group;
      for (int i = 0; i < count; ++i) {
        sl.t[i].gram = planes[i].k_major[kGramA];
        sl.t[i].rest = planes[i].k_major[kQa];
        sl.t[i].k_stages = (int)((Shape(tensors[i]).m + BK - 1) / BK);
      }
      if (err == cudaSuccess) err = launch_small(sl, count, st);
      sq = rest_scale(group - 1);
      for (int k = 1; k < group; ++k) q0 *= kA;
    }
    for (int k = small ? group : 0; k < group; ++k) {
      const Matrix poly = k == 0 ? kQa : kPoly;  // R; the first one is also the first S
      for (int i = 0; i < count; ++i) {
        Problem& p = symmetric(i, kGramA, kScaleA, kGramA, kScaleA, poly, kC * kScaleP);
        p.alpha = poly_alpha();
        p.add1 = planes[i].at[kGramA]; p.c1 = poly_c1();
      }
      run();
      // S <- a S + q0 R + R S, for the tensors of one parity: between them the two launches that follow have room for it
      const Matrix next = q == kQa ? kQb : kQa;
      const float sn = rest_scale(k);
      auto rest = [&](int parity) {
        if (k == 0) return;
        for (int i = parity; i < count; i += 2) {
          Problem& p = symmetric(i, poly, kScaleP, q, sq, next, sn);
          p.add1 = planes[i].at[q]; p.c1 = kA * sn / sq / p.alpha;
          p.add2 = planes[i].at[poly]; p.c2 = q0 * sn / kScaleP / p.alpha;
        }
      };
      if (k + 1 < group) {  // A <- p A p, one factor at a time
        for (int i = 0; i < count; ++i) {
          Problem& p = symmetric(i, poly, kScaleP, kGramA, kScaleA, kPA, kScaleA);
          p.add1 = planes[i].at[kGramA]; p.c1 = kA / p.alpha;
        }
        rest(0);
        run();
        for (int i = 0; i < count; ++i) {
          Problem& p = symmetric(i, poly, kScaleP, kPA, kScaleA, kGramA, kScaleA);
          p.add1 = planes[i].at[kPA]; p.c1 = kA / p.alpha;
        }
        rest(1);
        run();
      } else if (k > 0) {
        rest(0);
        rest(1);
        run();
      }
      if (k > 0) {
        q = next;
        sq = sn;
        q0 *= kA;
      }
    }
    done += group;
    for (int i = 0; i < count; ++i) {
      const vgg19_muon_tensor& t = tensors[i];
      const Shape s(t);
      narrow[L.count] = nullptr;
      Problem& p = L.p[L.count++];
      p = Problem{};
      p.a = planes[i].k_major[q]; p.b = planes[i].box64[x];
      p.b_mn = 1;
      p.m = (int)s.m; p.n = (int)s.n;
      p.k_stages = (int)((s.m + BK - 1) / BK);
      p.ld = s.ldn; p.plane = s.m * s.ldn;
      p.add1 = planes[i].at[x]; p.c1 = q0 * sq;
      if (done < o.steps) {
        p.alpha = 1.f / sq;
        p.out = planes[i].at[x ^ 1];
      } else {
        const double scale = t.rows > t.cols ? sqrt((double)t.rows / (double)t.cols) : 1.0;
        p.alpha = (float)(-(double)o.lr * scale / ((double)sq * kScaleX));
        p.keep = (float)(1.0 - (double)o.lr * o.decay);
        p.w = t.w; p.w16 = static_cast<bf16*>(t.w_bf16);
        p.w_ld = t.cols;
        p.transposed = s.transposed;
        p.w_vec = t.cols % 4 == 0 && reinterpret_cast<uintptr_t>(t.w) % 16 == 0 && reinterpret_cast<uintptr_t>(t.w_bf16) % 8 == 0;
      }
    }
    run();
    x ^= 1;
  }
  return err;
}

int check_tensors(const vgg19_muon_tensor* t, int32_t count) {
  if (count < 0 || (count && !t)) return note_error(VGG19_ERR_ARG, "%d tensors, or a null list", count);
  for (int i = 0; i < count; ++i)
    if (t[i].rows < 1 || t[i].cols < 1 || t[i].rows > (1 << 24) || t[i].cols > (1 << 24) ||
        (t[i].rows < t[i].cols ? t[i].rows : t[i].cols) > (1 << 15) || t[i].rows * t[i].cols > (1LL << 34))
      return note_error(VGG19_ERR_SHAPE, "tensor %d is %lld x %lld: sides in [1, 2^24], the smaller at most 2^15, 2^34 elements", i,
                        (long long)t[i].rows, (long long)t[i].cols);
  return VGG19_OK;
}

// Blocks read and write in no order, so what is written may overlap nothing: neither another tensor (or the same one
// twice), nor the workspace.  Gradients are only read.
int check_overlaps(const vgg19_muon_tensor* t, int32_t count, const void* workspace, size_t bytes) {
  struct Range {
    uintptr_t begin, end;
    bool written;
  };
  try {
    std::vector<Range> r;
    r.reserve(4 * (size_t)count + 1);
    auto add = [&r](const void* p, size_t n, bool written) {
      const uintptr_t b = reinterpret_cast<uintptr_t>(p);
      if (p) r.push_back(Range{b, b + n, written});
    };
    add(workspace, bytes, true);
    for (int i = 0; i < count; ++i) {
      const size_t n = (size_t)(t[i].rows * t[i].cols);
      add(t[i].w, 4 * n, true);
      add(t[i].w_bf16, 2 * n, true);
      add(t[i].momentum, 4 * n, true);
      add(t[i].grad, 4 * n, false);
    }
    std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
    uintptr_t end = 0, written_end = 0;  // of what began before
    for (const Range& x : r) {
      if (x.begin < written_end || (x.written && x.begin < end))
        return note_error(VGG19_ERR_ARG, "a weight, its copy, a momentum or the workspace overlaps another tensor of the call");
      if (x.end > end) end = x.end;
      if (x.written && x.end > written_end) written_end = x.end;
    }
  } catch (...) {
    return note_error(VGG19_ERR_ARG, "no host memory for the list of %d tensors", count);
  }
  return VGG19_OK;
}

size_t workspace_bytes(const vgg19_muon_tensor* t, int32_t count) {
  size_t most = 256;
  for (int i = 0; i < count; i += kMaxTensors) {
    const size_t b = batch_bytes(t + i, count - i < kMaxTensors ? count - i : kMaxTensors);
    if (b > most) most = b;
  }
  return most;
}

}  // namespace

cudaError_t muon_take_error(int* code, cudaStream_t st) {
  void* word = nullptr;
  const cudaError_t e = cudaGetSymbolAddress(&word, g_muon_error);
  return e == cudaSuccess ? take_error(static_cast<int*>(word), code, st) : e;
}

cudaError_t muon_vector_update(const MuonVector* v, int count, float lr, float mu, bool nesterov, cudaStream_t st) {
  Vectors a{};
  a.nesterov = nesterov; a.mu = mu; a.lr = lr;
  for (int i = 0; i < count; ++i) {
    a.t[a.count].grad = v[i].grad; a.t[a.count].momentum = v[i].momentum; a.t[a.count].w = v[i].w;
    a.t[a.count].w16 = v[i].w16; a.t[a.count].n = v[i].n;
    if (++a.count == 32 || i + 1 == count) {
      vector_update_kernel<<<(unsigned)a.count, 256, 0, st>>>(a);
      a.count = 0;
    }
  }
  return cudaGetLastError();
}

}  // namespace vgg

extern "C" size_t vgg19_muon_workspace_bytes(const vgg19_muon_tensor* tensors, int32_t count) {
  return vgg::check_tensors(tensors, count) == VGG19_OK ? vgg::workspace_bytes(tensors, count) : 0;
}

int vgg::muon_update(const vgg19_muon_tensor* tensors, int32_t count, float lr, float momentum, float decay, int32_t steps, int32_t nesterov,
                     void* workspace, size_t bytes, const Waits& products, const Waits& small_steps, void* stream) {
  const int rc = check_tensors(tensors, count);
  if (rc != VGG19_OK) return rc;
  if (!(lr == lr) || !(momentum == momentum) || !(decay == decay))
    return note_error(VGG19_ERR_ARG, "NaN learning rate, momentum or decay");
  if (steps < 1 || steps > 16) return note_error(VGG19_ERR_ARG, "%d steps outside [1, 16]", steps);
  for (int i = 0; i < count; ++i) {
    const vgg19_muon_tensor& t = tensors[i];
    if (!t.w || !t.grad || !t.momentum) return note_error(VGG19_ERR_ARG, "tensor %d has a null weight, gradient or momentum", i);
    if (reinterpret_cast<uintptr_t>(t.w) % 4 || reinterpret_cast<uintptr_t>(t.grad) % 4 || reinterpret_cast<uintptr_t>(t.momentum) % 4 ||
        reinterpret_cast<uintptr_t>(t.w_bf16) % 2)
      return note_error(VGG19_ERR_ARG, "tensor %d is not aligned to its type", i);
  }
  if (count == 0) return VGG19_OK;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256)
    return note_error(VGG19_ERR_WORKSPACE, "the workspace is null or not 256-byte aligned");
  if (bytes < workspace_bytes(tensors, count))
    return note_error(VGG19_ERR_WORKSPACE, "workspace has %zu bytes, this call needs %zu", bytes, workspace_bytes(tensors, count));
  const int apart = check_overlaps(tensors, count, workspace, workspace_bytes(tensors, count));
  if (apart != VGG19_OK) return apart;
  const Options o{lr, momentum, decay, steps, nesterov != 0, products, small_steps};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  for (int i = 0; i < count; i += kMaxTensors) {
    const int n = count - i < kMaxTensors ? count - i : kMaxTensors;
    const cudaError_t e = n <= 2 ? update_batch<4>(tensors + i, n, o, static_cast<char*>(workspace), st)
                                 : update_batch<kMaxProblems>(tensors + i, n, o, static_cast<char*>(workspace), st);
    if (e != cudaSuccess) return note_error(VGG19_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
  }
  return VGG19_OK;
}

extern "C" int vgg19_muon_update(const vgg19_muon_tensor* tensors, int32_t count, float lr, float momentum, float decay,
                                 int32_t steps, int32_t nesterov, void* workspace, size_t bytes, void* stream) {
  return vgg::muon_update(tensors, count, lr, momentum, decay, steps, nesterov, workspace, bytes, vgg::Waits{}, vgg::Waits{}, stream);
}
