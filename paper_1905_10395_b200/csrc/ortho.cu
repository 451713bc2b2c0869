// Orthogonalised updates (include/lsgd.h): momentum and norm, then Newton-Schulz steps on the 5th-generation tensor cores.
//
//   G = X X^T,   Q = a I + b G + c G G,   X <- Q X        (X is the smaller side by the larger: rows r <= columns)
//
// Three batched products a step, with the polynomial in the second one's epilogue (a I belongs to Q, whose diagonal is then what
// singular values are multiplied by, about 1 in the last steps; stored without it, it would be about -2.5 and its rounding count
// 2.5 times).  G and Q are symmetric: only tiles on and above the diagonal are computed, each stored twice, the second time
// transposed, so a step costs 1.5 r r n + 0.5 r r r multiply-adds instead of 2 r r n + r r r.
//
// Operands are fp16 times 2^10, sums fp32.  Entries of X and G are below 2 (singular values stay below 1.3 with the usual
// coefficients) and those that matter are not below 2^-13 of their matrix's largest, so fp16's range holds them and its 11 bits
// lose an eighth of what bf16's 8 would.
//
// A rounding of X also falls on directions whose singular values are small or zero, where every later step multiplies it by a = 3.4: by
// 485 from the first X on, which a result of few large singular values (a gradient of few tokens) does not hide.  So what X is
// rounded by, R, is kept too, in fp16, and X <- Q X + diag(Q) R: on directions that Q stretches by about a, so does its diagonal, and
// elsewhere a rounding is not amplified.  That costs R's way from and to memory; the whole product Q R would take a third more time (2048 x
// 8192: 958 us instead of 778, without R 720).  Up to kTwofoldRows rows the diagonal holds too much of the few large singular values (64 x
// 64 of rank 1: off by 0.8 %, 16 x 16: 2.8), and the contraction is short: there it is the whole product.  The last step goes
// without R: what X is rounded by in front of it is amplified once.
// Off the exact result, relative to its norm (rounding to bf16 alone: 0.17 %), with and without R, by 1024 x 1024 matrices of rank 1:
// 0.32 and 15 %; 4: 0.24, 7.4; 16: 0.24, 4.6; 64: 0.24, 2.4; 256: 0.23, 0.9; full: 0.195, 0.205.
//
// product_kernel is a persistent kernel of one CTA an SM on tiles of 128 x 128 or 128 x 64, or of pairs of CTAs on 256 x 256, with the roles of the
// batched product of gemm_tc.cu: one thread fetches operands by tiled bulk copies into a ring, one issues tcgen05.mma into one of two
// accumulators in tensor memory, one fetches the tiles that are added, eight warps run the epilogue.  Every wait is bounded by a clock
// budget; on expiry the kernel raises a status bit, drains its copies, frees tensor memory and returns.
//
// What bounds it: large batches (2 x 4096 x 4096: 2.6 ms, 1070 TFLOP/s; 32 x 1024 x 1024 with momentum: 1.2 ms, 570) the operands' way from L2, at
// 8 TB/s; a few small matrices (8 x 256 x 256: 88 us) the chain of 15 dependent products of about 6 us each: its first operands'
// latency 1.2, the contraction 1.3, the epilogue with its store 1, the change of kernels 1.6.
#include <cuda_fp16.h>

#include "seq.h"
#include "tc.h"

namespace lsgd {
namespace ortho {
using namespace tc;
namespace {

__device__ uint32_t g_status;                    // of the device

constexpr float kScale = 1024.f;                 // of X, G and Q as stored
constexpr int BM = 128, BK = 64, kBoxBytes = 64 * 64 * 2, kTileBytes = BM * 128 * 2;
constexpr int kTwofoldRows = 128;
// The products' forms: 128 columns a tile or 64, or pairs of CTAs of 128 rows and 256 columns each.
template <bool PAIR, int BN>
struct Form {
  static constexpr int kM = PAIR ? 256 : 128, kN = PAIR ? 256 : BN;      // of a tile
  static constexpr int kBoxesB = PAIR ? 2 : BN / 64;                     // of B, a CTA fetches 64 rows or columns at a time
  static constexpr int kStageBytes = (2 + kBoxesB) * kBoxBytes, kStages = BN == 64 ? 6 : 5;
  static constexpr int kSmemBytes = kStages * kStageBytes + 2 * kTileBytes + 1024;
};
constexpr int kEpiWarps = 8, kThreads = 96 + 32 * kEpiWarps;    // operands, products, the added tile; the epilogue

// ------------------------------------------------------------------------------------------------ momentum and norm
struct Prep {
  lsgd_ortho_desc d;
  double* part;              // [P][blocks] sums of squares
  uint32_t blocks;
  uint32_t* done;            // counters of the products, cleared: n_done of them
  uint32_t n_done;
  __half *x, *lo;            // [P][r][ld]: X and what it was rounded by
  int32_t r, n, tall;        // rows and columns of X; tall: X is the matrix transposed
  int32_t out_wide;          // out's rows can be written 8 values at a time
  int64_t ld, stride;
};

// A piece of the update: its gradient and momentum, and what becomes of them.
template <typename T, int VEC>
struct Piece {
  Pack<T, VEC> g;
  Pack<float, VEC> m;
  __device__ __forceinline__ void load(const Prep& a, int p, int row, int col) {
    g.load(Rows<T>{static_cast<T*>(a.d.grad.data), a.d.grad.ld, a.d.grad.stride}.row(p, row) + col);
    if (a.d.momentum.data) m.load(momentum(a, p, row, col));
  }
  // u: the update; `step`: the momentum moves first, and is written
  __device__ __forceinline__ void update(const Prep& a, int p, int row, int col, bool step, float (&u)[VEC]) {
    g.get(u);
    if (!a.d.momentum.data) return;
    float v[VEC];
    m.get(v);
    if (step) {
#pragma unroll
      for (int k = 0; k < VEC; ++k) v[k] = fmaf(a.d.mu, v[k], u[k]);
      m.set(v);
      m.store(momentum(a, p, row, col));
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) u[k] = a.d.nesterov ? fmaf(a.d.mu, v[k], u[k]) : v[k];
  }
  static __device__ __forceinline__ float* momentum(const Prep& a, int p, int row, int col) {
    return Rows<float>{static_cast<float*>(a.d.momentum.data), a.d.momentum.ld, a.d.momentum.stride}.row(p, row) + col;
  }
};

// The momentum's step, and every block's sum of squares of the update: in 64 bits, since squares of small gradients leave fp32's range.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) norm_kernel(const __grid_constant__ Prep a) {
  pdl_wait();
  pdl_launch_dependents();
  const int p = blockIdx.y;
  if (blockIdx.x == 0 && p == 0)
    for (uint32_t i = threadIdx.x; i < a.n_done; i += 256) a.done[i] = 0;
  const uint32_t per = (a.d.n + VEC - 1) / VEC;
  const int64_t pieces = (int64_t)a.d.m * per;
  double s = 0.0;
  constexpr int kTake = 4;           // pieces fetched before the first is used
  const int64_t apart = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += kTake * apart) {
    Piece<T, VEC> piece[kTake];
    int row[kTake], col[kTake];
#pragma unroll
    for (int k = 0; k < kTake; ++k) {
      row[k] = (int)((uint32_t)(i + k * apart) / per), col[k] = (int)((uint32_t)(i + k * apart) % per) * VEC;
      if (i + k * apart < pieces) piece[k].load(a, p, row[k], col[k]);
    }
#pragma unroll
    for (int k = 0; k < kTake; ++k) {
      if (i + k * apart >= pieces) break;
      float u[VEC];
      piece[k].update(a, p, row[k], col[k], true, u);
#pragma unroll
      for (int v = 0; v < VEC; ++v) s = fma((double)u[v], (double)u[v], s);
    }
  }
  __shared__ double warps[8];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < 8; ++w) t += warps[w];
    a.part[(int64_t)p * a.blocks + blockIdx.x] = t;
  }
}

// 1 / (|U| + eps) from the sum of squares, as a power of two and a factor of like size, which a value is multiplied by one after the
// other: |U| may be that of the least subnormal or 2^31 times the largest value, whose inverse leaves fp32.  0 for a zero matrix, NaN
// where a value is not finite.
struct Inverse {
  float power, factor;
  __device__ __forceinline__ float times(float u) const { return u * power * factor; }
};
__device__ __forceinline__ Inverse inverse_of(double sum, float eps) {
  const double t = sqrt(sum) + (double)eps;
  if (!(t > 0.0 && t < 1e300)) return {1.f, t == 0.0 ? 0.f : __int_as_float(0x7FC00000)};
  const int half = -ilogb(t) / 2;
  return {ldexpf(1.f, half), (float)(ldexp(1.0, -half) / t)};
}
__device__ __forceinline__ Inverse inverse_norm(const Prep& a, int p) {
  __shared__ Inverse s;
  if (threadIdx.x < 32) {
    const Inverse t = inverse_of(warp_sum_fixed(a.part + (int64_t)p * a.blocks, a.blocks), a.d.eps);
    if (threadIdx.x == 0) s = t;
  }
  __syncthreads();
  return s;
}

// X as fp16, transposed where the matrix is tall: tiles of 64 x 64 through shared memory.  Without steps: out itself.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) scale_kernel(const __grid_constant__ Prep a) {
  pdl_wait();
  pdl_launch_dependents();
  const int p = blockIdx.z, r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;       // of the matrix as given
  Inverse inv = {};
  __shared__ float tile[64][65];
  constexpr int kPieces = 64 * (64 / VEC) / 256, kTake = kPieces < 8 ? kPieces : 8;
#pragma unroll 1
  for (int k0 = 0; k0 < kPieces; k0 += kTake) {
    Piece<T, VEC> piece[kTake];
#pragma unroll
    for (int k = 0; k < kTake; ++k) {
      const int i = threadIdx.x + (k0 + k) * 256, row = i / (64 / VEC), col = i % (64 / VEC) * VEC;
      if (r0 + row < a.d.m && c0 + col < a.d.n) piece[k].load(a, p, r0 + row, c0 + col);
    }
    if (k0 == 0) inv = inverse_norm(a, p);         // behind the first pieces' loads
#pragma unroll
    for (int k = 0; k < kTake; ++k) {
      const int i = threadIdx.x + (k0 + k) * 256, row = i / (64 / VEC), col = i % (64 / VEC) * VEC;
      float u[VEC] = {};
      if (r0 + row < a.d.m && c0 + col < a.d.n) piece[k].update(a, p, r0 + row, c0 + col, false, u);
#pragma unroll
      for (int v = 0; v < VEC; ++v) tile[row][col + v] = inv.times(u[v]);
    }
  }
  __syncthreads();
  if (a.d.steps == 0) {
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.d.out.data) + p * a.d.out.stride;
    for (int i = threadIdx.x; i < 64 * 64; i += 256) {
      const int row = i / 64, col = i % 64;
      if (r0 + row < a.d.m && c0 + col < a.d.n) out[(r0 + row) * a.d.out.ld + c0 + col] = __float2bfloat16_rn(a.d.scale * tile[row][col]);
    }
    return;
  }
  for (int i = threadIdx.x; i < 64 * 8; i += 256) {
    const int row = i / 8, col = i % 8 * 8;                                  // of X within its tile
    const int xr = (a.tall ? c0 : r0) + row, xc = (a.tall ? r0 : c0) + col;
    if (xr >= a.r || xc >= a.ld) continue;
    uint4 hi, lo;
    __half2 *h = reinterpret_cast<__half2*>(&hi), *l = reinterpret_cast<__half2*>(&lo);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float f0 = kScale * (a.tall ? tile[col + 2 * v][row] : tile[row][col + 2 * v]);
      const float f1 = kScale * (a.tall ? tile[col + 2 * v + 1][row] : tile[row][col + 2 * v + 1]);
      h[v] = __floats2half2_rn(f0, f1);
      l[v] = __floats2half2_rn(f0 - __low2float(h[v]), f1 - __high2float(h[v]));
    }
    *reinterpret_cast<uint4*>(a.x + p * a.stride + xr * a.ld + xc) = hi;
    if (a.lo) *reinterpret_cast<uint4*>(a.lo + p * a.stride + xr * a.ld + xc) = lo;
  }
}

// ------------------------------------------------------------------------------------------------ products
struct Product {
  int M, N, K, batch;
  int b_mn;                  // B is stored [K][N] (else [N][K])
  int symmetric;             // square: tiles on and above the diagonal, stored twice
  int split;                 // blocks that share a tile's contraction (1: none do); the last of them to finish adds up
  float* partial;            // split: [tiles][split][columns of a tile][128 rows]
  uint32_t* done;            // split: blocks of a tile that have finished, 0 between products
  int add;                   // C = alpha acc + beta D + diag I
  const __half* rows;        // NULL, or beta counts times a value for every row: rows[batch][row (rows_ld)]
  int64_t rows_ld, rows_stride;
  int twofold;               // C = A B + A D, D of B's layout (instead of an added tile)
  int rest;                  // what C is rounded by is stored too
  float alpha, beta, diag;
  __nv_bfloat16* out;        // last product: bf16 rows instead of C, times scale
  int64_t out_ld, out_stride;
  int out_transposed, out_wide;
  float scale;

  __device__ __forceinline__ int nk1() const { return (K + BK - 1) / BK; }
  __device__ __forceinline__ int nk() const { return twofold ? 2 * nk1() : nk1(); }
};

struct TileAt {
  int z, m0, n0;
  int part, k0, k1;          // of the contraction's slices, [k0, k1)
  int number;                // of the tile, without its parts
};
// Tile number t: all of a row of tiles, or those from the diagonal on (of 64 columns: both halves of each square).
template <typename F>
__device__ __forceinline__ TileAt tile_of(const Product& p, int t, int nt, int per) {
  TileAt q;
  const int nk = p.nk();
  q.part = 0, q.k0 = 0, q.k1 = nk;
  if (p.split > 1) {
    q.part = t % p.split;
    t /= p.split;
    const int share = (nk + p.split - 1) / p.split;
    q.k0 = q.part * share;
    q.k1 = min(nk, q.k0 + share);
  }
  q.number = t;
  q.z = t / per;
  t -= q.z * per;
  int i = 0;
  if (p.symmetric) {
    constexpr int kHalves = F::kM / F::kN;
    const int half = t % kHalves;
    t /= kHalves;
    while (t >= nt - i) t -= nt - i++;
    q.m0 = i * F::kM;
    q.n0 = (i + t) * F::kM + half * F::kN;
  } else {
    q.m0 = t / nt * F::kM;
    q.n0 = t % nt * F::kN;
  }
  return q;
}

__device__ __forceinline__ void epi_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kEpiWarps) : "memory"); }

// What all of the epilogue's threads say: after a wait that ran out for some of them all leave together, none at a barrier alone.
__device__ __forceinline__ bool epi_all(bool ok) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.red.and.pred q, 1, %2, p;\n selp.u32 %0, 1, 0, q;\n}"
      : "=r"(r)
      : "r"((uint32_t)ok), "n"(32 * kEpiWarps)
      : "memory");
  return r;
}

// 16 bytes `unit` of row `row` of a [128][256 bytes] buffer; a warp that writes a unit of 32 rows, or reads a row, meets no bank twice
__device__ __forceinline__ int out_at(int row, int unit) { return row * 256 + ((unit ^ (row & 15)) << 4); }

__device__ __forceinline__ uint32_t half_pair(float lo, float hi) {
  __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&h);
}

// What a pair is rounded by.
__device__ __forceinline__ uint32_t rest_pair(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return half_pair(lo - __low2float(h), hi - __high2float(h));
}

// PAIR: a cluster of two CTAs computes a 256 x 256 tile, each fetching its half of the rows of A and of B; the first one's issuer
// drives both tensor cores (cta_group::2).  Its barriers count both CTAs' copies and epilogues.
template <bool PAIR, int BN>
__global__ void __launch_bounds__(kThreads, 1)
product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const __grid_constant__ CUtensorMap map_c, const __grid_constant__ CUtensorMap map_d, const __grid_constant__ CUtensorMap map_rest,
               const __grid_constant__ Product p) {
  using F = Form<PAIR, BN>;
  constexpr int kStages = F::kStages, kStageBytes = F::kStageBytes, kHalves = PAIR ? 2 : 1;
  constexpr uint32_t kTmemCols = 2 * F::kN;      // two accumulators
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* buf = smem + kStages * kStageBytes;   // 128 x BN: D in, C out; boxes of [128][64]
  uint8_t* mirror = buf + kTileBytes;            // C transposed; or its rest, laid out as C
  __shared__ uint64_t full_bar[kStages], empty_bar[kStages], acc_full[2], acc_empty[2], in_full, in_free;
  __shared__ uint32_t tmem_base_s;
  __shared__ int abort_s, last_s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = PAIR ? (int)cluster_rank() : 0;
  const int mt = (p.M + F::kM - 1) / F::kM, nt = p.symmetric ? mt : (p.N + F::kN - 1) / F::kN;
  const int per = p.symmetric ? mt * (mt + 1) / 2 * (F::kM / F::kN) : mt * nt;
  const int n_tiles = per * p.batch * p.split, nk1 = p.nk1();
  const int first = PAIR ? blockIdx.x >> 1 : blockIdx.x, stride = PAIR ? gridDim.x >> 1 : gridDim.x;
  uint32_t* status = &g_status;
  if (threadIdx.x == 0) {
    abort_s = 0;
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&acc_full[b], 1);
      mbar_init(&acc_empty[b], (PAIR ? 2 : 1) * kEpiWarps);
    }
    mbar_init(&in_full, 1);
    mbar_init(&in_free, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_c) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_d) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_rest) : "memory");
  }
  if (warp == 1) {
    if (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"(kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"(kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (PAIR) cluster_sync_all();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = tmem_base_s;
  volatile int* abort_flag = &abort_s;
  pdl_wait();
  pdl_launch_dependents();

  if (warp == 0 && lane == 0) {
    // ---------------------------------------------------------------- operands
    uint32_t it = 0;
    bool ok = true;
    for (int t = first; t < n_tiles && ok; t += stride) {
      const TileAt q = tile_of<F>(p, t, nt, per);
      const int m0 = q.m0 + rank * 128, n0 = q.n0 + rank * 128;      // (of B a CTA of a pair fetches half)
      for (int kt = q.k0; kt < q.k1; ++kt, ++it) {
        const int s = it % kStages;
        ok = mbar_wait(&empty_bar[s], ((it / kStages) & 1) ^ 1, abort_flag, status);
        if (!ok) break;
        uint8_t* sa = smem + s * kStageBytes;
        uint8_t* sb = sa + BM * BK * 2;
        const int k0 = (kt < nk1 ? kt : kt - nk1) * BK;
        const CUtensorMap* from_b = kt < nk1 ? &map_b : &map_d;
        if (rank == 0) mbar_expect_tx(&full_bar[s], (PAIR ? 2 : 1) * kStageBytes);
        const uint32_t bar = PAIR ? map_to_rank(smem_u32(&full_bar[s]), 0) : 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int bx = p.b_mn ? n0 + 64 * j : k0, by = p.b_mn ? k0 : n0 + 64 * j;
          if (PAIR) tma_load_3d_pair(sa + j * kBoxBytes, &map_a, bar, k0, m0 + 64 * j, q.z);
          else tma_load_3d(sa + j * kBoxBytes, &map_a, &full_bar[s], k0, m0 + 64 * j, q.z);
          if (j >= F::kBoxesB) break;
          if (PAIR) tma_load_3d_pair(sb + j * kBoxBytes, from_b, bar, bx, by, q.z);
          else tma_load_3d(sb + j * kBoxBytes, from_b, &full_bar[s], bx, by, q.z);
        }
      }
    }
    if (!ok && rank == 0) {       // copies in flight land before the CTAs leave (the other CTA waits at the last cluster barrier)
      const long long t0 = clock64();
      for (uint32_t j = it > kStages ? it - kStages : 0; j < it; ++j)
        while (!mbar_try(&full_bar[j % kStages], (j / kStages) & 1) && clock64() - t0 < kWaitBudgetCycles / 4) {
        }
    }
  } else if (warp == 1 && lane == 0 && rank == 0) {
    // ---------------------------------------------------------------- products
    const uint32_t idesc = (1u << 4) | ((uint32_t)(p.b_mn ? 1 : 0) << 16) | ((uint32_t)(F::kN >> 3) << 17) | ((uint32_t)(F::kM >> 4) << 24);
    uint32_t it = 0;
    int local = 0;
    bool ok = true;
    for (int t = first; t < n_tiles && ok; t += stride, ++local) {
      const int b = local & 1;
      ok = mbar_wait(&acc_empty[b], ((local >> 1) & 1) ^ 1, abort_flag, status);
      if (!ok) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t tacc = tmem_base + (uint32_t)(b * F::kN);
      const TileAt q = tile_of<F>(p, t, nt, per);
      for (int kt = q.k0; kt < q.k1; ++kt, ++it) {
        const int s = it % kStages;
        ok = mbar_wait(&full_bar[s], (it / kStages) & 1, abort_flag, status);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t sa = smem_u32(smem + s * kStageBytes), sb = sa + BM * BK * 2;
#pragma unroll
        for (int k = 0; k < BK / 16; ++k) {
          const uint64_t da = smem_desc(sa + k * 32, 16, 1024);
          const uint64_t db = p.b_mn ? smem_desc(sb + k * 2048, 8192, 1024) : smem_desc(sb + k * 32, 16, 1024);
          if (PAIR) mma_f16_pair(tacc, da, db, idesc, kt > q.k0 || k > 0 ? 1u : 0u);
          else mma_f16(tacc, da, db, idesc, kt > q.k0 || k > 0 ? 1u : 0u);
        }
        if (PAIR) {
          mma_commit_pair(map_to_rank(smem_u32(&empty_bar[s]), 0));
          mma_commit_pair(map_to_rank(smem_u32(&empty_bar[s]), 1));
        } else {
          mma_commit(&empty_bar[s]);
        }
      }
      if (!ok) break;
      if (PAIR) {
        mma_commit_pair(map_to_rank(smem_u32(&acc_full[b]), 0));
        mma_commit_pair(map_to_rank(smem_u32(&acc_full[b]), 1));
      } else {
        mma_commit(&acc_full[b]);
      }
    }
  } else if (warp == 2 + kEpiWarps && lane == 0 && p.add) {
    // ---------------------------------------------------------------- the tiles that are added
    uint32_t use = 0;
    bool ok = true;
    for (int t = first; t < n_tiles && ok; t += stride) {
      const TileAt q = tile_of<F>(p, t, nt, per);
      const int m0 = q.m0 + rank * 128;
      for (int half = 0; half < kHalves; ++half) {
        const int n0 = q.n0 + half * 128;
        if (n0 >= p.N || m0 >= p.M) break;
        ok = mbar_wait(&in_free, (use & 1) ^ 1, abort_flag, status);
        if (!ok) break;
        ++use;
        mbar_expect_tx(&in_full, BN / 64 * 2 * kBoxBytes);
#pragma unroll
        for (int j = 0; j < BN / 64; ++j) tma_load_3d(buf + j * 2 * kBoxBytes, &map_d, &in_full, n0 + 64 * j, m0, q.z);
      }
    }
    if (!ok && use > 0) {
      const long long t0 = clock64();
      while (!mbar_try(&in_full, (use - 1) & 1) && clock64() - t0 < kWaitBudgetCycles / 4) {
      }
    }
  } else if (warp >= 2 && warp < 2 + kEpiWarps) {
    // ---------------------------------------------------------------- epilogue: this CTA's 128 rows, 128 columns at a time
    constexpr int kEach = BN / 64;                 // pieces of 32 columns of a warp
    const int q4 = warp & 3, part = (warp - 2) >> 2, row = q4 * 32 + lane;
    const bool leader = threadIdx.x == 64;
    int local = 0;
    uint32_t use = 0;
    bool ok = true;
    for (int t = first; t < n_tiles && ok; t += stride, ++local) {
      const TileAt q = tile_of<F>(p, t, nt, per);
      const int b = local & 1, m0 = q.m0 + rank * 128;
      const bool twice = p.symmetric && q.n0 >= q.m0 + F::kM;
      float beta = p.beta;
      if (p.rows) beta *= m0 + row < p.M ? __half2float(p.rows[q.z * p.rows_stride + (m0 + row) * p.rows_ld]) : 0.f;
      ok = mbar_wait(&acc_full[b], (local >> 1) & 1, abort_flag, status);
#pragma unroll 1
      for (int half = 0; half < kHalves; ++half) {
        const int n0 = q.n0 + half * 128;
        const bool there = n0 < p.N && m0 < p.M;
        if (there && p.add && ok) ok = mbar_wait(&in_full, use++ & 1, abort_flag, status);
        ok = epi_all(ok);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t tacc = tmem_base + ((uint32_t)(q4 * 32) << 16) + (uint32_t)(b * F::kN + half * 128);
        float* partial = nullptr;                                // of the tile, where its contraction is shared
        if (!PAIR && p.split > 1) {
          partial = p.partial + (int64_t)q.number * p.split * BM * BN + row;
#pragma unroll 1
          for (int c = kEach * part; c < kEach * part + kEach; ++c) {
            if (n0 + c * 32 >= p.N) break;
            uint32_t r[32];
            tmem_ld32(tacc + (uint32_t)(c * 32), r);
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
            float* to = partial + ((int64_t)q.part * BN + c * 32) * BM;
#pragma unroll
            for (int j = 0; j < 32; ++j) __stcg(to + j * BM, __uint_as_float(r[j]));
          }
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(&acc_empty[b]);
          __threadfence();
          epi_barrier();
          if (leader) last_s = atomicAdd(p.done + q.number, 1u) == (uint32_t)p.split - 1;
          epi_barrier();
          if (!last_s) continue;
          __threadfence();
          if (leader) p.done[q.number] = 0;
        }
#pragma unroll 1
        for (int c = kEach * part; c < kEach * part + kEach; ++c) {
          if (!there || n0 + c * 32 >= p.N) break;
          uint32_t r[32];
          if (partial) {                                         // the parts in order
            float sum[32] = {};
#pragma unroll 1
            for (int k = 0; k < p.split; k += 2) {               // two of them fetched at a time
              const float *from = partial + ((int64_t)k * BN + c * 32) * BM, *then = k + 1 < p.split ? from + (int64_t)BN * BM : nullptr;
              float f[32], g[32];
#pragma unroll
              for (int j = 0; j < 32; ++j) f[j] = __ldcg(from + j * BM);
#pragma unroll
              for (int j = 0; j < 32; ++j) g[j] = then ? __ldcg(then + j * BM) : 0.f;
#pragma unroll
              for (int j = 0; j < 32; ++j) sum[j] = (sum[j] + f[j]) + g[j];
            }
#pragma unroll
            for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(sum[j]);
          } else {
            tmem_ld32(tacc + (uint32_t)(c * 32), r);
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          }
          uint8_t* box = buf + (c >> 1) * 2 * kBoxBytes;
          const int u0 = (c & 1) * 4;
          float v[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = p.alpha * __uint_as_float(r[j]);
          if (p.add) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const uint4 w = *reinterpret_cast<const uint4*>(box + swz(row, u0 + u));
              const __half2* h = reinterpret_cast<const __half2*>(&w);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float2 f = __half22float2(h[j]);
                v[8 * u + 2 * j] = fmaf(beta, f.x, v[8 * u + 2 * j]);
                v[8 * u + 2 * j + 1] = fmaf(beta, f.y, v[8 * u + 2 * j + 1]);
              }
            }
          }
          if (p.add && !p.rows) {
            const int d = m0 + row - n0 - c * 32;                // the diagonal's column in this piece
            // selects: every lane has its own j, and 32 branches in turn made this the slowest warp (8 x 256 x 256: 118 us for 113, with
            // squares)
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = fmaf(j == d ? 1.f : 0.f, p.diag, v[j]);
          }
          if (p.out) {
            const int gr = m0 + row, gc = n0 + c * 32;
            if (gr < p.M) {
              __nv_bfloat16* o = p.out + q.z * p.out_stride;
              if (p.out_transposed) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                  if (gc + j < p.N) o[(gc + j) * p.out_ld + gr] = __float2bfloat16_rn(v[j] * p.scale);
              } else if (p.out_wide) {
#pragma unroll
                for (int u = 0; u < 4; ++u)
                  if (gc + 8 * u < p.N) {
                    float f[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] = v[8 * u + j] * p.scale;
                    Pack<__nv_bfloat16, 8> k;
                    k.set(f);
                    k.store(o + gr * p.out_ld + gc + 8 * u);
                  }
              }
            }
            if (!p.out_transposed && !p.out_wide) {              // through the buffer: 16 columns a row, turned by the row
#pragma unroll
              for (int u = 0; u < 4; ++u)
                *reinterpret_cast<uint4*>(buf + out_at(row, c * 4 + u)) =
                    make_uint4(bf16_pair(v[8 * u] * p.scale, v[8 * u + 1] * p.scale), bf16_pair(v[8 * u + 2] * p.scale, v[8 * u + 3] * p.scale),
                               bf16_pair(v[8 * u + 4] * p.scale, v[8 * u + 5] * p.scale), bf16_pair(v[8 * u + 6] * p.scale, v[8 * u + 7] * p.scale));
            }
            continue;
          }
#pragma unroll
          for (int u = 0; u < 4; ++u)
            *reinterpret_cast<uint4*>(box + swz(row, u0 + u)) =
                make_uint4(half_pair(v[8 * u], v[8 * u + 1]), half_pair(v[8 * u + 2], v[8 * u + 3]),
                           half_pair(v[8 * u + 4], v[8 * u + 5]), half_pair(v[8 * u + 6], v[8 * u + 7]));
          if (p.rest) {
            uint8_t* rbox = mirror + (c >> 1) * 2 * kBoxBytes;
#pragma unroll
            for (int u = 0; u < 4; ++u)
              *reinterpret_cast<uint4*>(rbox + swz(row, u0 + u)) =
                  make_uint4(rest_pair(v[8 * u], v[8 * u + 1]), rest_pair(v[8 * u + 2], v[8 * u + 3]),
                             rest_pair(v[8 * u + 4], v[8 * u + 5]), rest_pair(v[8 * u + 6], v[8 * u + 7]));
          }
          if (twice) {
            uint8_t* mbox = mirror + (row >> 6) * (BN * 128);
#pragma unroll
            for (int j = 0; j < 32; ++j)
              *reinterpret_cast<__half*>(mbox + swz(c * 32 + j, (row & 63) >> 3) + (row & 7) * 2) = __float2half_rn(v[j]);
          }
        }
        if (half == kHalves - 1 && !partial) {                   // the accumulator has been read
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            if (PAIR) mbar_arrive_cluster(map_to_rank(smem_u32(&acc_empty[b]), 0));
            else mbar_arrive(&acc_empty[b]);
          }
        }
        if (there && p.out && !p.out_transposed && !p.out_wide) {
          // a warp a row, 32 neighbouring columns at a time (a lane a row, 2 bytes each, took 16 us of a tile)
          epi_barrier();
          for (int k = warp - 2; k < BM && m0 + k < p.M; k += kEpiWarps) {
            __nv_bfloat16* o = p.out + q.z * p.out_stride + (m0 + k) * p.out_ld + n0;
#pragma unroll
            for (int col = lane; col < BN; col += 32)
              if (n0 + col < p.N) o[col] = *reinterpret_cast<const __nv_bfloat16*>(buf + out_at(k, col >> 3) + (col & 7) * 2);
          }
          epi_barrier();
        }
        if (!there || p.out) continue;                           // neither an added tile nor a stored one
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        epi_barrier();
        if (leader) {
          // boxes of BN rows: of C's 128 rows one or two
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            if (BN == 64 && m0 + 64 * j < p.M) tma_store_3d(buf + j * kBoxBytes, &map_c, n0, m0 + 64 * j, q.z);
            if (BN == 128 && n0 + 64 * j < p.N) tma_store_3d(buf + j * 2 * kBoxBytes, &map_c, n0 + 64 * j, m0, q.z);
            if (BN == 64 && p.rest && m0 + 64 * j < p.M) tma_store_3d(mirror + j * kBoxBytes, &map_rest, n0, m0 + 64 * j, q.z);
            if (BN == 128 && p.rest && n0 + 64 * j < p.N) tma_store_3d(mirror + j * 2 * kBoxBytes, &map_rest, n0 + 64 * j, m0, q.z);
            if (twice && m0 + 64 * j < p.M) tma_store_3d(mirror + j * (BN * 128), &map_c, m0 + 64 * j, n0, q.z);
          }
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          if (p.add) mbar_arrive(&in_free);
        }
        epi_barrier();
      }
    }
    if (leader) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (PAIR) cluster_sync_all();
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

// ------------------------------------------------------------------------------------------------ small matrices
// X of at most 128 x 256 (and G, Q): one block a matrix does everything in one launch.  Operands stay in shared memory as the tensor
// cores read them: 64 columns a box, 128 rows of 128 bytes, 128-byte swizzle.  The same box serves as rows of a K-major operand (G = X
// X^T) and as the K index of an MN-major one (Q X).  A product is issued by one thread, everybody waits for it and takes part
// in the epilogue; what bounds it is that chain of latencies, about 1 us a product.
constexpr int kSmallRows = 128, kSmallCols = 256, kSmallThreads = 512, kSmallParts = kSmallThreads / 128;
constexpr int kSmallBox = kSmallRows * 128;

__device__ __forceinline__ uint32_t two(__half a, __half b) { return (uint32_t)__half_as_ushort(a) | (uint32_t)__half_as_ushort(b) << 16; }
__device__ __forceinline__ int small_at(int row, int col) { return (col >> 6) * kSmallBox + (int)swz(row, (col & 63) >> 3) + (col & 7) * 2; }

template <typename T, int VEC>
__global__ void __launch_bounds__(kSmallThreads, 1) small_kernel(const __grid_constant__ Prep a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sx = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int boxes = (a.n + 63) / 64;
  uint8_t *slo = sx + boxes * kSmallBox, *sg = slo + boxes * kSmallBox, *sq = sg + 2 * kSmallBox;
  __shared__ uint64_t bar;
  __shared__ uint32_t tmem_s;
  __shared__ int abort_s;
  __shared__ double warp_sums[kSmallThreads / 32];
  const int p = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr uint32_t kTmemCols = 512;            // 128 of G and Q, 256 of X
  if (threadIdx.x == 0) {
    abort_s = 0;
    mbar_init(&bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  for (int i = threadIdx.x; i < (2 * boxes + 4) * kSmallBox / 16; i += kSmallThreads) reinterpret_cast<uint4*>(sx)[i] = make_uint4(0, 0, 0, 0);
  pdl_wait();
  pdl_launch_dependents();
  // momentum and norm; the update stays in registers
  constexpr int kMost = kSmallRows * kSmallCols / VEC / kSmallThreads;
  const int per = a.d.n / VEC, pieces = a.d.m * per;
  float u[kMost][VEC];
  double sum = 0.0;
  constexpr int kTake = 8;                       // pieces fetched before the first is used
#pragma unroll
  for (int k0 = 0; k0 < kMost; k0 += kTake) {
    Piece<T, VEC> piece[kTake];
#pragma unroll
    for (int k = 0; k < kTake; ++k) {
      const int i = threadIdx.x + (k0 + k) * kSmallThreads;
      if (i < pieces) piece[k].load(a, p, i / per, i % per * VEC);
    }
#pragma unroll
    for (int k = 0; k < kTake; ++k) {
      const int i = threadIdx.x + (k0 + k) * kSmallThreads;
#pragma unroll
      for (int v = 0; v < VEC; ++v) u[k0 + k][v] = 0.f;
      if (i < pieces) piece[k].update(a, p, i / per, i % per * VEC, true, u[k0 + k]);
    }
  }
#pragma unroll
  for (int k = 0; k < kMost; ++k)
#pragma unroll
    for (int v = 0; v < VEC; ++v) sum = fma((double)u[k][v], (double)u[k][v], sum);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if (lane == 0) warp_sums[warp] = sum;
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_s;
  double total = 0.0;
  for (int w = 0; w < kSmallThreads / 32; ++w) total += warp_sums[w];
  Inverse inv = inverse_of(total, a.d.eps);
  inv.factor *= kScale;
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
    const int i = threadIdx.x + k * kSmallThreads;
    if (i >= pieces) break;
    const int row = i / per, col = i % per * VEC;
    __half hi[VEC], lo[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const float f = inv.times(u[k][v]);
      hi[v] = __float2half_rn(f);
      lo[v] = __float2half_rn(f - __half2float(hi[v]));
    }
    if (VEC == 4 && !a.tall) {
      *reinterpret_cast<uint2*>(sx + small_at(row, col)) = make_uint2(two(hi[0], hi[VEC > 1]), two(hi[VEC / 2], hi[VEC - 1]));
      *reinterpret_cast<uint2*>(slo + small_at(row, col)) = make_uint2(two(lo[0], lo[VEC > 1]), two(lo[VEC / 2], lo[VEC - 1]));
    } else {
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const int at = a.tall ? small_at(col + v, row) : small_at(row, col + v);
        *reinterpret_cast<__half*>(sx + at) = hi[v];
        *reinterpret_cast<__half*>(slo + at) = lo[v];
      }
    }
  }
  // the products' shapes, padded with the zeros above to what an instruction takes
  const int rows16 = (a.r + 15) / 16, cols16 = (a.n + 15) / 16;
  const uint32_t idesc = (1u << 4) | ((uint32_t)(rows16 * 2) << 17) | ((uint32_t)(kSmallRows >> 4) << 24);
  const uint32_t idesc_x = (1u << 4) | (1u << 16) | ((uint32_t)(cols16 * 2) << 17) | ((uint32_t)(kSmallRows >> 4) << 24);
  const uint32_t ax = smem_u32(sx), alo = smem_u32(slo), ag = smem_u32(sg), aq = smem_u32(sq);
  const int q4 = warp & 3, part = warp >> 2, row = q4 * 32 + lane;
  const uint32_t tg = tmem, tx = tmem + 128, quarter = (uint32_t)(q4 * 32) << 16;
  uint32_t phase = 0;
  // shared memory and tensor memory as everybody has left them -> one thread's products -> everybody
  auto product = [&](auto issue) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      issue();
      mma_commit(&bar);
    }
    const bool ok = mbar_wait(&bar, phase, &abort_s, &g_status);
    phase ^= 1;
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    return ok;
  };
  bool ok = true;
  for (int step = 0; step < a.d.steps; ++step) {
    ok = product([&] {
      for (int k = 0; k < cols16; ++k) {
        const uint64_t d = smem_desc(ax + (k >> 2) * kSmallBox + (k & 3) * 32, 16, 1024);
        mma_f16(tg, d, d, idesc, k > 0);
      }
    });
    if (__syncthreads_or(!ok)) break;
    for (int c = part * 32; c < rows16 * 16; c += 32 * kSmallParts) {
      uint32_t r[32];
      tmem_ld32(tg + quarter + c, r);
      asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        uint4 w;
        w.x = half_pair(__uint_as_float(r[8 * u]) * (1 / kScale), __uint_as_float(r[8 * u + 1]) * (1 / kScale));
        w.y = half_pair(__uint_as_float(r[8 * u + 2]) * (1 / kScale), __uint_as_float(r[8 * u + 3]) * (1 / kScale));
        w.z = half_pair(__uint_as_float(r[8 * u + 4]) * (1 / kScale), __uint_as_float(r[8 * u + 5]) * (1 / kScale));
        w.w = half_pair(__uint_as_float(r[8 * u + 6]) * (1 / kScale), __uint_as_float(r[8 * u + 7]) * (1 / kScale));
        if (c + 8 * u < rows16 * 16) *reinterpret_cast<uint4*>(sg + small_at(row, c + 8 * u)) = w;
      }
    }
    ok = product([&] {
      for (int k = 0; k < rows16; ++k) {
        const uint64_t d = smem_desc(ag + (k >> 2) * kSmallBox + (k & 3) * 32, 16, 1024);
        mma_f16(tg, d, d, idesc, k > 0);
      }
    });
    if (__syncthreads_or(!ok)) break;
    for (int c = part * 32; c < rows16 * 16; c += 32 * kSmallParts) {
      uint32_t r[32];
      tmem_ld32(tg + quarter + c, r);
      asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (c + 8 * u >= rows16 * 16) continue;
        const uint4 g = *reinterpret_cast<const uint4*>(sg + small_at(row, c + 8 * u));
        const __half2* h = reinterpret_cast<const __half2*>(&g);
        float v[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = __half22float2(h[j]);
          v[2 * j] = fmaf(a.d.b, f.x, a.d.c * (1 / kScale) * __uint_as_float(r[8 * u + 2 * j]));
          v[2 * j + 1] = fmaf(a.d.b, f.y, a.d.c * (1 / kScale) * __uint_as_float(r[8 * u + 2 * j + 1]));
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(c + 8 * u + j == row && row < a.r ? 1.f : 0.f, a.d.a * kScale, v[j]);
        *reinterpret_cast<uint4*>(sq + small_at(row, c + 8 * u)) =
            make_uint4(half_pair(v[0], v[1]), half_pair(v[2], v[3]), half_pair(v[4], v[5]), half_pair(v[6], v[7]));
      }
    }
    ok = product([&] {
      for (int twice = 0; twice < (step + 1 < a.d.steps ? 2 : 1); ++twice)
        for (int k = 0; k < rows16; ++k) {
          const uint64_t da = smem_desc(aq + (k >> 2) * kSmallBox + (k & 3) * 32, 16, 1024);
          mma_f16(tx, da, smem_desc((twice ? alo : ax) + k * 2048, kSmallBox, 1024), idesc_x, (k | twice) > 0);
        }
    });
    if (__syncthreads_or(!ok)) break;
    const bool last = step + 1 == a.d.steps;
    const float down = last ? a.d.scale / kScale / kScale : 1 / kScale;
    for (int c = part * 32; c < cols16 * 16; c += 32 * kSmallParts) {
      uint32_t r[32];
      tmem_ld32(tx + quarter + c, r);
      asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
      if (last) {
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(a.d.out.data) + p * a.d.out.stride;
        if (row < a.r && !a.tall && a.out_wide) {
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (c + 8 * u < a.n) {
              float f[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(r[8 * u + j]) * down;
              Pack<__nv_bfloat16, 8> k;
              k.set(f);
              k.store(o + row * a.d.out.ld + c + 8 * u);
            }
        } else if (a.tall) {
          if (row < a.r) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (c + j < a.n) o[(c + j) * a.d.out.ld + row] = __float2bfloat16_rn(__uint_as_float(r[j]) * down);
          }
        } else if (!a.out_wide) {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            uint4 w;
            w.x = bf16_pair(__uint_as_float(r[8 * u]) * down, __uint_as_float(r[8 * u + 1]) * down);
            w.y = bf16_pair(__uint_as_float(r[8 * u + 2]) * down, __uint_as_float(r[8 * u + 3]) * down);
            w.z = bf16_pair(__uint_as_float(r[8 * u + 4]) * down, __uint_as_float(r[8 * u + 5]) * down);
            w.w = bf16_pair(__uint_as_float(r[8 * u + 6]) * down, __uint_as_float(r[8 * u + 7]) * down);
            if (c + 8 * u < cols16 * 16) *reinterpret_cast<uint4*>(sx + small_at(row, c + 8 * u)) = w;
          }
        }
        continue;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (c + 8 * u >= cols16 * 16) continue;
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(r[8 * u + j]) * down;
        *reinterpret_cast<uint4*>(sx + small_at(row, c + 8 * u)) =
            make_uint4(half_pair(f[0], f[1]), half_pair(f[2], f[3]), half_pair(f[4], f[5]), half_pair(f[6], f[7]));
        if (step + 2 < a.d.steps)
          *reinterpret_cast<uint4*>(slo + small_at(row, c + 8 * u)) =
              make_uint4(rest_pair(f[0], f[1]), rest_pair(f[2], f[3]), rest_pair(f[4], f[5]), rest_pair(f[6], f[7]));
      }
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == 0) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
  if (ok && !a.tall && !a.out_wide) {            // from X's place, a warp a row
    for (int k = warp; k < a.r; k += kSmallThreads / 32) {
      __nv_bfloat16* o = static_cast<__nv_bfloat16*>(a.d.out.data) + p * a.d.out.stride + k * a.d.out.ld;
      for (int col = lane; col < a.n; col += 32) o[col] = *reinterpret_cast<const __nv_bfloat16*>(sx + small_at(k, col));
    }
  }
}
template <typename T, int VEC>
cudaError_t launch_small(const Prep& a, cudaStream_t s) {
  static OncePerDevice attr;
  const auto bytes = [](int n) { return (2 * ((n + 63) / 64) + 4) * kSmallBox + 1024; };
  if (!attr.here()) {
    const cudaError_t e = cudaFuncSetAttribute(small_kernel<T, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes(kSmallCols));
    if (e != cudaSuccess) return e;
    attr.here() = true;
  }
  return launch_pdl(small_kernel<T, VEC>, dim3(a.d.P), dim3(kSmallThreads), (size_t)bytes(a.n), s, a);
}

// ------------------------------------------------------------------------------------------------ host
lsgd_status check_ortho(const lsgd_ortho_desc* d) {
  if (!d || d->struct_size != sizeof(lsgd_ortho_desc)) return LSGD_ERR_INVALID_ARG;
  if (d->P < 1 || d->m < 1 || d->n < 1 || d->steps < 0) return LSGD_ERR_INVALID_ARG;
  if (d->P > 65535 || d->m > 65536 || d->n > 65536 || d->steps > 32) return LSGD_ERR_UNSUPPORTED;
  if ((int64_t)d->m * d->n >= int64_t(1) << 31) return LSGD_ERR_TOO_LARGE;
  if (d->grad_dtype < LSGD_F32 || d->grad_dtype > LSGD_BF16) return LSGD_ERR_INVALID_ARG;
  if (!(fabsf(d->a) <= 16.f) || !(fabsf(d->b) <= 16.f) || !(fabsf(d->c) <= 16.f)) return LSGD_ERR_INVALID_ARG;
  if (!(d->mu >= 0.f && d->mu < 1.f) || !(d->eps >= 0.f && d->eps < 1e30f) || !(d->scale - d->scale == 0.f)) return LSGD_ERR_INVALID_ARG;
  if (!d->grad.data || !d->out.data) return LSGD_ERR_INVALID_ARG;
  lsgd_status st;
  if ((st = check_rows(d->grad, d->P, d->m, d->n, elem_bytes(d->grad_dtype), false)) != LSGD_OK) return st;
  if (d->momentum.data && (st = check_rows(d->momentum, d->P, d->m, d->n, 4, true)) != LSGD_OK) return st;
  if ((st = check_rows(d->out, d->P, d->m, d->n, 2, true)) != LSGD_OK) return st;
  const Extent ins[] = {extent(d->grad, d->P, d->m, d->n, elem_bytes(d->grad_dtype))};
  const Extent outs[] = {extent(d->out, d->P, d->m, d->n, 2), extent(d->momentum, d->P, d->m, d->n, 4)};
  return all_apart(outs, 2, ins, 1) ? LSGD_OK : LSGD_ERR_INVALID_ARG;
}

// Blocks that share the contraction of G's tiles, where there are few of them and many columns.  In units of 10 ns a block takes 33
// for a slice of 64 columns (45 with tiles of 128), and where it is shared 100 and 60 for every part that the last one adds up (300 x
// 5000: 233 us unshared, 143 so; 256 x 4096: 194, 128; 1024 x 4096: 274, 231).
int split_of(int r, int n, int P) {
  const int64_t mt = (r + BM - 1) / BM, tiles = mt * (mt + 1) / 2 * P, nk = (n + BK - 1) / BK;
  int64_t best = 1, least = INT64_MAX;
  for (int64_t s = 1; s <= 16 && s * tiles <= sm_count(); ++s) {
    const int64_t share = (nk + s - 1) / s;
    if (s > 1 && share * (s - 1) >= nk) continue;            // every part has a slice
    const bool half = 2 * s * tiles <= sm_count();
    const int64_t cost = (half ? 33 : 45) * share + (s > 1 ? 100 + 60 * s : 0);
    if (cost < least) best = s, least = cost;
  }
  return (int)best;
}
struct Plan {
  int r, n;                  // rows and columns of X
  int64_t ldx, ldg;
  uint32_t blocks, tiles;    // of the norm; of G, of 64 columns
  bool small;                // one block a matrix
  int split;                 // of G's contraction
  uint64_t part, done, partial, x[2], rest[2], g, q, total;      // X of even and odd steps, and what it was rounded by
};
Plan plan_of(const lsgd_ortho_desc* d) {
  Plan m{};
  m.r = d->m < d->n ? d->m : d->n;
  m.n = d->m < d->n ? d->n : d->m;
  m.ldx = (m.n + 7) / 8 * 8;
  m.ldg = (m.r + 7) / 8 * 8;
  const int64_t each = d->n % 4 == 0 ? 4096 : 1024;       // values of a block: 4 pieces a thread, all under way at once
  const int64_t want = ((int64_t)d->m * d->n + each - 1) / each, cap = (4 * (int64_t)sm_count() + d->P - 1) / d->P;
  m.blocks = (uint32_t)(want < cap ? want : cap);
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) {
    const uint64_t here = at;
    at += (bytes + 255) & ~uint64_t(255);
    return here;
  };
  m.small = m.r <= kSmallRows && m.n <= kSmallCols && d->steps > 0;
  if (m.small) return m;
  m.part = take(sizeof(double) * (uint64_t)d->P * m.blocks);
  if (d->steps > 0) {
    const uint64_t x = 2 * (uint64_t)d->P * m.r * m.ldx, g = 2 * (uint64_t)d->P * m.r * m.ldg;
    for (int i = 0; i < 2 && i < d->steps; ++i) m.x[i] = take(x);
    for (int i = 0; i < 2 && i + 1 < d->steps; ++i) m.rest[i] = take(x);
    m.split = split_of(m.r, m.n, d->P);
    m.tiles = (uint32_t)(((m.r + BM - 1) / BM) * ((m.r + BM - 1) / BM + 1) * (int64_t)d->P);
    if (m.split > 1) {
      m.done = take(sizeof(uint32_t) * m.tiles);             // (of 64 columns)
      m.partial = take(sizeof(float) * (uint64_t)BM * 64 * m.tiles * m.split);
    }
    m.g = take(g);
    m.q = take(g);
  }
  m.total = at;
  return m;
}

bool encode_boxes(CUtensorMap* map, const void* base, int64_t inner, int64_t outer, int64_t ld, int64_t P, int rows) {
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, base, inner, outer, ld, P, ld * outer, 64, rows);
}

template <bool PAIR, int BN>
cudaError_t launch_form(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& c, const CUtensorMap& d, const CUtensorMap& rest, const Product& p,
                        int64_t tiles, cudaStream_t s) {
  static OncePerDevice attr;
  constexpr int kSmemBytes = Form<PAIR, BN>::kSmemBytes;
  if (!attr.here()) {
    const cudaError_t e = cudaFuncSetAttribute(product_kernel<PAIR, BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    if (e != cudaSuccess) return e;
    attr.here() = true;
  }
  const int64_t cap = PAIR ? sm_count() / 2 : sm_count(), n = tiles < cap ? tiles : cap;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(PAIR ? 2 * n : n));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemBytes;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = 2;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = PAIR ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, product_kernel<PAIR, BN>, a, b, c, d, rest, p);
}
template <typename F>
int64_t tiles_of(const Product& p) {
  const int64_t mt = (p.M + F::kM - 1) / F::kM, nt = (p.N + F::kN - 1) / F::kN;
  return (p.symmetric ? mt * (mt + 1) / 2 * (F::kM / F::kN) : mt * nt) * p.batch * p.split;
}
// The form whose rounds over the machine take least.  A pair's tile is four of 128 x 128 on two SMs and runs at about 1.4 times their
// rate (32 x 1024 x 1024: 1131 us instead of 1334 when it was chosen).  One of 64 columns fetches three quarters of a square's operands and has half its
// epilogue, so it takes about 11 of its 14: where there are few (3 x 1001 x 333: 131 us instead of 147; 768 x 768: 140 instead of 158; 8 x 256
// x 256: 93 instead of 113).  c64, rest64: the stored tensors in boxes of 64 rows.
struct Chosen {
  int columns;               // 64, 128, or 256: pairs
  int64_t tiles, each;       // in all; most that a block (a pair) takes
};
Chosen form_of(const Product& p) {
  const int64_t half = tiles_of<Form<false, 64>>(p), one = tiles_of<Form<false, 128>>(p), two = tiles_of<Form<true, 128>>(p), sms = sm_count();
  const int64_t n_half = (half + sms - 1) / sms, n_one = (one + sms - 1) / sms, n_two = (two + sms / 2 - 1) / (sms / 2);
  if (11 * n_half < 14 * n_one && 11 * n_half < 20 * n_two) return {64, half, n_half};
  return 20 * n_two <= 14 * n_one && p.split == 1 ? Chosen{256, two, n_two} : Chosen{128, one, n_one};
}
cudaError_t launch_product(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& c, const CUtensorMap& c64, const CUtensorMap& d,
                           const CUtensorMap& rest, const CUtensorMap& rest64, const Product& p, cudaStream_t s) {
  if (tiles_of<Form<false, 64>>(p) >= int64_t(1) << 31) return cudaErrorInvalidValue;
  const Chosen f = form_of(p);
  return f.columns == 64    ? launch_form<false, 64>(a, b, c64, d, rest64, p, f.tiles, s)
         : f.columns == 256 ? launch_form<true, 128>(a, b, c, d, rest, p, f.tiles, s)
                            : launch_form<false, 128>(a, b, c, d, rest, p, f.tiles, s);
}

template <typename T>
cudaError_t launch_prep(const Prep& a, int vec, cudaStream_t s) {
  const dim3 norm(a.blocks, a.d.P), tiles((a.d.n + 63) / 64, (a.d.m + 63) / 64, a.d.P);
  cudaError_t e = vec == 4 ? launch_pdl(norm_kernel<T, 4>, norm, dim3(256), 0, s, a) : launch_pdl(norm_kernel<T, 1>, norm, dim3(256), 0, s, a);
  if (e != cudaSuccess) return e;
  return vec == 4 ? launch_pdl(scale_kernel<T, 4>, tiles, dim3(256), 0, s, a) : launch_pdl(scale_kernel<T, 1>, tiles, dim3(256), 0, s, a);
}

lsgd_status run_ortho(const lsgd_ortho_desc* d, cudaStream_t s) {
  const Plan m = plan_of(d);
  char* scratch = static_cast<char*>(d->scratch);
  Prep a{};
  a.d = *d;
  a.part = reinterpret_cast<double*>(scratch + m.part);
  a.blocks = m.blocks;
  a.done = reinterpret_cast<uint32_t*>(scratch + m.done);
  a.n_done = m.split > 1 ? m.tiles : 0;
  a.x = reinterpret_cast<__half*>(scratch + m.x[0]);
  a.lo = d->steps > 1 ? reinterpret_cast<__half*>(scratch + m.rest[0]) : nullptr;
  a.r = m.r;
  a.n = m.n;
  a.tall = d->m > d->n;
  a.out_wide = row_vec(d->out, d->P, d->m, d->n, 2) == 8;
  a.ld = m.ldx;
  a.stride = m.ldx * m.r;
  const int gb = elem_bytes(d->grad_dtype);
  auto fits = [&](const lsgd_rows& r, int bytes) {
    return !r.data || (d->n % 4 == 0 && reinterpret_cast<uintptr_t>(r.data) % (4 * bytes) == 0 && (d->m <= 1 || r.ld % 4 == 0) && (d->P <= 1 || r.stride % 4 == 0));
  };
  const int vec = fits(d->grad, gb) && fits(d->momentum, 4) ? 4 : 1;
  cudaError_t e = cudaSuccess;
  if (m.small)
    e = d->grad_dtype == LSGD_BF16 ? (vec == 4 ? launch_small<__nv_bfloat16, 4>(a, s) : launch_small<__nv_bfloat16, 1>(a, s))
                                   : (vec == 4 ? launch_small<float, 4>(a, s) : launch_small<float, 1>(a, s));
  if (m.small) return e == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
  e = d->grad_dtype == LSGD_BF16 ? launch_prep<__nv_bfloat16>(a, vec, s) : launch_prep<float>(a, vec, s);
  if (e != cudaSuccess) return LSGD_ERR_CUDA;
  if (d->steps == 0) return LSGD_OK;
  // a matrix in boxes of 64 and of 128 rows; those without a place (few steps) are not reached
  struct Maps {
    CUtensorMap op, tile;
  } x[2], rest[2], g, q;
  auto map = [&](Maps& t, uint64_t at, int64_t inner, int64_t ld) {
    return encode_boxes(&t.op, scratch + at, inner, m.r, ld, d->P, 64) && encode_boxes(&t.tile, scratch + at, inner, m.r, ld, d->P, 128);
  };
  if (!map(g, m.g, m.r, m.ldg) || !map(q, m.q, m.r, m.ldg)) return LSGD_ERR_CUDA;
  for (int i = 0; i < 2; ++i)
    if (!map(x[i], m.x[i], m.n, m.ldx) || !map(rest[i], m.rest[i], m.n, m.ldx)) return LSGD_ERR_CUDA;
  const float down = 1.f / kScale;
  for (int step = 0; step < d->steps; ++step) {
    const bool last = step + 1 == d->steps;          // takes no rest of X, and stores neither X nor a rest
    const Maps &from = x[step & 1], &to = x[(step & 1) ^ 1], &from_rest = rest[step & 1], &to_rest = rest[(step & 1) ^ 1];
    Product p{};
    p.batch = d->P;
    p.M = p.N = m.r;
    p.K = m.n;
    p.symmetric = 1;
    p.split = m.split;
    p.partial = reinterpret_cast<float*>(scratch + m.partial);
    p.done = a.done;
    p.alpha = down;
    if (launch_product(from.op, from.op, g.tile, g.op, g.tile, g.tile, g.op, p, s) != cudaSuccess) return LSGD_ERR_CUDA;
    p.K = m.r;
    p.split = 1;
    p.add = 1;
    p.alpha = d->c * down;
    p.beta = d->b;
    p.diag = d->a * kScale;
    if (launch_product(g.op, g.op, q.tile, q.op, g.tile, q.tile, q.op, p, s) != cudaSuccess) return LSGD_ERR_CUDA;
    p.N = m.n;
    p.symmetric = 0;
    p.b_mn = 1;
    p.twofold = !last && m.r <= kTwofoldRows;
    p.add = !last && !p.twofold;
    p.alpha = p.beta = down;
    p.diag = 0.f;
    p.rows = p.add ? reinterpret_cast<const __half*>(scratch + m.q) : nullptr;    // Q's diagonal
    p.rows_ld = m.ldg + 1;
    p.rows_stride = m.ldg * m.r;
    p.rest = step + 2 < d->steps;
    if (last) {
      p.out = static_cast<__nv_bfloat16*>(d->out.data);
      p.out_ld = d->out.ld;
      p.out_stride = d->out.stride;
      p.out_transposed = a.tall;
      p.out_wide = a.out_wide;
      p.scale = d->scale * down;
    }
    if (launch_product(q.op, from.op, to.tile, to.op, p.twofold ? from_rest.op : from_rest.tile, to_rest.tile, to_rest.op, p, s) != cudaSuccess)
      return LSGD_ERR_CUDA;
  }
  return LSGD_OK;
}

}  // namespace
}  // namespace ortho
}  // namespace lsgd

extern "C" {

uint64_t lsgd_ortho_scratch_bytes(const lsgd_ortho_desc* d) {
  using namespace lsgd::ortho;
  if (!d || d->struct_size != sizeof(lsgd_ortho_desc) || d->P < 1 || d->P > 65535 || d->m < 1 || d->m > 65536 || d->n < 1 || d->n > 65536 || d->steps < 0) return 0;
  return plan_of(d).total;
}

lsgd_status lsgd_ortho(const lsgd_ortho_desc* d, void* stream) {
  using namespace lsgd::ortho;
  const lsgd_status st = check_ortho(d);
  if (st != LSGD_OK) return st;
  const uint64_t need = lsgd_ortho_scratch_bytes(d);
  if (need && (!d->scratch || d->scratch_bytes < need)) return LSGD_ERR_INVALID_ARG;
  if (need && reinterpret_cast<uintptr_t>(d->scratch) % 256) return LSGD_ERR_ALIGNMENT;
  return run_ortho(d, static_cast<cudaStream_t>(stream));
}

lsgd_status lsgd_ortho_plan(const lsgd_ortho_desc* d, int32_t plan[7]) {
  using namespace lsgd::ortho;
  const lsgd_status st = check_ortho(d);
  if (st != LSGD_OK || !plan) return st != LSGD_OK ? st : LSGD_ERR_INVALID_ARG;
  const Plan m = plan_of(d);
  for (int i = 0; i < 7; ++i) plan[i] = 0;
  if (m.small || d->steps == 0) return LSGD_OK;
  for (int i = 0; i < 3; ++i) {
    Product p{};
    p.batch = d->P;
    p.M = m.r;
    p.N = i < 2 ? m.r : m.n;
    p.symmetric = i < 2;
    p.split = i == 0 ? m.split : 1;
    const Chosen f = form_of(p);
    plan[i] = f.columns;
    plan[3 + i] = (int32_t)f.each;
  }
  plan[6] = m.split;
  return LSGD_OK;
}

lsgd_status lsgd_ortho_check_device(uint32_t* flag_out) {
  uint32_t f = 0;
  if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&f, lsgd::ortho::g_status, sizeof(f)) != cudaSuccess) return LSGD_ERR_CUDA;
  const uint32_t zero = 0;
  if (f && cudaMemcpyToSymbol(lsgd::ortho::g_status, &zero, sizeof(zero)) != cudaSuccess) return LSGD_ERR_CUDA;
  if (flag_out) *flag_out = f;
  return f ? LSGD_ERR_DEVICE_FLAG : LSGD_OK;
}

}  // extern "C"
