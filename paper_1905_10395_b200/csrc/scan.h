// Selective state space scan and its gradient (include/lsgd.h): the kernels of one activation type.
//
//   h_t = exp(delta_t A) h_(t-1) + delta_t x_t B_t,   y_t = C_t . h_t
//
// for N states of every channel.  L lanes (2, 4, 8 or 16) share a channel and hold 4 of its states each in registers (N <= 4 L; states up
// to the next of 8, 16, 32 and 64 are computed and left out of the sums), two to an instruction.  A block takes some channels of a run of
// rows (a chain), a tile of rows at a time: the tile's next rows are fetched into registers while the present ones run, and are staged in
// shared memory as what the recurrence reads: delta and delta x (one softplus a row and channel), B and C as fp32.  delta and delta x lie [channel][row], so that a lane reads four rows at once.  The
// sums over a channel's states go through its L lanes, four rows at a time (each lane ends up with one row's sum), and are finished
// (skip, gate) by the thread that staged the row's piece of 8 channels.
//
// What bounds it: exponentials, one a state and row (16 a clock and SM), with 2 to 4 more a row and channel for softplus and gate.
//
// Chains.  Where workers, sequences and channels give enough blocks, a chain is a run of whole sequences and nothing else is
// needed.  Otherwise the rows are split into chains of equal length: a first pass finds what every chain adds to the state behind
// it and by how much it decays the state in front (one exp of the summed time steps), a short pass runs over the chains, and
// the last pass starts every chain from its own state.  The exps are then computed twice.
//
// Gradient.  The forward pass saves the state in front of every 8th row.  A chain goes backwards in groups of 8 rows: it recomputes
// the group's states from the saved one, keeps them and the decays in registers, and runs the adjoint
//   g_t = d_t C_t + a_(t+1) g_(t+1)
// back through them.  dB and dC are sums over channels: over a warp's by exchanges that halve the number of values at
// each step, over the warps in shared memory, over the blocks by a second kernel; all in a fixed order.
#pragma once
#include <cfloat>
#include <type_traits>

#include "activations.h"
#include "seq.h"

namespace lsgd {
namespace scan {

constexpr int kThreads = 128, kQuad = 4, kGroup = 8;
constexpr int kBlocks = 4;       // of either direction's kernels, resident on an SM
// Channels of a block, rows of a tile; at most one piece of 8 channels of a row a thread.
template <int L> struct Tile {
  static constexpr int kCh = kThreads / L;
  static constexpr int kFull = kThreads * 8 / kCh;                 // rows that give every thread a piece
  static constexpr int kRows = kFull > 32 ? 32 : kFull;
  static constexpr int kN = kQuad * L;                             // states, padded
  static constexpr int kPieces = kCh / 8 * kRows;
  static constexpr int kPitch = kRows + 4, kArray = kCh * kPitch;  // an array [channel][row]
  static constexpr int kQuads = (2 * kRows * L + kThreads - 1) / kThreads;   // pieces of 4 states of B and C a thread stages
  // A row's place: turned by 4 rows every 8 channels, so that neither a warp's pieces (8 channels apart) nor its lanes (one
  // channel apart, four rows at a time) meet in a bank.
  static __device__ __forceinline__ int at(int ch, int t) { return ch * kPitch + ((t + 4 * (ch >> 3)) & (kRows - 1)); }
};

struct Args {
  lsgd_scan_desc d;
  SeqView q;
  int32_t chains, per;       // chains of a worker; sequences of a chain, or (split) rows
  int32_t split, wide;       // wide: values that every row can be moved at a time (8, 4, 2 or 1)
  int32_t wide_bc;           // rows of b and c can be moved 4 values at a time
  uint32_t tiles;            // blocks of channels
  float* ends;               // split: [P][chains][D][N], what a chain adds, then the state (adjoint) it starts from
  float* sums;               // split: [P][chains][D], summed time steps; negative where a sequence begins inside
  float* old_state;          // split, with a state: its copy, [P][S][D][N]
  float* part_bc;            // backward: [P][tiles][T][2][N]
  float* part_a;             // backward: [P][chains][D][N]
  float* part_v;             // backward: [P][chains][2][D]
};

template <typename T>
__device__ __forceinline__ Rows<T> view(const lsgd_rows& r) {
  return Rows<T>{static_cast<T*>(r.data), r.ld, r.stride};
}
// exp(delta A) = 2^(delta A2).  The unit's results are 1e-8 low on average for the small arguments of slowly decaying states (its
// roundings, measured against 64 bits over [-0.1, 0)), which a thousand rows in front of such a state would all add: the argument is
// lifted by as much.  The gradient of a_log, of 2048 rows, is then off by 7e-7 of its norm instead of 1.4e-6.
constexpr float kLift = 1.7e-8f;
__device__ __forceinline__ float2 decay(float2 delta, float2 A2) { return ex2(fma2(delta, A2, make_float2(kLift, kLift))); }
// softplus(v) = max(v, 0) + log1p(e), e = exp(-|v|) <= 1; log1p(e) = 2 artanh(s), s = e / (2 + e) <= 1/3, with a polynomial in s^2
// for artanh(s) / s (interpolation at Chebyshev's points; within 2e-8).
__device__ __forceinline__ float2 softplus(float2 v, float2& e) {
  e = ex2(mul2(make_float2(fabsf(v.x), fabsf(v.y)), both(-kLog2e)));
  const float2 s = mul2(e, rcp(add2(e, both(2.f)))), s2 = mul2(s, s);
  float2 r = fma2(s2, both(0.13433775f), both(0.14116978f));
  r = fma2(s2, r, both(0.20003835f));
  r = fma2(s2, r, both(0.3333332f));
  r = fma2(mul2(s, s2), r, s);
  return fma2(r, both(2.f), make_float2(fmaxf(v.x, 0.f), fmaxf(v.y, 0.f)));
}
__device__ __forceinline__ float softplus(float v, float& e) {
  float2 e2;
  const float r = softplus(both(v), e2).x;
  e = e2.x;
  return r;
}
// 8 neighbouring channels of a row, `width` (8, 4, 2 or 1) at a time; those behind the last are zeros.
template <typename T, int W>
__device__ __forceinline__ void load_by(float (&f)[8], const T* row, int ch, int D) {
#pragma unroll
  for (int v = 0; v < 8; v += W) {
#pragma unroll
    for (int k = 0; k < W; ++k) f[v + k] = 0.f;
    if (ch + v < D) {
      Pack<T, W> k;
      k.load(row + ch + v);
      k.get(f + v);
    }
  }
}
template <typename T>
__device__ __forceinline__ void load8(Pack<T, 8>& k, const T* row, int ch, int D, int width) {
  if (width == 8) {
    k.load(row + ch);
    return;
  }
  float f[8];
  if (width == 4) load_by<T, 4>(f, row, ch, D);
  else if (width == 2) load_by<T, 2>(f, row, ch, D);
  else load_by<T, 1>(f, row, ch, D);
  k.set(f);
}
template <typename T, int W>
__device__ __forceinline__ void store_by(const float (&f)[8], T* row, int ch, int D) {
#pragma unroll
  for (int v = 0; v < 8; v += W)
    if (ch + v < D) {
      Pack<T, W> k;
      k.set(f + v);
      k.store(row + ch + v);
    }
}
template <typename T>
__device__ __forceinline__ void store8(const float (&f)[8], T* row, int ch, int D, int width) {
  if (width == 8) store_by<T, 8>(f, row, ch, ch + 8);
  else if (width == 4) store_by<T, 4>(f, row, ch, D);
  else if (width == 2) store_by<T, 2>(f, row, ch, D);
  else store_by<T, 1>(f, row, ch, D);
}
__device__ __forceinline__ void pairs8(const float (&f)[8], float2 (&q)[4]) {
#pragma unroll
  for (int v = 0; v < 4; ++v) q[v] = make_float2(f[2 * v], f[2 * v + 1]);
}
// A log2(e); of a finite a_log whose exponential leaves fp32, the largest there is: times a time step of zero (of rows of no sequence,
// or far below) it is no NaN.
__device__ __forceinline__ float rate_of(float a_log) {
  const float A2 = -expf(a_log) * kLog2e;
  return a_log < __int_as_float(0x7F800000) && A2 < -FLT_MAX ? -FLT_MAX : A2;
}
// ... of 4 states of a channel; 0 for those that do not exist (they stay zero, for B is zero there)
__device__ __forceinline__ void decay_rates(const Args& a, int p, int ch, int n0, float (&A2)[kQuad]) {
  const float* src = static_cast<const float*>(a.d.a_log.data) + p * a.d.a_log.stride + ch * a.d.a_log.ld + n0;
#pragma unroll
  for (int k = 0; k < kQuad; ++k) A2[k] = ch < a.d.D && n0 + k < a.d.N ? src[k] : 0.f;
#pragma unroll
  for (int k = 0; k < kQuad; ++k) A2[k] = ch < a.d.D && n0 + k < a.d.N ? rate_of(A2[k]) : 0.f;
}
__device__ __forceinline__ void load_vector8(const lsgd_rows& v, int p, int ch, int D, float2 (&f)[4]) {
  const float* src = static_cast<const float*>(v.data) + p * v.stride + ch;
#pragma unroll
  for (int k = 0; k < 4; ++k) f[k] = make_float2(v.data && ch + 2 * k < D ? src[2 * k] : 0.f, v.data && ch + 2 * k + 1 < D ? src[2 * k + 1] : 0.f);
}
__device__ __forceinline__ float vector_at(const lsgd_rows& v, int p, int ch, bool in) {
  return in && v.data ? static_cast<const float*>(v.data)[p * v.stride + ch] : 0.f;
}

// 4 states of a channel in a [..][D][N] array of fp32, whose row `row` is (.., channel)
__device__ __forceinline__ void load_states(const float* base, int64_t row, int n0, int N, float (&h)[kQuad]) {
  const float* src = base + row * N + n0;
  if ((N & 3) == 0) {
    const float4 v = *reinterpret_cast<const float4*>(src);
    h[0] = v.x, h[1] = v.y, h[2] = v.z, h[3] = v.w;
  } else {
#pragma unroll
    for (int k = 0; k < kQuad; ++k) h[k] = n0 + k < N ? src[k] : 0.f;
  }
}
__device__ __forceinline__ void store_states(float* base, int64_t row, int n0, int N, const float (&h)[kQuad]) {
  float* dst = base + row * N + n0;
  if ((N & 3) == 0) {
    *reinterpret_cast<float4*>(dst) = make_float4(h[0], h[1], h[2], h[3]);
  } else {
#pragma unroll
    for (int k = 0; k < kQuad; ++k)
      if (n0 + k < N) dst[k] = h[k];
  }
}

struct Range {
  int t0, t1, base;          // rows of the chain; base: t0 rounded down to a group
  int lo = 0, hi = 0;        // equal parts: the sequence that was asked for last
  __device__ __forceinline__ Range(const Args& a, int p, int c) {
    if (a.split) {
      t0 = min(a.q.T, c * a.per);
      t1 = min(a.q.T, t0 + a.per);
    } else {
      const int s0 = c * a.per, s1 = min(a.q.S, s0 + a.per);
      t0 = a.q.edge(p, s0);
      t1 = a.q.edge(p, s1);
    }
    base = t0 & ~(kGroup - 1);
  }
  // Whether rows [at, at + rows) are the chain's and one sequence's, which neither begins nor ends among them.
  __device__ __forceinline__ bool plain(const Args& a, int p, int at, int rows) {
    if (at < t0 || at + rows > t1) return false;
    if (a.q.starts) {
      const int code = a.q.code(p, at - 1);
      return code >= 0 && code == a.q.code(p, at + rows);
    }
    if (at < lo || at >= hi) {
      lo = at / a.q.len * a.q.len;
      hi = lo + a.q.len;
    }
    return at > lo && at + rows < hi;
  }
};
__device__ __forceinline__ bool row_lives(const Args& a, int p, const Range& r, int t) {
  return t >= r.t0 && t < r.t1 && (!a.q.starts || a.q.code(p, t) >= 0);
}
// Which rows of a tile begin and end a sequence (its number, else -1; of no sequence: kNoRow).
constexpr int kNoRow = -2;
template <int ROWS>
__device__ __forceinline__ void mark_rows(const Args& a, int p, const Range& r, int base, int* begins, int* ends, int i) {
  if (i >= ROWS) return;
  const int t = base + i;
  int b = kNoRow, e = kNoRow;
  if (t >= r.t0 && t < r.t1) {
    const int code = a.q.code(p, t);
    if (code >= 0) {
      b = e = -1;
      if (a.q.code(p, t - 1) != code) b = code;
      if (a.q.code(p, t + 1) != code) e = code;
    }
  }
  begins[i] = b;
  ends[i] = e;
}

// Sums over the L lanes of a channel for four rows.  L >= 4: lane l holds row row_of(l) in y[0]; L == 2: rows 2 (l & 1) and one more.
template <int L>
__device__ __forceinline__ void sum_states(float (&y)[4], int lane) {
  const bool b0 = lane & 1;
  const float s0 = b0 ? y[0] : y[2], s1 = b0 ? y[1] : y[3];
  y[0] = (b0 ? y[2] : y[0]) + __shfl_xor_sync(0xFFFFFFFFu, s0, 1);
  y[1] = (b0 ? y[3] : y[1]) + __shfl_xor_sync(0xFFFFFFFFu, s1, 1);
  if (L == 2) return;
  const bool b1 = lane & 2;
  const float s = b1 ? y[0] : y[1];
  y[0] = (b1 ? y[1] : y[0]) + __shfl_xor_sync(0xFFFFFFFFu, s, 2);
#pragma unroll
  for (int m = 4; m < L; m *= 2) y[0] += __shfl_xor_sync(0xFFFFFFFFu, y[0], m);
}
__device__ __forceinline__ int row_of(int lane) { return 2 * (lane & 1) + ((lane >> 1) & 1); }
// ... and stores them: rows t .. t + 3 of channel ch of an array
template <int L, typename Ti>
__device__ __forceinline__ void keep_sums(float (&y)[4], float* array, int ch, int t, int lane) {
  sum_states<L>(y, lane);
  float* at = array + Ti::at(ch, t);               // the four rows lie together
  if (L == 2) {
    *reinterpret_cast<float2*>(at + 2 * (lane & 1)) = make_float2(y[0], y[1]);
  } else if (lane % L < 4) {
    at[row_of(lane)] = y[0];
  }
}

// B and C of a tile: pieces of 4 states, fetched into registers and stored as fp32 [which][row][state].
template <typename T, int L, typename Ti>
struct StageBC {
  Pack<T, 4> k[Ti::kQuads];
  const T* from[Ti::kQuads];                       // at row 0; NULL: no such states
  int64_t ld[Ti::kQuads];
  __device__ __forceinline__ void init(const Args& a, int p, int tid, bool b_too) {
#pragma unroll
    for (int j = 0; j < Ti::kQuads; ++j) {
      const int i = tid + j * kThreads, which = i / (Ti::kRows * L), n = i % L * kQuad;
      from[j] = which > 1 || n >= a.d.N || (which == 0 && !b_too) ? nullptr
                : static_cast<const T*>(which ? a.d.c.data : a.d.b.data) + p * (which ? a.d.c.stride : a.d.b.stride) + n;
      ld[j] = which ? a.d.c.ld : a.d.b.ld;
    }
  }
  __device__ __forceinline__ void fetch(const Args& a, int p, const Range& r, int base, bool plain, int tid) {
#pragma unroll
    for (int j = 0; j < Ti::kQuads; ++j) {
      const int i = tid + j * kThreads, row = base + i / L % Ti::kRows, n = i % L * kQuad;
      const float zero[4] = {};
      k[j].set(zero);
      if (!from[j] || !(plain || row_lives(a, p, r, row))) continue;
      const T* src = from[j] + row * ld[j];
      if (a.wide_bc) {
        k[j].load(src);
      } else {
        float f[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          Pack<T, 1> one;
          f[v] = 0.f;
          if (n + v < a.d.N) {
            one.load(src + v);
            one.get(f + v);
          }
        }
        k[j].set(f);
      }
    }
  }
  __device__ __forceinline__ void store(float* bc, int tid) const {
#pragma unroll
    for (int j = 0; j < Ti::kQuads; ++j) {
      const int i = tid + j * kThreads;
      if (i >= 2 * Ti::kRows * L) continue;
      float f[4];
      k[j].get(f);
      *reinterpret_cast<float4*>(bc + i * kQuad) = make_float4(f[0], f[1], f[2], f[3]);
    }
  }
};

__device__ __forceinline__ void pairs(const float4& v, float2 (&f)[2]) {
  f[0] = make_float2(v.x, v.y);
  f[1] = make_float2(v.z, v.w);
}
__device__ __forceinline__ float part_of(const float4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// ------------------------------------------------------------------------------------------------ forward
// Named barriers of 2 kThreads threads, half of which wait.
__device__ __forceinline__ void barrier_wait(int id) { asm volatile("barrier.sync %0, %1;" ::"r"(id), "n"(2 * kThreads) : "memory"); }
__device__ __forceinline__ void barrier_arrive(int id) { asm volatile("barrier.arrive %0, %1;" ::"r"(id), "n"(2 * kThreads) : "memory"); }

// kEnds: only what the chain adds to the state behind it, and its summed time steps.
// kSome: some of a channel's 4 L states do not exist.  They stay out of the sums: their h is zero, but infinite inputs make it NaN
// (infinity times B's zero).
// Half of the block's warps run the recurrence, the others stage the next tile and finish the last one meanwhile (two buffers; barriers
// 1 + b: buffer b is staged, 3 + b: its tile is done), so that a block's staging, a chain of latencies, does not stop its recurrence:
// ragged prompts of 8191 x 1500 take 203 us instead of 258.  (Two channels a thread would halve what is read of B and C, but leave
// half the warps: the prompts took 304 us instead of 203, though 32768 x 384 in fp32, which lacks no warps, 172 instead of 197.)
template <typename T, int L, bool kEnds, bool kSome>
__global__ void __launch_bounds__(2 * kThreads, kBlocks) forward_kernel(const __grid_constant__ Args a) {
  using Ti = Tile<L>;
  pdl_wait();
  pdl_launch_dependents();
  __shared__ __align__(16) float s_delta[2][Ti::kArray], s_du[2][Ti::kArray], s_y[2][kEnds ? 4 : Ti::kArray];   // delta, delta x; C . h
  __shared__ __align__(16) float s_bc[2][2 * Ti::kRows * Ti::kN];
  __shared__ __align__(16) float s_bias[Ti::kCh], s_skip[Ti::kCh];
  __shared__ int s_begin[2][Ti::kRows], s_end[2][Ti::kRows], s_plain[2];
  const int p = blockIdx.z, c = blockIdx.y;
  Range r(a, p, c);
  const lsgd_scan_desc& d = a.d;
  const int n_tiles = r.base < r.t1 ? (r.t1 - r.base + Ti::kRows - 1) / Ti::kRows : 0;

  if (threadIdx.x >= kThreads) {
    // ---------------------------------------------------------------- stage and finish: a piece of 8 channels of a row a thread
    const int tid = threadIdx.x - kThreads, prow = tid / (Ti::kCh / 8), piece = (tid % (Ti::kCh / 8)) * 8;
    const int pch = blockIdx.x * Ti::kCh + piece, own = Ti::at(piece, prow);
    const bool has_piece = tid < Ti::kPieces && pch < d.D, gated = !kEnds && d.z.data != nullptr;
    for (int i = tid; i < Ti::kCh; i += kThreads) {
      const int col = blockIdx.x * Ti::kCh + i;
      s_bias[i] = vector_at(d.dt_bias, p, col, col < d.D);
      s_skip[i] = vector_at(d.skip, p, col, col < d.D);
    }
    asm volatile("barrier.sync 5, %0;" ::"n"(kThreads) : "memory");
    const int wide = a.wide;
    StageBC<T, L, Ti> bc;
    bc.init(a, p, tid, true);
    const T *px = view<T>(d.x).row(p, r.base + prow), *pdt = view<T>(d.dt).row(p, r.base + prow);
    Pack<T, 8> rx, rdt, rz;
    bool plain = false, live = false, was_live = false;
    auto fetch = [&](int base) {
      plain = r.plain(a, p, base, Ti::kRows);
      live = has_piece && (plain || row_lives(a, p, r, base + prow));
      if (live) {
        load8<T>(rx, px, pch, d.D, wide);
        load8<T>(rdt, pdt, pch, d.D, wide);
      }
      px += Ti::kRows * d.x.ld, pdt += Ti::kRows * d.dt.ld;
      bc.fetch(a, p, r, base, plain, tid);
    };
    auto stage = [&](int base, int b) {
      if (live) {
        float fx[8], fd[8];
        float2 x2[4], dt2[4];
        rx.get(fx);
        rdt.get(fd);
        pairs8(fx, x2);
        pairs8(fd, dt2);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          float2 e;
          const float2 delta = softplus(add2(dt2[v], *reinterpret_cast<const float2*>(s_bias + piece + 2 * v)), e), du = mul2(delta, x2[v]);
          s_delta[b][own + 2 * v * Ti::kPitch] = delta.x, s_delta[b][own + (2 * v + 1) * Ti::kPitch] = delta.y;
          s_du[b][own + 2 * v * Ti::kPitch] = du.x, s_du[b][own + (2 * v + 1) * Ti::kPitch] = du.y;
        }
      } else if (tid < Ti::kPieces) {
#pragma unroll
        for (int v = 0; v < 8; ++v) s_delta[b][own + v * Ti::kPitch] = s_du[b][own + v * Ti::kPitch] = 0.f;
      }
      bc.store(s_bc[b], tid);
      if (!plain) mark_rows<Ti::kRows>(a, p, r, base, s_begin[b], s_end[b], tid);
      if (tid == 0) s_plain[b] = plain;
    };
    if (n_tiles > 0) {
      fetch(r.base);
      stage(r.base, 0);
      barrier_arrive(1);
      was_live = live;
      if (n_tiles > 1) fetch(r.base + Ti::kRows);
    }
    for (int i = 0; i < n_tiles; ++i) {
      const int base = r.base + i * Ti::kRows, b = i & 1;
      const bool finish = !kEnds && was_live;
      if (i + 1 < n_tiles) {
        stage(base + Ti::kRows, b ^ 1);
        barrier_arrive(1 + (b ^ 1));
        was_live = live;
        if (i + 2 < n_tiles) fetch(base + 2 * Ti::kRows);
      }
      Pack<T, 8> kx;
      if (finish) {                                                // again, from the caches
        load8<T>(kx, view<T>(d.x).row(p, base + prow), pch, d.D, wide);
        if (gated) load8<T>(rz, view<T>(d.z).row(p, base + prow), pch, d.D, wide);
      }
      barrier_wait(3 + b);
      if (!finish) continue;
      float f[8];
      float2 x2[4], y2[4];
      kx.get(f);
      pairs8(f, x2);
#pragma unroll
      for (int v = 0; v < 4; ++v)
        y2[v] = fma2(*reinterpret_cast<const float2*>(s_skip + piece + 2 * v), x2[v],
                     make_float2(s_y[b][own + 2 * v * Ti::kPitch], s_y[b][own + (2 * v + 1) * Ti::kPitch]));
      if (gated) {
        float2 z2[4];
        rz.get(f);
        pairs8(f, z2);
#pragma unroll
        for (int v = 0; v < 4; ++v) y2[v] = mul2(y2[v], mul2(z2[v], sigmoid(z2[v])));
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) f[2 * v] = y2[v].x, f[2 * v + 1] = y2[v].y;
      store8<T>(f, view<T>(d.out).row(p, base + prow), pch, d.D, wide);
    }
    return;
  }

  // ------------------------------------------------------------------ the recurrence
  const int lane = threadIdx.x & 31, local = threadIdx.x / L, ch = blockIdx.x * Ti::kCh + local, n0 = (threadIdx.x % L) * kQuad;
  const bool mine = ch < d.D && n0 < d.N, with_state = d.state != nullptr;
  const int64_t chain_row = ((int64_t)p * a.chains + c) * d.D + ch;
  float2 A2[2], h[2];
  {
    float f[kQuad], g[kQuad] = {};
    decay_rates(a, p, ch, n0, f);
    if (!kEnds && a.split && mine) load_states(a.ends, chain_row, n0, d.N, g);
    A2[0] = make_float2(f[0], f[1]), A2[1] = make_float2(f[2], f[3]);
    h[0] = make_float2(g[0], g[1]), h[1] = make_float2(g[2], g[3]);
  }
  float sum = 0.f;
  bool fresh = false;                                              // a sequence began inside
  // the states in front of every 8th row
  const int64_t saved_step = (int64_t)d.D * d.N;
  float* saved = !kEnds && d.saved && mine ? d.saved + ((int64_t)p * ((a.q.T + kGroup - 1) / kGroup) + r.base / kGroup) * saved_step + (int64_t)ch * d.N : nullptr;
  const int turn = 4 * (local >> 3);
  auto only = [&](float2 v, int k) { return kSome ? make_float2(n0 + 2 * k < d.N ? v.x : 0.f, n0 + 2 * k + 1 < d.N ? v.y : 0.f) : v; };
  // four rows of the recurrence
  auto rows4 = [&](int base, int b, int t4, auto special) {
    if (!kEnds && saved && t4 % kGroup == 0) {
      if (!special || (base + t4 >= r.t0 && base + t4 < r.t1)) {
        const float f[kQuad] = {h[0].x, h[0].y, h[1].x, h[1].y};
        store_states(saved, 0, n0, d.N, f);
      }
      saved += saved_step;
    }
    const int place = local * Ti::kPitch + ((t4 + turn) & (Ti::kRows - 1));
    const float4 delta4 = *reinterpret_cast<const float4*>(s_delta[b] + place);
    const float4 du4 = *reinterpret_cast<const float4*>(s_du[b] + place);
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = t4 + i;
      if (special) {
        const int s = s_begin[b][t];
        if (s >= 0) {
          fresh = true;
          float f[kQuad] = {};
          if (with_state && mine) {
            const int64_t row = ((int64_t)p * a.q.S + s) * d.D + ch;
            load_states(a.split && !kEnds ? a.old_state : d.state, row, n0, d.N, f);
            if (kEnds) store_states(a.old_state, row, n0, d.N, f);
          }
          h[0] = make_float2(f[0], f[1]), h[1] = make_float2(f[2], f[3]);
        }
      }
      const float delta = part_of(delta4, i), du = part_of(du4, i);
      float2 B[2], C[2];
      pairs(*reinterpret_cast<const float4*>(s_bc[b] + t * Ti::kN + n0), B);
      h[0] = fma2(decay(both(delta), A2[0]), h[0], mul2(both(du), B[0]));
      h[1] = fma2(decay(both(delta), A2[1]), h[1], mul2(both(du), B[1]));
      if (kEnds) {
        sum += delta;
      } else {
        pairs(*reinterpret_cast<const float4*>(s_bc[b] + (Ti::kRows + t) * Ti::kN + n0), C);
        const float2 s = fma2(C[0], only(h[0], 0), mul2(C[1], only(h[1], 1)));
        y[i] = s.x + s.y;
        if (special && with_state && mine && s_end[b][t] >= 0) {
          const float f[kQuad] = {h[0].x, h[0].y, h[1].x, h[1].y};
          store_states(d.state, ((int64_t)p * a.q.S + s_end[b][t]) * d.D + ch, n0, d.N, f);
        }
      }
    }
    if (!kEnds) keep_sums<L, Ti>(y, s_y[b], local, t4, lane);
  };
  for (int i = 0; i < n_tiles; ++i) {
    const int base = r.base + i * Ti::kRows, b = i & 1;
    barrier_wait(1 + b);
    if (s_plain[b]) {
#pragma unroll 2
      for (int t4 = 0; t4 < Ti::kRows; t4 += 4) rows4(base, b, t4, std::false_type());
    } else {
#pragma unroll 1
      for (int t4 = 0; t4 < Ti::kRows; t4 += 4) rows4(base, b, t4, std::true_type());
    }
    barrier_arrive(3 + b);
  }
  if (kEnds && mine) {
    const float f[kQuad] = {h[0].x, h[0].y, h[1].x, h[1].y};
    store_states(a.ends, chain_row, n0, d.N, f);
    if (n0 == 0) a.sums[chain_row] = fresh ? -1.f : sum;
  }
}

// Sequences of one row each: a thread takes 4 states of a channel of one sequence after another.  Everything that a row needs is under
// way before the first of it, the decays' logarithms included, is used: what bounds a block is one latency of memory and its
// own work, so many small blocks overlap (64 x 4096 x 16: 12 us; four rows a thread at a time, in half the warps, 16).
template <typename T, int L, bool kSome>
__global__ void __launch_bounds__(kThreads, 10) single_kernel(const __grid_constant__ Args a) {
  pdl_wait();
  pdl_launch_dependents();
  const int p = blockIdx.z, lane = threadIdx.x & 31;
  const lsgd_scan_desc& d = a.d;
  const int ch = blockIdx.x * (kThreads / L) + threadIdx.x / L, n0 = (threadIdx.x % L) * kQuad;
  const bool in = ch < d.D, mine = in && n0 < d.N;
  auto one = [&](const lsgd_rows& m, int t) {
    Pack<T, 1> k;
    float f = 0.f;
    k.set(&f);
    if (in && m.data) k.load(view<T>(m).row(p, t) + ch);
    return k;
  };
  auto four = [&](const lsgd_rows& m, int t) {
    const T* src = view<T>(m).row(p, t) + n0;
    Pack<T, 4> k;
    float f[kQuad] = {};
    if (mine && a.wide_bc) {
      k.load(src);
      return k;
    }
#pragma unroll
    for (int i = 0; i < kQuad; ++i)
      if (mine && n0 + i < d.N) {
        Pack<T, 1> v;
        v.load(src + i);
        v.get(f + i);
      }
    k.set(f);
    return k;
  };
  auto value = [](const Pack<T, 1>& k) {
    float f;
    k.get(&f);
    return f;
  };
  float A2[kQuad];
  const float* logs = static_cast<const float*>(d.a_log.data) + p * d.a_log.stride + ch * d.a_log.ld + n0;
#pragma unroll
  for (int k = 0; k < kQuad; ++k) A2[k] = in && n0 + k < d.N ? logs[k] : 0.f;
  const float bias = vector_at(d.dt_bias, p, ch, in), skip = vector_at(d.skip, p, ch, in);
  bool rates = false;
  for (int t = blockIdx.y; t < a.q.S; t += gridDim.y) {
    const int64_t row = ((int64_t)p * a.q.S + t) * d.D + ch;
    float h[kQuad] = {}, B[kQuad], C[kQuad];
    if (d.state && mine) load_states(d.state, row, n0, d.N, h);
    const Pack<T, 1> kdt = one(d.dt, t), kx = one(d.x, t), kz = one(d.z, t);
    const Pack<T, 4> kb = four(d.b, t), kc = four(d.c, t);
    if (!rates) {
#pragma unroll
      for (int k = 0; k < kQuad; ++k) A2[k] = in && n0 + k < d.N ? rate_of(A2[k]) : 0.f;
      rates = true;
    }
    float e, y = 0.f;
    const float x = value(kx), delta = softplus(value(kdt) + bias, e), du = delta * x;
    kb.get(B);
    kc.get(C);
#pragma unroll
    for (int k = 0; k < kQuad; ++k) {
      h[k] = fmaf(ex2(fmaf(delta, A2[k], kLift)), h[k], du * B[k]);
      if (!kSome || n0 + k < d.N) y = fmaf(C[k], h[k], y);     // kSome: as for the forward kernel
    }
    if (d.state && mine) store_states(d.state, row, n0, d.N, h);
#pragma unroll
    for (int m = 1; m < L; m *= 2) y += __shfl_xor_sync(0xFFFFFFFFu, y, m);
    if (lane % L == 0 && in) {
      float o = fmaf(skip, x, y);
      if (d.z.data) {
        const float z = value(kz);
        o *= z * sigmoid(z);
      }
      Pack<T, 1> k;
      k.set(&o);
      k.store(view<T>(d.out).row(p, t) + ch);
    }
  }
}

// ------------------------------------------------------------------------------------------------ backward
// Split chains: what the chain's rows add to the adjoint in front of it, and its summed time steps.
template <typename T, int L>
__global__ void __launch_bounds__(kThreads, kBlocks) adjoint_kernel(const __grid_constant__ Args a) {
  using Ti = Tile<L>;
  pdl_wait();
  pdl_launch_dependents();
  __shared__ __align__(16) float s_delta[Ti::kArray], s_d[Ti::kArray], s_bc[2 * Ti::kRows * Ti::kN];
  __shared__ int s_begin[Ti::kRows], s_end[Ti::kRows];
  const int p = blockIdx.z, c = blockIdx.y;
  Range r(a, p, c);
  const lsgd_scan_desc& d = a.d;
  const int local = threadIdx.x / L, ch = blockIdx.x * Ti::kCh + local, n0 = (threadIdx.x % L) * kQuad;
  const bool mine = ch < d.D && n0 < d.N;
  const int64_t chain_row = ((int64_t)p * a.chains + c) * d.D + ch;
  float2 A2[2], carry[2] = {};                                     // carry: a_(t+1) g_(t+1)
  {
    float f[kQuad];
    decay_rates(a, p, ch, n0, f);
    A2[0] = make_float2(f[0], f[1]), A2[1] = make_float2(f[2], f[3]);
  }
  float sum = 0.f;
  bool fresh = false;
  const int prow = threadIdx.x / (Ti::kCh / 8), piece = (threadIdx.x % (Ti::kCh / 8)) * 8;
  const int pch = blockIdx.x * Ti::kCh + piece;
  const bool has_piece = threadIdx.x < Ti::kPieces && pch < d.D;
  const int wide = a.wide;
  const Rows<T> dt = view<T>(d.dt), z = view<T>(d.z), up = view<T>(d.d_out);
  float2 bias[4];
  load_vector8(d.dt_bias, p, pch, has_piece ? d.D : 0, bias);
  const int own = Ti::at(piece, prow);
  const bool gated = d.z.data != nullptr;
  Pack<T, 8> rup, rdt, rz;
  StageBC<T, L, Ti> bc;
  bc.init(a, p, threadIdx.x, false);
  bool live = false, plain = false;
  auto fetch = [&](int base) {
    const int t = base + prow;
    plain = r.plain(a, p, base, Ti::kRows);
    live = has_piece && (plain || row_lives(a, p, r, t));
    if (live) {
      load8<T>(rup, up.row(p, t), pch, d.D, wide);
      load8<T>(rdt, dt.row(p, t), pch, d.D, wide);
      if (d.z.data) load8<T>(rz, z.row(p, t), pch, d.D, wide);
    }
    bc.fetch(a, p, r, base, plain, threadIdx.x);
  };
  const int n_tiles = r.base < r.t1 ? (r.t1 - r.base + Ti::kRows - 1) / Ti::kRows : 0;
  if (n_tiles > 0) fetch(r.base + (n_tiles - 1) * Ti::kRows);
  for (int it = n_tiles - 1; it >= 0; --it) {
    const int base = r.base + it * Ti::kRows;
    if (live) {
      float f[8];
      float2 up2[4], dt2[4];
      rup.get(f);
      pairs8(f, up2);
      rdt.get(f);
      pairs8(f, dt2);
      if (gated) {
        float2 z2[4];
        rz.get(f);
        pairs8(f, z2);
#pragma unroll
        for (int v = 0; v < 4; ++v) up2[v] = mul2(up2[v], mul2(z2[v], sigmoid(z2[v])));
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        float2 e;
        const float2 delta = softplus(add2(dt2[v], bias[v]), e);
        s_delta[own + 2 * v * Ti::kPitch] = delta.x, s_delta[own + (2 * v + 1) * Ti::kPitch] = delta.y;
        s_d[own + 2 * v * Ti::kPitch] = up2[v].x, s_d[own + (2 * v + 1) * Ti::kPitch] = up2[v].y;
      }
    } else if (threadIdx.x < Ti::kPieces) {
#pragma unroll
      for (int v = 0; v < 8; ++v) s_delta[own + v * Ti::kPitch] = s_d[own + v * Ti::kPitch] = 0.f;
    }
    bc.store(s_bc, threadIdx.x);
    const bool special = !plain;
    if (special) mark_rows<Ti::kRows>(a, p, r, base, s_begin, s_end, threadIdx.x);
    __syncthreads();
    if (it > 0) fetch(base - Ti::kRows);
#pragma unroll 2
    for (int t4 = Ti::kRows - 4; t4 >= 0; t4 -= 4) {
      const float4 delta4 = *reinterpret_cast<const float4*>(s_delta + Ti::at(local, t4));
      const float4 d4 = *reinterpret_cast<const float4*>(s_d + Ti::at(local, t4));
#pragma unroll
      for (int i = 3; i >= 0; --i) {
        float2 C[2];
        pairs(*reinterpret_cast<const float4*>(s_bc + (Ti::kRows + t4 + i) * Ti::kN + n0), C);
        const float delta = part_of(delta4, i), g0 = part_of(d4, i);
        carry[0] = mul2(decay(both(delta), A2[0]), fma2(C[0], both(g0), carry[0]));
        carry[1] = mul2(decay(both(delta), A2[1]), fma2(C[1], both(g0), carry[1]));
        sum += delta;
        if (special && s_begin[t4 + i] >= 0) {
          fresh = true;
          carry[0] = carry[1] = make_float2(0.f, 0.f);
        }
      }
    }
    __syncthreads();
  }
  if (mine) {
    const float f[kQuad] = {carry[0].x, carry[0].y, carry[1].x, carry[1].y};
    store_states(a.ends, chain_row, n0, d.N, f);
    if (n0 == 0) a.sums[chain_row] = fresh ? -1.f : sum;
  }
}

// Sums of 8 values over the 32 / L channels of a warp; a lane ends up with `count` of them, from `first` on.
template <int L>
struct ChannelSum {
  static constexpr int kCount = L == 16 ? 4 : L == 8 ? 2 : 1;
  static __device__ __forceinline__ int first(int lane) {
    int i = (lane & L) ? 4 : 0;
    if (2 * L <= 16) i += (lane & (2 * L)) ? 2 : 0;
    if (4 * L <= 16) i += (lane & (4 * L)) ? 1 : 0;
    return i;
  }
  static __device__ __forceinline__ void run(float (&v)[8], int lane) {
    halve<4>(v, lane, L);
    if (2 * L <= 16) halve<2>(v, lane, 2 * L);
    if (4 * L <= 16) halve<1>(v, lane, 4 * L);
    if (8 * L <= 16) v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], 8 * L);
  }
  template <int H>
  static __device__ __forceinline__ void halve(float (&v)[8], int lane, int m) {
    const bool up = lane & m;
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const float send = up ? v[i] : v[i + H], keep = up ? v[i + H] : v[i];
      v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, m);
    }
  }
};

__device__ __forceinline__ void copy_async(void* dst, const void* src, int bytes) {       // 8 or 16
  const uint32_t to = (uint32_t)__cvta_generic_to_shared(dst);
  if (bytes == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(src) : "memory");
  else asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(src) : "memory");
}

// Shared memory of a block, the dynamic part: what a thread keeps for itself.
template <typename T, int L>
struct BackSmem {
  static constexpr int kBufs = L == 16 ? 1 : 2;
  static constexpr int kPart = kThreads / 32 * kGroup * 8 * L;     // warps x rows x (4 dB, 4 dC) x L
  static constexpr int kOwn = 8 * kThreads;                        // values of a thread's piece, [value][thread]
  static constexpr int kRaw = kThreads;                            // pieces of 8 values as they came, [thread]
  static constexpr size_t bytes = sizeof(float) * 2 * kOwn + sizeof(Pack<T, 8>) * 5 * kRaw + sizeof(Pack<T, 4>) * Tile<L>::kQuads * kThreads;
};
// Registers: the four rows in hand (states, decays, B, C and time steps, which both directions use), so that four blocks fit an SM;
// what is fetched for the next tile therefore goes to shared memory.
// kSome: some of a channel's 4 L states do not exist, or some of the last block's channels.  They stay out of the sums: they are zero, but
// infinite inputs make them NaN.
template <typename T, int L, bool kSome>
__global__ void __launch_bounds__(kThreads, kBlocks) backward_kernel(const __grid_constant__ Args a) {
  using Ti = Tile<L>;
  using Sm = BackSmem<T, L>;
  pdl_wait();
  pdl_launch_dependents();
  // what the recurrence reads (delta, delta x, d), and its sums over the states (g B, C h; q A log2(e) takes delta x's place)
  __shared__ __align__(16) float s_delta[Ti::kArray], s_du[Ti::kArray], s_d[Ti::kArray], s_gb[Ti::kArray], s_y[Ti::kArray];
  __shared__ __align__(16) float s_bc[2 * Ti::kRows * Ti::kN], s_part[Sm::kBufs * Sm::kPart];
  __shared__ int s_begin[Ti::kRows], s_end[Ti::kRows];
  extern __shared__ __align__(16) float s_own[];
  float *s_slope = s_own + threadIdx.x, *s_gate = s_slope + Sm::kOwn;
  Pack<T, 8>* raw = reinterpret_cast<Pack<T, 8>*>(s_own + 2 * Sm::kOwn) + threadIdx.x;       // dt, d_out, z, x, the other tile's x
  Pack<T, 4>* raw_bc = reinterpret_cast<Pack<T, 4>*>(reinterpret_cast<Pack<T, 8>*>(s_own + 2 * Sm::kOwn) + 5 * Sm::kRaw) + threadIdx.x;
  const int p = blockIdx.z, c = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Range r(a, p, c);
  const lsgd_scan_desc& d = a.d;
  const int local = threadIdx.x / L, ch = blockIdx.x * Ti::kCh + local, n0 = (threadIdx.x % L) * kQuad;
  const bool mine = ch < d.D && n0 < d.N;
  // carry: a_(t+1) g_(t+1); dA: of a tile's rows, total: of the tiles' (summed by fours, tiles and chains: 2048 terms in a row would
  // lose three bits)
  float2 A2[2], carry[2], dA[2] = {}, total[2] = {};
  {
    float f[kQuad], g[kQuad] = {};
    decay_rates(a, p, ch, n0, f);
    if (a.split && mine) load_states(a.ends, ((int64_t)p * a.chains + c) * d.D + ch, n0, d.N, g);
    A2[0] = make_float2(f[0], f[1]), A2[1] = make_float2(f[2], f[3]);
    carry[0] = make_float2(g[0], g[1]), carry[1] = make_float2(g[2], g[3]);
  }
  const int prow = threadIdx.x / (Ti::kCh / 8), piece = (threadIdx.x % (Ti::kCh / 8)) * 8;
  const int pch = blockIdx.x * Ti::kCh + piece, own = Ti::at(piece, prow);
  const bool has_piece = threadIdx.x < Ti::kPieces && pch < d.D;
  const bool gated = d.z.data != nullptr;
  const int n_tiles = r.base < r.t1 ? (r.t1 - r.base + Ti::kRows - 1) / Ti::kRows : 0;
  int base = r.base + (n_tiles - 1) * Ti::kRows;
  bool live = false, plain = false;
  auto fetch8 = [&](Pack<T, 8>* to, const lsgd_rows& m, int t) {
    const T* src = view<T>(m).row(p, t);
    if (a.wide == 8) {
#pragma unroll
      for (int k = 0; k < (int)sizeof(Pack<T, 8>); k += 16)
        copy_async(reinterpret_cast<char*>(to) + k, reinterpret_cast<const char*>(src + pch) + k, 16);
    } else {
      Pack<T, 8> k;
      load8<T>(k, src, pch, d.D, a.wide);
      *to = k;
    }
  };
  auto fetch = [&](int at, int which) {
    plain = r.plain(a, p, at, Ti::kRows);
    live = has_piece && (plain || row_lives(a, p, r, at + prow));
    if (live) {
      fetch8(raw, d.dt, at + prow);
      fetch8(raw + Sm::kRaw, d.d_out, at + prow);
      if (gated) fetch8(raw + 2 * Sm::kRaw, d.z, at + prow);
      fetch8(raw + (3 + which) * Sm::kRaw, d.x, at + prow);
    }
#pragma unroll
    for (int j = 0; j < Ti::kQuads; ++j) {
      const int i = threadIdx.x + j * kThreads, w = i / (Ti::kRows * L), row = at + i / L % Ti::kRows, n = i % L * kQuad;
      if (w > 1) continue;
      Pack<T, 4>* to = raw_bc + j * kThreads;
      if (n < d.N && (plain || row_lives(a, p, r, row))) {
        const T* src = view<T>(w ? d.c : d.b).row(p, row) + n;
        if (a.wide_bc) {
          copy_async(to, src, (int)sizeof(Pack<T, 4>));
          continue;
        }
        float f[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          Pack<T, 1> one;
          f[v] = 0.f;
          if (n + v < d.N) {
            one.load(src + v);
            one.get(f + v);
          }
        }
        to->set(f);
      } else {
        const float zero[4] = {};
        to->set(zero);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int parity = 0;
  if (n_tiles > 0) fetch(base, parity);
  const int place0 = local * Ti::kPitch, turn = 4 * (local >> 3);
  // the saved state in front of a group, fetched a group ahead
  const float* saved = d.saved + ((int64_t)p * ((a.q.T + kGroup - 1) / kGroup) * d.D + ch) * d.N;
  float next[kQuad] = {};
  auto fetch_state = [&](int row0) {
    if (mine && row0 >= r.t0 && row0 < r.t1) load_states(saved, (int64_t)(row0 / kGroup) * d.D, n0, d.N, next);
    else next[0] = next[1] = next[2] = next[3] = 0.f;
  };
  if (n_tiles > 0) fetch_state(base + Ti::kRows - kGroup);
  float* part_bc = a.part_bc + ((int64_t)p * a.tiles + blockIdx.x) * a.q.T * 2 * d.N;
  float column = 0.f;                                              // of d skip or d dt_bias
  int buf = 0;
  const int there = mine ? d.N - n0 : 0;
  // (beside the recurrences, not in them)
  auto only = [&](float2 v, int k) { return kSome ? make_float2(2 * k < there ? v.x : 0.f, 2 * k + 1 < there ? v.y : 0.f) : v; };
  // a group of 8 rows from row0 = base + g8: the later four first, whose states are found through the earlier ones'
  auto group = [&](int row0, int g8, auto special) {
    const float2 first[2] = {make_float2(next[0], next[1]), make_float2(next[2], next[3])};
    fetch_state(row0 - kGroup);
    float* part = s_part + buf * Sm::kPart + warp * kGroup * 8 * L;
    float2 h[2] = {first[0], first[1]};
    {
      const int place = place0 + ((g8 + turn) & (Ti::kRows - 1));
      const float4 delta4 = *reinterpret_cast<const float4*>(s_delta + place), du4 = *reinterpret_cast<const float4*>(s_du + place);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (special && s_begin[g8 + i] != -1) h[0] = h[1] = make_float2(0.f, 0.f);
        float2 B[2];
        pairs(*reinterpret_cast<const float4*>(s_bc + (g8 + i) * Ti::kN + n0), B);
        const float2 delta = both(part_of(delta4, i)), du = both(part_of(du4, i));
#pragma unroll
        for (int k = 0; k < 2; ++k) h[k] = fma2(decay(delta, A2[k]), h[k], mul2(du, B[k]));
      }
    }
#pragma unroll 1
    for (int half = 4; half >= 0; half -= 4) {
      if (half == 0) h[0] = first[0], h[1] = first[1];
      const float2 prior[2] = {h[0], h[1]};                        // the state in front of the four rows
      float2 hs[4][2], as[4][2], B[4][2], C[4][2];
      float y[4], gb[4], qa[4];
      const int place = place0 + ((g8 + half + turn) & (Ti::kRows - 1));
      const float4 delta4 = *reinterpret_cast<const float4*>(s_delta + place), du4 = *reinterpret_cast<const float4*>(s_du + place);
      const float4 d4 = *reinterpret_cast<const float4*>(s_d + place);
      const float *b_of = s_bc + (g8 + half) * Ti::kN + n0, *c_of = b_of + Ti::kRows * Ti::kN;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (special && s_begin[g8 + half + i] != -1) h[0] = h[1] = make_float2(0.f, 0.f);
        pairs(*reinterpret_cast<const float4*>(b_of + i * Ti::kN), B[i]);
        pairs(*reinterpret_cast<const float4*>(c_of + i * Ti::kN), C[i]);
        const float2 delta = both(part_of(delta4, i)), du = both(part_of(du4, i));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          as[i][k] = decay(delta, A2[k]);
          h[k] = fma2(as[i][k], h[k], mul2(du, B[i][k]));
          hs[i][k] = only(h[k], k);
        }
        if (gated) {
          const float2 s = fma2(C[i][0], hs[i][0], mul2(C[i][1], hs[i][1]));
          y[i] = s.x + s.y;
        }
      }
      float2 sum_a[2] = {};                                        // of the four rows
#pragma unroll
      for (int i = 3; i >= 0; --i) {
        float2 db[2], dc[2], sb, sq;
        const float2 delta = both(part_of(delta4, i)), du = both(part_of(du4, i)), dy = both(part_of(d4, i));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float2 all = fma2(C[i][k], dy, carry[k]), g = only(all, k);
          db[k] = mul2(g, du);
          dc[k] = mul2(dy, hs[i][k]);
          sb = k == 0 ? mul2(g, B[i][k]) : fma2(g, B[i][k], sb);
          carry[k] = mul2(as[i][k], all);
          float2 q = only(mul2(carry[k], i > 0 ? hs[i > 0 ? i - 1 : 0][k] : prior[k]), k);
          if (special && s_begin[g8 + half + i] != -1) carry[k] = q = make_float2(0.f, 0.f);
          sum_a[k] = fma2(q, delta, sum_a[k]);
          sq = k == 0 ? mul2(q, A2[k]) : fma2(q, A2[k], sq);
        }
        gb[i] = sb.x + sb.y;
        qa[i] = sq.x + sq.y;
        float v[8] = {db[0].x, db[0].y, db[1].x, db[1].y, dc[0].x, dc[0].y, dc[1].x, dc[1].y};
        ChannelSum<L>::run(v, lane);
        if (8 * L > 16 || !(lane & (8 * L))) {
          const int f = ChannelSum<L>::first(lane);
#pragma unroll
          for (int q = 0; q < ChannelSum<L>::kCount; ++q) part[((half + i) * 8 + f + q) * L + lane % L] = v[q];
        }
      }
      if (gated) keep_sums<L, Ti>(y, s_y, local, g8 + half, lane);
      keep_sums<L, Ti>(gb, s_gb, local, g8 + half, lane);
      keep_sums<L, Ti>(qa, s_du, local, g8 + half, lane);          // whose four rows every lane of the channel has read
#pragma unroll
      for (int k = 0; k < 2; ++k) dA[k] = add2(dA[k], sum_a[k]);
    }
    __syncthreads();
    // the block's sums over its channels, the warps' in order
#pragma unroll
    for (int i = threadIdx.x; i < kGroup * 8 * L; i += kThreads) {
      const int row = row0 + i / (8 * L), which = (i / L) % 8, n = (i % L) * kQuad + which % 4;
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < kThreads / 32; ++w) s += s_part[buf * Sm::kPart + w * kGroup * 8 * L + i];
      if (n < d.N && (!special || (row >= r.t0 && row < r.t1))) part_bc[(int64_t)row * 2 * d.N + which / 4 * d.N + n] = s;
    }
    if (Sm::kBufs == 1) __syncthreads();
    else buf ^= 1;
  };
  for (int it = n_tiles - 1; it >= 0; --it, base -= Ti::kRows, parity ^= 1) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");           // a thread reads only what it has copied
    if (live) {
      float f[8];
      float2 x2[4], up2[4], dt2[4], bias[4];
      raw[(3 + parity) * Sm::kRaw].get(f);
      pairs8(f, x2);
      raw[Sm::kRaw].get(f);
      pairs8(f, up2);
      raw[0].get(f);
      pairs8(f, dt2);
      load_vector8(d.dt_bias, p, pch, d.D, bias);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        float2 e;
        const float2 pre = add2(dt2[v], bias[v]), delta = softplus(pre, e), du = mul2(delta, x2[v]);
        const float2 slope = mul2(make_float2(pre.x >= 0.f ? 1.f : e.x, pre.y >= 0.f ? 1.f : e.y), rcp(add2(e, both(1.f))));
        s_delta[own + 2 * v * Ti::kPitch] = delta.x, s_delta[own + (2 * v + 1) * Ti::kPitch] = delta.y;
        s_du[own + 2 * v * Ti::kPitch] = du.x, s_du[own + (2 * v + 1) * Ti::kPitch] = du.y;
        s_slope[2 * v * kThreads] = slope.x, s_slope[(2 * v + 1) * kThreads] = slope.y;
      }
      if (gated) {
        float2 z2[4];
        raw[2 * Sm::kRaw].get(f);
        pairs8(f, z2);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float2 sg = sigmoid(z2[v]), sl = mul2(z2[v], sg);
          const float2 gate = mul2(up2[v], fma2(sl, make_float2(1.f - sg.x, 1.f - sg.y), sg));
          s_gate[2 * v * kThreads] = gate.x, s_gate[(2 * v + 1) * kThreads] = gate.y;
          up2[v] = mul2(up2[v], sl);
        }
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) s_d[own + 2 * v * Ti::kPitch] = up2[v].x, s_d[own + (2 * v + 1) * Ti::kPitch] = up2[v].y;
    } else if (threadIdx.x < Ti::kPieces) {
#pragma unroll
      for (int v = 0; v < 8; ++v) s_delta[own + v * Ti::kPitch] = s_du[own + v * Ti::kPitch] = s_d[own + v * Ti::kPitch] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < Ti::kQuads; ++j) {
      const int i = threadIdx.x + j * kThreads;
      if (i >= 2 * Ti::kRows * L) continue;
      float f[4];
      raw_bc[j * kThreads].get(f);
      *reinterpret_cast<float4*>(s_bc + i * kQuad) = make_float4(f[0], f[1], f[2], f[3]);
    }
    const bool is_plain = plain, was_live = live;
    if (!is_plain) mark_rows<Ti::kRows>(a, p, r, base, s_begin, s_end, threadIdx.x);
    __syncthreads();
    if (it > 0) fetch(base - Ti::kRows, parity ^ 1);
    if (is_plain) {
#pragma unroll 1
      for (int g8 = Ti::kRows - kGroup; g8 >= 0; g8 -= kGroup) group(base + g8, g8, std::false_type());
    } else {
#pragma unroll 1
      for (int g8 = Ti::kRows - kGroup; g8 >= 0; g8 -= kGroup) {
        if (base + g8 < r.t1 && base + g8 + kGroup > r.t0) group(base + g8, g8, std::true_type());      // the same for the whole block
        else fetch_state(base + g8 - kGroup);
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) total[k] = add2(total[k], dA[k]), dA[k] = make_float2(0.f, 0.f);
    // the last group's barrier has passed: every warp's sums are there
    if (was_live) {
      float f[8];
      float2 x2[4], skip[4];
      raw[(3 + parity) * Sm::kRaw].get(f);
      pairs8(f, x2);
      load_vector8(d.skip, p, pch, d.D, skip);
      auto pair_of = [&](const float* array, int v) { return make_float2(array[own + 2 * v * Ti::kPitch], array[own + (2 * v + 1) * Ti::kPitch]); };
      auto mine_of = [&](const float* array, int v) { return make_float2(array[2 * v * kThreads], array[(2 * v + 1) * kThreads]); };
      const int t = base + prow;
      if (gated) {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float2 o = mul2(mine_of(s_gate, v), fma2(skip[v], x2[v], pair_of(s_y, v)));
          f[2 * v] = o.x, f[2 * v + 1] = o.y;
        }
        store8<T>(f, view<T>(d.dz).row(p, t), pch, d.D, a.wide);
      }
      float2 gB[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        gB[v] = pair_of(s_gb, v);
        const float2 g = pair_of(s_d, v), o = fma2(pair_of(s_delta, v), gB[v], mul2(skip[v], g)), gx = mul2(g, x2[v]);
        f[2 * v] = o.x, f[2 * v + 1] = o.y;
        s_y[own + 2 * v * Ti::kPitch] = gx.x, s_y[own + (2 * v + 1) * Ti::kPitch] = gx.y;
      }
      store8<T>(f, view<T>(d.dx).row(p, t), pch, d.D, a.wide);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float2 o = mul2(fma2(x2[v], gB[v], mul2(pair_of(s_du, v), both(kLn2))), mine_of(s_slope, v));
        f[2 * v] = o.x, f[2 * v + 1] = o.y;
        s_gb[own + 2 * v * Ti::kPitch] = o.x, s_gb[own + (2 * v + 1) * Ti::kPitch] = o.y;
      }
      store8<T>(f, view<T>(d.d_dt).row(p, t), pch, d.D, a.wide);
    } else if (threadIdx.x < Ti::kPieces) {
#pragma unroll
      for (int v = 0; v < 8; ++v) s_gb[own + v * Ti::kPitch] = s_y[own + v * Ti::kPitch] = 0.f;
    }
    __syncthreads();
    // d skip and d dt_bias: a channel's rows of the tile in order (these arrays are written again behind the next barrier)
    if (threadIdx.x < 2 * Ti::kCh) {
      const float* src = (threadIdx.x < Ti::kCh ? s_y : s_gb) + threadIdx.x % Ti::kCh * Ti::kPitch;
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < Ti::kRows; k += 4) {
        const float4 v = *reinterpret_cast<const float4*>(src + k);
        s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
      }
      column += (s.x + s.y) + (s.z + s.w);
    }
  }
  if (mine) {
    const float f[kQuad] = {total[0].x * (A2[0].x * kLn2), total[0].y * (A2[0].y * kLn2), total[1].x * (A2[1].x * kLn2), total[1].y * (A2[1].y * kLn2)};
    store_states(a.part_a, ((int64_t)p * a.chains + c) * d.D + ch, n0, d.N, f);
  }
  const int which = threadIdx.x / Ti::kCh, col = blockIdx.x * Ti::kCh + threadIdx.x % Ti::kCh;
  if (which < 2 && col < d.D) a.part_v[(((int64_t)p * a.chains + c) * 2 + which) * d.D + col] = column;
}

// The backward pass's last sums.  The first blocks, which take longest: gradients of a_log, skip and dt_bias, the chains' sums in order (of
// all workers where they share the vector); columns of a worker: D x N of a_log, D of skip, D of dt_bias.  The others: db and dc,
// the channel blocks' sums in order.
template <typename T>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ Args a, const uint32_t blocks_params) {
  pdl_wait();
  pdl_launch_dependents();
  const int p = blockIdx.y;
  if (blockIdx.x >= blocks_params) {
    const int64_t i = (int64_t)(blockIdx.x - blocks_params) * 256 + threadIdx.x, n2 = 2 * a.d.N;
    if (i >= (int64_t)a.q.T * n2) return;
    const int t = (int)(i / n2), which = (int)(i % n2) / a.d.N, n = (int)(i % n2) % a.d.N;
    if (a.q.starts && a.q.code(p, t) < 0) return;
    const float* src = a.part_bc + (int64_t)p * a.tiles * a.q.T * n2 + i;
    float s = 0.f;
#pragma unroll 8
    for (uint32_t k = 0; k < a.tiles; ++k) s += src[(int64_t)k * a.q.T * n2];
    Pack<T, 1> one;
    one.set(&s);
    one.store(view<T>(which ? a.d.dc : a.d.db).row(p, t) + n);
    return;
  }
  const int64_t n = (int64_t)a.d.D * a.d.N, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n + 2 * a.d.D) return;
  const int which = i < n ? 0 : i < n + a.d.D ? 1 : 2;
  const lsgd_rows& o = which == 0 ? a.d.d_a_log : which == 1 ? a.d.d_skip : a.d.d_dt_bias;
  const bool shared = a.d.P > 1 && o.stride == 0;
  if (!o.data || (shared && p > 0)) return;
  const int64_t width = which == 0 ? n : 2 * a.d.D;
  const float* src = which == 0 ? a.part_a + i : a.part_v + (i - n);
  float total = 0.f;
  const int p0 = shared ? 0 : p, p1 = shared ? a.d.P : p + 1;
  for (int w = p0; w < p1; ++w) {
    const float* s = src + (int64_t)w * a.chains * width;
#pragma unroll 8
    for (int c = 0; c < a.chains; ++c) total += s[c * width];
  }
  const int64_t col = which == 0 ? i / a.d.N * o.ld + i % a.d.N : i - n - (which == 1 ? 0 : a.d.D);
  float* dst = static_cast<float*>(o.data) + (shared ? 0 : p * o.stride) + col;
  *dst = a.d.accumulate ? *dst + total : total;
}
template <typename T>
cudaError_t launch_join(const Args& a, cudaStream_t s) {
  const int64_t bc = ((int64_t)a.q.T * 2 * a.d.N + 255) / 256, params = ((int64_t)a.d.D * (a.d.N + 2) + 255) / 256;
  return launch_pdl(join_kernel<T>, dim3((unsigned)(bc + params), a.d.P), dim3(256), 0, s, a, (uint32_t)params);
}

struct Launch {
  int L;
  bool single;
  dim3 grid;
};
cudaError_t launch_forward_f32(const Args& a, const Launch& l, cudaStream_t s);
cudaError_t launch_forward_bf16(const Args& a, const Launch& l, cudaStream_t s);
cudaError_t launch_backward_f32(const Args& a, const Launch& l, cudaStream_t s);
cudaError_t launch_backward_bf16(const Args& a, const Launch& l, cudaStream_t s);
cudaError_t launch_join_f32(const Args& a, cudaStream_t s);
// split: from what every chain adds to what every chain starts from, forwards or backwards (scan.cu)
cudaError_t launch_chain_join(const Args& a, bool reverse, cudaStream_t s);

template <typename T, int L>
cudaError_t forward_of(const Args& a, const Launch& l, cudaStream_t s) {
  const bool some = a.d.N % Tile<L>::kN;
  if (l.single) return some ? launch_pdl(single_kernel<T, L, true>, l.grid, dim3(kThreads), 0, s, a) : launch_pdl(single_kernel<T, L, false>, l.grid, dim3(kThreads), 0, s, a);
  if (a.split) {
    cudaError_t e = launch_pdl(forward_kernel<T, L, true, false>, l.grid, dim3(2 * kThreads), 0, s, a);
    if (e == cudaSuccess) e = launch_chain_join(a, false, s);
    if (e != cudaSuccess) return e;
  }
  return some ? launch_pdl(forward_kernel<T, L, false, true>, l.grid, dim3(2 * kThreads), 0, s, a)
              : launch_pdl(forward_kernel<T, L, false, false>, l.grid, dim3(2 * kThreads), 0, s, a);
}
template <typename T, int L, bool kSome>
cudaError_t launch_backward(const Args& a, const Launch& l, cudaStream_t s) {
  constexpr size_t smem = BackSmem<T, L>::bytes;
  static OncePerDevice attr;
  if (!attr.here()) {
    const cudaError_t e = cudaFuncSetAttribute(backward_kernel<T, L, kSome>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    attr.here() = true;
  }
  return launch_pdl(backward_kernel<T, L, kSome>, l.grid, dim3(kThreads), smem, s, a);
}
template <typename T, int L>
cudaError_t backward_of(const Args& a, const Launch& l, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  if (a.split) {
    e = launch_pdl(adjoint_kernel<T, L>, l.grid, dim3(kThreads), 0, s, a);
    if (e == cudaSuccess) e = launch_chain_join(a, true, s);
  }
  const bool some = a.d.N % Tile<L>::kN || a.d.D % Tile<L>::kCh;
  if (e == cudaSuccess) e = some ? launch_backward<T, L, true>(a, l, s) : launch_backward<T, L, false>(a, l, s);
  return e == cudaSuccess ? launch_join<T>(a, s) : e;
}
template <typename T>
cudaError_t forward_any(const Args& a, const Launch& l, cudaStream_t s) {
  switch (l.L) {
    case 2: return forward_of<T, 2>(a, l, s);
    case 4: return forward_of<T, 4>(a, l, s);
    case 8: return forward_of<T, 8>(a, l, s);
    default: return forward_of<T, 16>(a, l, s);
  }
}
template <typename T>
cudaError_t backward_any(const Args& a, const Launch& l, cudaStream_t s) {
  switch (l.L) {
    case 2: return backward_of<T, 2>(a, l, s);
    case 4: return backward_of<T, 4>(a, l, s);
    case 8: return backward_of<T, 8>(a, l, s);
    default: return backward_of<T, 16>(a, l, s);
  }
}

}  // namespace scan
}  // namespace lsgd
