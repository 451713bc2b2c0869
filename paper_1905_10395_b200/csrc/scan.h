// Selective state space scan and its gradient (include/lsgd.h): the kernels of one activation type.
//
//   h_t = exp(delta_t A) h_(t-1) + delta_t x_t B_t,   y_t = C_t . h_t
//
// for N states of every channel.  L lanes share a channel and hold 4 of its states each in registers (N <= 4 L), two to an
// instruction.  A block takes some channels of a run of rows (a chain), a tile of rows at a time: the tile's next rows are fetched into
// registers while the present ones run, and are staged in shared memory as what the recurrence reads: delta and delta x (one
// softplus a row and channel), B and C as fp32.  delta and delta x lie [channel][row], so that a lane reads four rows at once.  The
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
// back through them.  dB and dC are sums over channels: over a thread's two, over the warp's by exchanges that halve the number of
// values at each step, over the warps in shared memory, over the blocks by a second kernel; all in a fixed order.
#pragma once
#include <type_traits>

#include "seq.h"

namespace lsgd {
namespace scan {

constexpr int kThreads = 128, kQuad = 4, kGroup = 8;
// CH channels of a block, rows of a tile; at most one piece of 8 channels of a row a thread.
template <int L, int KD> struct Tile {
  static constexpr int kCh = KD * kThreads / L;
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
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Args {
  lsgd_scan_desc d;
  SeqView q;
  int32_t chains, per;       // chains of a worker; sequences of a chain, or (split) rows
  int32_t split, wide;       // wide: every row can be moved 8 values at a time
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
__device__ __forceinline__ float ex2(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float2 ex2(float2 v) { return make_float2(ex2(v.x), ex2(v.y)); }
// softplus(v) = max(v, 0) + log1p(e), e = exp(-|v|) <= 1; log1p(e) = 2 artanh(s), s = e / (2 + e) <= 1/3, by its series.
__device__ __forceinline__ float softplus(float v, float& e) {
  e = ex2(-kLog2e * fabsf(v));
  const float s = __fdividef(e, 2.f + e), s2 = s * s;
  float r = fmaf(s2, 1.f / 13, 1.f / 11);
  r = fmaf(s2, r, 1.f / 9);
  r = fmaf(s2, r, 1.f / 7);
  r = fmaf(s2, r, 1.f / 5);
  r = fmaf(s2, r, 1.f / 3);
  return fmaxf(v, 0.f) + 2.f * fmaf(s * s2, r, s);
}
__device__ __forceinline__ float sigmoid(float v) { return __fdividef(1.f, 1.f + ex2(-kLog2e * v)); }

// 8 neighbouring channels of a row; those behind the last are zeros.
template <typename T>
__device__ __forceinline__ void load8(Pack<T, 8>& k, const T* row, int ch, int D, bool wide) {
  if (wide) {
    k.load(row + ch);
    return;
  }
  float f[8];
#pragma unroll
  for (int v = 0; v < 8; ++v) {
    Pack<T, 1> one;
    f[v] = 0.f;
    if (ch + v < D) {
      one.load(row + ch + v);
      one.get(f + v);
    }
  }
  k.set(f);
}
template <typename T>
__device__ __forceinline__ void store8(const float (&f)[8], T* row, int ch, int D, bool wide) {
  if (wide) {
    Pack<T, 8> k;
    k.set(f);
    k.store(row + ch);
    return;
  }
#pragma unroll
  for (int v = 0; v < 8; ++v)
    if (ch + v < D) {
      Pack<T, 1> one;
      one.set(f + v);
      one.store(row + ch + v);
    }
}

// A log2(e) of 4 states of a channel; 0 for those that do not exist (they stay zero, for B is zero there)
__device__ __forceinline__ void decay_rates(const Args& a, int p, int ch, int n0, float (&A2)[kQuad]) {
#pragma unroll
  for (int k = 0; k < kQuad; ++k) {
    A2[k] = 0.f;
    if (ch < a.d.D && n0 + k < a.d.N)
      A2[k] = -expf(static_cast<const float*>(a.d.a_log.data)[p * a.d.a_log.stride + ch * a.d.a_log.ld + n0 + k]) * kLog2e;
  }
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
  // Whether rows [base, base + rows) are the chain's and one sequence's, which neither begins nor ends among them.
  __device__ __forceinline__ bool plain(const Args& a, int p, int base_, int rows) const {
    if (base_ < t0 || base_ + rows > t1) return false;
    const int code = a.q.code(p, base_ - 1);
    return code >= 0 && code == a.q.code(p, base_ + rows);
  }
};
__device__ __forceinline__ bool row_lives(const Args& a, int p, const Range& r, int t) {
  return t >= r.t0 && t < r.t1 && (!a.q.starts || a.q.code(p, t) >= 0);
}
// Which rows of a tile begin and end a sequence (its number, else -1).
template <int ROWS>
__device__ __forceinline__ void mark_rows(const Args& a, int p, const Range& r, int base, int* begins, int* ends) {
  const int i = threadIdx.x;
  if (i >= ROWS) return;
  const int t = base + i;
  int b = -1, e = -1;
  if (t >= r.t0 && t < r.t1) {
    const int code = a.q.code(p, t);
    if (code >= 0) {
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
  if (L == 2) {
    array[Ti::at(ch, t + 2 * (lane & 1))] = y[0];
    array[Ti::at(ch, t + 2 * (lane & 1) + 1)] = y[1];
  } else if (lane % L < 4) {
    array[Ti::at(ch, t + row_of(lane))] = y[0];
  }
}

// B and C of a tile: pieces of 4 states, fetched into registers and stored as fp32 [which][row][state].
template <typename T, int L, typename Ti>
struct StageBC {
  Pack<T, 4> k[Ti::kQuads];
  __device__ __forceinline__ void fetch(const Args& a, int p, const Range& r, int base, bool plain, bool b_too) {
#pragma unroll
    for (int j = 0; j < Ti::kQuads; ++j) {
      const int i = threadIdx.x + j * kThreads, which = i / (Ti::kRows * L), row = base + i / L % Ti::kRows, n = i % L * kQuad;
      const float zero[4] = {};
      k[j].set(zero);
      if (which > 1 || n >= a.d.N || (which == 0 && !b_too) || !(plain || row_lives(a, p, r, row))) continue;
      const T* src = view<T>(which ? a.d.c : a.d.b).row(p, row) + n;
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
  __device__ __forceinline__ void store(float* bc) const {
#pragma unroll
    for (int j = 0; j < Ti::kQuads; ++j) {
      const int i = threadIdx.x + j * kThreads;
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
// kEnds: only what the chain adds to the state behind it, and its summed time steps.
template <typename T, int L, bool kEnds>
__global__ void __launch_bounds__(kThreads, 4) forward_kernel(const __grid_constant__ Args a) {
  using Ti = Tile<L, 1>;
  pdl_wait();
  pdl_launch_dependents();
  __shared__ __align__(16) float s_delta[Ti::kArray], s_du[Ti::kArray];      // delta, then the sum over the states; delta x
  __shared__ __align__(16) float s_bc[2 * Ti::kRows * Ti::kN];
  __shared__ int s_begin[Ti::kRows], s_end[Ti::kRows];
  const int p = blockIdx.z, c = blockIdx.y, lane = threadIdx.x & 31;
  const Range r(a, p, c);
  const lsgd_scan_desc& d = a.d;
  const int local = threadIdx.x / L, ch = blockIdx.x * Ti::kCh + local, n0 = (threadIdx.x % L) * kQuad;
  const bool mine = ch < d.D && n0 < d.N;
  const int64_t chain_row = ((int64_t)p * a.chains + c) * d.D + ch;
  float2 A2[2], h[2];
  {
    float f[kQuad], g[kQuad] = {};
    decay_rates(a, p, ch, n0, f);
    if (!kEnds && a.split && mine) load_states(a.ends, chain_row, n0, d.N, g);
    A2[0] = make_float2(f[0], f[1]), A2[1] = make_float2(f[2], f[3]);
    h[0] = make_float2(g[0], g[1]), h[1] = make_float2(g[2], g[3]);
  }
  const float* from = a.split && !kEnds ? a.old_state : d.state;
  float sum = 0.f;
  bool fresh = false;                                              // a sequence began inside

  // the piece of 8 channels of a row that this thread stages and finishes
  const int prow = threadIdx.x / (Ti::kCh / 8), piece = (threadIdx.x % (Ti::kCh / 8)) * 8;
  const int pch = blockIdx.x * Ti::kCh + piece;
  const bool has_piece = threadIdx.x < Ti::kPieces && pch < d.D;
  const bool wide = a.wide;
  const Rows<T> x = view<T>(d.x), dt = view<T>(d.dt), z = view<T>(d.z), out = view<T>(d.out);
  float bias[8], skip[8];
#pragma unroll
  for (int v = 0; v < 8; ++v) {
    bias[v] = vector_at(d.dt_bias, p, pch + v, has_piece && pch + v < d.D);
    skip[v] = vector_at(d.skip, p, pch + v, !kEnds && has_piece && pch + v < d.D);
  }
  Pack<T, 8> rx, rdt, rz;
  StageBC<T, L, Ti> bc;
  bool live = false, plain = false;
  auto fetch = [&](int base) {
    const int t = base + prow;
    plain = r.plain(a, p, base, Ti::kRows);
    live = has_piece && (plain || row_lives(a, p, r, t));
    if (live) {
      load8<T>(rx, x.row(p, t), pch, d.D, wide);
      load8<T>(rdt, dt.row(p, t), pch, d.D, wide);
      if (!kEnds && d.z.data) load8<T>(rz, z.row(p, t), pch, d.D, wide);
    }
    bc.fetch(a, p, r, base, plain, true);
  };
  if (r.base < r.t1) fetch(r.base);
  const int64_t groups = (a.q.T + kGroup - 1) / kGroup;
  // four rows of the recurrence
  auto rows4 = [&](int base, int t4, auto special) {
    if (!kEnds && d.saved && t4 % kGroup == 0 && mine && (!special || (base + t4 >= r.t0 && base + t4 < r.t1))) {
      const float f[kQuad] = {h[0].x, h[0].y, h[1].x, h[1].y};
      store_states(d.saved, ((int64_t)p * groups + (base + t4) / kGroup) * d.D + ch, n0, d.N, f);
    }
    const float4 delta4 = *reinterpret_cast<const float4*>(s_delta + Ti::at(local, t4));
    const float4 du4 = *reinterpret_cast<const float4*>(s_du + Ti::at(local, t4));
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = t4 + i;
      if (special) {
        const int s = s_begin[t];
        if (s >= 0) {
          fresh = true;
          float f[kQuad] = {};
          if (d.state && mine) {
            const int64_t row = ((int64_t)p * a.q.S + s) * d.D + ch;
            load_states(from, row, n0, d.N, f);
            if (kEnds) store_states(a.old_state, row, n0, d.N, f);
          }
          h[0] = make_float2(f[0], f[1]), h[1] = make_float2(f[2], f[3]);
        }
      }
      const float delta = part_of(delta4, i), du = part_of(du4, i);
      float2 B[2], C[2];
      pairs(*reinterpret_cast<const float4*>(s_bc + t * Ti::kN + n0), B);
      h[0] = fma2(ex2(mul2(both(delta), A2[0])), h[0], mul2(both(du), B[0]));
      h[1] = fma2(ex2(mul2(both(delta), A2[1])), h[1], mul2(both(du), B[1]));
      if (kEnds) {
        sum += delta;
      } else {
        pairs(*reinterpret_cast<const float4*>(s_bc + (Ti::kRows + t) * Ti::kN + n0), C);
        const float2 s = fma2(C[0], h[0], mul2(C[1], h[1]));
        y[i] = s.x + s.y;
        if (special && d.state && mine && s_end[t] >= 0) {
          const float f[kQuad] = {h[0].x, h[0].y, h[1].x, h[1].y};
          store_states(d.state, ((int64_t)p * a.q.S + s_end[t]) * d.D + ch, n0, d.N, f);
        }
      }
    }
    if (!kEnds) keep_sums<L, Ti>(y, s_delta, local, t4, lane);     // every lane of the channel has read these rows
  };
  for (int base = r.base; base < r.t1; base += Ti::kRows) {
    // stage
    if (threadIdx.x < Ti::kPieces) {
      float fx[8] = {}, fd[8] = {};
      if (live) {
        rx.get(fx);
        rdt.get(fd);
      }
#pragma unroll
      for (int v = 0; v < 8; ++v) {
        float e;
        const float delta = live ? softplus(fd[v] + bias[v], e) : 0.f;
        s_delta[Ti::at(piece + v, prow)] = delta;
        s_du[Ti::at(piece + v, prow)] = delta * fx[v];
      }
    }
    bc.store(s_bc);
    const bool is_plain = plain, was_live = live;
    if (!is_plain) mark_rows<Ti::kRows>(a, p, r, base, s_begin, s_end);
    const Pack<T, 8> kx = rx, kz = rz;
    __syncthreads();
    if (base + Ti::kRows < r.t1) fetch(base + Ti::kRows);
    if (is_plain) {
#pragma unroll 2
      for (int t4 = 0; t4 < Ti::kRows; t4 += 4) rows4(base, t4, std::false_type());
    } else {
#pragma unroll 1
      for (int t4 = 0; t4 < Ti::kRows; t4 += 4) rows4(base, t4, std::true_type());
    }
    __syncthreads();
    if (kEnds || !was_live) continue;
    // finish: the thread reads and later overwrites its own piece only
    float fx[8], fz[8], o[8];
    kx.get(fx);
    if (d.z.data) kz.get(fz);
#pragma unroll
    for (int v = 0; v < 8; ++v) {
      o[v] = fmaf(skip[v], fx[v], s_delta[Ti::at(piece + v, prow)]);
      if (d.z.data) o[v] *= fz[v] * sigmoid(fz[v]);
    }
    store8<T>(o, out.row(p, base + prow), pch, d.D, wide);
  }
  if (kEnds && mine) {
    const float f[kQuad] = {h[0].x, h[0].y, h[1].x, h[1].y};
    store_states(a.ends, chain_row, n0, d.N, f);
    if (n0 == 0) a.sums[chain_row] = fresh ? -1.f : sum;
  }
}

// Sequences of one row each: a thread takes 4 states of a channel of one sequence, read and written once.
template <typename T, int L>
__global__ void __launch_bounds__(kThreads) single_kernel(const __grid_constant__ Args a) {
  pdl_wait();
  pdl_launch_dependents();
  const int p = blockIdx.z, lane = threadIdx.x & 31;
  const lsgd_scan_desc& d = a.d;
  const int ch = blockIdx.x * (kThreads / L) + threadIdx.x / L, n0 = (threadIdx.x % L) * kQuad;
  const bool in = ch < d.D, mine = in && n0 < d.N;
  float A2[kQuad];
  decay_rates(a, p, ch, n0, A2);
  const float bias = vector_at(d.dt_bias, p, ch, in), skip = vector_at(d.skip, p, ch, in);
  auto one = [&](const lsgd_rows& m, int t, int i, bool there) {
    float f = 0.f;
    if (there) {
      Pack<T, 1> k;
      k.load(view<T>(m).row(p, t) + i);
      k.get(&f);
    }
    return f;
  };
  for (int t = blockIdx.y; t < a.q.S; t += gridDim.y) {
    const int64_t row = ((int64_t)p * a.q.S + t) * d.D + ch;
    float h[kQuad] = {};
    if (d.state && mine) load_states(d.state, row, n0, d.N, h);
    const float x = one(d.x, t, ch, in), z = one(d.z, t, ch, in && d.z.data);
    float e;
    const float delta = softplus(one(d.dt, t, ch, in) + bias, e), du = delta * x;
    float y = 0.f;
#pragma unroll
    for (int k = 0; k < kQuad; ++k) {
      const bool there = n0 + k < d.N;
      h[k] = fmaf(ex2(delta * A2[k]), h[k], du * one(d.b, t, n0 + k, there));
      y = fmaf(one(d.c, t, n0 + k, there), h[k], y);
    }
    if (d.state && mine) store_states(d.state, row, n0, d.N, h);
#pragma unroll
    for (int m = 1; m < L; m *= 2) y += __shfl_xor_sync(0xFFFFFFFFu, y, m);
    if (lane % L == 0 && in) {
      float o = fmaf(skip, x, y);
      if (d.z.data) o *= z * sigmoid(z);
      Pack<T, 1> k;
      k.set(&o);
      k.store(view<T>(d.out).row(p, t) + ch);
    }
  }
}

// ------------------------------------------------------------------------------------------------ backward
// Split chains: what the chain's rows add to the adjoint in front of it, and its summed time steps.
template <typename T, int L>
__global__ void __launch_bounds__(kThreads, 4) adjoint_kernel(const __grid_constant__ Args a) {
  using Ti = Tile<L, 1>;
  pdl_wait();
  pdl_launch_dependents();
  __shared__ __align__(16) float s_delta[Ti::kArray], s_d[Ti::kArray], s_bc[2 * Ti::kRows * Ti::kN];
  __shared__ int s_begin[Ti::kRows], s_end[Ti::kRows];
  const int p = blockIdx.z, c = blockIdx.y;
  const Range r(a, p, c);
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
  const bool wide = a.wide;
  const Rows<T> dt = view<T>(d.dt), z = view<T>(d.z), up = view<T>(d.d_out);
  float bias[8];
#pragma unroll
  for (int v = 0; v < 8; ++v) bias[v] = vector_at(d.dt_bias, p, pch + v, has_piece && pch + v < d.D);
  Pack<T, 8> rup, rdt, rz;
  StageBC<T, L, Ti> bc;
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
    bc.fetch(a, p, r, base, plain, false);
  };
  const int n_tiles = r.base < r.t1 ? (r.t1 - r.base + Ti::kRows - 1) / Ti::kRows : 0;
  if (n_tiles > 0) fetch(r.base + (n_tiles - 1) * Ti::kRows);
  for (int it = n_tiles - 1; it >= 0; --it) {
    const int base = r.base + it * Ti::kRows;
    if (threadIdx.x < Ti::kPieces) {
      float fu[8] = {}, fd[8] = {}, fz[8] = {};
      if (live) {
        rup.get(fu);
        rdt.get(fd);
        if (d.z.data) rz.get(fz);
      }
#pragma unroll
      for (int v = 0; v < 8; ++v) {
        float e;
        s_delta[Ti::at(piece + v, prow)] = live ? softplus(fd[v] + bias[v], e) : 0.f;
        s_d[Ti::at(piece + v, prow)] = d.z.data ? fu[v] * (fz[v] * sigmoid(fz[v])) : fu[v];
      }
    }
    bc.store(s_bc);
    const bool special = !plain;
    if (special) mark_rows<Ti::kRows>(a, p, r, base, s_begin, s_end);
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
        carry[0] = mul2(ex2(mul2(both(delta), A2[0])), fma2(C[0], both(g0), carry[0]));
        carry[1] = mul2(ex2(mul2(both(delta), A2[1])), fma2(C[1], both(g0), carry[1]));
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

// A thread takes two channels, a warp's lanes apart, so that B and C are read and dB and dC exchanged for both at once.
template <int L>
struct BackSmem {
  using Ti = Tile<L, 2>;
  static constexpr int kOwn = 8 * kThreads;                        // values of a thread's own piece, [value][thread]
  static constexpr int kPart = kThreads / 32 * kGroup * 8 * L;     // warps x rows x (4 dB, 4 dC) x L
  static constexpr size_t bytes = sizeof(float) * (6 * Ti::kArray + 3 * kOwn + 2 * Ti::kRows * Ti::kN + 2 * kPart) + 2 * sizeof(int) * Ti::kRows;
};
template <typename T, int L>
__global__ void __launch_bounds__(kThreads, 2) backward_kernel(const __grid_constant__ Args a) {
  using Ti = Tile<L, 2>;
  using Sm = BackSmem<L>;
  pdl_wait();
  pdl_launch_dependents();
  extern __shared__ __align__(16) float smem[];
  float* s_delta = smem;                                           // what the recurrence reads
  float* s_du = s_delta + Ti::kArray;
  float* s_d = s_du + Ti::kArray;
  float* s_qa = s_d + Ti::kArray;                                  // its sums over the states: q A log2(e), g B, C h
  float* s_gb = s_qa + Ti::kArray;
  float* s_y = s_gb + Ti::kArray;
  float* s_bc = s_y + Ti::kArray;
  float* s_part = s_bc + 2 * Ti::kRows * Ti::kN;
  float* s_x = s_part + 2 * Sm::kPart + threadIdx.x;               // the thread's own: x, the slopes of softplus and of the gate
  float* s_slope = s_x + Sm::kOwn;
  float* s_gate = s_slope + Sm::kOwn;
  int* s_begin = reinterpret_cast<int*>(s_part + 2 * Sm::kPart + 3 * Sm::kOwn);
  int* s_end = s_begin + Ti::kRows;
  const int p = blockIdx.z, c = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Range r(a, p, c);
  const lsgd_scan_desc& d = a.d;
  constexpr int kWarpCh = 32 / L;                                  // a thread's channels: this far apart
  const int local = warp * 2 * kWarpCh + lane / L, ch0 = blockIdx.x * Ti::kCh + local, n0 = (threadIdx.x % L) * kQuad;
  const bool states = n0 < d.N;
  const int64_t chain_row = ((int64_t)p * a.chains + c) * d.D;
  float2 A2[2][2], carry[2][2], dA[2][2] = {};                     // carry: a_(t+1) g_(t+1)
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int ch = ch0 + j * kWarpCh;
    float f[kQuad], g[kQuad] = {};
    decay_rates(a, p, ch, n0, f);
    if (a.split && states && ch < d.D) load_states(a.ends, chain_row + ch, n0, d.N, g);
    A2[j][0] = make_float2(f[0], f[1]), A2[j][1] = make_float2(f[2], f[3]);
    carry[j][0] = make_float2(g[0], g[1]), carry[j][1] = make_float2(g[2], g[3]);
  }
  const int prow = threadIdx.x / (Ti::kCh / 8), piece = (threadIdx.x % (Ti::kCh / 8)) * 8;
  const int pch = blockIdx.x * Ti::kCh + piece;
  const bool has_piece = threadIdx.x < Ti::kPieces && pch < d.D;
  const bool wide = a.wide;
  const Rows<T> x = view<T>(d.x), dt = view<T>(d.dt), z = view<T>(d.z), up = view<T>(d.d_out);
  float d_skip[8] = {}, d_bias[8] = {};
  Pack<T, 8> rx, rdt, rz, rup;
  constexpr bool kAhead = Ti::kQuads <= 2;
  StageBC<T, L, Ti> bc;
  bool live = false, plain = false;
  auto fetch = [&](int base) {
    const int t = base + prow;
    plain = r.plain(a, p, base, Ti::kRows);
    live = has_piece && (plain || row_lives(a, p, r, t));
    if (live) {
      load8<T>(rx, x.row(p, t), pch, d.D, wide);
      load8<T>(rdt, dt.row(p, t), pch, d.D, wide);
      load8<T>(rup, up.row(p, t), pch, d.D, wide);
      if (d.z.data) load8<T>(rz, z.row(p, t), pch, d.D, wide);
    }
    if (kAhead) bc.fetch(a, p, r, base, plain, true);
  };
  const int64_t groups = (a.q.T + kGroup - 1) / kGroup;
  const int n_tiles = r.base < r.t1 ? (r.t1 - r.base + Ti::kRows - 1) / Ti::kRows : 0;
  if (n_tiles > 0) fetch(r.base + (n_tiles - 1) * Ti::kRows);
  int buf = 0;
  // a group of 8 rows from row0 = base + g8
  auto group = [&](int base, int g8, auto special) {
    const int row0 = base + g8;
    float2 hs[kGroup][2][2], as[kGroup][2][2], first[2][2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float f[kQuad] = {};
      const int ch = ch0 + j * kWarpCh;
      if (states && ch < d.D && (!special || row0 >= r.t0)) load_states(d.saved, ((int64_t)p * groups + row0 / kGroup) * d.D + ch, n0, d.N, f);
      first[j][0] = make_float2(f[0], f[1]), first[j][1] = make_float2(f[2], f[3]);
    }
    float2 h[2][2] = {{first[0][0], first[0][1]}, {first[1][0], first[1][1]}};
#pragma unroll
    for (int half = 0; half < kGroup; half += 4) {
      float y[2][4];
      float4 delta4[2], du4[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        delta4[j] = *reinterpret_cast<const float4*>(s_delta + Ti::at(local + j * kWarpCh, g8 + half));
        du4[j] = *reinterpret_cast<const float4*>(s_du + Ti::at(local + j * kWarpCh, g8 + half));
      }
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const int i = half + i4, t = g8 + i;
        if (special && s_begin[t] >= 0) {
#pragma unroll
          for (int j = 0; j < 2; ++j) h[j][0] = h[j][1] = make_float2(0.f, 0.f);
        }
        float2 B[2], C[2];
        pairs(*reinterpret_cast<const float4*>(s_bc + t * Ti::kN + n0), B);
        pairs(*reinterpret_cast<const float4*>(s_bc + (Ti::kRows + t) * Ti::kN + n0), C);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 delta = both(part_of(delta4[j], i4)), du = both(part_of(du4[j], i4));
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            as[i][j][k] = ex2(mul2(delta, A2[j][k]));
            h[j][k] = fma2(as[i][j][k], h[j][k], mul2(du, B[k]));
            hs[i][j][k] = h[j][k];
          }
          const float2 s = fma2(C[0], h[j][0], mul2(C[1], h[j][1]));
          y[j][i4] = s.x + s.y;
        }
      }
      if (d.z.data) {
#pragma unroll
        for (int j = 0; j < 2; ++j) keep_sums<L, Ti>(y[j], s_y, local + j * kWarpCh, g8 + half, lane);
      }
    }
    float* part = s_part + buf * Sm::kPart + warp * kGroup * 8 * L;
    float2 sum_a[2][2] = {};                                       // of the group's rows
#pragma unroll
    for (int half = kGroup - 4; half >= 0; half -= 4) {
      float gb[2][4], qa[2][4];
      float4 delta4[2], du4[2], d4[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        delta4[j] = *reinterpret_cast<const float4*>(s_delta + Ti::at(local + j * kWarpCh, g8 + half));
        du4[j] = *reinterpret_cast<const float4*>(s_du + Ti::at(local + j * kWarpCh, g8 + half));
        d4[j] = *reinterpret_cast<const float4*>(s_d + Ti::at(local + j * kWarpCh, g8 + half));
      }
#pragma unroll
      for (int i4 = 3; i4 >= 0; --i4) {
        const int i = half + i4, t = g8 + i;
        const bool begins = special && s_begin[t] >= 0;
        float2 B[2], C[2], db[2], dc[2];
        pairs(*reinterpret_cast<const float4*>(s_bc + t * Ti::kN + n0), B);
        pairs(*reinterpret_cast<const float4*>(s_bc + (Ti::kRows + t) * Ti::kN + n0), C);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 delta = both(part_of(delta4[j], i4)), du = both(part_of(du4[j], i4)), dy = both(part_of(d4[j], i4));
          float2 sb = make_float2(0.f, 0.f), sq = sb;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float2 g = fma2(C[k], dy, carry[j][k]);
            db[k] = j == 0 ? mul2(g, du) : fma2(g, du, db[k]);
            dc[k] = j == 0 ? mul2(dy, hs[i][j][k]) : fma2(dy, hs[i][j][k], dc[k]);
            sb = k == 0 ? mul2(g, B[k]) : fma2(g, B[k], sb);
            carry[j][k] = mul2(as[i][j][k], g);
            float2 q = mul2(carry[j][k], i > 0 ? hs[i > 0 ? i - 1 : 0][j][k] : first[j][k]);
            if (begins) carry[j][k] = q = make_float2(0.f, 0.f);
            sum_a[j][k] = fma2(q, delta, sum_a[j][k]);
            sq = k == 0 ? mul2(q, A2[j][k]) : fma2(q, A2[j][k], sq);
          }
          gb[j][i4] = sb.x + sb.y;
          qa[j][i4] = sq.x + sq.y;
        }
        float v[8] = {db[0].x, db[0].y, db[1].x, db[1].y, dc[0].x, dc[0].y, dc[1].x, dc[1].y};
        ChannelSum<L>::run(v, lane);
        const int f = ChannelSum<L>::first(lane);
        if (8 * L > 16 || !(lane & (8 * L))) {
#pragma unroll
          for (int q = 0; q < ChannelSum<L>::kCount; ++q) part[(i * 8 + f + q) * L + lane % L] = v[q];
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        keep_sums<L, Ti>(gb[j], s_gb, local + j * kWarpCh, g8 + half, lane);
        keep_sums<L, Ti>(qa[j], s_qa, local + j * kWarpCh, g8 + half, lane);
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int k = 0; k < 2; ++k) dA[j][k] = make_float2(dA[j][k].x + sum_a[j][k].x, dA[j][k].y + sum_a[j][k].y);
    __syncthreads();
    // the block's sums over its channels, the warps' in order
#pragma unroll
    for (int i = threadIdx.x; i < kGroup * 8 * L; i += kThreads) {
      const int row = row0 + i / (8 * L), which = (i / L) % 8, n = (i % L) * kQuad + which % 4;
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < kThreads / 32; ++w) s += s_part[buf * Sm::kPart + w * kGroup * 8 * L + i];
      if (n < d.N && (!special || (row >= r.t0 && row < r.t1)))
        a.part_bc[((((int64_t)p * a.tiles + blockIdx.x) * a.q.T + row) * 2 + which / 4) * d.N + n] = s;
    }
    buf ^= 1;
  };
  for (int it = n_tiles - 1; it >= 0; --it) {
    const int base = r.base + it * Ti::kRows;
    if (threadIdx.x < Ti::kPieces) {
      float fx[8] = {}, fd[8] = {}, fu[8] = {}, fz[8] = {};
      if (live) {
        rx.get(fx);
        rdt.get(fd);
        rup.get(fu);
        if (d.z.data) rz.get(fz);
      }
#pragma unroll
      for (int v = 0; v < 8; ++v) {
        float e;
        const float pre = fd[v] + vector_at(d.dt_bias, p, pch + v, has_piece && pch + v < d.D), delta = live ? softplus(pre, e) : 0.f;
        const int o = Ti::at(piece + v, prow);
        s_delta[o] = delta;
        s_du[o] = delta * fx[v];
        s_x[v * kThreads] = fx[v];
        s_slope[v * kThreads] = live ? __fdividef(pre >= 0.f ? 1.f : e, 1.f + e) : 0.f;
        if (d.z.data) {
          const float sg = sigmoid(fz[v]), sl = fz[v] * sg;
          s_gate[v * kThreads] = fu[v] * fmaf(sl, 1.f - sg, sg);
          fu[v] *= sl;
        }
        s_d[o] = fu[v];
      }
    }
    if (!kAhead) bc.fetch(a, p, r, base, plain, true);
    bc.store(s_bc);
    const bool is_plain = plain, was_live = live;
    if (!is_plain) mark_rows<Ti::kRows>(a, p, r, base, s_begin, s_end);
    __syncthreads();
    if (it > 0) fetch(base - Ti::kRows);
    if (is_plain) {
#pragma unroll 1
      for (int g8 = Ti::kRows - kGroup; g8 >= 0; g8 -= kGroup) group(base, g8, std::false_type());
    } else {
#pragma unroll 1
      for (int g8 = Ti::kRows - kGroup; g8 >= 0; g8 -= kGroup)
        if (base + g8 < r.t1 && base + g8 + kGroup > r.t0) group(base, g8, std::true_type());      // the same for the whole block
    }
    // the last group's barrier has passed: every warp's sums are there
    if (was_live) {
      float o_x[8], o_dt[8], o_z[8];
#pragma unroll
      for (int v = 0; v < 8; ++v) {
        const int o = Ti::at(piece + v, prow);
        const float fx = s_x[v * kThreads], gB = s_gb[o], g = s_d[o];
        const float skip = vector_at(d.skip, p, pch + v, pch + v < d.D);
        o_x[v] = fmaf(s_delta[o], gB, skip * g);
        o_dt[v] = fmaf(fx, gB, s_qa[o] * kLn2) * s_slope[v * kThreads];
        if (d.z.data) o_z[v] = s_gate[v * kThreads] * fmaf(skip, fx, s_y[o]);
        d_skip[v] = fmaf(g, fx, d_skip[v]);
        d_bias[v] += o_dt[v];
      }
      const int t = base + prow;
      store8<T>(o_x, view<T>(d.dx).row(p, t), pch, d.D, wide);
      store8<T>(o_dt, view<T>(d.d_dt).row(p, t), pch, d.D, wide);
      if (d.z.data) store8<T>(o_z, view<T>(d.dz).row(p, t), pch, d.D, wide);
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int ch = ch0 + j * kWarpCh;
    if (!states || ch >= d.D) continue;
    float f[kQuad];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      f[2 * k] = dA[j][k].x * (A2[j][k].x * kLn2);
      f[2 * k + 1] = dA[j][k].y * (A2[j][k].y * kLn2);
    }
    store_states(a.part_a, chain_row + ch, n0, d.N, f);
  }
  // the rows' sums of d skip and d dt_bias, in order
  if (threadIdx.x < Ti::kPieces) {
#pragma unroll
    for (int v = 0; v < 8; ++v) {
      s_gb[Ti::at(piece + v, prow)] = d_skip[v];
      s_y[Ti::at(piece + v, prow)] = d_bias[v];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * Ti::kCh; i += kThreads) {
    const int which = i / Ti::kCh, ch = i % Ti::kCh;
    const float* src = which ? s_y : s_gb;
    float s = 0.f;
#pragma unroll 8
    for (int row = 0; row < Ti::kRows; ++row) s += src[Ti::at(ch, row)];
    const int col = blockIdx.x * Ti::kCh + ch;
    if (col < d.D) a.part_v[(((int64_t)p * a.chains + c) * 2 + which) * d.D + col] = s;
  }
}

// db and dc: the channel blocks' sums in order.
template <typename T>
__global__ void __launch_bounds__(256) join_bc_kernel(const __grid_constant__ Args a) {
  pdl_wait();
  pdl_launch_dependents();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n2 = 2 * a.d.N;
  const int p = blockIdx.y;
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
}

struct Launch {
  int L;
  bool single;
  dim3 grid, back;           // blocks of one and of two channels a thread
};
cudaError_t launch_forward_f32(const Args& a, const Launch& l, cudaStream_t s);
cudaError_t launch_forward_bf16(const Args& a, const Launch& l, cudaStream_t s);
cudaError_t launch_backward_f32(const Args& a, const Launch& l, cudaStream_t s);
cudaError_t launch_backward_bf16(const Args& a, const Launch& l, cudaStream_t s);
// split: from what every chain adds to what every chain starts from, forwards or backwards (scan.cu)
cudaError_t launch_chain_join(const Args& a, bool reverse, cudaStream_t s);

template <typename T, int L>
cudaError_t forward_of(const Args& a, const Launch& l, cudaStream_t s) {
  if (l.single) return launch_pdl(single_kernel<T, L>, l.grid, dim3(kThreads), 0, s, a);
  if (a.split) {
    cudaError_t e = launch_pdl(forward_kernel<T, L, true>, l.grid, dim3(kThreads), 0, s, a);
    if (e == cudaSuccess) e = launch_chain_join(a, false, s);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(forward_kernel<T, L, false>, l.grid, dim3(kThreads), 0, s, a);
}
template <typename T, int L>
cudaError_t backward_of(const Args& a, const Launch& l, cudaStream_t s) {
  constexpr size_t smem = BackSmem<L>::bytes;
  static OncePerDevice attr;
  if (!attr.here()) {
    const cudaError_t e = cudaFuncSetAttribute(backward_kernel<T, L>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    attr.here() = true;
  }
  cudaError_t e = cudaSuccess;
  if (a.split) {
    e = launch_pdl(adjoint_kernel<T, L>, l.grid, dim3(kThreads), 0, s, a);
    if (e == cudaSuccess) e = launch_chain_join(a, true, s);
  }
  if (e == cudaSuccess) e = launch_pdl(backward_kernel<T, L>, l.back, dim3(kThreads), smem, s, a);
  if (e != cudaSuccess) return e;
  const int64_t values = (int64_t)a.q.T * 2 * a.d.N;
  return launch_pdl(join_bc_kernel<T>, dim3((unsigned)((values + 255) / 256), a.d.P), dim3(256), 0, s, a);
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
