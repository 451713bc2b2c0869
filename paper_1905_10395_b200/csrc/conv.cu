// Short causal convolution of every channel along its sequences, and its gradient (include/lsgd.h).
//
// A thread owns `VEC` neighbouring channels of a run of rows and keeps the last W - 1 inputs in registers, so each input is read
// once (and W - 1 rows again where a run begins) and each output written once: the operator is bound by memory.  The next rows are
// fetched while the present ones are used (8 x 2048 x 2048 in bf16: 31 us forward, 38 with one set of rows in flight; 21 at the rate
// of a copy; a ring of 16 rows in shared memory, copied asynchronously: 34 and 75 backward), and a run's rows are found span by
// span of a sequence, not row by row.
//
// The gradient walks W - 1 rows further than its run: row t's d = d_out act'(pre) is made from the window of inputs and added to
// the W sums dx[t - k] that wait in registers; the sums of dw and d_bias stay in registers over the run, are added up by
// the block and then by a second kernel in a fixed order (56 us for the above; 31 at the rate of a copy).
#include <type_traits>

#include "activations.h"
#include "seq.h"

namespace lsgd {
namespace {

constexpr int kMaxW = 4, kAhead = 8, kLanes = 32, kRuns = 4;       // a block: 32 channel pieces x 4 runs of rows
constexpr int kMostRows = 64;                                      // of a run
// Blocks of a kernel that are resident on an SM: as many as leave a thread the registers for two sets of rows in flight.
constexpr int forward_blocks(int vec) { return vec == 4 ? 5 : 7; }
constexpr int backward_blocks(int vec) { return vec == 2 ? 5 : 4; }

__global__ void __launch_bounds__(256) codes_kernel(const SeqView q, int32_t* codes) {
  pdl_wait();
  pdl_launch_dependents();
  const int p = blockIdx.y, t = blockIdx.x * 256 + threadIdx.x;
  if (t >= q.T) return;
  int lo = 0, hi = q.S + 1;                      // edges at or before t: [0, lo); behind t: [hi, S]
  while (lo < hi) {
    const int mid = lo + ((hi - lo) >> 1);       // (lo + hi may pass 2^31)
    if (q.edge(p, mid) <= t) lo = mid + 1; else hi = mid;
  }
  codes[(int64_t)p * q.T + t] = lo == 0 || lo > q.S ? -1 : lo - 1;
}

struct ConvArgs {
  lsgd_conv_desc d;
  SeqView q;
  int32_t run;               // rows of a thread
  float* part;               // [P][blocks of rows][D][W + 1]
  uint32_t blocks_t;
};

template <typename T>
__device__ __forceinline__ Rows<T> view(const lsgd_rows& r) {
  return Rows<T>{static_cast<T*>(r.data), r.ld, r.stride};
}

// VEC (4, 2 or 1) neighbouring values as pairs, two to an instruction (of a single value the second is idle).
template <int VEC>
struct Vals {
  static constexpr int kPairs = (VEC + 1) / 2;
  float2 v[kPairs];
};
template <typename T, int VEC>
__device__ __forceinline__ Vals<VEC> values(const Pack<T, VEC>& k) {
  float f[VEC + 1];
  k.get(f);
  if (VEC == 1) f[1] = 0.f;
  Vals<VEC> r;
#pragma unroll
  for (int i = 0; i < Vals<VEC>::kPairs; ++i) r.v[i] = make_float2(f[2 * i], f[2 * i + 1]);
  return r;
}
template <typename T, int VEC>
__device__ __forceinline__ void put(const Vals<VEC>& r, T* to) {
  float f[VEC + 1];
#pragma unroll
  for (int i = 0; i < Vals<VEC>::kPairs; ++i) f[2 * i] = r.v[i].x, f[2 * i + 1] = r.v[i].y;
  Pack<T, VEC> k;
  k.set(f);
  k.store(to);
}
// A thread's weights: tap j multiplies the input W - 1 - j rows back.  (The number of taps is a template parameter: a weight of zero
// would not keep an infinite input out.)
template <int VEC, int W>
struct Taps {
  Vals<VEC> w[W], bias;
  __device__ __forceinline__ void load(const lsgd_conv_desc& d, int p, int ch) {
    const float* wp = static_cast<const float*>(d.w.data) + p * d.w.stride + ch * d.w.ld;
    const float* bp = static_cast<const float*>(d.bias.data) + p * d.bias.stride + ch;
#pragma unroll
    for (int i = 0; i < Vals<VEC>::kPairs; ++i) {
      const bool x = ch + 2 * i < d.D, y = VEC > 1 && ch + 2 * i + 1 < d.D;
#pragma unroll
      for (int j = 0; j < W; ++j) w[j].v[i] = make_float2(x ? wp[2 * i * d.w.ld + j] : 0.f, y ? wp[(2 * i + 1) * d.w.ld + j] : 0.f);
      bias.v[i] = make_float2(x && d.bias.data ? bp[2 * i] : 0.f, y && d.bias.data ? bp[2 * i + 1] : 0.f);
    }
  }
  // win[0 .. W - 2]: the inputs in front of a row, oldest first; last: the row's own
  __device__ __forceinline__ Vals<VEC> apply(const Vals<VEC> (&win)[W], const Vals<VEC>& last) const {
    Vals<VEC> s = bias;
#pragma unroll
    for (int i = 0; i < Vals<VEC>::kPairs; ++i) {
#pragma unroll
      for (int j = 0; j < W - 1; ++j) s.v[i] = fma2(w[j].v[i], win[j].v[i], s.v[i]);
      s.v[i] = fma2(w[W - 1].v[i], last.v[i], s.v[i]);
    }
    return s;
  }
};
template <int VEC>
__device__ __forceinline__ Vals<VEC> activate(Vals<VEC> s, bool silu) {
  if (silu) {
#pragma unroll
    for (int i = 0; i < Vals<VEC>::kPairs; ++i) s.v[i] = mul2(s.v[i], sigmoid(s.v[i]));
  }
  return s;
}

// The W - 1 inputs in front of row t (oldest first) of its own sequence, whose rows begin at lo, from the rows or the state; zeros
// where there is none.
template <typename T, int VEC, int W>
__device__ __forceinline__ void window(const ConvArgs& a, int p, int t, int ch, const SeqView::Span& q, Vals<VEC> (&win)[W]) {
  const Rows<T> x = view<T>(a.d.x);
  const T* state = static_cast<const T*>(a.d.state);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) {
    const int row = t - (W - 1) + j;
    Pack<T, VEC> k;
    const float zero[VEC] = {};
    if (row >= q.lo) k.load(x.row(p, row) + ch);
    else if (state) k.load(state + (((int64_t)p * a.q.S + q.code) * (W - 1) + (row - q.lo + W - 1)) * a.d.D + ch);
    else k.set(zero);
    win[j] = values<T, VEC>(k);
  }
}

template <typename T, int VEC, int W>
__global__ void __launch_bounds__(kLanes * kRuns, forward_blocks(VEC)) conv_forward_kernel(const __grid_constant__ ConvArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int ch = (blockIdx.x * kLanes + threadIdx.x) * VEC, p = blockIdx.z;
  int t = (blockIdx.y * kRuns + threadIdx.y) * a.run;
  const int t1 = min(a.q.T, t + a.run);
  if (ch >= a.d.D || t >= t1) return;
  const bool silu = a.d.act == LSGD_CONV_SILU;
  const int64_t ldx = a.d.x.ld, ldo = a.d.out.ld;
  Taps<VEC, W> taps;
  taps.load(a.d, p, ch);
  while (t < t1) {
    const SeqView::Span q = a.q.span(p, t);
    const int end = min(t1, q.hi);
    if (q.code < 0) {
      t = end;
      continue;
    }
    Vals<VEC> win[W];
    window<T, VEC, W>(a, p, t, ch, q, win);
    const T* px = view<T>(a.d.x).row(p, t) + ch;
    T* po = view<T>(a.d.out).row(p, t) + ch;
    Pack<T, VEC> next[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (t + i < end) next[i].load(px + i * ldx);
    for (; t < end; t += kAhead) {
      Pack<T, VEC> in[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        in[i] = next[i];
        if (t + kAhead + i < end) next[i].load(px + (kAhead + i) * ldx);
      }
      auto row = [&](int i) {
        const Vals<VEC> last = values<T, VEC>(in[i]);
        put<T, VEC>(activate(taps.apply(win, last), silu), po + i * ldo);
#pragma unroll
        for (int j = 0; j + 1 < W - 1; ++j) win[j] = win[j + 1];
        if (W > 1) win[W > 1 ? W - 2 : 0] = last;
      };
      if (t + kAhead <= end) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) row(i);
      } else {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          if (t + i >= end) break;
          row(i);
        }
      }
      px += kAhead * ldx;
      po += kAhead * ldo;
    }
    t = end;
  }
}

// The states behind the sequences: a thread takes VEC channels of one sequence, all of whose kept inputs it reads before it writes.
// SINGLE, for sequences of one row each: the row's output as well, in one launch.
template <typename T, int VEC, int W, bool SINGLE>
__global__ void __launch_bounds__(kLanes * kRuns) conv_state_kernel(const __grid_constant__ ConvArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int ch = (blockIdx.x * kLanes + threadIdx.x) * VEC, p = blockIdx.z;
  if (ch >= a.d.D) return;
  const Rows<T> x = view<T>(a.d.x);
  for (int s = blockIdx.y * kRuns + threadIdx.y; s < a.q.S; s += gridDim.y * kRuns) {
    const int lo = a.q.edge(p, s), n = a.q.edge(p, s + 1) - lo;
    if (n <= 0) continue;
    T* state = a.d.state ? static_cast<T*>(a.d.state) + ((int64_t)p * a.q.S + s) * (W - 1) * a.d.D + ch : nullptr;
    // inputs `from` on of the old state with the sequence behind it; the single row's window begins with the state's first
    const int from = SINGLE ? 0 : n;
    constexpr int kTake = SINGLE ? W : W - 1;
    Pack<T, VEC> kept[W];
#pragma unroll
    for (int k = 0; k < kTake; ++k) {
      const int i = from + k;
      const float zero[VEC] = {};
      if (i >= W - 1) kept[k].load(x.row(p, lo + i - (W - 1)) + ch);
      else if (state) kept[k].load(state + (int64_t)i * a.d.D);
      else kept[k].set(zero);
    }
    if (SINGLE) {
      Taps<VEC, W> taps;
      taps.load(a.d, p, ch);
      Vals<VEC> win[W];
#pragma unroll
      for (int k = 0; k < W; ++k) win[k] = values<T, VEC>(kept[k]);
      put<T, VEC>(activate(taps.apply(win, win[W - 1]), a.d.act == LSGD_CONV_SILU), view<T>(a.d.out).row(p, lo) + ch);
    }
    if (!state) continue;
#pragma unroll
    for (int k = 0; k < W - 1; ++k) kept[k + SINGLE].store(state + (int64_t)k * a.d.D);
  }
}

template <typename T, int VEC, int W>
__global__ void __launch_bounds__(kLanes * kRuns, backward_blocks(VEC)) conv_backward_kernel(const __grid_constant__ ConvArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int kPairs = Vals<VEC>::kPairs, kTake = VEC * sizeof(T) <= 4 ? 8 : 4;      // rows a set
  const int ch = (blockIdx.x * kLanes + threadIdx.x) * VEC, p = blockIdx.z;
  int t = (blockIdx.y * kRuns + threadIdx.y) * a.run;
  const int t1 = min(a.q.T, t + a.run);
  const bool silu = a.d.act == LSGD_CONV_SILU;
  Vals<VEC> dw[W] = {}, db = {};
  if (ch < a.d.D && t < t1) {
    const int64_t ldx = a.d.x.ld, ldu = a.d.d_out.ld, ldd = a.d.dx.ld;
    Taps<VEC, W> taps;
    taps.load(a.d, p, ch);
    while (t < t1) {
      const SeqView::Span q = a.q.span(p, t);
      const int own = min(t1, q.hi), end = min(q.hi, t1 + W - 1);       // rows of this run; rows that reach into it
      if (q.code < 0) {
        t = own;
        continue;
      }
      Vals<VEC> win[W], wait[W] = {};              // wait[j]: dx of row t - (W - 1) + j as far as it is known
      window<T, VEC, W>(a, p, t, ch, q, win);
      const int first = t;                         // dx of the rows in front belongs to another thread
      const T* px = view<T>(a.d.x).row(p, t) + ch;
      const T* pu = view<T>(a.d.d_out).row(p, t) + ch;
      T* pd = view<T>(a.d.dx).row(p, t) + ch;
      Pack<T, VEC> next_in[kTake], next_up[kTake];
#pragma unroll
      for (int i = 0; i < kTake; ++i)
        if (t + i < end) {
          next_in[i].load(px + i * ldx);
          next_up[i].load(pu + i * ldu);
        }
      for (; t < end; t += kTake) {
        Pack<T, VEC> in[kTake], up[kTake];
#pragma unroll
        for (int i = 0; i < kTake; ++i) {
          in[i] = next_in[i], up[i] = next_up[i];
          if (t + kTake + i < end) {
            next_in[i].load(px + (kTake + i) * ldx);
            next_up[i].load(pu + (kTake + i) * ldu);
          }
        }
        // row t + i; plain: it is this run's, as is the row W - 1 before it
        auto row = [&](int i, auto plain) {
          const Vals<VEC> last = values<T, VEC>(in[i]);
          Vals<VEC> g = values<T, VEC>(up[i]);
          if (silu) {
            const Vals<VEC> s = taps.apply(win, last);
#pragma unroll
            for (int v = 0; v < kPairs; ++v) {
              const float2 sg = sigmoid(s.v[v]), sl = mul2(s.v[v], sg);
              g.v[v] = mul2(g.v[v], fma2(sl, fma2(sg, both(-1.f), both(1.f)), sg));
            }
          }
          const bool mine = plain || t + i < own;
#pragma unroll
          for (int v = 0; v < kPairs; ++v) {
#pragma unroll
            for (int j = 0; j < W - 1; ++j) wait[j].v[v] = fma2(taps.w[j].v[v], g.v[v], wait[j].v[v]);
            wait[W - 1].v[v] = mul2(taps.w[W - 1].v[v], g.v[v]);
            if (mine) {
              db.v[v] = add2(db.v[v], g.v[v]);
#pragma unroll
              for (int j = 0; j < W - 1; ++j) dw[j].v[v] = fma2(win[j].v[v], g.v[v], dw[j].v[v]);
              dw[W - 1].v[v] = fma2(last.v[v], g.v[v], dw[W - 1].v[v]);
            }
          }
          if (plain || t + i - (W - 1) >= first) put<T, VEC>(wait[0], pd + (i - (W - 1)) * ldd);      // complete W - 1 rows on
#pragma unroll
          for (int j = 0; j + 1 < W; ++j) wait[j] = wait[j + 1];
#pragma unroll
          for (int j = 0; j + 1 < W - 1; ++j) win[j] = win[j + 1];
          if (W > 1) win[W > 1 ? W - 2 : 0] = last;
        };
        if (t - (W - 1) >= first && t + kTake <= own) {
#pragma unroll
          for (int i = 0; i < kTake; ++i) row(i, std::true_type());
        } else {
#pragma unroll
          for (int i = 0; i < kTake; ++i) {
            if (t + i >= end) break;
            row(i, std::false_type());
          }
        }
        px += kTake * ldx;
        pu += kTake * ldu;
        pd += kTake * ldd;
      }
      // the rows that wait are complete where their sequence ends
      if (end == q.hi) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
          const int row = end - (W - 1) + j;
          if (row >= first && row < own) put<T, VEC>(wait[j], view<T>(a.d.dx).row(p, row) + ch);
        }
      }
      t = own;
    }
  }
  // the block's sums: the runs' in order
  __shared__ float sums[kRuns][kLanes * VEC];
#pragma unroll
  for (int j = 0; j <= W; ++j) {
    __syncthreads();
    const Vals<VEC>& mine = j < W ? dw[j < W ? j : 0] : db;
#pragma unroll
    for (int v = 0; v < VEC; ++v) sums[threadIdx.y][threadIdx.x * VEC + v] = v % 2 ? mine.v[v / 2].y : mine.v[v / 2].x;
    __syncthreads();
    for (int i = threadIdx.y * kLanes + threadIdx.x; i < kLanes * VEC; i += kLanes * kRuns) {
      const int c = blockIdx.x * kLanes * VEC + i;
      if (c >= a.d.D) continue;
      float s = 0.f;
#pragma unroll
      for (int r = 0; r < kRuns; ++r) s += sums[r][i];
      a.part[(((int64_t)p * a.blocks_t + blockIdx.y) * a.d.D + c) * (W + 1) + j] = s;
    }
  }
}

// Adds the blocks' sums in order: columns of a worker (of all workers where they share the vector), a thread a column where there are
// few sums of each (SPLIT 1), else 8 warps 32 columns.
template <int SPLIT>
__global__ void __launch_bounds__(256) conv_join_kernel(const __grid_constant__ ConvArgs a) {
  pdl_wait();
  const int per = a.d.W + 1, n = a.d.D * per;
  const int part = SPLIT == 1 ? 0 : threadIdx.x >> 5;
  const int i = SPLIT == 1 ? blockIdx.x * 256 + threadIdx.x : blockIdx.x * 32 + (threadIdx.x & 31);
  __shared__ float s[SPLIT][33];
  const int k = i % per, c = i / per;
  const lsgd_rows& o = k < a.d.W ? a.d.dw : a.d.d_bias;
  const bool shared = a.d.P > 1 && o.stride == 0, idle = i >= n || !o.data || (shared && blockIdx.y > 0);
  const uint32_t rows = a.blocks_t, share = (rows + SPLIT - 1) / SPLIT, r0 = min(rows, part * share), r1 = min(rows, r0 + share);
  float total = 0.f;
  if (!idle) {
    for (int p = shared ? 0 : blockIdx.y, last = shared ? a.d.P - 1 : p; p <= last; ++p) {
      const float* src = a.part + (int64_t)p * rows * n + i;
#pragma unroll 8
      for (uint32_t r = r0; r < r1; ++r) total += src[(int64_t)r * n];
    }
  }
  if (SPLIT > 1) {
    s[part][threadIdx.x & 31] = total;
    __syncthreads();
    if (part > 0) return;
    total = 0.f;
    for (int q = 0; q < SPLIT; ++q) total += s[q][threadIdx.x & 31];
  }
  if (idle) return;
  float* dst = static_cast<float*>(o.data) + (shared ? 0 : blockIdx.y * o.stride) + (k < a.d.W ? c * o.ld + k : c);
  *dst = a.d.accumulate ? *dst + total : total;
}

// ------------------------------------------------------------------------------------------------ host
lsgd_status check_conv(const lsgd_conv_desc* d, bool backward) {
  if (!d || d->struct_size != sizeof(lsgd_conv_desc)) return LSGD_ERR_INVALID_ARG;
  if (d->P < 1 || d->T < 0 || d->D < 1 || d->W < 1) return LSGD_ERR_INVALID_ARG;
  if (d->act_dtype < LSGD_F32 || d->act_dtype > LSGD_BF16 || d->act < LSGD_CONV_IDENTITY || d->act > LSGD_CONV_SILU) return LSGD_ERR_INVALID_ARG;
  if (d->D > 65536 || d->W > kMaxW || d->P > 65535) return LSGD_ERR_UNSUPPORTED;
  if (d->T >= kMaxRows / d->P) return LSGD_ERR_TOO_LARGE;
  lsgd_status st;
  if ((st = check_sequences(d->seq, d->P, d->T)) != LSGD_OK) return st;
  const int64_t P = d->P, T = d->T, D = d->D;
  const int ab = elem_bytes(d->act_dtype);
  const bool rows = T > 0;
  if (!d->w.data || (rows && !d->x.data)) return LSGD_ERR_INVALID_ARG;
#define LSGD_ROWS(r, t, w, bytes, written, shared)                                                 \
  do {                                                                                            \
    if ((r).data && (st = check_rows(r, P, t, w, bytes, written, shared)) != LSGD_OK) return st;  \
  } while (0)
  LSGD_ROWS(d->x, T, D, ab, false, false);
  LSGD_ROWS(d->w, D, d->W, 4, false, false);
  LSGD_ROWS(d->bias, 1, D, 4, false, false);
  if (!backward) {
    if (rows && !d->out.data) return LSGD_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(d->state) % ab) return LSGD_ERR_ALIGNMENT;
    LSGD_ROWS(d->out, T, D, ab, true, false);
    const Extent ins[] = {extent(d->x, P, T, D, ab), extent(d->w, P, D, d->W, 4), extent(d->bias, P, 1, D, 4)};
    const Extent outs[] = {extent(d->out, P, T, D, ab), extent({d->state, D, (int64_t)d->seq.S * (d->W - 1) * D}, P, (int64_t)d->seq.S * (d->W - 1), D, ab)};
    return all_apart(outs, 2, ins, 3) ? LSGD_OK : LSGD_ERR_INVALID_ARG;
  }
  if (d->state) return LSGD_ERR_INVALID_ARG;
  if (rows && (!d->d_out.data || !d->dx.data)) return LSGD_ERR_INVALID_ARG;
  if (!d->dw.data || (d->bias.data != nullptr) != (d->d_bias.data != nullptr)) return LSGD_ERR_INVALID_ARG;
  LSGD_ROWS(d->d_out, T, D, ab, false, false);
  LSGD_ROWS(d->dx, T, D, ab, true, false);
  LSGD_ROWS(d->dw, D, d->W, 4, true, true);
  LSGD_ROWS(d->d_bias, 1, D, 4, true, true);
#undef LSGD_ROWS
  const Extent ins[] = {extent(d->x, P, T, D, ab), extent(d->d_out, P, T, D, ab), extent(d->w, P, D, d->W, 4), extent(d->bias, P, 1, D, 4)};
  const Extent outs[] = {extent(d->dx, P, T, D, ab), extent(d->dw, P, D, d->W, 4), extent(d->d_bias, P, 1, D, 4)};
  return all_apart(outs, 3, ins, 4) ? LSGD_OK : LSGD_ERR_INVALID_ARG;
}

// Values a thread: 8 bytes of a row where every row allows it (of fp32, four would not fit the registers: 8 x 2048 x 2048 took 66 + 129
// us instead of 46 + 77).  In bf16 two do where four leave SMs with few blocks (8 x 1024 x 512: 8.5 + 15 us instead of 6.1
// + 13.5; 3 x 1000 x 256: 4.4 + 11 instead of 3.6 + 10).
int conv_vec(const lsgd_conv_desc* d, bool backward) {
  const int ab = elem_bytes(d->act_dtype);
  auto fits = [&](const lsgd_rows& r, int v) {
    return !r.data || (reinterpret_cast<uintptr_t>(r.data) % (v * ab) == 0 && (d->T <= 1 || r.ld % v == 0) && (d->P <= 1 || r.stride % v == 0));
  };
  auto all = [&](int v) {
    return d->D % v == 0 && fits(d->x, v) &&
           (backward ? fits(d->d_out, v) && fits(d->dx, v) : fits(d->out, v) && reinterpret_cast<uintptr_t>(d->state) % (v * ab) == 0);
  };
  const int64_t blocks = (d->D + kLanes * 4 - 1) / (kLanes * 4) * d->P * ((d->T + 8 * kRuns - 1) / (8 * kRuns));      // of 8 rows a thread
  return ab == 2 && blocks >= 32 * sm_count() && all(4) ? 4 : all(2) ? 2 : 1;
}

struct ConvPlan {
  int vec, run, join;        // values and rows of a thread; warps of a last sum
  uint32_t blocks_d, blocks_t;
};
ConvPlan conv_plan(const lsgd_conv_desc* d, bool backward) {
  ConvPlan c{};
  c.vec = conv_vec(d, backward);
  c.blocks_d = (uint32_t)((d->D + kLanes * c.vec - 1) / (kLanes * c.vec));
  // rows of a thread: those that take the least time by the rounds of blocks over the machine, each of as many rows and what a run
  // begins with.  Forwards by whole rounds; backwards, where a run begins and ends with more, between whole rounds and their fraction, and
  // powers of two, which seldom cross from one sequence to the next (8 x 2048 x 2048 in two sequences each: 56 us with runs of 64 rows, 64 with
  // 40, 62 with 32)
  const int64_t resident = (int64_t)sm_count() * (backward ? backward_blocks(c.vec) : forward_blocks(c.vec)), columns = (int64_t)c.blocks_d * d->P;
  int64_t least = INT64_MAX;
  for (int run = 8; run <= kMostRows; run = backward ? 2 * run : run + 8) {
    const int64_t blocks = columns * ((d->T + (int64_t)run * kRuns - 1) / ((int64_t)run * kRuns)), rounds = (blocks + resident - 1) / resident;
    const int64_t cost = backward ? (rounds * resident + blocks) * (run + 16) : rounds * (run + d->W + 2);
    if (cost < least) {
      least = cost;
      c.run = run;
    }
  }
  // no more than 65535 blocks of rows (gridDim.y)
  while ((d->T + (int64_t)c.run * kRuns - 1) / ((int64_t)c.run * kRuns) > 65535) c.run *= 2;
  c.blocks_t = (uint32_t)((d->T + (int64_t)c.run * kRuns - 1) / ((int64_t)c.run * kRuns));
  c.join = !backward ? 0 : c.blocks_t <= 32 ? 1 : 8;
  return c;
}

template <typename T, int VEC, int W>
cudaError_t launch_conv(const ConvArgs& a, const ConvPlan& c, bool backward, cudaStream_t s) {
  const dim3 block(kLanes, kRuns), grid(c.blocks_d, c.blocks_t, a.d.P);
  if (backward) return launch_pdl(conv_backward_kernel<T, VEC, W>, grid, block, 0, s, a);
  const int64_t groups = (a.q.S + kRuns - 1) / kRuns;
  const dim3 states(c.blocks_d, (unsigned)(groups < 65535 ? groups : 65535), a.d.P);
  if (!a.q.starts && a.q.len == 1) return launch_pdl(conv_state_kernel<T, VEC, W, true>, states, block, 0, s, a);
  const cudaError_t e = launch_pdl(conv_forward_kernel<T, VEC, W>, grid, block, 0, s, a);
  if (e != cudaSuccess || !a.d.state || W == 1) return e;
  // in a launch of its own: other threads read the states of the first rows above
  return launch_pdl(conv_state_kernel<T, VEC, W, false>, states, block, 0, s, a);
}
template <typename T, int VEC>
cudaError_t launch_conv(const ConvArgs& a, const ConvPlan& c, bool backward, cudaStream_t s) {
  switch (a.d.W) {
    case 1: return launch_conv<T, VEC, 1>(a, c, backward, s);
    case 2: return launch_conv<T, VEC, 2>(a, c, backward, s);
    case 3: return launch_conv<T, VEC, 3>(a, c, backward, s);
    default: return launch_conv<T, VEC, 4>(a, c, backward, s);
  }
}

lsgd_status run_conv(const lsgd_conv_desc* d, bool backward, cudaStream_t s) {
  const ConvPlan c = conv_plan(d, backward);
  int32_t* codes = static_cast<int32_t*>(d->scratch);
  ConvArgs a{};
  a.d = *d;
  a.q = seq_view(d->seq, d->T, codes);
  a.run = c.run;
  a.blocks_t = c.blocks_t;
  a.part = reinterpret_cast<float*>(static_cast<char*>(d->scratch) + codes_bytes(d->seq, d->P, d->T));
  cudaError_t e = cudaSuccess;
  if (d->T > 0) {
    if (d->seq.starts) e = launch_codes(a.q, codes, d->P, s);
    if (e == cudaSuccess)
      e = d->act_dtype == LSGD_F32 ? (c.vec == 2 ? launch_conv<float, 2>(a, c, backward, s) : launch_conv<float, 1>(a, c, backward, s))
          : c.vec == 4             ? launch_conv<__nv_bfloat16, 4>(a, c, backward, s)
          : c.vec == 2             ? launch_conv<__nv_bfloat16, 2>(a, c, backward, s)
                                   : launch_conv<__nv_bfloat16, 1>(a, c, backward, s);
  }
  if (e == cudaSuccess && backward) {
    const unsigned n = (unsigned)d->D * (d->W + 1);
    e = c.join == 1      ? launch_pdl(conv_join_kernel<1>, dim3((n + 255) / 256, d->P), dim3(256), 0, s, a)
                         : launch_pdl(conv_join_kernel<8>, dim3((n + 31) / 32, d->P), dim3(256), 0, s, a);
  }
  return e == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
}

}  // namespace

cudaError_t launch_codes(const SeqView& q, int32_t* codes, int32_t P, cudaStream_t s) {
  return launch_pdl(codes_kernel, dim3((q.T + 255) / 256, P), dim3(256), 0, s, q, codes);
}

}  // namespace lsgd

extern "C" {

uint64_t lsgd_conv_scratch_bytes(const lsgd_conv_desc* d, int32_t backward) {
  using namespace lsgd;
  if (!d || d->struct_size != sizeof(lsgd_conv_desc) || d->P < 1 || d->T < 0 || d->D < 1 || d->D > 65536 || d->W < 1 || d->W > kMaxW ||
      d->act_dtype < LSGD_F32 || d->act_dtype > LSGD_BF16 || d->T >= kMaxRows / d->P)
    return 0;
  uint64_t n = codes_bytes(d->seq, d->P, d->T);
  if (backward) n += sizeof(float) * (uint64_t)d->P * conv_plan(d, true).blocks_t * d->D * (d->W + 1);
  return align256(n);
}

lsgd_status lsgd_conv_plan(const lsgd_conv_desc* d, int32_t backward, int32_t plan[3]) {
  using namespace lsgd;
  const lsgd_status st = check_conv(d, backward);
  if (st != LSGD_OK || !plan) return st != LSGD_OK ? st : LSGD_ERR_INVALID_ARG;
  const ConvPlan c = conv_plan(d, backward);
  plan[0] = c.vec, plan[1] = c.run, plan[2] = c.join;
  return LSGD_OK;
}

#define LSGD_CONV_CALL(name, backward)                                                            \
  lsgd_status name(const lsgd_conv_desc* d, void* stream) {                                       \
    using namespace lsgd;                                                                         \
    const lsgd_status st = check_conv(d, backward);                                               \
    if (st != LSGD_OK) return st;                                                                 \
    const uint64_t need = lsgd_conv_scratch_bytes(d, backward);                                   \
    if (need && (!d->scratch || d->scratch_bytes < need)) return LSGD_ERR_INVALID_ARG;            \
    if (need && reinterpret_cast<uintptr_t>(d->scratch) % 256) return LSGD_ERR_ALIGNMENT;         \
    return run_conv(d, backward, static_cast<cudaStream_t>(stream));                              \
  }
LSGD_CONV_CALL(lsgd_conv_forward, false)
LSGD_CONV_CALL(lsgd_conv_backward, true)
#undef LSGD_CONV_CALL

}  // extern "C"
