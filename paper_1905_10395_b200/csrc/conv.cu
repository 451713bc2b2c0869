// Short causal convolution of every channel along its sequences, and its gradient (include/lsgd.h).
//
// A thread owns `VEC` neighbouring channels of a run of rows and keeps the last W - 1 inputs in registers, so each input is read
// once (and W - 1 rows again where a run begins) and each output written once: the operator is bound by memory.  Rows are
// fetched kAhead at a time before the first of them is used.
//
// The gradient walks W - 1 rows further than its run: row t's d = d_out act'(pre) is made from the window of inputs and added to
// the W sums dx[t - k] that wait in registers; the sums of dw and d_bias stay in registers over the run, are added up by
// the block and then by a second kernel in a fixed order.
#include "seq.h"

namespace lsgd {
namespace {

constexpr int kMaxW = 4, kAhead = 8, kLanes = 32, kRuns = 4;       // a block: 32 channel pieces x 4 runs of rows
constexpr int kBackRun = 64;                                       // rows of a backward run at most

__global__ void __launch_bounds__(256) codes_kernel(const SeqView q, int32_t* codes) {
  pdl_wait();
  pdl_launch_dependents();
  const int p = blockIdx.y, t = blockIdx.x * 256 + threadIdx.x;
  if (t >= q.T) return;
  int lo = 0, hi = q.S + 1;                      // edges at or before t: [0, lo); behind t: [hi, S]
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
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

// pre and its factor: out = pre * s, d out / d pre = s + pre s (1 - s)
__device__ __forceinline__ float sigmoid(float v) { return __fdividef(1.f, 1.f + __expf(-v)); }

// A thread's weights: tap j multiplies the input W - 1 - j rows back.  (The number of taps is a template parameter: a weight of zero
// would not keep an infinite input out.)
template <int VEC, int W>
struct Taps {
  float w[W][VEC], bias[VEC];
  __device__ __forceinline__ void load(const lsgd_conv_desc& d, int p, int ch) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const bool in = ch + v < d.D;
#pragma unroll
      for (int j = 0; j < W; ++j) w[j][v] = in ? static_cast<const float*>(d.w.data)[p * d.w.stride + (ch + v) * d.w.ld + j] : 0.f;
      bias[v] = in && d.bias.data ? static_cast<const float*>(d.bias.data)[p * d.bias.stride + ch + v] : 0.f;
    }
  }
};

template <typename T, int VEC>
__device__ __forceinline__ void fetch(const T* row, int ch, float (&f)[VEC]) {
  Pack<T, VEC> k;
  k.load(row + ch);
  k.get(f);
}

// The W - 1 inputs in front of row t (oldest first) of its own sequence, from the rows or the state; zeros where there is none.
// Returns how many rows of the sequence lie in front of t, at most W - 1.
template <typename T, int VEC, int W>
__device__ __forceinline__ int window(const ConvArgs& a, int p, int t, int ch, int code, float (&win)[W][VEC]) {
  const Rows<T> x = view<T>(a.d.x);
  int pos = 0;
  while (pos < W - 1 && a.q.code(p, t - 1 - pos) == code) ++pos;
  const T* state = static_cast<const T*>(a.d.state);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) {
    const int back = W - 1 - j;                  // rows in front of t
#pragma unroll
    for (int v = 0; v < VEC; ++v) win[j][v] = 0.f;
    if (back <= pos) fetch<T, VEC>(x.row(p, t - back), ch, win[j]);
    else if (state) fetch<T, VEC>(state + (((int64_t)p * a.q.S + code) * (W - 1) + j + pos) * a.d.D, ch, win[j]);
  }
  return pos;
}

template <typename T, int VEC, int W>
__global__ void __launch_bounds__(kLanes * kRuns) conv_forward_kernel(const __grid_constant__ ConvArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int ch = (blockIdx.x * kLanes + threadIdx.x) * VEC, p = blockIdx.z;
  const int t0 = (blockIdx.y * kRuns + threadIdx.y) * a.run, t1 = min(a.q.T, t0 + a.run);
  if (ch >= a.d.D || t0 >= t1) return;
  const Rows<T> x = view<T>(a.d.x), out = view<T>(a.d.out);
  Taps<VEC, W> taps;
  taps.load(a.d, p, ch);
  float win[W][VEC];                             // the last W - 1 inputs and row t's
  int before = -2;                               // no row's code
  for (int t = t0; t < t1; t += kAhead) {
    Pack<T, VEC> in[kAhead];
    int code[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      code[i] = t + i < t1 ? a.q.code(p, t + i) : -1;
      if (code[i] >= 0) in[i].load(x.row(p, t + i) + ch);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (code[i] < 0) {
        before = -2;
        continue;
      }
      if (code[i] != before) {
        window<T, VEC, W>(a, p, t + i, ch, code[i], win);
        before = code[i];
      }
      in[i].get(win[W - 1]);
      float o[VEC];
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        float s = taps.bias[v];
#pragma unroll
        for (int j = 0; j < W; ++j) s = fmaf(taps.w[j][v], win[j][v], s);
        o[v] = a.d.act == LSGD_CONV_SILU ? s * sigmoid(s) : s;
      }
      Pack<T, VEC> k;
      k.set(o);
      k.store(out.row(p, t + i) + ch);
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
#pragma unroll
        for (int v = 0; v < VEC; ++v) win[j][v] = win[j + 1][v];
    }
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
      float o[VEC];
#pragma unroll
      for (int v = 0; v < VEC; ++v) o[v] = taps.bias[v];
#pragma unroll
      for (int k = 0; k < W; ++k) {
        float f[VEC];
        kept[k].get(f);
#pragma unroll
        for (int v = 0; v < VEC; ++v) o[v] = fmaf(taps.w[k][v], f[v], o[v]);
      }
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        if (a.d.act == LSGD_CONV_SILU) o[v] *= sigmoid(o[v]);
      Pack<T, VEC> k;
      k.set(o);
      k.store(view<T>(a.d.out).row(p, lo) + ch);
    }
    if (!state) continue;
#pragma unroll
    for (int k = 0; k < W - 1; ++k) kept[k + SINGLE].store(state + (int64_t)k * a.d.D);
  }
}

template <typename T, int VEC, int W>
__global__ void __launch_bounds__(kLanes * kRuns) conv_backward_kernel(const __grid_constant__ ConvArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int ch = (blockIdx.x * kLanes + threadIdx.x) * VEC, p = blockIdx.z;
  const int t0 = (blockIdx.y * kRuns + threadIdx.y) * a.run, t1 = min(a.q.T, t0 + a.run);
  const Rows<T> x = view<T>(a.d.x), d_out = view<T>(a.d.d_out), dx = view<T>(a.d.dx);
  Taps<VEC, W> taps;
  float dw[W][VEC] = {}, db[VEC] = {};
  if (ch < a.d.D && t0 < t1) {
    taps.load(a.d, p, ch);
    float win[W][VEC];
    float wait[W][VEC];                          // dx of rows t - W + 1 .. t as far as it is known
    int before = -2, pos = 0;                    // code of row t - 1; rows of its sequence in front of t, at most W - 1
    const int last = min(a.q.T, t1 + W - 1);
    for (int t = t0; t < last; t += 4) {
      Pack<T, VEC> in[4], up[4];
      int code[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        code[i] = t + i < last ? a.q.code(p, t + i) : -1;
        if (code[i] >= 0) {
          in[i].load(x.row(p, t + i) + ch);
          up[i].load(d_out.row(p, t + i) + ch);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = t + i;
        if (r >= t1 && (code[i] < 0 || code[i] != before)) {       // nothing behind the run reaches into it any more
          t = last;
          break;
        }
        if (code[i] < 0) {
          before = -2;
          continue;
        }
        if (code[i] != before) {
          // the run's first row may lie inside a sequence; dx of the rows in front of the run belongs to another thread
          pos = window<T, VEC, W>(a, p, r, ch, code[i], win);
#pragma unroll
          for (int j = 0; j < W - 1; ++j)
#pragma unroll
            for (int v = 0; v < VEC; ++v) wait[j][v] = 0.f;
          before = code[i];
        }
        in[i].get(win[W - 1]);
        float g[VEC];
        up[i].get(g);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          wait[W - 1][v] = 0.f;
          if (a.d.act == LSGD_CONV_SILU) {
            float s = taps.bias[v];
#pragma unroll
            for (int j = 0; j < W; ++j) s = fmaf(taps.w[j][v], win[j][v], s);
            const float sg = sigmoid(s);
            g[v] *= fmaf(s * sg, 1.f - sg, sg);
          }
#pragma unroll
          for (int j = 0; j < W; ++j) wait[j][v] = fmaf(taps.w[j][v], g[v], wait[j][v]);
          if (r < t1) {
            db[v] += g[v];
#pragma unroll
            for (int j = 0; j < W; ++j) dw[j][v] = fmaf(win[j][v], g[v], dw[j][v]);
          }
        }
        // a row's dx is complete W - 1 rows on, or where its sequence ends
        const bool ends = a.q.code(p, r + 1) != code[i];
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const int row = r - (W - 1) + j;
          if ((j == 0 || ends) && row >= t0 && row < t1 && row >= r - pos) {
            Pack<T, VEC> k;
            k.set(wait[j]);
            k.store(dx.row(p, row) + ch);
          }
        }
        pos = min(pos + 1, W - 1);
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
#pragma unroll
          for (int v = 0; v < VEC; ++v) win[j][v] = win[j + 1][v], wait[j][v] = wait[j + 1][v];
      }
    }
  }
  // the block's sums: the runs' in order
  __shared__ float sums[kRuns][kLanes * VEC];
#pragma unroll
  for (int j = 0; j <= W; ++j) {
    __syncthreads();
#pragma unroll
    for (int v = 0; v < VEC; ++v) sums[threadIdx.y][threadIdx.x * VEC + v] = j < W ? dw[j < W ? j : 0][v] : db[v];
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

// Adds the blocks' sums in order: a warp takes 32 neighbouring sums of a worker (of all workers where they share the vector).
__global__ void __launch_bounds__(1024) conv_join_kernel(const __grid_constant__ ConvArgs a) {
  pdl_wait();
  const int per = a.d.W + 1, n = a.d.D * per;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
  __shared__ float s[32][33];
  const int k = i % per, c = i / per;
  const lsgd_rows& o = k < a.d.W ? a.d.dw : a.d.d_bias;
  const bool share_w = a.d.P > 1 && a.d.dw.stride == 0, share_b = a.d.P > 1 && a.d.d_bias.stride == 0;
  const int workers = share_w || share_b ? a.d.P : 1;
  // where only one of the two is shared, a sum is one worker's or all workers' by its own kind
  const bool shared = k < a.d.W ? share_w : share_b;
  const uint32_t rows = a.blocks_t, share = (rows + 31) / 32, r0 = min(rows, warp * share), r1 = min(rows, r0 + share);
  float total = 0.f;
  for (int w = 0; w < workers; ++w) {
    const int p = workers > 1 && shared ? w : blockIdx.z;
    float v = 0.f;
    if (i < n && (shared ? blockIdx.z == 0 : w == 0)) {
      const float* src = a.part + (int64_t)p * rows * n + i;
#pragma unroll 4
      for (uint32_t r = r0; r < r1; ++r) v += src[(int64_t)r * n];
    }
    __syncthreads();
    s[warp][lane] = v;
    __syncthreads();
    if (warp == 0)
      for (int q = 0; q < 32; ++q) total += s[q][lane];
  }
  if (warp != 0 || i >= n || !o.data || (shared && blockIdx.z > 0)) return;
  float* dst = static_cast<float*>(o.data) + (shared ? 0 : blockIdx.z * o.stride) + (k < a.d.W ? c * o.ld + k : c);
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
  if ((int64_t)d->seq.S * d->P >= int64_t(1) << 31) return LSGD_ERR_TOO_LARGE;
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
    if (rows && (!d->out.data || d->out.data == d->x.data)) return LSGD_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(d->state) % ab) return LSGD_ERR_ALIGNMENT;
    LSGD_ROWS(d->out, T, D, ab, true, false);
    return LSGD_OK;
  }
  if (d->state) return LSGD_ERR_INVALID_ARG;
  if (rows && (!d->d_out.data || !d->dx.data || d->dx.data == d->x.data || d->dx.data == d->d_out.data)) return LSGD_ERR_INVALID_ARG;
  if (!d->dw.data || (d->bias.data != nullptr) != (d->d_bias.data != nullptr)) return LSGD_ERR_INVALID_ARG;
  LSGD_ROWS(d->d_out, T, D, ab, false, false);
  LSGD_ROWS(d->dx, T, D, ab, true, false);
  if (D > 1 && d->dw.ld < d->W) return LSGD_ERR_INVALID_ARG;
  LSGD_ROWS(d->dw, D, d->W, 4, true, true);
  LSGD_ROWS(d->d_bias, 1, D, 4, true, true);
#undef LSGD_ROWS
  return LSGD_OK;
}

// Four values a thread where every row allows it, else one.
int conv_vec(const lsgd_conv_desc* d, bool backward) {
  const int ab = elem_bytes(d->act_dtype);
  auto fits = [&](const lsgd_rows& r) {
    return !r.data || (reinterpret_cast<uintptr_t>(r.data) % (4 * ab) == 0 && (d->T <= 1 || r.ld % 4 == 0) && (d->P <= 1 || r.stride % 4 == 0));
  };
  const bool ok = d->D % 4 == 0 && fits(d->x) &&
                  (backward ? fits(d->d_out) && fits(d->dx) : fits(d->out) && reinterpret_cast<uintptr_t>(d->state) % (4 * ab) == 0);
  return ok ? 4 : 1;
}

struct ConvPlan {
  int vec, run;
  uint32_t blocks_d, blocks_t;
};
ConvPlan conv_plan(const lsgd_conv_desc* d, bool backward) {
  ConvPlan c{};
  c.vec = conv_vec(d, backward);
  c.blocks_d = (uint32_t)((d->D + kLanes * c.vec - 1) / (kLanes * c.vec));
  // rows of a thread: as many as leave every SM several blocks, so that the rows read twice are few
  const int most = kBackRun, least = 8;
  c.run = least;
  while (c.run < most && (int64_t)c.blocks_d * d->P * ((d->T + 2 * c.run * kRuns - 1) / (2 * c.run * kRuns)) >= 8 * sm_count()) c.run *= 2;
  // no more than 65535 blocks of rows (gridDim.y)
  while ((d->T + (int64_t)c.run * kRuns - 1) / ((int64_t)c.run * kRuns) > 65535) c.run *= 2;
  c.blocks_t = (uint32_t)((d->T + (int64_t)c.run * kRuns - 1) / ((int64_t)c.run * kRuns));
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
      e = d->act_dtype == LSGD_BF16 ? (c.vec == 4 ? launch_conv<__nv_bfloat16, 4>(a, c, backward, s) : launch_conv<__nv_bfloat16, 1>(a, c, backward, s))
                                    : (c.vec == 4 ? launch_conv<float, 4>(a, c, backward, s) : launch_conv<float, 1>(a, c, backward, s));
  }
  if (e == cudaSuccess && backward)
    e = launch_pdl(conv_join_kernel, dim3((d->D * (d->W + 1) + 31) / 32, 1, d->P), dim3(1024), 0, s, a);
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
