// Host side and the last sums of the block-boundary norms; the mathematics and the kernels are in blocknorm.h.
#include "blocknorm.h"

namespace lsgd {
namespace blocknorm {
namespace {

// Adds the blocks' partial rows in order: columns of one of the three sums of one worker (of all workers where they share the
// vector).  `split` warps share 32 columns, each adding a run of rows, then the runs are added.
constexpr int kJoinMaxSplit = 32;
struct Join {
  int which[3];              // of the sums, per blockIdx.y
  int split;
};
__global__ void __launch_bounds__(1024)
blocknorm_join_kernel(const __grid_constant__ Args a, const __grid_constant__ Join join) {
  pdl_wait();
  const lsgd_blocknorm_desc& d = a.d;
  const int j = join.which[blockIdx.y];  // 0: w_pre, 1: w_post, 2: channel gate -- the last two from the same sums
  const lsgd_rows& o = j == 0 ? d.d_w_pre : j == 1 ? d.d_w_post : d.d_gate;
  const bool channel = d.gate_kind == LSGD_GATE_CHANNEL;
  const bool shared = d.P > 1 && o.stride == 0;
  if (shared && blockIdx.z > 0) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = warp % join.split, group = warp / join.split;
  const int col = (blockIdx.x * (blockDim.x / (32 * join.split)) + group) * 32 + lane;
  __shared__ float s[kJoinMaxSplit][32];
  float total = 0.f;
  const uint32_t per = (a.blocks_w + join.split - 1) / join.split, i0 = min(a.blocks_w, sub * per), i1 = min(a.blocks_w, i0 + per);
  for (uint32_t w = shared ? 0 : blockIdx.z, last = shared ? d.P - 1 : w; w <= last; ++w) {
    float v = 0.f;
    if (col < d.D) {
      const float* src = a.part + ((size_t)w * a.blocks_w * 2 + (j > 0)) * d.D + col;
#pragma unroll 8
      for (uint32_t i = i0; i < i1; ++i) v += src[(size_t)i * 2 * d.D];
    }
    if (join.split > 1) {
      __syncthreads();
      s[warp][lane] = v;
      __syncthreads();
      v = 0.f;
      if (sub == 0)
        for (int q = 0; q < join.split; ++q) v += s[warp + q][lane];
    }
    if (sub == 0 && col < d.D && j > 0) {
      const float ga = channel ? gate_value(static_cast<const float*>(d.gate.data)[w * d.gate.stride + col], d.gate_act) : 1.f;
      v *= d.beta;
      if (j == 1) v *= ga;
      else v *= gate_slope(ga, d.gate_act) * (d.post_norm ? static_cast<const float*>(d.w_post.data)[w * d.w_post.stride + col] : 1.f);
    }
    total += v;
  }
  if (sub != 0 || col >= d.D) return;
  float* dst = static_cast<float*>(o.data) + (shared ? 0 : blockIdx.z) * o.stride + col;
  *dst = d.accumulate ? *dst + total : total;
}

// ------------------------------------------------------------------------------------------------ host
constexpr int kMaxD = 8192;

lsgd_status check_norm(const lsgd_blocknorm_desc* d, bool backward) {
  if (!d || d->struct_size != sizeof(lsgd_blocknorm_desc)) return LSGD_ERR_INVALID_ARG;
  if (d->P < 1 || d->T < 0 || d->D < 1) return LSGD_ERR_INVALID_ARG;
  if (d->resid_dtype < LSGD_F32 || d->resid_dtype > LSGD_BF16 || d->act_dtype < LSGD_F32 || d->act_dtype > LSGD_BF16)
    return LSGD_ERR_INVALID_ARG;
  if (d->resid_dtype == LSGD_BF16 && d->act_dtype == LSGD_F32) return LSGD_ERR_UNSUPPORTED;
  if (d->D > kMaxD || d->P > 65535) return LSGD_ERR_UNSUPPORTED;
  if (d->T >= (int64_t(1) << 31) / d->P) return LSGD_ERR_TOO_LARGE;
  if (d->gate_kind < LSGD_GATE_NONE || d->gate_kind > LSGD_GATE_TOKEN || d->gate_act < LSGD_GATE_IDENTITY ||
      d->gate_act > LSGD_GATE_TANH)
    return LSGD_ERR_INVALID_ARG;
  if (!(d->eps > 0.f) || !(d->eps < 1e30f) || !(d->alpha - d->alpha == 0.f) || !(d->beta - d->beta == 0.f)) return LSGD_ERR_INVALID_ARG;
  const bool has_y = d->y.data != nullptr, pre = d->w_pre.data != nullptr, rows = d->T > 0;
  const bool gated = d->gate_kind != LSGD_GATE_NONE, channel = d->gate_kind == LSGD_GATE_CHANNEL;
  if (!has_y && rows && (d->post_norm || gated || !pre)) return LSGD_ERR_INVALID_ARG;
  // what would be left unwritten, or unread, for want of the operand it belongs to
  if (!pre && (backward ? d->d_w_pre.data || d->d_h.data : d->h.data != nullptr)) return LSGD_ERR_INVALID_ARG;
  if (backward && ((!d->post_norm && d->d_w_post.data) || (!gated && d->d_gate.data) || (!has_y && rows && d->dy.data)))
    return LSGD_ERR_INVALID_ARG;
  const int rb = elem_bytes(d->resid_dtype), ab = elem_bytes(d->act_dtype);
  const int64_t P = d->P, T = d->T, D = d->D;
  if (d->post_norm && (!d->w_post.data || (rows && !d->rstd_post))) return LSGD_ERR_INVALID_ARG;
  if (pre && rows && !d->rstd_pre) return LSGD_ERR_INVALID_ARG;
  if (gated && (rows || channel) && !d->gate.data) return LSGD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(d->rstd_post) | reinterpret_cast<uintptr_t>(d->rstd_pre)) % 4) return LSGD_ERR_ALIGNMENT;
  lsgd_status st;
#define LSGD_ROWS(r, t, bytes, written, shared)                                                   \
  do {                                                                                            \
    if ((r).data && (st = check_rows(r, P, t, D, bytes, written, shared)) != LSGD_OK) return st;  \
  } while (0)
  LSGD_ROWS(d->y, T, ab, false, false);
  LSGD_ROWS(d->gate, channel ? 1 : T, channel ? 4 : ab, false, false);
  LSGD_ROWS(d->w_post, 1, 4, false, false);
  LSGD_ROWS(d->w_pre, 1, 4, false, false);
  LSGD_ROWS(d->out, T, rb, !backward && has_y, false);      // without y it is only the backward pass's input
  if (!backward) {
    if (rows && (!d->x.data || (has_y && !d->out.data) || (pre && !d->h.data))) return LSGD_ERR_INVALID_ARG;
    LSGD_ROWS(d->x, T, rb, false, false);
    LSGD_ROWS(d->h, T, ab, true, false);
    return LSGD_OK;
  }
  if (rows && ((pre && (!d->out.data || !d->d_h.data)) || (!pre && !d->d_out.data) || !d->dx.data || (has_y && !d->dy.data)))
    return LSGD_ERR_INVALID_ARG;
  if (rows && d->gate_kind == LSGD_GATE_TOKEN && !d->d_gate.data) return LSGD_ERR_INVALID_ARG;
  LSGD_ROWS(d->d_out, T, rb, false, false);
  LSGD_ROWS(d->d_h, T, ab, false, false);
  LSGD_ROWS(d->dx, T, rb, true, false);
  LSGD_ROWS(d->dy, T, ab, true, false);
  LSGD_ROWS(d->d_gate, channel ? 1 : T, channel ? 4 : ab, true, channel);
  LSGD_ROWS(d->d_w_post, 1, 4, true, true);
  LSGD_ROWS(d->d_w_pre, 1, 4, true, true);
#undef LSGD_ROWS
  return LSGD_OK;
}

struct Shape {
  Launch l;
  int tpr, rpb, slots, phased;
  uint32_t blocks_w;
};

Shape shape_of(const lsgd_blocknorm_desc* d, bool backward) {
  const int rb = elem_bytes(d->resid_dtype), ab = elem_bytes(d->act_dtype);
  Shape s{};
  s.l.mode = mode_of(*d);
  s.l.backward = backward;
  const bool pre = s.l.mode & kPre, has_y = s.l.mode & kY, token = s.l.mode & kToken;
  // pieces of 8 values: every matrix starts on the boundary of one, and all rows have the same offset from one in every matrix
  bool pieces = true, first = true;
  int64_t ld = 0, stride = 0;
  auto see = [&](const lsgd_rows& r, int bytes) {
    if (!r.data) return;
    const int64_t l = d->T > 1 ? r.ld & 7 : 0, p = d->P > 1 ? r.stride & 7 : 0;
    if (first) ld = l, stride = p;
    first = false;
    pieces = pieces && reinterpret_cast<uintptr_t>(r.data) % (8 * bytes) == 0 && l == ld && p == stride;
  };
  if (has_y) see(d->y, ab);
  if (token) see(d->gate, ab);
  if (backward) {
    see(d->d_out, rb);
    if (pre) see(d->out, rb), see(d->d_h, ab);
    see(d->dx, rb);
    if (has_y) see(d->dy, ab);
    if (token) see(d->d_gate, ab);
  } else {
    see(d->x, rb);
    if (has_y) see(d->out, rb);
    if (pre) see(d->h, ab);
  }
  s.phased = ld != 0 || stride != 0;
  int need = (d->D + (s.phased ? 7 : 0) + E - 1) / E;
  if (!pieces || need > 512) {            // one value at a time
    s.l.mode = kDirect;
    s.phased = 0;
    need = (d->D + E - 1) / E;
  }
  s.tpr = 4;
  while (s.tpr < 32 && s.tpr < need) s.tpr *= 2;
  if (need > 32) s.tpr = (need + 31) / 32 * 32;
  if (s.l.mode != kDirect && (s.phased || d->D != s.tpr * E)) s.l.mode |= kRagged;
  const int wish = backward ? 256 : 128;  // threads of a block; backward fewer and larger blocks, since each leaves a partial row
  s.rpb = s.tpr >= wish ? 1 : wish / s.tpr;
  // few rows: smaller blocks (of whole warps) until there are two for every SM
  while (s.rpb > 1 && s.tpr * s.rpb >= 64 && (d->T + s.rpb - 1) / s.rpb * d->P < 2 * sm_count()) s.rpb = (s.rpb + 1) / 2;
  s.l.threads = (s.tpr * s.rpb + 31) / 32 * 32;
  s.rpb = s.l.threads / s.tpr;
  const size_t per = (size_t)E * s.l.threads;                         // values of a tensor's rows
  const size_t factors = 4 * per * ((pre ? 1 : 0) + (has_y ? 1 : 0));
  const size_t row = per * (backward ? rb + (pre ? rb + ab : 0) + (has_y ? ab : 0) + (token ? ab : 0)
                                     : rb + (has_y ? ab : 0) + (token ? ab : 0));
  const size_t sums = backward && s.rpb > 1 ? sizeof(float) * (size_t)s.rpb * d->D : 0;
  const int64_t groups = (d->T + s.rpb - 1) / s.rpb;
  // persistent: as many blocks as the SMs hold at once (registers, shared memory), and no more than rows
  const auto plan = [&](int slots) {
    s.slots = slots;
    s.l.smem = factors + (s.l.mode == kDirect ? 0 : slots * row);    // one slot: at most 64 + 160 KiB (5 fp32 tensors, D = 8192)
    if (s.l.smem < sums) s.l.smem = sums;
    int per_sm = (backward ? kBackwardThreads : kForwardThreads) / s.l.threads;
    const int fit = (int)(size_t(228) * 1024 / (s.l.smem + 2048));
    if (per_sm > fit) per_sm = fit;
    if (per_sm < 1) per_sm = 1;
    int64_t n = (int64_t)sm_count() * per_sm / d->P;                 // rounded down: one block more would be a second round
    if (n < 1) n = 1;
    if (s.phased && n < groups) n = n < 8 ? 8 : n & ~int64_t(7);     // a block's rows are a multiple of 8 apart
    s.blocks_w = (uint32_t)(groups < n ? groups : n);
  };
  if (s.l.mode != kDirect && factors + 2 * row <= (size_t)kSmemMax) {
    plan(2);
    if (groups <= (int64_t)s.blocks_w) plan(1);                      // one group of rows a block: nothing is fetched ahead
  } else {
    plan(1);
  }
  return s;
}

cudaError_t run(const lsgd_blocknorm_desc* d, bool backward, cudaStream_t st) {
  const Shape s = shape_of(d, backward);
  Args a{};
  a.d = *d;
  a.T = (uint32_t)d->T;
  a.tpr = s.tpr;
  a.rpb = s.rpb;
  a.phased = s.phased;
  a.slots = s.slots;
  a.inv_d = 1.f / (float)d->D;
  a.blocks_w = s.blocks_w;
  a.part = backward ? static_cast<float*>(d->scratch) : nullptr;
  cudaError_t e = cudaSuccess;
  if (d->T > 0)
    e = d->resid_dtype == LSGD_BF16 ? launch_bf16_bf16(a, s.l, st)
        : d->act_dtype == LSGD_BF16 ? launch_f32_bf16(a, s.l, st) : launch_f32_f32(a, s.l, st);
  if (e != cudaSuccess || !backward) return e;
  Join join{};
  int n = 0;
  if (d->w_pre.data && d->d_w_pre.data) join.which[n++] = 0;
  if (d->post_norm && d->d_w_post.data) join.which[n++] = 1;
  if (d->gate_kind == LSGD_GATE_CHANNEL && d->d_gate.data) join.which[n++] = 2;
  if (n == 0) return cudaSuccess;
  join.split = s.blocks_w <= 16 ? 1 : s.blocks_w <= 64 ? 8 : kJoinMaxSplit;
  const int threads = join.split == kJoinMaxSplit ? 1024 : 256, cols = threads / join.split;
  return launch_pdl(blocknorm_join_kernel, dim3((d->D + cols - 1) / cols, n, d->P), dim3(threads), 0, st, a, join);
}

}  // namespace
}  // namespace blocknorm
}  // namespace lsgd

extern "C" {

uint64_t lsgd_blocknorm_scratch_bytes(const lsgd_blocknorm_desc* d) {
  using namespace lsgd;
  using namespace lsgd::blocknorm;
  if (!d || d->struct_size != sizeof(lsgd_blocknorm_desc) || d->P < 1 || d->T < 0 || d->D < 1 || d->D > kMaxD) return 0;
  return sizeof(float) * 2 * (uint64_t)d->D * d->P * shape_of(d, true).blocks_w;
}

lsgd_status lsgd_blocknorm_forward(const lsgd_blocknorm_desc* d, void* stream) {
  using namespace lsgd;
  using namespace lsgd::blocknorm;
  const lsgd_status st = check_norm(d, false);
  if (st != LSGD_OK) return st;
  return run(d, false, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
}

lsgd_status lsgd_blocknorm_backward(const lsgd_blocknorm_desc* d, void* stream) {
  using namespace lsgd;
  using namespace lsgd::blocknorm;
  const lsgd_status st = check_norm(d, true);
  if (st != LSGD_OK) return st;
  const uint64_t need = lsgd_blocknorm_scratch_bytes(d);
  if (need && (!d->scratch || d->scratch_bytes < need)) return LSGD_ERR_INVALID_ARG;
  if (need && reinterpret_cast<uintptr_t>(d->scratch) % 256) return LSGD_ERR_ALIGNMENT;
  return run(d, true, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
}

}  // extern "C"
