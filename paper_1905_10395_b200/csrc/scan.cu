// Host side of the selective state space scan, and the passes over its chains; the mathematics and the kernels are in scan.h.
#include "scan.h"

namespace lsgd {
namespace scan {
namespace {

// What a chain starts from: a thread takes one state of a channel through the chains of its worker.
template <bool REVERSE>
__global__ void __launch_bounds__(256) chain_kernel(const __grid_constant__ Args a) {
  pdl_wait();
  pdl_launch_dependents();
  const int64_t n = (int64_t)a.d.D * a.d.N, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int p = blockIdx.y;
  if (i >= n) return;
  const int ch = (int)(i / a.d.N), st = (int)(i % a.d.N);
  const float A2 = rate_of(static_cast<const float*>(a.d.a_log.data)[p * a.d.a_log.stride + ch * a.d.a_log.ld + st]);
  float* ends = a.ends + (int64_t)p * a.chains * n + i;
  const float* sums = a.sums + (int64_t)p * a.chains * a.d.D + ch;
  float carry = 0.f;
  constexpr int kTake = 16;                      // chains fetched before the first is used
  for (int k0 = 0; k0 < a.chains; k0 += kTake) {
    float e[kTake], s[kTake];
#pragma unroll
    for (int k = 0; k < kTake; ++k) {
      if (k0 + k >= a.chains) break;
      const int c = REVERSE ? a.chains - 1 - k0 - k : k0 + k;
      e[k] = ends[c * n];
      s[k] = sums[(int64_t)c * a.d.D];
    }
#pragma unroll
    for (int k = 0; k < kTake; ++k) {
      if (k0 + k >= a.chains) break;
      const int c = REVERSE ? a.chains - 1 - k0 - k : k0 + k;
      ends[c * n] = carry;
      carry = s[k] < 0.f ? e[k] : fmaf(ex2(s[k] * A2), carry, e[k]);
    }
  }
}

// ------------------------------------------------------------------------------------------------ host
lsgd_status check_scan(const lsgd_scan_desc* d, bool backward) {
  if (!d || d->struct_size != sizeof(lsgd_scan_desc)) return LSGD_ERR_INVALID_ARG;
  if (d->P < 1 || d->T < 0 || d->D < 1 || d->N < 1) return LSGD_ERR_INVALID_ARG;
  if (d->act_dtype < LSGD_F32 || d->act_dtype > LSGD_BF16) return LSGD_ERR_INVALID_ARG;
  if (d->D > 65536 || d->N > 64 || d->P > 65535) return LSGD_ERR_UNSUPPORTED;
  if (d->T >= kMaxRows / d->P) return LSGD_ERR_TOO_LARGE;
  lsgd_status st;
  if ((st = check_sequences(d->seq, d->P, d->T)) != LSGD_OK) return st;
  const int64_t P = d->P, T = d->T, D = d->D, N = d->N;
  const int ab = elem_bytes(d->act_dtype);
  const bool rows = T > 0;
  const int64_t states = D * N, groups = (T + kGroup - 1) / kGroup;
  if (!d->a_log.data || (rows && (!d->x.data || !d->dt.data || !d->b.data || !d->c.data))) return LSGD_ERR_INVALID_ARG;
#define LSGD_ROWS(r, t, w, bytes, written, shared)                                                 \
  do {                                                                                            \
    if ((r).data && (st = check_rows(r, P, t, w, bytes, written, shared)) != LSGD_OK) return st;  \
  } while (0)
  LSGD_ROWS(d->x, T, D, ab, false, false);
  LSGD_ROWS(d->dt, T, D, ab, false, false);
  LSGD_ROWS(d->z, T, D, ab, false, false);
  LSGD_ROWS(d->b, T, N, ab, false, false);
  LSGD_ROWS(d->c, T, N, ab, false, false);
  LSGD_ROWS(d->a_log, D, N, 4, false, false);
  LSGD_ROWS(d->skip, 1, D, 4, false, false);
  LSGD_ROWS(d->dt_bias, 1, D, 4, false, false);
  if ((reinterpret_cast<uintptr_t>(d->state) | reinterpret_cast<uintptr_t>(d->saved)) % 16) return LSGD_ERR_ALIGNMENT;
  if (!backward) {
    if (rows && !d->out.data) return LSGD_ERR_INVALID_ARG;
    LSGD_ROWS(d->out, T, D, ab, true, false);
    const int64_t kept = (int64_t)d->seq.S;
    const Extent ins[] = {extent(d->x, P, T, D, ab), extent(d->dt, P, T, D, ab),  extent(d->z, P, T, D, ab),   extent(d->b, P, T, N, ab),
                          extent(d->c, P, T, N, ab), extent(d->a_log, P, D, N, 4), extent(d->skip, P, 1, D, 4), extent(d->dt_bias, P, 1, D, 4)};
    const Extent outs[] = {extent(d->out, P, T, D, ab), extent({d->state, states, kept * states}, P, kept, states, 4),
                           extent({d->saved, states, groups * states}, P, groups, states, 4)};
    return all_apart(outs, 3, ins, 8) ? LSGD_OK : LSGD_ERR_INVALID_ARG;
  }
  if (d->state || (rows && (!d->saved || !d->d_out.data || !d->dx.data || !d->d_dt.data || !d->db.data || !d->dc.data))) return LSGD_ERR_INVALID_ARG;
  if (!d->d_a_log.data) return LSGD_ERR_INVALID_ARG;
  if ((rows && (d->z.data != nullptr) != (d->dz.data != nullptr)) || (d->skip.data != nullptr) != (d->d_skip.data != nullptr) ||
      (d->dt_bias.data != nullptr) != (d->d_dt_bias.data != nullptr))
    return LSGD_ERR_INVALID_ARG;
  LSGD_ROWS(d->d_out, T, D, ab, false, false);
  LSGD_ROWS(d->dx, T, D, ab, true, false);
  LSGD_ROWS(d->d_dt, T, D, ab, true, false);
  LSGD_ROWS(d->dz, T, D, ab, true, false);
  LSGD_ROWS(d->db, T, N, ab, true, false);
  LSGD_ROWS(d->dc, T, N, ab, true, false);
  LSGD_ROWS(d->d_a_log, D, N, 4, true, true);
  LSGD_ROWS(d->d_skip, 1, D, 4, true, true);
  LSGD_ROWS(d->d_dt_bias, 1, D, 4, true, true);
#undef LSGD_ROWS
  const Extent ins[] = {extent(d->x, P, T, D, ab), extent(d->dt, P, T, D, ab),   extent(d->z, P, T, D, ab),     extent(d->b, P, T, N, ab),
                        extent(d->c, P, T, N, ab), extent(d->d_out, P, T, D, ab), extent(d->a_log, P, D, N, 4), extent(d->skip, P, 1, D, 4),
                        extent(d->dt_bias, P, 1, D, 4), extent({d->saved, states, groups * states}, P, groups, states, 4)};
  const Extent outs[] = {extent(d->dx, P, T, D, ab),     extent(d->d_dt, P, T, D, ab),  extent(d->dz, P, T, D, ab),    extent(d->db, P, T, N, ab),
                         extent(d->dc, P, T, N, ab),     extent(d->d_a_log, P, D, N, 4), extent(d->d_skip, P, 1, D, 4), extent(d->d_dt_bias, P, 1, D, 4)};
  return all_apart(outs, 8, ins, 10) ? LSGD_OK : LSGD_ERR_INVALID_ARG;
}

bool row_vec4(const lsgd_rows& r, int64_t P, int64_t T, int bytes) {
  return reinterpret_cast<uintptr_t>(r.data) % (4 * bytes) == 0 && (T <= 1 || r.ld % 4 == 0) && (P <= 1 || r.stride % 4 == 0);
}

struct Plan {
  Launch l;
  int32_t chains, per, split, wide, wide_bc;
  uint32_t tiles;
  uint64_t codes, ends, sums, old_state, part_bc, part_a, part_v, total;   // offsets in the scratch
};

Plan plan_of(const lsgd_scan_desc* d, bool backward) {
  Plan m{};
  const int64_t P = d->P, T = d->T, D = d->D, N = d->N, S = d->seq.S;
  m.l.L = N <= 8 ? 2 : N <= 16 ? 4 : N <= 32 ? 8 : 16;
  const bool equal = !d->seq.starts;
  m.l.single = !backward && equal && S == T && !d->saved;
  const int ch = kThreads / m.l.L, rows = 32;              // channels of a block; a chain's rows are a multiple of any tile's
  m.tiles = (uint32_t)((D + ch - 1) / ch);
  const int ab = elem_bytes(d->act_dtype);
  m.wide = 8;
  auto fits = [&](const lsgd_rows& r) {
    while (m.wide > 1 && r.data && !(D % m.wide == 0 && reinterpret_cast<uintptr_t>(r.data) % (m.wide * ab) == 0 &&
                                     (T <= 1 || r.ld % m.wide == 0) && (P <= 1 || r.stride % m.wide == 0)))
      m.wide /= 2;
  };
  for (const lsgd_rows* r : {&d->x, &d->dt, &d->z}) fits(*r);
  if (backward)
    for (const lsgd_rows* r : {&d->d_out, &d->dx, &d->d_dt, &d->dz}) fits(*r);
  else
    fits(d->out);
  // Chains: whole sequences where that gives every SM a block; else equal runs of rows, as many as are resident.
  m.wide_bc = N % 4 == 0 && row_vec4(d->b, P, T, ab) && row_vec4(d->c, P, T, ab);
  const int64_t columns = P * m.tiles, sms = sm_count(), resident = sms * kBlocks;
  int64_t chains;
  if (columns >= sms) {
    chains = 1;
    m.per = (int32_t)S;
  } else if (equal && columns * S >= sms) {
    int64_t want = resident / columns;
    if (want > S) want = S;
    m.per = (int32_t)((S + want - 1) / want);
    chains = (S + m.per - 1) / m.per;
  } else {
    m.split = 1;
    const int64_t want = resident / columns;        // all of them at once: one block more would be a second round
    int64_t per = (T + want - 1) / want;
    per = (per + rows - 1) / rows * rows;
    if (per < 2 * rows) per = 2 * rows;
    if (per > T) per = (T + rows - 1) / rows * rows;
    m.per = (int32_t)(per < 1 ? 1 : per);
    chains = T > 0 ? (T + m.per - 1) / m.per : 1;
    if (chains <= 1) {       // one chain is a run of all sequences
      chains = 1;
      m.split = 0;
      m.per = (int32_t)S;
    }
  }
  m.chains = (int32_t)chains;
  // single rows: several sequences a block one after another, which share its decays, while 32 blocks an SM are left
  int64_t singles = 32 * sms / columns < S ? 32 * sms / columns : S;
  if (singles < (S + 15) / 16) singles = (S + 15) / 16;
  if (singles > 65535) singles = 65535;
  m.l.grid = dim3(m.tiles, (unsigned)(m.l.single ? singles : chains), (unsigned)P);
  uint64_t at = codes_bytes(d->seq, P, T);
  auto take = [&](uint64_t floats) {
    const uint64_t here = at;
    at += align256(sizeof(float) * floats);
    return here;
  };
  if (m.split) {
    m.ends = take((uint64_t)P * chains * D * N);
    m.sums = take((uint64_t)P * chains * D);
    if (d->state) m.old_state = take((uint64_t)P * S * D * N);
  }
  if (backward) {
    m.part_bc = take((uint64_t)P * m.tiles * T * 2 * N);
    m.part_a = take((uint64_t)P * chains * D * N);
    m.part_v = take((uint64_t)P * chains * 2 * D);
  }
  m.total = at;
  return m;
}

lsgd_status run_scan(const lsgd_scan_desc* d, bool backward, cudaStream_t s) {
  const Plan m = plan_of(d, backward);
  char* scratch = static_cast<char*>(d->scratch);
  Args a{};
  a.d = *d;
  a.q = seq_view(d->seq, d->T, reinterpret_cast<int32_t*>(scratch));
  a.chains = m.chains;
  a.per = m.per;
  a.split = m.split;
  a.wide = m.wide;
  a.wide_bc = m.wide_bc;
  a.tiles = m.tiles;
  auto at = [&](uint64_t offset) { return reinterpret_cast<float*>(scratch + offset); };
  a.ends = at(m.ends);
  a.sums = at(m.sums);
  a.old_state = at(m.old_state);
  a.part_bc = at(m.part_bc);
  a.part_a = at(m.part_a);
  a.part_v = at(m.part_v);
  cudaError_t e = cudaSuccess;
  if (d->T > 0) {
    if (d->seq.starts) e = launch_codes(a.q, reinterpret_cast<int32_t*>(scratch), d->P, s);
    const bool f32 = d->act_dtype == LSGD_F32;
    if (e == cudaSuccess)
      e = backward ? (f32 ? launch_backward_f32(a, m.l, s) : launch_backward_bf16(a, m.l, s))
                   : (f32 ? launch_forward_f32(a, m.l, s) : launch_forward_bf16(a, m.l, s));
  }
  if (e == cudaSuccess && backward && d->T == 0) {
    a.chains = 0;
    e = launch_join_f32(a, s);                               // no rows, whatever their type
  }
  return e == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
}

}  // namespace

cudaError_t launch_chain_join(const Args& a, bool reverse, cudaStream_t s) {
  const dim3 grid((unsigned)(((int64_t)a.d.D * a.d.N + 255) / 256), a.d.P);
  return reverse ? launch_pdl(chain_kernel<true>, grid, dim3(256), 0, s, a) : launch_pdl(chain_kernel<false>, grid, dim3(256), 0, s, a);
}

}  // namespace scan
}  // namespace lsgd

extern "C" {

uint64_t lsgd_scan_scratch_bytes(const lsgd_scan_desc* d, int32_t backward) {
  using namespace lsgd;
  using namespace lsgd::scan;
  if (!d || d->struct_size != sizeof(lsgd_scan_desc) || d->P < 1 || d->T < 0 || d->D < 1 || d->D > 65536 || d->N < 1 || d->N > 64 ||
      d->seq.S < 1 || d->act_dtype < LSGD_F32 || d->act_dtype > LSGD_BF16 || d->T >= kMaxRows / d->P)
    return 0;
  return plan_of(d, backward).total;
}

lsgd_status lsgd_scan_plan(const lsgd_scan_desc* d, int32_t backward, int32_t plan[4]) {
  using namespace lsgd;
  const lsgd_status st = scan::check_scan(d, backward);
  if (st != LSGD_OK || !plan) return st != LSGD_OK ? st : LSGD_ERR_INVALID_ARG;
  const scan::Plan m = scan::plan_of(d, backward);
  plan[0] = m.l.L, plan[1] = m.chains, plan[2] = m.split ? m.per : 0, plan[3] = m.l.single;
  return LSGD_OK;
}

#define LSGD_SCAN_CALL(name, backward)                                                            \
  lsgd_status name(const lsgd_scan_desc* d, void* stream) {                                       \
    using namespace lsgd;                                                                         \
    const lsgd_status st = scan::check_scan(d, backward);                                         \
    if (st != LSGD_OK) return st;                                                                 \
    const uint64_t need = lsgd_scan_scratch_bytes(d, backward);                                   \
    if (need && (!d->scratch || d->scratch_bytes < need)) return LSGD_ERR_INVALID_ARG;            \
    if (need && reinterpret_cast<uintptr_t>(d->scratch) % 256) return LSGD_ERR_ALIGNMENT;         \
    return scan::run_scan(d, backward, static_cast<cudaStream_t>(stream));                        \
  }
LSGD_SCAN_CALL(lsgd_scan_forward, false)
LSGD_SCAN_CALL(lsgd_scan_backward, true)
#undef LSGD_SCAN_CALL

}  // extern "C"
