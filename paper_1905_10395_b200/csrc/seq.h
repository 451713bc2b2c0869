// Sequences in a worker's rows, for the operators that run along them (conv.cu, scan*.cu): which sequence a row belongs to.
#pragma once
#include "lm_ops.h"

namespace lsgd {

// Rows of all workers, and sequences of all: a loop's next step behind the last (65535 blocks of 4 sequences, a chain, a tile) is still
// a number of 32 bits.
constexpr int64_t kMaxRows = (int64_t(1) << 31) - (int64_t(1) << 20);

// Sequences given by their starts are looked up once: codes[p][t] is the sequence of row t, -1 in front of the first and behind
// the last.  A row begins a sequence where its code differs from the row's before it (an empty sequence has no row).  Equal parts
// need no table.
struct SeqView {
  const int32_t* starts;     // NULL: equal parts of `len` rows
  int64_t stride;
  const int32_t* codes;      // [P][T], with starts
  int32_t S, T, len;

  __device__ __forceinline__ int code(int p, int t) const {
    if ((unsigned)t >= (unsigned)T) return -1;
    return starts ? codes[(int64_t)p * T + t] : t / len;
  }
  __device__ __forceinline__ int edge(int p, int s) const {      // first row of sequence s (s == S: the end of all)
    if (!starts) return s * len;
    const int v = starts[p * stride + s];
    return v < 0 ? 0 : v > T ? T : v;
  }
  // The rows around row t that are of one sequence, or of none (code -1).
  struct Span {
    int code, lo, hi;
  };
  __device__ __forceinline__ Span span(int p, int t) const {
    Span s;
    if (!starts) {
      s.code = t / len;
      s.lo = s.code * len;
      s.hi = s.lo + len;
    } else {
      s.code = codes[(int64_t)p * T + t];
      if (s.code >= 0) {
        s.lo = edge(p, s.code);
        s.hi = max(edge(p, s.code + 1), t + 1);
      } else {
        const int first = edge(p, 0);
        s.lo = t < first ? 0 : t;
        s.hi = t < first ? first : T;
      }
    }
    return s;
  }
};

inline lsgd_status check_sequences(const lsgd_sequences& q, int64_t P, int64_t T) {
  if (q.S < 1) return LSGD_ERR_INVALID_ARG;
  if (q.S >= kMaxRows / P) return LSGD_ERR_TOO_LARGE;
  if (!q.starts) return T % q.S == 0 ? LSGD_OK : LSGD_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(q.starts) % 4) return LSGD_ERR_ALIGNMENT;
  if (q.stride < 0 || (q.stride > 0 && q.stride < q.S + 1 && P > 1)) return LSGD_ERR_INVALID_ARG;
  if (P > 1 && q.stride > (int64_t(1) << 56) / P) return LSGD_ERR_TOO_LARGE;
  return LSGD_OK;
}
inline SeqView seq_view(const lsgd_sequences& q, int64_t T, const int32_t* codes) {
  return SeqView{q.starts, q.stride, codes, q.S, (int32_t)T, q.starts ? 0 : (int32_t)(T / q.S)};
}
// A matrix of rows in memory, for the check that outputs overlap no input.
struct Extent {
  uintptr_t at, end;         // first byte, one behind the last
  uint64_t ld, stride, width, block;     // in bytes; block: one worker's rows, from the first to the last
};
inline Extent extent(const lsgd_rows& r, int64_t P, int64_t T, int64_t D, int bytes) {
  Extent e{};
  if (!r.data || P < 1 || T < 1 || D < 1) return e;
  e.at = reinterpret_cast<uintptr_t>(r.data);
  e.ld = T > 1 ? (uint64_t)r.ld * bytes : 0;
  e.stride = P > 1 ? (uint64_t)r.stride * bytes : 0;
  e.width = (uint64_t)D * bytes;
  e.block = (uint64_t)(T - 1) * e.ld + e.width;
  e.end = e.at + (uint64_t)(P - 1) * e.stride + e.block;
  return e;
}
// Whether pieces of `wa` and `wb` bytes, each set a multiple of `unit` apart, never meet.
inline bool interleaved(uintptr_t a, uint64_t wa, uintptr_t b, uint64_t wb, uint64_t unit) {
  if (unit == 0) return false;
  const uint64_t from = (a % unit + unit - b % unit) % unit;      // where a's pieces begin, from b's
  return from >= wb && from + wa <= unit;
}
// Whether two matrices certainly have no byte in common: apart as a whole, workers' blocks between one another (tensors of one
// parameter row), or columns of one buffer's rows.
inline bool apart(const Extent& a, const Extent& b) {
  if (a.at == a.end || b.at == b.end || a.end <= b.at || b.end <= a.at) return true;
  if (a.stride == b.stride && interleaved(a.at, a.block, b.at, b.block, a.stride)) return true;
  if (a.ld != b.ld || a.stride != b.stride) return false;
  // both matrices' rows begin at multiples of one number, each from its own place
  const uint64_t unit = a.stride == 0 ? a.ld : a.ld == 0 || a.ld % a.stride == 0 ? a.stride : a.stride % a.ld == 0 ? a.ld : 0;
  return interleaved(a.at, a.width, b.at, b.width, unit);
}
inline bool all_apart(const Extent* outs, int n_outs, const Extent* ins, int n_ins) {
  for (int i = 0; i < n_outs; ++i) {
    for (int j = 0; j < n_ins; ++j)
      if (!apart(outs[i], ins[j])) return false;
    for (int j = 0; j < i; ++j)
      if (!apart(outs[i], outs[j])) return false;
  }
  return true;
}
inline uint64_t align256(uint64_t n) { return (n + 255) & ~uint64_t(255); }
inline uint64_t codes_bytes(const lsgd_sequences& q, int64_t P, int64_t T) {
  return q.starts ? align256(sizeof(int32_t) * (uint64_t)(P * T)) : 0;
}
// Fills the table (conv.cu).
cudaError_t launch_codes(const SeqView& q, int32_t* codes, int32_t P, cudaStream_t s);

}  // namespace lsgd
