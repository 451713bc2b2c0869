// Embedding lookup with scaling, and its gradient by sorted tokens.
//
//     out[p][t] = scale * table[p][token]          d_table[p][v] = scale * sum_{t: token = v} d_out[p][t]
//
// Both only move rows: the lookup reads and writes each value once, the gradient reads every row of d_out once and
// writes every row of d_table, the rows of absent tokens with zeros.  A row is written once, except for the last rows of a
// table whose tokens are sorted by a cluster: those are cleared during the sort, before it is known which of them have a token.
//
// The gradient must not depend on timing, so no row is added with atomics.  Two ways to the same sums:
//   few tokens   one launch.  Every block reads all tokens; a warp takes a position, leaves if an earlier one holds the same
//                token, and otherwise lists the later ones and adds their rows in order.
//   many tokens  positions are sorted by (worker, token) with a stable radix sort -- up to 131072 positions in the shared
//                memory of one cluster, in one launch, more with a histogram and a scatter launch per pass; a warp then
//                walks a piece of the sorted list, adding rows while the token stays the same.  A token that lies within
//                one piece is written at once; pieces of a token that crosses piece ends leave fp32 partial rows, which a
//                last launch adds in order.  Work is split by positions, never by token, so it stays even however often
//                one token occurs.
#include "lm_ops.h"

namespace lsgd {
namespace {

__device__ uint32_t g_embed_status;      // LSGD_DEVFLAG_BAD_INDEX, read and cleared by lsgd_embed_check_device

constexpr int kMaxD = 65536;
constexpr uint32_t kNone = 0xFFFFFFFFu;  // key of a position that adds to no row

struct Tokens {
  const void* p;
  int64_t stride;
  int64_t V, padding;
  uint32_t T, N;
  uint32_t key_stride;                   // V, or 0 where all workers share one table's gradient
  int bytes;
  __device__ __forceinline__ int64_t token(uint32_t worker, uint32_t t) const {
    const int64_t i = worker * stride + t;
    return bytes == 8 ? static_cast<const int64_t*>(p)[i] : (int64_t) static_cast<const int32_t*>(p)[i];
  }
  // (worker, token) as one number, or kNone
  __device__ __forceinline__ uint32_t key(uint32_t pos) const {
    const uint32_t w = pos / T;
    return key_of(w, token(w, pos - w * T));
  }
  __device__ __forceinline__ uint32_t key_of(uint32_t w, int64_t v) const {
    if (v < 0 || v >= V) {
      atomicOr(&g_embed_status, FLAG_BAD_INDEX);
      return kNone;
    }
    return v == padding ? kNone : w * key_stride + (uint32_t)v;
  }
};

// ------------------------------------------------------------------------------------------------ lookup
// A block copies kLookupRows rows for each group of tx threads.  8 x 4096 rows of 1024 fp32 values into bf16: 27 us, 1.4 times
// what the 124 MB of distinct rows and outputs take at the measured copy bandwidth.  No unit is at its limit (DRAM 35 %, L2
// 30 %, issue 47 %): a row waits for its token, and a block has no row in flight meanwhile.  1, 2 or 4 rows a thread, 3 to 8
// blocks an SM and a persistent form with the tokens ahead measured 27 to 30 us.  Rows that are moved in pairs or one by one
// (rows of 1022 and 1023 values): 61 us.
constexpr int kLookupThreads = 256;
constexpr int kLookupRows = 4;           // rows whose loads a thread issues before the first store

template <typename TT, typename TA, int VEC>
__global__ void __launch_bounds__(kLookupThreads)
embed_lookup_kernel(Tokens tok, Rows<const TT> table, Rows<TA> out, uint32_t nvec, uint32_t tx, float scale) {
  pdl_wait();
  const uint32_t ty = kLookupThreads / tx;
  const uint32_t cx = threadIdx.x % tx, ry = threadIdx.x / tx;
  const uint32_t base = (blockIdx.x * ty + ry) * kLookupRows;
  const TT* src[kLookupRows];
  TA* dst[kLookupRows];
#pragma unroll
  for (int u = 0; u < kLookupRows; ++u) {
    src[u] = nullptr;
    dst[u] = nullptr;
    const uint32_t pos = base + u;
    if (pos < tok.N) {
      const uint32_t w = pos / tok.T, t = pos - w * tok.T;
      const int64_t v = tok.token(w, t);
      dst[u] = out.row(w, t);
      if (v >= 0 && v < tok.V) src[u] = table.p + w * table.stride + v * table.ld;
      else if (cx == 0 && blockIdx.y == 0) atomicOr(&g_embed_status, FLAG_BAD_INDEX);
    }
  }
  constexpr int kPieces = VEC == 8 ? 1 : 4;      // narrow pieces: several in flight
  for (uint32_t c0 = blockIdx.y * tx + cx; c0 < nvec; c0 += kPieces * gridDim.y * tx) {
    Pack<TT, VEC> in[kPieces][kLookupRows];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const uint32_t c = c0 + i * gridDim.y * tx;
#pragma unroll
      for (int u = 0; u < kLookupRows; ++u)
        if (src[u] && c < nvec) in[i][u].load(src[u] + (int64_t)c * VEC);
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const uint32_t c = c0 + i * gridDim.y * tx;
#pragma unroll
      for (int u = 0; u < kLookupRows; ++u) {
        if (!dst[u] || c >= nvec) continue;
        float f[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) f[k] = 0.f;
        if (src[u]) {
          in[i][u].get(f);
#pragma unroll
          for (int k = 0; k < VEC; ++k) f[k] *= scale;
        }
        Pack<TA, VEC> o;
        o.set(f);
        o.store(dst[u] + (int64_t)c * VEC);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ rows of the gradient
constexpr int kSlab = 256;               // columns that one warp carries: 8 values a lane

template <typename TG>
struct GradRows {
  TG* p;
  int64_t ld, stride;
  uint32_t key_stride;
  __device__ __forceinline__ TG* row(uint32_t key) const {
    const uint32_t w = key_stride ? key / key_stride : 0;
    return p + w * stride + (int64_t)(key - w * key_stride) * ld;
  }
};

// A lane's 8 columns of a slab: one piece of 8, or pieces of VEC that are 32 VEC columns apart.
template <int VEC>
__device__ __forceinline__ int slab_col(int slab, int lane, int i) { return slab * kSlab + i * 32 * VEC + lane * VEC; }

template <typename TG, int VEC>
__device__ __forceinline__ void write_row(TG* row, int slab, int lane, int D, const float* acc, float scale, bool add) {
  constexpr int N = 8 / VEC;
  float f[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) f[k] = acc[k] * scale;
  if (add) {                             // all of what is there before the first is written: the stores would hold the loads up
    Pack<TG, VEC> o[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (slab_col<VEC>(slab, lane, i) < D) o[i].load(row + slab_col<VEC>(slab, lane, i));
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (slab_col<VEC>(slab, lane, i) >= D) break;
      float e[VEC];
      o[i].get(e);
#pragma unroll
      for (int k = 0; k < VEC; ++k) f[i * VEC + k] += e[k];
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int col = slab_col<VEC>(slab, lane, i);
    if (col >= D) break;
    Pack<TG, VEC> o;
    o.set(f + i * VEC);
    o.store(row + col);
  }
}

// A row of zeros, by a warp: single values up to a 16-byte boundary and behind the last, 16 bytes at a time between, so that
// rows of odd length are cleared as fast as others (gradient of 3 tables of 32698 x 1019 bf16 values from 480 tokens: 51 us, 70
// value by value).
template <typename TG>
__device__ __forceinline__ void clear_row(TG* row, int lane, int D) {
  constexpr int n = 16 / (int)sizeof(TG);
  const int head = min(D, (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(TG));
  const int body = (D - head) / n;
  TG zero{};
  if (lane < head) row[lane] = zero;
  uint4* wide = reinterpret_cast<uint4*>(row + head);
  for (int i = lane; i < body; i += 32) wide[i] = make_uint4(0, 0, 0, 0);
  const int tail = head + body * n;
  if (lane < D - tail) row[tail + lane] = zero;
}

// Adds rows list[j0 .. j1) of d_out to a lane's columns of a slab, kAhead rows in flight.
template <typename TA, int VEC, typename List>
__device__ __forceinline__ void add_rows(const Tokens& tok, const Rows<const TA>& d_out, const List* list, uint32_t j0, uint32_t j1,
                                         int slab, int lane, int D, float (&acc)[8]) {
  constexpr int kAhead = VEC < 8 ? 3 : sizeof(TA) == 2 ? 8 : 4;   // what the registers of 4 blocks an SM hold
  for (uint32_t j = j0; j < j1; j += kAhead) {
    Pack<TA, VEC> in[kAhead][8 / VEC];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (j + u >= j1) break;
      const uint32_t pos = list[j + u], w = pos / tok.T;
      const TA* row = d_out.row(w, pos - w * tok.T);
#pragma unroll
      for (int i = 0; i < 8 / VEC; ++i)
        if (slab_col<VEC>(slab, lane, i) < D) in[u][i].load(row + slab_col<VEC>(slab, lane, i));
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (j + u >= j1) break;
#pragma unroll
      for (int i = 0; i < 8 / VEC; ++i) {
        if (slab_col<VEC>(slab, lane, i) >= D) break;
        float f[VEC];
        in[u][i].get(f);
#pragma unroll
        for (int k = 0; k < VEC; ++k) acc[i * VEC + k] += f[k];
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ few tokens
// One launch instead of three: 16 to 17 us against 23 us for 3 x 1021 tokens of 250 values.  It is a chain of latencies (tokens, the
// search for equal ones, rows, the write), so blocks are small enough for all of them to be resident.
constexpr int kFewTokens = 4096;
constexpr int kFewThreads = 256;
constexpr int kFewWarps = kFewThreads / 32;
constexpr int kFewLoads = 8;                        // tokens that a thread loads together; divides kFewTokens / kFewThreads
constexpr int kFewAlone = 32;                       // rows that one warp adds alone

// The positions after `mine`'s that hold the same key, in order, into list[0 .. cap): returns how many there are with
// itself, or 0 if there is an earlier one.  512 keys at a time, 4 times 4 to a lane; a whole warp calls it.
__device__ __forceinline__ uint32_t find_same(const uint32_t* s_key, uint32_t N, uint32_t me, uint32_t mine, uint16_t* list, uint32_t cap) {
  const int lane = threadIdx.x & 31;
  uint32_t count = 0;
  for (uint32_t j = 0; j < N; j += 512) {           // the keys behind the last are none's
    uint32_t hits = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint4 k = *reinterpret_cast<const uint4*>(s_key + j + u * 128 + lane * 4);
      hits |= ((k.x == mine) | (k.y == mine) << 1 | (k.z == mine) << 2 | (k.w == mine) << 3) << (4 * u);
    }
    if (!__any_sync(0xFFFFFFFFu, hits)) continue;
    for (int u = 0; u < 4; ++u) {
      const uint32_t j0 = j + u * 128, hit = hits >> (4 * u) & 15u;
      const uint32_t lanes = __ballot_sync(0xFFFFFFFFu, hit != 0);
      if (lanes == 0) continue;
      if (count == 0) {
        const int l = __ffs(lanes) - 1;
        if (j0 + l * 4 + __ffs(__shfl_sync(0xFFFFFFFFu, hit, l)) - 1 != me) return 0;
      }
      const uint32_t n = __popc(hit);
      uint32_t incl = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += v;
      }
      uint32_t place = count + incl - n;
      for (uint32_t b = hit; b; b &= b - 1, ++place)
        if (place < cap) list[place] = (uint16_t)(j0 + lane * 4 + __ffs(b) - 1);
      count += __shfl_sync(0xFFFFFFFFu, incl, 31);
    }
  }
  __syncwarp();
  return count;
}

template <typename TG, typename TA, int VEC>
__global__ void __launch_bounds__(kFewThreads, 4)
embed_grad_few_kernel(Tokens tok, Rows<const TA> d_out, GradRows<TG> grad, uint32_t rows, uint32_t rows_per_block, uint32_t sum_blocks,
                      int slabs, int D, float scale, bool add) {
  pdl_wait();
  __shared__ __align__(16) uint32_t s_key[kFewTokens];
  __shared__ __align__(16) uint16_t s_list[kFewTokens];   // kFewAlone for each warp, or one long list; or words of row bits
  __shared__ float s_part[kFewWarps][kSlab];
  __shared__ uint32_t s_count[kFewWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (blockIdx.x >= sum_blocks && blockIdx.y > 0) return;
  for (uint32_t j0 = 0; j0 < tok.N; j0 += kFewLoads * kFewThreads) {
    int64_t t[kFewLoads];                           // in flight together
    uint32_t w[kFewLoads];
#pragma unroll
    for (int u = 0; u < kFewLoads; ++u) {
      const uint32_t j = j0 + u * kFewThreads + threadIdx.x;
      w[u] = tok.T < tok.N ? j / tok.T : 0;
      t[u] = j < tok.N ? tok.token(w[u], j - w[u] * tok.T) : 0;
    }
#pragma unroll
    for (int u = 0; u < kFewLoads; ++u) {
      const uint32_t j = j0 + u * kFewThreads + threadIdx.x;
      s_key[j] = j < tok.N ? tok.key_of(w[u], t[u]) : kNone;
    }
  }
  if (blockIdx.x >= sum_blocks) {                   // rows of absent tokens: zeros
    uint32_t* s_bits = reinterpret_cast<uint32_t*>(s_list);
    const uint32_t r0 = (blockIdx.x - sum_blocks) * rows_per_block;
    const uint32_t n = min(rows_per_block, rows - r0);
    for (uint32_t i = threadIdx.x; i < (n + 31) / 32; i += kFewThreads) s_bits[i] = 0;
    __syncthreads();
    for (uint32_t j = threadIdx.x; j < tok.N; j += kFewThreads) {
      const uint32_t k = s_key[j];
      if (k >= r0 && k - r0 < n) atomicOr(&s_bits[(k - r0) >> 5], 1u << ((k - r0) & 31));
    }
    __syncthreads();
    for (uint32_t r = warp; r < n; r += kFewWarps)
      if (!(s_bits[r >> 5] >> (r & 31) & 1)) clear_row(grad.row(r0 + r), lane, D);
    return;
  }
  __syncthreads();
  const uint32_t i = blockIdx.x + warp * sum_blocks;   // frequent tokens have their first position early: spread over the blocks
  const uint32_t mine = i < tok.N ? s_key[i] : kNone;
  uint16_t* l = s_list + warp * kFewAlone;
  const uint32_t count = mine == kNone ? 0 : find_same(s_key, tok.N, i, mine, l, kFewAlone);
  if (count > 0 && count <= kFewAlone) {
    for (int slab = blockIdx.y; slab < slabs; slab += gridDim.y) {
      float acc[8] = {};
      add_rows<TA, VEC>(tok, d_out, l, 0, count, slab, lane, D, acc);
      write_row<TG, VEC>(grad.row(mine), slab, lane, D, acc, scale, add);
    }
  }
  if (lane == 0) s_count[warp] = count > kFewAlone ? count : 0;
  for (int h = 0; h < kFewWarps; ++h) {             // frequent tokens: the whole block
    __syncthreads();
    const uint32_t n = s_count[h];
    if (n == 0) continue;
    if (warp == h) find_same(s_key, tok.N, i, mine, s_list, kFewTokens);
    __syncthreads();
    const uint32_t per = (n + kFewWarps - 1) / kFewWarps, used = (n + per - 1) / per;
    const uint32_t key = s_key[blockIdx.x + h * sum_blocks];
    for (int slab = blockIdx.y; slab < slabs; slab += gridDim.y) {
      float acc[8] = {};
      add_rows<TA, VEC>(tok, d_out, s_list, min(n, warp * per), min(n, (warp + 1) * per), slab, lane, D, acc);
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 8; ++k) s_part[warp][k * 32 + lane] = acc[k];
      __syncthreads();
      if (warp != 0) continue;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float v = 0.f;
        for (uint32_t w = 0; w < used; ++w) v += s_part[w][k * 32 + lane];
        acc[k] = v;
      }
      write_row<TG, VEC>(grad.row(key), slab, lane, D, acc, scale, add);
    }
  }
}

// ------------------------------------------------------------------------------------------------ sort
// The lanes whose digit is this lane's: one vote per bit.
template <int BITS>
__device__ __forceinline__ uint32_t same_digit(uint32_t d, bool live) {
  uint32_t same = __ballot_sync(0xFFFFFFFFu, live);
#pragma unroll
  for (int b = 0; b < BITS; ++b) {
    const int one = (int)(d << (31 - b)) >> 31;                // all bits are bit b
    same &= ~(__ballot_sync(0xFFFFFFFFu, one) ^ (uint32_t)one);
  }
  return same;
}

constexpr int kDigitBits = 10;
constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortItems = 4;                                  // keys a thread holds
constexpr int kSortTile = kSortThreads * kSortItems;           // 2048
constexpr int kMaxTiles = 128;

struct SortPass {
  const uint32_t* key_in;     // nullptr: keys are made from the tokens, positions count from 0
  const uint32_t* pos_in;
  uint32_t *key_out, *pos_out;
  uint32_t* counts;           // [tiles][bins]
  uint8_t* touched;           // first histogram only: rows that have a token
  uint32_t N, per_tile, none_key;
  int shift, bits, tiles;
};

__device__ __forceinline__ uint32_t sort_key(const Tokens& tok, const SortPass& a, uint32_t i) {
  if (a.key_in) return a.key_in[i];
  const uint32_t k = tok.key(i);
  return k == kNone ? a.none_key : k;      // past every row: sorted last
}

__global__ void __launch_bounds__(kSortThreads)
embed_histogram_kernel(Tokens tok, SortPass a) {
  pdl_wait();
  pdl_launch_dependents();
  extern __shared__ uint32_t s_hist[];
  const uint32_t bins = 1u << a.bits;
  for (uint32_t b = threadIdx.x; b < bins; b += kSortThreads) s_hist[b] = 0;
  __syncthreads();
  const uint32_t i0 = blockIdx.x * a.per_tile, i1 = min(a.N, i0 + a.per_tile);
  for (uint32_t i = i0 + threadIdx.x; i < i1; i += kSortThreads) {
    const uint32_t k = sort_key(tok, a, i);
    if (a.touched && k != a.none_key) a.touched[k] = 1;
    atomicAdd(&s_hist[(k >> a.shift) & (bins - 1)], 1u);
  }
  __syncthreads();
  for (uint32_t b = threadIdx.x; b < bins; b += kSortThreads) a.counts[(size_t)blockIdx.x * bins + b] = s_hist[b];
}

__global__ void __launch_bounds__(kSortThreads)
embed_scatter_kernel(Tokens tok, SortPass a) {
  pdl_wait();
  pdl_launch_dependents();
  extern __shared__ __align__(16) uint32_t smem[];
  const uint32_t bins = 1u << a.bits;
  uint32_t* s_base = smem;                                                   // [bins] next place of each digit
  uint16_t* s_cnt = reinterpret_cast<uint16_t*>(smem + bins);                // [warps][bins]
  __shared__ uint32_t s_warp[kSortWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;

  // first place of each digit in this tile: all smaller digits, and this digit in earlier tiles
  const uint32_t per = (bins + kSortThreads - 1) / kSortThreads;             // bins a thread owns, 1 or 2
  uint32_t total[2] = {0, 0}, before[2] = {0, 0};
  for (uint32_t q = 0; q < per; ++q) {
    const uint32_t b = threadIdx.x * per + q;
    if (b < bins) {
#pragma unroll 16
      for (int t = 0; t < a.tiles; ++t) {
        const uint32_t n = a.counts[(size_t)t * bins + b];
        total[q] += n;
        if (t < (int)blockIdx.x) before[q] += n;
      }
    }
  }
  uint32_t sum = total[0] + total[1], incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t n = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += n;
  }
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  uint32_t start = incl - sum;
  for (int w = 0; w < warp; ++w) start += s_warp[w];
  for (uint32_t q = 0; q < per; ++q) {
    const uint32_t b = threadIdx.x * per + q;
    if (b < bins) s_base[b] = start + before[q];
    start += total[q];
  }
  __syncthreads();

  const uint32_t i0 = blockIdx.x * a.per_tile, i1 = min(a.N, i0 + a.per_tile);
  for (uint32_t s = i0; s < i1; s += kSortTile) {
    for (uint32_t j = threadIdx.x; j < bins * kSortWarps / 2; j += kSortThreads) reinterpret_cast<uint32_t*>(s_cnt)[j] = 0;
    __syncthreads();
    uint16_t* cnt = s_cnt + warp * bins;
    uint32_t key[kSortItems], rank[kSortItems];
#pragma unroll
    for (int q = 0; q < kSortItems; ++q) {                                   // a warp's keys are consecutive: the sort is stable
      const uint32_t i = s + warp * (32 * kSortItems) + q * 32 + lane;
      key[q] = i < i1 ? sort_key(tok, a, i) : 0;
    }
#pragma unroll
    for (int q = 0; q < kSortItems; ++q) {
      const uint32_t i = s + warp * (32 * kSortItems) + q * 32 + lane;
      const uint32_t d = (key[q] >> a.shift) & (bins - 1);
      const bool live = i < i1;
      const uint32_t same = same_digit<kDigitBits>(d, live);
      uint32_t prev = 0;
      if (live) prev = cnt[d];
      rank[q] = prev + __popc(same & ((1u << lane) - 1));
      __syncwarp();
      if (live && (same >> lane) == 1u) cnt[d] = (uint16_t)(prev + __popc(same));   // the last lane of the group
      __syncwarp();
    }
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < bins; b += kSortThreads) {            // running count over the warps
      uint32_t run = 0;
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t n = s_cnt[w * bins + b];
        s_cnt[w * bins + b] = (uint16_t)run;
        run += n;
      }
      if (b < kSortThreads) total[0] = run;                                  // added to s_base once this sub-tile is written
      else total[1] = run;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kSortItems; ++q) {
      const uint32_t i = s + warp * (32 * kSortItems) + q * 32 + lane;
      if (i < i1) {
        const uint32_t d = (key[q] >> a.shift) & (bins - 1);
        const uint32_t at = s_base[d] + cnt[d] + rank[q];
        a.key_out[at] = key[q];
        a.pos_out[at] = a.pos_in ? a.pos_in[i] : i;
      }
    }
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < bins; b += kSortThreads) s_base[b] += b < kSortThreads ? total[0] : total[1];
  }
}

// ---- up to kClusterKeys keys: the whole sort in the shared memory of one cluster.  A block holds 1024 ITEMS consecutive
// places.  A pass orders the block's own keys by digit in its shared memory, adds up the blocks' digit counts through
// distributed shared memory, and copies the keys to their places in whichever block holds them: in the order of the digits,
// so that a warp's stores to another block are runs of consecutive places.  Two cluster barriers a pass instead of two
// launches.
constexpr int kClusterThreads = 1024;
constexpr int kClusterWarps = kClusterThreads / 32;
constexpr int kClusterBlocks = 16;                             // 8 (the portable size) of twice the keys: 30 us instead of 20 for 65536
constexpr int kClusterItems = 8;                               // keys of a thread: 1, 2, 4 or 8, the fewest that 16 blocks hold
constexpr int kClusterKeys = kClusterThreads * kClusterItems * kClusterBlocks;
constexpr int kClusterBits = 9;
constexpr int kClearBlocks = 112;                              // blocks of all clusters where some of them clear rows
constexpr int kClusterBins = 1 << kClusterBits;

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t remote(const void* smem, uint32_t block) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(smem)), "r"(block));
  return r;
}
__device__ __forceinline__ uint32_t load_remote(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void store_remote(uint32_t a, uint2 v) {
  asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(a), "r"(v.x), "r"(v.y) : "memory");
}

struct ClusterSort {
  uint32_t *key_out, *pos_out;
  uint8_t* touched;           // nullptr: not wanted
  uint32_t N, none_key, rows;
  int bits, passes, blocks;
  uint32_t clear_from;        // further clusters clear rows clear_from .. rows
  int D;
};
template <int ITEMS>
struct ClusterMemory {
  uint2 stage[kClusterThreads * ITEMS];    // (key, position): this block's keys in the order of their digits
  uint2 place[kClusterThreads * ITEMS];    // what the blocks have put in this block's places
  uint32_t count[kClusterBins];                    // this block's digits; read by all blocks
  uint32_t base[kClusterBins];                     // first place of this block's digit
  uint32_t local[kClusterBins];                    // first place of the digit in `stage`
  uint16_t warp[kClusterWarps][kClusterBins];
  uint32_t scan[2][kClusterWarps];
};

// Sum of the values of the threads before this one, of the whole block.
__device__ __forceinline__ uint32_t scan_before(uint32_t v, uint32_t* s_scan) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t n = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += n;
  }
  if (lane == 31) s_scan[warp] = incl;
  __syncthreads();
  uint32_t sums = lane < warp ? s_scan[lane] : 0;
  sums = __reduce_add_sync(0xFFFFFFFFu, sums);
  return sums + incl - v;
}

// Cluster 0 sorts.  The sort leaves most of the machine idle and waits more than it works, so further clusters clear rows
// meanwhile, whether they have a token or not: the last ones, since vocabularies tend to begin with the frequent tokens, and
// no more than takes about as long as the sort (65536 tokens into 50000 rows of 2048 fp32 values: 125 us instead of 135).
template <int ITEMS, typename TG>
__global__ void __launch_bounds__(kClusterThreads, 1)
embed_cluster_sort_kernel(Tokens tok, ClusterSort a, GradRows<TG> grad) {
  pdl_wait();
  pdl_launch_dependents();
  if (blockIdx.x >= (uint32_t)a.blocks) {
    const uint32_t warps = (gridDim.x - a.blocks) * kClusterWarps;
    for (uint32_t r = a.clear_from + (blockIdx.x - a.blocks) * kClusterWarps + (threadIdx.x >> 5); r < a.rows; r += warps)
      clear_row(grad.row(r), threadIdx.x & 31, a.D);
    return;
  }
  extern __shared__ __align__(16) uint32_t smem[];
  constexpr uint32_t kBlockKeys = kClusterThreads * ITEMS;
  ClusterMemory<ITEMS>& s = *reinterpret_cast<ClusterMemory<ITEMS>*>(smem);
  const uint32_t bins = 1u << a.bits;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t me = cluster_rank();
  const uint32_t first = me * kBlockKeys;
  const uint32_t n = a.N > first ? min(a.N - first, (uint32_t)kBlockKeys) : 0;   // places of this block
  const uint32_t at = warp * (32 * ITEMS) + lane;                     // of the thread's first key; 32 apart

  uint2 item[ITEMS];
  int64_t token[ITEMS];            // all of them before the first is looked at
#pragma unroll
  for (int q = 0; q < ITEMS; ++q) {
    const uint32_t pos = first + at + q * 32, w = pos / tok.T;
    item[q].y = pos;
    token[q] = at + q * 32 < n ? tok.token(w, pos - w * tok.T) : 0;
  }
#pragma unroll
  for (int q = 0; q < ITEMS; ++q) {
    item[q].x = a.none_key;
    if (at + q * 32 < n) {
      const uint32_t k = tok.key_of(item[q].y / tok.T, token[q]);
      if (k != kNone) item[q].x = k;
    }
  }
  if (a.touched)
    for (uint32_t i = (me * kClusterThreads + threadIdx.x) * 16; i < a.rows; i += a.blocks * kClusterThreads * 16)
      *reinterpret_cast<uint4*>(a.touched + i) = make_uint4(0, 0, 0, 0);      // the buffer is a multiple of 256 bytes

  for (int pass = 0; pass < a.passes; ++pass) {
    const int shift = pass * a.bits;
    const uint32_t mask = bins - 1;
    for (uint32_t b = lane; b < bins; b += 32) s.warp[warp][b] = 0;
    __syncwarp();
    uint16_t* cnt = s.warp[warp];
    uint32_t rank[ITEMS];
#pragma unroll
    for (int q = 0; q < ITEMS; ++q) {
      rank[q] = 0;
      if (warp * (32 * ITEMS) + q * 32 >= n) break;                   // the whole warp
      const uint32_t d = (item[q].x >> shift) & mask;
      const bool live = at + q * 32 < n;
      const uint32_t same = same_digit<kClusterBits>(d, live);
      uint32_t prev = 0;
      if (live) prev = cnt[d];
      rank[q] = prev + __popc(same & ((1u << lane) - 1));
      __syncwarp();
      if (live && (same >> lane) == 1u) cnt[d] = (uint16_t)(prev + __popc(same));
      __syncwarp();
    }
    __syncthreads();
    uint32_t mine = 0;
    if (threadIdx.x < bins) {
      uint32_t c[kClusterWarps];
#pragma unroll
      for (int w = 0; w < kClusterWarps; ++w) c[w] = s.warp[w][threadIdx.x];
#pragma unroll
      for (int w = 0; w < kClusterWarps; ++w) {
        s.warp[w][threadIdx.x] = (uint16_t)mine;
        mine += c[w];
      }
      s.count[threadIdx.x] = mine;
    }
    const uint32_t local = scan_before(mine, s.scan[0]);
    if (threadIdx.x < bins) s.local[threadIdx.x] = local;
    cluster_sync();                        // every block's counts are there; its keys are in registers
    uint32_t total = 0, before = 0;
    if (threadIdx.x < bins) {
#pragma unroll
      for (int r = 0; r < kClusterBlocks; ++r) {
        const uint32_t c = r < a.blocks ? load_remote(remote(&s.count[threadIdx.x], r)) : 0;
        total += c;
        before += r < (int)me ? c : 0;
      }
    }
    const uint32_t start = scan_before(total, s.scan[1]);
    if (threadIdx.x < bins) s.base[threadIdx.x] = start + before;
#pragma unroll
    for (int q = 0; q < ITEMS; ++q) {
      if (at + q * 32 < n) {
        const uint32_t d = (item[q].x >> shift) & mask;
        s.stage[s.local[d] + cnt[d] + rank[q]] = item[q];
      }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < ITEMS; ++q) {
      const uint32_t i = threadIdx.x + q * kClusterThreads;
      if (i < n) {
        const uint2 v = s.stage[i];
        const uint32_t d = (v.x >> shift) & mask;
        const uint32_t to = s.base[d] + (i - s.local[d]);                     // < N
        store_remote(remote(&s.place[to % kBlockKeys], to / kBlockKeys), v);
      }
    }
    cluster_sync();                        // every key is in its place
#pragma unroll
    for (int q = 0; q < ITEMS; ++q)
      if (at + q * 32 < n) item[q] = s.place[at + q * 32];
    if (pass + 1 == a.passes) {
#pragma unroll
      for (int q = 0; q < ITEMS; ++q) {
        const uint32_t i = at + q * 32;
        if (i < n) {
          a.key_out[first + i] = item[q].x;
          a.pos_out[first + i] = item[q].y;
          // a row's first place marks it (flags were cleared before the cluster barriers)
          if (a.touched && item[q].x != a.none_key && (i == 0 || s.place[i - 1].x != item[q].x)) a.touched[item[q].x] = 1;
        }
      }
    }
    __syncthreads();                       // the digit tables are written again
  }
}

// ------------------------------------------------------------------------------------------------ sums over the sorted list
constexpr int kSumThreads = 256;
constexpr int kSumWarps = kSumThreads / 32;
constexpr uint32_t kMaxPiece = 128;

// A warp carries 256 columns of a piece.  65536 tokens of 2048 bf16 values into a table of 50000 fp32 rows: 104 us for all 652 MB
// of rows read and written, 6.3 TB/s or 0.96 of the measured copy bandwidth, and so many fewer as the sort's launch has
// cleared rows; sort and join add 20 and 8 us of latency.
struct SumArgs {
  const uint32_t *key, *pos;  // sorted
  const uint8_t* touched;     // nullptr: rows of absent tokens are left alone
  float* part;                // [pieces][2][slabs * 256]
  uint32_t N, T, none_key;
  uint32_t piece, pieces, slabs;
  uint32_t sum_blocks, rows_per_block;
  uint32_t clear_rows;        // the absent ones of the first clear_rows rows are cleared here
  int D;
  float scale;
  bool add;
};

template <typename TG, typename TA, int VEC>
__global__ void __launch_bounds__(kSumThreads)
embed_sum_kernel(SumArgs a, Rows<const TA> d_out, GradRows<TG> grad) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (blockIdx.x >= a.sum_blocks) {      // rows of absent tokens: zeros
    const uint32_t r0 = (blockIdx.x - a.sum_blocks) * a.rows_per_block, r1 = min(a.clear_rows, r0 + a.rows_per_block);
    for (uint32_t r = r0; r < r1; r += 32) {
      const uint32_t absent = __ballot_sync(0xFFFFFFFFu, r + lane < r1 && !a.touched[min(r + lane, r1 - 1)]);
      for (uint32_t k = warp; k < min(32u, r1 - r); k += kSumWarps)
        if (absent >> k & 1) clear_row(grad.row(r + k), lane, a.D);
    }
    return;
  }
  const uint32_t item = blockIdx.x * kSumWarps + warp;
  const uint32_t c = item / a.slabs;
  const int slab = item - c * a.slabs;
  if (c >= a.pieces) return;
  const uint32_t i0 = c * a.piece, i1 = min(a.N, i0 + a.piece);
  uint32_t cur = a.key[i0];
  bool inside = i0 == 0 || a.key[i0 - 1] != cur;     // the current token began in this piece
  float* part = a.part + ((size_t)c * 2 * a.slabs + slab) * kSlab;
  float acc[8] = {};
  const auto to_part = [&](int which) {
    float* o = part + (size_t)which * a.slabs * kSlab + lane * 8;
    Pack<float, 8> v;
#pragma unroll
    for (int k = 0; k < 8; ++k) v.v[k] = acc[k];
    v.store(o);
  };
  constexpr int U = 4;
  for (uint32_t i = i0; i < i1; i += 32) {
    const bool live = i + lane < i1;
    const uint32_t key = live ? a.key[i + lane] : a.none_key;
    int64_t off = 0;
    if (live && key != a.none_key) {
      const uint32_t pos = a.pos[i + lane], p = pos / a.T;
      off = p * d_out.stride + (int64_t)(pos - p * a.T) * d_out.ld;
    }
    const int n = min(32u, i1 - i);
    for (int j = 0; j < n; j += U) {
      Pack<TA, VEC> in[U][8 / VEC];
      uint32_t kk[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int jj = min(j + u, 31);
        kk[u] = __shfl_sync(0xFFFFFFFFu, key, jj);
        const int64_t o = __shfl_sync(0xFFFFFFFFu, off, jj);
        if (j + u < n && kk[u] != a.none_key) {
          const TA* row = d_out.p + o;
#pragma unroll
          for (int i2 = 0; i2 < 8 / VEC; ++i2)
            if (slab_col<VEC>(slab, lane, i2) < a.D) in[u][i2].load(row + slab_col<VEC>(slab, lane, i2));
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (j + u >= n) break;
        if (kk[u] != cur) {
          if (inside) write_row<TG, VEC>(grad.row(cur), slab, lane, a.D, acc, a.scale, a.add);
          else to_part(0);
          cur = kk[u];
          inside = true;
#pragma unroll
          for (int k = 0; k < 8; ++k) acc[k] = 0.f;
        }
        if (cur == a.none_key) return;   // the rest of the list adds to no row
#pragma unroll
        for (int i2 = 0; i2 < 8 / VEC; ++i2) {
          if (slab_col<VEC>(slab, lane, i2) >= a.D) break;
          float f[VEC];
          in[u][i2].get(f);
#pragma unroll
          for (int k = 0; k < VEC; ++k) acc[i2 * VEC + k] += f[k];
        }
      }
    }
  }
  const bool goes_on = i1 < a.N && a.key[i1] == cur;
  if (!inside) to_part(0);
  else if (goes_on) to_part(1);
  else write_row<TG, VEC>(grad.row(cur), slab, lane, a.D, acc, a.scale, a.add);
}

// A warp takes a piece: if a token begins in it and goes on in the next ones, its partial rows are added in order.  Few: by
// the warp alone; many: by the block, each warp a run of them, then the runs.
constexpr uint32_t kJoinFew = 16;

template <typename TG, int VEC>
__global__ void __launch_bounds__(kSumThreads)
embed_join_kernel(SumArgs a, GradRows<TG> grad) {
  pdl_wait();
  __shared__ uint32_t s_n[kSumWarps], s_key[kSumWarps];
  __shared__ float s_part[kSumWarps][kSlab];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t c = blockIdx.x + warp * gridDim.x;  // spread: a long token's pieces are neighbours
  uint32_t n = 0, k = 0;                             // partial rows: the first piece's end, then whole beginnings
  if (c + 1 < a.pieces) {
    const uint32_t next = (c + 1) * a.piece;
    k = a.key[next];
    const uint32_t mine = a.key[next - 1], before = c > 0 ? a.key[c * a.piece - 1] : ~k;
    if (k != a.none_key && mine == k && before != k) {
      uint32_t last = c + 1;                         // last piece that begins with the token
      for (;;) {
        const uint32_t q = last + 1 + lane;
        const bool same = q < a.pieces && a.key[q * a.piece] == k;
        const uint32_t bits = __ballot_sync(0xFFFFFFFFu, same);
        last += bits == 0xFFFFFFFFu ? 32 : __ffs(~bits) - 1;
        if (bits != 0xFFFFFFFFu) break;
      }
      n = last - c + 1;
    }
  }
  const size_t row = (size_t)a.slabs * kSlab;
  const auto add = [&](uint32_t first, int slab, uint32_t j0, uint32_t j1, float (&acc)[8]) {
    const float* src = a.part + (size_t)slab * kSlab + lane * 8;
    constexpr int kAhead = 4;
    for (uint32_t j = j0; j < j1; j += kAhead) {
      Pack<float, 8> v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (j + u < j1) v[u].load(src + ((size_t)(first + j + u) * 2 + (j + u == 0)) * row);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (j + u >= j1) break;
#pragma unroll
        for (int q = 0; q < 8; ++q) acc[q] += v[u].v[q];
      }
    }
  };
  if (n > 0 && n <= kJoinFew) {
    for (int slab = blockIdx.y; slab < (int)a.slabs; slab += gridDim.y) {
      float acc[8] = {};
      add(c, slab, 0, n, acc);
      write_row<TG, VEC>(grad.row(k), slab, lane, a.D, acc, a.scale, a.add);
    }
  }
  if (lane == 0) {
    s_n[warp] = n > kJoinFew ? n : 0;
    s_key[warp] = k;
  }
  __syncthreads();
  for (int h = 0; h < kSumWarps; ++h) {
    const uint32_t m = s_n[h];
    if (m == 0) continue;                            // the same for the whole block
    const uint32_t per = (m + kSumWarps - 1) / kSumWarps, used = (m + per - 1) / per, first = blockIdx.x + h * gridDim.x;
    for (int slab = blockIdx.y; slab < (int)a.slabs; slab += gridDim.y) {
      float acc[8] = {};
      add(first, slab, min(m, warp * per), min(m, (warp + 1) * per), acc);
      __syncthreads();
#pragma unroll
      for (int q = 0; q < 8; ++q) s_part[warp][q * 32 + lane] = acc[q];
      __syncthreads();
      if (warp != 0) continue;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        float v = 0.f;
        for (uint32_t w = 0; w < used; ++w) v += s_part[w][q * 32 + lane];
        acc[q] = v;
      }
      write_row<TG, VEC>(grad.row(s_key[h]), slab, lane, a.D, acc, a.scale, a.add);
    }
  }
}

// ------------------------------------------------------------------------------------------------ host
struct SortPlan {
  uint32_t N, rows, piece, pieces, slabs, per_tile;
  int passes, bits, tiles, items;
  bool cluster;
  size_t o_touched, o_key[2], o_pos[2], o_counts, o_part, bytes;
};

template <int ITEMS>
cudaLaunchConfig_t cluster_config(int blocks, cudaStream_t s, cudaLaunchAttribute (&at)[2]) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(kClusterThreads);
  cfg.dynamicSmemBytes = sizeof(ClusterMemory<ITEMS>);
  cfg.stream = s;
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = blocks;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = LSGD_NO_PDL ? 1 : 2;
  return cfg;
}

// Whether the device can hold a cluster of kClusterBlocks (16 is more than the portable 8).  Looked up once per device.
template <int ITEMS, typename TG>
bool cluster_fits() {
  static OncePerDevice once, fits;
  if (!once.here()) {
    int n = 0;
    cudaLaunchAttribute at[2];
    cudaLaunchConfig_t cfg = cluster_config<ITEMS>(kClusterBlocks, nullptr, at);
    cfg.numAttrs = 1;
    const auto kernel = embed_cluster_sort_kernel<ITEMS, TG>;
    fits.here() = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg.dynamicSmemBytes) == cudaSuccess &&
                  cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                  cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess && n > 0;
    if (!fits.here()) (void)cudaGetLastError();
    once.here() = true;
  }
  return fits.here();
}

SortPlan sort_plan(uint32_t N, uint32_t rows, int D) {
  SortPlan s{};
  s.N = N;
  s.rows = rows;
  int need = 1;
  while ((rows >> need) != 0) ++need;      // keys 0 .. rows (rows: no row)
  s.items = 1;
  while (s.items < kClusterItems && (uint32_t)(kClusterThreads * kClusterBlocks * s.items) < N) s.items *= 2;
  s.cluster = N <= kClusterKeys && (s.items == 1   ? cluster_fits<1, float>() && cluster_fits<1, __nv_bfloat16>()
                                    : s.items == 2 ? cluster_fits<2, float>() && cluster_fits<2, __nv_bfloat16>()
                                    : s.items == 4 ? cluster_fits<4, float>() && cluster_fits<4, __nv_bfloat16>()
                                                   : cluster_fits<8, float>() && cluster_fits<8, __nv_bfloat16>());
  s.passes = s.cluster ? (need + kClusterBits - 1) / kClusterBits : (need + kDigitBits - 1) / kDigitBits;
  s.bits = (need + s.passes - 1) / s.passes;
  const uint32_t sub = (N + kSortTile - 1) / kSortTile;
  s.per_tile = ((sub + kMaxTiles - 1) / kMaxTiles) * kSortTile;
  s.tiles = (int)((N + s.per_tile - 1) / s.per_tile);
  s.slabs = (uint32_t)((D + kSlab - 1) / kSlab);
  // pieces as long as there are still enough of them to fill the machine: every piece end can cost two partial rows
  s.piece = 8;
  while (s.piece < kMaxPiece && (uint64_t)(N / (2 * s.piece)) * s.slabs >= 4096) s.piece *= 2;
  s.pieces = (N + s.piece - 1) / s.piece;
  size_t off = 0;
  auto take = [&](size_t b) { size_t o = off; off += (b + 255) & ~size_t(255); return o; };
  s.o_touched = take(rows);
  for (int i = 0; i < (s.cluster ? 1 : 2); ++i) {
    s.o_key[i] = take(sizeof(uint32_t) * (size_t)N);
    s.o_pos[i] = take(sizeof(uint32_t) * (size_t)N);
  }
  if (!s.cluster) s.o_counts = take(sizeof(uint32_t) * ((size_t)s.tiles << s.bits));
  s.o_part = take(sizeof(float) * 2 * (size_t)s.pieces * s.slabs * kSlab);
  s.bytes = off;
  return s;
}

lsgd_status check_embed(const lsgd_embed_desc* e, bool backward) {
  if (!e || e->struct_size != sizeof(lsgd_embed_desc)) return LSGD_ERR_INVALID_ARG;
  if (e->P < 1 || e->T < 0 || e->V < 1 || e->D < 1) return LSGD_ERR_INVALID_ARG;
  if (e->token_bytes != 4 && e->token_bytes != 8) return LSGD_ERR_INVALID_ARG;
  if (e->table_dtype < LSGD_F32 || e->table_dtype > LSGD_BF16 || e->act_dtype < LSGD_F32 || e->act_dtype > LSGD_BF16)
    return LSGD_ERR_INVALID_ARG;
  if (e->D > kMaxD) return LSGD_ERR_UNSUPPORTED;
  if (e->T >= (int64_t(1) << 31) / e->P || e->V >= (int64_t(1) << 31) / e->P) return LSGD_ERR_TOO_LARGE;
  if (e->padding < -1 || e->padding >= e->V || e->token_stride < 0) return LSGD_ERR_INVALID_ARG;
  if (e->P > 1 && e->token_stride > (int64_t(1) << 56) / e->P) return LSGD_ERR_TOO_LARGE;
  if (e->T > 0 && !e->tokens) return LSGD_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(e->tokens) % e->token_bytes) return LSGD_ERR_ALIGNMENT;
  const int tb = elem_bytes(e->table_dtype), ab = elem_bytes(e->act_dtype);
  lsgd_status st;
  if (!backward) {
    if (e->T > 0 && (!e->table.data || !e->out.data)) return LSGD_ERR_INVALID_ARG;
    if ((st = check_rows(e->table, e->P, e->V, e->D, tb, false)) != LSGD_OK) return st;
    return check_rows(e->out, e->P, e->T, e->D, ab, true);
  }
  if (!e->d_table.data || (e->T > 0 && !e->d_out.data)) return LSGD_ERR_INVALID_ARG;
  if ((st = check_rows(e->d_out, e->P, e->T, e->D, ab, false)) != LSGD_OK) return st;
  return check_rows(e->d_table, e->P, e->V, e->D, tb, true, true);
}

bool shared_grad(const lsgd_embed_desc* e) { return e->P > 1 && e->d_table.stride == 0; }

Tokens tokens_of(const lsgd_embed_desc* e, bool shared) {
  Tokens t{};
  t.p = e->tokens;
  t.stride = e->token_stride;
  t.V = e->V;
  t.padding = e->padding;
  t.T = (uint32_t)(e->T > 0 ? e->T : 1);
  t.N = (uint32_t)(e->T * e->P);
  t.key_stride = shared ? 0 : (uint32_t)e->V;
  t.bytes = e->token_bytes;
  return t;
}

template <typename TT, typename TA, int VEC>
cudaError_t launch_lookup(const lsgd_embed_desc* e, cudaStream_t s) {
  const Tokens tok = tokens_of(e, false);
  const uint32_t nvec = (uint32_t)(e->D / VEC);
  uint32_t tx = 1;
  while (tx < nvec && tx < kLookupThreads) tx *= 2;
  const uint32_t rows_per_block = kLookupThreads / tx * kLookupRows;
  const uint32_t gx = (tok.N + rows_per_block - 1) / rows_per_block;
  uint32_t gy = (nvec + tx - 1) / tx;      // wide rows: column groups side by side while rows alone do not fill the machine
  const uint32_t most = ((uint32_t)sm_count() * 8 + gx - 1) / gx;
  if (gy > most) gy = most;
  return launch_pdl(embed_lookup_kernel<TT, TA, VEC>, dim3(gx, gy), dim3(kLookupThreads), 0, s, tok,
                    rows_of<const TT>(e->table), rows_of<TA>(e->out), nvec, tx, e->scale);
}

// `cleared`: how many of the last rows further clusters clear.
template <int ITEMS, typename TG>
cudaError_t launch_cluster_sort(const SortPlan& p, const Tokens& tok, char* w, uint8_t* touched, uint32_t cleared, const GradRows<TG>& grad, int D,
                                cudaStream_t s) {
  ClusterSort a{};
  a.key_out = reinterpret_cast<uint32_t*>(w + p.o_key[0]);
  a.pos_out = reinterpret_cast<uint32_t*>(w + p.o_pos[0]);
  a.touched = touched;
  a.N = p.N;
  a.none_key = a.rows = p.rows;
  a.bits = p.bits;
  a.passes = p.passes;
  a.blocks = kClusterBlocks / 2;             // the fewest that more than kFewTokens positions take
  while ((uint32_t)a.blocks * kClusterThreads * ITEMS < p.N) a.blocks *= 2;
  a.clear_from = p.rows - cleared;
  a.D = D;
  cudaLaunchAttribute at[2];
  cudaLaunchConfig_t cfg = cluster_config<ITEMS>(a.blocks, s, at);
  if (cleared) cfg.gridDim.x = kClearBlocks;                       // whole clusters: a.blocks divides it
  return cudaLaunchKernelEx(&cfg, embed_cluster_sort_kernel<ITEMS, TG>, tok, a, grad);
}

template <typename TG, typename TA, int VEC>
cudaError_t launch_grad(const lsgd_embed_desc* e, cudaStream_t s) {
  const bool shared = shared_grad(e);
  const Tokens tok = tokens_of(e, shared);
  const uint32_t rows = shared ? (uint32_t)e->V : (uint32_t)(e->V * e->P);
  const GradRows<TG> grad{static_cast<TG*>(e->d_table.data), e->d_table.ld, e->d_table.stride, tok.key_stride};
  const Rows<const TA> d_out = rows_of<const TA>(e->d_out);
  const bool add = e->accumulate != 0;
  const uint32_t slabs = (uint32_t)((e->D + kSlab - 1) / kSlab);
  const size_t row_bytes = (size_t)e->D * sizeof(TG);
  uint32_t rows_per_block = (uint32_t)(65536 / (row_bytes < 64 ? 64 : row_bytes));   // about 64 KiB of zeros a block
  if (rows_per_block < 1) rows_per_block = 1;
  if (tok.N <= kFewTokens) {
    // each block reads all tokens first: one block an SM beside those that add rows (four are resident), two where there is
    // more to clear than to add, and at least 32 rows and 64 KiB a block
    const uint32_t blocks = (uint32_t)sm_count() * ((uint64_t)rows * row_bytes > (64u << 20) ? 2 : 1);
    const uint32_t even = (rows + blocks - 1) / blocks;
    if (rows_per_block < even) rows_per_block = even;
    if (rows_per_block < 32) rows_per_block = 32;
    if (rows_per_block > kFewTokens * 16) rows_per_block = kFewTokens * 16;      // bits in s_list
    const uint32_t zero_blocks = add ? 0 : (rows + rows_per_block - 1) / rows_per_block;
    const uint32_t sum_blocks = (tok.N + kFewWarps - 1) / kFewWarps;
    if (sum_blocks + zero_blocks == 0) return cudaSuccess;
    return launch_pdl(embed_grad_few_kernel<TG, TA, VEC>, dim3(sum_blocks + zero_blocks, slabs < 4 ? slabs : 4), dim3(kFewThreads), 0, s,
                      tok, d_out, grad, rows, rows_per_block, sum_blocks, (int)slabs, (int)e->D, e->scale, add);
  }
  const SortPlan p = sort_plan(tok.N, rows, e->D);
  char* w = static_cast<char*>(e->scratch);
  uint8_t* touched = add ? nullptr : reinterpret_cast<uint8_t*>(w + p.o_touched);
  cudaError_t err;
  // rows cleared during the sort: about 4.5 MB for each of the 6 us and 1 us per 4096 tokens that it takes
  uint32_t cleared = 0;
  if (p.cluster && touched) {
    const uint64_t n = (uint64_t)(6 + p.N / 4096) * 4500000 / row_bytes;
    cleared = n < rows ? (uint32_t)n : rows;
  }
  if (cleared == rows) touched = nullptr;  // nothing is left to be cleared
  if (p.cluster) {
    const auto sort = p.items == 1   ? launch_cluster_sort<1, TG>
                      : p.items == 2 ? launch_cluster_sort<2, TG>
                      : p.items == 4 ? launch_cluster_sort<4, TG> : launch_cluster_sort<8, TG>;
    err = sort(p, tok, w, touched, cleared, grad, (int)e->D, s);
    if (err != cudaSuccess) return err;
  }
  if (!p.cluster && touched && (err = cudaMemsetAsync(touched, 0, rows, s)) != cudaSuccess) return err;
  const size_t bins = size_t(1) << p.bits;
  for (int i = 0; i < (p.cluster ? 0 : p.passes); ++i) {
    SortPass a{};
    a.key_in = i ? reinterpret_cast<uint32_t*>(w + p.o_key[(i - 1) & 1]) : nullptr;
    a.pos_in = i ? reinterpret_cast<uint32_t*>(w + p.o_pos[(i - 1) & 1]) : nullptr;
    a.key_out = reinterpret_cast<uint32_t*>(w + p.o_key[i & 1]);
    a.pos_out = reinterpret_cast<uint32_t*>(w + p.o_pos[i & 1]);
    a.counts = reinterpret_cast<uint32_t*>(w + p.o_counts);
    a.touched = i ? nullptr : touched;
    a.N = p.N;
    a.per_tile = p.per_tile;
    a.none_key = rows;
    a.shift = i * p.bits;
    a.bits = p.bits;
    a.tiles = p.tiles;
    if ((err = launch_pdl(embed_histogram_kernel, dim3(p.tiles), dim3(kSortThreads), bins * sizeof(uint32_t), s, tok, a)) != cudaSuccess)
      return err;
    if ((err = launch_pdl(embed_scatter_kernel, dim3(p.tiles), dim3(kSortThreads),
                          bins * (sizeof(uint32_t) + kSortWarps * sizeof(uint16_t)), s, tok, a)) != cudaSuccess)
      return err;
  }
  SumArgs a{};
  const int last = p.cluster ? 0 : (p.passes - 1) & 1;
  a.key = reinterpret_cast<uint32_t*>(w + p.o_key[last]);
  a.pos = reinterpret_cast<uint32_t*>(w + p.o_pos[last]);
  a.touched = touched;
  a.part = reinterpret_cast<float*>(w + p.o_part);
  a.N = p.N;
  a.T = tok.T;
  a.none_key = rows;
  a.piece = p.piece;
  a.pieces = p.pieces;
  a.slabs = slabs;
  a.sum_blocks = (uint32_t)(((uint64_t)p.pieces * slabs + kSumWarps - 1) / kSumWarps);
  a.rows_per_block = rows_per_block;
  a.D = e->D;
  a.scale = e->scale;
  a.add = add;
  a.clear_rows = add ? 0 : rows - cleared;
  const uint32_t zero_blocks = (a.clear_rows + rows_per_block - 1) / rows_per_block;
  if ((err = launch_pdl(embed_sum_kernel<TG, TA, VEC>, dim3(a.sum_blocks + zero_blocks), dim3(kSumThreads), 0, s, a, d_out, grad)) != cudaSuccess)
    return err;
  return launch_pdl(embed_join_kernel<TG, VEC>, dim3((p.pieces - 1 + kSumWarps - 1) / kSumWarps, slabs < 8 ? slabs : 8), dim3(kSumThreads), 0, s,
                    a, grad);                // more than kFewTokens positions are many pieces
}

template <int VEC>
cudaError_t dispatch(const lsgd_embed_desc* e, bool backward, cudaStream_t s) {
  using B = __nv_bfloat16;
  const bool tb = e->table_dtype == LSGD_BF16, ab = e->act_dtype == LSGD_BF16;
  if (!backward)
    return tb ? (ab ? launch_lookup<B, B, VEC>(e, s) : launch_lookup<B, float, VEC>(e, s))
              : (ab ? launch_lookup<float, B, VEC>(e, s) : launch_lookup<float, float, VEC>(e, s));
  return tb ? (ab ? launch_grad<B, B, VEC>(e, s) : launch_grad<B, float, VEC>(e, s))
            : (ab ? launch_grad<float, B, VEC>(e, s) : launch_grad<float, float, VEC>(e, s));
}

cudaError_t embed(const lsgd_embed_desc* e, bool backward, cudaStream_t s) {
  const int tb = elem_bytes(e->table_dtype), ab = elem_bytes(e->act_dtype);
  const lsgd_rows &table = backward ? e->d_table : e->table, &act = backward ? e->d_out : e->out;
  const int vec = min_vec(row_vec(table, e->P, e->V, e->D, tb), row_vec(act, e->P, e->T, e->D, ab));
  return vec == 8 ? dispatch<8>(e, backward, s) : vec == 2 ? dispatch<2>(e, backward, s) : dispatch<1>(e, backward, s);
}

}  // namespace
}  // namespace lsgd

extern "C" {

uint64_t lsgd_embed_scratch_bytes(const lsgd_embed_desc* e) {
  using namespace lsgd;
  if (!e || e->struct_size != sizeof(lsgd_embed_desc) || e->P < 1 || e->T < 0 || e->V < 1 || e->D < 1 || e->D > kMaxD) return 0;
  if (e->T >= (int64_t(1) << 31) / e->P || e->V >= (int64_t(1) << 31) / e->P) return 0;
  const uint32_t N = (uint32_t)(e->T * e->P);
  if (N <= kFewTokens) return 0;
  return sort_plan(N, shared_grad(e) ? (uint32_t)e->V : (uint32_t)(e->V * e->P), e->D).bytes;
}

lsgd_status lsgd_embed_forward(const lsgd_embed_desc* e, void* stream) {
  using namespace lsgd;
  const lsgd_status st = check_embed(e, false);
  if (st != LSGD_OK) return st;
  if (e->T == 0) return LSGD_OK;
  return embed(e, false, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
}

lsgd_status lsgd_embed_backward(const lsgd_embed_desc* e, void* stream) {
  using namespace lsgd;
  const lsgd_status st = check_embed(e, true);
  if (st != LSGD_OK) return st;
  const uint64_t need = lsgd_embed_scratch_bytes(e);
  if (need && (!e->scratch || e->scratch_bytes < need)) return LSGD_ERR_INVALID_ARG;
  if (need && reinterpret_cast<uintptr_t>(e->scratch) % 256) return LSGD_ERR_ALIGNMENT;
  return embed(e, true, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LSGD_OK : LSGD_ERR_CUDA;
}

lsgd_status lsgd_embed_check_device(uint32_t* flag_out) {
  using namespace lsgd;
  uint32_t f = 0, zero = 0;
  if (cudaDeviceSynchronize() != cudaSuccess) return LSGD_ERR_CUDA;
  if (cudaMemcpyFromSymbol(&f, g_embed_status, sizeof(f)) != cudaSuccess) return LSGD_ERR_CUDA;
  if (f && cudaMemcpyToSymbol(g_embed_status, &zero, sizeof(zero)) != cudaSuccess) return LSGD_ERR_CUDA;
  if (flag_out) *flag_out = f;
  return f ? LSGD_ERR_DEVICE_FLAG : LSGD_OK;
}

}  // extern "C"
