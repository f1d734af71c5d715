// embed_grad: the gradient of an embedding lookup by sorted tokens.
//
//   rows[u] = scale * sum of grad[p] over the positions p with key keys[u]
//
// The (key, position) pairs come sorted.  They are cut into spans, a block
// each, and a span into chunks, a row group each: a group walks its chunk's
// rows with several loads in flight, keeps the running sum of the current key
// in registers (fp32), and writes the sum of a key whose rows lie inside the
// chunk straight to its place.  Keys cut by a chunk's end leave partial sums
// in shared memory that the block adds in chunk order; keys that run past a
// span leave theirs in memory and grad_combine adds them in span order.  So
// each row is read once, each sum written once, a hot token's rows are spread
// over many groups, and the order of every sum is fixed by the input alone.
// Bound by memory where rows are many (64 x 4096 rows of 1024 bf16 elements of
// 62,000 tokens: grad_sum 126 us, 6.3 TB/s; the sort in front 26, the rest 8),
// by the latency of its launches where they are few (3 x 2003 rows of 200:
// sort 10, grad_sum 6.6, grad_combine 3 us).
//
// Where a sum goes: the index of its key among the distinct ones, which is the
// number of keys that begin before it: grad_heads counts those of each span,
// and a block of grad_sum adds the counts of the spans before its own (of a few
// thousand keys it counts them itself, which saves the launch).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "embed.cuh"
#include "rowgroup.cuh"

namespace adapm {

namespace {

constexpr int kGradSpan = 2048;   // sorted rows staged per block, at most
// grad_sum blocks per SM.  Two keep enough loads in flight; a third takes its
// shared memory from L1, which holds what is in flight (the case above 162 us in
// all with two, 165 to 188 with three, 167 with four; while a block took 67 KB
// of shared memory 205 with three and 240 and more with four).
constexpr int kGradBlocks = 2;
constexpr uint64_t kSpansSummed = 2048;   // spans whose counts every block of grad_sum sums up itself

// V elements of type T as they travel.
template <int BYTES>
struct Raw;
template <>
struct Raw<16> {
  using type = uint4;
};
template <>
struct Raw<8> {
  using type = uint2;
};
template <>
struct Raw<4> {
  using type = uint32_t;
};
template <>
struct Raw<2> {
  using type = uint16_t;
};
template <class T, int V>
using RawOf = typename Raw<(int)sizeof(T) * V>::type;

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }

template <class T, int V>
__device__ __forceinline__ void add_raw(float (&sum)[V], const RawOf<T, V>& raw) {
  const T* x = reinterpret_cast<const T*>(&raw);
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] += as_float(x[j]);
}
template <class T, int V>
__device__ __forceinline__ void set_raw(float (&sum)[V], const RawOf<T, V>& raw) {
  const T* x = reinterpret_cast<const T*>(&raw);
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] = as_float(x[j]);
}
// V floats to or from a row that begins on a multiple of min(V, 4) floats.
template <int V>
__device__ __forceinline__ void put_floats(float* p, const float (&x)[V], float scale) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int j = 0; j < V; j += 4)
      *reinterpret_cast<float4*>(p + j) =
          make_float4(x[j] * scale, x[j + 1] * scale, x[j + 2] * scale, x[j + 3] * scale);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) p[j] = x[j] * scale;
  }
}
template <int V>
__device__ __forceinline__ void add_floats(float (&x)[V], const float* p) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      const float4 v = *reinterpret_cast<const float4*>(p + j);
      x[j] += v.x;
      x[j + 1] += v.y;
      x[j + 2] += v.z;
      x[j + 3] += v.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] += p[j];
  }
}

// Whether a sort before gave up, or which arrays hold the sorted pairs.
__device__ __forceinline__ bool grad_resolve(GradArgs& a) {
  if (sort_failed(a.st)) return false;
  if (a.plan_word != nullptr && *a.plan_word == a.plan_seq) {
    a.skeys = a.alt_keys;
    a.spos = a.alt_pos;
  }
  return true;
}
__device__ __forceinline__ bool grad_valid(const GradArgs& a, uint32_t k) { return k < a.K && k != a.pad_key; }

// heads[b] = distinct keys that begin in span b.
__global__ void __launch_bounds__(kThreads) grad_heads_kernel(const GradArgs args, uint32_t span) {
  after_previous();
  GradArgs a = args;
  if (!grad_resolve(a)) return;
  const uint64_t p0 = (uint64_t)blockIdx.x * span;
  const uint64_t p1 = p0 + span < a.n ? p0 + span : a.n;
  uint32_t heads = 0, unused = 0;
  for (uint64_t p = p0 + threadIdx.x; p < p1; p += kThreads) {
    const uint32_t k = a.skeys[p];
    heads += grad_valid(a, k) && (p == 0 || a.skeys[p - 1] != k) ? 1u : 0u;
  }
  block_sum2(heads, unused);
  if (threadIdx.x == 0) a.heads[blockIdx.x] = heads;
}

// Very many spans: their counts summed up by one block, so that grad_sum need
// not read all of them.  heads[b] becomes the keys that begin before span b,
// heads[spans] all.
__global__ void __launch_bounds__(kThreads) grad_scan_kernel(const GradArgs args, uint32_t spans) {
  after_previous();
  if (sort_failed(args.st)) return;
  uint32_t run = 0;
  for (uint32_t b0 = 0; b0 < spans; b0 += kThreads) {
    const uint32_t b = b0 + threadIdx.x;
    uint32_t h = b < spans ? args.heads[b] : 0u, unused = 0, total, none;
    block_exclusive_scan2(h, unused, total, none);
    if (b < spans) args.heads[b] = run + h;
    run += total;
  }
  if (threadIdx.x == 0) args.heads[spans] = run;
}

// A thread's share of the distinct keys that begin before span b, and in all:
// from the spans' counts, or from the keys themselves where there are few.
__device__ __forceinline__ void grad_ranks(const GradArgs& a, uint32_t b, uint32_t spans, uint64_t P0, uint32_t& below,
                                           uint32_t& all) {
  below = all = 0;
  if (a.scanned) {
    if (threadIdx.x == 0) {
      below = a.heads[b];
      all = a.heads[spans];
    }
    return;
  }
  if (a.heads != nullptr) {
#pragma unroll 4
    for (uint32_t m = threadIdx.x; m < spans; m += kThreads) {
      const uint32_t h = a.heads[m];
      all += h;
      if (m < b) below += h;
    }
    return;
  }
  const uint32_t n = (uint32_t)a.n;
  auto count = [&](uint32_t p, uint32_t k, uint32_t prev) {
    const uint32_t h = grad_valid(a, k) && prev != k ? 1u : 0u;
    all += h;
    if (p < P0) below += h;
  };
#pragma unroll 4
  for (uint32_t p = 4 * threadIdx.x; p + 4 <= n; p += 4 * kThreads) {
    const uint4 v = *reinterpret_cast<const uint4*>(a.skeys + p);
    count(p, v.x, p > 0 ? a.skeys[p - 1] : kNoKey);
    count(p + 1, v.y, v.x);
    count(p + 2, v.z, v.y);
    count(p + 3, v.w, v.z);
  }
  const uint32_t p = n / 4 * 4 + threadIdx.x;
  if (p < n) count(p, a.skeys[p], p > 0 ? a.skeys[p - 1] : kNoKey);
}

// Dynamic shared memory of grad_sum: the head piece of every chunk, then the
// span's keys (with the one before and the one after), rows and flags.  What it
// takes, L1 lacks for the loads in flight.
template <int C, int V>
constexpr size_t grad_smem() {
  return (size_t)kThreads * C * V * sizeof(float) +
         kGradSpan * (2 * sizeof(uint32_t) + sizeof(uint8_t)) + (kGradSpan + 2) * sizeof(uint32_t);
}

// Row flags: the first of its key in its chunk; the last of its key, or of the
// chunk; the key begins in the chunk; it ends at this row; the row counts.
constexpr uint8_t kBegin = 1, kEnd = 2, kStarted = 4, kLast = 8, kCounts = 16;

// Blocks of one span are next to each other, one per tile of columns.
template <class T, int V, int G, int C, int R>
__global__ void __launch_bounds__(kThreads, kGradBlocks) grad_sum_kernel(const GradArgs args, uint32_t spans,
                                                                         uint32_t tiles, uint32_t tile) {
  after_previous();
  GradArgs a = args;
  if (!grad_resolve(a)) return;
  constexpr int NG = kThreads / G;
  const uint32_t CH = a.chunk, span = NG * CH;
  extern __shared__ __align__(16) unsigned char dsm[];
  float* ph = reinterpret_cast<float*>(dsm);                 // head piece of each chunk
  uint32_t* sp = reinterpret_cast<uint32_t*>(ph + kThreads * C * V);   // position of each row
  uint32_t* su = sp + kGradSpan;                             // index of its key among the distinct ones
  uint32_t* sk = su + kGradSpan;                             // sk[0]: key before the span; sk[1 + len]: after it
  uint8_t* sf = reinterpret_cast<uint8_t*>(sk + kGradSpan + 2);
  const int lane = threadIdx.x & (G - 1);
  const uint32_t gi = threadIdx.x / G;
  const uint32_t b = blockIdx.x / tiles, q0 = (blockIdx.x - b * tiles) * tile;   // first vector of the tile
  const uint32_t nv = (a.dim + V - 1) / V - q0 < tile ? (a.dim + V - 1) / V - q0 : tile;
  const T* grad = reinterpret_cast<const T*>(a.grad.data) + q0 * V;
  float* rows = a.rows + q0 * V;
  float* parts = a.parts + q0 * V;
  const uint64_t P0 = (uint64_t)b * span;
  const uint32_t len = (uint32_t)(a.n - P0 < (uint64_t)span ? a.n - P0 : span);
  // the span's keys and positions, and the counts in front of it, in one
  // latency; then one scan: a row's rank is the heads of the rounds and warps
  // before it plus those of the lanes before
  constexpr int NR = kGradSpan / kThreads, NW = kThreads / 32;
  __shared__ uint32_t heads[NR * NW], sums[2][NW];
  const int lane32 = threadIdx.x & 31, warp = threadIdx.x / 32;
  uint32_t pos[NR];
#pragma unroll
  for (int j = 0; j < NR; ++j) {
    const uint32_t i = j * kThreads + threadIdx.x;
    pos[j] = i < len ? a.spos[P0 + i] : 0u;
    if (i < len) sk[1 + i] = a.skeys[P0 + i];
  }
  if (threadIdx.x == 0) {
    sk[0] = P0 > 0 ? a.skeys[P0 - 1] : kNoKey;
    sk[1 + len] = P0 + len < a.n ? a.skeys[P0 + len] : kNoKey;
  }
  uint32_t below, all;
  grad_ranks(a, b, spans, P0, below, all);
  below = __reduce_add_sync(0xFFFFFFFFu, below);
  all = __reduce_add_sync(0xFFFFFFFFu, all);
  if (lane32 == 0) {
    sums[0][warp] = below;
    sums[1][warp] = all;
  }
  __syncthreads();
  uint32_t head[NR];   // lanes of the warp whose row is the first of its key
#pragma unroll
  for (int j = 0; j < NR; ++j) {
    const uint32_t i = j * kThreads + threadIdx.x;
    const bool h = i < len && grad_valid(a, sk[1 + i]) && sk[i] != sk[1 + i];   // (sk[0] is kNoKey in front of the first)
    head[j] = __ballot_sync(0xFFFFFFFFu, h);
    if (lane32 == 0) heads[j * NW + warp] = __popc(head[j]);
  }
  __syncthreads();
  if (warp == 0) {   // exclusive scan of the NR * NW counts, two a lane
    static_assert(NR * NW == 64, "");
    const uint32_t h0 = heads[2 * lane32], h1 = heads[2 * lane32 + 1];
    uint32_t x = h0 + h1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, x, o);
      if (lane32 >= o) x += y;
    }
    heads[2 * lane32] = x - h0 - h1;
    heads[2 * lane32 + 1] = x - h1;
  }
  uint32_t first = 0, total = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    first += sums[0][w];
    total += sums[1][w];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.count = total;
  __syncthreads();
  bool wrong = false;
#pragma unroll
  for (int j = 0; j < NR; ++j) {
    const uint32_t i = j * kThreads + threadIdx.x;
    if (i >= len) break;
    const uint32_t k = sk[1 + i];
    const bool counts = grad_valid(a, k), begins = (head[j] >> lane32) & 1u;
    uint8_t f = 0;
    if (counts && pos[j] < a.n) {
      const uint32_t cs = i - i % CH, ce = cs + CH < len ? cs + CH : len;
      const bool ends = sk[2 + i] != k;
      f = kCounts | (begins || i == cs ? kBegin : 0) | (ends || i + 1 == ce ? kEnd : 0) |
          (sk[cs] != k ? kStarted : 0) | (ends ? kLast : 0);
      sp[i] = pos[j];
    } else if (counts || (k >= a.K && k != kNoKey)) {
      wrong = true;
    }
    sf[i] = f;
    // heads up to and including this row, less one
    const uint32_t u = first + heads[j * NW + warp] + __popc(head[j] & (0xFFFFFFFFu >> (31 - lane32))) - 1;
    su[i] = u;
    if (q0 == 0) {
      if (begins) a.keys[u] = k;
      if (i + 1 == len) a.crossing[b] = u;
      if (P0 + i >= total) a.keys[P0 + i] = kNoKey;
    }
  }
  if (__syncthreads_or(wrong) && threadIdx.x == 0) set_error(a.st, ERR_INTERNAL);
  const uint32_t p0 = gi * CH < len ? gi * CH : len;
  const uint32_t p1 = p0 + CH < len ? p0 + CH : len;
  float run[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int j = 0; j < V; ++j) run[c][j] = 0.f;
  auto fetch = [&](uint32_t p, uint8_t (&f)[R], RawOf<T, V> (&d)[R][C]) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      f[r] = p + r < p1 ? sf[p + r] : 0;
      const T* row = grad + (f[r] & kCounts ? row_offset(a.grad, sp[p + r]) : 0);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const uint32_t q = lane + c * G;
        if ((f[r] & kCounts) && q < nv)
          d[r][c] = *reinterpret_cast<const RawOf<T, V>*>(row + q * V);
        else
          d[r][c] = RawOf<T, V>{};
      }
    }
  };
  auto add = [&](uint32_t p, const uint8_t (&f)[R], const RawOf<T, V> (&d)[R][C]) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (!(f[r] & kCounts)) continue;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if (f[r] & kBegin) set_raw<T, V>(run[c], d[r][c]);
        else add_raw<T, V>(run[c], d[r][c]);
      }
      if (!(f[r] & kEnd)) continue;
      if ((f[r] & (kStarted | kLast)) == (kStarted | kLast)) {
        float* row = rows + (uint64_t)su[p + r] * a.dim;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const uint32_t q = lane + c * G;
          if (q < nv) put_floats<V>(row + q * V, run[c], a.scale);
        }
      } else if (!(f[r] & kStarted)) {   // the chunk's head piece (a tail piece stays in the registers)
#pragma unroll
        for (int c = 0; c < C; ++c) put_floats<V>(ph + (gi * G * C + lane + c * G) * V, run[c], 1.f);
      }
    }
  };
  for (uint32_t p = p0; p < p1; p += R) {
    uint8_t f[R];
    RawOf<T, V> d[R][C];
    fetch(p, f, d);
    add(p, f, d);
  }
  __syncthreads();
  // A key that begins in chunk gi and goes on is summed here by group gi: its
  // tail piece (the running sum), then the head pieces of the chunks it covers.
  const uint32_t nch = (len + CH - 1) / CH;
  auto chunk_end = [&](uint32_t m) { return (m + 1) * CH < len ? (m + 1) * CH : len; };
  auto walk = [&](uint32_t m, uint32_t kk, bool& out) {   // last chunk from m on that kk covers; past the span?
    while (true) {
      const uint32_t e = chunk_end(m);
      const bool through = sk[e] == kk && sk[1 + e] == kk;
      if (!through || m + 1 >= nch) {
        out = through;
        return m;
      }
      ++m;
    }
  };
  auto add_pieces = [&](uint32_t m0, uint32_t m1) {
    for (uint32_t m = m0; m <= m1; ++m)
#pragma unroll
      for (int c = 0; c < C; ++c) add_floats<V>(run[c], ph + (m * G * C + lane + c * G) * V);
  };
  auto put_row = [&](float* row, float scale) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint32_t q = lane + c * G;
      if (q < nv) put_floats<V>(row + q * V, run[c], scale);
    }
  };
  if (gi < nch) {
    const uint32_t kl = sk[p1];   // the chunk's last row
    if (grad_valid(a, kl) && sk[1 + p1] == kl && sk[p0] != kl) {
      bool out = true;
      const uint32_t m1 = gi + 1 < nch ? walk(gi + 1, kl, out) : gi;
      add_pieces(gi + 1, m1);
      if (out) put_row(parts + (2 * (uint64_t)b + 1) * a.dim, 1.f);
      else put_row(rows + (uint64_t)su[p1 - 1] * a.dim, a.scale);
    }
  }
  if (gi == 0 && sk[0] == sk[1] && grad_valid(a, sk[1])) {   // the span's first key began before it
    bool out = false;
    const uint32_t m1 = walk(0, sk[1], out);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < V; ++j) run[c][j] = 0.f;
    add_pieces(0, m1);
    put_row(parts + 2 * (uint64_t)b * a.dim, 1.f);
  }
}

// Keys that run past a span: the tail piece of the span where one begins plus
// the head pieces of the spans that it continues into.  A block per span and
// tile of 32 vectors; its warps take the head pieces in strides, in increasing
// order and several in flight, then the warps' sums are added in warp order.
template <int V>
__global__ void __launch_bounds__(kThreads) grad_combine_kernel(const GradArgs args, uint32_t span, uint32_t spans,
                                                                uint32_t tiles) {
  after_previous();
  GradArgs a = args;
  if (!grad_resolve(a)) return;
  constexpr int NW = kThreads / 32, UB = 8;
  __shared__ float part[NW][32 * V];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const uint32_t b = blockIdx.x / tiles, c0 = ((blockIdx.x - b * tiles) * 32 + lane) * V;
  const uint64_t st = (uint64_t)b * span, en = st + span;
  // the keys around the span's end and before its start, and the first keys of
  // the spans after it, in one latency
  const uint32_t kl = a.skeys[en - 1], kn = a.skeys[en], kb = st > 0 ? a.skeys[st - 1] : kNoKey;
  uint32_t kf = b + 1 + threadIdx.x < spans ? a.skeys[(uint64_t)(b + 1 + threadIdx.x) * span] : kNoKey;
  const uint32_t u = a.crossing[b];
  if (!grad_valid(a, kl) || kn != kl || kb == kl) return;   // (uniform) none, or it began in an earlier span
  // the last span whose first row has the key: those after b that do are a prefix
  uint32_t lo = b;
  for (uint32_t m0 = b + 1; m0 < spans; m0 += kThreads) {
    if (m0 > b + 1) kf = m0 + threadIdx.x < spans ? a.skeys[(uint64_t)(m0 + threadIdx.x) * span] : kNoKey;
    const int same = __syncthreads_count(kf == kl);
    lo += (uint32_t)same;
    if (same < kThreads) break;
  }
  float sum[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] = 0.f;
  if (c0 < a.dim) {
    for (uint32_t m0 = b + 1 + warp; m0 <= lo; m0 += NW * UB) {
      float x[UB][V];
#pragma unroll
      for (int r = 0; r < UB; ++r) {
#pragma unroll
        for (int j = 0; j < V; ++j) x[r][j] = 0.f;
        if (m0 + r * NW <= lo) add_floats<V>(x[r], a.parts + 2 * (uint64_t)(m0 + r * NW) * a.dim + c0);
      }
#pragma unroll
      for (int r = 0; r < UB; ++r)
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += x[r][j];
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) part[warp][j * 32 + lane] = sum[j];
  __syncthreads();
  if (warp == 0 && c0 < a.dim) {
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = 0.f;
    add_floats<V>(sum, a.parts + (2 * (uint64_t)b + 1) * a.dim + c0);
#pragma unroll
    for (int w = 0; w < NW; ++w)
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] += part[w][j * 32 + lane];
    put_floats<V>(a.rows + (uint64_t)u * a.dim + c0, sum, a.scale);
  }
}

// Columns are cut into tiles of at most 32 * most_vectors(V) vectors, so that a
// lane's sums and the rows it has in flight leave registers for kGradBlocks
// blocks per SM.  Few rows take one vector per lane (more, shorter blocks).
constexpr int most_vectors(int V) { return V == 8 ? 2 : (V == 4 ? 4 : 8); }
constexpr uint64_t kFewRows = 4096;

struct GradTiles {
  uint32_t tiles, tile;   // of so many vectors
};
template <int V>
GradTiles grad_tiles(const GradArgs& a) {
  const uint32_t nv = (a.dim + V - 1) / V, most = 32 * (a.n <= kFewRows ? 1 : most_vectors(V));
  const uint32_t tiles = (nv + most - 1) / most;
  return {tiles, (nv + tiles - 1) / tiles};
}

// Lanes per row group and vectors of a tile's row per lane.
template <int V, class F>
void dispatch_grad(uint32_t tile, F&& f) {
  if (tile <= 4) f(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
  else if (tile <= 8) f(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
  else if (tile <= 16) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
  else if (tile <= 32) f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
  else if (tile <= 64) f(std::integral_constant<int, 32>{}, std::integral_constant<int, 2>{});
  else if constexpr (V < 8) {
    if (V >= 4 && tile <= 96) f(std::integral_constant<int, 32>{}, std::integral_constant<int, 3>{});
    else if (tile <= 128) f(std::integral_constant<int, 32>{}, std::integral_constant<int, 4>{});
    else if constexpr (V < 4) f(std::integral_constant<int, 32>{}, std::integral_constant<int, 8>{});
  }
}

// Elements a lane loads at a time: the most that every row's start and length
// are a multiple of.  (Sums of four and more are written as vectors.)
template <class T>
int grad_vector(const GradArgs& a) {
  for (int v = 16 / (int)sizeof(T); v > 1; v /= 2) {
    if (reinterpret_cast<uintptr_t>(a.grad.data) % (v * sizeof(T)) == 0 && a.dim % v == 0 &&
        a.grad.inner_stride % v == 0 && (a.grad.flat || a.grad.outer_stride % v == 0) &&
        (v < 4 || reinterpret_cast<uintptr_t>(a.rows) % 16 == 0))
      return v;
  }
  return 1;
}

template <class T, class F>
void dispatch_grad_args(const GradArgs& a, F&& f) {
  const int v = grad_vector<T>(a);
  auto by_v = [&](auto Vc) {
    const GradTiles t = grad_tiles<decltype(Vc)::value>(a);
    dispatch_grad<decltype(Vc)::value>(t.tile, [&](auto Gc, auto Cc) { f(Vc, Gc, Cc, t); });
  };
  if constexpr (sizeof(T) == 2)
    if (v == 8) return by_v(std::integral_constant<int, 8>{});
  if (v >= 4) return by_v(std::integral_constant<int, 4>{});
  if (v == 2) return by_v(std::integral_constant<int, 2>{});
  by_v(std::integral_constant<int, 1>{});
}

template <class T>
GradPlan grad_plan_typed(const GradArgs& a, int sms) {
  GradPlan p{};
  dispatch_grad_args<T>(a, [&](auto, auto Gc, auto, GradTiles t) {
    constexpr uint64_t NG = kThreads / decltype(Gc)::value, most = kGradSpan / NG;
    // one span per resident block, or as few full waves of them as spans allow
    const uint64_t groups = NG * std::max<uint64_t>(1, (uint64_t)sms * kGradBlocks / t.tiles);
    const uint64_t waves = (a.n + groups * most - 1) / (groups * most);
    uint64_t ch = (a.n + groups * waves - 1) / (groups * waves);
    if (ch < 8) ch = 8;
    if (ch > most) ch = most;
    p.chunk = (uint32_t)ch;
    p.spans = (a.n + NG * ch - 1) / (NG * ch);
  });
  p.count_heads = a.n > kCountSort;
  p.scan_heads = p.spans > kSpansSummed;
  return p;
}

template <class T>
void launch_grad_typed(const GradArgs& a, const GradPlan& p, cudaStream_t stream) {
  dispatch_grad_args<T>(a, [&](auto Vc, auto Gc, auto Cc, GradTiles t) {
    constexpr int V = decltype(Vc)::value, G = decltype(Gc)::value, C = decltype(Cc)::value;
    constexpr int R = 8 / C;
    const uint32_t span = p.chunk * (kThreads / G), spans = (uint32_t)p.spans;
    note_launches((p.count_heads ? 1 : 0) + (p.scan_heads ? 1 : 0) + (spans > 1 ? 2 : 1));
    if (p.count_heads) launch_after(grad_heads_kernel, spans, kThreads, 0, stream, a, span);
    if (p.scan_heads) launch_after(grad_scan_kernel, 1, kThreads, 0, stream, a, spans);
    constexpr size_t smem = grad_smem<C, V>();
    // the kernel's dynamic shared-memory limit is a per-device attribute
    static bool attr_set[64] = {false};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
      cudaFuncSetAttribute(grad_sum_kernel<T, V, G, C, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
      if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    launch_after(grad_sum_kernel<T, V, G, C, R>, spans * t.tiles, kThreads, smem, stream, a, spans, t.tiles, t.tile);
    if (spans > 1) {
      const uint32_t tiles = (a.dim + 32 * V - 1) / (32 * V);
      launch_after(grad_combine_kernel<V>, (spans - 1) * tiles, kThreads, 0, stream, a, span, spans, tiles);
    }
  });
}

}  // namespace
}  // namespace adapm
