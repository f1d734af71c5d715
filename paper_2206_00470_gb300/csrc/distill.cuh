// Distillation from a teacher's top logits: the loss of every row of student
// logits and its gradient.
//
// Row r has student logits s_v, a list of (id_j, t_j), and perhaps a label y:
//
//   p = softmax over the list of t_j / T,  q = softmax of s / T,  c = softmax of s
//   loss = soft T^2 sum_j p_j (ln p_j - ln q_id_j) + hard (-ln c_y)
//   grad_v = f (soft T (q_v - sum_{id_j = v} p_j) + hard (c_v - [v = y])),  f = scale weights[r]
//
// Three launches, or one where there are few rows (distill_few).  distill_lists,
// a warp per row: the list's p, one entry for all that share an id, and the
// logits at its ids and at the label.  distill_rows: sums of exponentials of
// each row and the part of the gradient that every element has, from one
// reading.  distill_marks, a warp per row: the loss, and the few elements that
// list and label change.
//
// The second launch comes in three forms.  distill_rows, for rows of up to 16
// KB: a block keeps its row in registers, packed as it came.  distill_slices,
// up to 1 MB: the blocks of a cluster keep a slice of the row each, which was
// copied to shared memory while they worked on the row before it, and exchange
// their sums.  distill_long: the blocks of a cluster read a slice twice, the
// second time from L2.
// Every warp sums relative to its own maximum, so one exchange per row is
// enough.  Bound by memory, a read and a write of the logits: 4096 rows of
// 250,000 bf16 646 to 655 us, 6.3 TB/s.  3060 rows of 50,021, a quarter of them
// padding, each by two blocks: 134 to 143 us (two exponentials: 152), 79 at the
// memory's rate; a row's exchange takes as long as its slices' work, and only two
// blocks an SM run beside it.  Seven rows of 32,000 by the one launch 9 us.  Far
// from that rate: short rows by their lists (34,584 rows of 384 bf16 92 us, 9 at
// the rate), rows read twice (16 of 700,000 fp32 54, 13).
#pragma once

#include <cooperative_groups.h>

#include <algorithm>

#include "barrier.cuh"
#include "dense.cuh"

namespace adapm {

namespace {

namespace cg = cooperative_groups;

constexpr float kLog2E = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kMaxCluster = 16;
constexpr uint32_t kEmpty = 0x7FFFFFFFu;

template <int TYPE>
struct Word {
  static constexpr int kSize = TYPE == ADAPM_F32 ? 4 : 2;
  static constexpr int kElements = 16 / kSize;
  static constexpr uint32_t kNone = TYPE == ADAPM_F32 ? 0xFF800000u : (TYPE == ADAPM_BF16 ? 0xFF80FF80u : 0xFC00FC00u);   // -inf
};
template <int TYPE>
__device__ __forceinline__ void unpack_word(const uint4& v, float (&x)[Word<TYPE>::kElements]) {
  if constexpr (TYPE == ADAPM_F32) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  } else {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = unpack2<TYPE>(w[j]);
      x[2 * j] = f.x;
      x[2 * j + 1] = f.y;
    }
  }
}

// A row in aligned 16-byte words from `base` on: elements [head, head + vocab)
// of them.  Its first and last word may hold elements that are not the row's;
// those are neither read nor written.
struct RowWords {
  char* base;
  uint32_t head;
  uint32_t words;
  uint32_t full0, full1;   // the words that hold nothing else
};
template <int TYPE>
__device__ __forceinline__ RowWords row_words(const RowView& v, uint64_t row, uint32_t vocab) {
  constexpr uint32_t S = Word<TYPE>::kSize, E = Word<TYPE>::kElements;
  char* p = v.data + row_offset(v, (uint32_t)row) * S;
  const uint32_t in = (uint32_t)reinterpret_cast<uintptr_t>(p) & 15u;
  RowWords b;
  b.head = in / S;
  b.base = p - in;
  b.words = (b.head + vocab + E - 1) / E;
  b.full0 = b.head != 0 ? 1 : 0;
  b.full1 = (b.head + vocab) / E;
  return b;
}
// Word w of a row; elements that are not the row's are -inf.
template <int TYPE>
__device__ __noinline__ uint4 load_edge(const char* base, uint32_t head, uint32_t vocab, uint32_t w) {
  constexpr uint32_t S = Word<TYPE>::kSize, E = Word<TYPE>::kElements;
  const char* p = base + (uint64_t)w * 16;
  uint32_t x[4] = {Word<TYPE>::kNone, Word<TYPE>::kNone, Word<TYPE>::kNone, Word<TYPE>::kNone};
#pragma unroll
  for (uint32_t j = 0; j < E; ++j) {
    if (w * E + j - head >= vocab) continue;   // (unsigned: in front of the row too)
    if constexpr (S == 4) x[j] = *reinterpret_cast<const uint32_t*>(p + j * S);
    else x[j / 2] = (x[j / 2] & (0xFFFFu << (16 * (1 - (j & 1))))) |
                    ((uint32_t)*reinterpret_cast<const uint16_t*>(p + j * S) << (16 * (j & 1)));
  }
  return make_uint4(x[0], x[1], x[2], x[3]);
}
template <int TYPE>
__device__ __forceinline__ uint4 load_word(const RowWords& b, uint32_t vocab, uint32_t w) {
  if (w >= b.full0 && w < b.full1) return *reinterpret_cast<const uint4*>(b.base + (uint64_t)w * 16);
  if (w < b.words) return load_edge<TYPE>(b.base, b.head, vocab, w);
  return make_uint4(Word<TYPE>::kNone, Word<TYPE>::kNone, Word<TYPE>::kNone, Word<TYPE>::kNone);
}
// A word's worth of elements from number `shift` (less than a word's) of two
// words on.
template <int TYPE>
__device__ __forceinline__ uint4 shift_words(const uint4& lo, const uint4& hi, uint32_t shift) {
  uint32_t x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  const uint32_t bytes = shift * Word<TYPE>::kSize;
  if (bytes & 8u)
#pragma unroll
    for (int j = 0; j < 6; ++j) x[j] = x[j + 2];
  if (bytes & 4u)
#pragma unroll
    for (int j = 0; j < 5; ++j) x[j] = x[j + 1];
  const uint32_t bits = (bytes & 3u) * 8u;
  return make_uint4(__funnelshift_r(x[0], x[1], bits), __funnelshift_r(x[1], x[2], bits), __funnelshift_r(x[2], x[3], bits),
                    __funnelshift_r(x[3], x[4], bits));
}
// The elements of word w of another row of the same elements, whose words
// begin `shift` elements further on in b's.
template <int TYPE>
__device__ __forceinline__ uint4 load_shifted(const RowWords& b, uint32_t vocab, uint32_t w, uint32_t shift) {
  const uint4 lo = load_word<TYPE>(b, vocab, w);
  if (shift == 0) return lo;
  return shift_words<TYPE>(lo, load_word<TYPE>(b, vocab, w + 1), shift);
}
template <int TYPE>
__device__ __noinline__ void store_edge(char* base, uint32_t head, uint32_t vocab, uint32_t w, uint4 v) {
  constexpr uint32_t S = Word<TYPE>::kSize, E = Word<TYPE>::kElements;
  char* p = base + (uint64_t)w * 16;
  const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (uint32_t j = 0; j < E; ++j) {
    if (w * E + j - head >= vocab) continue;
    if constexpr (S == 4) *reinterpret_cast<uint32_t*>(p + j * S) = x[j];
    else *reinterpret_cast<uint16_t*>(p + j * S) = (uint16_t)(x[j / 2] >> (16 * (j & 1)));
  }
}
template <int TYPE>
__device__ __forceinline__ void store_word(const RowWords& g, uint32_t vocab, uint32_t w, uint4 v) {
  if (w >= g.full0 && w < g.full1) *reinterpret_cast<uint4*>(g.base + (uint64_t)w * 16) = v;
  else if (w < g.words) store_edge<TYPE>(g.base, g.head, vocab, w, v);
}
template <int TYPE>
__device__ __forceinline__ uint4 pack_word(const float (&y)[Word<TYPE>::kElements]) {
  if constexpr (TYPE == ADAPM_F32)
    return make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]));
  else
    return make_uint4(pack2<TYPE>(y[0], y[1]), pack2<TYPE>(y[2], y[3]), pack2<TYPE>(y[4], y[5]), pack2<TYPE>(y[6], y[7]));
}

// What distill_lists finds out about a row.
struct RowTask {
  float plogp;      // sum of p ln p over the list
  float label_s;    // the label's logit
  int32_t label;    // -1: none
  int32_t some;     // whether the list has entries
};
// What distill_rows finds out: largest logit, and sums of exp((s - max) / T)
// and, with two temperatures, of exp(s - max).
struct RowSums {
  float max, t, one;
};
// An entry: the p of all that share its id, and the id's logit.
struct Entry {
  uint32_t id;   // kNoKey: none, or another one speaks for it
  float p, s;
};

static_assert(sizeof(RowTask) == kTaskBytes && sizeof(RowSums) == kRowSumBytes && sizeof(Entry) == kEntryBytes);

__device__ __forceinline__ int64_t id_at(const void* ids, bool wide, uint64_t i) {
  return wide ? static_cast<const int64_t*>(ids)[i] : (int64_t)static_cast<const int32_t*>(ids)[i];
}
__device__ __forceinline__ float lanes_max(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
  return x;
}

// A warp's entries of a row in shared memory, and the table of slots (`table`,
// a power of two of at least twice as many) that finds ids listed twice.
struct Lists {
  uint32_t *id, *slot, *tab;
  float *t, *s;
  static __host__ __device__ constexpr uint32_t words(uint32_t top, uint32_t table) { return 4 * top + table; }
  __device__ __forceinline__ Lists(uint32_t* at, uint32_t top)
      : id(at), slot(at + top), tab(at + 4 * top), t(reinterpret_cast<float*>(at + 2 * top)), s(reinterpret_cast<float*>(at + 3 * top)) {}
};
// Warp-wide: what there is to learn from a row's list and label.  Afterwards
// l.id[j] is the id of entry j (kNoKey: none, or another one speaks for it),
// l.t[j] its p and l.s[j] its logit.  The loads are in two steps, each all at
// once: entries, then logits.
template <int TYPE>
__device__ __forceinline__ RowTask read_lists(const DistillArgs& a, uint64_t row, const Lists& l, uint32_t table) {
  const int lane = threadIdx.x & 31;
  const char* const logits = a.logits.data + row_offset(a.logits, (uint32_t)row) * Word<TYPE>::kSize;
  RowTask task{0.f, 0.f, -1, 0};
  bool bad = false;
  if (a.labels != nullptr) {
    const int64_t y = id_at(a.labels, a.wide_labels, row);
    if (!(a.has_pad && y == a.pad)) {
      if (y >= 0 && y < (int64_t)a.vocab) task.label = (int32_t)y;
      else bad = true;
    }
    if (task.label >= 0) task.label_s = load_as(logits, TYPE, task.label);
  }
  if (a.top > 0) {
    for (uint32_t j = lane; j < table; j += 32) l.tab[j] = kEmpty;
    // T ln p_j = t_j - t_max - T ln(sum)
    float largest = -INFINITY;
#pragma unroll 4
    for (uint32_t j = lane; j < a.top; j += 32) {
      const uint64_t at = row * a.top + j;
      const int64_t id = id_at(a.ids, a.wide, at);
      const float t = load_as(static_cast<const char*>(a.teacher), a.teacher_type, at);
      const bool here = id >= 0 && id < (int64_t)a.vocab && t != -INFINITY;
      bad = bad || id >= (int64_t)a.vocab || id < -1;
      l.id[j] = here ? (uint32_t)id : kNoKey;
      l.t[j] = t;
      l.s[j] = here ? load_as(logits, TYPE, id) : 0.f;
      if (here) {
        task.some = 1;
        largest = fmaxf(largest, t);
      }
    }
    __syncwarp();
    largest = lanes_max(largest);
    task.some = __any_sync(0xFFFFFFFFu, task.some);
    const float per_t = kLog2E / a.temperature, inv_t = 1.f / a.temperature;
    bool doubled = false;
    float sum = 0.f;
    for (uint32_t j = lane; j < a.top; j += 32) {
      const uint32_t id = l.id[j];
      if (id == kNoKey) continue;
      sum += exp2_of((l.t[j] - largest) * per_t);
      // the first entry of an id speaks for all (the table has twice as many slots as there are entries)
      uint32_t h = (id * 2654435761u) & (table - 1);
      while (true) {
        const uint32_t old = atomicCAS(&l.tab[h], kEmpty, j);
        if (old == kEmpty) break;
        if (l.id[old] == id) {
          atomicMin(&l.tab[h], j);
          doubled = true;
          break;
        }
        h = (h + 1) & (table - 1);
      }
      l.slot[j] = h;
    }
    __syncwarp();
    doubled = __any_sync(0xFFFFFFFFu, doubled);
    sum = lanes_sum(sum, 32);
    const float log_sum = logf(sum);
    for (uint32_t j = lane; j < a.top; j += 32) {
      if (l.id[j] == kNoKey) continue;
      const float d = l.t[j] - largest, p = exp2_of(d * per_t) / sum;
      if (p != 0.f) task.plogp += p * (d * inv_t - log_sum);
      l.t[j] = p;
    }
    task.plogp = lanes_sum(task.plogp, 32);
    __syncwarp();
    if (doubled) {
      for (uint32_t j = lane; j < a.top; j += 32) {
        if (l.id[j] == kNoKey || l.tab[l.slot[j]] != j) continue;
        float p = l.t[j];
        for (uint32_t i = j + 1; i < a.top; ++i)
          if (l.id[i] == l.id[j]) p += l.t[i];
        l.t[j] = p;   // (an entry that speaks is no other one's)
      }
      __syncwarp();
      for (uint32_t j = lane; j < a.top; j += 32)
        if (l.id[j] != kNoKey && l.tab[l.slot[j]] != j) l.id[j] = kNoKey;
      __syncwarp();
    }
  }
  if (bad) set_error(a.st, ERR_KEY_RANGE);
  return task;
}

constexpr int kListWarps = 4;
template <int TYPE>
__global__ void __launch_bounds__(kListWarps * 32)
distill_lists_kernel(const __grid_constant__ DistillArgs a, uint32_t table) {
  after_previous();
  extern __shared__ uint32_t lists[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Lists l(lists + warp * Lists::words(a.top, table), a.top);
  for (uint64_t row = (uint64_t)blockIdx.x * kListWarps + warp; row < a.n; row += (uint64_t)gridDim.x * kListWarps) {
    const RowTask task = read_lists<TYPE>(a, row, l, table);
    for (uint32_t j = lane; j < a.top; j += 32) static_cast<Entry*>(a.entries)[row * a.top + j] = Entry{l.id[j], l.t[j], l.s[j]};
    __syncwarp();
    if (lane == 0) static_cast<RowTask*>(a.tasks)[row] = task;
  }
}

// Coefficients of a row's two exponentials in its gradient.
struct RowScale {
  float t, one;
};
__device__ __forceinline__ float row_weight(const DistillArgs& a, uint64_t row) {
  return a.weights != nullptr ? a.scale * a.weights[row] : a.scale;
}
__device__ __forceinline__ RowScale row_scale(const DistillArgs& a, float f, const RowTask& task, const RowSums& sums, bool two) {
  const float soft = task.some ? a.soft * a.temperature * f : 0.f, hard = task.label >= 0 ? a.hard * f : 0.f;
  if (two) return RowScale{soft / sums.t, hard / sums.one};
  return RowScale{(soft + hard) / sums.t, 0.f};
}

// The elements of a word, two by two.
template <int TYPE>
__device__ __forceinline__ uint64_t pair_at(const uint4& v, int j) {
  if constexpr (TYPE == ADAPM_F32) {
    return j == 0 ? ((uint64_t)v.x | ((uint64_t)v.y << 32)) : ((uint64_t)v.z | ((uint64_t)v.w << 32));
  } else {
    const uint32_t w = j == 0 ? v.x : (j == 1 ? v.y : (j == 2 ? v.z : v.w));
    const float2 f = unpack2<TYPE>(w);
    return pair_of(f.x, f.y);
  }
}
// The largest of the elements seen, kept packed.
template <int TYPE>
struct Largest {
  using H = typename std::conditional<TYPE == ADAPM_BF16, __nv_bfloat162, __half2>::type;
  uint32_t m = Word<TYPE>::kNone;
  __device__ __forceinline__ void see(uint32_t w) {
    if constexpr (TYPE == ADAPM_F32) {
      m = __float_as_uint(fmaxf(__uint_as_float(m), __uint_as_float(w)));
    } else {
      const H x = __hmax2(*reinterpret_cast<const H*>(&m), *reinterpret_cast<const H*>(&w));
      m = *reinterpret_cast<const uint32_t*>(&x);
    }
  }
  __device__ __forceinline__ void see(const uint4& v) {
    see(v.x);
    see(v.y);
    see(v.z);
    see(v.w);
  }
  __device__ __forceinline__ float value() const {
    if constexpr (TYPE == ADAPM_F32) {
      return __uint_as_float(m);
    } else {
      const float2 f = unpack2<TYPE>(m);
      return fmaxf(f.x, f.y);
    }
  }
};
// Where max c is this large, for one of the temperatures, logits are taken
// relative to the largest before they are multiplied (which would lose too
// much, or overflow): in fp32, so that a difference serves both temperatures.
constexpr float kHuge = 1e5f;

// 2^(s c - k) with k = max c, rounded, is off by the rounding of k alone; times
// this it is 2^((s - max) c).
__device__ __forceinline__ float unround(float max, float c) {
  const float k = max * c;
  return exp2_of(-fmaf(max, c, -k));
}

__device__ __forceinline__ float finite_shift(float m) { return m == -INFINITY ? 0.f : m; }

// Which sums a row has: at one temperature; at two; at two of which the first is
// 2, where e^d = (e^(d/2))^2 (3063 rows of 50,021 bf16, both terms: 164 -> 122 us).
enum { ONE_SUM = 0, TWO_SUMS = 1, SQUARES = 2 };
template <int MODE>
__device__ __forceinline__ bool is_huge(float max, float per) {
  return fabsf(max * per) > kHuge || (MODE == TWO_SUMS && fabsf(max * kLog2E) > kHuge);
}

// Constants of 2^(s c - k) at both temperatures, as pairs; off: what is taken
// off first where the largest is huge (k: 0).
struct Exponents {
  uint64_t c, m, c1, m1, off;
  __device__ __forceinline__ Exponents(float per, float k, float largest)
      : c(pair_of(per, per)), m(pair_of(-(k * per), -(k * per))), c1(pair_of(kLog2E, kLog2E)), m1(pair_of(-(k * kLog2E), -(k * kLog2E))),
        off(pair_of(-largest, -largest)) {}
};
// Adds the exponentials of the elements of a word, two by two.
template <int TYPE, int MODE, bool HUGE>
__device__ __forceinline__ void add_word(const uint4& word, const Exponents& e, uint64_t& t, uint64_t& one) {
#pragma unroll
  for (int j = 0; j < Word<TYPE>::kElements / 2; ++j) {
    uint64_t s = pair_at<TYPE>(word, j);
    if (HUGE) s = add_pair(s, e.off);
    const float2 d = floats_of(fma_pair(s, e.c, e.m));
    const uint64_t x = pair_of(exp2_of(d.x), exp2_of(d.y));
    t = add_pair(t, x);
    if (MODE == TWO_SUMS) {
      const float2 d1 = floats_of(fma_pair(s, e.c1, e.m1));
      one = add_pair(one, pair_of(exp2_of(d1.x), exp2_of(d1.y)));
    } else if (MODE == SQUARES) {
      one = fma_pair(x, x, one);
    }
  }
}
// What the rounding of k costs the two sums: see unround.
template <int MODE>
__device__ __forceinline__ float2 unround_both(float k, float per) {
  const float u = unround(k, per);
  return make_float2(u, MODE == TWO_SUMS ? unround(k, kLog2E) : (MODE == SQUARES ? u * u : 0.f));
}

// What turns a row's logits into the part of the gradient that every element
// has: st 2^(s per - k) + so 2^(s log2(e) - k1).
struct RowFactors {
  float minus_k, st, minus_k1, so;
  float max;
  bool huge;
  bool folded;   // st is part of the exponent
};
template <int TYPE, int MODE>
__device__ __forceinline__ RowFactors row_factors(const DistillArgs& a, float weight, const RowTask& task, const RowSums& all, float per) {
  const RowScale scale = row_scale(a, weight, task, all, MODE != ONE_SUM);
  RowFactors f;
  f.max = all.max;
  f.huge = is_huge<MODE>(all.max, per);
  const float k = f.huge ? 0.f : all.max;
  const float2 u = unround_both<MODE>(k, per);
  f.st = scale.t * u.x;
  f.so = scale.one * u.y;
  // 16-bit gradients of one exponential: the factor is added to the exponent, where the sum is below 128 and its
  // logarithm at most 64: both round by 2^-18, so a gradient is off by 2^-17 of itself at most, a 64th of a half step
  // of fp16.  (Around 20,000 it would be 7e-4, more than that half step.)
  f.minus_k = -(k * per);
  f.folded = false;
  if (MODE == ONE_SUM && TYPE != ADAPM_F32 && !f.huge && f.st >= 0x1p-64f && f.st <= 0x1p64f) {
    const float sum = f.minus_k + log2f(f.st);
    f.folded = fabsf(sum) < 128.f;
    if (f.folded) f.minus_k = sum;
  }
  f.minus_k1 = -(k * kLog2E);
  return f;
}
template <int TYPE, int MODE, bool FOLD, bool HUGE>
struct Gradient {
  uint64_t c, m, ct, c1, m1, co, off;
  __device__ __forceinline__ Gradient(const RowFactors& f, float per)
      : c(pair_of(per, per)), m(pair_of(f.minus_k, f.minus_k)), ct(pair_of(f.st, f.st)), c1(pair_of(kLog2E, kLog2E)),
        m1(pair_of(f.minus_k1, f.minus_k1)), co(pair_of(f.so, f.so)), off(pair_of(-f.max, -f.max)) {}
  __device__ __forceinline__ uint4 of(const uint4& word) const {
    constexpr int E = Word<TYPE>::kElements;
    float x[E];
#pragma unroll
    for (int j = 0; j < E / 2; ++j) {
      uint64_t s = pair_at<TYPE>(word, j);
      if (HUGE) s = add_pair(s, off);
      const float2 d = floats_of(fma_pair(s, c, m));
      float2 f = make_float2(exp2_of(d.x), exp2_of(d.y));
      if (!FOLD) {
        const uint64_t x = pair_of(f.x, f.y);
        uint64_t y = mul_pair(x, ct);
        if (MODE == TWO_SUMS) {
          const float2 d1 = floats_of(fma_pair(s, c1, m1));
          y = fma_pair(pair_of(exp2_of(d1.x), exp2_of(d1.y)), co, y);
        } else if (MODE == SQUARES) {
          y = mul_pair(x, fma_pair(x, co, ct));
        }
        f = floats_of(y);
      }
      x[2 * j] = f.x;
      x[2 * j + 1] = f.y;
    }
    return pack_word<TYPE>(x);
  }
};
// fn(Gradient) in the form that the row's factors ask for.
template <int TYPE, int MODE, class F>
__device__ __forceinline__ void with_gradient(const RowFactors& f, float per, F&& fn) {
  if (f.huge) return fn(Gradient<TYPE, MODE, false, true>(f, per));
  if constexpr (MODE == ONE_SUM && TYPE != ADAPM_F32) {
    if (f.folded) return fn(Gradient<TYPE, MODE, true, false>(f, per));
  }
  fn(Gradient<TYPE, MODE, false, false>(f, per));
}

// How far a part's largest lies below that of all (-inf: a part without logits
// above it, whose sums are 0).  Parts of -inf alone stay as they are: their
// sums are 0, or NaN where they hold one, and a row of nothing else becomes NaN
// by the division by its sum.
__device__ __forceinline__ float below(float part, float all) { return all == -INFINITY ? 0.f : part - all; }

// Sums of several parts of a row, relative to the largest of all: `count` of
// them, of which the lane has number `lane` (at most 32).
template <int MODE>
__device__ __forceinline__ RowSums merge_sums(const RowSums& s, int count, float per) {
  const int lane = threadIdx.x & 31;
  RowSums all;
  all.max = lanes_max(lane < count ? s.max : -INFINITY);
  const float down = below(s.max, all.max);
  all.t = lanes_sum(lane < count ? s.t * exp2_of(down * per) : 0.f, 32);
  all.one = MODE != ONE_SUM ? lanes_sum(lane < count ? s.one * exp2_of(down * kLog2E) : 0.f, 32) : 0.f;
  return all;
}

// The same by every lane for itself, for few parts that part(i) reads from
// shared memory: no lane waits for another.
template <int MODE, class F>
__device__ __forceinline__ RowSums merge_few(int count, float per, F&& part) {
  RowSums all{-INFINITY, 0.f, 0.f};
#pragma unroll 8
  for (int i = 0; i < count; ++i) all.max = fmaxf(all.max, part(i).max);
#pragma unroll 8
  for (int i = 0; i < count; ++i) {
    const RowSums s = part(i);
    const float down = below(s.max, all.max);
    all.t = fmaf(s.t, exp2_of(down * per), all.t);
    if (MODE != ONE_SUM) all.one = fmaf(s.one, exp2_of(down * kLog2E), all.one);
  }
  return all;
}

// ---- rows in registers ------------------------------------------------------------
// Blocks per SM that the registers allow: 32 of a thread hold eight words.
constexpr int resident_blocks(int threads, int words) { return (words == 8 ? 1024 : 1536) / threads; }

// NV words a thread.
template <int TYPE, int THREADS, int NV, int MODE>
__global__ void __launch_bounds__(THREADS, resident_blocks(THREADS, NV))
distill_rows_kernel(const __grid_constant__ DistillArgs a) {
  after_previous();
  constexpr int E = Word<TYPE>::kElements, WARPS = THREADS / 32;
  __shared__ RowSums warps[2][WARPS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // exp((s - m) / T) = 2^((s - m) per); the one temperature of a row with one sum
  const float per = a.top > 0 ? kLog2E / a.temperature : kLog2E;
  const RowTask* const tasks = static_cast<const RowTask*>(a.tasks);
  uint64_t row = blockIdx.x;
  RowTask next = tasks[row];
  for (int turn = 0; row < a.n; row += gridDim.x, turn ^= 1) {
    const RowTask task = next;
    const bool live = task.some || task.label >= 0;
    const RowWords b = row_words<TYPE>(a.logits, row, a.vocab);
    uint4 v[NV];
    if (live) {
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i] = load_word<TYPE>(b, a.vocab, i * THREADS + threadIdx.x);
    }
    if (row + gridDim.x < a.n) next = tasks[row + gridDim.x];
    RowSums all{-INFINITY, 0.f, 0.f};
    if (live) {
      Largest<TYPE> largest;
#pragma unroll
      for (int i = 0; i < NV; ++i) largest.see(v[i]);
      RowSums mine;
      mine.max = lanes_max(largest.value());
      const float shift = finite_shift(mine.max);
      const bool huge = is_huge<MODE>(shift, per);
      const float k = huge ? 0.f : shift;
      const Exponents e(per, k, shift);
      uint64_t st = 0, so = 0;
      if (!huge) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (i * THREADS >= (int)b.words) break;
          add_word<TYPE, MODE, false>(v[i], e, st, so);
        }
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (i * THREADS >= (int)b.words) break;
          add_word<TYPE, MODE, true>(v[i], e, st, so);
        }
      }
      const float2 t = floats_of(st), o = floats_of(so), u = unround_both<MODE>(k, per);
      mine.t = lanes_sum((t.x + t.y) * u.x, 32);
      mine.one = MODE != ONE_SUM ? lanes_sum((o.x + o.y) * u.y, 32) : 0.f;
      if (lane == 0) warps[turn][warp] = mine;
    }
    __syncthreads();
    if (live) {
      all = merge_few<MODE>(WARPS, per, [&](int i) { return warps[turn][i]; });
      if (threadIdx.x == 0) static_cast<RowSums*>(a.sums)[row] = all;
    }
    if (a.grad.data == nullptr) continue;
    const RowWords g = row_words<TYPE>(a.grad, row, a.vocab);
    if (!live) {
      for (uint32_t w = threadIdx.x; w < g.words; w += THREADS) store_word<TYPE>(g, a.vocab, w, make_uint4(0, 0, 0, 0));
      continue;
    }
    const RowFactors f = row_factors<TYPE, MODE>(a, row_weight(a, row), task, all, per);
    with_gradient<TYPE, MODE>(f, per, [&](const auto& gradient) {
      if (g.head == b.head) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (i * THREADS >= (int)g.words) break;
          store_word<TYPE>(g, a.vocab, i * THREADS + threadIdx.x, gradient.of(v[i]));
        }
      } else {
        // words of the gradient that begin elsewhere: the row again, from L1 and L2
        const uint32_t shift = (b.head - g.head) & (E - 1), back = b.head < g.head ? 1 : 0;
        for (uint32_t w = threadIdx.x; w < g.words; w += THREADS) {
          store_word<TYPE>(g, a.vocab, w, gradient.of(load_shifted<TYPE>(b, a.vocab, w - back, shift)));
        }
      }
    });
  }
}

// ---- rows in slices -----------------------------------------------------------------
// A cluster of `split` blocks takes a row, each a slice of it: kSliceWarps warps
// work, one copies the next row's slice to shared memory as soon as they have
// taken this one's to their registers (NV words a thread), adds up their sums,
// exchanges the blocks', and prepares the row's factors.  With two or three
// blocks an SM, one's exchange and stores run beside another's sums.
constexpr int kSliceWarps = 7, kSliceWork = 32 * kSliceWarps, kSliceThreads = kSliceWork + 32;
// Words of a thread, and blocks per SM: of the 128 registers that eight warps of
// two blocks have 72 hold words, of the 80 of three blocks' 36.
constexpr int kManyWords = 18, kFewWords = 9;
constexpr int slice_blocks(int words) { return words == kManyWords ? 2 : 3; }
constexpr uint32_t kNap = 40;
// A block's part of a row: words [g0, g1) of the gradient, whose elements lie in
// words [e0, e1) of the logits, in which they begin `shift` elements further on.
struct Slice {
  char* to;            // the gradient's words
  uint32_t head;       // of the gradient's row
  uint32_t g0, g1, e0, held;
  uint32_t in0, in1;   // of [g0, g1): the words that hold nothing else
  uint32_t shift, back;
  bool live;
};
struct SliceShared {
  uint64_t full, taken;                // of the place that slices are copied to
  uint64_t summed, arrived[2], ready;  // of the live rows; arrivals by turns
  RowSums warps[kSliceWarps];
  float4 blocks[2][kMaxCluster];
  RowFactors factors;
  Slice slice;
  int gave_up;
};
// Who writes where while others may still read: the warps write their sums of a
// row after they have read the factors of the row before, which were made
// from the sums before; the copier writes a slice's description after all have
// taken the slice before, and its factors when all have summed, behind the
// stores of the row before.  A block sends sums of row r + 2 when all have sent
// those of row r + 1, behind their reading of row r's.
template <int TYPE, int NV, int MODE>
__global__ void __launch_bounds__(kSliceThreads) __maxnreg__(NV == kManyWords ? 128 : 80)
distill_slices_kernel(const __grid_constant__ DistillArgs a, int split) {
  extern __shared__ __align__(128) uint8_t place_bytes[];
  __shared__ SliceShared sh;
  constexpr int E = Word<TYPE>::kElements;
  uint4* const place = reinterpret_cast<uint4*>(place_bytes);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rank = split > 1 ? (int)(blockIdx.x % split) : 0;
  const uint64_t rows = gridDim.x / split, first = blockIdx.x / split;
  const uint32_t full = shared_at(&sh.full), taken = shared_at(&sh.taken), summed = shared_at(&sh.summed), ready = shared_at(&sh.ready);
  if (threadIdx.x == 0) {
    barrier_init(full, 1);
    barrier_init(taken, kSliceWarps);
    barrier_init(summed, kSliceWarps);
    barrier_init(ready, 1);
    for (int i = 0; i < 2; ++i) {
      barrier_init(shared_at(&sh.arrived[i]), 1);
      barrier_expect(shared_at(&sh.arrived[i]), split * 16);
    }
    sh.gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (split > 1) cg::this_cluster().sync();
  else __syncthreads();
  after_previous();
  const float per = a.top > 0 ? kLog2E / a.temperature : kLog2E;
  bool ok = true;
  if (warp == kSliceWarps) {
    const RowTask* const tasks = static_cast<const RowTask*>(a.tasks);
    uint32_t copies = 0, landed = 0;   // (those that somebody has waited for)
    // copies the slice of `row` and describes it
    auto copy = [&](uint64_t row, const RowTask& task) {
      const RowWords b = row_words<TYPE>(a.logits, row, a.vocab);
      const RowWords g = a.grad.data != nullptr ? row_words<TYPE>(a.grad, row, a.vocab) : b;
      Slice s;
      s.to = g.base;
      s.head = g.head;
      const uint32_t size = (g.words + split - 1) / split;
      s.g0 = min(g.words, rank * size);
      s.g1 = min(g.words, s.g0 + size);
      s.in0 = max(s.g0, g.full0);
      s.in1 = max(s.in0, min(s.g1, g.full1));
      s.shift = (b.head - g.head) & (E - 1);
      s.back = b.head < g.head ? 1 : 0;
      s.e0 = s.g0 - (s.g0 > 0 ? s.back : 0);
      const uint32_t e1 = min(b.words, s.g1 + (s.shift != 0 && s.back == 0 ? 1 : 0));
      s.held = e1 > s.e0 ? e1 - s.e0 : 0;
      s.live = task.some || task.label >= 0;
      uint32_t bytes = 0, in0 = 0;
      if (s.live && s.held > 0) {
        in0 = max(s.e0, b.full0);
        const uint32_t in1 = min(e1, b.full1);
        bytes = in1 > in0 ? (in1 - in0) * 16 : 0;
        // the row's first and last word, where they hold other elements too
        if (lane == 0 && s.e0 < b.full0) place[0] = load_word<TYPE>(b, a.vocab, s.e0);
        if (lane == 1 && e1 > b.full1) place[e1 - 1 - s.e0] = load_word<TYPE>(b, a.vocab, e1 - 1);
      }
      __syncwarp();
      if (lane == 0) {
        sh.slice = s;
        barrier_expect(full, bytes);
        if (bytes > 0) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (words written plainly for the row before)
          asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                           shared_at(place + (in0 - s.e0))),
                       "l"(b.base + (uint64_t)in0 * 16), "r"(bytes), "r"(full)
                       : "memory");
        }
      }
      ++copies;
      __syncwarp();
    };
    uint32_t it = 0, lives = 0;
    RowTask task = tasks[first < a.n ? first : 0];
    if (first < a.n) copy(first, task);
    for (uint64_t row = first; row < a.n; row += rows, ++it) {
      const bool more = row + rows < a.n;
      const RowTask next = tasks[more ? row + rows : row];
      if (!(ok = barrier_wait(taken, it & 1u, kNap))) break;
      ++landed;
      if (more) copy(row + rows, next);
      if (task.some || task.label >= 0) {
        const uint32_t parity = lives & 1u, q = lives & 1u;
        const float weight = row_weight(a, row);
        if (!(ok = barrier_wait(summed, parity))) break;
        RowSums all = merge_few<MODE>(kSliceWarps, per, [&](int i) { return sh.warps[i]; });
        if (split > 1) {
          const uint32_t bar = shared_at(&sh.arrived[q]);
          if (lane < split)
            store_and_count(shared_of(shared_at(&sh.blocks[q][rank]), lane), make_float4(all.max, all.t, all.one, 0.f), shared_of(bar, lane));
          if (!(ok = barrier_wait(bar, (lives >> 1) & 1u))) break;
          if (lane == 0) barrier_expect(bar, split * 16);   // (for two live rows on)
          all = merge_few<MODE>(split, per, [&](int i) {
            const float4 v = sh.blocks[q][i];
            return RowSums{v.x, v.y, v.z};
          });
        }
        ++lives;
        if (lane == 0) {
          sh.factors = row_factors<TYPE, MODE>(a, weight, task, all, per);
          barrier_arrive(ready);
          if (rank == 0) static_cast<RowSums*>(a.sums)[row] = all;
        }
        __syncwarp();
      }
      task = next;
    }
    if (!ok) {
      if (lane == 0) atomicExch(&sh.gave_up, 1);
      if (copies > landed) barrier_wait(full, landed & 1u);   // (it lands before the block ends)
    }
  } else {
    uint32_t it = 0, lives = 0;
    for (uint64_t row = first; row < a.n; row += rows, ++it) {
      if (!(ok = barrier_wait(full, it & 1u))) break;
      const Slice& s = sh.slice;
      const uint32_t g0 = s.g0, g1 = s.g1, count = g1 - g0, in0 = s.in0, in1 = s.in1, head = s.head;
      char* const to = s.to;
      const bool live = s.live;
      const uint4 none = make_uint4(Word<TYPE>::kNone, Word<TYPE>::kNone, Word<TYPE>::kNone, Word<TYPE>::kNone);
      uint4 v[NV];
      if (live) {
        const uint32_t shift = s.shift, held = s.held, from = g0 + threadIdx.x - s.back - s.e0;
        if (shift == 0) {
          const uint4* const p = place + threadIdx.x;   // (word g0 is the first that is held)
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            if (i * kSliceWork >= count) break;         // (the same for the block)
            if ((i + 1) * kSliceWork <= held) {
              v[i] = p[i * kSliceWork];
            } else {
              v[i] = none;
              if (threadIdx.x + i * kSliceWork < held) v[i] = p[i * kSliceWork];
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            if (i * kSliceWork >= count) break;
            const uint32_t w = from + i * kSliceWork;
            v[i] = none;
            if (threadIdx.x + i * kSliceWork < count)
              v[i] = shift_words<TYPE>(w < held ? place[w] : none, w + 1 < held ? place[w + 1] : none, shift);
          }
        }
      }
      __syncwarp();
      if (lane == 0) barrier_arrive(taken);
      if (!live) {
        if (a.grad.data != nullptr) {
          for (uint32_t w = g0 + threadIdx.x; w < g1; w += kSliceWork) {
            if (w >= in0 && w < in1) *reinterpret_cast<uint4*>(to + (uint64_t)w * 16) = make_uint4(0, 0, 0, 0);
            else store_edge<TYPE>(to, head, a.vocab, w, make_uint4(0, 0, 0, 0));
          }
        }
        continue;
      }
      Largest<TYPE> largest;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (i * kSliceWork >= count) break;
        largest.see(v[i]);
      }
      RowSums mine;
      mine.max = lanes_max(largest.value());
      const float shift = finite_shift(mine.max);
      const bool huge = is_huge<MODE>(shift, per);
      const float k = huge ? 0.f : shift;
      const Exponents e(per, k, shift);
      uint64_t st = 0, so = 0;
      if (!huge) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (i * kSliceWork >= count) break;
          add_word<TYPE, MODE, false>(v[i], e, st, so);
        }
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (i * kSliceWork >= count) break;
          add_word<TYPE, MODE, true>(v[i], e, st, so);
        }
      }
      const float2 t = floats_of(st), o = floats_of(so), u = unround_both<MODE>(k, per);
      mine.t = lanes_sum((t.x + t.y) * u.x, 32);
      mine.one = MODE != ONE_SUM ? lanes_sum((o.x + o.y) * u.y, 32) : 0.f;
      if (lane == 0) {
        sh.warps[warp] = mine;
        barrier_arrive(summed);
      }
      if (!(ok = barrier_wait(ready, lives & 1u))) break;
      ++lives;
      if (a.grad.data == nullptr) continue;
      const RowFactors f = sh.factors;
      with_gradient<TYPE, MODE>(f, per, [&](const auto& gradient) {
        const uint32_t w = g0 + threadIdx.x;
        char* const p = to + (uint64_t)w * 16;
        // (the row's first and last word may hold other elements too)
        const uint32_t inside = w - in0, size = in1 - in0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (i * kSliceWork >= count) break;
          const uint4 y = gradient.of(v[i]);
          if (inside + i * kSliceWork < size) *reinterpret_cast<uint4*>(p + i * kSliceWork * 16) = y;
          else if (w + i * kSliceWork < g1) store_edge<TYPE>(to, head, a.vocab, w + i * kSliceWork, y);
        }
      });
    }
    if (!ok && lane == 0) atomicExch(&sh.gave_up, 1);
  }
  __syncwarp();
  if (split > 1) cg::this_cluster().sync();   // (no block leaves while others send to it)
  else __syncthreads();
  if (threadIdx.x == 0 && sh.gave_up) set_error(a.st, ERR_TIMEOUT);
}

// ---- rows read twice ---------------------------------------------------------------
constexpr int kLongThreads = 512, kLongBlocks = 8;   // of a cluster
template <int TYPE, int MODE>
__global__ void __launch_bounds__(kLongThreads, 2) __cluster_dims__(kLongBlocks)
distill_long_kernel(const __grid_constant__ DistillArgs a) {
  after_previous();
  constexpr int E = Word<TYPE>::kElements, WARPS = kLongThreads / 32;
  __shared__ RowSums warps[WARPS];
  __shared__ RowSums blocks[2][kLongBlocks];
  cg::cluster_group cluster = cg::this_cluster();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = blockIdx.x % kLongBlocks;
  const float per = a.top > 0 ? kLog2E / a.temperature : kLog2E;
  int turn = 0;
  for (uint64_t row = blockIdx.x / kLongBlocks; row < a.n; row += gridDim.x / kLongBlocks) {
    const RowTask task = static_cast<const RowTask*>(a.tasks)[row];
    const bool live = task.some || task.label >= 0;
    const RowWords b = row_words<TYPE>(a.logits, row, a.vocab);
    const uint32_t size = (b.words + kLongBlocks - 1) / kLongBlocks;
    const uint32_t w0 = min(b.words, rank * size), w1 = min(b.words, w0 + size);
    RowSums all{-INFINITY, 0.f, 0.f};
    if (live) {
      RowSums mine{-INFINITY, 0.f, 0.f};   // relative to the largest so far
#pragma unroll 4
      for (uint32_t w = w0 + threadIdx.x; w < w1; w += kLongThreads) {
        const uint4 word = load_word<TYPE>(b, a.vocab, w);
        Largest<TYPE> here;
        here.see(word);
        const float max = fmaxf(mine.max, here.value());
        if (max > mine.max && mine.max != -INFINITY) {   // (sums of nothing are 0)
          mine.t *= exp2_of((mine.max - max) * per);
          mine.one *= exp2_of((mine.max - max) * kLog2E);
        }
        mine.max = max;
        const float shift = finite_shift(max);
        float x[E];
        unpack_word<TYPE>(word, x);
#pragma unroll
        for (int j = 0; j < E; ++j) {
          mine.t += exp2_of((x[j] - shift) * per);
          if (MODE != ONE_SUM) mine.one += exp2_of((x[j] - shift) * kLog2E);
        }
      }
      const float top = lanes_max(mine.max);
      if (mine.max != -INFINITY) {
        mine.t *= exp2_of((mine.max - top) * per);
        mine.one *= exp2_of((mine.max - top) * kLog2E);
      }
      mine.max = top;
      mine.t = lanes_sum(mine.t, 32);
      mine.one = lanes_sum(mine.one, 32);
      if (lane == 0) warps[warp] = mine;
      __syncthreads();
      if (warp == 0) {
        const RowSums ours = merge_sums<MODE>(lane < WARPS ? warps[lane] : RowSums{-INFINITY, 0.f, 0.f}, WARPS, per);
        if (lane < kLongBlocks) cluster.map_shared_rank(&blocks[turn][0], lane)[rank] = ours;
      }
      cluster.sync();
      all = merge_sums<MODE>(lane < kLongBlocks ? blocks[turn][lane] : RowSums{-INFINITY, 0.f, 0.f}, kLongBlocks, per);
      if (rank == 0 && threadIdx.x == 0) static_cast<RowSums*>(a.sums)[row] = all;
      turn ^= 1;
    }
    if (a.grad.data == nullptr) continue;
    const RowWords g = row_words<TYPE>(a.grad, row, a.vocab);
    const uint32_t g0 = min(g.words, rank * size), g1 = rank == kLongBlocks - 1 ? g.words : min(g.words, (rank + 1) * size);
    if (!live) {
      for (uint32_t w = g0 + threadIdx.x; w < g1; w += kLongThreads) store_word<TYPE>(g, a.vocab, w, make_uint4(0, 0, 0, 0));
      continue;
    }
    const RowFactors f = row_factors<TYPE, MODE>(a, row_weight(a, row), task, all, per);
    const uint32_t shift = (b.head - g.head) & (E - 1), back = b.head < g.head ? 1 : 0;
    with_gradient<TYPE, MODE>(f, per, [&](const auto& gradient) {
#pragma unroll 4
      for (uint32_t w = g0 + threadIdx.x; w < g1; w += kLongThreads) {
        store_word<TYPE>(g, a.vocab, w, gradient.of(load_shifted<TYPE>(b, a.vocab, w - back, shift)));
      }
    });
  }
  cluster.sync();   // (others may still write here)
}

// Warp-wide: a row's loss, and the elements that list and label change;
// entry(j): entry j of its list.
template <int TYPE, class F>
__device__ __forceinline__ void write_marks(const DistillArgs& a, uint64_t row, const RowTask& task, const RowSums& all, bool two, F&& entry) {
  const int lane = threadIdx.x & 31;
  if (!task.some && task.label < 0) {
    if (lane == 0) a.loss[row] = 0.f;
    return;
  }
  const float per = a.top > 0 ? kLog2E / a.temperature : kLog2E;
  const float inv_t = 1.f / a.temperature;
  const float f = row_weight(a, row);
  const RowScale scale = row_scale(a, f, task, all, two);
  const float log_st = logf(all.t), log_s1 = two ? logf(all.one) : log_st;
  const bool write = a.grad.data != nullptr;
  char* const grad = write ? a.grad.data + row_offset(a.grad, (uint32_t)row) * Word<TYPE>::kSize : nullptr;
  auto dense = [&](float s) {   // the part that every element has
    const float d = s - all.max;
    const float x = exp2_of(d * per) * scale.t;
    return two ? fmaf(exp2_of(d * kLog2E), scale.one, x) : x;
  };
  float cross = 0.f;   // sum of p ln q
  bool label_met = false;
  if (task.some) {
#pragma unroll 4
    for (uint32_t j = lane; j < a.top; j += 32) {
      const Entry e = entry(j);
      if (e.id == kNoKey) continue;
      if (e.p != 0.f) cross += e.p * ((e.s - all.max) * inv_t - log_st);
      const bool labelled = task.label == (int32_t)e.id;
      label_met = label_met || labelled;
      if (write) store_as(grad, TYPE, e.id, dense(e.s) - f * (a.soft * a.temperature * e.p + (labelled ? a.hard : 0.f)));
    }
    label_met = __any_sync(0xFFFFFFFFu, label_met);
    cross = lanes_sum(cross, 32);
  }
  if (lane != 0) return;
  float loss = task.some ? a.soft * a.temperature * a.temperature * (task.plogp - cross) : 0.f;
  if (task.label >= 0) {
    loss -= a.hard * ((task.label_s - all.max) - log_s1);
    if (write && !label_met) store_as(grad, TYPE, task.label, dense(task.label_s) - f * a.hard);
  }
  a.loss[row] = loss;
}
template <int TYPE>
__global__ void __launch_bounds__(kListWarps * 32)
distill_marks_kernel(const __grid_constant__ DistillArgs a, bool two) {
  after_previous();
  const int warp = threadIdx.x >> 5;
  for (uint64_t row = (uint64_t)blockIdx.x * kListWarps + warp; row < a.n; row += (uint64_t)gridDim.x * kListWarps)
    write_marks<TYPE>(a, row, static_cast<const RowTask*>(a.tasks)[row], static_cast<const RowSums*>(a.sums)[row], two,
                      [&](uint32_t j) { return static_cast<const Entry*>(a.entries)[row * a.top + j]; });
}

// ---- few rows ---------------------------------------------------------------------------
// All of it in one launch, a block per row that fits its registers: warp 0 reads
// the list while the row is on its way, and writes what it changes behind the
// others' gradient.
constexpr int kFewThreads = 1024;
template <int TYPE, int NV, int MODE>
__global__ void __launch_bounds__(kFewThreads)
distill_few_kernel(const __grid_constant__ DistillArgs a, uint32_t table) {
  after_previous();
  extern __shared__ uint32_t lists[];
  __shared__ RowSums warps[32];
  __shared__ RowTask shared_task;
  constexpr int E = Word<TYPE>::kElements;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t row = blockIdx.x;
  const float per = a.top > 0 ? kLog2E / a.temperature : kLog2E;
  const RowWords b = row_words<TYPE>(a.logits, row, a.vocab);
  uint4 v[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i] = load_word<TYPE>(b, a.vocab, i * kFewThreads + threadIdx.x);
  const Lists l(lists, a.top);
  if (warp == 0) {
    const RowTask task = read_lists<TYPE>(a, row, l, table);
    if (lane == 0) shared_task = task;
  }
  Largest<TYPE> largest;
#pragma unroll
  for (int i = 0; i < NV; ++i) largest.see(v[i]);
  RowSums mine;
  mine.max = lanes_max(largest.value());
  const float shift = finite_shift(mine.max);
  const bool huge = is_huge<MODE>(shift, per);
  const float k = huge ? 0.f : shift;
  const Exponents e(per, k, shift);
  uint64_t st = 0, so = 0;
  if (!huge) {
#pragma unroll
    for (int i = 0; i < NV; ++i) add_word<TYPE, MODE, false>(v[i], e, st, so);
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) add_word<TYPE, MODE, true>(v[i], e, st, so);
  }
  const float2 t = floats_of(st), o = floats_of(so), u = unround_both<MODE>(k, per);
  mine.t = lanes_sum((t.x + t.y) * u.x, 32);
  mine.one = MODE != ONE_SUM ? lanes_sum((o.x + o.y) * u.y, 32) : 0.f;
  if (lane == 0) warps[warp] = mine;
  __syncthreads();
  const RowTask task = shared_task;
  const bool live = task.some || task.label >= 0;
  const RowSums all = merge_sums<MODE>(warps[lane], 32, per);
  if (a.grad.data != nullptr) {
    const RowWords g = row_words<TYPE>(a.grad, row, a.vocab);
    if (!live) {
      for (uint32_t w = threadIdx.x; w < g.words; w += kFewThreads) store_word<TYPE>(g, a.vocab, w, make_uint4(0, 0, 0, 0));
    } else {
      const RowFactors f = row_factors<TYPE, MODE>(a, row_weight(a, row), task, all, per);
      with_gradient<TYPE, MODE>(f, per, [&](const auto& gradient) {
        if (g.head == b.head) {
#pragma unroll
          for (int i = 0; i < NV; ++i) store_word<TYPE>(g, a.vocab, i * kFewThreads + threadIdx.x, gradient.of(v[i]));
        } else {
          // words of the gradient that begin elsewhere: the row again, from L2
          const uint32_t shift_by = (b.head - g.head) & (E - 1), back = b.head < g.head ? 1 : 0;
          for (uint32_t w = threadIdx.x; w < g.words; w += kFewThreads) {
            store_word<TYPE>(g, a.vocab, w, gradient.of(load_shifted<TYPE>(b, a.vocab, w - back, shift_by)));
          }
        }
      });
    }
    __syncthreads();   // the marks are written over it
  }
  if (warp == 0) write_marks<TYPE>(a, row, task, all, MODE != ONE_SUM, [&](uint32_t j) { return Entry{l.id[j], l.t[j], l.s[j]}; });
}

// Smallest power of two that is at least n.
inline uint32_t power_of_two(uint64_t n) {
  uint32_t p = 1;
  while (p < n) p *= 2;
  return p;
}
inline int distill_mode(const DistillArgs& a) {
  return a.top == 0 || a.labels == nullptr || a.temperature == 1.f ? ONE_SUM : (a.temperature == 2.f ? SQUARES : TWO_SUMS);
}

template <int TYPE, int THREADS, int NV>
void launch_rows_as(const DistillArgs& a, int sms, cudaStream_t stream) {
  const unsigned grid = (unsigned)std::min<uint64_t>(a.n, (uint64_t)sms * resident_blocks(THREADS, NV));
  const int mode = distill_mode(a);
  if (mode == ONE_SUM) launch_after(distill_rows_kernel<TYPE, THREADS, NV, ONE_SUM>, grid, THREADS, 0, stream, a);
  else if (mode == SQUARES) launch_after(distill_rows_kernel<TYPE, THREADS, NV, SQUARES>, grid, THREADS, 0, stream, a);
  else launch_after(distill_rows_kernel<TYPE, THREADS, NV, TWO_SUMS>, grid, THREADS, 0, stream, a);
}

// As many clusters of a kernel as run at once: rows are dealt out beforehand,
// and one cluster more would double the time.  (Not all SMs of a GPC fill up
// with clusters.  Asked for once per kernel and size.)
inline int clusters_at_once(const void* kernel, const cudaLaunchConfig_t& c, int split, int otherwise) {
  struct Known {
    const void* kernel;
    size_t smem;
    int split, clusters;
  };
  static thread_local Known known[8]{};
  static thread_local unsigned next = 0;
  for (const Known& k : known)
    if (k.kernel == kernel && k.smem == c.dynamicSmemBytes && k.split == split) return k.clusters;
  int clusters = 0;
  if (split == 1 || cudaOccupancyMaxActiveClusters(&clusters, kernel, &c) != cudaSuccess || clusters < 1) {
    cudaGetLastError();
    clusters = std::max(1, otherwise / split);
  }
  known[next++ % 8] = Known{kernel, c.dynamicSmemBytes, split, clusters};
  return clusters;
}

template <int TYPE, int NV>
void launch_slices(const DistillArgs& a, int split, int sms, cudaStream_t stream) {
  const int mode = distill_mode(a);
  void (*kernel)(DistillArgs, int) = mode == ONE_SUM ? distill_slices_kernel<TYPE, NV, ONE_SUM>
                                     : (mode == SQUARES ? distill_slices_kernel<TYPE, NV, SQUARES> : distill_slices_kernel<TYPE, NV, TWO_SUMS>);
  cudaLaunchAttribute at[2]{};
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)split;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t c{};
  c.gridDim = dim3((unsigned)split);
  c.blockDim = dim3(kSliceThreads);
  c.dynamicSmemBytes = (NV * kSliceWork + 2) * 16;   // (a neighbour where the gradient's words begin elsewhere)
  c.stream = stream;
  c.attrs = at;
  c.numAttrs = split > 1 ? 2 : 1;
  static Asked asked[3];
  asked[mode].allow(kernel, c.dynamicSmemBytes, true);   // (an error shows in the launch)
  const int clusters = clusters_at_once((const void*)kernel, c, split, sms * slice_blocks(NV));
  c.gridDim = dim3((unsigned)(std::min<uint64_t>(a.n, clusters) * split));
  cudaLaunchKernelEx(&c, kernel, a, split);
}

template <int TYPE>
void launch_rows(const DistillArgs& a, int sms, cudaStream_t stream) {
  // (slices are cut by the gradient's words)
  const uint64_t words = std::max(words_of_row(a.vocab, a.logits, a.n), a.grad.data ? words_of_row(a.vocab, a.grad, a.n) : 0);
  if (words <= 256) return launch_rows_as<TYPE, 128, 2>(a, sms, stream);
  if (words <= 1024) return launch_rows_as<TYPE, 128, 8>(a, sms, stream);
  constexpr uint64_t most = kManyWords * kSliceWork, few = kFewWords * kSliceWork;   // words of a slice
  if (words <= kMaxCluster * most) {
    uint32_t split = (uint32_t)((words + most - 1) / most);
    // few rows: more blocks for each
    while (split <= 4 && a.n * split * 2 <= (uint64_t)sms && words / split > 1024) split *= 2;
    if (words <= split * few) return launch_slices<TYPE, kFewWords>(a, (int)split, sms, stream);
    return launch_slices<TYPE, kManyWords>(a, (int)split, sms, stream);
  }
  const unsigned grid = (unsigned)std::min<uint64_t>(a.n, std::max(1, sms * 2 / kLongBlocks)) * kLongBlocks;
  if (distill_mode(a) == ONE_SUM) launch_after(distill_long_kernel<TYPE, ONE_SUM>, grid, kLongThreads, 0, stream, a);
  else launch_after(distill_long_kernel<TYPE, TWO_SUMS>, grid, kLongThreads, 0, stream, a);
}

template <int TYPE, int NV>
void launch_few(const DistillArgs& a, uint32_t table, cudaStream_t stream) {
  const size_t smem = Lists::words(a.top, table) * sizeof(uint32_t);
  const int mode = distill_mode(a);
  note_launches(1);
  if (mode == ONE_SUM) launch_after(distill_few_kernel<TYPE, NV, ONE_SUM>, (unsigned)a.n, kFewThreads, smem, stream, a, table);
  else if (mode == SQUARES) launch_after(distill_few_kernel<TYPE, NV, SQUARES>, (unsigned)a.n, kFewThreads, smem, stream, a, table);
  else launch_after(distill_few_kernel<TYPE, NV, TWO_SUMS>, (unsigned)a.n, kFewThreads, smem, stream, a, table);
}

template <int TYPE>
void launch_distill_type(const DistillArgs& a, int sms, cudaStream_t stream) {
  const uint32_t table = a.top > 0 ? power_of_two(2 * a.top) : 0;
  if (distill_in_one(a.logits, a.n, a.vocab, sms)) {
    if (words_of_row(a.vocab, a.logits, a.n) <= 2 * kFewThreads) return launch_few<TYPE, 2>(a, table, stream);
    return launch_few<TYPE, 8>(a, table, stream);
  }
  const unsigned grid = (unsigned)std::min<uint64_t>((a.n + kListWarps - 1) / kListWarps, (uint64_t)sms * 16);
  const size_t smem = kListWarps * (size_t)Lists::words(a.top, table) * sizeof(uint32_t);
  static Asked asked;
  if (smem > 48 * 1024) asked.allow(distill_lists_kernel<TYPE>, kListWarps * 6 * (size_t)kMaxTop * sizeof(uint32_t));
  note_launches(3);
  launch_after(distill_lists_kernel<TYPE>, grid, kListWarps * 32, smem, stream, a, table);
  launch_rows<TYPE>(a, sms, stream);
  launch_after(distill_marks_kernel<TYPE>, grid, kListWarps * 32, 0, stream, a, distill_mode(a) != ONE_SUM);
}

}  // namespace

}  // namespace adapm
