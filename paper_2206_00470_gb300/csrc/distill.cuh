// Distillation from a teacher's top logits: the loss of every row of student
// logits and its gradient, in one pass over them.
//
// Row r has student logits s_v, a list of (id_j, t_j), and perhaps a label y:
//
//   p = softmax over the list of t_j / T,  q = softmax of s / T,  c = softmax of s
//   loss = soft T^2 sum_j p_j (ln p_j - ln q_id_j) + hard (-ln c_y)
//   grad_v = f (soft T (q_v - sum_{id_j = v} p_j) + hard (c_v - [v = y])),  f = scale weights[r]
//
// A row is read once and kept in registers, packed as it came: eight 16-byte
// words a thread, 512 threads a block, and where that is too little the blocks
// of a cluster take a slice of the row each and exchange their warps' maxima
// and sums through shared memory.  Every warp sums relative to its own maximum,
// so one exchange per row is enough.  The dense part of the gradient is
// written from the registers; warp 0, which has read the list and the logits
// at its ids meanwhile, then writes the few elements that the list and the
// label change.
// Bound by memory: a read and a write of the logits.
#pragma once

#include <cooperative_groups.h>

#include <algorithm>

#include "dense.cuh"

namespace adapm {

namespace {

namespace cg = cooperative_groups;

constexpr float kLog2E = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kMaxCluster = 16;
constexpr uint32_t kEmpty = 0x7FFFFFFFu;

__device__ __forceinline__ float exp2_of(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

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
// The elements of word w of another row of the same elements, whose words
// begin `shift` elements (less than a word's) further on in b's.
template <int TYPE>
__device__ __forceinline__ uint4 load_shifted(const RowWords& b, uint32_t vocab, uint32_t w, uint32_t shift) {
  const uint4 lo = load_word<TYPE>(b, vocab, w);
  if (shift == 0) return lo;
  const uint4 hi = load_word<TYPE>(b, vocab, w + 1);
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

// Maximum, and sums of exp((s - max) / T) and of exp(s - max), of some logits.
struct Sums {
  float max, t, one;
};
__device__ __forceinline__ float finite_shift(float m) { return m == -INFINITY ? 0.f : m; }

__device__ __forceinline__ int64_t id_at(const void* ids, bool wide, uint64_t i) {
  return wide ? static_cast<const int64_t*>(ids)[i] : (int64_t)static_cast<const int32_t*>(ids)[i];
}

// Blocks per SM that the registers allow: 32 of a thread hold eight words.
constexpr int resident_blocks(int threads, int words) { return (words == 8 ? 1024 : 1536) / threads; }

// What a row has to learn from.
struct RowTask {
  int64_t label;    // -1: none
  bool listed;      // the list has an id
};
__device__ __forceinline__ RowTask row_task(const DistillArgs& a, uint64_t row) {
  RowTask t{-1, false};
  if (a.labels != nullptr) {
    const int64_t y = id_at(a.labels, a.wide_labels, row);
    if (!(a.has_pad && y == a.pad)) {
      if (y >= 0 && y < (int64_t)a.vocab) t.label = y;
      else if (threadIdx.x == 0) set_error(a.st, ERR_KEY_RANGE);
    }
  }
  // (the first 32 entries say it nearly always)
  const int lane = threadIdx.x & 31;
  for (uint32_t j0 = 0; j0 < a.top && !t.listed; j0 += 32) {
    const int64_t id = j0 + lane < a.top ? id_at(a.ids, a.wide, row * a.top + j0 + lane) : -1;
    t.listed = __any_sync(0xFFFFFFFFu, id >= 0 && id < (int64_t)a.vocab);
  }
  return t;
}

// NV words a thread in registers (0: the row is read again for its gradient).
// TWO: sums at both temperatures.  Launched in clusters of `split` blocks per row.
template <int TYPE, int THREADS, int NV, bool TWO>
__global__ void __launch_bounds__(THREADS, resident_blocks(THREADS, NV))
distill_kernel(const __grid_constant__ DistillArgs a, int split, uint32_t table) {
  after_previous();
  constexpr int E = Word<TYPE>::kElements, WARPS = THREADS / 32, KEPT = NV > 0 ? NV : 1;
  __shared__ Sums sums[2][kMaxCluster * WARPS];
  __shared__ float teacher_part[2][4];   // whether there are entries, largest t, sum of exponentials
  extern __shared__ uint32_t lists[];    // warp 0: id, t, s, slot of every entry; the table
  uint32_t* const l_id = lists;
  float* const l_t = reinterpret_cast<float*>(lists + a.top);
  float* const l_s = l_t + a.top;
  uint32_t* const l_slot = lists + 3 * a.top;
  uint32_t* const l_table = lists + 4 * a.top;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rank = split > 1 ? (int)(blockIdx.x % split) : 0;
  const uint64_t rows = gridDim.x / split;
  const float per_t = kLog2E / a.temperature;             // exp((s - m) / T) = 2^((s - m) per_t)
  const float per = a.top > 0 ? per_t : kLog2E;           // the one temperature of a row without TWO
  uint64_t row = blockIdx.x / split;
  RowTask next = row < a.n ? row_task(a, row) : RowTask{-1, false};
  for (int turn = 0; row < a.n; row += rows, turn ^= 1) {
    const RowTask task = next;
    const bool live = task.listed || task.label >= 0;
    const RowWords b = row_words<TYPE>(a.logits, row, a.vocab);
    const uint32_t slice = (b.words + split - 1) / split;
    const uint32_t w0 = rank * slice, w1 = min(b.words, w0 + slice);
    uint4 v[KEPT];
    float label_s = 0.f;   // the label's logit (warp 0)
    Sums mine{-INFINITY, 0.f, 0.f};
    if (live) {
      if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const uint32_t w = w0 + i * THREADS + threadIdx.x;
          v[i] = make_uint4(Word<TYPE>::kNone, Word<TYPE>::kNone, Word<TYPE>::kNone, Word<TYPE>::kNone);
          if (w < w1) v[i] = load_word<TYPE>(b, a.vocab, w);
        }
      }
    }
    if (row + rows < a.n) next = row_task(a, row + rows);
    if (live) {
      if (warp == 0) {
        // the list: ids, teacher and student logits; its largest t and sum
        float tm = -INFINITY;
        bool bad = false;
        for (uint32_t j = lane; j < a.top; j += 32) {
          const uint64_t at = row * a.top + j;
          const int64_t id = id_at(a.ids, a.wide, at);
          float t = load_as(static_cast<const char*>(a.teacher), a.teacher_type, at);
          const bool here = id >= 0 && id < (int64_t)a.vocab && t != -INFINITY;
          bad = bad || (id >= (int64_t)a.vocab) || id < -1;
          l_id[j] = here ? (uint32_t)id : kNoKey;
          l_t[j] = here ? t : -INFINITY;
          l_s[j] = here ? load_as(b.base, TYPE, b.head + id) : 0.f;
          if (here) tm = fmaxf(tm, t);
        }
        if (task.label >= 0) label_s = load_as(b.base, TYPE, b.head + task.label);
        if (bad) set_error(a.st, ERR_KEY_RANGE);
        for (uint32_t j = lane; j < table; j += 32) l_table[j] = kEmpty;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) tm = fmaxf(tm, __shfl_xor_sync(0xFFFFFFFFu, tm, o));
        float ts = 0.f;
        bool some = false;
        for (uint32_t j = lane; j < a.top; j += 32) {
          if (l_id[j] == kNoKey) continue;
          some = true;
          ts += exp2_of((l_t[j] - tm) * per_t);
        }
        some = __any_sync(0xFFFFFFFFu, some);
        ts = lanes_sum(ts, 32);
        if (lane == 0) {
          teacher_part[turn][0] = some ? 1.f : 0.f;
          teacher_part[turn][1] = tm;
          teacher_part[turn][2] = ts;
        }
      }
      // the warp's largest logit, then its sums relative to it
      auto largest = [&](const uint4& word) {
        float x[E];
        unpack_word<TYPE>(word, x);
#pragma unroll
        for (int j = 0; j < E; ++j) mine.max = fmaxf(mine.max, x[j]);
      };
      auto add = [&](const uint4& word, float shift) {
        float x[E];
        unpack_word<TYPE>(word, x);
#pragma unroll
        for (int j = 0; j < E; ++j) {
          const float d = x[j] - shift;
          mine.t += exp2_of(d * per);
          if (TWO) mine.one += exp2_of(d * kLog2E);
        }
      };
      if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) largest(v[i]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mine.max = fmaxf(mine.max, __shfl_xor_sync(0xFFFFFFFFu, mine.max, o));
        const float shift = finite_shift(mine.max);
#pragma unroll
        for (int i = 0; i < NV; ++i) add(v[i], shift);
      } else {
        float max = -INFINITY;   // of the words so far, which the sums are relative to
        for (uint32_t w = w0 + threadIdx.x; w < w1; w += THREADS) {
          const uint4 word = load_word<TYPE>(b, a.vocab, w);
          mine.max = max;
          largest(word);
          const float shift = finite_shift(mine.max), down = finite_shift(max) - shift;
          if (down != 0.f) {
            mine.t *= exp2_of(down * per);
            mine.one *= exp2_of(down * kLog2E);
          }
          max = mine.max;
          add(word, shift);
        }
        float top = max;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        const float down = finite_shift(max) - finite_shift(top);
        mine.t *= exp2_of(down * per);
        mine.one *= exp2_of(down * kLog2E);
        mine.max = top;
      }
      mine.t = lanes_sum(mine.t, 32);
      if (TWO) mine.one = lanes_sum(mine.one, 32);
    }
    // one exchange: every warp's sums to every block of the cluster
    if (split > 1) {
      cg::cluster_group cluster = cg::this_cluster();
      if (lane < split) cluster.map_shared_rank(&sums[turn][0], lane)[rank * WARPS + warp] = mine;
      cluster.sync();
    } else {
      if (lane == 0) sums[turn][warp] = mine;
      __syncthreads();
    }
    Sums all{-INFINITY, 0.f, 0.f};
    if (live) {
      for (int i = lane; i < split * WARPS; i += 32) all.max = fmaxf(all.max, sums[turn][i].max);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) all.max = fmaxf(all.max, __shfl_xor_sync(0xFFFFFFFFu, all.max, o));
      for (int i = lane; i < split * WARPS; i += 32) {
        const Sums& s = sums[turn][i];
        const float down = s.max - all.max;   // (-inf: the warp has no logit above -inf, its sums are 0)
        all.t += s.t * exp2_of(down * per);
        if (TWO) all.one += s.one * exp2_of(down * kLog2E);
      }
      all.t = lanes_sum(all.t, 32);
      if (TWO) all.one = lanes_sum(all.one, 32);
    }
    const bool some = live && teacher_part[turn][0] != 0.f && a.top > 0;
    const float factor = a.weights != nullptr ? a.scale * a.weights[row] : a.scale;
    const float soft = some ? a.soft * a.temperature : 0.f, hard = task.label >= 0 ? a.hard : 0.f;
    const bool any = some || task.label >= 0;
    // coefficients of the two exponentials
    const float ct = TWO ? soft * factor / all.t : (soft + hard) * factor / all.t;
    const float co = TWO ? hard * factor / all.one : 0.f;
    RowWords g{};
    uint32_t w1g = 0;
    if (a.grad.data != nullptr) {
      g = row_words<TYPE>(a.grad, row, a.vocab);
      w1g = rank == split - 1 ? g.words : min(g.words, w0 + slice);
      auto gradient = [&](const uint4& word) {
        float x[E];
        unpack_word<TYPE>(word, x);
#pragma unroll
        for (int j = 0; j < E; ++j) {
          const float d = x[j] - all.max;
          x[j] = exp2_of(d * per) * ct;
          if (TWO) x[j] = fmaf(exp2_of(d * kLog2E), co, x[j]);
        }
        return pack_word<TYPE>(x);
      };
      if (!any) {
        for (uint32_t w = w0 + threadIdx.x; w < w1g; w += THREADS) store_word<TYPE>(g, a.vocab, w, make_uint4(0, 0, 0, 0));
      } else if (NV > 0 && g.head == b.head) {
#pragma unroll
        for (int i = 0; i < KEPT; ++i) {
          const uint32_t w = w0 + i * THREADS + threadIdx.x;
          if (w < w1) store_word<TYPE>(g, a.vocab, w, gradient(v[i]));
        }
      } else {
        // words of the gradient that begin elsewhere: the row again, from L2
        const uint32_t shift = (b.head - g.head) & (E - 1), back = b.head < g.head ? 1 : 0;
        for (uint32_t w = w0 + threadIdx.x; w < w1g; w += THREADS)
          store_word<TYPE>(g, a.vocab, w, gradient(load_shifted<TYPE>(b, a.vocab, w - back, shift)));
      }
      if (any) __syncthreads();   // the elements below are written over
    }
    if (warp != 0) continue;
    if (!any) {
      if (rank == 0 && lane == 0) a.loss[row] = 0.f;
      continue;
    }
    const float tm = teacher_part[turn][1], ts = teacher_part[turn][2];
    const float inv_t = 1.f / a.temperature;
    const float log_st = logf(all.t), log_s1 = TWO ? logf(all.one) : log_st, log_ts = logf(ts);
    // entries that share an id: the first of them speaks for all
    bool doubled = false;
    if (some && a.grad.data != nullptr) {
      __syncwarp();
      for (uint32_t j = lane; j < a.top; j += 32) {
        const uint32_t id = l_id[j];
        if (id == kNoKey) continue;
        uint32_t h = (id * 2654435761u) & (table - 1);
        while (true) {   // (the table has twice as many slots as there are entries)
          const uint32_t old = atomicCAS(&l_table[h], kEmpty, j);
          if (old == kEmpty) break;
          if (l_id[old] == id) {
            atomicMin(&l_table[h], j);
            doubled = true;
            break;
          }
          h = (h + 1) & (table - 1);
        }
        l_slot[j] = h;
      }
      doubled = __any_sync(0xFFFFFFFFu, doubled);
      __syncwarp();
    }
    float kl = 0.f;
    bool label_met = false;
    auto mine_to_write = [&](uint32_t id) {
      const uint32_t w = (g.head + id) / E;
      return a.grad.data != nullptr && w >= w0 && w < w1g;
    };
    auto dense = [&](float s) {   // the part of every element, as written above
      const float d = s - all.max;
      const float x = exp2_of(d * per) * ct;
      return TWO ? fmaf(exp2_of(d * kLog2E), co, x) : x;
    };
    if (some) {
      for (uint32_t j = lane; j < a.top; j += 32) {
        const uint32_t id = l_id[j];
        if (id == kNoKey) continue;
        const float log_p = (l_t[j] - tm) * inv_t - log_ts;
        float p = exp2_of((l_t[j] - tm) * per_t) / ts;
        if (rank == 0 && p != 0.f) kl += p * (log_p - ((l_s[j] - all.max) * inv_t - log_st));
        const bool labelled = task.label == (int64_t)id;
        label_met = label_met || labelled;
        if (!mine_to_write(id)) continue;
        if (doubled) {
          if (l_table[l_slot[j]] != j) continue;
          for (uint32_t i = j + 1; i < a.top; ++i)
            if (l_id[i] == id) p += exp2_of((l_t[i] - tm) * per_t) / ts;
        }
        store_as(g.base, TYPE, (int64_t)g.head + id, dense(l_s[j]) - factor * (soft * p + (labelled ? hard : 0.f)));
      }
      label_met = __any_sync(0xFFFFFFFFu, label_met);
    }
    if (rank == 0) kl = lanes_sum(kl, 32);
    if (lane != 0) continue;
    if (task.label >= 0 && !label_met && mine_to_write((uint32_t)task.label))
      store_as(g.base, TYPE, g.head + task.label, dense(label_s) - factor * hard);
    if (rank != 0) continue;
    float loss = some ? a.soft * a.temperature * a.temperature * kl : 0.f;
    if (task.label >= 0) loss -= a.hard * ((label_s - all.max) - log_s1);
    a.loss[row] = loss;
  }
}

// Smallest power of two that is at least n.
inline uint32_t power_of_two(uint64_t n) {
  uint32_t p = 1;
  while (p < n) p *= 2;
  return p;
}

template <int TYPE, int THREADS, int NV>
void launch_distill_as(const DistillArgs& a, int split, int sms, cudaStream_t stream) {
  const bool two = a.top > 0 && a.labels != nullptr && a.temperature != 1.f;
  const uint32_t table = a.top > 0 ? power_of_two(2 * a.top) : 0;
  void (*kernel)(DistillArgs, int, uint32_t) = two ? distill_kernel<TYPE, THREADS, NV, true> : distill_kernel<TYPE, THREADS, NV, false>;
  cudaLaunchAttribute at[2]{};
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)split;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  if (split > 8) cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  const uint64_t clusters = std::max<uint64_t>(1, (uint64_t)sms * resident_blocks(THREADS, NV) / split);
  cudaLaunchConfig_t c{};
  c.gridDim = dim3((unsigned)(std::min<uint64_t>(a.n, clusters) * split));
  c.blockDim = dim3(THREADS);
  c.dynamicSmemBytes = (4 * (size_t)a.top + table) * sizeof(uint32_t);
  c.stream = stream;
  c.attrs = at;
  c.numAttrs = split > 1 ? 2 : 1;
  note_launches(1);
  cudaLaunchKernelEx(&c, kernel, a, split, table);
}

template <int TYPE>
void launch_distill_type(const DistillArgs& a, int sms, cudaStream_t stream) {
  const uint64_t words = ((uint64_t)a.vocab * Word<TYPE>::kSize + 15) / 16 + 1;   // (a row may begin inside a word)
  if (words <= 256) return launch_distill_as<TYPE, 128, 2>(a, 1, sms, stream);
  if (words <= 1024) return launch_distill_as<TYPE, 128, 8>(a, 1, sms, stream);
  if (words <= 2048) return launch_distill_as<TYPE, 512, 4>(a, 1, sms, stream);
  uint32_t split = power_of_two((words + 4095) / 4096);
  if (split > kMaxCluster) return launch_distill_as<TYPE, 512, 0>(a, 8, sms, stream);
  // few rows: more blocks for each
  while (split < 8 && a.n * split * 2 <= (uint64_t)sms && words / split > 1024) split *= 2;
  launch_distill_as<TYPE, 512, 8>(a, (int)split, sms, stream);
}

}  // namespace

}  // namespace adapm
