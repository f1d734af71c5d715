// The Euclidean norm over many gradient tensors, and clipping by it.
//
//   norm = |scale| * sqrt(sum of x^2 over all elements of all tensors)
//   out  = round(scale * min(1, max_norm / norm) * x)
//
// Both run over units: a unit is an aligned window of kUnit bytes of one
// tensor, taken by a warp with eight 128-bit loads in flight.  So tensors of any
// number, size and alignment are one grid's work and one launch (per
// kTableLarge tensors: the list travels in the kernel's parameters, no copy in
// front of it); only a tensor's first and last unit look at element bounds.
// Bound by memory: 500M bf16 elements, norm 142 us (7.0 TB/s), clipping 300 us
// (6.7 TB/s); 24 tensors of 100,003 floats in all by two launches, 9.7 us.
// (At five and six blocks per SM the registers do not hold a unit: 473 and 567
// us for both, 460 at four.)
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "adapm.h"
#include "embed.cuh"
#include "rowgroup.cuh"

namespace adapm {

namespace {

constexpr uint32_t kUnit = 4096;   // bytes
constexpr int kLoads = kUnit / (32 * 16);
constexpr int kTableSmall = 32, kTableLarge = 400;   // tensors per launch
constexpr int kNormBlocks = 4;     // blocks per SM

template <int N>
struct Table {
  GradTensor t[N];
  uint32_t unit[N + 1];   // first unit of each tensor; all units
  int n;
};

__device__ __forceinline__ int size_of(int type) { return type == ADAPM_F32 ? 4 : 2; }

// The tensor of unit u, one of lo .. hi.
template <int N>
__device__ __forceinline__ int tensor_of(const Table<N>& tab, uint32_t u, int lo, int hi) {
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab.unit[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ uint64_t live_count(const GradTensor& t) {
  if (t.live == nullptr) return t.count;
  const uint64_t c = (uint64_t)*t.live * t.row_len;
  return c < t.count ? c : t.count;
}

// Element j of eight (or the low four) from a 128-bit word.
template <int TYPE>
__device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (TYPE == ADAPM_F32) {
      x[j] = __uint_as_float(w[j]);
    } else if (TYPE == ADAPM_BF16) {
      x[2 * j] = __uint_as_float(w[j] << 16);
      x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
      x[2 * j] = f.x;
      x[2 * j + 1] = f.y;
    }
  }
}
template <int TYPE>
__device__ __forceinline__ float load_one(const char* p) {
  if (TYPE == ADAPM_F32) return *reinterpret_cast<const float*>(p);
  if (TYPE == ADAPM_BF16) return __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(p));
  return __half2float(*reinterpret_cast<const __half*>(p));
}
__device__ __forceinline__ void store_one(char* p, int type, float v) {
  if (type == ADAPM_F32) *reinterpret_cast<float*>(p) = v;
  else if (type == ADAPM_BF16) *reinterpret_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(v);
  else *reinterpret_cast<__half*>(p) = __float2half_rn(v);
}

// The unit's words that hold elements of the tensor: words outside it, and
// elements of the first and last word that belong to a neighbour, read as 0.
template <int TYPE>
__device__ __forceinline__ void load_unit(const char* p0, const char* p1, const char* at, uint4 (&v)[kLoads]) {
  const int lane = threadIdx.x & 31;
  if (at >= p0 && at + kUnit <= p1) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) v[i] = *reinterpret_cast<const uint4*>(at + (i * 32 + lane) * 16);
    return;
  }
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const char* w = at + (i * 32 + lane) * 16;
    v[i] = make_uint4(0u, 0u, 0u, 0u);
    if (w >= p0 && w + 16 <= p1) {
      v[i] = *reinterpret_cast<const uint4*>(w);
    } else if (w + 16 > p0 && w < p1) {
      constexpr int S = TYPE == ADAPM_F32 ? 4 : 2;
      uint32_t x[4] = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int j = 0; j < 16 / S; ++j) {
        const char* e = w + j * S;
        if (e >= p0 && e < p1) {
          if (S == 4) x[j] = *reinterpret_cast<const uint32_t*>(e);
          else x[j / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(e) << (16 * (j & 1));
        }
      }
      v[i] = make_uint4(x[0], x[1], x[2], x[3]);
    }
  }
}

// Sum of the unit's squares of one lane: fp32 over its 32 or 64 elements,
// which errs by a few parts in 10^7 at most, unless squares overflow or
// vanish there: then again in fp64, from memory (the words need not be kept
// for that, which would cost the usual case registers).
template <int TYPE>
__device__ __forceinline__ double norm_unit(const GradTensor& t, uint32_t k) {
  constexpr int E = TYPE == ADAPM_F32 ? 4 : 8;
  const char* p0 = t.in;
  const char* p1 = p0 + live_count(t) * (TYPE == ADAPM_F32 ? 4 : 2);
  const char* at = p0 - (reinterpret_cast<uintptr_t>(p0) & 15) + (uint64_t)k * kUnit;
  if (at >= p1) return 0.0;
  uint4 v[kLoads];
  load_unit<TYPE>(p0, p1, at, v);
  float sum[2] = {0.f, 0.f};
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    any |= v[i].x | v[i].y | v[i].z | v[i].w;
    float x[8];
    unpack<TYPE>(v[i], x);
#pragma unroll
    for (int j = 0; j < E; ++j) sum[i & 1] = fmaf(x[j], x[j], sum[i & 1]);
  }
  const float both = sum[0] + sum[1];
  if (both > 1e-25f && both < 1e37f) return (double)both;
  if ((any & (TYPE == ADAPM_F32 ? 0x7FFFFFFFu : 0x7FFF7FFFu)) == 0u) return 0.0;   // zeros, as untouched rows have
  double s = 0.0;
#pragma unroll 1
  for (int i = 0; i < kLoads; ++i) {
    const char* w = at + (i * 32 + (threadIdx.x & 31)) * 16;
    constexpr int S = 16 / E;
#pragma unroll 1
    for (int j = 0; j < E; ++j) {
      const char* e = w + j * S;
      const double x = e >= p0 && e < p1 ? (double)load_one<TYPE>(e) : 0.0;
      s += x * x;
    }
  }
  return s;
}

// part: one sum per block of every launch of the call; the last block of the
// last launch (`total` set) adds them in order and writes the norm.
template <int N>
__global__ void __launch_bounds__(kThreads, kNormBlocks)
grad_norm_kernel(const __grid_constant__ Table<N> tab, double* part, uint32_t part0, uint32_t total, float scale, float* norm,
                 DevState* st) {
  after_previous();
  __shared__ double sums[kThreads / 32];
  __shared__ bool last;
  const uint32_t units = tab.unit[tab.n];
  const uint32_t warps = gridDim.x * (kThreads / 32);
  double sum = 0.0;
  int i = 0;
  for (uint32_t u = blockIdx.x * (kThreads / 32) + threadIdx.x / 32; u < units; u += warps) {
    i = tensor_of(tab, u, i, tab.n - 1);
    const GradTensor& t = tab.t[i];
    const uint32_t k = u - tab.unit[i];
    sum += t.type == ADAPM_F32 ? norm_unit<ADAPM_F32>(t, k)
                               : (t.type == ADAPM_BF16 ? norm_unit<ADAPM_BF16>(t, k) : norm_unit<ADAPM_F16>(t, k));
  }
  auto block_sum = [&](double x) {   // to thread 0, in a fixed order
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x / 32] = x;
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x == 0)
      for (int w = 0; w < kThreads / 32; ++w) s += sums[w];
    return s;
  };
  sum = block_sum(sum);
  if (threadIdx.x == 0) {
    part[part0 + blockIdx.x] = sum;
    __threadfence();
    last = total != 0u && atomicAdd(&st->norm_done, 1u) == gridDim.x - 1;
    __threadfence();
  }
  __syncthreads();
  if (!last) return;
  double all = 0.0;
  for (uint32_t b = threadIdx.x; b < total; b += kThreads) all += __ldcg(part + b);
  all = block_sum(all);
  if (threadIdx.x == 0) {
    *norm = (float)(fabs((double)scale) * sqrt(all));
    st->norm_done = 0u;
  }
}

template <int TYPE>
__device__ __forceinline__ void clip_unit(const GradTensor& t, uint32_t k, float f) {
  constexpr int S = TYPE == ADAPM_F32 ? 4 : 2, E = 16 / S;
  const int lane = threadIdx.x & 31;
  const char* p0 = t.in;
  const char* p1 = p0 + live_count(t) * S;
  const char* at = p0 - (reinterpret_cast<uintptr_t>(p0) & 15) + (uint64_t)k * kUnit;
  if (at >= p1) return;
  const int os = size_of(t.out_type);
  uint4 v[kLoads];
  load_unit<TYPE>(p0, p1, at, v);
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const char* w = at + (i * 32 + lane) * 16;
    if (w + 16 <= p0 || w >= p1) continue;
    float x[8];
    unpack<TYPE>(v[i], x);
#pragma unroll
    for (int j = 0; j < E; ++j) x[j] *= f;
    const int64_t e0 = (w - p0) / S;   // (exact; negative in the first word of an unaligned tensor)
    char* o = t.out + e0 * os;
    if (w >= p0 && w + 16 <= p1 && t.out_type == TYPE && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
      uint32_t r[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (TYPE == ADAPM_F32) {
          r[j] = __float_as_uint(x[j]);
        } else if (TYPE == ADAPM_BF16) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
          r[j] = *reinterpret_cast<const uint32_t*>(&b);
        } else {
          const __half2 b = __floats2half2_rn(x[2 * j], x[2 * j + 1]);
          r[j] = *reinterpret_cast<const uint32_t*>(&b);
        }
      }
      *reinterpret_cast<uint4*>(o) = make_uint4(r[0], r[1], r[2], r[3]);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const char* e = w + j * S;
        if (e >= p0 && e < p1) store_one(o + j * os, t.out_type, x[j]);
      }
    }
  }
}

template <int N>
__global__ void __launch_bounds__(kThreads, kNormBlocks)
clip_grads_kernel(const __grid_constant__ Table<N> tab, float scale, float max_norm, const float* norm, bool in_place) {
  after_previous();
  const float f = clip_factor(scale, *norm, max_norm);
  if (in_place && f == 1.f) return;
  const uint32_t units = tab.unit[tab.n];
  const uint32_t warps = gridDim.x * (kThreads / 32);
  int i = tab.n - 1;
  // last units first: the norm's pass left them in L2 (clip_mixed 62.9 -> 59.4 us)
  for (uint32_t v = blockIdx.x * (kThreads / 32) + threadIdx.x / 32; v < units; v += warps) {
    const uint32_t u = units - 1 - v;
    i = tensor_of(tab, u, 0, i);
    const GradTensor& t = tab.t[i];
    const uint32_t k = u - tab.unit[i];
    if (t.type == ADAPM_F32) clip_unit<ADAPM_F32>(t, k, f);
    else if (t.type == ADAPM_BF16) clip_unit<ADAPM_BF16>(t, k, f);
    else clip_unit<ADAPM_F16>(t, k, f);
  }
}

// A launch per table of at most N tensors, and of fewer than 2^31 units; the
// blocks of launch j begin at part0[j].  fn(table, blocks, first, last).
uint64_t units_of(const GradTensor& t) {
  const uint64_t bytes = t.count * (t.type == ADAPM_F32 ? 4 : 2);
  return t.count == 0 ? 0 : ((reinterpret_cast<uintptr_t>(t.in) & 15) + bytes + kUnit - 1) / kUnit;
}

template <int N, class F>
void for_tables(const GradTensor* t, uint64_t n, int sms, F&& fn) {
  static thread_local Table<N> tab;
  uint64_t i = 0;
  do {
    tab.n = 0;
    uint64_t units = 0;
    for (; i < n && tab.n < N; ++i) {
      const uint64_t u = units_of(t[i]);
      if (u == 0) continue;
      if (tab.n > 0 && units + u >= (1ull << 31)) break;
      tab.t[tab.n] = t[i];
      tab.unit[tab.n++] = (uint32_t)units;
      units += u;
    }
    tab.unit[tab.n] = (uint32_t)units;
    const uint64_t most = (uint64_t)sms * kNormBlocks;
    const uint64_t blocks = std::max<uint64_t>(1, std::min(most, (units + kThreads / 32 - 1) / (kThreads / 32)));
    fn(tab, (unsigned)blocks, i >= n);
  } while (i < n);
}

template <int N>
void norm_tables(const GradTensor* t, uint64_t n, float scale, double* part, float* norm, DevState* st, int sms,
                 cudaStream_t stream) {
  uint32_t part0 = 0;
  for_tables<N>(t, n, sms, [&](const Table<N>& tab, unsigned blocks, bool last) {
    note_launches(1);
    launch_after(grad_norm_kernel<N>, blocks, kThreads, 0, stream, tab, part, part0, last ? part0 + blocks : 0u, scale,
                 norm, st);
    part0 += blocks;
  });
}

template <int N>
void clip_tables(const GradTensor* t, uint64_t n, float scale, float max_norm, const float* norm, bool in_place,
                 int sms, cudaStream_t stream) {
  for_tables<N>(t, n, sms, [&](const Table<N>& tab, unsigned blocks, bool) {
    note_launches(1);
    launch_after(clip_grads_kernel<N>, blocks, kThreads, 0, stream, tab, scale, max_norm, norm, in_place);
  });
}

}  // namespace

size_t norm_scratch_doubles(uint64_t n, int sms) {
  // (a table closes early only where its units reach 2^31: tensors of 8 TB)
  return (size_t)(n / kTableLarge + 2) * sms * kNormBlocks;
}

void launch_grad_norm(const GradTensor* t, uint64_t n, float scale, double* part, float* norm, DevState* st, int sms,
                      cudaStream_t stream) {
  if (n <= kTableSmall) norm_tables<kTableSmall>(t, n, scale, part, norm, st, sms, stream);
  else norm_tables<kTableLarge>(t, n, scale, part, norm, st, sms, stream);
}

void launch_clip_grads(const GradTensor* t, uint64_t n, float scale, float max_norm, const float* norm, bool in_place,
                       int sms, cudaStream_t stream) {
  if (n <= kTableSmall) clip_tables<kTableSmall>(t, n, scale, max_norm, norm, in_place, sms, stream);
  else clip_tables<kTableLarge>(t, n, scale, max_norm, norm, in_place, sms, stream);
}

}  // namespace adapm
