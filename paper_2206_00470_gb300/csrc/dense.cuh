// The dense operators of a token model: what the entry points (capi.cu) hand
// to the kernels of norm.cu, distill.cu and linear.cu, and how those read and
// write elements of the three types.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "adapm.h"
#include "embed.cuh"

namespace adapm {

// `count` elements without gaps (device memory; null: none).
struct VectorView {
  char* data;
  int type;
};

// Asks once per device for what a kernel may use beyond the usual (asking takes
// the host 0.5 us): dynamic shared memory, and clusters of more than 8 blocks.
struct Asked {
  std::atomic<uint32_t> devices{0};
  template <class K>
  cudaError_t allow(K kernel, size_t smem, bool large_clusters = false) {
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    const uint32_t bit = 1u << (device & 31);
    if (e != cudaSuccess || (devices.load(std::memory_order_relaxed) & bit) != 0) return e;
    if (smem > 48 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e == cudaSuccess && large_clusters) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess && device < 32) devices.fetch_or(bit, std::memory_order_relaxed);
    return e;
  }
};

// ---- layer norm (norm.cu) -------------------------------------------------------
struct NormArgs {
  uint64_t n;          // rows
  uint32_t dim;
  RowView x, out;      // out: dx in the backward pass (null data: not wanted)
  RowView grad;        // backward only
  VectorView weight, bias;     // backward: bias unused
  VectorView dweight, dbias;   // backward only (null data: not wanted)
  float eps;
  float* stats;        // n pairs (mean, reciprocal deviation); forward: may be null
  float* parts;        // backward: norm_grad_scratch floats
};
size_t norm_grad_scratch(const NormArgs& a, int sms);
void launch_layer_norm(const NormArgs& a, int sms, cudaStream_t stream);
void launch_layer_norm_grad(const NormArgs& a, int sms, cudaStream_t stream);

// Columns of `count` rows of sums (`width` floats each) added up in a fixed
// order; the first `dim` go to low, the others to high.
void launch_column_join(const float* parts, uint32_t count, uint64_t width, uint32_t dim, const VectorView& low,
                        const VectorView& high, cudaStream_t stream);

// ---- distillation (distill.cuh) ---------------------------------------------------
constexpr uint32_t kMaxTop = 1024;   // entries of a teacher's list
struct DistillArgs {
  uint64_t n;            // rows
  uint32_t vocab;
  RowView logits, grad;  // grad: null data: not wanted
  const void* ids;       // n x top, without gaps
  const void* teacher;   // n x top, without gaps
  const void* labels;    // n, null: none
  bool wide;             // 64-bit ids
  bool wide_labels;
  bool has_pad;
  int64_t pad;           // of the labels
  uint32_t top;          // 0: no teacher
  int teacher_type;
  float temperature, soft, hard, scale;
  const float* weights;  // n factors of the gradient's rows, null: ones
  float* loss;           // n
  void *tasks, *sums, *entries;   // scratch: n, n and n * top of them
  DevState* st;
};
constexpr size_t kTaskBytes = 16, kRowSumBytes = 12, kEntryBytes = 12;
// Whether every row of the view begins on a multiple of `elements` elements.
inline bool rows_on(const RowView& v, uint64_t n, uint32_t elements);
// 16-byte words of a row, one more where rows may begin inside one; and whether
// all rows are done by one launch, which needs no scratch: at most one per SM,
// of up to 128 KB.
inline uint64_t words_of_row(uint32_t vocab, const RowView& v, uint64_t n) {
  const uint32_t size = v.type == ADAPM_F32 ? 4 : 2;
  return ((uint64_t)vocab * size + 15) / 16 + (rows_on(v, n, 16 / size) ? 0 : 1);
}
inline bool distill_in_one(const RowView& logits, uint64_t n, uint32_t vocab, int sms) {
  return n <= (uint64_t)sms && words_of_row(vocab, logits, n) <= 8192;
}
// The kernels of one type of logits (a translation unit each).
void launch_distill_f32(const DistillArgs& a, int sms, cudaStream_t stream);
void launch_distill_f16(const DistillArgs& a, int sms, cudaStream_t stream);
void launch_distill_bf16(const DistillArgs& a, int sms, cudaStream_t stream);
inline void launch_distill(const DistillArgs& a, int sms, cudaStream_t stream) {
  if (a.logits.type == ADAPM_F32) launch_distill_f32(a, sms, stream);
  else if (a.logits.type == ADAPM_F16) launch_distill_f16(a, sms, stream);
  else launch_distill_bf16(a, sms, stream);
}

// ---- matrix products (linear.cu) ----------------------------------------------------
// Element (i, j) is at i * row_stride + j * col_stride.
struct MatrixView {
  char* data;
  int type;
  int64_t row_stride, col_stride;
};
struct LinearArgs {
  uint64_t rows;
  uint32_t ins, outs;
  MatrixView x, weight;      // rows x ins, ins x outs, of one 16-bit type
  VectorView bias;           // null data: none
  MatrixView residual, out, pre;   // rows x outs, col_stride 1; null data: none
  int activation;            // ADAPM_ACTIVATION_*
  // backward: the gradient of out, and what is wanted of x, weight, bias
  MatrixView grad, dx, dweight;
  VectorView dbias;
  DevState* st;
};
// Bytes of scratch; the launches take a pointer to that many (aligned to 256),
// and return a CUDA error of their host side.
size_t linear_scratch(const LinearArgs& a, int sms);
cudaError_t launch_linear(const LinearArgs& a, char* scratch, int sms, cudaStream_t stream);
size_t linear_grad_scratch(const LinearArgs& a, int sms);
cudaError_t launch_linear_grad(const LinearArgs& a, char* scratch, int sms, cudaStream_t stream);

#ifdef __CUDACC__
namespace {

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// fn(type) for a type known when compiled, or (TYPE -1) for the one known at run
// time: the branch stands outside of fn's loops, so that their loads go out together.
template <int T>
struct Type {
  static constexpr int value = T;
};
template <int TYPE, class F>
__device__ __forceinline__ void by_type(int type, F&& fn) {
  if constexpr (TYPE >= 0) fn(Type<TYPE>());
  else if (type == ADAPM_F32) fn(Type<ADAPM_F32>());
  else if (type == ADAPM_BF16) fn(Type<ADAPM_BF16>());
  else fn(Type<ADAPM_F16>());
}

// One element of a type known at run time.
__device__ __forceinline__ float load_as(const char* p, int type, int64_t i) {
  if (type == ADAPM_F32) return reinterpret_cast<const float*>(p)[i];
  if (type == ADAPM_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[i]);
  return __half2float(reinterpret_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_as(char* p, int type, int64_t i, float v) {
  if (type == ADAPM_F32) reinterpret_cast<float*>(p)[i] = v;
  else if (type == ADAPM_BF16) reinterpret_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else reinterpret_cast<__half*>(p)[i] = __float2half_rn(v);
}

// Two elements of a 16-bit type from a word, and back.
template <int TYPE>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if (TYPE == ADAPM_BF16) return make_float2(bf16_low(w), bf16_high(w));
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <int TYPE>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  if (TYPE == ADAPM_BF16) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&b);
  }
  const __half2 h = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// N elements of a type known when compiled from an address aligned to all of
// them (N * size is 4, 8 or 16 bytes), and back.
template <int TYPE, int N>
__device__ __forceinline__ void load_n(const char* p, float* x) {
  if constexpr (TYPE == ADAPM_F32) {
    if constexpr (N == 4) {
      const float4 v = *reinterpret_cast<const float4*>(p);
      x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else if constexpr (N == 8) {
      load_n<TYPE, 4>(p, x);
      load_n<TYPE, 4>(p + 16, x + 4);
    } else {
      static_assert(N == 1);
      x[0] = *reinterpret_cast<const float*>(p);
    }
  } else if constexpr (N == 1) {
    x[0] = load_as(p, TYPE, 0);
  } else {
    uint32_t w[N / 2];
    if constexpr (N == 8) {
      const uint4 v = *reinterpret_cast<const uint4*>(p);
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else {
      static_assert(N == 4);
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      w[0] = v.x; w[1] = v.y;
    }
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
      const float2 f = unpack2<TYPE>(w[j]);
      x[2 * j] = f.x;
      x[2 * j + 1] = f.y;
    }
  }
}
template <int TYPE, int N>
__device__ __forceinline__ void store_n(char* p, const float* x) {
  if constexpr (TYPE == ADAPM_F32) {
    if constexpr (N == 4) {
      *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    } else if constexpr (N == 8) {
      store_n<TYPE, 4>(p, x);
      store_n<TYPE, 4>(p + 16, x + 4);
    } else {
      static_assert(N == 1);
      *reinterpret_cast<float*>(p) = x[0];
    }
  } else if constexpr (N == 1) {
    store_as(p, TYPE, 0, x[0]);
  } else if constexpr (N == 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2<TYPE>(x[0], x[1]), pack2<TYPE>(x[2], x[3]),
                                              pack2<TYPE>(x[4], x[5]), pack2<TYPE>(x[6], x[7]));
  } else {
    static_assert(N == 4);
    *reinterpret_cast<uint2*>(p) = make_uint2(pack2<TYPE>(x[0], x[1]), pack2<TYPE>(x[2], x[3]));
  }
}

__host__ __device__ __forceinline__ int type_size(int type) { return type == ADAPM_F32 ? 4 : 2; }

// ---- two floats at a time ------------------------------------------------------
__device__ __forceinline__ uint64_t pair_of(float x, float y) {
  return (uint64_t)__float_as_uint(x) | ((uint64_t)__float_as_uint(y) << 32);
}
__device__ __forceinline__ float2 floats_of(uint64_t v) { return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))); }
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// 2^x and 1 / x, off by a few units in the last place; 2^x is 0 below the normal numbers.
__device__ __forceinline__ float exp2_of(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float over(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Sum over `width` lanes (a power of two) that begin at a multiple of it; every lane gets it.
__device__ __forceinline__ float lanes_sum(float x, int width) {
  for (int o = width >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  return x;
}

}  // namespace

// Whether every row of the view begins on a multiple of `elements` elements.
inline bool rows_on(const RowView& v, uint64_t n, uint32_t elements) {
  const uint64_t bytes = (uint64_t)elements * type_size(v.type);
  if (reinterpret_cast<uintptr_t>(v.data) % bytes != 0) return false;
  const bool one = n <= 1;
  if (!one && v.inner_stride % (int64_t)elements != 0) return false;
  return v.flat || v.outer_stride % (int64_t)elements == 0;
}
#endif

}  // namespace adapm
