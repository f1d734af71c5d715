// embed: the rows of a batch of tokens, scaled, in the type of the model.
//
//   out[t][c] = round(scale * value(worker, token t)[c]),  c < dim
//
// One pass: the gather of pull (store.cu) with the multiplication and the
// rounding to 16 bits on the way, so that the fp32 rows never travel.  Bound by
// memory: 4 dim bytes in per distinct token (repeats come from L2), dim
// elements out per token.  64 x 4096 tokens of 62,000 distinct ones, rows of
// 1024, bf16 out: 139 us, 5.7 TB/s of those bytes; 64 x 2048 tokens of 250,000
// at random, fp32 out, 157 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "adapm.h"
#include "embed.cuh"
#include "rowgroup.cuh"

namespace adapm {

namespace {

__device__ __forceinline__ uint2 pack4(float4 v, __half) {
  const __half2 a = __floats2half2_rn(v.x, v.y), b = __floats2half2_rn(v.z, v.w);
  return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ uint2 pack4(float4 v, __nv_bfloat16) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ float4 pack4(float4 v, float) { return v; }
template <class T>
__device__ __forceinline__ T round_to(float v) {
  return (T)v;
}
template <>
__device__ __forceinline__ __half round_to<__half>(float v) {
  return __float2half_rn(v);
}
template <>
__device__ __forceinline__ __nv_bfloat16 round_to<__nv_bfloat16>(float v) {
  return __float2bfloat16_rn(v);
}

__device__ __forceinline__ uint32_t pack2(float x, float y, __half) {
  const __half2 a = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&a);
}
__device__ __forceinline__ uint32_t pack2(float x, float y, __nv_bfloat16) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&a);
}
__device__ __forceinline__ float2 pack2(float x, float y, float) { return make_float2(x, y); }

// Up to four elements of a row from column c; rows begin on a multiple of
// `align` (4, 2 or 1) elements.
template <class T>
__device__ __forceinline__ void put4(T* row, uint32_t c, uint32_t dim, float4 v, int align) {
  if (align == 4 && c + 4 <= dim) {
    auto p = pack4(v, T());
    __stcs(reinterpret_cast<decltype(p)*>(row + c), p);
    return;
  }
  if (align == 2 && c + 4 <= dim) {
    auto p = pack2(v.x, v.y, T()), q = pack2(v.z, v.w, T());
    *reinterpret_cast<decltype(p)*>(row + c) = p;
    *reinterpret_cast<decltype(p)*>(row + c + 2) = q;
    return;
  }
  const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (c + j < dim) row[c + j] = round_to<T>(x[j]);
}

__device__ __forceinline__ float4 f4scale(float4 v, float s) {
  return make_float4(v.x * s, v.y * s, v.z * s, v.w * s);
}

// 256 bits at once, from a 32-byte boundary.
__device__ __forceinline__ void load8(const float4* p, float4& a, float4& b) {
  asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(a.x), "=f"(a.y), "=f"(a.z), "=f"(a.w), "=f"(b.x), "=f"(b.y), "=f"(b.z), "=f"(b.w)
               : "l"(p));
}

__device__ __forceinline__ void store8(float* p, float4 a, float4 b) {
  asm volatile("st.global.cs.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(a.x), "f"(a.y), "f"(a.z),
               "f"(a.w), "f"(b.x), "f"(b.y), "f"(b.z), "f"(b.w)
               : "memory");
}

// A warp takes a batch of up to 32 tokens: a lane per token for what a token
// needs (its id, two divisions for strided ones, map entry, state, addresses),
// then the warp's row groups for the rows, which learn the addresses from the
// lane that has them.  (Every lane of a row group working that out for itself is
// a hundred instructions per row: 2^20 rows of 100 floats 196 us, now 141.)  The
// block scheduler hands the batches out: warps that take one after the other
// (two to four times as many blocks as are resident) lose up to a tenth on wide
// rows.
//
// A lane moves units of W float4 of a row, U of them.  W = 2 (rows of a multiple
// of eight elements): 256-bit loads, 256-bit or (16-bit types) 128-bit stores,
// half as many of each (2^20 rows of 64 floats 106 us, now 75).  Blocks per SM,
// by what the registers hold and what was fastest: 2^20 rows of 100 floats 171
// us at five, 142 at eight; 2^18 of 300 floats 104 at four, 110 at five.  At eight
// the kernels of W = 2, U = 1 spill one word of a thread (G = 32: four) to local
// memory.
constexpr int embed_blocks_per_sm(int U, int W) { return U == 1 ? 8 : (U * W <= 3 ? 4 : 3); }
// Tokens per batch, at most.
constexpr uint32_t embed_batch(int U) { return U == 1 ? 32 : 4; }

template <class T, int W, int G, int U>
__global__ void __launch_bounds__(kThreads, embed_blocks_per_sm(U, W))
embed_kernel(Store s, uint32_t w, const TokenView tv, uint32_t per, uint32_t dim, float scale, const RowView ov,
             int align) {
  after_previous();
  constexpr int C = U * W, GW = 32 / G;
  const uint32_t lane32 = threadIdx.x & 31, lane = lane32 & (G - 1), sub = lane32 / G;
  const uint32_t n4 = (dim + 3) >> 2, n = (uint32_t)tv.n;
  const uint64_t base = ((uint64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32) * per;
  if (base >= n) return;   // warp-uniform
  const uint32_t cnt = n - base < per ? (uint32_t)(n - base) : per;
  const uint32_t k = lane32 < cnt ? token_key(tv, base + lane32, s.K) : kNoKey;
  s.par = s.st->par;
  const bool mapped = s.st->live != 0;   // without replicas every map entry is -1
  const float4 *src = nullptr, *add = nullptr;
  if (k < s.K) src = row_source(s, mapped ? s.map[(uint64_t)w * s.K + k] : -1, k, &add);
  else if (k == kBadKey) set_error(s.st, ERR_KEY_RANGE);
  T* out = reinterpret_cast<T*>(ov.data) + (lane32 < cnt ? row_offset(ov, (uint32_t)base + lane32) : 0);
  const bool adds = __any_sync(0xFFFFFFFFu, add != nullptr);
  auto col_of = [&](int c) { return W * (uint32_t)(lane + c / W * G) + c % W; };
  auto of_token = [&](const void* p, uint32_t t) {   // what the lane of token t has
    return __shfl_sync(0xFFFFFFFFu, reinterpret_cast<unsigned long long>(p), t & 31);
  };
  for (uint32_t j = 0; j < cnt; j += GW) {
    const uint32_t t = j + sub;
    const float4* from = reinterpret_cast<const float4*>(of_token(src, t));
    T* row = reinterpret_cast<T*>(of_token(out, t));
    float4 v[C];
#pragma unroll
    for (int c = 0; c < C; c += W) {
      const uint32_t col = col_of(c);
#pragma unroll
      for (int q = 0; q < W; ++q) v[c + q] = f4zero();
      if (t >= cnt || from == nullptr || col >= n4) continue;
      if constexpr (W == 2) load8(from + col, v[c], v[c + 1]);
      else v[c] = from[col];
    }
    if (adds) {
      const float4* more = reinterpret_cast<const float4*>(of_token(add, t));
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const uint32_t col = col_of(c);
        if (t < cnt && more != nullptr && col < n4) v[c] = f4add(v[c], more[col]);
      }
    }
    if (t >= cnt) continue;
#pragma unroll
    for (int c = 0; c < C; c += W) {
      const uint32_t col = col_of(c);
      if (col >= n4) continue;
      if constexpr (W == 2 && sizeof(T) == 4) {
        store8(row + 4 * col, f4scale(v[c], scale), f4scale(v[c + 1], scale));
      } else if constexpr (W == 2) {
        const uint2 x = pack4(f4scale(v[c], scale), T()), y = pack4(f4scale(v[c + 1], scale), T());
        __stcs(reinterpret_cast<uint4*>(row + 4 * col), make_uint4(x.x, x.y, y.x, y.y));
      } else {
        put4(row, 4 * col, dim, f4scale(v[c], scale), align);
      }
    }
  }
}

// Whether every row begins on a multiple of `elements` elements.
bool rows_aligned(const RowView& r, size_t size, int64_t elements) {
  return reinterpret_cast<uintptr_t>(r.data) % (elements * size) == 0 && r.inner_stride % elements == 0 &&
         (r.flat || r.outer_stride % elements == 0);
}

template <class T>
void launch_typed(const Store& s, uint32_t w, const TokenView& t, uint32_t dim, float scale, const RowView& out,
                  int sms, cudaStream_t stream) {
  auto go = [&](auto Wc, auto Gc, auto Uc) {
    constexpr int W = decltype(Wc)::value, G = decltype(Gc)::value, U = decltype(Uc)::value;
    // few tokens: batches (of whole rounds of the warp's groups) that give every resident warp some (of six
    // blocks per SM: 24 x 1023 rows of 256 5.3 us, of eight 5.8)
    constexpr uint64_t round = 32 / G, most = std::max<uint64_t>(round, embed_batch(U));
    const uint64_t warps = (uint64_t)sms * std::min(embed_blocks_per_sm(U, W), 6) * (kThreads / 32);
    const uint64_t per = std::min<uint64_t>(most, ((t.n + warps - 1) / warps + round - 1) / round * round);
    const uint64_t blocks = (t.n + per * (kThreads / 32) - 1) / (per * (kThreads / 32));
    launch_after(embed_kernel<T, W, G, U>, (unsigned)blocks, kThreads, 0, stream, s, w, t, (uint32_t)per, dim, scale,
                 out, rows_aligned(out, sizeof(T), 4) ? 4 : (rows_aligned(out, sizeof(T), 2) ? 2 : 1));
  };
  using std::integral_constant;
  if (dim % 8 == 0 && s.D % 8 == 0 && rows_aligned(out, sizeof(T), 8)) {
    const integral_constant<int, 2> two{};
    const uint32_t units = dim / 8;
    if (units <= 4) go(two, integral_constant<int, 4>{}, integral_constant<int, 1>{});
    else if (units <= 8) go(two, integral_constant<int, 8>{}, integral_constant<int, 1>{});
    else if (units <= 16) go(two, integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (units <= 32) go(two, integral_constant<int, 32>{}, integral_constant<int, 1>{});
    else if (units <= 64) go(two, integral_constant<int, 32>{}, integral_constant<int, 2>{});
    else if (units <= 96) go(two, integral_constant<int, 32>{}, integral_constant<int, 3>{});
    else go(two, integral_constant<int, 32>{}, integral_constant<int, 4>{});
    return;
  }
  dispatch_gc((dim + 3) / 4, [&](auto Gc, auto Cc) { go(integral_constant<int, 1>{}, Gc, Cc); });
}

}  // namespace

void launch_embed(const Store& s, uint32_t w, const TokenView& t, uint32_t dim, float scale, const RowView& out,
                  int sms, cudaStream_t stream) {
  if (t.n == 0) return;
  note_launches(1);
  if (out.type == ADAPM_F32) launch_typed<float>(s, w, t, dim, scale, out, sms, stream);
  else if (out.type == ADAPM_F16) launch_typed<__half>(s, w, t, dim, scale, out, sms, stream);
  else launch_typed<__nv_bfloat16>(s, w, t, dim, scale, out, sms, stream);
}

}  // namespace adapm
