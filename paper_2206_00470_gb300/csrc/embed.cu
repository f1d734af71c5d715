// embed: the rows of a batch of tokens, scaled, in the type of the model.
//
//   out[t][c] = round(scale * value(worker, token t)[c]),  c < dim
//
// One pass: the gather of pull (store.cu) with the multiplication and the
// rounding to 16 bits on the way, so that the fp32 rows never travel.  Bound by
// memory: 4 dim bytes in per distinct token (repeats come from L2), dim
// elements out per token.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

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

// Up to four elements of a row from column c; `vec`: rows begin on a multiple
// of four elements.
template <class T>
__device__ __forceinline__ void put4(T* row, uint32_t c, uint32_t dim, float4 v, bool vec) {
  if (vec && c + 4 <= dim) {
    auto p = pack4(v, T());
    __stcs(reinterpret_cast<decltype(p)*>(row + c), p);
    return;
  }
  const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (c + j < dim) row[c + j] = round_to<T>(x[j]);
}

// Rows per group and round, as in pull.
constexpr int embed_rows(int C) { return C == 1 ? 4 : (8 / C > 0 ? 8 / C : 1); }

template <class T, int G, int C, int R>
__global__ void __launch_bounds__(kThreads, C == 1 ? 5 : 1)
embed_kernel(Store s, uint32_t w, const TokenView tv, uint32_t dim, float scale, const RowView ov, bool vec) {
  after_previous();
  const int lane = threadIdx.x & (G - 1);
  const uint64_t g = group_id<G>(), ng = group_count<G>();
  const uint32_t D4 = s.D >> 2, n4 = (dim + 3) >> 2;
  const uint64_t n = tv.n;
  const int32_t* mapw = s.map + (uint64_t)w * s.K;
  s.par = s.st->par;
  const bool mapped = s.st->live != 0;   // without replicas every map entry is -1
  const uint64_t step = ng * R;
  bool bad = false;
  auto load_keys = [&](uint64_t b, uint32_t (&k)[R]) {
#pragma unroll
    for (int r = 0; r < R; ++r) k[r] = b + r < n ? token_key(tv, b + r, s.K) : kNoKey;
  };
  auto load_slots = [&](const uint32_t (&k)[R], int32_t (&sl)[R]) {
#pragma unroll
    for (int r = 0; r < R; ++r) sl[r] = mapped && k[r] < s.K ? mapw[k[r]] : -1;
  };
  uint64_t base = g * R;
  uint32_t k0[R], k1[R];
  int32_t sl0[R];
  load_keys(base, k0);
  load_keys(base + step, k1);
  load_slots(k0, sl0);
  for (; base < n; base += step) {
    const float4* src[R];
    const float4* add[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      src[r] = add[r] = nullptr;
      if (k0[r] < s.K) src[r] = row_source(s, sl0[r], k0[r], &add[r]);
      else if (k0[r] == kBadKey) bad = true;
    }
    float4 v[R][C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint32_t col = lane + c * G;
#pragma unroll
      for (int r = 0; r < R; ++r) v[r][c] = (src[r] != nullptr && col < n4) ? src[r][col] : f4zero();
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (add[r] != nullptr)
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const uint32_t col = lane + c * G;
          if (col < n4) v[r][c] = f4add(v[r][c], add[r][col]);
        }
    int32_t sl1[R];
    uint32_t k2[R];
    load_slots(k1, sl1);
    load_keys(base + 2 * step, k2);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (base + r >= n) break;
      T* row = reinterpret_cast<T*>(ov.data) + row_offset(ov, (uint32_t)(base + r));
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const uint32_t col = lane + c * G;
        const float4 x = v[r][c];
        if (col < n4)
          put4(row, 4 * col, dim, make_float4(x.x * scale, x.y * scale, x.z * scale, x.w * scale), vec);
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      k0[r] = k1[r];
      sl0[r] = sl1[r];
      k1[r] = k2[r];
    }
  }
  if (bad && lane == 0) set_error(s.st, ERR_KEY_RANGE);
}

template <class T>
void launch_typed(const Store& s, uint32_t w, const TokenView& t, uint32_t dim, float scale, const RowView& out,
                  bool vec, int sms, cudaStream_t stream) {
  dispatch_gc((dim + 3) / 4, [&](auto Gc, auto Cc) {
    constexpr int G = decltype(Gc)::value, C = decltype(Cc)::value, R = embed_rows(C);
    launch_after(embed_kernel<T, G, C, R>, grid_for((t.n + R - 1) / R, G, sms), kThreads, 0, stream, s, w, t, dim,
                 scale, out, vec);
  });
}

}  // namespace

void launch_embed(const Store& s, uint32_t w, const TokenView& t, uint32_t dim, float scale, const RowView& out,
                  int sms, cudaStream_t stream) {
  if (t.n == 0) return;
  const size_t size = out.type == ADAPM_F32 ? 4 : 2;
  const bool vec = reinterpret_cast<uintptr_t>(out.data) % (4 * size) == 0 && out.inner_stride % 4 == 0 &&
                   (out.flat || out.outer_stride % 4 == 0);
  note_launches(1);
  if (out.type == ADAPM_F32) launch_typed<float>(s, w, t, dim, scale, out, vec, sms, stream);
  else if (out.type == ADAPM_F16) launch_typed<__half>(s, w, t, dim, scale, out, vec, sms, stream);
  else launch_typed<__nv_bfloat16>(s, w, t, dim, scale, out, vec, sms, stream);
}

}  // namespace adapm
