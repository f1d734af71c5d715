// embed: the rows of a batch of tokens, scaled, in the type of the model.
//
//   out[t][c] = round(scale * value(worker, token t)[c]),  c < dim
//
// One pass: the gather of pull (store.cu) with the multiplication and the
// rounding to 16 bits on the way, so that the fp32 rows never travel.  Bound by
// memory: 4 dim bytes in per distinct token (repeats come from L2), dim
// elements out per token.  64 x 4096 tokens of 62,000 distinct ones, rows of
// 1024, bf16 out: 142 us, 5.6 TB/s of those bytes; 64 x 2048 distinct rows, fp32
// out, 160 us, 6.7 TB/s.
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

__device__ __forceinline__ float4 f4scale(float4 v, float s) {
  return make_float4(v.x * s, v.y * s, v.z * s, v.w * s);
}

// 256 bits at once, from a 32-byte boundary.
__device__ __forceinline__ void load8(const float4* p, float4& a, float4& b) {
  asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(a.x), "=f"(a.y), "=f"(a.z), "=f"(a.w), "=f"(b.x), "=f"(b.y), "=f"(b.z), "=f"(b.w)
               : "l"(p));
}

// A lane takes units of W float4 of a row, U of them.  W = 2 (16-bit rows of a
// multiple of eight elements): 256-bit loads and 128-bit stores, half as many
// of each (262,144 rows of 1024 floats out of a table in L2, where the stores
// are what counts, 97 -> 93 us).  Rows per group and round: four to eight
// float4 per lane in flight, at three blocks per SM (64 x 4096 rows of 1024
// floats: 157 us with as many registers as the compiler likes, 147 at three
// blocks, 151 at four).
constexpr int embed_rows(int U, int W) {
  return W == 2 ? (U == 1 ? 2 : 1) : (U == 1 ? 4 : (U == 2 ? 2 : 1));
}

template <class T, int W, int G, int U, int R>
__global__ void __launch_bounds__(kThreads, U * W == 1 ? 5 : 3)
embed_kernel(Store s, uint32_t w, const TokenView tv, uint32_t dim, float scale, const RowView ov, bool vec) {
  after_previous();
  constexpr int C = U * W;
  const int lane = threadIdx.x & (G - 1);
  const uint64_t g = group_id<G>(), ng = group_count<G>();
  const uint32_t n4 = (dim + 3) >> 2;
  const uint64_t n = tv.n;
  const int32_t* mapw = s.map + (uint64_t)w * s.K;
  s.par = s.st->par;
  const bool mapped = s.st->live != 0;   // without replicas every map entry is -1
  const uint64_t step = ng * R;
  bool bad = false;
  auto col_of = [&](int c) { return W * (uint32_t)(lane + c / W * G) + c % W; };
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
    for (int c = 0; c < C; c += W) {
      const uint32_t col = col_of(c);
#pragma unroll
      for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int j = 0; j < W; ++j) v[r][c + j] = f4zero();
        if (src[r] == nullptr || col >= n4) continue;
        if constexpr (W == 2) load8(src[r] + col, v[r][c], v[r][c + 1]);
        else v[r][c] = src[r][col];
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (add[r] != nullptr)
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const uint32_t col = col_of(c);
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
      for (int c = 0; c < C; c += W) {
        const uint32_t col = col_of(c);
        if (col >= n4) continue;
        if constexpr (W == 2) {
          const uint2 a = pack4(f4scale(v[r][c], scale), T()), b = pack4(f4scale(v[r][c + 1], scale), T());
          __stcs(reinterpret_cast<uint4*>(row + 4 * col), make_uint4(a.x, a.y, b.x, b.y));
        } else {
          put4(row, 4 * col, dim, f4scale(v[r][c], scale), vec);
        }
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

// Whether every row begins on a multiple of `elements` elements.
bool rows_aligned(const RowView& r, size_t size, int64_t elements) {
  return reinterpret_cast<uintptr_t>(r.data) % (elements * size) == 0 && r.inner_stride % elements == 0 &&
         (r.flat || r.outer_stride % elements == 0);
}

template <class T>
void launch_typed(const Store& s, uint32_t w, const TokenView& t, uint32_t dim, float scale, const RowView& out,
                  int sms, cudaStream_t stream) {
  auto go = [&](auto Wc, auto Gc, auto Uc) {
    constexpr int W = decltype(Wc)::value, G = decltype(Gc)::value, U = decltype(Uc)::value, R = embed_rows(U, W);
    launch_after(embed_kernel<T, W, G, U, R>, grid_for((t.n + R - 1) / R, G, sms), kThreads, 0, stream, s, w, t, dim,
                 scale, out, rows_aligned(out, sizeof(T), 4));
  };
  using std::integral_constant;
  if constexpr (sizeof(T) == 2) {
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
