// Layer norm over rows of `dim` elements, forward and backward.
//
//   m = sum x / dim, r = 1 / sqrt(sum (x - m)^2 / dim + eps), h = (x - m) r
//   forward    y = h w + b
//   backward   g = dy w,  dx = r (g - sum g / dim - h (sum g h) / dim),
//              dw = sum over rows of dy h,  db = sum over rows of dy
//
// A row is taken by a group of lanes, 8 to 32 elements each, that stay in
// registers, so that both sums are over values already there: the squares are
// of differences from the mean, which costs no second pass over memory and
// loses nothing where the mean is large.  Rows of up to 512 elements are taken
// by (parts of) a warp, of up to 8192 by a block (forward, 16-bit rows in wide
// accesses: 1024 and 16,384), which has its next row on the way while it works
// on one; longer ones are read again from L2.  Arithmetic is on pairs of floats:
// one issue for two.  dweight and dbias are summed by every block over its rows,
// in registers, and joined in the order of the blocks.
// Bound by memory: 65,472 rows of 1024 bf16 forward 48 us, 5.5 TB/s, 262,144
// rows backward 271 us, 6.0 TB/s; one row of 4096 by the launch, 6.9 us.  Odd
// rows of 16 bits, which no wide access fits, are bound by instructions: 5105
// rows of 1001 fp16 backward 15 us, 8011 of 6511 bf16 133 forward (31 at the
// memory's rate) and 120 backward (46).  So are rows beyond a block's registers,
// which are read three times in such accesses: 1617 of 38,946 bf16 139 (37) and
// 504 (56), 4096 of 12,000 backward 346 (43).
#include <algorithm>

#include "dense.cuh"

namespace adapm {

namespace {

// A row is taken by `lanes` lanes (a power of two up to 32, or whole warps up
// to kMaxLanes), of which lane l holds elements ((j / VEC) * lanes + l) * VEC + j % VEC
// for j < EL; blocks of kSmallBlock threads hold several rows of few lanes.
constexpr int kMaxLanes = 512;
constexpr int kSmallBlock = 128;
struct Spread {
  int lanes, threads;
};
Spread spread_of(uint32_t dim, int el) {
  const uint32_t units = (dim + el - 1) / el;
  Spread s{1, kSmallBlock};
  if (units <= 32) {
    while ((uint32_t)s.lanes < units) s.lanes *= 2;
  } else {
    s.lanes = s.threads = (int)((units + 31) / 32 * 32);
  }
  return s;
}

// Elements of a lane: 8 where a warp's lanes are enough for the row; else as
// many as the registers hold beside the parameters (and, backward, their sums).
constexpr int kFew = 8;
constexpr int many(int type, int vec, bool backward) {
  return backward || type < 0 || type == ADAPM_F32 || vec == 1 ? 16 : 32;
}

// Sums of two numbers over a row's lanes; `part` is shared memory that
// successive calls use in turn (`turn` 0 and 1), so that one barrier a call is enough.
__device__ __forceinline__ float2 row_sum2(float a, float b, int lanes, float2 (*part)[32], int turn) {
  const int w = lanes < 32 ? lanes : 32;
  a = lanes_sum(a, w);
  b = lanes_sum(b, w);
  if (lanes <= 32) return make_float2(a, b);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = lanes >> 5;
  if (lane == 0) part[turn][warp] = make_float2(a, b);
  __syncthreads();
  if (warps > 8) {
    const float2 v = lane < warps ? part[turn][lane] : make_float2(0.f, 0.f);
    return make_float2(lanes_sum(v.x, 32), lanes_sum(v.y, 32));
  }
  float2 s = part[turn][0];
  for (int i = 1; i < warps; ++i) {
    s.x += part[turn][i].x;
    s.y += part[turn][i].y;
  }
  return s;
}

// Elements of a row that warp `warp` of its lanes holds, in accesses of VEC.
template <int VEC, int EL>
__device__ __forceinline__ float warp_elements(uint32_t dim, int lanes, int warp) {
  const int w = lanes < 32 ? lanes : 32;
  int n = 0;
#pragma unroll
  for (int i = 0; i < EL / VEC; ++i) {
    const int64_t left = (int64_t)dim - ((int64_t)i * lanes + warp * w) * VEC;
    n += left <= 0 ? 0 : (left < w * VEC ? (int)left : w * VEC);
  }
  return (float)n;
}

// Mean of a row and sum of squared differences from it.  Warps find both for
// their own elements first, so one exchange serves both: with n_w elements of
// sum s_w, the row's sum is sum q_w + sum n_w (s_w / n_w - m)^2.  counts: n_w of
// every warp, mine: this one's.  x (pairs; absent elements are zero) becomes
// its differences from the mean.
template <bool FULL, int VEC, int EL>
__device__ __forceinline__ float2 row_moments(uint64_t (&x)[EL / 2], float mine, const float* counts, uint32_t dim, int lane,
                                              int lanes, float2 (*part)[32], int turn) {
  const int w = lanes < 32 ? lanes : 32;
  uint64_t sum = x[0];
#pragma unroll
  for (int j = 1; j < EL / 2; ++j) sum = add_pair(sum, x[j]);
  const float s = lanes_sum(floats_of(sum).x + floats_of(sum).y, w);
  const float mean_w = mine > 0.f ? __fdividef(s, mine) : 0.f;
  const uint64_t minus = pair_of(-mean_w, -mean_w);
  uint64_t sq = 0;
#pragma unroll
  for (int j = 0; j < EL / 2; ++j) {
    x[j] = add_pair(x[j], minus);
    if constexpr (!FULL) {
      const float2 d = floats_of(x[j]);
      auto here = [&](int e) { return (uint32_t)((e / VEC) * lanes + lane) * VEC + e % VEC < dim; };
      x[j] = pair_of(here(2 * j) ? d.x : 0.f, here(2 * j + 1) ? d.y : 0.f);
    }
    sq = fma_pair(x[j], x[j], sq);
  }
  const float q = lanes_sum(floats_of(sq).x + floats_of(sq).y, w);
  if (lanes <= 32) return make_float2(mean_w, q);
  const int wl = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = lanes >> 5;
  if (wl == 0) part[turn][warp] = make_float2(s, q);
  __syncthreads();
  float total = 0.f;
  for (int i = 0; i < warps; ++i) total += part[turn][i].x;
  const float mean = total / (float)dim;
  float all = 0.f;
  for (int i = 0; i < warps; ++i) {
    const float2 v = part[turn][i];
    const float n = counts[i], d = n > 0.f ? v.x / n - mean : 0.f;
    all += fmaf(n * d, d, v.y);
  }
  const uint64_t more = pair_of(mean_w - mean, mean_w - mean);
#pragma unroll
  for (int j = 0; j < EL / 2; ++j) x[j] = add_pair(x[j], more);
  return make_float2(mean, all);
}

// A lane's elements as they come from memory (TYPE -1: a type known at run
// time alone, as floats), so that the next row's can be on their way while
// this one is worked on.
template <int TYPE, int VEC, int EL>
struct Raw {
  static constexpr int kSize = TYPE == ADAPM_F32 || TYPE < 0 ? 4 : 2;
  static constexpr int kWords = VEC == 1 ? EL : EL * kSize / 4;
  uint32_t w[kWords];
};
template <bool FULL, int TYPE, int VEC, int EL>
__device__ __forceinline__ void fetch(const RowView& v, uint64_t row, uint32_t dim, int lane, int lanes, Raw<TYPE, VEC, EL>& r) {
  const int type = TYPE < 0 ? v.type : TYPE;
  const char* p = v.data + (row_offset(v, (uint32_t)row) + (int64_t)lane * VEC) * type_size(type);
  constexpr int A = EL / VEC, W = Raw<TYPE, VEC, EL>::kWords / A;   // accesses; words of one
  if constexpr (!FULL) {
#pragma unroll
    for (int j = 0; j < Raw<TYPE, VEC, EL>::kWords; ++j) r.w[j] = 0u;
  }
  auto all = [&](auto kind) {
    constexpr int T = decltype(kind)::value, S = T == ADAPM_F32 ? 4 : 2;
    const char* q = p;
#pragma unroll
    for (int i = 0; i < A; ++i, q += (int64_t)lanes * VEC * S) {
      if (!FULL && (uint32_t)(i * lanes + lane) * VEC >= dim) continue;
      if constexpr (W == 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(q);
        r.w[4 * i] = x.x; r.w[4 * i + 1] = x.y; r.w[4 * i + 2] = x.z; r.w[4 * i + 3] = x.w;
      } else if constexpr (W == 2) {
        const uint2 x = *reinterpret_cast<const uint2*>(q);
        r.w[2 * i] = x.x; r.w[2 * i + 1] = x.y;
      } else if constexpr (TYPE < 0) {
        r.w[i] = __float_as_uint(load_as(q, T, 0));
      } else {
        static_assert(W == 1 && VEC == 1);
        if constexpr (S == 4) r.w[i] = *reinterpret_cast<const uint32_t*>(q);
        else r.w[i] = *reinterpret_cast<const uint16_t*>(q);
      }
    }
  };
  by_type<TYPE>(type, all);
}
// The elements as pairs of floats.
template <int TYPE, int VEC, int EL>
__device__ __forceinline__ void unpack_raw(const Raw<TYPE, VEC, EL>& r, uint64_t (&x)[EL / 2]) {
#pragma unroll
  for (int j = 0; j < EL / 2; ++j) {
    if constexpr (TYPE == ADAPM_F32 || TYPE < 0) {
      x[j] = (uint64_t)r.w[2 * j] | ((uint64_t)r.w[2 * j + 1] << 32);
    } else if constexpr (VEC == 1) {
      x[j] = pair_of(unpack2<TYPE>(r.w[2 * j]).x, unpack2<TYPE>(r.w[2 * j + 1]).x);
    } else {
      const float2 f = unpack2<TYPE>(r.w[j]);
      x[j] = pair_of(f.x, f.y);
    }
  }
}
template <bool FULL, int VEC, int EL>
__device__ __forceinline__ void store_row(const RowView& v, uint64_t row, uint32_t dim, int lane, int lanes, const uint64_t (&pairs)[EL / 2]) {
  float y[EL];
#pragma unroll
  for (int j = 0; j < EL / 2; ++j) {
    y[2 * j] = floats_of(pairs[j]).x;
    y[2 * j + 1] = floats_of(pairs[j]).y;
  }
  auto all = [&](auto kind) {
    constexpr int T = decltype(kind)::value, S = T == ADAPM_F32 ? 4 : 2;
    char* p = v.data + (row_offset(v, (uint32_t)row) + (int64_t)lane * VEC) * S;
#pragma unroll
    for (int i = 0; i < EL / VEC; ++i, p += (int64_t)lanes * VEC * S)
      if (FULL || (uint32_t)(i * lanes + lane) * VEC < dim) store_n<T, VEC>(p, y + i * VEC);
  };
  by_type<-1>(v.type, all);
}
template <int VEC, int EL>
__device__ __forceinline__ void load_params(const VectorView& v, uint32_t dim, int lane, int lanes, float none, uint64_t (&pairs)[EL / 2]) {
  if (v.data == nullptr) {
#pragma unroll
    for (int j = 0; j < EL / 2; ++j) pairs[j] = pair_of(none, none);
    return;
  }
  float w[EL];
  auto all = [&](auto kind) {
    constexpr int T = decltype(kind)::value;
#pragma unroll
    for (int j = 0; j < EL; ++j) {
      const uint32_t c = (uint32_t)((j / VEC) * lanes + lane) * VEC + j % VEC;
      w[j] = c < dim ? load_as(v.data, T, c) : 0.f;
    }
  };
  by_type<-1>(v.type, all);
#pragma unroll
  for (int j = 0; j < EL / 2; ++j) pairs[j] = pair_of(w[2 * j], w[2 * j + 1]);
}

// FULL: the lanes hold nothing but elements.
template <bool FULL, int TYPE, int VEC, int EL>
__global__ void __launch_bounds__(kMaxLanes)
norm_kernel(const __grid_constant__ NormArgs a, int lanes) {
  after_previous();
  __shared__ float2 part[2][32];
  __shared__ float counts[32];
  const int lane = threadIdx.x % lanes, group = threadIdx.x / lanes, rows = blockDim.x / lanes;
  const uint64_t step = (uint64_t)gridDim.x * rows;
  // (the rows of a warp are taken together: lanes without a row take the last one, and leave it)
  uint64_t row = (uint64_t)blockIdx.x * rows + group;
  auto held = [&](uint64_t r) { return r < a.n ? r : a.n - 1; };
  Raw<TYPE, VEC, EL> raw;
  fetch<FULL>(a.x, held(row), a.dim, lane, lanes, raw);
  uint64_t w[EL / 2], b[EL / 2];
  load_params<VEC, EL>(a.weight, a.dim, lane, lanes, 1.f, w);
  load_params<VEC, EL>(a.bias, a.dim, lane, lanes, 0.f, b);
  if (threadIdx.x < 32) counts[threadIdx.x] = (int)threadIdx.x * 32 < lanes ? warp_elements<VEC, EL>(a.dim, lanes, threadIdx.x) : 0.f;
  const float mine = warp_elements<VEC, EL>(a.dim, lanes, lane >> 5);
  if (lanes > 32) __syncthreads();
  int turn = 0;
  for (uint64_t r0 = (uint64_t)blockIdx.x * rows; r0 < a.n; r0 += step, row += step, turn ^= 1) {
    uint64_t x[EL / 2];
    unpack_raw(raw, x);
    if (r0 + step < a.n) fetch<FULL>(a.x, held(row + step), a.dim, lane, lanes, raw);
    const float2 m = row_moments<FULL, VEC, EL>(x, mine, counts, a.dim, lane, lanes, part, turn);
    const float r = 1.f / sqrtf(m.y / (float)a.dim + a.eps);
    if (row >= a.n) continue;
    const uint64_t rr = pair_of(r, r);
#pragma unroll
    for (int j = 0; j < EL / 2; ++j) x[j] = fma_pair(mul_pair(x[j], rr), w[j], b[j]);
    store_row<FULL, VEC, EL>(a.out, row, a.dim, lane, lanes, x);
    if (a.stats != nullptr && lane == 0) reinterpret_cast<float2*>(a.stats)[row] = make_float2(m.x, r);
  }
}

// Rows that do not fit a block's registers: three passes, of which the second
// and third find the row in L2.
__global__ void __launch_bounds__(1024)
norm_long_kernel(const __grid_constant__ NormArgs a) {
  after_previous();
  __shared__ float2 part[2][32];
  for (uint64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const char* x = a.x.data + row_offset(a.x, (uint32_t)row) * type_size(a.x.type);
    char* y = a.out.data + row_offset(a.out, (uint32_t)row) * type_size(a.out.type);
    by_type<-1>(a.x.type, [&](auto kind) {
      constexpr int T = decltype(kind)::value;
      float s = 0.f;
#pragma unroll 8
      for (uint32_t c = threadIdx.x; c < a.dim; c += 1024) s += load_as(x, T, c);
      const float mean = row_sum2(s, 0.f, 1024, part, 0).x / (float)a.dim;
      float q = 0.f;
#pragma unroll 8
      for (uint32_t c = threadIdx.x; c < a.dim; c += 1024) {
        const float d = load_as(x, T, c) - mean;
        q = fmaf(d, d, q);
      }
      const float r = 1.f / sqrtf(row_sum2(q, 0.f, 1024, part, 1).x / (float)a.dim + a.eps);
      auto write = [&](auto wkind) {
        constexpr int W = decltype(wkind)::value;
#pragma unroll 4
        for (uint32_t c = threadIdx.x; c < a.dim; c += 1024) {
          const float w = a.weight.data ? load_as(a.weight.data, W, c) : 1.f;
          const float b = a.bias.data ? load_as(a.bias.data, a.bias.type, c) : 0.f;
          store_as(y, a.out.type, c, fmaf((load_as(x, T, c) - mean) * r, w, b));
        }
      };
      by_type<-1>(a.weight.type, write);
      if (a.stats != nullptr && threadIdx.x == 0) reinterpret_cast<float2*>(a.stats)[row] = make_float2(mean, r);
    });
  }
}

// dx, and every block's sums of dy h and dy over its rows.
template <bool FULL, int TYPE, int VEC, int EL>
__global__ void __launch_bounds__(kMaxLanes)
norm_grad_kernel(const __grid_constant__ NormArgs a, int lanes) {
  after_previous();
  __shared__ float2 part[2][32];
  __shared__ float sums[kSmallBlock * EL];
  const int lane = threadIdx.x % lanes, group = threadIdx.x / lanes, rows = blockDim.x / lanes;
  const uint64_t step = (uint64_t)gridDim.x * rows;
  uint64_t row = (uint64_t)blockIdx.x * rows + group;
  auto held = [&](uint64_t r) { return r < a.n ? r : a.n - 1; };
  Raw<TYPE, VEC, EL> rx, rg;
  fetch<FULL>(a.x, held(row), a.dim, lane, lanes, rx);
  fetch<FULL>(a.grad, held(row), a.dim, lane, lanes, rg);
  float2 next = reinterpret_cast<const float2*>(a.stats)[held(row)];
  uint64_t w[EL / 2], dw[EL / 2], db[EL / 2];
  load_params<VEC, EL>(a.weight, a.dim, lane, lanes, 1.f, w);
#pragma unroll
  for (int j = 0; j < EL / 2; ++j) dw[j] = db[j] = 0;
  const float inv = 1.f / (float)a.dim;
  int turn = 0;
  for (uint64_t r0 = (uint64_t)blockIdx.x * rows; r0 < a.n; r0 += step, row += step, turn ^= 1) {
    const bool live = row < a.n;
    const float2 st = next;
    uint64_t x[EL / 2], g[EL / 2];
    unpack_raw(rx, x);
    unpack_raw(rg, g);
    if (r0 + step < a.n) {
      fetch<FULL>(a.x, held(row + step), a.dim, lane, lanes, rx);
      fetch<FULL>(a.grad, held(row + step), a.dim, lane, lanes, rg);
      next = reinterpret_cast<const float2*>(a.stats)[held(row + step)];
    }
    const uint64_t minus = pair_of(-st.x, -st.x), rr = pair_of(st.y, st.y);
    uint64_t s0 = 0, s1 = 0;
    // (where there is no element g is zero; lanes without a row add to sums that nobody reads)
#pragma unroll
    for (int j = 0; j < EL / 2; ++j) {
      x[j] = mul_pair(add_pair(x[j], minus), rr);   // h
      if (live) {
        dw[j] = fma_pair(g[j], x[j], dw[j]);
        db[j] = add_pair(db[j], g[j]);
      }
      g[j] = mul_pair(g[j], w[j]);
      s0 = add_pair(s0, g[j]);
      s1 = fma_pair(g[j], x[j], s1);
    }
    if (a.out.data == nullptr) continue;
    const float2 p0 = floats_of(s0), p1 = floats_of(s1);
    const float2 s = row_sum2(p0.x + p0.y, p1.x + p1.y, lanes, part, turn);
    if (!live) continue;
    const float c0 = -s.x * inv, c1 = -s.y * inv;
    const uint64_t m0 = pair_of(c0, c0), m1 = pair_of(c1, c1);
#pragma unroll
    for (int j = 0; j < EL / 2; ++j) x[j] = mul_pair(fma_pair(x[j], m1, add_pair(g[j], m0)), rr);
    store_row<FULL, VEC, EL>(a.out, row, a.dim, lane, lanes, x);
  }
  if (a.parts == nullptr) return;
  // the block's rows together, group after group
  float* out = a.parts + (uint64_t)blockIdx.x * 2 * a.dim;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    auto element = [&](int j) {
      const float2 f = floats_of(which ? db[j / 2] : dw[j / 2]);
      return j % 2 ? f.y : f.x;
    };
    if (lanes > 32) {   // one row at a time
#pragma unroll
      for (int j = 0; j < EL; ++j) {
        const uint32_t c = (uint32_t)((j / VEC) * lanes + lane) * VEC + j % VEC;
        if (c < a.dim) out[which * a.dim + c] = element(j);
      }
      continue;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < EL; ++j)
      sums[group * lanes * EL + ((j / VEC) * lanes + lane) * VEC + j % VEC] = element(j);
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < a.dim; c += blockDim.x) {
      float s = 0.f;
      for (int g = 0; g < rows; ++g) s += sums[g * lanes * EL + c];
      out[which * a.dim + c] = s;
    }
  }
}

// Rows that do not fit a block: dx by two passes ...
__global__ void __launch_bounds__(1024)
norm_grad_long_kernel(const __grid_constant__ NormArgs a) {
  after_previous();
  __shared__ float2 part[2][32];
  int turn = 0;
  for (uint64_t row = blockIdx.x; row < a.n; row += gridDim.x, turn ^= 1) {
    const char* x = a.x.data + row_offset(a.x, (uint32_t)row) * type_size(a.x.type);
    const char* g = a.grad.data + row_offset(a.grad, (uint32_t)row) * type_size(a.grad.type);
    char* dx = a.out.data + row_offset(a.out, (uint32_t)row) * type_size(a.out.type);
    const float2 st = reinterpret_cast<const float2*>(a.stats)[row];
    auto both = [&](auto xkind, auto gkind) {
      constexpr int X = decltype(xkind)::value, G = decltype(gkind)::value;
      auto gw_at = [&](uint32_t c) { return load_as(g, G, c) * (a.weight.data ? load_as(a.weight.data, a.weight.type, c) : 1.f); };
      float s0 = 0.f, s1 = 0.f;
#pragma unroll 4
      for (uint32_t c = threadIdx.x; c < a.dim; c += 1024) {
        const float gw = gw_at(c);
        s0 += gw;
        s1 = fmaf(gw, (load_as(x, X, c) - st.x) * st.y, s1);
      }
      const float2 s = row_sum2(s0, s1, 1024, part, turn);
      const float c0 = s.x / (float)a.dim, c1 = s.y / (float)a.dim;
#pragma unroll 4
      for (uint32_t c = threadIdx.x; c < a.dim; c += 1024)
        store_as(dx, a.out.type, c, st.y * (gw_at(c) - c0 - (load_as(x, X, c) - st.x) * st.y * c1));
    };
    by_type<-1>(a.x.type, [&](auto xkind) {
      if (a.grad.type == a.x.type) both(xkind, xkind);
      else by_type<-1>(a.grad.type, [&](auto gkind) { both(xkind, gkind); });
    });
  }
}

// ... and the sums over rows before that (dx may be written over x or dy):
// block (i, j) takes 256 columns of every gridDim.y-th row.
__global__ void __launch_bounds__(256)
norm_columns_kernel(const __grid_constant__ NormArgs a) {
  after_previous();
  const uint64_t c = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= a.dim) return;
  float dw = 0.f, db = 0.f;
  by_type<-1>(a.x.type, [&](auto xkind) {
    by_type<-1>(a.grad.type, [&](auto gkind) {
      constexpr int X = decltype(xkind)::value, G = decltype(gkind)::value;
#pragma unroll 4
      for (uint64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
        const float2 st = reinterpret_cast<const float2*>(a.stats)[row];
        const float g = load_as(a.grad.data + row_offset(a.grad, (uint32_t)row) * type_size(G), G, c);
        const float x = load_as(a.x.data + row_offset(a.x, (uint32_t)row) * type_size(X), X, c);
        dw = fmaf(g, (x - st.x) * st.y, dw);
        db += g;
      }
    });
  });
  float* out = a.parts + (uint64_t)blockIdx.y * 2 * a.dim;
  out[c] = dw;
  out[a.dim + c] = db;
}

// The sums of `count` blocks over `width` columns, in a fixed order: a block
// takes kJoinColumns of them, each by kJoinRows threads, which take every
// kJoinRows-th block's sums, four of them on their way at a time.  Few columns a
// block: more blocks, and fewer loads one after the other.
constexpr uint32_t kJoinColumns = 16, kJoinRows = 1024 / kJoinColumns;
__global__ void __launch_bounds__(1024)
column_join_kernel(const float* parts, uint32_t count, uint64_t width, uint32_t dim, VectorView low, VectorView high) {
  after_previous();
  __shared__ float sums[kJoinColumns][kJoinRows + 1];
  const uint32_t column = threadIdx.x % kJoinColumns, first = threadIdx.x / kJoinColumns;
  const uint64_t c = (uint64_t)blockIdx.x * kJoinColumns + column;
  float s = 0.f;
  if (c < width) {
    uint32_t p = first;
    for (; p + 3 * kJoinRows < count; p += 4 * kJoinRows) {
      const float x0 = parts[p * width + c], x1 = parts[(p + kJoinRows) * width + c], x2 = parts[(p + 2 * kJoinRows) * width + c],
                  x3 = parts[(p + 3 * kJoinRows) * width + c];
      s = (((s + x0) + x1) + x2) + x3;
    }
    for (; p < count; p += kJoinRows) s += parts[p * width + c];
  }
  sums[column][first] = s;
  __syncthreads();
  // a warp adds up a column
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  if (warp >= kJoinColumns) return;
  s = 0.f;
  for (uint32_t i = lane; i < kJoinRows; i += 32) s += sums[warp][i];
  s = lanes_sum(s, 32);
  const uint64_t mine = (uint64_t)blockIdx.x * kJoinColumns + warp;
  if (lane != 0 || mine >= width) return;
  const VectorView& v = mine < dim ? low : high;
  if (v.data != nullptr) store_as(v.data, v.type, mine < dim ? mine : mine - dim, s);
}

// Elements that every access takes: rows begin and end on a multiple of it.
template <class... V>
int width_of(const NormArgs& a, const V&... views) {
  for (int vec : {8, 4}) {
    if (a.x.type == ADAPM_F32 && vec == 8) continue;
    bool ok = a.dim % vec == 0;
    ((ok = ok && rows_on(views, a.n, vec)), ...);
    if (ok) return vec;
  }
  return 1;
}

// How the kernels take the rows: types known when compiled or not, the width of
// an access, elements of a lane.
struct Plan {
  int type, vec, el;
  Spread s;
  unsigned grid;
  bool wide;   // too wide for a block
};
Plan plan_of(const NormArgs& a, bool backward, int sms) {
  Plan p{};
  const bool mixed = backward && a.grad.type != a.x.type;
  p.type = mixed ? -1 : a.x.type;
  p.vec = mixed ? 1 : (!backward ? width_of(a, a.x, a.out) : (a.out.data ? width_of(a, a.x, a.grad, a.out) : width_of(a, a.x, a.grad)));
  p.el = a.dim <= 32 * kFew ? kFew : many(p.type, p.vec, backward);
  p.s = spread_of(a.dim, p.el);
  p.wide = p.s.lanes > kMaxLanes;
  const uint64_t rows = p.s.threads / p.s.lanes;
  // blocks per SM that the registers hold
  const uint64_t per_sm = std::max(1, (p.el == kFew ? 1024 : 512) / p.s.threads);
  p.grid = (unsigned)std::max<uint64_t>(1, std::min<uint64_t>((a.n + rows - 1) / rows, (uint64_t)sms * per_sm));
  return p;
}
constexpr int kLongRows = 64;   // row classes of norm_columns_kernel
uint64_t part_count(const NormArgs& a, const Plan& p) { return p.wide ? std::min<uint64_t>(a.n, kLongRows) : p.grid; }

template <bool BACK, bool FULL, int TYPE, int VEC, int EL>
void launch_el(const NormArgs& a, const Plan& p, cudaStream_t stream) {
  if constexpr (BACK) launch_after(norm_grad_kernel<FULL, TYPE, VEC, EL>, p.grid, p.s.threads, 0, stream, a, p.s.lanes);
  else launch_after(norm_kernel<FULL, TYPE, VEC, EL>, p.grid, p.s.threads, 0, stream, a, p.s.lanes);
}
template <bool BACK, int TYPE, int VEC>
void launch_as(const NormArgs& a, const Plan& p, cudaStream_t stream) {
  constexpr int MANY = many(TYPE, VEC, BACK);
  const bool full = (uint64_t)p.s.lanes * p.el == a.dim;
  if constexpr (VEC > 1) {   // (rows of full lanes are read in wide accesses)
    if (full && p.el == kFew) return launch_el<BACK, true, TYPE, VEC, kFew>(a, p, stream);
    if (full) return launch_el<BACK, true, TYPE, VEC, MANY>(a, p, stream);
  }
  if (p.el == kFew) launch_el<BACK, false, TYPE, VEC, kFew>(a, p, stream);
  else launch_el<BACK, false, TYPE, VEC, MANY>(a, p, stream);
}
template <bool BACK, int TYPE>
void launch_type(const NormArgs& a, const Plan& p, cudaStream_t stream) {
  if constexpr (TYPE == ADAPM_F16 || TYPE == ADAPM_BF16)
    if (p.vec == 8) return launch_as<BACK, TYPE, 8>(a, p, stream);
  if (p.vec == 4) launch_as<BACK, TYPE, 4>(a, p, stream);
  else launch_as<BACK, TYPE, 1>(a, p, stream);
}
template <bool BACK>
void launch(const NormArgs& a, const Plan& p, cudaStream_t stream) {
  note_launches(1);
  if (p.type == ADAPM_F32) launch_type<BACK, ADAPM_F32>(a, p, stream);
  else if (p.type == ADAPM_F16) launch_type<BACK, ADAPM_F16>(a, p, stream);
  else if (p.type == ADAPM_BF16) launch_type<BACK, ADAPM_BF16>(a, p, stream);
  else if constexpr (BACK) launch_as<BACK, -1, 1>(a, p, stream);
}

}  // namespace

void launch_layer_norm(const NormArgs& a, int sms, cudaStream_t stream) {
  const Plan p = plan_of(a, false, sms);
  if (!p.wide) return launch<false>(a, p, stream);
  note_launches(1);
  launch_after(norm_long_kernel, (unsigned)std::min<uint64_t>(a.n, (uint64_t)sms * 2), 1024, 0, stream, a);
}

size_t norm_grad_scratch(const NormArgs& a, int sms) {
  return a.dweight.data || a.dbias.data ? part_count(a, plan_of(a, true, sms)) * 2 * a.dim : 0;
}

void launch_layer_norm_grad(const NormArgs& a, int sms, cudaStream_t stream) {
  const Plan p = plan_of(a, true, sms);
  const uint64_t count = part_count(a, p);
  if (!p.wide) {
    launch<true>(a, p, stream);
  } else {
    if (a.parts != nullptr) {
      note_launches(1);
      // (the grid has two dimensions: launched plainly)
      norm_columns_kernel<<<dim3((a.dim + 255) / 256, (unsigned)count), 256, 0, stream>>>(a);
    }
    if (a.out.data != nullptr) {
      note_launches(1);
      launch_after(norm_grad_long_kernel, (unsigned)std::min<uint64_t>(a.n, (uint64_t)sms * 2), 1024, 0, stream, a);
    }
  }
  if (a.parts != nullptr) {
    launch_column_join(a.parts, (uint32_t)count, 2ull * a.dim, a.dim, a.dweight, a.dbias, stream);
  }
}

void launch_column_join(const float* parts, uint32_t count, uint64_t width, uint32_t dim, const VectorView& low,
                        const VectorView& high, cudaStream_t stream) {
  note_launches(1);
  launch_after(column_join_kernel, (unsigned)((width + kJoinColumns - 1) / kJoinColumns), 1024, 0, stream, parts, count, width, dim, low, high);
}

}  // namespace adapm
