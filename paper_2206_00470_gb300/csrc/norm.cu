// Layer norm over rows of `dim` elements, forward and backward.
//
//   m = sum x / dim, r = 1 / sqrt(sum (x - m)^2 / dim + eps), h = (x - m) r
//   forward    y = h w + b
//   backward   g = dy w,  dx = r (g - sum g / dim - h (sum g h) / dim),
//              dw = sum over rows of dy h,  db = sum over rows of dy
//
// A row is taken by a group of lanes, eight elements each, that stay in
// registers, so that both sums of squares and sums are over values already
// there: the squares are of differences from the mean, which costs no second
// pass over memory and loses nothing where the mean is large.  Rows of up to
// 256 elements are taken by (parts of) a warp, of up to 8192 by a block.
// Bound by memory.
#include <algorithm>

#include "dense.cuh"

namespace adapm {

namespace {

constexpr int kUnit = 8;             // elements of a lane
constexpr uint32_t kBlockRow = 1024 * kUnit;   // elements of a row that one block holds
constexpr int kSmallBlock = 256;     // threads where several rows share a block

// How a row is spread: `lanes` lanes per row (a power of two up to 32, or whole
// warps), `rows` rows per block of `threads` threads.
struct Spread {
  int lanes, rows, threads;
};
Spread spread_of(uint32_t dim) {
  const uint32_t units = (dim + kUnit - 1) / kUnit;
  Spread s{};
  if (units <= 32) {
    s.lanes = 1;
    while ((uint32_t)s.lanes < units) s.lanes *= 2;
    s.threads = kSmallBlock;
    s.rows = kSmallBlock / s.lanes;
  } else {
    s.lanes = s.threads = (int)((units + 31) / 32 * 32);
    s.rows = 1;
  }
  return s;
}

// Sums of two numbers over a row's lanes; `part` is shared memory of two
// float2 per warp, used in turn by successive calls (`turn` 0 and 1), so that
// one barrier a call is enough.
__device__ __forceinline__ float2 row_sum2(float a, float b, int lanes, float2 (*part)[32], int turn) {
  const int w = lanes < 32 ? lanes : 32;
  a = lanes_sum(a, w);
  b = lanes_sum(b, w);
  if (lanes <= 32) return make_float2(a, b);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = lanes >> 5;
  if (lane == 0) part[turn][warp] = make_float2(a, b);
  __syncthreads();
  const float2 v = lane < warps ? part[turn][lane] : make_float2(0.f, 0.f);
  return make_float2(lanes_sum(v.x, 32), lanes_sum(v.y, 32));
}

// Mean and sum of squared differences from it over a row's lanes.  Warps find
// both for their own elements first, so one exchange serves both: with n_w
// elements of mean m_w, the row's sum is sum S_w + sum n_w (m_w - m)^2.
template <int N>
__device__ __forceinline__ float2 row_moments(const float (&x)[N], const bool (&has)[N], float own, float warp_n, uint32_t dim,
                                              int lanes, float2 (*part)[32], int turn) {
  const int w = lanes < 32 ? lanes : 32;
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < N; ++j) s += x[j];   // (absent elements are zero)
  s = lanes_sum(s, w);
  const float mean_w = warp_n > 0.f ? s / warp_n : 0.f;
  float q = 0.f;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float d = has[j] ? x[j] - mean_w : 0.f;
    q = fmaf(d, d, q);
  }
  q = lanes_sum(q, w);
  if (lanes <= 32) return make_float2(mean_w, q);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = lanes >> 5;
  if (lane == 0) part[turn][warp] = make_float2(s, q);
  __syncthreads();
  const float2 v = lane < warps ? part[turn][lane] : make_float2(0.f, 0.f);
  const float mean = lanes_sum(v.x, 32) / (float)dim;
  // `own`: elements of the warp whose sums this lane looks at
  const float d = own > 0.f ? v.x / own - mean : 0.f;
  return make_float2(mean, lanes_sum(fmaf(own * d, d, v.y), 32));
}

// Elements of a row that warp `warp` of `lanes` holds, in accesses of VEC.
template <int VEC>
__device__ __forceinline__ float warp_elements(uint32_t dim, int lanes, int warp) {
  const int w = lanes < 32 ? lanes : 32;
  int n = 0;
#pragma unroll
  for (int i = 0; i < kUnit / VEC; ++i) {
    const int64_t first = ((int64_t)i * lanes + warp * w) * VEC;
    const int64_t left = (int64_t)dim - first;
    n += left <= 0 ? 0 : (left < w * VEC ? (int)left : w * VEC);
  }
  return (float)n;
}

// Lane `lane` of `lanes` holds elements ((j / VEC) * lanes + lane) * VEC + j % VEC.
// TYPE -1: types are known at run time alone.
template <int TYPE, int VEC>
__device__ __forceinline__ void load_row(const RowView& v, uint64_t row, uint32_t dim, int lane, int lanes, float (&x)[kUnit]) {
  const int type = TYPE < 0 ? v.type : TYPE;
  const char* p = v.data + row_offset(v, (uint32_t)row) * type_size(type);
#pragma unroll
  for (int i = 0; i < kUnit / VEC; ++i) {
    const uint32_t c = (uint32_t)(i * lanes + lane) * VEC;
    if (c < dim) {
      if constexpr (TYPE < 0) load_n_as<VEC>(p + (uint64_t)c * type_size(type), type, x + i * VEC);
      else load_n<TYPE, VEC>(p + (uint64_t)c * type_size(type), x + i * VEC);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[i * VEC + j] = 0.f;
    }
  }
}
template <int VEC>
__device__ __forceinline__ void store_row(const RowView& v, uint64_t row, uint32_t dim, int lane, int lanes, const float (&y)[kUnit]) {
  char* p = v.data + row_offset(v, (uint32_t)row) * type_size(v.type);
#pragma unroll
  for (int i = 0; i < kUnit / VEC; ++i) {
    const uint32_t c = (uint32_t)(i * lanes + lane) * VEC;
    if (c < dim) store_n_as<VEC>(p + (uint64_t)c * type_size(v.type), v.type, y + i * VEC);
  }
}
template <int VEC>
__device__ __forceinline__ void load_params(const VectorView& v, uint32_t dim, int lane, int lanes, float none, float (&w)[kUnit]) {
#pragma unroll
  for (int j = 0; j < kUnit; ++j) {
    const uint32_t c = (uint32_t)((j / VEC) * lanes + lane) * VEC + j % VEC;
    w[j] = v.data == nullptr ? none : (c < dim ? load_as(v.data, v.type, c) : 0.f);
  }
}

template <int TYPE, int VEC>
__global__ void __launch_bounds__(1024)
norm_kernel(const __grid_constant__ NormArgs a, int lanes) {
  after_previous();
  __shared__ float2 part[2][32];
  const int lane = threadIdx.x % lanes, group = threadIdx.x / lanes, rows = blockDim.x / lanes;
  float w[kUnit], b[kUnit];
  load_params<VEC>(a.weight, a.dim, lane, lanes, 1.f, w);
  load_params<VEC>(a.bias, a.dim, lane, lanes, 0.f, b);
  bool has[kUnit];
#pragma unroll
  for (int j = 0; j < kUnit; ++j) has[j] = (uint32_t)((j / VEC) * lanes + lane) * VEC + j % VEC < a.dim;
  const float mine = warp_elements<VEC>(a.dim, lanes, lane >> 5);
  const float own = (threadIdx.x & 31) * 32 < lanes ? warp_elements<VEC>(a.dim, lanes, threadIdx.x & 31) : 0.f;
  int turn = 0;
  // (the rows of a warp are taken together: a lane without a row follows with zeros)
  for (uint64_t r0 = (uint64_t)blockIdx.x * rows; r0 < a.n; r0 += (uint64_t)gridDim.x * rows, turn ^= 1) {
    const uint64_t row = r0 + group;
    const bool live = row < a.n;
    float x[kUnit];
    load_row<TYPE, VEC>(a.x, live ? row : r0, a.dim, lane, lanes, x);
    const float2 m = row_moments(x, has, own, mine, a.dim, lanes, part, turn);
    const float r = 1.f / sqrtf(m.y / (float)a.dim + a.eps);
    if (!live) continue;
#pragma unroll
    for (int j = 0; j < kUnit; ++j) x[j] = fmaf((x[j] - m.x) * r, w[j], b[j]);
    store_row<VEC>(a.out, row, a.dim, lane, lanes, x);
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
    float s = 0.f;
    for (uint32_t c = threadIdx.x; c < a.dim; c += 1024) s += load_as(x, a.x.type, c);
    const float mean = row_sum2(s, 0.f, 1024, part, 0).x / (float)a.dim;
    float q = 0.f;
    for (uint32_t c = threadIdx.x; c < a.dim; c += 1024) {
      const float d = load_as(x, a.x.type, c) - mean;
      q = fmaf(d, d, q);
    }
    const float r = 1.f / sqrtf(row_sum2(q, 0.f, 1024, part, 1).x / (float)a.dim + a.eps);
    for (uint32_t c = threadIdx.x; c < a.dim; c += 1024) {
      const float w = a.weight.data ? load_as(a.weight.data, a.weight.type, c) : 1.f;
      const float b = a.bias.data ? load_as(a.bias.data, a.bias.type, c) : 0.f;
      store_as(y, a.out.type, c, fmaf((load_as(x, a.x.type, c) - mean) * r, w, b));
    }
    if (a.stats != nullptr && threadIdx.x == 0) reinterpret_cast<float2*>(a.stats)[row] = make_float2(mean, r);
  }
}

// dx, and every block's sums of dy h and dy over its rows.
template <int TYPE, int VEC>
__global__ void __launch_bounds__(1024)
norm_grad_kernel(const __grid_constant__ NormArgs a, int lanes) {
  after_previous();
  __shared__ float2 part[2][32];
  __shared__ float sums[kSmallBlock * kUnit];
  const int lane = threadIdx.x % lanes, group = threadIdx.x / lanes, rows = blockDim.x / lanes;
  float w[kUnit], dw[kUnit], db[kUnit];
  load_params<VEC>(a.weight, a.dim, lane, lanes, 1.f, w);
#pragma unroll
  for (int j = 0; j < kUnit; ++j) dw[j] = db[j] = 0.f;
  const float inv = 1.f / (float)a.dim;
  int turn = 0;
  for (uint64_t r0 = (uint64_t)blockIdx.x * rows; r0 < a.n; r0 += (uint64_t)gridDim.x * rows, turn ^= 1) {
    const uint64_t row = r0 + group;
    const bool live = row < a.n;
    float x[kUnit], g[kUnit];
    load_row<TYPE, VEC>(a.x, live ? row : r0, a.dim, lane, lanes, x);
    load_row<TYPE, VEC>(a.grad, live ? row : r0, a.dim, lane, lanes, g);
    const float2 st = reinterpret_cast<const float2*>(a.stats)[live ? row : r0];
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int j = 0; j < kUnit; ++j) {
      const float h = (x[j] - st.x) * st.y;
      if (live) {
        dw[j] = fmaf(g[j], h, dw[j]);
        db[j] += g[j];
      }
      const float gw = g[j] * w[j];   // (zero where there is no element)
      s0 += gw;
      s1 = fmaf(gw, h, s1);
    }
    if (a.out.data == nullptr) continue;
    const float2 s = row_sum2(s0, s1, lanes, part, turn);
    if (!live) continue;
    const float c0 = s.x * inv, c1 = s.y * inv;
#pragma unroll
    for (int j = 0; j < kUnit; ++j) {
      const float h = (x[j] - st.x) * st.y;
      x[j] = st.y * (g[j] * w[j] - c0 - h * c1);
    }
    store_row<VEC>(a.out, row, a.dim, lane, lanes, x);
  }
  if (a.parts == nullptr) return;
  // the block's rows together, group after group
  float* out = a.parts + (uint64_t)blockIdx.x * 2 * a.dim;
  for (int which = 0; which < 2; ++which) {
    const float(&d)[kUnit] = which ? db : dw;
    if (lanes > 32) {   // one row at a time
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        const uint32_t c = (uint32_t)((j / VEC) * lanes + lane) * VEC + j % VEC;
        if (c < a.dim) out[which * a.dim + c] = d[j];
      }
      continue;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kUnit; ++j)
      sums[group * lanes * kUnit + ((j / VEC) * lanes + lane) * VEC + j % VEC] = d[j];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < a.dim; c += blockDim.x) {
      float s = 0.f;
      for (int g = 0; g < rows; ++g) s += sums[g * lanes * kUnit + c];
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
    float s0 = 0.f, s1 = 0.f;
    for (uint32_t c = threadIdx.x; c < a.dim; c += 1024) {
      const float gw = load_as(g, a.grad.type, c) * (a.weight.data ? load_as(a.weight.data, a.weight.type, c) : 1.f);
      s0 += gw;
      s1 = fmaf(gw, (load_as(x, a.x.type, c) - st.x) * st.y, s1);
    }
    const float2 s = row_sum2(s0, s1, 1024, part, turn);
    const float c0 = s.x / (float)a.dim, c1 = s.y / (float)a.dim;
    for (uint32_t c = threadIdx.x; c < a.dim; c += 1024) {
      const float gw = load_as(g, a.grad.type, c) * (a.weight.data ? load_as(a.weight.data, a.weight.type, c) : 1.f);
      const float h = (load_as(x, a.x.type, c) - st.x) * st.y;
      store_as(dx, a.out.type, c, st.y * (gw - c0 - h * c1));
    }
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
  for (uint64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
    const float2 st = reinterpret_cast<const float2*>(a.stats)[row];
    const float g = load_as(a.grad.data + row_offset(a.grad, (uint32_t)row) * type_size(a.grad.type), a.grad.type, c);
    const float x = load_as(a.x.data + row_offset(a.x, (uint32_t)row) * type_size(a.x.type), a.x.type, c);
    dw = fmaf(g, (x - st.x) * st.y, dw);
    db += g;
  }
  float* out = a.parts + (uint64_t)blockIdx.y * 2 * a.dim;
  out[c] = dw;
  out[a.dim + c] = db;
}

// The sums of `count` blocks, in a fixed order: 32 columns a block, every warp
// takes each 8th block's sums.
__global__ void __launch_bounds__(256)
norm_join_kernel(const float* parts, uint32_t count, uint32_t dim, VectorView dweight, VectorView dbias) {
  after_previous();
  __shared__ float sums[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t c = (uint64_t)blockIdx.x * 32 + lane;   // of 2 dim columns
  const uint64_t width = 2ull * dim;
  float s = 0.f;
  if (c < width)
    for (uint32_t p = warp; p < count; p += 8) s += parts[p * width + c];
  sums[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || c >= width) return;
  for (int w = 1; w < 8; ++w) s += sums[w][lane];
  const VectorView& v = c < dim ? dweight : dbias;
  if (v.data != nullptr) store_as(v.data, v.type, c < dim ? c : c - dim, s);
}

// Elements that every access of the vectors kernels takes: rows begin and end on a multiple of it.
template <class... V>
uint32_t width_of(const NormArgs& a, const V&... views) {
  const int type = a.x.type;
  for (uint32_t vec : {8u, 4u}) {
    if (type == ADAPM_F32 && vec == 8) continue;
    bool ok = a.dim % vec == 0;
    ((ok = ok && rows_on(views, a.n, vec)), ...);
    if (ok) return vec;
  }
  return 1;
}

unsigned grid_of(uint64_t n, const Spread& s, int sms, int threads_per_sm) {
  const uint64_t per_sm = std::min(32, std::max(1, threads_per_sm / s.threads));
  return (unsigned)std::max<uint64_t>(1, std::min<uint64_t>((n + s.rows - 1) / s.rows, (uint64_t)sms * per_sm));
}

constexpr int kNormThreads = 1536, kNormGradThreads = 1024;   // per SM
constexpr int kLongRows = 64;   // row classes of norm_columns_kernel

bool long_rows(const NormArgs& a) { return a.dim > kBlockRow; }
uint64_t part_count(const NormArgs& a, int sms) {
  if (long_rows(a)) return std::min<uint64_t>(a.n, kLongRows);
  return grid_of(a.n, spread_of(a.dim), sms, kNormGradThreads);
}

template <int TYPE>
void launch_norm_type(const NormArgs& a, uint32_t vec, const Spread& s, unsigned grid, cudaStream_t stream) {
  if (vec == 8) {
    if constexpr (TYPE != ADAPM_F32) launch_after(norm_kernel<TYPE, 8>, grid, s.threads, 0, stream, a, s.lanes);
  } else {
    launch_after(norm_kernel<TYPE, 4>, grid, s.threads, 0, stream, a, s.lanes);
  }
}
template <int TYPE>
void launch_grad_type(const NormArgs& a, uint32_t vec, const Spread& s, unsigned grid, cudaStream_t stream) {
  if (vec == 8) {
    if constexpr (TYPE != ADAPM_F32) launch_after(norm_grad_kernel<TYPE, 8>, grid, s.threads, 0, stream, a, s.lanes);
  } else {
    launch_after(norm_grad_kernel<TYPE, 4>, grid, s.threads, 0, stream, a, s.lanes);
  }
}

}  // namespace

void launch_layer_norm(const NormArgs& a, int sms, cudaStream_t stream) {
  note_launches(1);
  if (long_rows(a)) {
    launch_after(norm_long_kernel, (unsigned)std::min<uint64_t>(a.n, (uint64_t)sms * 2), 1024, 0, stream, a);
    return;
  }
  const Spread s = spread_of(a.dim);
  const unsigned grid = grid_of(a.n, s, sms, kNormThreads);
  const uint32_t vec = width_of(a, a.x, a.out);
  if (vec == 1) launch_after(norm_kernel<-1, 1>, grid, s.threads, 0, stream, a, s.lanes);
  else if (a.x.type == ADAPM_F32) launch_norm_type<ADAPM_F32>(a, vec, s, grid, stream);
  else if (a.x.type == ADAPM_F16) launch_norm_type<ADAPM_F16>(a, vec, s, grid, stream);
  else launch_norm_type<ADAPM_BF16>(a, vec, s, grid, stream);
}

size_t norm_grad_scratch(const NormArgs& a, int sms) {
  return a.dweight.data || a.dbias.data ? part_count(a, sms) * 2 * a.dim : 0;
}

void launch_layer_norm_grad(const NormArgs& a, int sms, cudaStream_t stream) {
  const uint64_t count = part_count(a, sms);
  if (long_rows(a)) {
    if (a.parts != nullptr) {
      note_launches(1);
      // (the grid has two dimensions: launched plainly)
      norm_columns_kernel<<<dim3((a.dim + 255) / 256, (unsigned)count), 256, 0, stream>>>(a);
    }
    if (a.out.data != nullptr) {
      note_launches(1);
      launch_after(norm_grad_long_kernel, (unsigned)std::min<uint64_t>(a.n, (uint64_t)sms * 2), 1024, 0, stream, a);
    }
  } else {
    const Spread s = spread_of(a.dim);
    uint32_t vec = a.grad.type != a.x.type ? 1 : (a.out.data ? width_of(a, a.x, a.grad, a.out) : width_of(a, a.x, a.grad));
    note_launches(1);
    if (vec == 1) launch_after(norm_grad_kernel<-1, 1>, (unsigned)count, s.threads, 0, stream, a, s.lanes);
    else if (a.x.type == ADAPM_F32) launch_grad_type<ADAPM_F32>(a, vec, s, (unsigned)count, stream);
    else if (a.x.type == ADAPM_F16) launch_grad_type<ADAPM_F16>(a, vec, s, (unsigned)count, stream);
    else launch_grad_type<ADAPM_BF16>(a, vec, s, (unsigned)count, stream);
  }
  if (a.parts != nullptr) {
    note_launches(1);
    launch_after(norm_join_kernel, (unsigned)((2ull * a.dim + 31) / 32), 256, 0, stream, (const float*)a.parts, (uint32_t)count, a.dim,
                 a.dweight, a.dbias);
  }
}

}  // namespace adapm
