// Dense layers: products with bias, activation and residual, and their gradients.
//
//   z = x w + b,  out = act(z) + residual
//   dz = grad act'(z),  dx = dz w^T,  dw = x^T dz,  db = sum over rows of dz
//
// All three products run in one kernel on the tensor cores: tiles of 128 x bn,
// operands copied by the tensor memory accelerator into a ring of swizzled
// blocks of 64 k, sums in tensor memory (two accumulators, so that one tile's
// epilogue runs beside the next one's products), one warp that issues copies,
// one that issues products, four for the epilogue.  Operands are taken as they
// lie in memory, with k contiguous or across it; what the accelerator cannot
// address (rows that do not begin on 16 bytes) is copied first.
// Bound by the tensor cores where all three sizes are large, by memory where
// one is small: then k is summed in parts, so that every SM reads.
#include <algorithm>
#include <cmath>

#include "gemm.cuh"

namespace adapm {

namespace {

constexpr int kGemmThreads = 192;
constexpr uint32_t kMaxStages = 12;
constexpr uint32_t kStage = 32 * 36;        // floats of a warp's staging tile (rows of 32, apart by 36)
constexpr uint32_t kSmem = 232448;          // shared memory of a block
constexpr uint32_t kGroupM = 16;            // tiles of m taken together, for L2
constexpr uint32_t kTurnedRows = 64;        // up to so many rows the weight's columns are m

// ---- activations -----------------------------------------------------------------
__device__ __forceinline__ float act(float z, int kind) {
  switch (kind) {
    case ADAPM_ACTIVATION_RELU: return fmaxf(z, 0.f) + (z != z ? z : 0.f);   // (a NaN stays one)
    case ADAPM_ACTIVATION_GELU: return 0.5f * z * (1.f + erff(z * 0.70710678f));
    case ADAPM_ACTIVATION_GELU_TANH: return 0.5f * z * (1.f + tanhf(0.79788456f * (z + 0.044715f * z * z * z)));
    case ADAPM_ACTIVATION_SILU: return z / (1.f + expf(-z));
    case ADAPM_ACTIVATION_TANH: return tanhf(z);
    default: return z;
  }
}
__device__ __forceinline__ float slope(float z, int kind) {
  switch (kind) {
    case ADAPM_ACTIVATION_RELU: return z > 0.f ? 1.f : (z != z ? z : 0.f);
    case ADAPM_ACTIVATION_GELU: return 0.5f * (1.f + erff(z * 0.70710678f)) + z * 0.39894228f * expf(-0.5f * z * z);
    case ADAPM_ACTIVATION_GELU_TANH: {
      const float t = tanhf(0.79788456f * (z + 0.044715f * z * z * z));
      return 0.5f * (1.f + t) + 0.5f * z * (1.f - t * t) * 0.79788456f * (1.f + 0.134145f * z * z);
    }
    case ADAPM_ACTIVATION_SILU: {
      const float s = 1.f / (1.f + expf(-z));
      return s * (1.f + z * (1.f - s));
    }
    case ADAPM_ACTIVATION_TANH: {
      const float t = tanhf(z);
      return 1.f - t * t;
    }
    default: return 1.f;
  }
}

// One element of a product.
__device__ __forceinline__ void finish_one(const Epilogue& e, uint64_t r, uint64_t c, float z) {
  if (e.bias.data) z += load_as(e.bias.data, e.bias.type, c);
  if (e.pre.data) store_as(e.pre.data, e.pre.type, r * e.pre.row_stride + c, z);
  z = act(z, e.activation);
  if (e.residual.data) z += load_as(e.residual.data, e.residual.type, r * e.residual.row_stride + c);
  store_as(e.out.data, e.out.type, r * e.out.row_stride + c, z);
}
// Four neighbours of a row, on addresses that are multiples of four elements.
__device__ __forceinline__ void finish_four(const Epilogue& e, uint64_t r, uint64_t c, float (&z)[4], const float (&bias)[4]) {
  float add[4] = {0.f, 0.f, 0.f, 0.f};
  if (e.residual.data) load_n_as<4>(e.residual.data + (r * e.residual.row_stride + c) * type_size(e.residual.type), e.residual.type, add);
#pragma unroll
  for (int j = 0; j < 4; ++j) z[j] += bias[j];
  if (e.pre.data) store_n_as<4>(e.pre.data + (r * e.pre.row_stride + c) * type_size(e.pre.type), e.pre.type, z);
#pragma unroll
  for (int j = 0; j < 4; ++j) z[j] = act(z[j], e.activation) + add[j];
  store_n_as<4>(e.out.data + (r * e.out.row_stride + c) * type_size(e.out.type), e.out.type, z);
}

// ---- the product -------------------------------------------------------------------
struct Item {
  uint32_t m0, n0, k0, k1, split;
};
__device__ __forceinline__ Item item_of(const GemmArgs& g, uint32_t i) {
  Item t;
  const uint32_t tiles = g.tiles_m * g.tiles_n;
  t.split = i / tiles;
  const uint32_t tile = i - t.split * tiles;
  // groups of kGroupM tiles of m, n by n inside
  const uint32_t in_group = kGroupM * g.tiles_n, group = tile / in_group, at = tile - group * in_group;
  const uint32_t height = min(kGroupM, g.tiles_m - group * kGroupM);
  t.m0 = (group * kGroupM + at % height) * kTileM;
  t.n0 = at / height * g.bn;
  t.k0 = t.split * g.per_split;
  t.k1 = min(g.k_blocks, t.k0 + g.per_split);
  return t;
}

__global__ void __launch_bounds__(kGemmThreads, 1)
gemm_kernel(const __grid_constant__ GemmArgs g, bool aligned) {
  extern __shared__ uint8_t smem[];
  __shared__ uint64_t bars[2 * kMaxStages + 4];
  __shared__ uint32_t tmem_at;
  __shared__ uint32_t gave_up;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t a_bytes = kTileM * 128, stage_bytes = a_bytes + g.bn * 128;
  const uint32_t ring = (shared_at(smem) + 1023u) & ~1023u;
  float* const staging = reinterpret_cast<float*>(smem + (ring - shared_at(smem)) + g.stages * stage_bytes);
  const uint32_t full = shared_at(bars), empty = full + 8 * kMaxStages, sum_full = empty + 8 * kMaxStages, sum_empty = sum_full + 16;
  const uint32_t columns = 2 * max(16u, g.bn) <= 32 ? 32 : 2 * g.bn;   // (bn is a power of two)
  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < g.stages; ++s) {
      barrier_init(full + 8 * s, 1);
      barrier_init(empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      barrier_init(sum_full + 8 * b, 1);
      barrier_init(sum_empty + 8 * b, 4);
    }
    gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_take(&tmem_at, columns);
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  after_previous();
  const uint32_t tmem = tmem_at;
  const uint32_t items = g.tiles_m * g.tiles_n * g.splits;
  if (warp == 0) {
    if (lane == 0) {
      asm volatile("fence.proxy.async;" ::: "memory");
      uint32_t n = 0, stage = 0, parity = 1;   // copies issued; a fresh ring is empty
      bool ok = true;
      for (uint32_t i = blockIdx.x; i < items && ok; i += gridDim.x) {
        const Item t = item_of(g, i);
        for (uint32_t k = t.k0; k < t.k1; ++k) {
          if (!(ok = barrier_wait(empty + 8 * stage, parity))) break;
          const uint32_t bar = full + 8 * stage, at = ring + stage * stage_bytes;
          barrier_expect(bar, stage_bytes);
          if (!g.a_across) {
            copy_tile(at, &g.a, (int)(k * kBlockK), (int)t.m0, bar);
          } else {
            for (uint32_t j = 0; j < kTileM; j += 64) copy_tile(at + j * 128, &g.a, (int)(t.m0 + j), (int)(k * kBlockK), bar);
          }
          if (!g.b_across) {
            copy_tile(at + a_bytes, &g.b, (int)(k * kBlockK), (int)t.n0, bar);
          } else {
            for (uint32_t j = 0; j < g.bn; j += 64) copy_tile(at + a_bytes + j * 128, &g.b, (int)(t.n0 + j), (int)(k * kBlockK), bar);
          }
          ++n;
          if (++stage == g.stages) {
            stage = 0;
            parity ^= 1u;
          }
        }
      }
      if (!ok) {
        atomicExch(&gave_up, 1u);
        // copies in flight land before the block ends
        for (uint32_t j = n > g.stages ? n - g.stages : 0; j < n; ++j)
          if (!barrier_wait(full + 8 * (j % g.stages), (j / g.stages) & 1u)) break;
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t shape = mma_shape(g.bf16, g.a_across, g.b_across, g.bn);
      const uint32_t a_step = tile_step(g.a_across), b_step = tile_step(g.b_across);
      uint32_t stage = 0, parity = 0, turn = 0;
      bool ok = true;
      for (uint32_t i = blockIdx.x; i < items && ok; i += gridDim.x, ++turn) {
        const Item t = item_of(g, i);
        const uint32_t b = turn & 1u;
        if (!(ok = barrier_wait(sum_empty + 8 * b, ((turn >> 1) & 1u) ^ 1u))) break;
        tmem_fence_after();
        for (uint32_t k = t.k0; k < t.k1; ++k) {
          if (!(ok = barrier_wait(full + 8 * stage, parity))) break;
          tmem_fence_after();
          const uint32_t at = ring + stage * stage_bytes;
          const uint64_t da = tile_descriptor(at, g.a_across), db = tile_descriptor(at + a_bytes, g.b_across);
#pragma unroll
          for (uint32_t j = 0; j < kBlockK / 16; ++j)
            mma(tmem + b * g.bn, da + j * a_step, db + j * b_step, shape, k > t.k0 || j > 0);
          mma_commit(empty + 8 * stage);
          if (++stage == g.stages) {
            stage = 0;
            parity ^= 1u;
          }
        }
        mma_commit(sum_full + 8 * b);
      }
      if (!ok) atomicExch(&gave_up, 1u);
    }
  } else {
    const uint32_t quarter = (uint32_t)warp & 3u;   // of the rows of tensor memory that this warp reaches
    float* const tile = staging + (warp - 2) * kStage;
    uint32_t turn = 0;
    for (uint32_t i = blockIdx.x; i < items; i += gridDim.x, ++turn) {
      const Item t = item_of(g, i);
      const uint32_t b = turn & 1u;
      if (!barrier_wait(sum_full + 8 * b, (turn >> 1) & 1u)) {
        if (lane == 0) atomicExch(&gave_up, 1u);
        break;
      }
      __syncwarp();
      tmem_fence_after();
      const uint32_t from = tmem + ((quarter * 32u) << 16) + b * g.bn;
      const uint32_t m1 = t.m0 + quarter * 32;   // the warp's first row
      float* const part = g.splits > 1 ? g.parts + (uint64_t)t.split * g.m * g.n : nullptr;
      if (g.turned) {
        // lanes are neighbours in the product's rows
        for (uint32_t c0 = 0; c0 < g.bn; c0 += 16) {
          float v[16];
          __syncwarp();
          tmem_load16(from + c0, v);
          const uint64_t c = m1 + lane;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const uint64_t r = t.n0 + c0 + j;
            if (c >= g.m || r >= g.n) continue;
            if (part) part[r * g.m + c] = v[j];
            else finish_one(g.e, r, c, v[j]);
          }
        }
      } else {
        for (uint32_t c0 = 0; c0 < g.bn && t.n0 + c0 < g.n; c0 += 32) {
          float v[32];
          __syncwarp();
          tmem_load(from + c0, v);
          // through shared memory, so that neighbouring lanes hold neighbouring columns
#pragma unroll
          for (int j = 0; j < 32; j += 4)
            *reinterpret_cast<float4*>(tile + lane * 36 + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
          __syncwarp();
          const uint32_t c = t.n0 + c0 + (lane & 7) * 4;
          float bias[4] = {0.f, 0.f, 0.f, 0.f};
          if (!part && g.e.bias.data)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (c + j < g.n) bias[j] = load_as(g.e.bias.data, g.e.bias.type, c + j);
          for (int p = 0; p < 8; ++p) {
            const uint32_t row = p * 4 + (lane >> 3);
            const uint64_t r = m1 + row;
            const float4 q = *reinterpret_cast<const float4*>(tile + row * 36 + (lane & 7) * 4);
            if (r >= g.m) break;
            float z[4] = {q.x, q.y, q.z, q.w};
            if (aligned && c + 4 <= g.n) {
              if (part) *reinterpret_cast<float4*>(part + r * g.n + c) = q;
              else finish_four(g.e, r, c, z, bias);
            } else {
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if (c + j >= g.n) break;
                if (part) part[r * g.n + c + j] = z[j];
                else finish_one(g.e, r, c + j, z[j]);
              }
            }
          }
        }
      }
      tmem_fence_before();
      __syncwarp();
      if (lane == 0) barrier_arrive(sum_empty + 8 * b);
    }
  }
  __syncwarp();
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  if (threadIdx.x == 0 && gave_up) set_error(g.st, ERR_TIMEOUT);
  if (warp == 1) tmem_give(tmem, columns);
}

// The parts of a product of rows x columns, in order, and what becomes of their sum.
__global__ void __launch_bounds__(256)
gemm_join_kernel(const float* parts, uint32_t splits, uint64_t rows, uint32_t columns, const __grid_constant__ Epilogue e) {
  after_previous();
  const uint64_t count = rows * columns;
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (uint64_t)gridDim.x * 256) {
    float z = 0.f;
    for (uint32_t s = 0; s < splits; ++s) z += parts[s * count + i];
    const uint64_t r = i / columns;
    finish_one(e, r, i - r * columns, z);
  }
}

// ---- operands ------------------------------------------------------------------------
// rows x columns elements of a 16-bit type to rows without gaps but for `pitch`.
__global__ void __launch_bounds__(256)
pack_kernel(const uint16_t* from, int64_t row_stride, int64_t col_stride, uint16_t* to, uint64_t rows, uint32_t columns, uint32_t pitch) {
  after_previous();
  for (uint64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (uint32_t c = threadIdx.x; c < columns; c += 256) to[r * pitch + c] = from[(int64_t)r * row_stride + (int64_t)c * col_stride];
}

// A matrix of mn x k elements as an operand: how it is stored, and whether it
// has to be copied for that.
struct Operand {
  const char* data;
  uint64_t mn;
  uint32_t k;
  int64_t mn_stride, k_stride;
  bool across;      // mn contiguous
  bool packed;
  uint64_t pitch;   // elements from one row (k: across) to the next
  size_t bytes;     // of the copy
};
Operand operand(const char* data, uint64_t mn, uint32_t k, int64_t mn_stride, int64_t k_stride, bool along_k_only) {
  Operand o{data, mn, k, mn_stride, k_stride, false, false, 0, 0};
  // (rows that overlap each other are copied too)
  auto fits = [&](int64_t one, int64_t step, uint64_t steps, uint64_t width) {
    return one == 1 && (steps <= 1 || (step >= (int64_t)width && step % 8 == 0 && step < (1ll << 38))) &&
           reinterpret_cast<uintptr_t>(data) % 16 == 0;
  };
  const uint64_t k8 = ((uint64_t)k + 7) / 8 * 8, mn8 = (mn + 7) / 8 * 8;
  // (a row of one element has any stride)
  const int64_t k_one = k <= 1 ? 1 : k_stride, mn_one = mn <= 1 ? 1 : mn_stride;
  if (fits(k_one, mn_stride, mn, k)) {
    o.pitch = mn <= 1 ? k8 : (uint64_t)mn_stride;
  } else if (!along_k_only && fits(mn_one, k_stride, k, mn)) {
    o.across = true;
    o.pitch = k <= 1 ? mn8 : (uint64_t)k_stride;
  } else {
    o.packed = true;
    o.across = !along_k_only && k_one != 1 && mn_one == 1;
    o.pitch = o.across ? mn8 : k8;
    o.bytes = (o.across ? k : mn) * o.pitch * 2;
  }
  return o;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// Copies the operand to `at` if it has to be; returns what it takes there.
size_t pack(Operand& o, char* at, int sms, cudaStream_t stream) {
  if (!o.packed) return 0;
  const uint64_t rows = o.across ? o.k : o.mn;
  const uint32_t columns = (uint32_t)(o.across ? o.mn : o.k);
  note_launches(1);
  launch_after(pack_kernel, (unsigned)std::min<uint64_t>(rows, (uint64_t)sms * 8), 256, 0, stream,
               reinterpret_cast<const uint16_t*>(o.data), o.across ? o.k_stride : o.mn_stride, o.across ? o.mn_stride : o.k_stride,
               reinterpret_cast<uint16_t*>(at), rows, columns, (uint32_t)o.pitch);
  o.data = at;
  return round256(o.bytes);
}

// The tensor map of an operand whose tiles have `height` rows of mn.
cudaError_t tensor_map(const Operand& o, bool bf16, uint32_t height, CUtensorMap* map) {
  using Fn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                          const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                          CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Fn encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult got;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &got) != cudaSuccess ||
        got != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      f = nullptr;
    }
    return reinterpret_cast<Fn>(f);
  }();
  if (!encode) return cudaErrorNotSupported;
  const cuuint64_t size[2] = {o.across ? o.mn : o.k, o.across ? o.k : o.mn};
  const cuuint64_t stride[1] = {o.pitch * 2};
  const cuuint32_t box[2] = {kBlockK, o.across ? kBlockK : height}, step[2] = {1, 1};
  const CUresult r = encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                            const_cast<char*>(o.data), size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// ---- sizes of a product -----------------------------------------------------------------
struct GemmPlan {
  bool turned;
  uint32_t bn, tiles_m, tiles_n, k_blocks, splits, per_split, stages;
  size_t part_bytes;
};
// The product of `rows` x `columns` elements over k.
GemmPlan gemm_plan(uint64_t rows, uint32_t columns, uint64_t k, int sms) {
  GemmPlan p{};
  p.turned = rows <= kTurnedRows;
  const uint64_t m = p.turned ? columns : rows, n = p.turned ? rows : columns;
  if (p.turned) p.bn = n <= 16 ? 16 : (n <= 32 ? 32 : 64);
  else p.bn = n <= 64 ? 64 : (n <= 128 ? 128 : 256);
  p.tiles_m = (uint32_t)((m + kTileM - 1) / kTileM);
  // narrower tiles while there are too few for every SM
  while (!p.turned && p.bn > 64 && (uint64_t)p.tiles_m * ((n + p.bn - 1) / p.bn) < (uint64_t)sms) p.bn /= 2;
  p.tiles_n = (uint32_t)((n + p.bn - 1) / p.bn);
  p.k_blocks = (uint32_t)((k + kBlockK - 1) / kBlockK);
  // parts of k, of at least four blocks, while SMs are idle
  const uint64_t tiles = (uint64_t)p.tiles_m * p.tiles_n;
  const uint64_t want = std::max<uint64_t>(1, std::min<uint64_t>((uint64_t)sms / tiles, p.k_blocks / 4));
  p.per_split = (uint32_t)((p.k_blocks + want - 1) / want);
  p.splits = (p.k_blocks + p.per_split - 1) / p.per_split;
  p.part_bytes = p.splits > 1 ? (size_t)p.splits * rows * columns * sizeof(float) : 0;
  const uint32_t stage = kTileM * 128 + p.bn * 128;
  p.stages = std::min(kMaxStages, (kSmem - 1024 - 512 - 4 * kStage * (uint32_t)sizeof(float)) / stage);
  return p;
}

bool on_four(const MatrixView& v, uint64_t rows) {
  return v.data == nullptr || (reinterpret_cast<uintptr_t>(v.data) % (4 * type_size(v.type)) == 0 && (rows <= 1 || v.row_stride % 4 == 0));
}

// rows x columns = left (rows x k) right (k x columns); `at`: scratch for the parts.
cudaError_t launch_gemm(const GemmPlan& p, const Operand& left, const Operand& right, bool bf16, const Epilogue& e, char* at,
                        DevState* st, int sms, cudaStream_t stream) {
  GemmArgs g{};
  const Operand& a = p.turned ? right : left;
  const Operand& b = p.turned ? left : right;
  cudaError_t err = tensor_map(a, bf16, kTileM, &g.a);
  if (err == cudaSuccess) err = tensor_map(b, bf16, p.bn, &g.b);
  if (err != cudaSuccess) return err;
  g.a_across = a.across;
  g.b_across = b.across;
  g.turned = p.turned;
  g.m = (uint32_t)a.mn;
  g.n = (uint32_t)b.mn;
  g.bn = p.bn;
  g.stages = p.stages;
  g.tiles_m = p.tiles_m;
  g.tiles_n = p.tiles_n;
  g.k_blocks = p.k_blocks;
  g.splits = p.splits;
  g.per_split = p.per_split;
  g.bf16 = bf16;
  g.parts = p.splits > 1 ? reinterpret_cast<float*>(at) : nullptr;
  g.e = e;
  g.st = st;
  const uint64_t rows = left.mn;
  const uint32_t columns = (uint32_t)right.mn;
  const bool aligned = p.splits > 1 ? columns % 4 == 0
                                    : on_four(e.out, rows) && on_four(e.pre, rows) && on_four(e.residual, rows);
  const size_t smem = 1024 + (size_t)p.stages * (kTileM + p.bn) * 128 + 4 * kStage * sizeof(float);
  err = cudaFuncSetAttribute(gemm_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kSmem - 1024));
  if (err != cudaSuccess) return err;
  const uint64_t items = (uint64_t)p.tiles_m * p.tiles_n * p.splits;
  note_launches(1);
  launch_after(gemm_kernel, (unsigned)std::min<uint64_t>(items, (uint64_t)sms), kGemmThreads, smem, stream, g, aligned);
  if (p.splits > 1) {
    note_launches(1);
    launch_after(gemm_join_kernel, (unsigned)std::min<uint64_t>((rows * columns + 255) / 256, (uint64_t)sms * 8), 256, 0, stream,
                 (const float*)g.parts, p.splits, rows, columns, e);
  }
  return cudaSuccess;
}

// ---- the gradient of z ----------------------------------------------------------------------
// dz = grad act'(pre) to rows of `pitch` elements (to null: grad itself serves),
// and sums of its columns over every gridDim.y-th group of 8 rows.
__global__ void __launch_bounds__(256)
dz_kernel(const MatrixView grad, const MatrixView pre, int activation, char* to, uint32_t pitch, uint64_t rows, uint32_t columns, float* parts) {
  after_previous();
  __shared__ float sums[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t c = (uint64_t)blockIdx.x * 32 + lane;
  float sum = 0.f;
  if (c < columns)
    for (uint64_t r = (uint64_t)blockIdx.y * 8 + warp; r < rows; r += (uint64_t)gridDim.y * 8) {
      float d = load_as(grad.data, grad.type, (int64_t)r * grad.row_stride + (int64_t)c * grad.col_stride);
      if (activation != ADAPM_ACTIVATION_NONE)
        d *= slope(load_as(pre.data, pre.type, (int64_t)r * pre.row_stride + (int64_t)c * pre.col_stride), activation);
      if (to != nullptr) store_as(to, grad.type, r * pitch + c, d);
      sum += d;
    }
  if (parts == nullptr) return;
  sums[warp][lane] = sum;
  __syncthreads();
  if (warp != 0 || c >= columns) return;
  for (int w = 1; w < 8; ++w) sum += sums[w][lane];
  parts[blockIdx.y * (uint64_t)columns + c] = sum;
}
__global__ void __launch_bounds__(256)
bias_join_kernel(const float* parts, uint32_t count, uint32_t columns, VectorView out) {
  after_previous();
  const uint64_t c = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= columns) return;
  float s = 0.f;
  for (uint32_t p = 0; p < count; ++p) s += parts[p * (uint64_t)columns + c];
  store_as(out.data, out.type, c, s);
}

bool by_rows(const MatrixView& m, uint64_t rows, uint32_t columns) {   // stored with a row's elements contiguous
  return columns <= 1 || m.col_stride == 1 || !(rows <= 1 || m.row_stride == 1);
}

}  // namespace

size_t linear_scratch(const LinearArgs& a, int sms) {
  const GemmPlan p = gemm_plan(a.rows, a.outs, a.ins, sms);
  const Operand x = operand(a.x.data, a.rows, a.ins, a.x.row_stride, a.x.col_stride, p.turned);
  const Operand w = operand(a.weight.data, a.outs, a.ins, a.weight.col_stride, a.weight.row_stride, false);
  return round256(x.bytes) + round256(w.bytes) + p.part_bytes;
}

cudaError_t launch_linear(const LinearArgs& a, char* scratch, int sms, cudaStream_t stream) {
  const GemmPlan p = gemm_plan(a.rows, a.outs, a.ins, sms);
  Operand x = operand(a.x.data, a.rows, a.ins, a.x.row_stride, a.x.col_stride, p.turned);
  Operand w = operand(a.weight.data, a.outs, a.ins, a.weight.col_stride, a.weight.row_stride, false);
  scratch += pack(x, scratch, sms, stream);
  scratch += pack(w, scratch, sms, stream);
  const Epilogue e{a.bias, a.residual, a.out, a.pre, a.activation};
  return launch_gemm(p, x, w, a.x.type == ADAPM_BF16, e, scratch, a.st, sms, stream);
}

namespace {

// What the backward pass needs: dz (its own, or grad), the operands of both
// products, and their scratch, one after the other.
struct Backward {
  bool own_dz;
  uint32_t pitch, chunks;
  MatrixView dz;
  bool across_out;   // dweight is stored by output: its transpose is computed
  size_t dz_bytes, sum_bytes;
};
constexpr uint32_t kRowChunks = 64;
Backward backward_of(const LinearArgs& a, char* scratch) {
  Backward b{};
  b.own_dz = a.activation != ADAPM_ACTIVATION_NONE && (a.dx.data || a.dweight.data);
  b.pitch = (a.outs + 7) / 8 * 8;
  b.dz_bytes = b.own_dz ? round256(a.rows * (size_t)b.pitch * 2) : 0;
  b.chunks = (uint32_t)std::min<uint64_t>((a.rows + 7) / 8, kRowChunks);
  b.sum_bytes = a.dbias.data ? round256((size_t)b.chunks * a.outs * sizeof(float)) : 0;
  b.dz = b.own_dz ? MatrixView{scratch, a.grad.type, (int64_t)b.pitch, 1} : a.grad;
  b.across_out = a.dweight.data && !by_rows(a.dweight, a.ins, a.outs);
  return b;
}
struct Product {
  GemmPlan p;
  Operand left, right;
  size_t bytes() const { return round256(left.bytes) + round256(right.bytes) + round256(p.part_bytes); }
};
Product dx_product(const LinearArgs& a, const Backward& b, int sms) {   // rows x ins over outs
  Product q;
  q.p = gemm_plan(a.rows, a.ins, a.outs, sms);
  q.left = operand(b.dz.data, a.rows, a.outs, b.dz.row_stride, b.dz.col_stride, q.p.turned);
  q.right = operand(a.weight.data, a.ins, a.outs, a.weight.row_stride, a.weight.col_stride, false);
  return q;
}
Product dweight_product(const LinearArgs& a, const Backward& b, int sms) {   // ins x outs over rows, or its transpose
  Product q;
  const uint32_t k = (uint32_t)a.rows;
  q.p = b.across_out ? gemm_plan(a.outs, a.ins, k, sms) : gemm_plan(a.ins, a.outs, k, sms);
  const bool turned = q.p.turned;
  const Operand x = operand(a.x.data, a.ins, k, a.x.col_stride, a.x.row_stride, turned && !b.across_out);
  const Operand d = operand(b.dz.data, a.outs, k, b.dz.col_stride, b.dz.row_stride, turned && b.across_out);
  q.left = b.across_out ? d : x;
  q.right = b.across_out ? x : d;
  return q;
}

}  // namespace

size_t linear_grad_scratch(const LinearArgs& a, int sms) {
  const Backward b = backward_of(a, nullptr);
  size_t most = 0;   // (the products follow each other: they share)
  if (a.dx.data) most = std::max(most, dx_product(a, b, sms).bytes());
  if (a.dweight.data) most = std::max(most, dweight_product(a, b, sms).bytes());
  return b.dz_bytes + b.sum_bytes + most;
}

cudaError_t launch_linear_grad(const LinearArgs& a, char* scratch, int sms, cudaStream_t stream) {
  const Backward b = backward_of(a, scratch);
  float* const sums = a.dbias.data ? reinterpret_cast<float*>(scratch + b.dz_bytes) : nullptr;
  char* const rest = scratch + b.dz_bytes + b.sum_bytes;
  const bool bf16 = a.x.type == ADAPM_BF16;
  if (b.own_dz || a.dbias.data) {
    note_launches(1);
    // (the grid has two dimensions: launched plainly)
    dz_kernel<<<dim3((a.outs + 31) / 32, b.chunks), 256, 0, stream>>>(a.grad, a.pre, a.activation, b.own_dz ? b.dz.data : nullptr,
                                                                      b.pitch, a.rows, a.outs, sums);
  }
  if (a.dbias.data) {
    note_launches(1);
    launch_after(bias_join_kernel, (a.outs + 255) / 256, 256, 0, stream, (const float*)sums, b.chunks, a.outs, a.dbias);
  }
  for (int which = 0; which < 2; ++which) {
    if ((which ? a.dweight.data : a.dx.data) == nullptr) continue;
    Product q = which ? dweight_product(a, b, sms) : dx_product(a, b, sms);
    char* at = rest;
    at += pack(q.left, at, sms, stream);
    at += pack(q.right, at, sms, stream);
    Epilogue e{};
    e.out = which ? a.dweight : a.dx;
    if (which && b.across_out) std::swap(e.out.row_stride, e.out.col_stride);
    const cudaError_t err = launch_gemm(q.p, q.left, q.right, bf16, e, at, a.st, sms, stream);
    if (err != cudaSuccess) return err;
  }
  return cudaSuccess;
}

}  // namespace adapm
