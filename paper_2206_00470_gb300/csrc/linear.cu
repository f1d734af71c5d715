// Dense layers: products with bias, activation and residual, and their gradients.
//
//   z = x w + b,  out = act(z) + residual
//   dz = grad act'(z),  dx = dz w^T,  dw = x^T dz,  db = sum over rows of dz
//
// All three products run in one kernel on the tensor cores: tiles of 128 x bn,
// operands copied by the tensor memory accelerator into a ring of swizzled
// blocks of 64 k, sums in tensor memory (two accumulators, so that one tile's
// epilogue runs beside the next one's products), one warp that issues copies,
// one that issues products, eight for the epilogue.  Large products are taken
// by pairs of blocks, 256 x 256 a tile.  Operands are taken as they lie in
// memory, with k contiguous or across it; what the accelerator cannot address
// (rows that do not begin on 16 bytes) is copied first.  Up to 64 rows are the
// columns of a tile whose rows are the weight's columns.
// Bound by the tensor cores where all three sizes are large, by memory where
// one is small: then k is summed in parts, so that every SM reads.  bf16, 8192
// x 4096 x 8192 with bias, activation, z kept and residual 362 to 379 us, 1.5
// PFLOP/s (320 us alone, 1.7; at full power the clock falls); gradients of 8192
// x 4096 x 4096 390 us, of which dz 36; one row by 4096 x 4096 9 us, 3.7 TB/s.
// Logits of 4092 x 1024 by 50,021 words 345 us (226 at the tensor cores' rate), of
// one row 27 (15 at the memory's).
#include <cooperative_groups.h>

#include <algorithm>

#include "gemm.cuh"

namespace adapm {

namespace {

namespace cg = cooperative_groups;

constexpr int kFinishWarps = 8, kGemmThreads = 32 * (2 + kFinishWarps);
constexpr uint32_t kMaxStages = 12;
constexpr uint32_t kStage = 32 * 36;        // floats of a warp's staging tile (rows of 32, apart by 36)
constexpr uint32_t kSmem = 232448;          // shared memory of a block
constexpr uint32_t kGroupM = 16;            // tiles of m taken together, for L2 (8192 x 4096 x 8192: 4 384 us, 8 381, 16 366, 32 372)
constexpr uint32_t kTurnedRows = 64;        // up to so many rows the weight's columns are m
constexpr uint32_t kMostSplits = 8;         // parts of k: the blocks of a cluster
// Blocks of k that the tensor cores add up at most, by the output's type; such
// chains' sums are added by the epilogue's warps.  The tensor cores cut what
// does not fit fp32 towards zero, which grows with the number of products:
// positive fp16 numbers lose 2.6e-6 of a sum of 512, 2.5e-5 of 4096, 4.1e-4 of
// 65,536, 1.7e-3 of 262,144; bf16 up to as much.
// fp32 outputs: short chains, whose sums stay in registers, for which tiles of
// 256 columns leave no room (4096 x 4096 x 4096 96 -> 141 us, 8192 x 4096 x
// 8192 351 -> 538, 133 x 4096 x 2048 16.1 -> 17.5).
// 16-bit outputs: up to a tenth of the half step that they are rounded by, 8192
// products for fp16's 4.9e-4 and 65,536 for bf16's 3.9e-3; sums of chains that
// long wait in memory, written and read beside the next chain's products.
constexpr uint32_t chain_of(int type) { return type == ADAPM_F32 ? 8 : (type == ADAPM_F16 ? 128 : 1024); }
// Where the sums of chains stay.
enum { ONE_CHAIN = 0, IN_REGISTERS = 1, IN_MEMORY = 2 };

// ---- activations -----------------------------------------------------------------
// 1 / (1 + 2^x); 0 where 2^x is beyond fp32, as in the limit.
__device__ __forceinline__ float logistic(float x) { return over(1.f + exp2_of(x)); }
constexpr float kLog2E = 1.4426950408889634f;
// 1/2 (1 + tanh u) = 1 / (1 + e^-2u); -2 u log2(e) = z (kTanhA z^2 + kTanhB) with u = sqrt(2 / pi) (z + 0.044715 z^3)
constexpr float kTanhB = -2.f * 0.7978845608f * kLog2E, kTanhA = 0.044715f * kTanhB;

// act(z) of N numbers; the branch stands outside of the loop.
template <int N>
__device__ __forceinline__ void activate(float (&z)[N], int kind) {
  switch (kind) {
    case ADAPM_ACTIVATION_RELU:
#pragma unroll
      for (int j = 0; j < N; ++j) z[j] = z[j] < 0.f ? 0.f : z[j];   // (a NaN stays one)
      break;
    case ADAPM_ACTIVATION_GELU:
#pragma unroll
      for (int j = 0; j < N; ++j) z[j] = 0.5f * z[j] * (1.f + erff(z[j] * 0.70710678f));
      break;
    case ADAPM_ACTIVATION_GELU_TANH:
#pragma unroll
      for (int j = 0; j < N; ++j) z[j] *= logistic(z[j] * fmaf(kTanhA, z[j] * z[j], kTanhB));
      break;
    case ADAPM_ACTIVATION_SILU:
#pragma unroll
      for (int j = 0; j < N; ++j) z[j] *= logistic(-kLog2E * z[j]);
      break;
    case ADAPM_ACTIVATION_TANH:
#pragma unroll
      for (int j = 0; j < N; ++j) z[j] = tanhf(z[j]);
      break;
    default: break;
  }
}
// d times act'(z), N of them.
template <int N>
__device__ __forceinline__ void times_slope(float (&d)[N], const float (&z)[N], int kind) {
  switch (kind) {
    case ADAPM_ACTIVATION_RELU:
#pragma unroll
      for (int j = 0; j < N; ++j) d[j] = z[j] > 0.f ? d[j] : (z[j] != z[j] ? z[j] : d[j] * 0.f);
      break;
    case ADAPM_ACTIVATION_GELU:
#pragma unroll
      for (int j = 0; j < N; ++j)
        d[j] *= 0.5f * (1.f + erff(z[j] * 0.70710678f)) + z[j] * 0.39894228f * exp2_of(-0.5f * kLog2E * z[j] * z[j]);
      break;
    case ADAPM_ACTIVATION_GELU_TANH:
#pragma unroll
      for (int j = 0; j < N; ++j) {
        // s = 1 / (1 + e^-2u), its slope s (1 - s) 2 u'; where z^2 is beyond 10^30, s is 0 or 1 and its slope 0
        const float q = fminf(z[j] * z[j], 1e30f);
        const float s = logistic(z[j] * fmaf(kTanhA, q, kTanhB)), t = s * z[j];
        d[j] *= fmaf(fmaf(-s, t, t), fmaf(-3.f * kTanhA / kLog2E, q, -kTanhB / kLog2E), s);
      }
      break;
    case ADAPM_ACTIVATION_SILU:
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float s = logistic(-kLog2E * z[j]), t = s * z[j];
        d[j] *= fmaf(-s, t, t) + s;
      }
      break;
    case ADAPM_ACTIVATION_TANH:
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float t = tanhf(z[j]);
        d[j] *= 1.f - t * t;
      }
      break;
    default: break;
  }
}

// ---- the product -------------------------------------------------------------------
struct Tile {
  uint32_t m0, n0;
};
template <bool PAIR>
__device__ __forceinline__ Tile tile_of(const GemmProduct& p, uint32_t bn, uint32_t tile) {
  Tile t;
  // groups of kGroupM tiles of m, n by n inside
  const uint32_t in_group = kGroupM * p.tiles_n, group = tile / in_group, at = tile - group * in_group;
  const uint32_t height = min(kGroupM, p.tiles_m - group * kGroupM);
  t.m0 = (group * kGroupM + at % height) * (PAIR ? 2 * kTileM : kTileM);
  t.n0 = at / height * bn;
  return t;
}
// The tiles of a worker (a block, or a pair or cluster of them), one after the
// other; TWO: of both products.
template <bool TWO>
struct Items {
  uint32_t worker, workers;
  uint32_t which = 0, tile, head = 0;   // of which product, its number, how many before the common rounds
  bool any;
  __device__ __forceinline__ Items(const GemmArgs& g, uint32_t w, uint32_t all) : worker(w), workers(all), tile(w) { check(g); }
  __device__ __forceinline__ void check(const GemmArgs& g) {
    const GemmProduct& p = g.p[TWO ? which : 0];
    any = tile < p.tiles_m * p.tiles_n;
    if (!TWO || any || which == 1) return;
    which = 1;
    if (worker >= g.late && ahead(g) != 0 && g.head != 0) {
      head = g.head;
      tile = worker - g.late;
    } else {
      tile = common(g);
    }
    any = tile < g.p[1].tiles_m * g.p[1].tiles_n;
  }
  __device__ __forceinline__ uint32_t ahead(const GemmArgs& g) const { return g.late != 0 ? workers - g.late : 0; }
  __device__ __forceinline__ uint32_t common(const GemmArgs& g) const { return g.head * ahead(g) + (workers - 1 - worker); }
  __device__ __forceinline__ void next(const GemmArgs& g) {
    if (!TWO || head == 0) tile += workers;
    else tile = --head != 0 ? tile + ahead(g) : common(g);
    check(g);
  }
};

// ---- epilogue ------------------------------------------------------------------------
// N neighbours of a row, on a multiple of N where N > 1.  (What is read or
// written once stays out of the way of the operands in L2.)
template <int TYPE, int N>
__device__ __forceinline__ void load_once(const char* p, float* x) {
  if constexpr (N == 4 && TYPE == ADAPM_F32) {
    const float4 v = __ldcs(reinterpret_cast<const float4*>(p));
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
  } else if constexpr (N == 4) {
    const uint2 v = __ldcs(reinterpret_cast<const uint2*>(p));
    const float2 low = unpack2<TYPE>(v.x), high = unpack2<TYPE>(v.y);
    x[0] = low.x; x[1] = low.y; x[2] = high.x; x[3] = high.y;
  } else {
    load_n<TYPE, N>(p, x);
  }
}
template <int TYPE, int N>
__device__ __forceinline__ void store_once(char* p, const float* x) {
  if constexpr (N == 4 && TYPE == ADAPM_F32) __stcs(reinterpret_cast<float4*>(p), make_float4(x[0], x[1], x[2], x[3]));
  else if constexpr (N == 4) __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack2<TYPE>(x[0], x[1]), pack2<TYPE>(x[2], x[3])));
  else store_n<TYPE, N>(p, x);
}
// The places (r + i * step, c), i < ROWS, of a matrix.
template <int TYPE>
struct Places {
  char* at;
  int64_t step;
  __device__ __forceinline__ Places(const MatrixView& v, uint64_t r, uint32_t c, uint32_t rows)
      : at(v.data + ((int64_t)r * v.row_stride + c) * (TYPE == ADAPM_F32 ? 4 : 2)),
        step((int64_t)rows * v.row_stride * (TYPE == ADAPM_F32 ? 4 : 2)) {}
  __device__ __forceinline__ char* operator[](int i) const { return at + i * step; }
};
// ROWS such places of N columns: z becomes what is stored; bias: of the
// columns.  Those from `count` on do not exist.
template <int TYPE, bool OUT32, int N, int ROWS>
__device__ __forceinline__ void finish(const Epilogue& e, uint64_t r, uint32_t step, uint32_t c, uint32_t count,
                                       const float (&bias)[N], float (&z)[ROWS * N]) {
  constexpr int kOut = OUT32 ? ADAPM_F32 : TYPE;
  float add[ROWS][N];
  const bool more = e.residual.data != nullptr;
  if (more) {
    const Places<kOut> from(e.residual, r, c, step);
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
      if (i < (int)count) load_once<kOut, N>(from[i], add[i]);
  }
#pragma unroll
  for (int j = 0; j < ROWS * N; ++j) z[j] += bias[j % N];
  if (e.pre.data != nullptr) {
    const Places<TYPE> to(e.pre, r, c, step);
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
      if (i < (int)count) store_once<TYPE, N>(to[i], z + i * N);
  }
  activate(z, e.activation);
  if (more) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) z[i * N + j] += add[i][j];
  }
  const Places<kOut> to(e.out, r, c, step);
#pragma unroll
  for (int i = 0; i < ROWS; ++i)
    if (i < (int)count) store_once<kOut, N>(to[i], z + i * N);
}

// 32 x 32 elements that a warp has staged, rows apart by 36: rows [m0, m0 + 32),
// columns [n0, n0 + 32) of m x n.
template <int TYPE, bool OUT32>
__device__ __forceinline__ void finish_tile(const Epilogue& e, bool aligned, const float* tile, uint32_t m, uint32_t n, uint32_t m0, uint32_t n0) {
  const uint32_t lane = threadIdx.x & 31u, rows = m - m0;
  if (aligned && n0 + 32 <= n) {
    // a lane holds four neighbours of each fourth row
    const uint32_t c = n0 + (lane & 7u) * 4, mine = lane >> 3;
    float bias[4] = {0.f, 0.f, 0.f, 0.f};
    if (e.bias.data)
#pragma unroll
      for (int j = 0; j < 4; ++j) bias[j] = load_as(e.bias.data, e.bias.type, c + j);
#pragma unroll
    for (uint32_t r0 = mine; r0 < 32; r0 += 16) {
      float z[16];
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) {
        const float4 q = *reinterpret_cast<const float4*>(tile + (r0 + i * 4) * 36 + (lane & 7u) * 4);
        z[4 * i] = q.x; z[4 * i + 1] = q.y; z[4 * i + 2] = q.z; z[4 * i + 3] = q.w;
      }
      finish<TYPE, OUT32, 4, 4>(e, (uint64_t)m0 + r0, 4, c, r0 < rows ? (rows - r0 + 3) / 4 : 0, bias, z);
    }
  } else if (n0 + lane < n) {
    // a lane holds a column: whatever the alignment, a row's stores are neighbours
    float bias[1] = {0.f};
    if (e.bias.data) bias[0] = load_as(e.bias.data, e.bias.type, n0 + lane);
#pragma unroll 1
    for (uint32_t r0 = 0; r0 < 32; r0 += 16) {
      float z[16];
#pragma unroll
      for (uint32_t i = 0; i < 16; ++i) z[i] = tile[(r0 + i) * 36 + lane];
      finish<TYPE, OUT32, 1, 16>(e, (uint64_t)m0 + r0, 1, n0 + lane, r0 < rows ? rows - r0 : 0, bias, z);
    }
  }
}

// Block `block` of `blocks`: 32 columns at a time, every warp its share of the
// rows, the warps' sums in their order.
__device__ __forceinline__ void add_columns(const ColumnSums& s, float* shared, uint32_t block, uint32_t blocks) {
  constexpr uint32_t kWarps = kGemmThreads / 32;
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  for (uint32_t c0 = block * 32; c0 < s.columns; c0 += blocks * 32) {
    const uint32_t c = c0 + lane;
    float sum = 0.f;
    if (c < s.columns)
#pragma unroll 4
      for (uint32_t i = warp; i < s.count; i += kWarps) sum += s.parts[(uint64_t)i * s.columns + c];
    shared[warp * 32 + lane] = sum;
    __syncthreads();
    if (warp == 0 && c < s.columns) {
      for (uint32_t w = 1; w < kWarps; ++w) sum += shared[w * 32 + lane];
      store_as(s.out.data, s.out.type, c, sum);
    }
    __syncthreads();
  }
}

// kGemmThreads threads: warp 0 copies, warp 1 multiplies, the others finish.
// PAIR: tiles of 256 x bn by two blocks; each copies its halves of the operands
// and finishes its half of the rows, the first one multiplies.  An SM then
// holds, and writes to its shared memory, half of b's tile: with tiles of 128 x
// 256 copies and products move 96 KB through it per block of k, 188 bytes a clock at
// full rate, with pairs 64 KB.
// CHAIN: for more blocks of k than a chain has: fp32 outputs in tiles of up to
// 128 columns (IN_REGISTERS), 16-bit ones (IN_MEMORY).
// TWO: of two products, both without more of an epilogue than the output, each of a type of its own.
template <bool BF16, bool OUT32, bool PAIR, bool TWO, int CHAIN>
__global__ void __launch_bounds__(kGemmThreads, 1)
gemm_kernel(const __grid_constant__ GemmArgs g) {
  constexpr int TYPE = BF16 ? ADAPM_BF16 : ADAPM_F16;
  extern __shared__ uint8_t smem[];
  __shared__ uint64_t bars[2 * kMaxStages + 4];
  __shared__ uint32_t tmem_at;
  __shared__ uint32_t gave_up;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t b_rows = PAIR ? g.bn / 2 : g.bn;   // of b's tile, in this block
  const uint32_t a_bytes = kTileM * 128, stage_bytes = a_bytes + b_rows * 128;
  const uint32_t ring = (shared_at(smem) + 1023u) & ~1023u;
  float* const ring_floats = reinterpret_cast<float*>(smem + (ring - shared_at(smem)));
  float* const staging = ring_floats + g.stages * stage_bytes / 4;
  const uint32_t full = shared_at(bars), empty = full + 8 * kMaxStages, sum_full = empty + 8 * kMaxStages, sum_empty = sum_full + 16;
  const uint32_t columns = 2 * g.bn;   // (bn is a power of two, at least 16)
  const uint32_t rank = PAIR ? blockIdx.x & 1u : 0;
  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < g.stages; ++s) {
      barrier_init(full + 8 * s, 1);
      barrier_init(empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      barrier_init(sum_full + 8 * b, 1);
      barrier_init(sum_empty + 8 * b, (PAIR ? 2 : 1) * kFinishWarps);
    }
    gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if constexpr (PAIR) cg::this_cluster().sync();
  if (warp == 1) tmem_take<PAIR>(&tmem_at, columns);
  tmem_fence_before();
  if constexpr (PAIR) cg::this_cluster().sync();
  else __syncthreads();
  tmem_fence_after();
  after_previous();
  const uint32_t tmem = tmem_at;
  // with parts of k, each block of a cluster sums one part of one tile
  const uint32_t part = g.splits > 1 ? blockIdx.x % g.splits : 0, team = PAIR ? 2 : g.splits;
  const uint32_t worker = blockIdx.x / team, workers = TWO ? g.workers : gridDim.x / team, k0 = part * g.per_split;
  auto k_end = [&](const GemmProduct& p) { return !TWO && g.splits > 1 ? min(p.k_blocks, k0 + g.per_split) : p.k_blocks; };
  if (TWO && worker >= workers) {
    add_columns(g.sums, staging, worker - workers, gridDim.x - workers);
  } else if (warp == 0) {
    if (lane == 0) {
      asm volatile("fence.proxy.async;" ::: "memory");
      uint32_t n = 0, stage = 0, parity = 1;   // copies issued; a fresh ring is empty
      bool ok = true;
      for (Items<TWO> i(g, worker, workers); i.any && ok; i.next(g)) {
        const GemmProduct& p = g.p[TWO ? i.which : 0];
        const Tile t = tile_of<PAIR>(p, g.bn, i.tile);
        const uint32_t m0 = t.m0 + rank * kTileM, n0 = t.n0 + rank * b_rows, k1 = k_end(p);
        for (uint32_t k = k0; k < k1; ++k) {
          if (!(ok = barrier_wait(empty + 8 * stage, parity))) break;
          const uint32_t at = ring + stage * stage_bytes;
          uint32_t bar = full + 8 * stage;
          // (the first block's barrier counts both blocks' bytes, before or after it expects them)
          if (!PAIR || rank == 0) barrier_expect(bar, (PAIR ? 2 : 1) * stage_bytes);
          if (PAIR) bar = shared_of(bar, 0);
          auto copy = [&](uint32_t to, const CUtensorMap* map, uint32_t x, uint32_t y) {
            if constexpr (PAIR) copy_tile_pair(to, map, (int)x, (int)y, bar);
            else copy_tile(to, map, (int)x, (int)y, bar);
          };
          if (!p.a_across) {
            copy(at, &p.a, k * kBlockK, m0);
          } else {
            for (uint32_t j = 0; j < kTileM; j += 64) copy(at + j * 128, &p.a, m0 + j, k * kBlockK);
          }
          if (!p.b_across) {
            copy(at + a_bytes, &p.b, k * kBlockK, n0);
          } else {
            for (uint32_t j = 0; j < b_rows; j += 64) copy(at + a_bytes + j * 128, &p.b, n0 + j, k * kBlockK);
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
        // copies in flight land before the block ends (of a pair's second block: its share of the first one's barriers)
        for (uint32_t j = n > g.stages ? n - g.stages : 0; j < n; ++j)
          if (!barrier_wait(rank == 0 ? full + 8 * (j % g.stages) : empty + 8 * (j % g.stages), (j / g.stages) & 1u)) break;
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      uint32_t stage = 0, parity = 0, turn = 0;
      bool ok = true;
      for (Items<TWO> i(g, worker, workers); i.any && ok; i.next(g)) {
        const GemmProduct& p = g.p[TWO ? i.which : 0];
        const uint32_t shape = mma_shape(BF16, p.a_across, p.b_across, PAIR ? 2 * kTileM : kTileM, g.bn);
        const uint32_t a_step = tile_step(p.a_across), b_step = tile_step(p.b_across), k1 = k_end(p);
        for (uint32_t from = k0, to; from < k1 && ok; from = to, ++turn) {   // a chain of them
          to = CHAIN ? min(k1, from + p.chain) : k1;
          const uint32_t b = turn & 1u;
          if (!(ok = barrier_wait(sum_empty + 8 * b, ((turn >> 1) & 1u) ^ 1u))) break;
          tmem_fence_after();
          for (uint32_t k = from; k < to; ++k) {
            if (!(ok = barrier_wait(full + 8 * stage, parity))) break;
            tmem_fence_after();
            const uint32_t at = ring + stage * stage_bytes;
            const uint64_t da = tile_descriptor(at, p.a_across), db = tile_descriptor(at + a_bytes, p.b_across);
#pragma unroll
            for (uint32_t j = 0; j < kBlockK / 16; ++j)
              mma<PAIR>(tmem + b * g.bn, da + j * a_step, db + j * b_step, shape, k > from || j > 0);
            mma_commit<PAIR>(empty + 8 * stage);
            if (++stage == g.stages) {
              stage = 0;
              parity ^= 1u;
            }
          }
          mma_commit<PAIR>(sum_full + 8 * b);
        }
      }
      if (!ok) atomicExch(&gave_up, 1u);
    }
  } else {
    const uint32_t quarter = (uint32_t)warp & 3u;      // of the rows of tensor memory that this warp reaches
    const uint32_t half = (uint32_t)(warp - 2) >> 2;   // of their columns, by turns
    float* const tile = staging + (warp - 2) * kStage;
    uint32_t turn = 0;
    float run[CHAIN == IN_REGISTERS ? 2 : 1][32];   // sums of the chains so far
    bool ok = true;
    for (Items<TWO> i(g, worker, workers); i.any && ok; i.next(g)) {
      const GemmProduct& p = g.p[TWO ? i.which : 0];
      const Tile t = tile_of<PAIR>(p, g.bn, i.tile);
      const uint32_t m0 = t.m0 + rank * kTileM + quarter * 32, k1 = k_end(p);
      for (uint32_t k = k0, to; k < k1; k = to, ++turn) {
        to = CHAIN ? min(k1, k + p.chain) : k1;
        const bool more = CHAIN && k > k0, last = !CHAIN || to == k1;
        const uint32_t b = turn & 1u;
        if (!(ok = barrier_wait(sum_full + 8 * b, (turn >> 1) & 1u))) {
          if (lane == 0) atomicExch(&gave_up, 1u);
          break;
        }
        __syncwarp();
        tmem_fence_after();
        const uint32_t from = tmem + ((quarter * 32u) << 16) + b * g.bn;
        // (column c of the lane's row: read and written by this lane alone)
        float* const waiting = CHAIN == IN_MEMORY ? g.chains + (uint64_t)blockIdx.x * g.bn * kTileM + quarter * 32 + lane : nullptr;
        if (!PAIR && !TWO && (g.splits > 1 || g.turned)) {
          // to shared memory (the ring is no longer read: there is one tile): see below
          const uint32_t row = quarter * 32 + lane;
#pragma unroll
          for (uint32_t n = 0; n < 2; ++n) {
            const uint32_t c0 = half * 16 + n * 32;
            if (c0 >= g.bn) break;
            float v[16];
            __syncwarp();
            tmem_load16(from + c0, v);
            if constexpr (CHAIN) {
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                if (more) v[j] += run[0][n * 16 + j];
                run[0][n * 16 + j] = v[j];
              }
            }
            if (!last) continue;
            if (g.turned) {
#pragma unroll
              for (int j = 0; j < 16; ++j) ring_floats[(c0 + j) * kTileM + row] = v[j];
            } else {
#pragma unroll
              for (int j = 0; j < 16; j += 4)
                *reinterpret_cast<float4*>(ring_floats + row * (g.bn + 4) + c0 + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
            }
          }
        } else if (!last) {
          if constexpr (CHAIN == IN_MEMORY) {
            for (uint32_t c0 = half * 32; c0 < g.bn && t.n0 + c0 < p.n; c0 += 64) {
              float v[32];
              float* const at = waiting + c0 * kTileM;
              __syncwarp();
              tmem_load(from + c0, v);
              if (more) {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] += at[j * kTileM];
              }
#pragma unroll
              for (int j = 0; j < 32; ++j) at[j * kTileM] = v[j];
            }
          }
          if constexpr (CHAIN == IN_REGISTERS) {
#pragma unroll
            for (uint32_t n = 0; n < 2; ++n) {
              const uint32_t c0 = half * 32 + n * 64;
              if (c0 >= g.bn || t.n0 + c0 >= p.n) break;
              float v[32];
              __syncwarp();
              tmem_load(from + c0, v);
#pragma unroll
              for (int j = 0; j < 32; ++j) run[n][j] = more ? run[n][j] + v[j] : v[j];
            }
          }
        } else {
          for (uint32_t c0 = half * 32, n = 0; c0 < g.bn && t.n0 + c0 < p.n; c0 += 64, ++n) {
            float v[32];
            __syncwarp();
            tmem_load(from + c0, v);
            if constexpr (CHAIN == IN_MEMORY) {
              if (more) {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] += waiting[(c0 + j) * kTileM];
              }
            }
            if constexpr (CHAIN == IN_REGISTERS) {
              // (an array of registers has no index)
              auto add = [&](const float (&sums)[32]) {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] += sums[j];
              };
              if (more) {
                if (n == 0) add(run[0]);
                else add(run[1]);
              }
            }
            // through shared memory, so that neighbouring lanes hold neighbouring columns
#pragma unroll
            for (int j = 0; j < 32; j += 4)
              *reinterpret_cast<float4*>(tile + lane * 36 + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
            __syncwarp();
            if (m0 >= p.m) continue;
            if constexpr (TWO) {
              Epilogue e{};
              e.out = p.e.out;
              if (e.out.type == ADAPM_F32) finish_tile<TYPE, true>(e, p.aligned, tile, p.m, p.n, m0, t.n0 + c0);
              else finish_tile<TYPE, false>(e, p.aligned, tile, p.m, p.n, m0, t.n0 + c0);
            } else {
              finish_tile<TYPE, OUT32>(p.e, p.aligned, tile, p.m, p.n, m0, t.n0 + c0);
            }
          }
        }
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) {
          if constexpr (PAIR) barrier_arrive_at(shared_of(sum_empty + 8 * b, 0));
          else barrier_arrive(sum_empty + 8 * b);
        }
      }
    }
  }
  __syncwarp();
  if (!PAIR && !TWO && (g.splits > 1 || g.turned)) {
    // One tile per block, or one part of it: the cluster's blocks add up a
    // share each, in the order of the parts.
    cg::cluster_group cluster = cg::this_cluster();
    if (g.splits > 1) cluster.sync();
    else __syncthreads();
    const GemmProduct& p = g.p[0];
    const Tile t = tile_of<PAIR>(p, g.bn, worker);
    const uint32_t shift = 31 - __clz(g.bn);
    // four neighbours at a time, of all parts at once
    for (uint32_t j = 4 * (part * kGemmThreads + threadIdx.x); j < kTileM * g.bn; j += 4 * g.splits * kGemmThreads) {
      const uint32_t m = g.turned ? j & (kTileM - 1) : j >> shift, n = g.turned ? j / kTileM : j & (g.bn - 1);
      const uint32_t at = g.turned ? j : m * (g.bn + 4) + n;
      if (t.m0 + m >= p.m || t.n0 + n >= p.n) continue;
      float4 v[kMostSplits];
#pragma unroll
      for (uint32_t s = 0; s < kMostSplits; ++s)
        if (s < g.splits)
          v[s] = *reinterpret_cast<const float4*>((g.splits > 1 ? cluster.map_shared_rank(ring_floats, s) : ring_floats) + at);
      float z[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
      for (uint32_t s = 1; s < kMostSplits; ++s) {
        if (s >= g.splits) break;
        z[0] += v[s].x; z[1] += v[s].y; z[2] += v[s].z; z[3] += v[s].w;
      }
      const uint32_t c = g.turned ? t.m0 + m : t.n0 + n, width = g.turned ? p.m : p.n;   // (columns of the product)
      const uint64_t r = g.turned ? t.n0 + n : t.m0 + m;
      float bias[4] = {0.f, 0.f, 0.f, 0.f};
      if (p.e.bias.data)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c + i < width) bias[i] = load_as(p.e.bias.data, p.e.bias.type, c + i);
      if (p.aligned && c + 4 <= width) {
        finish<TYPE, OUT32, 4, 1>(p.e, r, 0, c, 1, bias, z);
      } else {
#pragma unroll 1
        for (int i = 0; i < 4 && c + i < width; ++i) {
          const float b1[1] = {i == 0 ? bias[0] : (i == 1 ? bias[1] : (i == 2 ? bias[2] : bias[3]))};
          float z1[1] = {i == 0 ? z[0] : (i == 1 ? z[1] : (i == 2 ? z[2] : z[3]))};
          finish<TYPE, OUT32, 1, 1>(p.e, r, 0, c + i, 1, b1, z1);
        }
      }
    }
    if (g.splits > 1) cluster.sync();   // (others may still read here)
  }
  tmem_fence_before();
  if constexpr (PAIR) cg::this_cluster().sync();
  else __syncthreads();
  tmem_fence_after();
  if (threadIdx.x == 0 && gave_up) set_error(g.st, ERR_TIMEOUT);
  if (warp == 1) tmem_give<PAIR>(tmem, columns);
}

// ---- operands ------------------------------------------------------------------------
// rows x columns elements of a 16-bit type to rows that begin `pitch` (a
// multiple of eight) apart, of up to two matrices.  A thread writes eight
// neighbours; where a row's elements are neighbours too they come from the two
// 16-byte words that hold them, which may hold others of the matrix, but
// nothing in front of or behind it.
struct PackJob {
  const uint16_t* from;
  uint16_t* to;
  int64_t row_stride, col_stride;
  uint64_t rows;
  uint32_t columns, pitch, eights;   // eights: of a row
  uint32_t blocks;
};
__device__ __forceinline__ uint4 eight_of(const PackJob& p, uint64_t r, uint32_t c) {
  const uint16_t* const at = p.from + (int64_t)r * p.row_stride + (int64_t)c * p.col_stride;
  if (p.col_stride == 1 && c + 8 <= p.columns) {
    const uint32_t in = (uint32_t)reinterpret_cast<uintptr_t>(at) & 15u;
    const char* const word = reinterpret_cast<const char*>(at) - in;
    const char* const end = reinterpret_cast<const char*>(p.from + (int64_t)(p.rows - 1) * p.row_stride + p.columns);
    if (in == 0) return *reinterpret_cast<const uint4*>(word);
    if (word >= reinterpret_cast<const char*>(p.from) && word + 32 <= end) {
      const uint4 lo = *reinterpret_cast<const uint4*>(word), hi = *reinterpret_cast<const uint4*>(word + 16);
      uint32_t x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
      if (in & 8u)
#pragma unroll
        for (int j = 0; j < 6; ++j) x[j] = x[j + 2];
      if (in & 4u)
#pragma unroll
        for (int j = 0; j < 5; ++j) x[j] = x[j + 1];
      const uint32_t bits = (in & 3u) * 8u;
      return make_uint4(__funnelshift_r(x[0], x[1], bits), __funnelshift_r(x[1], x[2], bits), __funnelshift_r(x[2], x[3], bits),
                        __funnelshift_r(x[3], x[4], bits));
    }
  }
  uint32_t x[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (uint32_t j = 0; j < 8; ++j)
    if (c + j < p.columns) x[j / 2] |= (uint32_t)at[(int64_t)j * p.col_stride] << (16 * (j & 1));
  return make_uint4(x[0], x[1], x[2], x[3]);
}
__global__ void __launch_bounds__(256)
pack_kernel(const PackJob x, const PackJob y) {
  after_previous();
  const bool second = blockIdx.x >= x.blocks;
  const PackJob& p = second ? y : x;
  const uint32_t b = second ? blockIdx.x - x.blocks : blockIdx.x;
  const uint64_t i = (uint64_t)b * 256 + threadIdx.x, r = i / p.eights;
  const uint32_t c = (uint32_t)(i - r * p.eights) * 8;
  if (r < p.rows) *reinterpret_cast<uint4*>(p.to + r * p.pitch + c) = eight_of(p, r, c);
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

// Copies those of two operands to `at` that have to be.
void pack(Operand& x, Operand& y, char* at, cudaStream_t stream) {
  PackJob jobs[2]{};
  uint64_t blocks = 0;
  int i = 0;
  for (Operand* o : {&x, &y}) {
    PackJob& j = jobs[i++];
    j.eights = 1;
    if (!o->packed) continue;
    j.from = reinterpret_cast<const uint16_t*>(o->data);
    j.to = reinterpret_cast<uint16_t*>(at);
    j.row_stride = o->across ? o->k_stride : o->mn_stride;
    j.col_stride = o->across ? o->mn_stride : o->k_stride;
    j.rows = o->across ? o->k : o->mn;
    j.columns = (uint32_t)(o->across ? o->mn : o->k);
    j.pitch = (uint32_t)o->pitch;
    j.eights = (j.columns + 7) / 8;
    j.blocks = (uint32_t)((j.rows * j.eights + 255) / 256);
    blocks += j.blocks;
    o->data = at;
    at += round256(o->bytes);
  }
  if (blocks == 0) return;
  note_launches(1);
  launch_after(pack_kernel, (unsigned)blocks, 256, 0, stream, jobs[0], jobs[1]);
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
  uint64_t m, n;
  bool turned, pair;
  int chained;   // where the sums of chains stay (ONE_CHAIN, ...)
  uint32_t chain;   // blocks of k of one
  uint32_t bn, tiles_m, tiles_n, k_blocks, splits, per_split, stages;
  double us;   // that it takes, by kForms
};
// What a form of the kernel takes: microseconds before the first round of
// tiles, per block of k and per tile, as measured with fp16 outputs on sizes
// from 300 x 512 x 2048 to 4096 x 4096 x 4096.  The form is chosen by the sum,
// which is near what the sizes below take (rows x ins x outs, us):
//                        pairs  128 x 256  128 x 128  128 x 64
//   4096 x 4096 x 4096     89      121        125       215
//   2048 x 2048 x 2048     19       18         23        35
//   4096 x 4096 x 512      27       27         22        34
//   1024 x 1024 x 1024     13       12          9         8
//    256 x 8192 x 1000     47       67         44        15 (in parts)
struct Form {
  bool pair;
  uint32_t bn;
  double start, block, tile;
};
constexpr Form kForms[] = {
    {true, 256, 7.6, 0.284, 2.1}, {false, 256, 6.6, 0.345, 1.1}, {false, 128, 4.8, 0.24, 1.2}, {false, 64, 3.5, 0.22, 0.9}};
constexpr double kPartsCost = 3.0;   // of summing k in parts by a cluster
uint64_t tiles_of(const GemmPlan& p, uint32_t bn, bool pair) {
  const uint64_t height = pair ? 2 * kTileM : kTileM;
  return ((p.m + height - 1) / height) * ((p.n + bn - 1) / bn);
}
void set_form(GemmPlan& p, uint32_t bn, bool pair, uint64_t parts) {
  const uint32_t height = pair ? 2 * kTileM : kTileM;
  p.pair = pair;
  p.bn = bn;
  p.tiles_m = (uint32_t)((p.m + height - 1) / height);
  p.tiles_n = (uint32_t)((p.n + bn - 1) / bn);
  p.per_split = (uint32_t)((p.k_blocks + parts - 1) / parts);
  p.splits = (p.k_blocks + p.per_split - 1) / p.per_split;
  const uint32_t stage = kTileM * 128 + (pair ? bn / 2 : bn) * 128;
  p.stages = std::min(kMaxStages, (kSmem - 1024 - 512 - kFinishWarps * kStage * (uint32_t)sizeof(float)) / stage);
}
// The product of `rows` x `columns` elements of `type` over k.
GemmPlan gemm_plan(uint64_t rows, uint32_t columns, uint64_t k, int type, int sms) {
  GemmPlan p{};
  p.turned = rows <= kTurnedRows;
  p.m = p.turned ? columns : rows;
  p.n = p.turned ? rows : columns;
  p.k_blocks = (uint32_t)((k + kBlockK - 1) / kBlockK);
  p.chain = chain_of(type);
  if (type != ADAPM_F32 && p.k_blocks > p.chain) {   // chains of one length: none too short for the sums of the one before
    const uint32_t chains = (p.k_blocks + p.chain - 1) / p.chain;
    p.chain = (p.k_blocks + chains - 1) / chains;
  }
  p.chained = p.k_blocks <= chain_of(type) ? ONE_CHAIN : (type == ADAPM_F32 ? IN_REGISTERS : IN_MEMORY);
  // parts of k, of at least two blocks, while SMs are idle
  auto parts_of = [&](uint64_t tiles) {
    return std::max<uint64_t>(1, std::min<uint64_t>({(uint64_t)sms / tiles, p.k_blocks / 2, kMostSplits}));
  };
  if (p.turned) {
    const uint32_t bn = p.n <= 16 ? 16 : (p.n <= 32 ? 32 : 64);
    set_form(p, bn, false, parts_of(tiles_of(p, bn, false)));
    return p;
  }
  const Form* best = nullptr;
  uint64_t parts = 1;
  for (const Form& f : kForms) {
    if (p.chained == IN_REGISTERS && f.bn > 128) continue;   // (sums of chains that the registers hold)
    const uint64_t tiles = tiles_of(p, f.bn, f.pair), at_once = f.pair ? sms / 2 : sms;
    const double rounds = (double)((tiles + at_once - 1) / at_once);
    for (int in_parts = 0; in_parts < 2; ++in_parts) {
      const uint64_t s = in_parts ? parts_of(tiles) : 1;
      if (in_parts && (s == 1 || f.bn > 64)) continue;   // (128 x 128 in parts: 1327 x 3315 x 651 30 -> 35)
      const double us = f.start + (in_parts ? kPartsCost : 0.0) + rounds * ((double)((p.k_blocks + s - 1) / s) * f.block + f.tile);
      if (best && us >= p.us) continue;
      best = &f;
      p.us = us;
      parts = s;
    }
  }
  set_form(p, best->bn, best->pair, parts);
  return p;
}
// How two products share a launch.
struct Shared {
  uint32_t late, head;
};
// Whether one launch of one form does p (of as many blocks of k or more) and q
// sooner than each one's own: then they have that form.  A round of p that is
// not full is filled with tiles of q.  By a sixteenth at least, and not in
// pairs, which leave little idle (both gradients of rows x ins x outs, us):
//                          apart   one launch   of pairs
//     777 x  256 x 1000     16.2      10.5
//    1024 x 1024 x 1024     16.2      10.4
//    2048 x 2048 x 2048     34.1      30.1       35.0
//   16384 x 1024 x 1024     99.9      81.6
//    4096 x 4096 x 4096    185       205        182
//    8192 x 4096 x 4096    350                  361
bool share(GemmPlan& p, GemmPlan& q, int sms, Shared* how) {
  if (p.turned || q.turned || p.chained == IN_REGISTERS || q.chained == IN_REGISTERS) return false;
  double best = (p.us + q.us) * 15 / 16;
  const Form* form = nullptr;
  for (const Form& f : kForms) {
    if (f.pair) continue;
    const uint64_t of_p = tiles_of(p, f.bn, false), of_q = tiles_of(q, f.bn, false);
    const uint64_t workers = std::min<uint64_t>(sms, of_p + of_q);
    const double each_p = p.k_blocks * f.block + f.tile, each_q = q.k_blocks * f.block + f.tile;
    const uint64_t late = of_p % workers, head = late ? (uint64_t)(each_p / each_q) : 0;
    const uint64_t ahead = late ? head * (workers - late) : 0;
    const double rounds = (double)(of_p / workers), common = (double)(((of_q > ahead ? of_q - ahead : 0) + workers - 1) / workers);
    const double us = f.start + rounds * each_p + (late ? std::max(each_p, (double)head * each_q) : 0.0) + common * each_q;
    if (us >= best) continue;
    best = us;
    form = &f;
    *how = {(uint32_t)late, (uint32_t)head};
  }
  if (!form) return false;
  set_form(p, form->bn, false, 1);
  set_form(q, form->bn, false, 1);
  return true;
}

bool on_four(const MatrixView& v, uint64_t rows) {
  return v.data == nullptr || (reinterpret_cast<uintptr_t>(v.data) % (4 * type_size(v.type)) == 0 && (rows <= 1 || v.row_stride % 4 == 0));
}

// rows x columns = left (rows x k) right (k x columns), with its epilogue.
struct Product {
  GemmPlan p;
  Operand left, right;
  Epilogue e;
  size_t bytes() const { return round256(left.bytes) + round256(right.bytes); }   // of copies
  uint64_t tiles() const { return (uint64_t)p.tiles_m * p.tiles_n; }
};
// (a block whose tile goes through the ring to its epilogue takes one tile)
bool single(const GemmPlan& p) { return p.splits > 1 || p.turned; }
bool chains_wait(const Product& first, const Product* second) {
  return first.p.chained == IN_MEMORY || (second && second->p.chained == IN_MEMORY);
}
// Bytes of memory for the sums of chains (those of single tiles stay in registers).
size_t chain_bytes(const Product& first, const Product* second, int sms) {
  return chains_wait(first, second) && !single(first.p) ? (size_t)sms * first.p.bn * kTileM * sizeof(float) : 0;
}
// One product, or two that share a launch; chains: chain_bytes of memory.
cudaError_t launch_gemm(const Product& first, const Product* second, const Shared& how, const ColumnSums& sums, bool bf16, char* chains,
                        DevState* st, int sms, cudaStream_t stream) {
  const GemmPlan& p = first.p;
  GemmArgs g{};
  for (int i = 0; i < (second ? 2 : 1); ++i) {
    const Product& q = i ? *second : first;
    GemmProduct& to = g.p[i];
    const Operand& a = p.turned ? q.right : q.left;
    const Operand& b = p.turned ? q.left : q.right;
    cudaError_t err = tensor_map(a, bf16, kTileM, &to.a);
    if (err == cudaSuccess) err = tensor_map(b, bf16, p.pair ? p.bn / 2 : p.bn, &to.b);
    if (err != cudaSuccess) return err;
    to.a_across = a.across;
    to.b_across = b.across;
    to.aligned = on_four(q.e.out, q.left.mn) && on_four(q.e.pre, q.left.mn) && on_four(q.e.residual, q.left.mn);
    to.m = (uint32_t)a.mn;
    to.n = (uint32_t)b.mn;
    to.k_blocks = q.p.k_blocks;
    to.chain = q.p.chain;
    to.tiles_m = q.p.tiles_m;
    to.tiles_n = q.p.tiles_n;
    to.e = q.e;
  }
  g.late = how.late;
  g.head = how.head;
  g.turned = p.turned;
  g.bn = p.bn;
  g.stages = p.stages;
  g.splits = p.splits;
  g.per_split = p.per_split;
  g.chains = reinterpret_cast<float*>(chains);
  g.st = st;
  using Kernel = void (*)(GemmArgs);
  // (two products share no pairs, and chains in registers are none of theirs)
  static constexpr Kernel kernels[2][6][2] = {
      {{gemm_kernel<false, false, false, false, ONE_CHAIN>, gemm_kernel<false, false, true, false, ONE_CHAIN>},
       {gemm_kernel<false, true, false, false, ONE_CHAIN>, gemm_kernel<false, true, true, false, ONE_CHAIN>},
       {gemm_kernel<false, false, false, true, ONE_CHAIN>, nullptr},
       {gemm_kernel<false, true, false, false, IN_REGISTERS>, nullptr},
       {gemm_kernel<false, false, false, false, IN_MEMORY>, gemm_kernel<false, false, true, false, IN_MEMORY>},
       {gemm_kernel<false, false, false, true, IN_MEMORY>, nullptr}},
      {{gemm_kernel<true, false, false, false, ONE_CHAIN>, gemm_kernel<true, false, true, false, ONE_CHAIN>},
       {gemm_kernel<true, true, false, false, ONE_CHAIN>, gemm_kernel<true, true, true, false, ONE_CHAIN>},
       {gemm_kernel<true, false, false, true, ONE_CHAIN>, nullptr},
       {gemm_kernel<true, true, false, false, IN_REGISTERS>, nullptr},
       {gemm_kernel<true, false, false, false, IN_MEMORY>, gemm_kernel<true, false, true, false, IN_MEMORY>},
       {gemm_kernel<true, false, false, true, IN_MEMORY>, nullptr}}};
  const bool wait = chains_wait(first, second);
  const int what = second ? (wait ? 5 : 2) : (wait ? 4 : (p.chained ? 3 : (first.e.out.type == ADAPM_F32 ? 1 : 0)));
  const Kernel kernel = kernels[bf16][what][p.pair];
  static Asked asked[2][6][2];
  const cudaError_t err = asked[bf16][what][p.pair].allow(kernel, kSmem - 1024);
  if (err != cudaSuccess) return err;
  const uint64_t tiles = first.tiles() + (second ? second->tiles() : 0);
  g.workers = (uint32_t)std::min<uint64_t>(tiles, (uint64_t)sms);
  g.sums = sums;
  const uint32_t others = sums.parts ? std::min((uint32_t)sms - g.workers, (sums.columns + 31) / 32) : 0;
  const unsigned cluster = p.pair ? 2 : p.splits;
  cudaLaunchAttribute at[2]{};
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t c{};
  c.gridDim = dim3((unsigned)(p.pair ? 2 * std::min<uint64_t>(tiles, (uint64_t)sms / 2)
                                     : (single(p) ? tiles * p.splits : g.workers + others)));
  c.blockDim = dim3(kGemmThreads);
  c.dynamicSmemBytes = 1024 + (size_t)p.stages * (kTileM + (p.pair ? p.bn / 2 : p.bn)) * 128 + kFinishWarps * kStage * sizeof(float);
  c.stream = stream;
  c.attrs = at;
  c.numAttrs = cluster > 1 ? 2 : 1;
  note_launches(1);
  return cudaLaunchKernelEx(&c, kernel, g);
}

// ---- the gradient of z ----------------------------------------------------------------------
// dz = grad act'(pre) to rows of `pitch` elements (to null: grad itself
// serves), and the sums of its columns over a block's rows: 32 N columns a
// block, N neighbours a lane, warps take rows by turns, kDzRows at a time.
constexpr int kDzRows = 4;
// N elements of a 16-bit type as they come from memory.
template <int N>
struct Packed {
  uint4 v;
  __device__ __forceinline__ void fetch(const char* p) {
    if constexpr (N == 8) v = *reinterpret_cast<const uint4*>(p);
    else v.x = *reinterpret_cast<const uint16_t*>(p);
  }
  template <int TYPE>
  __device__ __forceinline__ void unpack(float (&x)[N]) const {
    if constexpr (N == 8) {
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = unpack2<TYPE>(w[j]);
        x[2 * j] = f.x;
        x[2 * j + 1] = f.y;
      }
    } else {
      x[0] = unpack2<TYPE>(v.x).x;
    }
  }
};
template <int TYPE, int N>
__global__ void __launch_bounds__(256, 3)
dz_kernel(const MatrixView grad, const MatrixView pre, int activation, char* to, uint32_t pitch, uint64_t rows, uint32_t columns,
          uint32_t per_block, float* parts) {
  after_previous();
  __shared__ float sums[8][32 * N];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t across = (columns + 32 * N - 1) / (32 * N);
  const uint32_t block = blockIdx.x / across;
  const uint64_t c = (uint64_t)(blockIdx.x % across) * 32 * N + lane * N;
  const uint64_t r1 = min(rows, (uint64_t)(block + 1) * per_block);
  float sum[N];
#pragma unroll
  for (int j = 0; j < N; ++j) sum[j] = 0.f;
  if (c < columns) {
    for (uint64_t r0 = (uint64_t)block * per_block + warp; r0 < r1; r0 += 8 * kDzRows) {
      Packed<N> d[kDzRows], z[kDzRows];
#pragma unroll
      for (int i = 0; i < kDzRows; ++i)
        if (r0 + i * 8 < r1) d[i].fetch(grad.data + ((int64_t)(r0 + i * 8) * grad.row_stride + (int64_t)c * grad.col_stride) * 2);
      if (activation != ADAPM_ACTIVATION_NONE) {
#pragma unroll
        for (int i = 0; i < kDzRows; ++i)
          if (r0 + i * 8 < r1) z[i].fetch(pre.data + ((int64_t)(r0 + i * 8) * pre.row_stride + (int64_t)c * pre.col_stride) * 2);
      }
#pragma unroll
      for (int i = 0; i < kDzRows; ++i) {
        if (r0 + i * 8 >= r1) continue;
        float x[N], y[N];
        d[i].template unpack<TYPE>(x);
        if (activation != ADAPM_ACTIVATION_NONE) {
          z[i].template unpack<TYPE>(y);
          times_slope(x, y, activation);
        }
        if (to != nullptr) store_n<TYPE, N>(to + ((r0 + i * 8) * pitch + c) * 2, x);
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] += x[j];
      }
    }
  }
  if (parts == nullptr) return;
#pragma unroll
  for (int j = 0; j < N; ++j) sums[warp][lane * N + j] = sum[j];
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * N; i += 256) {
    const uint64_t column = (uint64_t)(blockIdx.x % across) * 32 * N + i;
    if (column >= columns) continue;
    float s = 0.f;
    for (int w = 0; w < 8; ++w) s += sums[w][i];
    parts[block * (uint64_t)columns + column] = s;
  }
}

bool by_rows(const MatrixView& m, uint64_t rows, uint32_t columns) {   // stored with a row's elements contiguous
  return columns <= 1 || m.col_stride == 1 || !(rows <= 1 || m.row_stride == 1);
}

Product out_product(const LinearArgs& a, int sms) {   // rows x outs over ins
  Product q;
  q.p = gemm_plan(a.rows, a.outs, a.ins, a.out.type, sms);
  q.left = operand(a.x.data, a.rows, a.ins, a.x.row_stride, a.x.col_stride, q.p.turned);
  q.right = operand(a.weight.data, a.outs, a.ins, a.weight.col_stride, a.weight.row_stride, false);
  q.e = Epilogue{a.bias, a.residual, a.out, a.pre, a.activation};
  return q;
}

}  // namespace

size_t linear_scratch(const LinearArgs& a, int sms) {
  const Product q = out_product(a, sms);
  return q.bytes() + chain_bytes(q, nullptr, sms);
}

cudaError_t launch_linear(const LinearArgs& a, char* scratch, int sms, cudaStream_t stream) {
  Product q = out_product(a, sms);
  pack(q.left, q.right, scratch, stream);
  return launch_gemm(q, nullptr, Shared{}, ColumnSums{}, a.x.type == ADAPM_BF16, scratch + q.bytes(), a.st, sms, stream);
}

namespace {

// What the backward pass needs: dz (its own, or grad), the operands of both
// products, and their scratch, one after the other.
struct Backward {
  bool own_dz;
  uint32_t pitch;
  MatrixView dz;
  bool across_out;     // dweight is stored by output: its transpose is computed
  int vec;             // elements of an access of dz_kernel
  uint32_t across, blocks, per_block;   // its blocks: of columns, of rows, and their rows
  size_t dz_bytes, sum_bytes;
};
Backward backward_of(const LinearArgs& a, char* scratch, int sms) {
  Backward b{};
  b.own_dz = a.activation != ADAPM_ACTIVATION_NONE && (a.dx.data || a.dweight.data);
  b.pitch = (a.outs + 7) / 8 * 8;
  b.dz_bytes = b.own_dz ? round256(a.rows * (size_t)b.pitch * 2) : 0;
  b.dz = b.own_dz ? MatrixView{scratch, a.grad.type, (int64_t)b.pitch, 1} : a.grad;
  b.across_out = a.dweight.data && !by_rows(a.dweight, a.ins, a.outs);
  // eight neighbours where rows begin and end on them, else one
  auto on_eight = [&](const MatrixView& m) {
    return m.data == nullptr || (m.col_stride == 1 && reinterpret_cast<uintptr_t>(m.data) % 16 == 0 && (a.rows <= 1 || m.row_stride % 8 == 0));
  };
  b.vec = a.outs % 8 == 0 && on_eight(a.grad) && on_eight(a.pre) ? 8 : 1;
  b.across = (a.outs + 32 * b.vec - 1) / (32 * b.vec);
  // about six blocks an SM, of at least 32 rows
  const uint64_t want = std::max<uint64_t>(1, (uint64_t)sms * 6 / b.across);
  b.per_block = (uint32_t)std::max<uint64_t>(32, (a.rows + want - 1) / want);
  b.blocks = (uint32_t)((a.rows + b.per_block - 1) / b.per_block);
  b.sum_bytes = a.dbias.data ? round256((size_t)b.blocks * a.outs * sizeof(float)) : 0;
  return b;
}
Product dx_product(const LinearArgs& a, const Backward& b, int sms) {   // rows x ins over outs
  Product q;
  q.p = gemm_plan(a.rows, a.ins, a.outs, a.dx.type, sms);
  q.left = operand(b.dz.data, a.rows, a.outs, b.dz.row_stride, b.dz.col_stride, q.p.turned);
  q.right = operand(a.weight.data, a.ins, a.outs, a.weight.row_stride, a.weight.col_stride, false);
  q.e = Epilogue{};
  q.e.out = a.dx;
  return q;
}
Product dweight_product(const LinearArgs& a, const Backward& b, int sms) {   // ins x outs over rows, or its transpose
  Product q;
  const uint32_t k = (uint32_t)a.rows;
  q.p = b.across_out ? gemm_plan(a.outs, a.ins, k, a.dweight.type, sms) : gemm_plan(a.ins, a.outs, k, a.dweight.type, sms);
  const bool turned = q.p.turned;
  const Operand x = operand(a.x.data, a.ins, k, a.x.col_stride, a.x.row_stride, turned && !b.across_out);
  const Operand d = operand(b.dz.data, a.outs, k, b.dz.col_stride, b.dz.row_stride, turned && b.across_out);
  q.left = b.across_out ? d : x;
  q.right = b.across_out ? x : d;
  q.e = Epilogue{};
  q.e.out = a.dweight;
  if (b.across_out) std::swap(q.e.out.row_stride, q.e.out.col_stride);
  return q;
}
// Both, or the one that is wanted; the one of more blocks of k is the first.
struct Products {
  int n = 0;
  Product q[2];
  bool shared = false;   // in one launch
  Shared how{};
  size_t bytes(int sms) const {   // (launches that follow each other share scratch)
    if (shared) return q[0].bytes() + q[1].bytes() + chain_bytes(q[0], &q[1], sms);
    size_t most = 0;
    for (int i = 0; i < n; ++i) most = std::max(most, q[i].bytes() + chain_bytes(q[i], nullptr, sms));
    return most;
  }
};
Products backward_products(const LinearArgs& a, const Backward& b, int sms) {
  Products all;
  if (a.dx.data) all.q[all.n++] = dx_product(a, b, sms);
  if (a.dweight.data) all.q[all.n++] = dweight_product(a, b, sms);
  if (all.n == 2) {
    if (all.q[0].p.k_blocks < all.q[1].p.k_blocks) std::swap(all.q[0], all.q[1]);
    all.shared = share(all.q[0].p, all.q[1].p, sms, &all.how);
  }
  return all;
}

template <int TYPE>
void launch_dz(const LinearArgs& a, const Backward& b, float* sums, cudaStream_t stream) {
  note_launches(1);
  char* const to = b.own_dz ? b.dz.data : nullptr;
  const unsigned grid = b.across * b.blocks;
  if (b.vec == 8) launch_after(dz_kernel<TYPE, 8>, grid, 256, 0, stream, a.grad, a.pre, a.activation, to, b.pitch, a.rows, a.outs, b.per_block, sums);
  else launch_after(dz_kernel<TYPE, 1>, grid, 256, 0, stream, a.grad, a.pre, a.activation, to, b.pitch, a.rows, a.outs, b.per_block, sums);
}

}  // namespace

size_t linear_grad_scratch(const LinearArgs& a, int sms) {
  const Backward b = backward_of(a, nullptr, sms);
  return b.dz_bytes + b.sum_bytes + backward_products(a, b, sms).bytes(sms);
}

cudaError_t launch_linear_grad(const LinearArgs& a, char* scratch, int sms, cudaStream_t stream) {
  const Backward b = backward_of(a, scratch, sms);
  float* const sums = a.dbias.data ? reinterpret_cast<float*>(scratch + b.dz_bytes) : nullptr;
  char* const rest = scratch + b.dz_bytes + b.sum_bytes;
  const bool bf16 = a.x.type == ADAPM_BF16;
  if (b.own_dz || a.dbias.data) {
    if (bf16) launch_dz<ADAPM_BF16>(a, b, sums, stream);
    else launch_dz<ADAPM_F16>(a, b, sums, stream);
  }
  Products all = backward_products(a, b, sms);
  // the sums of dz's columns: beside the products where they leave blocks free
  ColumnSums beside{};
  if (a.dbias.data && all.shared && all.q[0].tiles() + all.q[1].tiles() < (uint64_t)sms) beside = ColumnSums{sums, b.blocks, a.outs, a.dbias};
  else if (a.dbias.data) launch_column_join(sums, b.blocks, a.outs, a.outs, a.dbias, VectorView{nullptr, ADAPM_F32}, stream);
  size_t at = 0;
  for (int i = 0; i < all.n; ++i) {
    Product& q = all.q[i];
    pack(q.left, q.right, rest + at, stream);
    at += q.bytes();
    if (all.shared && i == 0) continue;
    const cudaError_t err = launch_gemm(all.shared ? all.q[0] : q, all.shared ? &q : nullptr, all.how, beside, bf16, rest + at, a.st, sms, stream);
    if (err != cudaSuccess) return err;
    at = 0;
  }
  return cudaSuccess;
}

}  // namespace adapm
