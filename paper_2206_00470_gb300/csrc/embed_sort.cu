// Keys of a batch of tokens, without gaps or sorted with their positions, for
// embed_grad.
#include "embed.cuh"
#include "rowgroup.cuh"

namespace adapm {

namespace {

__global__ void __launch_bounds__(kThreads) copy_tokens_kernel(const TokenView t, uint64_t K, uint32_t* out,
                                                               DevState* st) {
  after_previous();
  bool bad = false;
  for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < t.n; i += (uint64_t)gridDim.x * kThreads) {
    const uint32_t k = token_key(t, i, K);
    bad |= k == kBadKey;
    out[i] = k == kBadKey ? kNoKey : k;
  }
  if (__syncthreads_or(bad) && threadIdx.x == 0) set_error(st, ERR_KEY_RANGE);
}

// Position of key i in the stable order: the keys below it, and those equal
// to it that come first.  Every block counts for kOwn keys against all n,
// staged in shared memory kTile at a time: kSlices threads share the others of
// kPer keys, four a load.  n^2 comparisons over the whole GPU in one launch and
// without a wait between blocks, where a radix sort of so few keys is a chain
// of passes in one block.
constexpr int kPer = 2, kSlices = 16, kOwn = kThreads / kSlices * kPer, kTile = 4096;

__global__ void __launch_bounds__(kThreads) count_sort_kernel(const TokenView t, uint64_t K, uint32_t* skeys,
                                                              uint32_t* spos, DevState* st) {
  after_previous();
  constexpr int NO = kThreads / kSlices;   // threads that hold different keys
  __shared__ __align__(16) uint32_t tile[kTile];
  __shared__ uint32_t cnt[kSlices][kOwn];
  const uint32_t n = (uint32_t)t.n;
  const int o = threadIdx.x % NO, part = threadIdx.x / NO;
  const uint32_t own0 = blockIdx.x * kOwn;
  uint32_t mine[kPer], before[kPer];
  bool bad = false;
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const uint32_t i = own0 + q * NO + o;
    mine[q] = i < n ? token_key(t, i, K) : kNoKey;
    bad |= mine[q] == kBadKey;
    if (mine[q] == kBadKey) mine[q] = kNoKey;
    before[q] = 0;
  }
  for (uint32_t t0 = 0; t0 < n; t0 += kTile) {
    const uint32_t len = n - t0 < (uint32_t)kTile ? n - t0 : (uint32_t)kTile;
    __syncthreads();
#pragma unroll 4
    for (uint32_t j = threadIdx.x; j < len; j += kThreads) {
      const uint32_t k = token_key(t, t0 + j, K);
      tile[j] = k == kBadKey ? kNoKey : k;
    }
    __syncthreads();
    // keys [lo, hi) of the tile, a multiple of four from lo: below mine, or
    // (before the block's own) not above it
    auto count = [&](uint32_t lo, uint32_t hi, bool equal) {
      const uint32_t whole = lo + (hi - lo) / 4 * 4;
#pragma unroll 4
      for (uint32_t j = lo + 4 * part; j < whole; j += 4 * kSlices) {
        const uint4 v = *reinterpret_cast<const uint4*>(tile + j);
        const uint32_t k[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int q = 0; q < kPer; ++q) before[q] += equal ? (k[e] <= mine[q]) : (k[e] < mine[q]);
      }
      for (uint32_t j = whole + part; j < hi; j += kSlices)
#pragma unroll
        for (int q = 0; q < kPer; ++q) before[q] += equal ? (tile[j] <= mine[q]) : (tile[j] < mine[q]);
    };
    // (own0 and the tiles' starts are multiples of kOwn)
    const uint32_t a = own0 < t0 ? 0u : (own0 - t0 < len ? own0 - t0 : len);
    const uint32_t b = own0 + kOwn < t0 ? 0u : (own0 + kOwn - t0 < len ? own0 + kOwn - t0 : len);
    count(0, a, true);
    count(b, len, false);
    for (uint32_t j = a + part; j < b; j += kSlices)
#pragma unroll
      for (int q = 0; q < kPer; ++q) {
        const uint32_t i = own0 + q * NO + o;
        before[q] += tile[j] < mine[q] || (tile[j] == mine[q] && t0 + j < i);
      }
  }
#pragma unroll
  for (int q = 0; q < kPer; ++q) cnt[part][q * NO + o] = before[q];
  __syncthreads();
  if (threadIdx.x < kOwn && own0 + threadIdx.x < n) {
    uint32_t at = 0;
#pragma unroll
    for (int p = 0; p < kSlices; ++p) at += cnt[p][threadIdx.x];
    const uint32_t k = token_key(t, own0 + threadIdx.x, K);
    skeys[at] = k == kBadKey ? kNoKey : k;
    spos[at] = own0 + threadIdx.x;
  }
  if (__syncthreads_or(bad) && threadIdx.x == 0) set_error(st, ERR_KEY_RANGE);
}

}  // namespace

void launch_copy_tokens(const TokenView& t, uint64_t K, uint32_t* out, DevState* st, int sms, cudaStream_t stream) {
  note_launches(1);
  launch_after(copy_tokens_kernel, grid_for(t.n, 1, sms), kThreads, 0, stream, t, K, out, st);
}

void launch_count_sort(const TokenView& t, uint64_t K, uint32_t* skeys, uint32_t* spos, DevState* st,
                       cudaStream_t stream) {
  note_launches(1);
  launch_after(count_sort_kernel, (unsigned)((t.n + kOwn - 1) / kOwn), kThreads, 0, stream, t, K, skeys, spos, st);
}

}  // namespace adapm
