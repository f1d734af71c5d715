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
// staged in shared memory kTile at a time: kThreads / kOwn threads share the
// others of one key.  n^2 comparisons over the whole GPU in one launch and
// without a wait between blocks, where a radix sort of so few keys is a chain
// of passes in one block.
constexpr int kOwn = 32, kTile = 4096;

__global__ void __launch_bounds__(kThreads) count_sort_kernel(const TokenView t, uint64_t K, uint32_t* skeys,
                                                              uint32_t* spos, DevState* st) {
  after_previous();
  constexpr int NS = kThreads / kOwn;
  __shared__ uint32_t tile[kTile];
  __shared__ uint32_t cnt[NS][kOwn];
  const uint32_t n = (uint32_t)t.n;
  const int o = threadIdx.x % kOwn, part = threadIdx.x / kOwn;
  const uint32_t i = blockIdx.x * kOwn + o;
  uint32_t mine = i < n ? token_key(t, i, K) : kNoKey;
  const bool bad = mine == kBadKey;
  if (bad) mine = kNoKey;
  uint32_t before = 0;
  for (uint32_t t0 = 0; t0 < n; t0 += kTile) {
    const uint32_t len = n - t0 < (uint32_t)kTile ? n - t0 : (uint32_t)kTile;
    __syncthreads();
    for (uint32_t j = threadIdx.x; j < len; j += kThreads) {
      const uint32_t k = token_key(t, t0 + j, K);
      tile[j] = k == kBadKey ? kNoKey : k;
    }
    __syncthreads();
    for (uint32_t j = part; j < len; j += NS) {
      const uint32_t k = tile[j];
      before += (k < mine || (k == mine && t0 + j < i)) ? 1u : 0u;
    }
  }
  cnt[part][o] = before;
  __syncthreads();
  if (part == 0 && i < n) {
    uint32_t at = 0;
#pragma unroll
    for (int p = 0; p < NS; ++p) at += cnt[p][o];
    skeys[at] = mine;
    spos[at] = i;
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
