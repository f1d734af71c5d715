// Keys of a batch of tokens, without gaps or sorted with their positions, for
// embed_grad.
#include "embed.cuh"
#include "radix.cuh"
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
// staged in shared memory: kSlices threads share the others of kPer keys, four
// a load.  n^2 comparisons over the whole GPU in one launch and without a wait
// between blocks, where a radix sort of so few keys is a chain of passes.
// Bound by latency up to 2,000 tokens (3.8 us), by the comparisons above: 4,096
// tokens 6.1 us, 6,000 9.5 us, 8,192 15 us.  The token sort below takes 12 us
// for any of these and needs grad_heads' launch; one block's sort (sort_small)
// 9, 13.5, 20 and 21 us.
constexpr int kThreadsC = 256, kPer = 2, kSlices = 32, kOwn = kThreadsC / kSlices * kPer;

__global__ void __launch_bounds__(kThreadsC) count_sort_kernel(const TokenView t, uint64_t K, uint32_t* skeys,
                                                              uint32_t* spos, DevState* st) {
  after_previous();
  constexpr int NO = kThreadsC / kSlices;   // threads that hold different keys
  __shared__ __align__(16) uint32_t all[kCountSort];
  __shared__ uint32_t cnt[kSlices][kOwn];
  const uint32_t n = (uint32_t)t.n;
  const int o = threadIdx.x % NO, part = threadIdx.x / NO;
  bool bad = false;
  constexpr int B = 8;   // ids in flight per thread
  for (uint32_t j0 = threadIdx.x; j0 < n; j0 += B * kThreadsC) {
    int64_t id[B];
    if (t.wide) {
#pragma unroll
      for (int e = 0; e < B; ++e)
        id[e] = j0 + e * kThreadsC < n ? static_cast<const int64_t*>(t.ids)[token_at(t, j0 + e * kThreadsC)] : 0;
    } else {
#pragma unroll
      for (int e = 0; e < B; ++e)
        id[e] = j0 + e * kThreadsC < n ? static_cast<const uint32_t*>(t.ids)[token_at(t, j0 + e * kThreadsC)] : 0;
    }
#pragma unroll
    for (int e = 0; e < B; ++e) {
      const uint32_t k = id_key(t, id[e], K);
      if (j0 + e * kThreadsC >= n) break;
      bad |= k == kBadKey;
      all[j0 + e * kThreadsC] = k == kBadKey ? kNoKey : k;
    }
  }
  __syncthreads();
  // the block's own keys [a, b), the thread's among them
  const uint32_t a = blockIdx.x * kOwn, b = a + kOwn < n ? a + kOwn : n;
  uint32_t mine[kPer], before[kPer];
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    mine[q] = a + q * NO + o < n ? all[a + q * NO + o] : kNoKey;
    before[q] = 0;
  }
  // keys [lo, hi), lo a multiple of four: those below mine, or (in front of the
  // block's own) not above it
  auto count = [&](uint32_t lo, uint32_t hi, bool equal) {
    const uint32_t whole = lo + (hi - lo) / 4 * 4;
#pragma unroll 4
    for (uint32_t j = lo + 4 * part; j < whole; j += 4 * kSlices) {
      const uint4 v = *reinterpret_cast<const uint4*>(all + j);
      const uint32_t k[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int q = 0; q < kPer; ++q) before[q] += equal ? (k[e] <= mine[q]) : (k[e] < mine[q]);
    }
    for (uint32_t j = whole + part; j < hi; j += kSlices)
#pragma unroll
      for (int q = 0; q < kPer; ++q) before[q] += equal ? (all[j] <= mine[q]) : (all[j] < mine[q]);
  };
  count(0, a, true);
  if (b < n) count(b, n, false);   // (b is then a multiple of kOwn)
  for (uint32_t j = a + part; j < b; j += kSlices)
#pragma unroll
    for (int q = 0; q < kPer; ++q) before[q] += all[j] < mine[q] || (all[j] == mine[q] && j < a + q * NO + o);
#pragma unroll
  for (int q = 0; q < kPer; ++q) cnt[part][q * NO + o] = before[q];
  __syncthreads();
  if (threadIdx.x < kOwn && a + threadIdx.x < n) {
    uint32_t at = 0;
#pragma unroll
    for (int p = 0; p < kSlices; ++p) at += cnt[p][threadIdx.x];
    skeys[at] = all[a + threadIdx.x];
    spos[at] = a + threadIdx.x;
  }
  if (blockIdx.x == 0 && __syncthreads_or(bad) && threadIdx.x == 0) set_error(st, ERR_KEY_RANGE);
}

// ---------------------------------------------------------------------------
// Token sort: a stable radix sort of up to kTokenSort tokens in one launch per
// pass of kTokenBits bits and one in front.  Every block owns a tile of
// consecutive items and finds the places of its own from a table (digit x
// tile) of the items that every tile holds, by summing the table's rows: no
// scan launch, no wait between blocks.  While it moves its items it counts
// them into the next pass's table (packed 16-bit counts; a tile holds at most
// 4096).  The first pass reads the tokens themselves, in whatever layout they
// have.  Bound by the latency of its launches, 3.5 to 8 us each.
//
// Grid sort (sort.cu) -> this, tokens of 1M keys: 16,384 26 -> 13.5 us, 65,536
// 31 -> 18, 131,072 31 -> 21, 262,144 34 -> 28, 524,288 50 -> 40; of 250,000
// keys 524,288 37 -> 34; 2^20, in tiles of 8192, 69 both.  (Digits of 10 bits
// take longer per launch than they save launches: 65,536 22 us, of 11 bits 24.)
// ---------------------------------------------------------------------------
constexpr uint32_t kTilesMost = 128;

struct TokenPass {
  const uint32_t* keys;   // null: the tokens
  const uint32_t* pos;
  uint32_t* keys_out;
  uint32_t* pos_out;
  const uint16_t* table;  // counts of this pass's digits
  uint32_t* next;         // packed counts of the next pass's, null: none
  uint32_t n, stride;     // stride: tiles of a table row, a multiple of eight
  int shift, bits, next_bits;
};

// The items of a thread: warp w owns ITEMS * 32 consecutive ones, 32 a round.
template <int ITEMS>
__device__ __forceinline__ uint32_t item_at(uint32_t tile0, int it) {
  return tile0 + ((threadIdx.x / 32) * ITEMS + it) * 32 + (threadIdx.x & 31);
}
template <int ITEMS>
__device__ __forceinline__ bool load_tokens(const TokenView& t, uint64_t K, uint32_t tile0, uint32_t (&key)[ITEMS]) {
  int64_t id[ITEMS];
  const uint32_t n = (uint32_t)t.n;
  if (t.wide) {
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
      const uint32_t i = item_at<ITEMS>(tile0, it);
      id[it] = i < n ? static_cast<const int64_t*>(t.ids)[token_at(t, i)] : 0;
    }
  } else {
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
      const uint32_t i = item_at<ITEMS>(tile0, it);
      id[it] = i < n ? static_cast<const uint32_t*>(t.ids)[token_at(t, i)] : 0;
    }
  }
  bool bad = false;
#pragma unroll
  for (int it = 0; it < ITEMS; ++it) {
    key[it] = id_key(t, id[it], K);
    if (key[it] == kBadKey) {
      key[it] = kNoKey;
      bad = true;
    }
  }
  return bad;
}

// The first pass's table, and the next ones cleared.
template <int NT, int ITEMS>
__global__ void __launch_bounds__(NT) token_count_kernel(const TokenView t, uint64_t K, uint16_t* table,
                                                                uint32_t* clear, uint32_t clear_words, uint32_t stride,
                                                                int bits, DevState* st) {
  after_previous();
  extern __shared__ __align__(16) unsigned char dsm[];
  uint32_t* cnt = reinterpret_cast<uint32_t*>(dsm);
  const uint32_t digits = 1u << bits, tile0 = blockIdx.x * (NT * ITEMS);
  for (uint32_t i = blockIdx.x * NT + threadIdx.x; i < clear_words; i += gridDim.x * NT) clear[i] = 0u;
  uint32_t key[ITEMS];
  const bool bad = load_tokens<ITEMS>(t, K, tile0, key);
  for (uint32_t d = threadIdx.x; d < digits; d += NT) cnt[d] = 0u;
  __syncthreads();
#pragma unroll
  for (int it = 0; it < ITEMS; ++it) {
    const bool in = item_at<ITEMS>(tile0, it) < (uint32_t)t.n;
    const uint32_t d = in ? key[it] & (digits - 1) : digits;
    const uint32_t peers = __match_any_sync(0xFFFFFFFFu, d);
    if (in && (peers & lanemask_lt()) == 0u) atomicAdd(cnt + d, (uint32_t)__popc(peers));
  }
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < digits; d += NT) table[d * stride + blockIdx.x] = (uint16_t)cnt[d];
  if (blockIdx.x == 0)   // tiles of the row that do not exist
    for (uint32_t d = threadIdx.x; d < digits; d += NT)
      for (uint32_t b = gridDim.x; b < stride; ++b) table[d * stride + b] = 0;
  if (__syncthreads_or(bad) && threadIdx.x == 0) set_error(st, ERR_KEY_RANGE);
}

// Dynamic shared memory of token_pass: the digits' places, the warps' digit
// counts, and the tile in order, so that a digit's items leave in one run
// (131,072 tokens 17 to 23 us so, 19 to 26 item by item; 262,144 22 to 29, 25
// to 35).
template <int NT, int ITEMS>
size_t token_smem(int bits) {
  return (((size_t)4 + NT / 16) << bits) + (size_t)NT * ITEMS * 8;
}

template <int NT, int ITEMS>
__global__ void __launch_bounds__(NT) token_pass_kernel(const TokenView t, uint64_t K, const TokenPass p) {
  after_previous();
  extern __shared__ __align__(16) unsigned char dsm[];
  const uint32_t digits = 1u << p.bits;
  uint32_t* place = reinterpret_cast<uint32_t*>(dsm);
  uint16_t* wcnt = reinterpret_cast<uint16_t*>(place + digits);   // [warp][digit]
  __shared__ uint32_t scan[(NT / 32)];
  const uint32_t tile0 = blockIdx.x * (NT * ITEMS);
  const int warp = threadIdx.x / 32;
  uint32_t key[ITEMS], pos[ITEMS], rank[ITEMS];
  if (p.keys == nullptr) {
    load_tokens<ITEMS>(t, K, tile0, key);
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) pos[it] = item_at<ITEMS>(tile0, it);
  } else {
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
      const uint32_t i = item_at<ITEMS>(tile0, it);
      key[it] = i < p.n ? p.keys[i] : kNoKey;
      pos[it] = i < p.n ? p.pos[i] : 0u;
    }
  }
  // items of the thread's digits (the next ones to each other): anywhere, and in
  // the tiles before this one
  constexpr int J = (1 << kTokenBits) / NT > 1 ? (1 << kTokenBits) / NT : 1;
  const uint32_t per = digits > (uint32_t)NT ? J : 1, d0 = threadIdx.x * per;
  uint32_t all[J], before[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    all[j] = before[j] = 0;
    if (j >= (int)per || d0 + j >= digits) continue;
    const uint4* row = reinterpret_cast<const uint4*>(p.table + (uint64_t)(d0 + j) * p.stride);
#pragma unroll 8
    for (uint32_t q = 0; q < p.stride / 8; ++q) {
      const uint4 v = row[q];
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t b = 8 * q + 2 * e, lo = w[e] & 0xFFFFu, hi = w[e] >> 16;
        all[j] += lo + hi;
        before[j] += (b < blockIdx.x ? lo : 0u) + (b + 1 < blockIdx.x ? hi : 0u);
      }
    }
  }
  for (uint32_t i = threadIdx.x; i < digits * (NT / 32) / 2; i += NT) reinterpret_cast<uint32_t*>(wcnt)[i] = 0u;
  __syncthreads();
  // ranks within the warp
  uint32_t peers[ITEMS];
#pragma unroll
  for (int it = 0; it < ITEMS; ++it)
    peers[it] = digit_peers((key[it] >> p.shift) & (digits - 1), item_at<ITEMS>(tile0, it) < p.n, p.bits);
#pragma unroll
  for (int it = 0; it < ITEMS; ++it) {
    const bool in = item_at<ITEMS>(tile0, it) < p.n;
    uint16_t* c = wcnt + warp * digits + ((key[it] >> p.shift) & (digits - 1));
    const uint32_t have = in ? *c : 0u;
    rank[it] = have + __popc(peers[it] & lanemask_lt());
    __syncwarp();
    if (in && (peers[it] & lanemask_lt()) == 0u) *c = (uint16_t)(have + __popc(peers[it]));
    __syncwarp();
  }
  // where the digit's items of this tile go: behind those of lower digits and
  // of the tiles before, warp by warp
  uint32_t sum = 0, total;
#pragma unroll
  for (int j = 0; j < J; ++j) sum += all[j];
  uint32_t base = block_exclusive_scan<NT>(sum, &total, scan);   // (a barrier: the warps' counts are final)
  uint32_t h[J][NT / 32], mine = 0;
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
      h[j][w] = j < (int)per && d0 + j < digits ? wcnt[w * digits + d0 + j] : 0u;
      mine += h[j][w];
    }
  uint32_t run = block_exclusive_scan<NT>(mine, &total, scan);   // in the ordered tile
#pragma unroll
  for (int j = 0; j < J; ++j) {
    if (j >= (int)per || d0 + j >= digits) continue;
    place[d0 + j] = base + before[j] - run;   // (of the ordered tile's begin)
    base += all[j];
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
      wcnt[w * digits + d0 + j] = (uint16_t)run;
      run += h[j][w];
    }
  }
  __syncthreads();
  uint32_t* tk = reinterpret_cast<uint32_t*>(wcnt + digits * (NT / 32));
  uint32_t* tp = tk + NT * ITEMS;
#pragma unroll
  for (int it = 0; it < ITEMS; ++it)
    if (item_at<ITEMS>(tile0, it) < p.n) {
      const uint32_t i = wcnt[warp * digits + ((key[it] >> p.shift) & (digits - 1))] + rank[it];
      tk[i] = key[it];
      tp[i] = pos[it];
    }
  __syncthreads();
  const uint32_t len = p.n - tile0 < (uint32_t)(NT * ITEMS) ? p.n - tile0 : (uint32_t)(NT * ITEMS);
  for (uint32_t i0 = 0; i0 < len; i0 += NT) {   // block-uniform
    const uint32_t i = i0 + threadIdx.x;
    const bool in = i < len;
    const uint32_t k = in ? tk[i] : 0u;
    const uint32_t at = in ? place[(k >> p.shift) & (digits - 1)] + i : 0u;
    if (in) {
      p.keys_out[at] = k;
      p.pos_out[at] = tp[i];
    }
    if (p.next != nullptr) {
      const uint32_t nd = (k >> (p.shift + p.bits)) & ((1u << p.next_bits) - 1);
      const uint32_t cell = in ? nd * p.stride + at / (NT * ITEMS) : 0xFFFFFFFFu;
      const uint32_t same = __match_any_sync(0xFFFFFFFFu, cell);
      if (in && (same & lanemask_lt()) == 0u) atomicAdd(p.next + cell / 2, (uint32_t)__popc(same) << (16 * (cell & 1)));
    }
  }
}

// Passes of a sort by `bits` bits.  Every thread of a block sums its digits' rows
// of the table, a load per eight tiles.  A pass of 9 bits has two digits per
// thread of a block of 256, so its sums are twice a pass of 8 bits' where rows
// are long; up to 16,384 tokens a row is four loads at most, and above 131,072 a
// block has 512 threads, a digit each: 9 bits there, else up to 8.  17 and 18 bits, two passes against three: 8,192
// tokens 10 and 12 us, 16,384 12.5 and 13.5, 262,144 26 and 28, 524,288 34 and
// 42; but 65,536 21 and 18, 131,072 23 and 20.
int token_passes(uint64_t n, int bits) {
  const int most = n <= 16384 || n > 131072 ? kTokenBits : 8;
  return (bits + most - 1) / most;
}

template <int NT, int ITEMS>
int token_sort_items(const TokenView& t, uint64_t K, int bits, uint32_t* const* keys, uint32_t* const* pos,
                     uint32_t* scratch, DevState* st, cudaStream_t stream) {
  const int passes = token_passes(t.n, bits), each = (bits + passes - 1) / passes;
  const uint32_t tiles = (uint32_t)((t.n + NT * ITEMS - 1) / (NT * ITEMS)), stride = (tiles + 7) / 8 * 8;
  const uint32_t words = (stride << each) / 2;   // of a table
  // the kernel's dynamic shared-memory limit is a per-device attribute
  static bool attr_set[64] = {false};
  int dev = 0;
  cudaGetDevice(&dev);
  if (token_smem<NT, ITEMS>(kTokenBits) > 48 * 1024 && (dev < 0 || dev >= 64 || !attr_set[dev])) {
    cudaFuncSetAttribute(token_pass_kernel<NT, ITEMS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                         (int)token_smem<NT, ITEMS>(kTokenBits));
    if (dev >= 0 && dev < 64) attr_set[dev] = true;
  }
  note_launches(1 + passes);
  launch_after(token_count_kernel<NT, ITEMS>, tiles, NT, sizeof(uint32_t) << each, stream, t, K,
               reinterpret_cast<uint16_t*>(scratch), scratch + words, (uint32_t)(passes - 1) * words, stride, each, st);
  for (int i = 0; i < passes; ++i) {
    TokenPass p{};
    p.keys = i == 0 ? nullptr : keys[(i - 1) & 1];
    p.pos = i == 0 ? nullptr : pos[(i - 1) & 1];
    p.keys_out = keys[i & 1];
    p.pos_out = pos[i & 1];
    p.table = reinterpret_cast<const uint16_t*>(scratch + i * words);
    p.next = i + 1 < passes ? scratch + (i + 1) * words : nullptr;
    p.n = (uint32_t)t.n;
    p.stride = stride;
    p.shift = i * each;
    p.bits = p.next_bits = each;
    launch_after(token_pass_kernel<NT, ITEMS>, tiles, NT, token_smem<NT, ITEMS>(each), stream, t, K, p);
  }
  return (passes - 1) & 1;
}

}  // namespace

void launch_copy_tokens(const TokenView& t, uint64_t K, uint32_t* out, DevState* st, int sms, cudaStream_t stream) {
  note_launches(1);
  launch_after(copy_tokens_kernel, grid_for(t.n, 1, sms), kThreads, 0, stream, t, K, out, st);
}

void launch_count_sort(const TokenView& t, uint64_t K, uint32_t* skeys, uint32_t* spos, DevState* st,
                       cudaStream_t stream) {
  note_launches(1);
  launch_after(count_sort_kernel, (unsigned)((t.n + kOwn - 1) / kOwn), kThreadsC, 0, stream, t, K, skeys, spos, st);
}

// Tiles of 512 tokens, doubled until there are at most kTilesMost.
uint32_t token_tile(uint64_t n) {
  uint32_t tile = 512;
  while ((uint64_t)tile * kTilesMost < n) tile *= 2;
  return tile;
}

size_t token_sort_words(uint64_t n, int bits) {
  const int passes = token_passes(n, bits), each = (bits + passes - 1) / passes;
  const uint64_t tile = token_tile(n), tiles = (n + tile - 1) / tile;
  return (size_t)passes * (((tiles + 7) / 8 * 8) << each) / 2;
}

int token_sort(const TokenView& t, uint64_t K, int bits, uint32_t* const* keys, uint32_t* const* pos,
               uint32_t* scratch, DevState* st, cudaStream_t stream) {
  switch (token_tile(t.n)) {
    case 512: return token_sort_items<256, 2>(t, K, bits, keys, pos, scratch, st, stream);
    case 1024: return token_sort_items<256, 4>(t, K, bits, keys, pos, scratch, st, stream);
    case 2048: return token_sort_items<512, 4>(t, K, bits, keys, pos, scratch, st, stream);
    default: return token_sort_items<512, 8>(t, K, bits, keys, pos, scratch, st, stream);
  }
}

}  // namespace adapm
