// Token embeddings: what the entry points (capi.cu) hand to the kernels of
// embed.cu, embed_sort.cu, embed_grad.cuh, push_grads.cu and grads.cu.
#pragma once

#include "internal.cuh"

namespace adapm {

constexpr uint32_t kBadKey = 0xFFFFFFFEu;   // an id outside [0, K); never a valid key (K < 2^32 - 1)

// n = outer * inner token ids (device memory).
struct TokenView {
  const void* ids;
  bool wide;      // 64-bit ids
  bool has_pad;
  bool flat;      // no gaps: id t is ids[t]
  int64_t pad;
  uint32_t inner;
  int64_t outer_stride, inner_stride;
  uint64_t n;
};

// The rows that belong to n tokens, in elements (device memory).
struct RowView {
  char* data;
  int type;       // ADAPM_F32, _F16, _BF16
  bool flat;      // no gaps: row t begins at t * inner_stride
  uint32_t inner;
  int64_t outer_stride, inner_stride;
};

#ifdef __CUDACC__
// Where token t's id is, the id, and its key: kNoKey for padding, kBadKey for an
// id that is none.
__device__ __forceinline__ int64_t token_at(const TokenView& v, uint32_t t) {
  if (v.flat) return t;
  const uint32_t o = t / v.inner, i = t - o * v.inner;
  return (int64_t)o * v.outer_stride + (int64_t)i * v.inner_stride;
}
__device__ __forceinline__ int64_t token_id(const TokenView& v, uint32_t t) {
  const int64_t at = token_at(v, t);
  return v.wide ? static_cast<const int64_t*>(v.ids)[at] : (int64_t)static_cast<const uint32_t*>(v.ids)[at];
}
__device__ __forceinline__ uint32_t id_key(const TokenView& v, int64_t id, uint64_t K) {
  if (v.has_pad && id == v.pad) return kNoKey;
  return id >= 0 && id < (int64_t)K ? (uint32_t)id : kBadKey;
}
__device__ __forceinline__ uint32_t token_key(const TokenView& v, uint64_t t, uint64_t K) {
  return id_key(v, token_id(v, (uint32_t)t), K);
}
// First element of the row of token t.
__device__ __forceinline__ int64_t row_offset(const RowView& v, uint32_t t) {
  if (v.flat) return (int64_t)t * v.inner_stride;
  const uint32_t o = t / v.inner;
  return (int64_t)o * v.outer_stride + (int64_t)(t - o * v.inner) * v.inner_stride;
}
#endif

void launch_embed(const Store& s, uint32_t w, const TokenView& t, uint32_t dim, float scale, const RowView& out,
                  int sms, cudaStream_t stream);

// ---- gradient by sorted tokens ----------------------------------------------
// Sorted (key, position) pairs of a batch, or the two places they may be in
// (a push plan or the sort made in its place, as in PushArgs).
struct GradArgs {
  const uint32_t* skeys;
  const uint32_t* spos;
  const uint32_t* alt_keys;
  const uint32_t* alt_pos;
  const uint32_t* plan_word;   // null: no plan
  uint32_t plan_seq;
  uint32_t pad_key;   // a key to leave out, kNoKey: none
  uint64_t n;
  uint64_t K;
  RowView grad;
  uint32_t dim;
  float scale;
  uint32_t* keys;     // out: distinct keys, ascending, then kNoKey
  float* rows;        // out
  uint32_t* count;    // out
  uint32_t chunk;     // rows a group sums, of a span of (groups per block) chunks
  uint32_t* heads;    // per span: distinct keys that begin in it; null: counted where they are needed
  bool scanned;       // heads holds sums: per span the keys that begin before it, then all
  uint32_t* crossing; // per span: index of the key whose rows run past its end
  float* parts;       // per span: a head and a tail row of `dim` floats
  DevState* st;
};
struct GradPlan {     // sizes of a batch's scratch
  uint32_t chunk;
  uint64_t spans;
  bool count_heads;   // heads is needed,
  bool scan_heads;    // summed up by a launch of its own
};
GradPlan grad_plan(const GradArgs& a, int sms);
void launch_embed_grad(const GradArgs& a, const GradPlan& p, cudaStream_t stream);

// The keys of n tokens without gaps; ids that are none become kNoKey and are
// reported.
void launch_copy_tokens(const TokenView& t, uint64_t K, uint32_t* out, DevState* st, int sms, cudaStream_t stream);
// Stable sort of a few tokens' keys with their positions by counting, for
// each, the keys that go before it; bad ids sort as padding and are reported.
constexpr uint64_t kCountSort = 6144;
void launch_count_sort(const TokenView& t, uint64_t K, uint32_t* skeys, uint32_t* spos, DevState* st,
                       cudaStream_t stream);

// Stable sort of up to kTokenSort tokens' keys by their low `bits` bits with
// their positions.  keys / pos: two arrays of n each; the result is in those
// whose index is returned.  scratch: token_sort_words(n, bits) words.  Bad ids sort as
// padding and are reported.
constexpr int kTokenBits = 9;   // of a pass, at most
constexpr uint64_t kTokenSort = 1u << 19;
size_t token_sort_words(uint64_t n, int bits);
int token_sort(const TokenView& t, uint64_t K, int bits, uint32_t* const* keys, uint32_t* const* pos,
               uint32_t* scratch, DevState* st, cudaStream_t stream);

// ---- update by gradient rows --------------------------------------------------
struct RowUpdate {
  const uint32_t* keys;
  const float* rows;
  uint64_t n;
  uint32_t dim;
  uint32_t worker;
  bool adagrad;
  float lr, eps, scale, max_norm;
  const float* norm;   // null: no clipping
};
void launch_push_grads(const Store& s, const RowUpdate& u, int sms, cudaStream_t stream);

// ---- norm and clipping over many tensors -----------------------------------------
struct GradTensor {
  const char* in;
  char* out;              // clipping only
  const uint32_t* live;   // null, or the number of live rows of row_len elements
  uint64_t count;
  uint32_t row_len;
  uint8_t type, out_type;
};
size_t norm_scratch_doubles(uint64_t n, int sms);
void launch_grad_norm(const GradTensor* t, uint64_t n, float scale, double* part, float* norm, DevState* st, int sms,
                      cudaStream_t stream);
void launch_clip_grads(const GradTensor* t, uint64_t n, float scale, float max_norm, const float* norm, bool in_place,
                       int sms, cudaStream_t stream);

#ifdef __CUDACC__
// scale times what clipping to max_norm multiplies a gradient by.
__device__ __forceinline__ float clip_factor(float scale, float norm, float max_norm) {
  return norm <= max_norm ? scale : scale * (max_norm / norm);
}
#endif

}  // namespace adapm
