// push_grads: the update of an embedding by its summed gradient rows.
//
//   g = scale * min(1, max_norm / norm) * rows[u]
//   SGD      value(worker, keys[u]) += -lr * g
//   AdaGrad  [theta | a] += [-lr * g / sqrt(a + g*g + eps) | g*g]
//
// The keys come distinct and ascending (embed_grad), so there is nothing to
// sort or to sum: a row group per key looks the target up as the push does
// (push_kernels.cuh) and applies the row it forms on the way.  Clipping is the
// factor, read from the norm's device word, so clipped rows never travel.
// Bound by memory: the gradient row in, the value row in and out (400,003
// AdaGrad rows of 2 x 256 floats: 2.05 GB in 325 us, 6.3 TB/s); few rows by the
// chain key -> map entry -> rows (20,011 of 64 floats 6 us).
#include "embed.cuh"
#include "push_kernels.cuh"

namespace adapm {

namespace {

__device__ __forceinline__ float4 get4(const float* row, uint32_t c, uint32_t dim, bool vec) {
  if (vec && c + 4 <= dim) return *reinterpret_cast<const float4*>(row + c);
  float x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = c + j < dim ? row[c + j] : 0.f;
  return make_float4(x[0], x[1], x[2], x[3]);
}

// Elements c .. c + 3 of a row; those behind the gradient's dim become -0, which
// changes no value it is added to (0 times a NaN or infinite factor would).
__device__ __forceinline__ float4 keep_dim(float4 v, uint32_t c, uint32_t dim) {
  return make_float4(c < dim ? v.x : -0.f, c + 1 < dim ? v.y : -0.f, c + 2 < dim ? v.z : -0.f,
                     c + 3 < dim ? v.w : -0.f);
}

// Blocks per SM that the registers are cut for: 400,003 AdaGrad rows of 2 x 256
// floats (C = 4) 363 us at two, 325 at three, 327 at four; 500,000 of 2 x 100
// (C = 2) 284 at three, 229 at four, 254 at five; 300,000 SGD rows of 300 (C =
// 3) 286 at three, 300 at four.
constexpr int update_blocks_per_sm(int C) { return C >= 8 ? 2 : (C >= 3 ? 3 : 4); }

template <int G, int C, int R, int SRC>
__global__ void __launch_bounds__(kThreads, update_blocks_per_sm(C)) push_grads_kernel(Store s, const RowUpdate u, bool vec) {
  after_previous();
  const int lane = threadIdx.x & (G - 1);
  const unsigned gmask = group_mask<G>();
  const uint32_t D4 = s.D >> 2;
  const uint32_t T4 = SRC == kSrcAda ? D4 / 2 : D4;
  constexpr int CT = SRC == kSrcAda ? C / 2 : C;   // vectors of a gradient row per lane
  s.par = s.st->par;
  if (sort_failed(s.st)) return;
  const bool any_replica = s.own == nullptr && s.st->live > 0;
  const float factor = u.norm != nullptr ? clip_factor(u.scale, *u.norm, u.max_norm) : u.scale;
  const float4* main4 = reinterpret_cast<const float4*>(s.main);
  const float4* val4 = reinterpret_cast<const float4*>(s.val);
  const float4* acc4 = reinterpret_cast<const float4*>(s.acc);
  bool bad = false, order = false;
  const uint64_t step = group_count<G>() * R;
  for (uint64_t base = group_id<G>() * R; base < u.n; base += step) {
    uint32_t k[R];
    Target t[R];
    float4 d[R][C];
    uint32_t prev = base > 0 ? u.keys[base - 1] : kNoKey;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      k[r] = base + r < u.n ? u.keys[base + r] : kNoKey;
      const uint32_t key = k[r];
      if (key >= s.K) {
        bad |= key != kNoKey;
        k[r] = kNoKey;
      } else if (base + r > 0 && prev >= key) {   // (also behind skipped keys, which sort last)
        order = true;
        k[r] = kNoKey;
      }
      prev = key;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      t[r] = Target{-2, REP_ALIAS, 0u};
      if (k[r] != kNoKey) t[r] = look_target(s, u.worker, k[r], any_replica);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float* row = u.rows + (base + r) * u.dim;
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const uint32_t q = lane + c * G;
        d[r][c] = k[r] != kNoKey && 4 * q < u.dim ? get4(row, 4 * q, u.dim, vec) : f4zero();
      }
      if (SRC == kSrcAda && k[r] != kNoKey) {   // the accumulators before
        const bool own = t[r].slot >= 0 && (t[r].state & REP_OWNVAL);
        const float4* from = own ? val4 + (uint64_t)t[r].slot * D4 : main4 + (uint64_t)k[r] * D4;
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          const uint32_t q = lane + c * G;
          d[r][CT + c] = q < T4 ? from[T4 + q] : f4zero();
          if (t[r].slot >= 0 && rep_adds(t[r].state) && q < T4)
            d[r][CT + c] = f4add(d[r][CT + c], acc4[(uint64_t)t[r].slot * D4 + T4 + q]);
        }
      }
    }
    __syncwarp(gmask);   // every lane has read the states
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (k[r] == kNoKey) continue;   // (uniform over the group)
      if (lane == 0) mark_target(s, u.worker, k[r], t[r]);
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const float4 g = f4mul(d[r][c], factor);
        if (SRC == kSrcAda) {
          d[r][c] = ada_theta4(g, d[r][CT + c], u.lr, u.eps);
          d[r][CT + c] = f4square(g);
        } else {
          d[r][c] = keep_dim(f4mul(g, -u.lr), 4 * (lane + c * G), u.dim);
        }
      }
      apply_sum<G, C, SRC>(s, k[r], t[r], d[r], lane, gmask);
    }
  }
  if (lane == 0 && (bad || order)) set_error(s.st, (bad ? ERR_KEY_RANGE : 0u) | (order ? ERR_KEY_ORDER : 0u));
}

template <int SRC>
void launch_source(const Store& s, const RowUpdate& u, bool vec, int sms, cudaStream_t stream) {
  dispatch_push_gc(s.D / 4, SRC == kSrcAda, [&](auto Gc, auto Cc) {
    constexpr int G = decltype(Gc)::value, C = decltype(Cc)::value;
    if constexpr (SRC != kSrcAda || C % 2 == 0) {
      constexpr int R = push_rows_in_flight(C);
      launch_after(push_grads_kernel<G, C, R, SRC>, grid_for((u.n + R - 1) / R, G, sms), kThreads, 0, stream, s, u,
                   vec);
    }
  });
}

}  // namespace

void launch_push_grads(const Store& s, const RowUpdate& u, int sms, cudaStream_t stream) {
  if (u.n == 0) return;
  const bool vec = reinterpret_cast<uintptr_t>(u.rows) % 16 == 0 && u.dim % 4 == 0;
  note_launches(1);
  if (u.adagrad) launch_source<kSrcAda>(s, u, vec, sms, stream);
  else launch_source<kSrcSgd>(s, u, vec, sms, stream);
}

}  // namespace adapm
