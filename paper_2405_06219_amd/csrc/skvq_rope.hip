// skvq_rope_apply: rotary positions of queries and keys in any strided order.
//
// Bound by memory: every value is read and written once, 3 flops each.  A workgroup takes up to four
// tokens and all heads of both tensors: cosine and sine of its (token, pair)s are computed once, by one
// thread each, and kept in LDS for rope_walk.
#include <hip/hip_runtime.h>

#include "skvq_paged.h"

namespace skvq {
namespace {

struct RopeSide {
  const void *x;
  void *y;
  long long xb, xt, xh, yb, yt, yh;
};
struct RopeArgs {
  RopeSide side[2];  // (the second unused where n_heads == first_heads)
  int first_heads, n_heads;
  int head_dim, tokens_per_group, copy_rest;
  unsigned n_tokens, total;  // tokens per sequence; over the batch
  const int *positions;
  long long positions_batch;
  int start;
  float sign;
};

// V: channels per access, 16 bytes' worth or 1.
template <class T, int V, bool STREAM>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(const RopeTable tab, const RopeArgs a) {
  __shared__ float2 cs[kRopeMaxTokens][kRopeMaxPairs];
  const int half = tab.half, n_here = a.tokens_per_group;
  const unsigned first = blockIdx.x * (unsigned)n_here;
  for (int x = threadIdx.x; x < n_here * half; x += kRopeThreads) {
    const int k = x / half, p = x - k * half;
    const unsigned token = first + k;
    if (token < a.total) {
      const unsigned b = token / a.n_tokens, t = token - b * a.n_tokens;
      const int position = a.positions ? a.positions[b * a.positions_batch + t] : a.start + (int)t;
      float2 f = rope_cos_sin(tab.turn[p], position, tab.amplitude);
      f.y *= a.sign;
      cs[k][p] = f;
    }
  }
  __syncthreads();
  rope_walk<T, V, STREAM>(tab, cs, n_here, a.head_dim, a.copy_rest, a.n_heads, [&](int k, int h, const T *&from, T *&to) {
    const unsigned token = first + k;
    if (token >= a.total) return false;
    const unsigned b = token / a.n_tokens, t = token - b * a.n_tokens;
    const bool second = h >= a.first_heads;
    const RopeSide &d = a.side[second];
    if (second) h -= a.first_heads;
    from = (const T *)d.x + (b * d.xb + t * d.xt + h * d.xh);
    to = (T *)d.y + (b * d.yb + t * d.yt + h * d.yh);
    return true;
  });
}

template <class T>
hipError_t launch_typed(const RopeTable &tab, const RopeArgs &a, bool wide, unsigned groups, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  if (wide && rope_streams(tab.half, a.head_dim, sizeof(T)))
    rope_kernel<T, V, true><<<groups, kRopeThreads, 0, s>>>(tab, a);
  else if (wide)
    rope_kernel<T, V, false><<<groups, kRopeThreads, 0, s>>>(tab, a);
  else
    rope_kernel<T, 1, false><<<groups, kRopeThreads, 0, s>>>(tab, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeTable &tab, int head_dim, const skvq_rope_tensor *tensors, int n_tensors, int dtype,
                       int batch, unsigned n_tokens, const int *positions, long long positions_batch, int start,
                       bool transpose, hipStream_t s) {
  RopeArgs a{};
  const int size = dtype == SKVQ_DTYPE_F32 ? 4 : 2, V = 16 / size;
  // 16-byte accesses where both members of a pair's neighbours lie in whole pieces and every row begins on one
  bool wide = tab.half % V == 0 && head_dim % V == 0;
  bool copy = false;
  for (int i = 0; i < n_tensors; ++i) {
    const skvq_rope_tensor &t = tensors[i];
    a.side[i] = RopeSide{t.x, t.y, t.x_batch, t.x_token, t.x_head, t.y_batch, t.y_token, t.y_head};
    a.n_heads += t.n_heads;
    wide = wide && !(((uintptr_t)t.x | (uintptr_t)t.y) & 15);
    for (long long d : {t.x_batch, t.x_token, t.x_head, t.y_batch, t.y_token, t.y_head}) wide = wide && d % V == 0;
    copy = copy || t.x != t.y;
  }
  a.first_heads = tensors[0].n_heads;
  a.head_dim = head_dim;
  a.copy_rest = copy && 2 * tab.half < head_dim;
  a.n_tokens = n_tokens;
  a.total = n_tokens * (unsigned)batch;
  a.tokens_per_group = rope_tokens_per_group(a.total, (a.copy_rest ? head_dim : 2 * tab.half) / (wide ? V : 1) / 2, a.n_heads);
  a.positions = positions;
  a.positions_batch = positions_batch;
  a.start = start;
  a.sign = transpose ? -1.0f : 1.0f;
  const unsigned groups = (a.total + a.tokens_per_group - 1) / a.tokens_per_group;
  switch (dtype) {
    case SKVQ_DTYPE_F16: return launch_typed<_Float16>(tab, a, wide, groups, s);
    case SKVQ_DTYPE_BF16: return launch_typed<__bf16>(tab, a, wide, groups, s);
    default: return launch_typed<float>(tab, a, wide, groups, s);
  }
}

}  // namespace skvq
