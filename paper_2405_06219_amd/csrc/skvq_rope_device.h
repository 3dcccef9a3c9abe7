// Rotary positions, device side: cosine and sine of position * frequency, and the rotation of a pair.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "skvq.h"

namespace skvq {

// A rotation as kernels take it, by value: 1 KB of kernel arguments, so a rope object holds no device memory.
struct RopeTable {
  uint64_t turn[SKVQ_ROPE_MAX_HEAD_DIM / 2];  // per pair: turns per token, mod 1, in units of 2^-64
  double amplitude;
  int half;         // pairs (0: nothing is rotated)
  int interleaved;  // pair i is channels (2i, 2i + 1), else (i, i + half)
};

// (cos, sin) of 2 pi * position * turn, times the amplitude, rounded to fp32.  position * turn wraps at 2^64,
// which is one turn: no range reduction is left to do but the quadrant, at any position.  Series of sine to
// x^13 and cosine to x^14 at |x| <= pi/4: the terms left out are below 2^-45, so the fp32 results are the
// rounded true ones (but for about one in 2^20 next to a border).  Some 40 double operations per (token,
// pair), shared by all heads.
__device__ __forceinline__ float2 rope_cos_sin(uint64_t turn, int position, double amplitude) {
  const uint64_t t = turn * (uint64_t)(int64_t)position;
  const unsigned quadrant = (unsigned)((t + (1ull << 61)) >> 62);
  const int64_t r = (int64_t)(t - ((uint64_t)quadrant << 62));  // [-1/8, 1/8) of a turn
  const double x = (double)r * (6.283185307179586476925286766559 / 18446744073709551616.0);
  const double z = x * x;
  double s = 1.0 / 6227020800.0;
  s = fma(s, z, -1.0 / 39916800.0);
  s = fma(s, z, 1.0 / 362880.0);
  s = fma(s, z, -1.0 / 5040.0);
  s = fma(s, z, 1.0 / 120.0);
  s = fma(s, z, -1.0 / 6.0);
  s = fma(s * z, x, x);
  double c = -1.0 / 87178291200.0;
  c = fma(c, z, 1.0 / 479001600.0);
  c = fma(c, z, -1.0 / 3628800.0);
  c = fma(c, z, 1.0 / 40320.0);
  c = fma(c, z, -1.0 / 720.0);
  c = fma(c, z, 1.0 / 24.0);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const bool swap = quadrant & 1u;
  const double cs = swap ? s : c, sn = swap ? c : s;
  const bool neg_c = (quadrant + 1u) & 2u, neg_s = quadrant & 2u;
  return make_float2((float)((neg_c ? -cs : cs) * amplitude), (float)((neg_s ? -sn : sn) * amplitude));
}

// One member of a rotated pair: x * c + other * s, each operation rounded once (the first member takes s
// negated: a c - b s = a c + b (-s), the same three roundings).
__device__ __forceinline__ float rope_turned(float x, float other, float c, float s) {
#pragma clang fp contract(off)
  const float p = x * c;
  const float q = other * s;
  return p + q;
}

// The rotation of a group of tokens by a workgroup of kRopeThreads.  cs: their cosines and sines, [token][pair],
// in LDS.  rows(k, h, &from, &to): head h's rows of token k, false where there is no such token.
//
// A thread keeps the cosines and sines of its place in the head in registers and walks over the heads, two
// pieces of V channels (2V members of V pairs) per head.  Few registers for many wavefronts, and STREAMing accesses
// where an instruction takes whole cache lines: a 32k prompt's rotation (671 MB) takes 121 - 123 us, with plain accesses
// and four heads' loads in flight 140.
constexpr int kRopeThreads = 256;
constexpr int kRopeMaxTokens = 4;  // tokens per workgroup
constexpr int kRopeAhead = 2;
constexpr int kRopeMaxPairs = SKVQ_ROPE_MAX_HEAD_DIM / 2;

// V values as one access.  (A vector type: a struct around an array may be moved to LDS by the compiler, whose addressing
// then waits for the dispatch packet in host memory, 10 us a launch.)
template <class T, int V>
using Piece = T __attribute__((ext_vector_type(V)));

template <bool STREAM, class P>
__device__ __forceinline__ P piece_load(const P *p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(p); else return *p;
}
template <bool STREAM, class P>
__device__ __forceinline__ void piece_store(P *p, P x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, p); else *p = x;
}
// Tokens per workgroup: about five heads a thread (more wait for memory in turn, fewer compute cosines for too little),
// one token where workgroups are few.
inline int rope_tokens_per_group(long long tokens, long long pieces, long long heads) {
  if (tokens < 4096) return 1;
  const long long n = 5 * kRopeThreads / (pieces * heads);
  return n >= kRopeMaxTokens ? kRopeMaxTokens : n >= 2 ? 2 : 1;
}
// whether each of the two pieces' runs over a head fills whole lines (of rows that begin on one)
inline __host__ __device__ bool rope_streams(int half, int head_dim, int size) { return half * size % 128 == 0 && head_dim * size % 128 == 0; }

template <class T, int V, bool STREAM, class Rows>
__device__ __forceinline__ void rope_walk(const RopeTable &tab, const float2 (*cs)[kRopeMaxPairs], int n_here, int head_dim,
                                          bool copy_rest, int n_heads, Rows rows) {
  typedef Piece<T, V> P;
  const int half = tab.half, rotated = half / V, rest = copy_rest ? (head_dim - 2 * half) / V : 0, pieces = rotated + (rest + 1) / 2;
  const int places = n_here * pieces, head_lanes = places < kRopeThreads ? kRopeThreads / places : 1;
  for (int x = threadIdx.x; x < places * head_lanes; x += kRopeThreads) {
    const int hl = x / places, place = x - hl * places;
    const int k = place / pieces, j = place - k * pieces;
    // Two pieces.  Of half layout half the rotated part apart, both members of pairs Vj .., and behind them two that are
    // copied (the last one twice if they are odd); likewise one channel at a time, where neighbours are a pair.  Whole
    // pieces of neighbouring pairs turn by themselves: half of all pieces apart, so that an access takes half a row in one
    // run (a head of 96 fp32 channels, 48 turned, 282 MB both ways: 62 us with the halves of either part, 58 so).
    const bool inside = V > 1 && tab.interleaved;
    bool turn_a = j < rotated, turn_b = turn_a;
    int oa = V == 1 && tab.interleaved ? 2 * j : V * j, ob = V == 1 && tab.interleaved ? oa + 1 : oa + half;
    if (inside) {
      const int second = j + pieces < 2 * rotated + rest ? j + pieces : j;
      ob = V * second;
      turn_a = j < 2 * rotated;
      turn_b = second < 2 * rotated;
    } else if (!turn_a) {
      const int first = j - rotated, second = first + (rest + 1) / 2;
      oa = 2 * half + V * first;
      ob = 2 * half + V * (second < rest ? second : rest - 1);
    }
    float c[V], s[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const bool turn = inside && e >= V / 2 ? turn_b : turn_a;
      const int pair = !inside ? j * V + e : e < V / 2 ? oa / 2 + e : ob / 2 + e - V / 2;
      const float2 f = turn ? cs[k][pair] : make_float2(1.0f, 0.0f);
      c[e] = f.x;
      s[e] = f.y;
    }
    for (int h0 = hl; h0 < n_heads; h0 += kRopeAhead * head_lanes) {
      P pa[kRopeAhead], pb[kRopeAhead];
      T *to[kRopeAhead];
#pragma unroll
      for (int u = 0; u < kRopeAhead; ++u) {
        const int h = h0 + u * head_lanes;
        const T *from;
        to[u] = nullptr;
        if (h < n_heads && rows(k, h, from, to[u])) {
          pa[u] = piece_load<STREAM>(reinterpret_cast<const P *>(from + oa));
          pb[u] = piece_load<STREAM>(reinterpret_cast<const P *>(from + ob));
        }
      }
#pragma unroll
      for (int u = 0; u < kRopeAhead; ++u)
        if (to[u]) {
          P ra, rb;
          if (inside) {
#pragma unroll
            for (int e = 0; e + 1 < V; e += 2) {  // (pairs within a piece)
              const int f = e / 2, g = V / 2 + e / 2;
              ra[e] = (T)rope_turned((float)pa[u][e], (float)pa[u][e + 1], c[f], -s[f]);
              ra[e + 1] = (T)rope_turned((float)pa[u][e + 1], (float)pa[u][e], c[f], s[f]);
              rb[e] = (T)rope_turned((float)pb[u][e], (float)pb[u][e + 1], c[g], -s[g]);
              rb[e + 1] = (T)rope_turned((float)pb[u][e + 1], (float)pb[u][e], c[g], s[g]);
            }
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              ra[e] = (T)rope_turned((float)pa[u][e], (float)pb[u][e], c[e], -s[e]);
              rb[e] = (T)rope_turned((float)pb[u][e], (float)pa[u][e], c[e], s[e]);
            }
          }
          piece_store<STREAM>(reinterpret_cast<P *>(to[u] + oa), turn_a ? ra : pa[u]);
          piece_store<STREAM>(reinterpret_cast<P *>(to[u] + ob), turn_b ? rb : pb[u]);
        }
    }
  }
}

}  // namespace skvq
