// skvq_paged_attention: the batch's query tokens over pages of 4-bit rows and the fp16 / bf16 rows (Eq. 1).
//
// A workgroup of four wavefronts takes one chunk of one sequence's tokens for one kv head and up to sixteen
// (query token, query head) rows; a wavefront takes every fourth tile of 32 tokens:
//   scores  S^T[token][row] = K Q^T by v_mfma_f32_16x16x32_f16, two blocks of 16 tokens.  The A operand is the
//           lane's 16 bytes of a key row: (w << 4, w, w >> 4, w >> 8) & 0x00f000f0 are its eight codes as fp16
//           subnormals code * 2^-20, in the order of the key dword's nibbles (kept at bits 4..7: the matrix core
//           aligns a subnormal by its unit, so lower bits would cost the sum precision).  A dword is 32 positions
//           of one quantization group, so there is one accumulator per group:
//           score = sum_g scale_g (codes . q)_g + zero_g (sum of q)_g, in fp32.
//   softmax in base 2, lazily re-referenced: the reference of a row moves when a weight would pass 2^15.
//   values  O^T[position][row] += V^T P^T, eight of the same instruction.  P^T is in the B operand's layout as it
//           leaves S^T (lane: row lane % 16, tokens 4 (lane / 16) + 0..3 of both blocks), and a lane's 16 bytes of
//           four value rows are the A operand's tokens of eight positions: nothing crosses lanes in the loop.
// The (scale, zero) pairs of a lane's four tokens sit in the lanes of its row of 16, one pair each (token x / NG, group
// x % NG in lane x): one load and one conversion per lane and block, and every use reads them by a lane broadcast that
// is part of the instruction.
//
// The weight that multiplies a code is weight * scale: the reference counts log2 of the token's largest scale in,
// so that this product, rounded to fp16 (half a step of 2^-10; a second part as in the fixed cache's kernel would refine
// what 16-bit outputs do not show), stays within fp16's normal numbers near the largest contributions.  The middle code
// goes into the zero and the rounded weights' own sum (one more matrix instruction, against ones) is taken off as often:
// only a code's distance from the middle feels the rounding (error of a flat average of 32k tokens against 64 bits,
// beside the output's own rounding: 1.8e-4 -> 0.9e-4).  Zeros enter by fp32 sums: out = sum (w scale) code + sum w zero.
//
// Lengths are device data: every workgroup sums up the batch, finds the chunk size that fills the chip's workgroups
// evenly (chunk_for) and its own units.  Bound by HBM for long contexts: 136 bytes per (token, kv head) at one group.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "skvq_paged.h"

namespace skvq {
namespace {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef unsigned uint4_t __attribute__((ext_vector_type(4)));
typedef unsigned uint2_t __attribute__((ext_vector_type(2)));

constexpr int kWaves = kPagedWaves, kTile = kPagedTile;
// workgroups that a compute unit holds: a third set of registers does not fit four accumulators per score
constexpr int groups_per_cu(int NG) { return NG == 4 ? 2 : 3; }
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kCodeUnit = 1048576.0f;      // 2^20: a code is the fp16 number code * 2^-20
constexpr float kWeightShift = 10.0f;        // a row's largest weight is 2^10 when its reference moves ...
constexpr float kSlack = 5.0f;               // ... and at most 2^15 before it moves again
constexpr float kLowestLog = -40.0f;         // of a scale: a group without spread has scale 0
constexpr float kMidCode = 7.5f;
constexpr float kNothing = -1e30f;           // reference of a row that has seen nothing
constexpr int kRowStride = kD + 4;           // floats per parked accumulator row

__device__ __forceinline__ float4_t mfma(half8_t a, half8_t b, float4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float4_t mfma(bf8_t a, bf8_t b, float4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ half8_t as_half8(unsigned a, unsigned b, unsigned c, unsigned d) {
  return __builtin_bit_cast(half8_t, uint4_t{a, b, c, d});
}

template <int I, int N, class F>
__device__ __forceinline__ void unrolled(F f) {  // f(I) .. f(N - 1), the numbers as types
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    unrolled<I + 1, N>(f);
  }
}

// Lane x's value of the row of 16 lanes.
template <int X>
__device__ __forceinline__ float of_lane(float v) {
  return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x150 + X, 0xF, 0xF, true));
}

// One (scale, zero) pair as it comes from memory.
template <int FMT>
struct PairWord {
  typename std::conditional<FMT == SKVQ_META_F32, uint2_t, typename std::conditional<FMT == SKVQ_META_F16, unsigned, unsigned short>::type>::type w;
  static constexpr int kSize = sizeof(w);
  __device__ __forceinline__ void load(const uint8_t *p) { w = *reinterpret_cast<const decltype(w) *>(p); }
  __device__ __forceinline__ float2 value() const {
    if constexpr (FMT == SKVQ_META_F32) {
      return make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
    } else if constexpr (FMT == SKVQ_META_F16) {
      typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
      const half2_t h = __builtin_bit_cast(half2_t, w);
      return make_float2((float)h[0], (float)h[1]);
    } else {
      return make_float2(__builtin_amdgcn_cvt_f32_fp8((int)w, 0), __builtin_amdgcn_cvt_f32_fp8((int)w, 1));
    }
  }
};

// A tile's packed data as a lane holds it.
template <int FMT>
struct Tile {
  uint4_t k[2], v[2];
  PairWord<FMT> km[2], vm[2];
};

struct Out {
  void *out;
  long long stride;
  float *f32;
};

// A unit's rows: up to 16 (query token, query head) rows of a kv head of one sequence.
struct RowBlock {
  int i;          // sequence
  Sequence s;
  int first;      // first of its rows, of n_new * R
  int count;      // rows here
};
// the query row's place in [n_tokens][Hq]
__device__ __forceinline__ long long query_row(const PagedLayout &L, const RowBlock &x, int h, int row) {
  const int y = x.first + row, j = y / L.R;
  return (long long)(x.s.row0 + j) * L.Hq + h * L.R + (y - j * L.R);
}

template <class T>
__device__ __forceinline__ void store_out(const PagedLayout &L, const Out &o, long long qrow, int channel, float x) {
  if (o.out) {
    const long long token = qrow / L.Hq, head = qrow - token * L.Hq;
    reinterpret_cast<T *>(o.out)[token * o.stride + head * kD + channel] = (T)x;
  }
  if (o.f32) o.f32[qrow * kD + channel] = x;
}

// What a workgroup needs to know of the batch: the chunk size, and the units per kv head.  (Units are counted in 32 bits:
// the host refuses a call that could have more.)
struct BatchPlan {
  int chunk, units;
};
// A sequence's blocks of 16 rows (none where its counts are bad) and its chunks.
__device__ __forceinline__ int blocks_of(const PagedLayout &L, const Sequence &s) {
  return s.counts_ok ? (int)(((long long)s.n_new * L.R + 15) >> 4) : 0;
}
__device__ __forceinline__ Chunks chunks_of_sequence(const PagedLayout &L, const Sequence &s, int chunk) {
  return chunks_of(s.counts_ok ? s.total : 1, L.W, L.S, chunk);
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long long wave_sum(long long x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  return (long long)(((unsigned long long)(unsigned)uniform((int)(x >> 32)) << 32) | (unsigned)uniform((int)x));
}
__device__ __forceinline__ BatchPlan plan_batch(const PagedLayout &L, const PagedBatch &b, int groups) {
  const int lane = threadIdx.x & 63;
  long long work = 0, extra = 0;
  bool bad = false;
  for (int i = lane; i < b.n_seqs; i += 64) {
    const Sequence s = sequence_of(b, L, i);
    bad = bad || !s.counts_ok;
    const int blocks = blocks_of(L, s);
    const Chunks c = chunks_of_sequence(L, s, kPagedMinChunk);
    work += (long long)blocks * c.nq;
    extra += (long long)blocks * (c.rows + (c.nq > 0));
  }
  if (bad && blockIdx.x == 0) atomicOr(L.errors, SKVQ_PAGED_BAD_COUNTS);
  BatchPlan p;
  p.chunk = chunk_for(wave_sum(work), wave_sum(extra), L.Hk, groups);
  int units = 0;
  for (int i = lane; i < b.n_seqs; i += 64) {
    const Sequence s = sequence_of(b, L, i);
    const Chunks c = chunks_of_sequence(L, s, p.chunk);
    units += blocks_of(L, s) * (c.rows + c.packed);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) units += __shfl_xor(units, d);
  p.units = uniform(units);
  return p;
}
// The unit's sequence, rows and chunk.  A chunk's row blocks are neighbours: they read the same rows.
__device__ __forceinline__ RowBlock find_unit(const PagedLayout &L, const PagedBatch &b, const BatchPlan &p, int unit, int &chunk) {
  const int lane = threadIdx.x & 63;
  RowBlock x;
  int rest = unit;
  for (int i0 = 0;; i0 += 64) {
    const int i = i0 + lane < b.n_seqs ? i0 + lane : b.n_seqs - 1;
    const Sequence s = sequence_of(b, L, i);
    const Chunks c = chunks_of_sequence(L, s, p.chunk);
    int upto = i0 + lane < b.n_seqs ? blocks_of(L, s) * (c.rows + c.packed) : 0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(upto, d);
      upto += lane >= d ? y : 0;
    }
    const unsigned long long behind = __ballot(upto > rest);  // (some lane, sooner or later: unit < p.units)
    if (behind || i0 + 64 >= b.n_seqs) {
      const int k = uniform(behind ? __ffsll(behind) - 1 : 63);
      if (k > 0) rest -= __builtin_amdgcn_readlane(upto, k - 1);
      x.i = i0 + k < b.n_seqs ? i0 + k : b.n_seqs - 1;
      break;
    }
    rest -= __builtin_amdgcn_readlane(upto, 63);
  }
  x.s = sequence_of(b, L, x.i);
  const int blocks = blocks_of(L, x.s);
  chunk = blocks > 1 ? rest / blocks : rest;
  x.first = blocks > 1 ? 16 * (rest % blocks) : 0;
  const int left = x.s.n_new * L.R - x.first;
  x.count = left < 16 ? left : 16;
  return x;
}

// A wavefront's running state: lane (g, c) = (lane / 16, lane % 16) holds row c's share.
template <int NG>
struct State {
  float4_t o[8];      // packed: positions 16n + 4g + reg; full rows: channels 8 (4g + reg) + n
  float4_t w[NG];     // packed: sum of the rounded weights that met the codes, in every register
  float m, l, z[NG];  // reference; this lane's share of the sum of weights, of weights times zeros
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int n = 0; n < 8; ++n) o[n] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    m = kNothing;
    l = 0.0f;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      w[g] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
      z[g] = 0.0f;
    }
  }
  // Moves the references up where a lane holds a logarithm too far above its row's.
  __device__ __forceinline__ void refer(float top) {
    if (!__any(top > m + (kWeightShift + kSlack))) return;
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float to = fmaxf(m, top - kWeightShift), f = __builtin_amdgcn_exp2f(m - to);
    m = to;
    l *= f;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      z[g] *= f;
      w[g] *= f;
    }
#pragma unroll
    for (int n = 0; n < 8; ++n) o[n] *= f;
  }
};

// One tile of packed rows.  MASKED: some of its rows are behind the chunk's end (what stands there may be anything) or
// behind what some query sees.  left: rows of the tile before the end; seen: before the last one that the lane's row
// sees.  alpha: on the scores, with the code's unit.
template <int NG, int FMT, bool MASKED>
__device__ __forceinline__ void take_tile(State<NG> &st, const Tile<FMT> &t, const half8_t (&qb)[4], const float (&qs)[NG], float alpha,
                                          int left, int seen, int g, int c) {
  float ks[2], kz[2], vs[2], vz[2], lg[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 k = t.km[i].value(), v = t.vm[i].value();
    const bool there = !MASKED || 16 * i + 4 * g + (c % (4 * NG)) / NG < left;
    ks[i] = there ? k.x * alpha : 0.0f;
    kz[i] = there ? k.y : 0.0f;
    vs[i] = there ? v.x : 0.0f;
    vz[i] = there ? fmaf(v.x, kMidCode, v.y) : 0.0f;
    float most = vs[i];
    if (NG >= 2) most = fmaxf(most, __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(most), 0xB1, 0xF, 0xF, true)));
    if (NG == 4) most = fmaxf(most, __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(most), 0x4E, 0xF, 0xF, true)));
    lg[i] = fmaxf(__builtin_amdgcn_logf(most), kLowestLog);
  }
  float s[8], top = -INFINITY;
  const unsigned mask = 0x00f000f0u;
  unrolled<0, 2>([&](auto I) {
    constexpr int i = I();
    float4_t acc[NG];
#pragma unroll
    for (int n = 0; n < NG; ++n) acc[n] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned w = t.k[i][j];
      acc[j * NG / 4] = mfma(as_half8((w << 4) & mask, w & mask, (w >> 4) & mask, (w >> 8) & mask), qb[j], acc[j * NG / 4]);
    }
    unrolled<0, 4>([&](auto R) {
      constexpr int r = R();
      float x = 0.0f;
      unrolled<0, NG>([&](auto N) {
        constexpr int n = N();
        x = n == 0 ? of_lane<r * NG>(kz[i]) * qs[0] : fmaf(of_lane<r * NG + n>(kz[i]), qs[n], x);
        x = fmaf(of_lane<r * NG + n>(ks[i]), acc[n][r], x);
      });
      const float u = of_lane<r * NG>(lg[i]) + x;
      const bool there = !MASKED || 16 * i + 4 * g + r < min(left, seen);
      s[4 * i + r] = there ? x : -INFINITY;
      top = fmaxf(top, there ? u : -INFINITY);
    });
  });
  st.refer(top);
  half8_t pb[NG];
  unrolled<0, 8>([&](auto I) {
    constexpr int i = I() / 4, r = I() % 4;
    const float p = __builtin_amdgcn_exp2f(s[I()] - st.m);
    st.l += p;
    unrolled<0, NG>([&](auto N) {
      constexpr int n = N();
      st.z[n] = fmaf(of_lane<r * NG + n>(vz[i]), p, st.z[n]);
      pb[n][I()] = (_Float16)(of_lane<r * NG + n>(vs[i]) * p);
    });
  });
  const half8_t one = as_half8(0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u);
#pragma unroll
  for (int n = 0; n < NG; ++n) st.w[n] = mfma(one, pb[n], st.w[n]);
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    unsigned a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned w = t.v[i / 2][2 * (i % 2) + n / 4];
      a[i] = (n % 4 == 0 ? w << 4 : n % 4 == 1 ? w : n % 4 == 2 ? w >> 4 : w >> 8) & mask;
    }
    st.o[n] = mfma(as_half8(a[0], a[1], a[2], a[3]), pb[n * NG / 8], st.o[n]);
  }
}

template <class T>
struct Lds {
  union alignas(16) {
    T q[16][kD + 8];
    float acc[kWaves][16][kRowStride];
  };
  float m[kWaves][16], l[kWaves][16];
  int bad;
};

// The wavefront's share of a chunk of packed rows.
template <class T, int NG, int FMT>
__device__ __forceinline__ void take_packed(const PagedLayout &L, const PagedBatch &b, const Lds<T> &lds, const RowBlock &x, const Chunks &ch,
                                            int chunk, int h, State<NG> &st, bool &bad) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
  const int last = x.s.total - x.s.n_new + (x.first + (c < x.count ? c : x.count - 1)) / L.R;  // lane's row: the last token it sees
  // B operand: row c's queries at the reordered positions of key dword 4g + j, as fp16 numbers.  bf16 queries are
  // brought to fp16's range by one power of two: what that makes subnormal is 2^-25 of the largest.
  half8_t qb[4];
  float qs[NG], scale = L.sm_scale * kLog2e, alpha = scale * kCodeUnit;
  {
    float v[4][8], most = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned long long at = *reinterpret_cast<const unsigned long long *>(L.k_channel + h * kD + 8 * (4 * g + j));
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[j][e] = (float)lds.q[c][(at >> (8 * e)) & 0xffu];
        most = fmaxf(most, fabsf(v[j][e]));
      }
    }
    float to_half = 1.0f;
    if constexpr (!__is_same(T, _Float16)) {
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));
      const int exponent = most > 0.0f ? __builtin_amdgcn_frexp_expf(most) : 0;  // most in [2^(e-1), 2^e)
      to_half = __builtin_amdgcn_ldexpf(1.0f, 14 - exponent < 126 ? 14 - exponent : 126);
      alpha /= to_half;
    }
#pragma unroll
    for (int t = 0; t < NG; ++t) qs[t] = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        qs[j * NG / 4] += v[j][e];
        qb[j][e] = (_Float16)(v[j][e] * to_half);
      }
#pragma unroll
    for (int t = 0; t < NG; ++t) {
      qs[t] += __shfl_xor(qs[t], 16);
      qs[t] += __shfl_xor(qs[t], 32);
      qs[t] *= scale;
    }
  }
  const int seen = last + 1 - L.S;  // packed rows that the lane's row sees; all of them see the first row's
  const int begin = chunk * ch.chunk, end = min(ch.nq, begin + ch.chunk);
  const int all_see = min(end, x.s.total - x.s.n_new + x.first / L.R + 1 - L.S);
  const int n_tiles = (end - begin + kTile - 1) / kTile, mine = n_tiles > wave ? (n_tiles - wave + kWaves - 1) / kWaves : 0;
  const uint8_t *head_part = L.pages + (long long)h * L.part_bytes;
  const long long page_stride = (long long)L.Hk * L.part_bytes;
  const int *table = b.table + (long long)x.i * b.table_stride;
  constexpr int kPair = PairWord<FMT>::kSize;
  const unsigned k_lane = c * (kD / 2) + 16 * g, v_lane = L.v_at + 256 * g + 16 * c;
  const unsigned m_lane = kPair * (4 * NG * g + c % (4 * NG));
  // Pages of the wavefront's next 32 tiles, two blocks of 16 tokens each: lane 2k + i holds tile k's block i.
  int ids = 0;
  auto look_up = [&](int k0) {
    const int te = begin + kTile * (wave + kWaves * (k0 + (lane >> 1))) + 16 * (lane & 1);
    ids = 0;
    if (te < end) {
      const int at = te >> L.page_log2;
      ids = page_known(at, b.table_stride) ? table[at] : -1;
      if (!page_valid(ids, L.n_pages)) {
        bad = true;
        ids = 0;
      }
    }
  };
  auto load = [&](Tile<FMT> &t, int k) {  // the wavefront's k-th tile, if there is one (blocks past the end: of page 0)
    if (k >= mine) return;
    if ((k & 31) == 0) look_up(k);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int id = __builtin_amdgcn_readlane(ids, 2 * (k & 31) + i);
      const int te = begin + kTile * (wave + kWaves * k) + 16 * i;
      const unsigned place = te & ((1 << L.page_log2) - 1);
      const uint8_t *p = head_part + id * page_stride;
      t.k[i] = *reinterpret_cast<const uint4_t *>(p + place * (kD / 2) + k_lane);
      t.v[i] = *reinterpret_cast<const uint4_t *>(p + place * (kD / 2) + v_lane);
      t.km[i].load(p + place * (NG * kPair) + L.km_at + m_lane);
      t.vm[i].load(p + place * (NG * kPair) + L.vm_at + m_lane);
    }
  };
  // Whole tiles that every query sees, two buffers in turn; then the others (at the chunk's end).
  const int whole_tiles = all_see > begin ? (all_see - begin) / kTile : 0;
  const int whole = whole_tiles > wave ? (whole_tiles - wave + kWaves - 1) / kWaves : 0;
  Tile<FMT> even, odd;
  load(even, 0);
  int k = 0;
  for (; k + 1 < whole; k += 2) {
    load(odd, k + 1);
    take_tile<NG, FMT, false>(st, even, qb, qs, alpha, 0, 0, g, c);
    load(even, k + 2);
    take_tile<NG, FMT, false>(st, odd, qb, qs, alpha, 0, 0, g, c);
  }
  for (; k < mine; ++k) {
    const int te0 = begin + kTile * (wave + kWaves * k);
    load(odd, k + 1);
    take_tile<NG, FMT, true>(st, even, qb, qs, alpha, end - te0, seen - te0, g, c);
    even = odd;
  }
}

// ... of a chunk of full-precision rows: the u-th of the kept and the ring tokens, in the order of their numbers.
template <class T, int NG>
__device__ __forceinline__ void take_rows(const PagedLayout &L, const Lds<T> &lds, const RowBlock &x, const Chunks &ch, int chunk, int h,
                                          State<NG> &st) {
  typedef T t8 __attribute__((ext_vector_type(8)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
  const int last = x.s.total - x.s.n_new + (x.first + (c < x.count ? c : x.count - 1)) / L.R;
  const float scale = L.sm_scale * kLog2e;
  const int n_full = ch.n_kept + ch.n_win, begin = chunk * kPagedRowsPerChunk, end = min(n_full, begin + kPagedRowsPerChunk);
  const long long head = ((long long)x.s.slot * L.Hk + h) * (L.W + L.S) * kD;
  const T *k_rows = reinterpret_cast<const T *>(L.k_rows) + head, *v_rows = reinterpret_cast<const T *>(L.v_rows) + head;
  const int first_recent = x.s.total - ch.n_win, first_slot = first_recent % L.W;
  auto row_of = [&](int u) {  // (rows past the end: the first, which holds a token)
    u = u < end ? u : begin;
    const int slot = first_slot + u - ch.n_kept;
    return u < ch.n_kept ? L.W + u : slot < L.W ? slot : slot - L.W;
  };
  auto token_of = [&](int u) { return u < ch.n_kept ? u : first_recent + u - ch.n_kept; };
  t8 qb[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) qb[j] = *reinterpret_cast<const t8 *>(&lds.q[c][32 * j + 8 * g]);
  for (int u0 = begin + kTile * wave; u0 < end; u0 += kTile * kWaves) {
    t8 kb[2][4], vb[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const T *kr = k_rows + (long long)row_of(u0 + 16 * i + c) * kD + 8 * g;
#pragma unroll
      for (int j = 0; j < 4; ++j) kb[i][j] = *reinterpret_cast<const t8 *>(kr + 32 * j);
#pragma unroll
      for (int r = 0; r < 4; ++r) vb[i][r] = *reinterpret_cast<const t8 *>(v_rows + (long long)row_of(u0 + 16 * i + 4 * g + r) * kD + 8 * c);
    }
    float s[2][4], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < 4; ++j) acc = mfma(kb[i][j], qb[j], acc);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int u = u0 + 16 * i + 4 * g + r;
        s[i][r] = u < end && token_of(u) <= last ? acc[r] * scale : -INFINITY;
        top = fmaxf(top, s[i][r]);
      }
    }
    st.refer(top);
    t8 hi, lo;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = __builtin_amdgcn_exp2f(s[i][r] - st.m);
        st.l += p;
        hi[4 * i + r] = (T)p;
        lo[4 * i + r] = (T)(p - (float)(T)p);
      }
    // a lane's 16 bytes of eight tokens, transposed: channel 8c + n of every one
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      t8 a;
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = vb[i / 4][i % 4][n];
      st.o[n] = mfma(a, hi, st.o[n]);
      if constexpr (!__is_same(T, _Float16)) st.o[n] = mfma(a, lo, st.o[n]);  // (fp16 holds 11 bits of a weight, bf16 8)
    }
  }
}

template <class T, int NG, int FMT>
__global__ __launch_bounds__(64 * kWaves, groups_per_cu(NG)) void paged_attention_kernel(const PagedLayout L, const PagedBatch b, const TokenRows q,
                                                                                    const Out out, int n_row_chunks) {
  typedef Piece<T, 8> P;
  __shared__ Lds<T> lds;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
  const BatchPlan plan = plan_batch(L, b, gridDim.x);
  for (int at = blockIdx.x; at < plan.units * L.Hk; at += gridDim.x) {
    const int unit = at / L.Hk, h = at - unit * L.Hk;
    int chunk;
    const RowBlock x = find_unit(L, b, plan, unit, chunk);
    const Chunks ch = chunks_of(x.s.total, L.W, L.S, plan.chunk);
    const bool packed = chunk >= ch.rows;
    __syncthreads();  // (the unit before has read its partials out of LDS)
    if (threadIdx.x == 0) {
      lds.bad = !x.s.slot_ok;
      if (!x.s.slot_ok) atomicOr(L.errors, SKVQ_PAGED_BAD_SLOT);
    }
    // the queries, rows past the last one repeat it
    for (int y = threadIdx.x; y < 16 * 16; y += 64 * kWaves) {
      const int row = y >> 4, m = y & 15;
      const long long qr = query_row(L, x, h, row < x.count ? row : x.count - 1);
      const long long token = qr / L.Hq, head = qr - token * L.Hq;
      *reinterpret_cast<P *>(&lds.q[row][8 * m]) = *reinterpret_cast<const P *>((const T *)q.p + token * q.stride + head * kD + 8 * m);
    }
    __syncthreads();
    State<NG> st;
    st.clear();
    bool bad = false;
    if (packed)
      take_packed<T, NG, FMT>(L, b, lds, x, ch, chunk - ch.rows, h, st, bad);
    else if (x.s.slot_ok)
      take_rows<T, NG>(L, lds, x, ch, chunk, h, st);

    // The wavefronts' states: sums over the lanes of a row, then one reference for the workgroup.
    st.l += __shfl_xor(st.l, 16);
    st.l += __shfl_xor(st.l, 32);
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      st.z[n] += __shfl_xor(st.z[n], 16);
      st.z[n] += __shfl_xor(st.z[n], 32);
      st.z[n] -= kMidCode * st.w[n][0];
    }
    if (g == 0) {
      lds.m[wave][c] = st.m;
      lds.l[wave][c] = st.l;
    }
    __syncthreads();  // (also: the queries in LDS are no longer needed)
    if (bad) {
      lds.bad = 1;
      atomicOr(L.errors, SKVQ_PAGED_BAD_PAGE);
    }
    float top = lds.m[0][c];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, lds.m[w][c]);
    const float f = __builtin_amdgcn_exp2f(st.m - top);
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      float4_t y = st.o[n];
      if (packed) {
        y = (y * kCodeUnit + st.z[n * NG / 8]) * f;
        *reinterpret_cast<float4_t *>(&lds.acc[wave][c][16 * n + 4 * g]) = y;
      } else {
        y *= f;
#pragma unroll
        for (int r = 0; r < 4; ++r) lds.acc[wave][c][8 * (4 * g + r) + n] = y[r];
      }
    }
    __syncthreads();
    const int n_partials = ch.rows + ch.packed, most = kPagedMaxSplits + n_row_chunks;
    for (int y = threadIdx.x; y < x.count * kD; y += 64 * kWaves) {
      const int row = y / kD, p = y % kD;
      float acc = lds.acc[0][row][p], m = lds.m[0][row], l = 0.0f;
#pragma unroll
      for (int w = 1; w < kWaves; ++w) {
        acc += lds.acc[w][row][p];
        m = fmaxf(m, lds.m[w][row]);
      }
#pragma unroll
      for (int w = 0; w < kWaves; ++w) l += lds.l[w][row] * __builtin_amdgcn_exp2f(lds.m[w][row] - m);
      if (lds.bad) l = NAN;
      const int channel = packed ? L.v_channel[h * kD + 8 * (p & 15) + (p >> 4)] : p;
      const long long qr = query_row(L, x, h, row);
      float *to = L.workspace + qr * most * kPartialStride;
      if (n_partials == 1) {
        store_out<T>(L, out, qr, channel, acc / l);
      } else {
        float *part = to + chunk * kPartialStride;
        part[4 + channel] = acc;
        if (p == 0) {
          part[0] = m;
          part[1] = l;
        }
      }
      if (p == 0 && chunk == 0) to[2] = __uint_as_float((unsigned)n_partials);  // (for the merge)
    }
  }
}

// Combines a row's partials: out = sum 2^(m_i - m) acc_i / sum 2^(m_i - m) l_i.  One workgroup per (query token, query
// head): eight groups of 32 threads read every eighth partial, thread t of a group channels 4t .. 4t+3.
constexpr int kMergeThreads = 256, kMergeGroups = kMergeThreads / 32;
template <class T>
__global__ __launch_bounds__(kMergeThreads) void paged_merge_kernel(const PagedLayout L, const PagedBatch b, const Out out, int n_row_chunks) {
  __shared__ float weight[kMergeThreads], red[2][kMergeThreads / 64];
  __shared__ float4_t parts[kMergeGroups][32];
  const int token = blockIdx.x, tid = threadIdx.x;
  const Sequence s = sequence_of(b, L, sequence_of_unit(b, token, kTokenDeal));
  if (!s.counts_ok || token < s.row0 || token >= s.row0 + s.n_new) return;
  const long long qr = (long long)token * L.Hq + blockIdx.y;
  const float *from = L.workspace + qr * (kPagedMaxSplits + n_row_chunks) * kPartialStride;
  const int n = (int)__float_as_uint(from[2]);
  if (n <= 1) return;
  auto partial = [&](int i) { return from + (long long)i * kPartialStride; };
  float m = kNothing, l = 0.0f;
  float4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i0 = 0; i0 < n; i0 += kMergeThreads) {  // (more than 256 only with windows of ten thousands of tokens)
    const int here = min(kMergeThreads, n - i0), t = tid & 31;
    const float mi = tid < here ? partial(i0 + tid)[0] : kNothing;
    const float li = tid < here ? partial(i0 + tid)[1] : 0.0f;
    float top = mi;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    if ((tid & 63) == 0) red[0][tid >> 6] = top;
    __syncthreads();
    top = m;
#pragma unroll
    for (int w = 0; w < kMergeThreads / 64; ++w) top = fmaxf(top, red[0][w]);
    const float w = tid < here ? __builtin_amdgcn_exp2f(mi - top) : 0.0f, before = __builtin_amdgcn_exp2f(m - top);
    weight[tid] = w;
    float sum = li * w;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    if ((tid & 63) == 0) red[1][tid >> 6] = sum;
    __syncthreads();
    l *= before;
#pragma unroll
    for (int w = 0; w < kMergeThreads / 64; ++w) l += red[1][w];
    acc *= before;
    m = top;
    int i = tid >> 5;
    for (; i + 3 * kMergeGroups < here; i += 4 * kMergeGroups) {
      float4_t a[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) a[u] = *reinterpret_cast<const float4_t *>(partial(i0 + i + u * kMergeGroups) + 4 + 4 * t);
#pragma unroll
      for (int u = 0; u < 4; ++u) acc += a[u] * weight[i + u * kMergeGroups];
    }
    for (; i < here; i += kMergeGroups) acc += *reinterpret_cast<const float4_t *>(partial(i0 + i) + 4 + 4 * t) * weight[i];
    __syncthreads();
  }
  parts[tid >> 5][tid & 31] = acc;
  __syncthreads();
  if (tid < kD) {
    float x = 0.0f;
#pragma unroll
    for (int k = 0; k < kMergeGroups; ++k) x += reinterpret_cast<const float *>(&parts[k][0])[tid];
    store_out<T>(L, out, qr, tid, x / l);
  }
}

template <class T, int NG>
void launch_chunks(const PagedLayout &L, const PagedBatch &b, TokenRows q, Out out, int row_chunks, unsigned groups, hipStream_t s) {
  const dim3 threads(64 * kWaves);
  switch (L.meta_fmt) {
    case SKVQ_META_F32: paged_attention_kernel<T, NG, SKVQ_META_F32><<<groups, threads, 0, s>>>(L, b, q, out, row_chunks); break;
    case SKVQ_META_F16: paged_attention_kernel<T, NG, SKVQ_META_F16><<<groups, threads, 0, s>>>(L, b, q, out, row_chunks); break;
    default: paged_attention_kernel<T, NG, SKVQ_META_FP8_E4M3><<<groups, threads, 0, s>>>(L, b, q, out, row_chunks); break;
  }
}

template <class T>
hipError_t launch_typed(const PagedLayout &L, const PagedBatch &b, TokenRows q, Out out, int row_chunks, unsigned groups, hipStream_t s) {
  switch (L.NG) {
    case 1: launch_chunks<T, 1>(L, b, q, out, row_chunks, groups, s); break;
    case 2: launch_chunks<T, 2>(L, b, q, out, row_chunks, groups, s); break;
    default: launch_chunks<T, 4>(L, b, q, out, row_chunks, groups, s); break;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  paged_merge_kernel<T><<<dim3((unsigned)b.n_tokens, L.Hq), kMergeThreads, 0, s>>>(L, b, out, row_chunks);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attention(const PagedLayout &L, const skvq_batch &batch, TokenRows q, void *out, long long out_stride,
                                  float *out_f32, int n_cus, hipStream_t s) {
  const PagedBatch b = batch_of(batch);
  const int row_chunks = paged_row_chunks(L.W, L.S);
  // Lengths are not known here: as many workgroups as the chip holds at once, unless there can be no more units than
  // that (every row in a block of its own sequence, every sequence as long as the page table allows).
  const long long rows = (long long)b.n_tokens * L.R, blocks = rows / 16 + (b.n_seqs < b.n_tokens ? b.n_seqs : b.n_tokens);
  long long splits = ((long long)b.table_stride << L.page_log2) / kPagedMinChunk + 1;
  if (splits > kPagedMaxSplits) splits = kPagedMaxSplits;
  const long long units = blocks * (row_chunks + splits) * L.Hk, most = (long long)groups_per_cu(L.NG) * n_cus;
  if (units > 0x7fffffff - most) return hipErrorInvalidValue;  // (counted in 32 bits)
  const unsigned groups = (unsigned)(units < most ? units : most);
  const Out o{out, out_stride, out_f32};
  return L.dtype == SKVQ_DTYPE_BF16 ? launch_typed<__bf16>(L, b, q, o, row_chunks, groups, s)
                                    : launch_typed<_Float16>(L, b, q, o, row_chunks, groups, s);
}

}  // namespace skvq
