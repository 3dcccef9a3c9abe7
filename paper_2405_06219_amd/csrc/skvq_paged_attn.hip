// skvq_paged_attention: the batch's query tokens over pages of 4-bit rows and the fp16 / bf16 rows (Eq. 1).
//
// A workgroup of four wavefronts takes some of one sequence's tokens for one kv head and RB blocks of sixteen
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
// The (scale, zero) pairs of a lane's eight tokens, of keys and values, sit in the lanes of its row of 16 (PairSlot): one
// load, conversion and logarithm per tile and group, and every use reads them by a lane broadcast.  What a tile's pairs, key
// codes and value codes leave free, the next tile's take in the same registers (a second buffer is 26 registers at four
// groups and hides no more: HBM answers within half a tile's work).
// Work on vectors bounds calls of many rows per kv head: two blocks share unpacking and broadcasts (RB = 2).
//
// The weight that multiplies a code is weight * scale: the reference counts log2 of the largest scale at hand in, so
// that this product stays within fp16's normal numbers near the largest contributions.  For fp16 outputs it is taken in
// two parts, rounded (half a step of 2^-10) and the rest: one alone is an error as large as the output's own rounding
// (16 sequences of 32k tokens, rms against 64 bits: 2.1e-4 with both, as of the rounding alone, 2.6e-4 with one; 390 us
// with one, 405 with two).  bf16 outputs, of 8 bits, make do with one (1.7e-3 either way); there the middle code goes into the zero
// and the rounded weights' own sum is taken off as often, so that only a code's distance from the middle feels the
// rounding.  Zeros enter by fp32 sums: out = sum (w scale) code + sum w zero.
//
// Lengths are device data: every workgroup sums up the batch's work, an equal share of it is its own, and it finds the
// sequences that its share lies in.
//
// Bound by HBM for long contexts of few rows per kv head, 136 bytes per (token, kv head) at one group: 16 sequences of
// 32k tokens, 32 heads, 2.3 GB in 385 - 405 us (its streaming loads alone 369); 128k tokens of 8 kv heads, 143 MB, 35 us and
// the merge's 5, of which the tiles 23; by vector instructions at two and four groups and for many rows: 64 sequences of
// 256 to 16k tokens, two groups, 311 MB, 72 us; up to 64 rows a kv head, four groups, 208 MB, 109 us.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "skvq_paged.h"

namespace skvq {
namespace {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef unsigned uint4_t __attribute__((ext_vector_type(4)));
typedef unsigned uint2_t __attribute__((ext_vector_type(2)));

constexpr int kWaves = kPagedWaves, kTile = kPagedTile;
// workgroups that a compute unit holds: a third set of registers does not fit four accumulators per score, or the state
// of two blocks of query rows
constexpr int groups_per_cu(int NG, int RB) { return NG == 4 || RB > 1 ? 2 : 3; }
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

// The largest of the row's 16 lanes, in all of them.
__device__ __forceinline__ float row_max(float v) {
  auto with = [](float x, auto ctrl) {
    return fmaxf(x, __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(ctrl)::value, 0xF, 0xF, true)));
  };
  v = with(v, std::integral_constant<int, 0xB1>{});   // lanes ^ 1, ^ 2, then mirror images of 8 and of 16
  v = with(v, std::integral_constant<int, 0x4E>{});
  v = with(v, std::integral_constant<int, 0x141>{});
  return with(v, std::integral_constant<int, 0x140>{});
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
      const half2_t h = __builtin_bit_cast(half2_t, w);
      return make_float2((float)h[0], (float)h[1]);
    } else {
      return make_float2(__builtin_amdgcn_cvt_f32_fp8((int)w, 0), __builtin_amdgcn_cvt_f32_fp8((int)w, 1));
    }
  }
};

// Whether a weight that meets codes has two parts.
template <class T>
constexpr bool two_parts() { return __is_same(T, _Float16); }

// A tile's packed data as a lane holds it.
template <int NG, int FMT>
struct Tile {
  uint4_t k[2], v[2];
  PairWord<FMT> pairs[NG];
};

// Which pair lane c of a row of 16 holds in pairs[q]: 16 NG pairs in the order [keys, values][block][token of four][group].
template <int NG>
struct PairSlot {
  int values, block, token, group;
  __device__ __forceinline__ PairSlot(int q, int c) {
    const int x = 16 * q + c;
    values = x / (8 * NG), block = x / (4 * NG) % 2, token = x / NG % 4, group = x % NG;
  }
  static constexpr int load_of(int values, int block, int token, int group) { return ((values * 2 + block) * 4 + token) * NG / 16 + 0 * group; }
  static constexpr int lane_of(int values, int block, int token, int group) { return (((values * 2 + block) * 4 + token) * NG + group) % 16; }
};

struct Out {
  void *out;
  long long stride;
  float *f32;
};

// A unit's rows: up to RB blocks of 16 (query token, query head) rows of a kv head of one sequence.
struct RowBlock {
  int i;      // sequence
  Sequence s;
  int first;  // first of its rows, of n_new * R
  int count;  // rows here
};
// Row y of the unit: its query token's row of the token arrays, its query head.
struct QueryRow {
  int token, head;
};
__device__ __forceinline__ QueryRow query_row(const PagedLayout &L, const RowBlock &x, int h, int row) {
  const int y = x.first + row, j = quotient(y, L.recip_R);
  return QueryRow{x.s.row0 + j, h * L.R + y - j * L.R};
}

template <class T>
__device__ __forceinline__ void store_out(const PagedLayout &L, const Out &o, const QueryRow &q, int channel, float x) {
  if (o.out) reinterpret_cast<T *>(o.out)[q.token * o.stride + q.head * kD + channel] = (T)x;
  if (o.f32) o.f32[((long long)q.token * L.Hq + q.head) * kD + channel] = x;
}

// Sum over the lanes up to this one, by moves within the register file (a shuffle goes through LDS).
template <class V>
__device__ __forceinline__ V lanes_up_to(V x) {
  auto moved = [](V v, auto ctrl, auto rows) {
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, decltype(rows)::value, 0xF, false));
  };
  typedef std::integral_constant<int, 0xF> all;
  x += moved(x, std::integral_constant<int, 0x111>{}, all{});  // one lane up within the row of 16; 2, 4, 8
  x += moved(x, std::integral_constant<int, 0x112>{}, all{});
  x += moved(x, std::integral_constant<int, 0x114>{}, all{});
  x += moved(x, std::integral_constant<int, 0x118>{}, all{});
  x += moved(x, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});  // the last lane of rows 0 and 2 to the next rows
  x += moved(x, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});  // lane 31 to the upper half
  return x;
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
template <class V>
__device__ __forceinline__ V last_lane(V x) {
  return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

// A sequence of the batch with its run, and how many: `blocks` units' worth of query rows (none where its counts are bad).
struct Member {
  Sequence s;
  Run run;
  int blocks;
};
__device__ __forceinline__ int table_capacity(const PagedLayout &L, const PagedBatch &b) {
  const long long n = (long long)b.table_stride << L.page_log2;
  return n < 0x7fffffff ? (int)n : 0x7fffffff;
}
template <int RB>
__device__ __forceinline__ Member member_in_lane(const PagedLayout &L, const PagedBatch &b, int i) {
  Member m;
  m.s = sequence_of(b, L, i < b.n_seqs ? i : b.n_seqs - 1);
  m.blocks = i < b.n_seqs && m.s.counts_ok ? (m.s.n_new * L.R + 16 * RB - 1) / (16 * RB) : 0;
  if (i >= b.n_seqs) m.s.counts_ok = true;
  m.run = run_of(m.s.counts_ok ? m.s.total : 1, L.W, L.S, table_capacity(L, b));
  return m;
}
// Work of all runs of a lane's sequence.  (No call has kPagedMostWork in all, the host refuses it; counts that contradict
// each other may.)
__device__ __forceinline__ unsigned work_in_lane(const Member &m) {
  const unsigned long long w = (unsigned long long)m.blocks * (unsigned)(m.run.row_weight + m.run.steps);
  return w < kPagedMostWork ? (unsigned)w : kPagedMostWork;
}
// What a workgroup needs to know of the batch.  The first 64 sequences are kept in LDS, written by the first wavefront.
struct BatchPlan {
  int share, work;  // a workgroup's, all (per kv head)
  unsigned upto;    // work of the sequences up to number `lane`
};
template <int RB>
__device__ __forceinline__ BatchPlan plan_batch(const PagedLayout &L, const PagedBatch &b, int groups, Member (&members)[64]) {
  const int lane = threadIdx.x & 63;
  BatchPlan p;
  Member m = member_in_lane<RB>(L, b, lane);
  if (threadIdx.x < 64) members[lane] = m;
  p.upto = lanes_up_to(work_in_lane(m));
  unsigned work = last_lane(p.upto);
  float about = last_lane(lanes_up_to((float)work_in_lane(m)));
  float most = m.blocks > 0 ? (float)m.run.steps : 0.0f;  // (at most 2^24)
  bool bad = !m.s.counts_ok;
  for (int i0 = 64; i0 < b.n_seqs; i0 += 64) {
    m = member_in_lane<RB>(L, b, i0 + lane);
    work += last_lane(lanes_up_to(work_in_lane(m)));
    about += last_lane(lanes_up_to((float)work_in_lane(m)));
    most = fmaxf(most, m.blocks > 0 ? (float)m.run.steps : 0.0f);
    bad = bad || !m.s.counts_ok;
  }
  if (about > 1.001f * kPagedMostWork) {
    bad = true;
    work = 0;
  }
  if (bad && blockIdx.x == 0 && blockIdx.y == 0) atomicOr(L.errors, SKVQ_PAGED_BAD_COUNTS);
  most = row_max(most);
  most = fmaxf(most, __shfl_xor(most, 16));
  most = fmaxf(most, __shfl_xor(most, 32));
  p.work = uniform((int)work);
  p.share = share_of(p.work, uniform((int)most), groups);
  return p;
}
// The run that work item `at` of the batch lies in: its sequence and rows, and how far into the run it is.
template <int RB>
__device__ __forceinline__ RowBlock find_run(const PagedLayout &L, const PagedBatch &b, const BatchPlan &p, const Member (&members)[64], int at,
                                             Run &run, int &done) {
  const int lane = threadIdx.x & 63;
  RowBlock x;
  int i0 = 0;
  unsigned upto = p.upto, y = (unsigned)at;
  while (last_lane(upto) <= y && i0 + 64 < b.n_seqs) {
    y -= last_lane(upto);
    i0 += 64;
    upto = lanes_up_to(work_in_lane(member_in_lane<RB>(L, b, i0 + lane)));
  }
  const unsigned long long behind = __ballot(upto > y);
  const int k = uniform(behind ? __ffsll(behind) - 1 : 63);
  if (k > 0) y -= (unsigned)__builtin_amdgcn_readlane((int)upto, k - 1);
  x.i = i0 + k < b.n_seqs ? i0 + k : b.n_seqs - 1;
  const Member m = i0 ? member_in_lane<RB>(L, b, x.i) : members[k];  // (the same in every lane)
  x.s = Sequence{uniform(m.s.row0), uniform(m.s.n_new), uniform(m.s.total), uniform(m.s.slot), true, false};
  x.s.slot_ok = x.s.slot >= 0 && x.s.slot < L.max_seqs;
  run = Run{uniform(m.run.n_kept), uniform(m.run.n_win), uniform(m.run.nq), uniform(m.run.rows), uniform(m.run.row_weight), uniform(m.run.steps)};
  done = (int)y;
  x.first = 0;
  if (uniform(m.blocks) > 1) {
    const int block = done / (run.row_weight + run.steps);
    done -= block * (run.row_weight + run.steps);
    x.first = 16 * RB * block;
  }
  const int left = x.s.n_new * L.R - x.first;
  x.count = left < 16 * RB ? left : 16 * RB;
  return x;
}

// A wavefront's running state: lane (g, c) = (lane / 16, lane % 16) holds row c's share.
template <int NG>
struct State {
  float4_t o[8];      // packed: positions 16n + 4g + reg; full rows: channels 8 (4g + reg) + n
  float m, l, z[NG];  // reference; this lane's share of the sum of weights, of weights times zeros less the middle codes
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int n = 0; n < 8; ++n) o[n] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    m = kNothing;
    l = 0.0f;
#pragma unroll
    for (int g = 0; g < NG; ++g) z[g] = 0.0f;
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
    for (int g = 0; g < NG; ++g) z[g] *= f;
#pragma unroll
    for (int n = 0; n < 8; ++n) o[n] *= f;
  }
};

// One tile of packed rows for RB blocks of query rows.  MASKED: some of its rows are behind the last (what stands
// there may be anything) or behind what some query sees.  left: rows of the tile before the end; seen: before the last one
// that the lane's row sees.  queries(r, j): block r's B operand for key dwords j; alpha: on the scores, with the code's unit.
template <class T, int NG, int FMT, int RB, bool MASKED, class Q, class Next>
__device__ __forceinline__ void take_tile(State<NG> (&st)[RB], Tile<NG, FMT> &t, const Next &next, const Q &queries, const float (&qs)[RB][NG],
                                          const float (&alpha)[RB], int left, const int (&seen)[RB], int g, int c) {
  typedef PairSlot<NG> Slot;
  // scale and zero (of values: with the middle code in it, see above); the logarithm of the largest scale of the lane's row of values
  float scale[NG], zero[NG], most = 0.0f;
#pragma unroll
  for (int q = 0; q < NG; ++q) {
    const Slot slot(q, c);
    const float2 pair = t.pairs[q].value();
    const bool there = !MASKED || 16 * slot.block + 4 * g + slot.token < left;
    const float x = there ? pair.x : 0.0f, z = there ? pair.y : 0.0f;
    scale[q] = x;
    if (NG == 1) {  // (keys and values side by side)
      zero[q] = two_parts<T>() ? z : fmaf(x, slot.values ? kMidCode : 0.0f, z);
      most = slot.values ? x : 0.0f;
    } else if (q < NG / 2) {
      zero[q] = z;
    } else {
      zero[q] = two_parts<T>() ? z : fmaf(x, kMidCode, z);
      most = fmaxf(most, x);
    }
  }
  next.pairs(t);
  most = fmaxf(__builtin_amdgcn_logf(row_max(most)), kLowestLog);
  // Broadcasts of a pair serve all blocks of rows; those of the next pairs wait (side by side they would fill the registers).
  auto separate = [] {
    if (RB > 1) __builtin_amdgcn_sched_barrier(0);
  };
  if (RB > 1) __atomic_signal_fence(__ATOMIC_ACQ_REL);  // (the queries are read again: holding them takes 32 registers)
  float s[RB][8], top[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) top[b] = -INFINITY;
  const unsigned mask = 0x00f000f0u;
  unrolled<0, 2>([&](auto I) {
    constexpr int i = I();
    float4_t acc[RB][NG], x[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      x[b] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int n = 0; n < NG; ++n) acc[b][n] = x[b];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned w = t.k[i][j];
      const half8_t codes = as_half8((w << 4) & mask, w & mask, (w >> 4) & mask, (w >> 8) & mask);
#pragma unroll
      for (int b = 0; b < RB; ++b) acc[b][j * NG / 4] = mfma(codes, queries(b, j), acc[b][j * NG / 4]);
    }
    separate();
    unrolled<0, 4>([&](auto R) {
      constexpr int r = R();
      float codes[RB];
      unrolled<0, NG>([&](auto N) {
        constexpr int n = N(), q = Slot::load_of(0, i, r, n), lane = Slot::lane_of(0, i, r, n);
        const float by = of_lane<lane>(scale[q]), z = of_lane<lane>(zero[q]);
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          x[b][r] = n == 0 ? z * qs[b][0] : fmaf(z, qs[b][n], x[b][r]);
          codes[b] = n == 0 ? by * acc[b][0][r] : fmaf(by, acc[b][n][r], codes[b]);
        }
      });
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const bool there = !MASKED || 16 * i + 4 * g + r < min(left, seen[b]);
        s[b][4 * i + r] = there ? fmaf(codes[b], alpha[b], x[b][r]) : -INFINITY;
        top[b] = fmaxf(top[b], s[b][4 * i + r]);
      }
      separate();
    });
  });
  next.keys(t);
#pragma unroll
  for (int b = 0; b < RB; ++b) st[b].refer(top[b] + most);
  half8_t pb[RB][NG], rest[RB][NG];
  unrolled<0, 8>([&](auto I) {
    constexpr int i = I() / 4, r = I() % 4;
    float p[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      p[b] = __builtin_amdgcn_exp2f(s[b][I()] - st[b].m);
      st[b].l += p[b];
    }
    unrolled<0, NG>([&](auto N) {
      constexpr int n = N(), q = Slot::load_of(1, i, r, n), lane = Slot::lane_of(1, i, r, n);
      const float by = of_lane<lane>(scale[q]), z = of_lane<lane>(zero[q]);
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        st[b].z[n] = fmaf(z, p[b], st[b].z[n]);
        const float w = by * p[b];
        pb[b][n][I()] = (_Float16)w;
        const half2_t middle = {-(_Float16)kMidCode, -(_Float16)kMidCode};
        if (two_parts<T>())
          rest[b][n][I()] = (_Float16)(w - (float)pb[b][n][I()]);
        else if (r % 2)
          st[b].z[n] = __builtin_amdgcn_fdot2(half2_t{pb[b][n][I() & ~1], pb[b][n][I()]}, middle, st[b].z[n], false);
      }
    });
    separate();
  });
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    unsigned a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned w = t.v[i / 2][2 * (i % 2) + n / 4];
      a[i] = (n % 4 == 0 ? w << 4 : n % 4 == 1 ? w : n % 4 == 2 ? w >> 4 : w >> 8) & mask;
    }
    const half8_t codes = as_half8(a[0], a[1], a[2], a[3]);
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      st[b].o[n] = mfma(codes, pb[b][n * NG / 8], st[b].o[n]);
      if (two_parts<T>()) st[b].o[n] = mfma(codes, rest[b][n * NG / 8], st[b].o[n]);
    }
  }
  next.values(t);
}

template <class T, int RB>
struct Lds {
  union alignas(16) {
    T q[16 * RB][kD + 8];         // the queries ...
    _Float16 h[16 * RB][kD + 8];  // ... for packed rows: as fp16 numbers, a head's channels in the order of the key codes
    float acc[kWaves][16][kRowStride];
  };
  float m[kWaves][16], l[kWaves][16];
  float unit[16 * RB];  // what 1 stands for in h
  int bad;
  Member members[64];
};

// The last token that a row of the unit sees (rows past the last one: as that).
__device__ __forceinline__ int last_token(const PagedLayout &L, const RowBlock &x, int row) {
  return x.s.total - x.s.n_new + quotient(x.first + (row < x.count ? row : x.count - 1), L.recip_R);
}

// Pages of the wavefront's tiles k0 .. k0 + 31 of packed rows begin .. end - 1, two blocks of 16 tokens each: lane
// 2k + i holds tile k0 + k's block i.
__device__ __forceinline__ int pages_of_tiles(const PagedLayout &L, const PagedBatch &b, int seq, int begin, int end, int k0, bool &bad) {
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int te = begin + kTile * (wave + kWaves * (k0 + (lane >> 1))) + 16 * (lane & 1);
  int id = 0;
  if (te < end) {
    const int at = te >> L.page_log2;
    id = page_known(at, b.table_stride) ? b.table[(long long)seq * b.table_stride + at] : -1;
    if (!page_valid(id, L.n_pages)) {
      bad = true;
      id = 0;
    }
  }
  return id;
}

// The wavefront's share of packed rows begin .. end - 1.  ids: pages_of_tiles of its first tiles.
template <class T, int NG, int FMT, int RB>
__device__ __forceinline__ void take_packed(const PagedLayout &L, const PagedBatch &b, const Lds<T, RB> &lds, const RowBlock &x, int begin, int end,
                                            int h, int ids, State<NG> (&st)[RB], bool &bad) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
  int seen[RB];  // packed rows that the lane's row sees; all rows see the first one's
#pragma unroll
  for (int r = 0; r < RB; ++r) seen[r] = last_token(L, x, 16 * r + c) + 1 - L.S;
  const int all_see = min(end, last_token(L, x, 0) + 1 - L.S);
  const int n_tiles = (end - begin + kTile - 1) / kTile, mine = n_tiles > wave ? (n_tiles - wave + kWaves - 1) / kWaves : 0;
  const uint8_t *head_part = L.pages + (long long)h * L.part_bytes;
  const long long page_stride = (long long)L.Hk * L.part_bytes;
  constexpr int kPair = PairWord<FMT>::kSize;
  const unsigned k_lane = c * (kD / 2) + 16 * g, v_lane = L.v_at + 256 * g + 16 * c;
  unsigned pair_lane[NG];
  bool pair_block[NG];
#pragma unroll
  for (int q = 0; q < NG; ++q) {
    const PairSlot<NG> slot(q, c);
    pair_lane[q] = (slot.values ? L.vm_at : L.km_at) + kPair * ((4 * g + slot.token) * NG + slot.group);
    pair_block[q] = slot.block;
  }
  // Loads of the wavefront's k-th tile, of those that `ids` holds from the k0-th on (blocks past the end: of page 0).
  // Codes are read once per unit, by instructions that take whole lines: streaming loads.
  struct Next {
    const PagedLayout &L;
    const unsigned k_lane, v_lane, (&pair_lane)[NG];
    const bool (&pair_block)[NG];
    const uint8_t *part[2];
    unsigned place[2];
    __device__ __forceinline__ uint4_t codes(int i, unsigned lane) const {
      return __builtin_nontemporal_load(reinterpret_cast<const uint4_t *>(part[i] + place[i] * (kD / 2) + lane));
    }
    __device__ __forceinline__ void pairs(Tile<NG, FMT> &t) const {
      const uint8_t *p0 = part[0] + place[0] * (NG * kPair), *p1 = part[1] + place[1] * (NG * kPair);
#pragma unroll
      for (int q = 0; q < NG; ++q) t.pairs[q].load((pair_block[q] ? p1 : p0) + pair_lane[q]);
    }
    __device__ __forceinline__ void keys(Tile<NG, FMT> &t) const {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        t.k[i] = codes(i, k_lane);
      }
    }
    __device__ __forceinline__ void values(Tile<NG, FMT> &t) const {
#pragma unroll
      for (int i = 0; i < 2; ++i) t.v[i] = codes(i, v_lane);
    }
  };
  auto tile = [&](int k, int k0) {
    Next x{L, k_lane, v_lane, pair_lane, pair_block, {}, {}};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int id = __builtin_amdgcn_readlane(ids, 2 * (k - k0) + i);
      const int te = begin + kTile * (wave + kWaves * k) + 16 * i;
      x.place[i] = te & ((1 << L.page_log2) - 1);
      x.part[i] = head_part + id * page_stride;
    }
    return x;
  };
  Tile<NG, FMT> t;
  if (mine > 0) {
    const Next x = tile(0, 0);
    x.pairs(t);
    x.keys(t);
    x.values(t);
  }
  // B operand of block r: row c's queries at the reordered positions of key dword 4g + j.  One block's stay in registers,
  // more are read for every tile.
  half8_t held[RB == 1 ? 4 : 1];
  auto queries = [&](int r, int j) { return RB == 1 ? held[j] : *reinterpret_cast<const half8_t *>(&lds.h[16 * r + c][8 * (4 * g + j)]); };
  float qs[RB][NG], alpha[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    const float scale = L.sm_scale * kLog2e * lds.unit[16 * r + c];
    alpha[r] = scale * kCodeUnit;
#pragma unroll
    for (int n = 0; n < NG; ++n) qs[r][n] = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const half8_t v = *reinterpret_cast<const half8_t *>(&lds.h[16 * r + c][8 * (4 * g + j)]);
      if (RB == 1) held[j] = v;
#pragma unroll
      for (int e = 0; e < 8; ++e) qs[r][j * NG / 4] += (float)v[e];
    }
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      qs[r][n] += __shfl_xor(qs[r][n], 16);
      qs[r][n] += __shfl_xor(qs[r][n], 32);
      qs[r][n] *= scale;
    }
  }
  // Whole tiles that every query sees, then the others (at the end).  The lanes hold the pages of 32 tiles, and the
  // next tile's pairs, key codes and value codes are asked for as soon as this one's have been used (the last one's loads are
  // repeated: no branch between loads and what they hide behind): 31 tiles a turn.
  const int whole_tiles = all_see > begin ? (all_see - begin) / kTile : 0;
  const int whole = whole_tiles > wave ? (whole_tiles - wave + kWaves - 1) / kWaves : 0;
  for (int k0 = 0; k0 < mine; k0 += 31) {
    if (k0 > 0) ids = pages_of_tiles(L, b, x.i, begin, end, k0, bad);
    const int stop = min(mine, k0 + 31), stop_whole = min(stop, whole);
    int k = k0;
    for (; k < stop_whole; ++k)
      take_tile<T, NG, FMT, RB, false>(st, t, tile(min(k + 1, mine - 1), k0), queries, qs, alpha, 0, seen, g, c);
    for (; k < stop; ++k) {
      const int te0 = begin + kTile * (wave + kWaves * k);
      int seen_here[RB];
#pragma unroll
      for (int r = 0; r < RB; ++r) seen_here[r] = seen[r] - te0;
      take_tile<T, NG, FMT, RB, true>(st, t, tile(min(k + 1, mine - 1), k0), queries, qs, alpha, end - te0, seen_here, g, c);
    }
  }
}

// ... of full-precision rows: the u-th of the kept and the ring tokens, in the order of their numbers.
template <class T, int NG, int RB>
__device__ __forceinline__ void take_rows(const PagedLayout &L, const Lds<T, RB> &lds, const RowBlock &x, const Run &ch, int begin, int end,
                                          int h, int block, State<NG> &st) {
  typedef T t8 __attribute__((ext_vector_type(8)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
  const int last = last_token(L, x, 16 * block + c);
  const float scale = L.sm_scale * kLog2e;
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
  for (int j = 0; j < 4; ++j) qb[j] = *reinterpret_cast<const t8 *>(&lds.q[16 * block + c][32 * j + 8 * g]);
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
      st.o[n] = mfma(a, lo, st.o[n]);
    }
  }
}

template <class T, int NG, int FMT, int RB>
__global__ __launch_bounds__(64 * kWaves, groups_per_cu(NG, RB)) void paged_attention_kernel(const PagedLayout L, const PagedBatch b,
                                                                                        const TokenRows q, const Out out, int n_row_chunks) {
  typedef Piece<T, 8> P;
  __shared__ Lds<T, RB> lds;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
  const int h = blockIdx.x;  // (heads side by side: a head's workgroups share a chiplet's L2)
  const unsigned long long places = *reinterpret_cast<const unsigned long long *>(L.k_place + h * kD + 8 * c);
  const int p = threadIdx.x % kD, packed_channel = L.v_offset[h * kD + 8 * (p & 15) + (p >> 4)] / 2;  // of the output place it writes
  const BatchPlan plan = plan_batch<RB>(L, b, gridDim.y, lds.members);
  __syncthreads();
  const long long mine_from = (long long)plan.share * blockIdx.y;
  const int stop = (int)min((long long)plan.work, mine_from + plan.share);
  int next = 0;
  for (int at = (int)min(mine_from, (long long)plan.work); at < stop; at += next) {
    Run run;
    int done;
    const RowBlock x = find_run<RB>(L, b, plan, lds.members, at, run, done);
    const Portion part = portion_of(run, done, at, stop, plan.share);
    next = part.work;
    if (!part.there) continue;
    const bool packed = part.packed;
    // the queries, sixteen threads a row, rows past the last one repeat it; the first pages meanwhile
    static_assert(64 * kWaves == 16 * 16, "one piece of a row per thread");
    const int query = threadIdx.x >> 4;
    P mine[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const QueryRow from = query_row(L, x, h, min(16 * r + query, x.count - 1));
      mine[r] = *reinterpret_cast<const P *>((const T *)q.p + from.token * q.stride + from.head * kD + 8 * c);
    }
    bool bad = run.nq > table_capacity(L, b);
    const int ids = packed ? pages_of_tiles(L, b, x.i, part.begin, part.end, 0, bad) : 0;
    __syncthreads();  // (the portion before has read its partials out of LDS)
    if (threadIdx.x == 0) {
      lds.bad = !x.s.slot_ok;
      if (!x.s.slot_ok) atomicOr(L.errors, SKVQ_PAGED_BAD_SLOT);
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      if (packed) {
        // bf16 queries are brought to fp16's range by one power of two: what that makes subnormal is 2^-25 of the largest.
        float to_half = 1.0f;
        if constexpr (!__is_same(T, _Float16)) {
          float largest = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) largest = fmaxf(largest, fabsf((float)mine[r][e]));
          largest = row_max(largest);
          const int exponent = largest > 0.0f ? 14 - __builtin_amdgcn_frexp_expf(largest) : 0;  // largest in [2^(e-1), 2^e)
          to_half = __builtin_amdgcn_ldexpf(1.0f, exponent < 126 ? exponent : 126);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          _Float16 &to = lds.h[16 * r + query][(places >> (8 * e)) & 0xffu];
          if constexpr (__is_same(T, _Float16))
            to = mine[r][e];
          else
            to = (_Float16)((float)mine[r][e] * to_half);
        }
        if (c == 0) lds.unit[16 * r + query] = 1.0f / to_half;
      } else {
        *reinterpret_cast<P *>(&lds.q[16 * r + query][8 * c]) = mine[r];
      }
    }
    __syncthreads();
    State<NG> st[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) st[r].clear();
    if (packed) {
      take_packed<T, NG, FMT, RB>(L, b, lds, x, part.begin, part.end, h, ids, st, bad);
    } else if (x.s.slot_ok) {
#pragma unroll
      for (int r = 0; r < RB; ++r) take_rows<T, NG, RB>(L, lds, x, run, part.begin, part.end, h, r, st[r]);
    }

    // The wavefronts' states: sums over the lanes of a row, then one reference for the workgroup.
    const int most = kPagedMaxSplits + n_row_chunks;
    const int channel = packed ? packed_channel : p;
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      State<NG> &own = st[r];
      own.l += __shfl_xor(own.l, 16);
      own.l += __shfl_xor(own.l, 32);
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        own.z[n] += __shfl_xor(own.z[n], 16);
        own.z[n] += __shfl_xor(own.z[n], 32);
      }
      if (r > 0) __syncthreads();  // (the block before has been read out of LDS)
      if (g == 0) {
        lds.m[wave][c] = own.m;
        lds.l[wave][c] = own.l;
      }
      __syncthreads();  // (also: the queries in LDS are no longer needed)
      if (r == 0 && bad) {
        lds.bad = 1;
        atomicOr(L.errors, SKVQ_PAGED_BAD_PAGE);
      }
      float top = lds.m[0][c];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) top = fmaxf(top, lds.m[w][c]);
      const float f = __builtin_amdgcn_exp2f(own.m - top);
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        float4_t y = own.o[n];
        if (packed) {
          y = (y * kCodeUnit + own.z[n * NG / 8]) * f;
          *reinterpret_cast<float4_t *>(&lds.acc[wave][c][16 * n + 4 * g]) = y;
        } else {
          y *= f;
#pragma unroll
          for (int k = 0; k < 4; ++k) lds.acc[wave][c][8 * (4 * g + k) + n] = y[k];
        }
      }
      __syncthreads();
      for (int row = threadIdx.x / kD; row < min(x.count - 16 * r, 16); row += 64 * kWaves / kD) {
        float acc = lds.acc[0][row][p], m = lds.m[0][row], l = 0.0f;
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
          acc += lds.acc[w][row][p];
          m = fmaxf(m, lds.m[w][row]);
        }
#pragma unroll
        for (int w = 0; w < kWaves; ++w) l += lds.l[w][row] * __builtin_amdgcn_exp2f(lds.m[w][row] - m);
        if (lds.bad) l = NAN;
        const QueryRow qr = query_row(L, x, h, 16 * r + row);
        float *to = L.workspace + ((long long)qr.token * L.Hq + qr.head) * most * kPartialStride;
        if (part.n_partials == 1) {
          store_out<T>(L, out, qr, channel, acc / l);
        } else {
          float *mine_to = to + part.partial * kPartialStride;
          mine_to[4 + channel] = acc;
          if (p == 0) {
            mine_to[0] = m;
            mine_to[1] = l;
          }
        }
        if (p == 0 && part.partial == 0) to[2] = __uint_as_float((unsigned)part.n_partials);  // (for the merge)
      }
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
  const int token = blockIdx.x, tid = threadIdx.x, group = tid >> 5, t = tid & 31;
  const QueryRow qr = {token, (int)blockIdx.y};
  const float *from = L.workspace + ((long long)token * L.Hq + qr.head) * (kPagedMaxSplits + n_row_chunks) * kPartialStride;
  auto partial = [&](int i) { return from + (long long)i * kPartialStride; };
  // (anything where the token is of no sequence, or nothing was done)
  const int n = min((int)__float_as_uint(from[2]), kPagedMaxSplits + n_row_chunks);
  const Sequence s = sequence_of(b, L, sequence_of_unit(b, token, kTokenDeal));
  if (!s.counts_ok || token < s.row0 || token >= s.row0 + s.n_new || n <= 1) return;
  float m = kNothing, l = 0.0f;
  float4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i0 = 0; i0 < n; i0 += kMergeThreads) {  // (more than 256 only with windows of ten thousands of tokens)
    const int here = min(kMergeThreads, n - i0);
    const float2 ml = tid < here ? *reinterpret_cast<const float2 *>(partial(i0 + tid)) : make_float2(kNothing, 0.0f);
    const float mi = ml.x;
    float top = row_max(mi);
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    if ((tid & 63) == 0) red[0][tid >> 6] = top;
    __syncthreads();
    top = m;
#pragma unroll
    for (int w = 0; w < kMergeThreads / 64; ++w) top = fmaxf(top, red[0][w]);
    const float w = tid < here ? __builtin_amdgcn_exp2f(mi - top) : 0.0f, before = __builtin_amdgcn_exp2f(m - top);
    weight[tid] = w;
    const float sum = last_lane(lanes_up_to(ml.y * w));
    if ((tid & 63) == 0) red[1][tid >> 6] = sum;
    __syncthreads();
    l *= before;
#pragma unroll
    for (int w = 0; w < kMergeThreads / 64; ++w) l += red[1][w];
    acc *= before;
    m = top;
    int i = group;
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
  parts[group][t] = acc;
  __syncthreads();
  if (tid < kD) {
    float x = 0.0f;
#pragma unroll
    for (int k = 0; k < kMergeGroups; ++k) x += reinterpret_cast<const float *>(&parts[k][0])[tid];
    store_out<T>(L, out, qr, tid, x / l);
  }
}

template <class T, int NG, int RB>
void launch_formats(const PagedLayout &L, const PagedBatch &b, TokenRows q, Out out, int row_chunks, unsigned groups, hipStream_t s) {
  const dim3 grid(L.Hk, groups), threads(64 * kWaves);
  switch (L.meta_fmt) {
    case SKVQ_META_F32: paged_attention_kernel<T, NG, SKVQ_META_F32, RB><<<grid, threads, 0, s>>>(L, b, q, out, row_chunks); break;
    case SKVQ_META_F16: paged_attention_kernel<T, NG, SKVQ_META_F16, RB><<<grid, threads, 0, s>>>(L, b, q, out, row_chunks); break;
    default: paged_attention_kernel<T, NG, SKVQ_META_FP8_E4M3, RB><<<grid, threads, 0, s>>>(L, b, q, out, row_chunks); break;
  }
}

template <class T, int RB>
hipError_t launch_typed(const PagedLayout &L, const PagedBatch &b, TokenRows q, Out out, int row_chunks, unsigned groups, hipStream_t s) {
  switch (L.NG) {
    case 1: launch_formats<T, 1, RB>(L, b, q, out, row_chunks, groups, s); break;
    case 2: launch_formats<T, 2, RB>(L, b, q, out, row_chunks, groups, s); break;
    default: launch_formats<T, 4, RB>(L, b, q, out, row_chunks, groups, s); break;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  paged_merge_kernel<T><<<dim3((unsigned)b.n_tokens, L.Hq), kMergeThreads, 0, s>>>(L, b, out, row_chunks);
  return hipGetLastError();
}

}  // namespace

// Two blocks a unit where sequences have more than 16 rows on average (us with one -> two, 8 kv heads): 8 sequences of 40k
// tokens with 64 rows each, one group 258 -> 209, two 257 -> 198, four 312 -> 269, with 20 rows 139 -> 123; 1024 rows of a
// sequence of 32k 343 -> 310.  With 16 rows at most the second block would be idle.
static int row_blocks_of(long long rows, int n_seqs) { return rows > 16LL * n_seqs ? 2 : 1; }

long long paged_most_work(const PagedLayout &L, const skvq_batch &b) {
  const long long rows = (long long)b.n_tokens * L.R, capacity = (long long)b.table_stride << L.page_log2;
  const long long blocks = rows / (16 * row_blocks_of(rows, b.n_seqs)) + (b.n_seqs < b.n_tokens ? b.n_seqs : b.n_tokens);
  return blocks * (row_weight_of(L.W + L.S) + (capacity < 0x7fffffff ? steps_of((int)capacity, kPagedStep) : 1 << 24));
}

hipError_t launch_paged_attention(const PagedLayout &L, const skvq_batch &batch, TokenRows q, void *out, long long out_stride,
                                  float *out_f32, int n_cus, hipStream_t s) {
  const PagedBatch b = batch_of(batch);
  const int row_chunks = paged_row_chunks(L.W, L.S);
  // Lengths are not known here: as many workgroups as the chip holds at once, over the kv heads, unless there can be no
  // more work than that (every query token of a sequence of its own, as long as the page table allows).  Where a sequence
  // has more than 16 rows per kv head on average, a unit holds two blocks of them.
  const long long work = paged_most_work(L, batch), rows = (long long)b.n_tokens * L.R;
  const int row_blocks = row_blocks_of(rows, b.n_seqs);
  const long long most = (long long)groups_per_cu(L.NG, row_blocks) * n_cus / L.Hk;
  const unsigned groups = (unsigned)(work < most ? work : most > 0 ? most : 1);
  const Out o{out, out_stride, out_f32};
  if (L.dtype == SKVQ_DTYPE_BF16)
    return row_blocks == 2 ? launch_typed<__bf16, 2>(L, b, q, o, row_chunks, groups, s) : launch_typed<__bf16, 1>(L, b, q, o, row_chunks, groups, s);
  return row_blocks == 2 ? launch_typed<_Float16, 2>(L, b, q, o, row_chunks, groups, s) : launch_typed<_Float16, 1>(L, b, q, o, row_chunks, groups, s);
}

}  // namespace skvq
