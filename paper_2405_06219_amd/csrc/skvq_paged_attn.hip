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
// The weight that multiplies a code is weight * scale: the reference counts log2 of the token's largest scale in,
// so that this product, rounded to fp16 (half a step, 2^-12 of itself; a second part as in the fixed cache's kernel
// would refine what 16-bit outputs do not show), stays within fp16's normal numbers near the largest contributions.
// Zeros enter by fp32 sums: out = sum (w scale) code + sum w zero.
//
// Bound by HBM for long contexts: 136 bytes per (token, kv head) at one group.
#include <hip/hip_runtime.h>

#include "skvq_paged.h"

namespace skvq {
namespace {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef unsigned uint4_t __attribute__((ext_vector_type(4)));
typedef unsigned uint2_t __attribute__((ext_vector_type(2)));

constexpr int kWaves = kPagedWaves, kTile = kPagedTile;
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

// The (scale, zero) pairs of a lane's four tokens, as they come from memory.
template <int NG, int FMT>
struct PairWords {
  static constexpr int kSize = FMT == SKVQ_META_F32 ? 8 : FMT == SKVQ_META_F16 ? 4 : 2;
  static constexpr int kWords = 4 * NG * kSize / 4;
  unsigned w[kWords];
  __device__ __forceinline__ void load(const uint8_t *p) {
    if constexpr (kWords == 2) {
      const uint2_t x = *reinterpret_cast<const uint2_t *>(p);
      w[0] = x.x, w[1] = x.y;
    } else {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) {
        const uint4_t x = reinterpret_cast<const uint4_t *>(p)[i];
        w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
      }
    }
  }
  // of token i, group g
  __device__ __forceinline__ float2 pair(int i, int g) const {
    const int x = i * NG + g;
    if constexpr (FMT == SKVQ_META_F32) {
      return make_float2(__uint_as_float(w[2 * x]), __uint_as_float(w[2 * x + 1]));
    } else if constexpr (FMT == SKVQ_META_F16) {
      typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
      const half2_t h = __builtin_bit_cast(half2_t, w[x]);
      return make_float2((float)h[0], (float)h[1]);
    } else {
      const int word = (int)w[x / 2];
      return x % 2 ? make_float2(__builtin_amdgcn_cvt_f32_fp8(word, 2), __builtin_amdgcn_cvt_f32_fp8(word, 3))
                   : make_float2(__builtin_amdgcn_cvt_f32_fp8(word, 0), __builtin_amdgcn_cvt_f32_fp8(word, 1));
    }
  }
};

// A tile's packed data as a lane holds it.
template <int NG, int FMT>
struct Tile {
  uint4_t k[2], v[2];
  PairWords<NG, FMT> km[2], vm[2];
};

struct Out {
  void *out;
  long long stride;
  float *f32;
};

// Row x of a row block: query token j, query head of the kv head.
struct RowBlock {
  int i;          // sequence
  Sequence s;
  int first;      // first of its rows, of n_new * R
  int count;      // rows here (<= 0: none)
};
__device__ __forceinline__ RowBlock row_block(const PagedLayout &L, const PagedBatch &b, long long unit) {
  RowBlock x;
  const UnitDeal deal = row_deal(L.R);
  x.i = sequence_of_unit(b, unit, deal);
  x.s = sequence_of(b, L, x.i);
  x.count = 0;
  x.first = 0;
  if (x.s.counts_ok) {
    const long long at = 16 * (unit - unit_start(deal, x.s.row0, x.i)), n = (long long)x.s.n_new * L.R;
    if (at >= 0 && at < n) {
      x.first = (int)at;
      x.count = n - at < 16 ? (int)(n - at) : 16;
    }
  }
  return x;
}
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

// A wavefront's running state: lane (g, c) = (lane / 16, lane % 16) holds row c's share.
template <int NG>
struct State {
  float4_t o[8];       // packed: positions 16n + 4g + reg; rows: channels 8 (4g + reg) + n
  float m, l, z[NG];   // reference; this lane's share of the sum of weights, of weights times zeros
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

template <class T, int NG, int FMT>
__global__ __launch_bounds__(64 * kWaves, 2) void paged_attention_kernel(const PagedLayout L, const PagedBatch b, const TokenRows q,
                                                                         const Out out, int n_row_chunks, int n_splits) {
  typedef T t8 __attribute__((ext_vector_type(8)));
  typedef Piece<T, 8> P;
  __shared__ __align__(16) union {
    T q[16][kD + 8];
    float acc[kWaves][16][kRowStride];
  } lds;
  __shared__ float lds_m[kWaves][16], lds_l[kWaves][16];
  __shared__ int lds_bad;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
  const int h = blockIdx.y, n_chunks = n_row_chunks + n_splits;
  const RowBlock x = row_block(L, b, blockIdx.x / n_chunks);
  if (!x.s.counts_ok) {
    if (threadIdx.x == 0) atomicOr(L.errors, SKVQ_PAGED_BAD_COUNTS);
    return;
  }
  if (x.count <= 0) return;
  const Chunks ch = chunks_of(x.s.total, L.W, L.S, n_splits);
  const int at_chunk = blockIdx.x % n_chunks;
  const bool packed = at_chunk >= n_row_chunks;
  const int chunk = packed ? at_chunk - n_row_chunks : at_chunk;
  if (chunk >= (packed ? ch.packed : ch.rows)) return;
  if (threadIdx.x == 0) {
    lds_bad = !x.s.slot_ok;
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
  // lane's row: the last token it sees
  const int last = x.s.total - x.s.n_new + (x.first + (c < x.count ? c : x.count - 1)) / L.R;
  const float scale = L.sm_scale * kLog2e;
  State<NG> st;
  st.clear();
  bool bad = false;

  if (packed) {
    // B operand: row c's queries at the reordered positions of key dword 4g + j, as fp16 numbers.  bf16 queries are
    // brought to fp16's range by a power of two per row: what that makes subnormal is 2^-25 of the row's largest.
    half8_t qb[4];
    float qs[NG], alpha = scale * kCodeUnit;
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
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        const int exponent = most > 0.0f ? __builtin_amdgcn_frexp_expf(most) : 0;  // most in [2^(e-1), 2^e)
        to_half = __builtin_amdgcn_ldexpf(1.0f, 14 - exponent < 127 ? 14 - exponent : 126);
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
    const int seen = last + 1 - L.S;  // packed rows this lane's row sees
    const int begin = chunk * ch.chunk, end = min(ch.nq, begin + ch.chunk);
    const int n_tiles = (end - begin + kTile - 1) / kTile;
    const uint8_t *head_part = L.pages + (long long)h * L.part_bytes;
    const long long page_stride = (long long)L.Hk * L.part_bytes;
    const int *table = b.table + (long long)x.i * b.table_stride;
    const unsigned k_lane = c * (kD / 2) + 16 * g, v_lane = L.v_at + 256 * g + 16 * c;
    const unsigned km_lane = L.km_at + 4 * g * NG * PairWords<NG, FMT>::kSize, vm_lane = L.vm_at + 4 * g * NG * PairWords<NG, FMT>::kSize;
    // Pages of the wavefront's next 32 tiles, two blocks of 16 tokens each: lane 2k + i holds tile k's block i.
    int ids = 0;
    auto look_up = [&](int k0) {
      const int te = begin + kTile * (wave + kWaves * (k0 + (lane >> 1))) + 16 * (lane & 1);
      ids = 0;
      if (te < end) {
        const int at = te >> L.page_log2;
        ids = at < b.table_stride ? table[at] : -1;
        if (ids < 0 || ids >= L.n_pages) {
          bad = true;
          ids = 0;
        }
      }
    };
    auto load = [&](Tile<NG, FMT> &t, int k) {  // the wavefront's k-th tile (any k: past the end page 0 is read)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int id = __builtin_amdgcn_readlane(ids, 2 * (k & 31) + i);
        const int te = begin + kTile * (wave + kWaves * k) + 16 * i;
        const int place = te & ((1 << L.page_log2) - 1);
        const uint8_t *p = head_part + id * page_stride;
        t.k[i] = *reinterpret_cast<const uint4_t *>(p + (unsigned)place * (kD / 2) + k_lane);
        t.v[i] = *reinterpret_cast<const uint4_t *>(p + (unsigned)place * (kD / 2) + v_lane);
        t.km[i].load(p + (unsigned)place * (NG * PairWords<NG, FMT>::kSize) + km_lane);
        t.vm[i].load(p + (unsigned)place * (NG * PairWords<NG, FMT>::kSize) + vm_lane);
      }
    };
    const int mine = n_tiles > wave ? (n_tiles - wave + kWaves - 1) / kWaves : 0;
    Tile<NG, FMT> next;
    if (mine > 0) {
      look_up(0);
      load(next, 0);
    }
    for (int k = 0; k < mine; ++k) {
      const Tile<NG, FMT> t = next;
      if (k + 1 < mine) {
        if (((k + 1) & 31) == 0) look_up(k + 1);
        load(next, k + 1);
      }
      const int te0 = begin + kTile * (wave + kWaves * k);
      // scores in base 2, and the logarithms of what will multiply codes
      float s[2][4], top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float4_t acc[NG];
#pragma unroll
        for (int n = 0; n < NG; ++n) acc[n] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const unsigned w = t.k[i][j], mask = 0x00f000f0u;
          acc[j * NG / 4] = mfma(as_half8((w << 4) & mask, w & mask, (w >> 4) & mask, (w >> 8) & mask), qb[j], acc[j * NG / 4]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float dot = 0.0f, most = 0.0f, z = 0.0f;
#pragma unroll
          for (int n = 0; n < NG; ++n) {
            const float2 pk = t.km[i].pair(r, n);
            dot = fmaf(pk.x, acc[n][r], dot);
            z = fmaf(pk.y, qs[n], z);
            most = fmaxf(most, t.vm[i].pair(r, n).x);
          }
          s[i][r] = fmaf(dot, alpha, z);
          const float lg = fmaxf(__builtin_amdgcn_logf(most), kLowestLog);
          const bool there = te0 + 16 * i + 4 * g + r < min(end, seen);
          s[i][r] = there ? s[i][r] : -INFINITY;
          top = fmaxf(top, there ? s[i][r] + lg : -INFINITY);
        }
      }
      st.refer(top);
      half8_t pb[NG];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float p = __builtin_amdgcn_exp2f(s[i][r] - st.m);
          const bool there = te0 + 16 * i + 4 * g + r < end;  // (what lies behind the last row may be anything)
          st.l += p;
#pragma unroll
          for (int n = 0; n < NG; ++n) {
            const float2 pv = t.vm[i].pair(r, n);
            const float w = p * (there ? pv.x : 0.0f);
            pb[n][4 * i + r] = (_Float16)w;
            st.z[n] = fmaf(p, there ? pv.y : 0.0f, st.z[n]);
            st.z[n] = fmaf(w - (float)pb[n][4 * i + r], kMidCode, st.z[n]);
          }
        }
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        unsigned a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned w = t.v[i / 2][2 * (i % 2) + n / 4], mask = 0x00f000f0u;
          a[i] = (n % 4 == 0 ? w << 4 : n % 4 == 1 ? w : n % 4 == 2 ? w >> 4 : w >> 8) & mask;
        }
        st.o[n] = mfma(as_half8(a[0], a[1], a[2], a[3]), pb[n * NG / 8], st.o[n]);
      }
    }
  } else if (x.s.slot_ok) {
    // Full-precision rows: u-th of the kept and the ring tokens, in the order of their numbers.
    const int n_full = ch.n_kept + ch.n_win, begin = chunk * kPagedRowsPerChunk, end = min(n_full, begin + kPagedRowsPerChunk);
    const long long head = ((long long)x.s.slot * L.Hk + h) * (L.W + L.S) * kD;
    const T *k_rows = reinterpret_cast<const T *>(L.k_rows) + head, *v_rows = reinterpret_cast<const T *>(L.v_rows) + head;
    const int first_recent = x.s.total - ch.n_win;
    auto row_of = [&](int u) {  // (rows past the end: the first, which holds a token)
      u = u < end ? u : begin;
      return u < ch.n_kept ? L.W + u : (first_recent + u - ch.n_kept) % L.W;
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

  // The wavefronts' states: sums over the lanes of a row, then one reference for the workgroup.
  st.l += __shfl_xor(st.l, 16);
  st.l += __shfl_xor(st.l, 32);
#pragma unroll
  for (int n = 0; n < NG; ++n) {
    st.z[n] += __shfl_xor(st.z[n], 16);
    st.z[n] += __shfl_xor(st.z[n], 32);
  }
  if (g == 0) {
    lds_m[wave][c] = st.m;
    lds_l[wave][c] = st.l;
  }
  __syncthreads();  // (also: the queries in LDS are no longer needed)
  if (bad) {
    lds_bad = 1;
    atomicOr(L.errors, SKVQ_PAGED_BAD_PAGE);
  }
  float top = lds_m[0][c];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) top = fmaxf(top, lds_m[w][c]);
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
  const bool alone = ch.rows + ch.packed == 1;
  const int partials = kPagedMaxSplits + n_row_chunks, part = packed ? n_row_chunks + chunk : chunk;
  for (int y = threadIdx.x; y < x.count * kD; y += 64 * kWaves) {
    const int row = y / kD, p = y % kD;
    float acc = lds.acc[0][row][p], m = lds_m[0][row], l = 0.0f;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
      acc += lds.acc[w][row][p];
      m = fmaxf(m, lds_m[w][row]);
    }
#pragma unroll
    for (int w = 0; w < kWaves; ++w) l += lds_l[w][row] * __builtin_amdgcn_exp2f(lds_m[w][row] - m);
    if (lds_bad) l = NAN;
    const int channel = packed ? L.v_channel[h * kD + 8 * (p & 15) + (p >> 4)] : p;
    const long long qr = query_row(L, x, h, row);
    if (alone) {
      store_out<T>(L, out, qr, channel, acc / l);
    } else {
      float *to = L.workspace + (qr * partials + part) * kPartialStride;
      to[4 + channel] = acc;
      if (p == 0) {
        to[0] = m;
        to[1] = l;
      }
    }
  }
}

// Combines a row's partials: out = sum 2^(m_i - m) acc_i / sum 2^(m_i - m) l_i.  One workgroup of 128 threads per
// (query token, kv head's query head): thread p owns channel p.
template <class T>
__global__ __launch_bounds__(kD) void paged_merge_kernel(const PagedLayout L, const PagedBatch b, const Out out, int n_row_chunks,
                                                         int n_splits) {
  const RowBlock x = row_block(L, b, blockIdx.x >> 4);
  const int row = blockIdx.x & 15;
  if (!x.s.counts_ok || row >= x.count) return;
  const Chunks ch = chunks_of(x.s.total, L.W, L.S, n_splits);
  if (ch.rows + ch.packed <= 1) return;
  const int partials = kPagedMaxSplits + n_row_chunks;
  const long long qr = query_row(L, x, blockIdx.y, row);
  const float *from = L.workspace + qr * partials * kPartialStride;
  const int p = threadIdx.x, n = ch.rows + ch.packed;
  __shared__ float weight[kD];
  __shared__ float part[2][kD / 64];
  auto partial = [&](int i) { return from + (i < ch.rows ? i : n_row_chunks + i - ch.rows) * (long long)kPartialStride; };
  float m = kNothing, l = 0.0f, acc = 0.0f;
  for (int i0 = 0; i0 < n; i0 += kD) {  // (more than 128 only with windows of thousands of tokens)
    const int here = min(kD, n - i0);
    const float mi = p < here ? partial(i0 + p)[0] : kNothing;
    const float li = p < here ? partial(i0 + p)[1] : 0.0f;
    float top = mi;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    if ((p & 63) == 0) part[0][p >> 6] = top;
    __syncthreads();
    top = fmaxf(m, fmaxf(part[0][0], part[0][1]));
    const float w = __builtin_amdgcn_exp2f(mi - top), before = __builtin_amdgcn_exp2f(m - top);
    weight[p] = p < here ? w : 0.0f;
    float sum = li * w;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    if ((p & 63) == 0) part[1][p >> 6] = sum;
    __syncthreads();
    l = l * before + part[1][0] + part[1][1];
    acc *= before;
    m = top;
    int i = 0;
    for (; i + 8 <= here; i += 8) {
      float a[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) a[u] = partial(i0 + i + u)[4 + p];
#pragma unroll
      for (int u = 0; u < 8; ++u) acc = fmaf(a[u], weight[i + u], acc);
    }
    for (; i < here; ++i) acc = fmaf(partial(i0 + i)[4 + p], weight[i], acc);
    __syncthreads();
  }
  store_out<T>(L, out, qr, p, acc / l);
}

template <class T, int NG>
void launch_chunks(const PagedLayout &L, const PagedBatch &b, TokenRows q, Out out, int row_chunks, int n_splits, dim3 grid, hipStream_t s) {
  const dim3 threads(64 * kWaves);
  switch (L.meta_fmt) {
    case SKVQ_META_F32: paged_attention_kernel<T, NG, SKVQ_META_F32><<<grid, threads, 0, s>>>(L, b, q, out, row_chunks, n_splits); break;
    case SKVQ_META_F16: paged_attention_kernel<T, NG, SKVQ_META_F16><<<grid, threads, 0, s>>>(L, b, q, out, row_chunks, n_splits); break;
    default: paged_attention_kernel<T, NG, SKVQ_META_FP8_E4M3><<<grid, threads, 0, s>>>(L, b, q, out, row_chunks, n_splits); break;
  }
}

template <class T>
hipError_t launch_typed(const PagedLayout &L, const PagedBatch &b, TokenRows q, Out out, int row_chunks, int n_splits, unsigned blocks,
                        hipStream_t s) {
  const dim3 grid((row_chunks + n_splits) * blocks, L.Hk);
  switch (L.NG) {
    case 1: launch_chunks<T, 1>(L, b, q, out, row_chunks, n_splits, grid, s); break;
    case 2: launch_chunks<T, 2>(L, b, q, out, row_chunks, n_splits, grid, s); break;
    default: launch_chunks<T, 4>(L, b, q, out, row_chunks, n_splits, grid, s); break;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  paged_merge_kernel<T><<<dim3(16 * blocks, L.Hk), kD, 0, s>>>(L, b, out, row_chunks, n_splits);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attention(const PagedLayout &L, const skvq_batch &batch, TokenRows q, void *out, long long out_stride,
                                  float *out_f32, int n_cus, hipStream_t s) {
  const PagedBatch b = batch_of(batch);
  const unsigned blocks = (unsigned)units_of(batch, row_deal(L.R));
  const int row_chunks = paged_row_chunks(L.W, L.S);
  // Lengths are not known here: enough chunks that sequences as long as the page table allows fill the chip
  // four workgroups to a compute unit; shorter ones use fewer (chunk_of).
  const long long groups = (long long)blocks * L.Hk, cap = ((long long)b.table_stride << L.page_log2) / kPagedMinChunk + 1;
  long long n = (4ll * n_cus + groups - 1) / groups;
  if (n > cap) n = cap;
  if (n > kPagedMaxSplits) n = kPagedMaxSplits;
  if (n < 1) n = 1;
  const Out o{out, out_stride, out_f32};
  return L.dtype == SKVQ_DTYPE_BF16 ? launch_typed<__bf16>(L, b, q, o, row_chunks, (int)n, blocks, s)
                                    : launch_typed<_Float16>(L, b, q, o, row_chunks, (int)n, blocks, s);
}

}  // namespace skvq
