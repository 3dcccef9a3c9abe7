// skvq_paged_append and skvq_paged_read: tokens into the paged cache and back out (Section 3.2, Eq. 2).
//
// Both work on eights of packed rows: one workgroup takes an eight of one sequence and some kv heads, one wavefront one
// head's keys or values at a time.  Lane (r, m) = (lane / 8, lane % 8) holds sixteen of row r's channels as they come and
// go, two pieces of 16 bytes that hold both members of the pairs it rotates (LanePieces); as codes it holds two dwords of
// a key row, of the same quantization groups, or row r's part of two value pieces: sixteen reordered positions either
// way.  The reorder goes through LDS, a row of values per (wavefront, r).
//
// Bound by memory and vector instructions for prompts (a row's 512 bytes in, 140 out; eight channels a lane and four rows
// a wavefront took twice as long: what a group needs once is computed by all its lanes; 25143 tokens of 8 kv heads, two
// groups, 53 us, read back in 28), by the chain of dependent loads
// for decode steps: sequence, its counts, its page, its ring row.
#include <hip/hip_runtime.h>

#include "skvq_append_device.h"
#include "skvq_paged.h"

namespace skvq {
namespace {

constexpr int kRowStride = 136;  // values per parked row: 272 B, so the rows' channels fall in different banks

__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The page of packed row te of a sequence, or null (with the error noted).
__device__ __forceinline__ uint8_t *page_of(const PagedLayout &L, const PagedBatch &b, int seq, int te) {
  const int x = te >> L.page_log2;
  const int id = page_known(x, b.table_stride) ? b.table[(long long)seq * b.table_stride + x] : -1;
  if (!page_valid(id, L.n_pages)) {
    atomicOr(L.errors, SKVQ_PAGED_BAD_PAGE);
    return nullptr;
  }
  return L.pages + (long long)id * L.Hk * L.part_bytes;
}

struct QueryRows {
  const void *q;
  void *out;
  long long stride, out_stride;
  int tokens_per_group;
};

// The rotation of the batch's queries: workgroups behind those of the keys and values.
template <class T>
__device__ __forceinline__ void rotate_queries(const PagedLayout &L, const RopeTable &tab, const PagedBatch &b, const QueryRows &q,
                                               int group, float2 (*cs)[kRopeMaxPairs]) {
  __shared__ int token_ok[kRopeMaxTokens], token_position[kRopeMaxTokens];
  const int first = group * q.tokens_per_group, wave = threadIdx.x >> 6;
  if (wave < q.tokens_per_group) {  // (four wavefronts, at most four tokens)
    const int token = first + wave;
    bool ok = token < b.n_tokens;
    int position = 0;
    if (ok) {
      int i;
      const Sequence s = locate(b, L, token, kTokenDeal, i);
      ok = s.counts_ok && s.slot_ok && token >= s.row0 && token < s.row0 + s.n_new;
      position = ok ? (b.positions ? b.positions[token] : s.total - s.n_new + token - s.row0) : 0;
    }
    if ((threadIdx.x & 63) == 0) {
      token_ok[wave] = ok;
      token_position[wave] = position;
    }
  }
  __syncthreads();
  for (int x = threadIdx.x; x < q.tokens_per_group * tab.half; x += kRopeThreads) {
    const int k = x / tab.half, p = x - k * tab.half;
    if (token_ok[k]) cs[k][p] = rope_cos_sin(tab.turn[p], token_position[k], tab.amplitude);
  }
  __syncthreads();
  auto rows = [&](int k, int h, const T *&from, T *&to) {
    if (!token_ok[k]) return false;
    from = (const T *)q.q + ((first + k) * q.stride + h * kD);
    to = (T *)q.out + ((first + k) * q.out_stride + h * kD);
    return true;
  };
  const bool copy = q.q != q.out;
  if (rope_streams(tab.half, kD, sizeof(T)))
    rope_walk<T, 8, true>(tab, cs, q.tokens_per_group, kD, copy, L.Hq, rows);
  else if (tab.half % 8 == 0)
    rope_walk<T, 8, false>(tab, cs, q.tokens_per_group, kD, copy, L.Hq, rows);
  else
    rope_walk<T, 1, false>(tab, cs, q.tokens_per_group, kD, copy, L.Hq, rows);
}

// The channels of a lane's two pieces: of half layout in whole pieces both members of pairs 8m .., else neighbours.
struct LanePieces {
  int a, b;    // first channels
  bool turns;  // both members of every pair are the lane's own, and there are some
};
__device__ __forceinline__ LanePieces lane_pieces(const RopeTable &tab, int m) {
  const int half = tab.half;
  if (half % 8 || tab.interleaved) return LanePieces{16 * m, 16 * m + 8, half % 8 == 0 && 16 * m < 2 * half};
  if (8 * m < half) return LanePieces{8 * m, half + 8 * m, true};
  return LanePieces{16 * m, 16 * m + 8, false};  // (lanes half/8 .. 7 have the channels from 2 half on)
}

// Sixteen channels of a row on their way to codes.
template <class T>
struct Pieces {
  Piece<T, 8> a, b;
};
template <class T>
__device__ __forceinline__ Pieces<T> load_pieces(const T *row, const LanePieces &at) {
  return Pieces<T>{*reinterpret_cast<const Piece<T, 8> *>(row + at.a), *reinterpret_cast<const Piece<T, 8> *>(row + at.b)};
}
template <class T>
__device__ __forceinline__ void store_pieces(T *row, const LanePieces &at, const Pieces<T> &x) {
  *reinterpret_cast<Piece<T, 8> *>(row + at.a) = x.a;
  *reinterpret_cast<Piece<T, 8> *>(row + at.b) = x.b;
}
// Rotates them.  WHOLE: the rotated part fills whole pieces, c and s are the cosines and sines of the lane's eight pairs
// (of lanes that turns).  Else channel by channel through LDS (row: this row's place; cs: the row's cosines and sines).
template <bool WHOLE, class T>
__device__ __forceinline__ void rotate_pieces(const RopeTable &tab, const LanePieces &at, const float (&c)[8], const float (&s)[8],
                                              const float2 *cs, T *row, Pieces<T> &x) {
  const int half = tab.half;
  if constexpr (WHOLE) {
    if (!at.turns) return;
    Pieces<T> y;
    if (tab.interleaved) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const int f = e / 2, g = 4 + e / 2;
        y.a[e] = (T)rope_turned((float)x.a[e], (float)x.a[e + 1], c[f], -s[f]);
        y.a[e + 1] = (T)rope_turned((float)x.a[e + 1], (float)x.a[e], c[f], s[f]);
        y.b[e] = (T)rope_turned((float)x.b[e], (float)x.b[e + 1], c[g], -s[g]);
        y.b[e + 1] = (T)rope_turned((float)x.b[e + 1], (float)x.b[e], c[g], s[g]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y.a[e] = (T)rope_turned((float)x.a[e], (float)x.b[e], c[e], -s[e]);
        y.b[e] = (T)rope_turned((float)x.b[e], (float)x.a[e], c[e], s[e]);
      }
    }
    x = y;
  } else {
    store_pieces(row, at, x);
    wave_lds_sync();
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int ch = (e < 8 ? at.a : at.b - 8) + e;
      if (ch < 2 * half) {
        const bool first = tab.interleaved ? !(ch & 1) : ch < half;
        const float2 f = cs[tab.interleaved ? ch >> 1 : first ? ch : ch - half];
        const float other = (float)row[tab.interleaved ? ch ^ 1 : first ? ch + half : ch - half];
        const float own = (float)(e < 8 ? x.a[e & 7] : x.b[e & 7]);
        const T y = (T)rope_turned(own, other, f.x, first ? -f.y : f.y);
        if (e < 8)
          x.a[e & 7] = y;
        else
          x.b[e & 7] = y;
      }
    }
    wave_lds_sync();
  }
}

__device__ __forceinline__ unsigned long long lane_bytes(const uint8_t *p) { return *reinterpret_cast<const unsigned long long *>(p); }
// The value of a parked row at the e-th of eight byte offsets.
template <class T>
__device__ __forceinline__ T &at_offset(T *row, unsigned long long offsets, int e) {
  const unsigned half = e < 4 ? (unsigned)offsets : (unsigned)(offsets >> 32);
  return *reinterpret_cast<T *>(reinterpret_cast<char *>(row) + ((half >> (8 * (e & 3))) & 0xffu));
}
// The element of a dword of key codes in nibble n: (0, 2, 4, 6, 1, 3, 5, 7).
constexpr int key_element(int n) { return n < 4 ? 2 * n : 2 * n - 7; }
// A lane's two dwords of a key row, and its two value pieces.
__device__ __forceinline__ int key_dword(int m, int i) { return 4 * (2 * (m & 1) + i) + (m >> 1); }  // 4g + j: g = 2 (m % 2) + i, j = m / 2
__device__ __forceinline__ int value_piece(int m, int i) { return 2 * m + i; }

// code = rint(clamp(y, 0, 15)), y = (x - lo) * inv with each operation rounded once: clamping first gives the same integer,
// and adding 1.5 * 2^23 rounds to the nearest integer, ties to even, and leaves the code in the low bits.
__device__ __forceinline__ unsigned code_in_low_bits(float x, const GroupParams &gp) {
#pragma clang fp contract(off)
  const float d = x - gp.lo;
  const float y = d * gp.inv;
  return __float_as_uint(__builtin_amdgcn_fmed3f(y, 0.0f, 15.0f) + 12582912.0f);
}

// Quantizes an eight's key rows of one head (parked in LDS) and stores codes and pairs.  part: the head's part
// of the page, or null; rp: the row's place in it.  offsets: of the channels of the lane's two dwords.
template <class T, int NG>
__device__ __forceinline__ void pack_keys(const PagedLayout &L, T *row, const unsigned long long (&offsets)[2], const float *clip,
                                          uint8_t *part, int rp, int m) {
  float x[2][8], mn, mx;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[i][e] = (float)at_offset(row, offsets[i], e);
      mn = i + e ? fminf(mn, x[i][e]) : x[i][e];
      mx = i + e ? fmaxf(mx, x[i][e]) : x[i][e];
    }
  // dword 4g + j holds positions 32j + 8g ..: a group is the two lanes of one j (NG = 4), four lanes, or all eight
  minmax_with<kLaneXor1>(mn, mx);
  if (NG <= 2) minmax_with<kLaneXor2>(mn, mx);
  if (NG == 1) minmax_with<kMirror8>(mn, mx);
  const int g = (m >> 1) * NG / 4;
  const GroupParams gp = group_params(mn, mx, clip[g], 15.0f, L.meta_fmt);
  unsigned w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int n = 0; n < 8; ++n) w[i] = __builtin_amdgcn_alignbit(code_in_low_bits(x[i][key_element(n)], gp), w[i], 4);
  if (part) {
#pragma unroll
    for (int i = 0; i < 2; ++i) reinterpret_cast<unsigned *>(part + rp * (kD / 2))[key_dword(m, i)] = w[i];
    if (m % (8 / NG) == 0) meta_store_pair(part + L.km_at, rp * NG + g, MetaPair{gp.scale, gp.lo, gp.stored}, L.meta_fmt);
  }
}

// ... its value rows: the lane's pieces hold positions 16n + piece, n = 0 .. 7, some of every group.
template <class T, int NG>
__device__ __forceinline__ void pack_values(const PagedLayout &L, T *row, const unsigned long long (&offsets)[2], const float *clip,
                                            uint8_t *part, int rp, int m) {
  unsigned w[2] = {0u, 0u};
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    float x[2][8 / NG], mn, mx;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 8 / NG; ++e) {
        x[i][e] = (float)at_offset(row, offsets[i], g * (8 / NG) + e);
        mn = i + e ? fminf(mn, x[i][e]) : x[i][e];
        mx = i + e ? fmaxf(mx, x[i][e]) : x[i][e];
      }
    minmax_with<kLaneXor1>(mn, mx);
    minmax_with<kLaneXor2>(mn, mx);
    minmax_with<kMirror8>(mn, mx);
    const GroupParams gp = group_params(mn, mx, clip[g], 15.0f, L.meta_fmt);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 8 / NG; ++e) w[i] = __builtin_amdgcn_alignbit(code_in_low_bits(x[i][e], gp), w[i], 4);
    if (part && m == g) meta_store_pair(part + L.vm_at, rp * NG + g, MetaPair{gp.scale, gp.lo, gp.stored}, L.meta_fmt);
  }
  // Two rows of a four share dwords: row 2p the low halves of both.  Where both are stored each lane takes one dword per
  // piece (the even row's the first four positions), else each its own halves.  (Lane ^ 8 is the row beside it.)
  const bool odd = rp & 1;
  const int here = part ? 1 : 0;
  const bool both = here & __builtin_amdgcn_update_dpp(0, here, 0x128, 0xF, 0xF, true);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const unsigned got = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(odd ? w[i] & 0xffffu : w[i] >> 16), 0x128, 0xF, 0xF, true);
    uint8_t *at = part + L.v_at + (rp >> 2) * (2 * kD) + 16 * value_piece(m, i) + 8 * ((rp & 3) >> 1);
    if (both) {
      reinterpret_cast<unsigned *>(at)[odd] = odd ? got | (w[i] & 0xffff0000u) : (w[i] & 0xffffu) | (got << 16);
    } else if (part) {
      unsigned short *to = reinterpret_cast<unsigned short *>(at) + odd;
      to[0] = (unsigned short)w[i];
      to[2] = (unsigned short)(w[i] >> 16);
    }
  }
}

// Append: see AppendPlan for which lanes do what.  WHOLE: see rotate_pieces.  QUERIES: workgroups from n_units on rotate
// the queries.
template <class T, int NG, bool WHOLE, bool QUERIES>
__global__ __launch_bounds__(kRopeThreads) void paged_append_kernel(const PagedLayout L, const RopeTable tab, const PagedBatch b,
                                                                    const TokenRows k, const TokenRows v, const QueryRows q,
                                                                    unsigned n_units, int heads_per_group) {
  __shared__ float2 cs[kEight][kRopeMaxPairs / 2];  // (a head of 128 channels has 64 pairs)
  __shared__ __align__(16) T parked[4][kEight][kRowStride];
  if (QUERIES && blockIdx.x >= n_units) {
    static_assert(sizeof cs >= sizeof(float2[kRopeMaxTokens][kRopeMaxPairs]), "queries use it with a stride of their own");
    if (blockIdx.y == 0) rotate_queries<T>(L, tab, b, q, blockIdx.x - n_units, reinterpret_cast<float2(*)[kRopeMaxPairs]>(cs));
    return;
  }
  int i;
  const Sequence s = locate(b, L, blockIdx.x, kAppendDeal, i);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane >> 3, m = lane & 7;
  const long long unit = blockIdx.x - unit_start(kAppendDeal, s.row0, i);
  if (!s.counts_ok || !s.slot_ok) {
    if (threadIdx.x == 0) atomicOr(L.errors, s.counts_ok ? SKVQ_PAGED_BAD_SLOT : SKVQ_PAGED_BAD_COUNTS);
    return;
  }
  const AppendPlan plan = append_plan(s.total, s.n_new, L.W, L.S);
  if (unit < 0 || unit >= plan.leaving + plan.vacant) return;
  const AppendRow x = append_row(plan, (int)unit, r);  // this lane's row
  const long long token = s.row0 + (x.fresh - plan.len);  // (of valid rows: a row of k and v)
  uint8_t *page = nullptr;
  if (x.valid && x.leaving && !x.sink) page = page_of(L, b, i, x.te);
  if (x.valid && tab.half) {
    // (eight lanes of each wavefront per row, all wavefronts together: 32 threads)
    const int position = b.positions ? b.positions[token] : x.fresh;
    for (int p = 8 * wave + m; p < tab.half; p += 32) cs[r][p] = rope_cos_sin(tab.turn[p], position, tab.amplitude);
  }
  __syncthreads();
  const bool keys = wave < 2;  // wavefronts 0, 1: keys; 2, 3: values
  const LanePieces at = lane_pieces(tab, m);
  float c[8] = {}, sn[8] = {};
  if (WHOLE && keys && at.turns) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 f = cs[r][8 * m + e];
      c[e] = f.x;
      sn[e] = f.y;
    }
  }
  const TokenRows src = keys ? k : v;
  T *rows = reinterpret_cast<T *>(keys ? L.k_rows : L.v_rows) + (long long)s.slot * L.Hk * (L.W + L.S) * kD;
  T *row = parked[wave][r];
  const int h1 = min(L.Hk, (int)(blockIdx.y + 1) * heads_per_group);
  for (int h = blockIdx.y * heads_per_group + (wave & 1); h < h1; h += 2) {
    T *head_rows = rows + (long long)h * (L.W + L.S) * kD;
    const uint8_t *order = (keys ? L.k_offset : L.v_offset) + h * kD;
    const unsigned long long offsets[2] = {lane_bytes(order + 8 * (keys ? key_dword(m, 0) : value_piece(m, 0))),
                                           lane_bytes(order + 8 * (keys ? key_dword(m, 1) : value_piece(m, 1)))};
    Pieces<T> fresh = {}, gone = {};
    if (x.valid) {
      fresh = load_pieces((const T *)src.p + token * src.stride + h * kD, at);
      if (x.old) gone = load_pieces(head_rows + (long long)x.ring * kD, at);
    }
    if (keys && tab.half) rotate_pieces<WHOLE>(tab, at, c, sn, cs[r], row, fresh);
    if (x.valid && x.ring >= 0) store_pieces(head_rows + (long long)x.ring * kD, at, fresh);
    if (!x.leaving) continue;
    if (!x.old) gone = fresh;
    if (x.valid && x.sink) store_pieces(head_rows + (long long)(L.W + x.token) * kD, at, gone);
    store_pieces(row, at, gone);
    wave_lds_sync();
    uint8_t *part = page ? page + (long long)h * L.part_bytes : nullptr;
    const int rp = x.te & ((1 << L.page_log2) - 1);
    if (keys)
      pack_keys<T, NG>(L, row, offsets, L.clip_k + h * NG, part, rp, m);
    else
      pack_values<T, NG>(L, row, offsets, L.clip_v + h * NG, part, rp, m);
    wave_lds_sync();
  }
}

// The queries of a large batch by themselves (their walk needs more registers than an eight of keys and values).
template <class T>
__global__ __launch_bounds__(kRopeThreads) void paged_queries_kernel(const PagedLayout L, const RopeTable tab, const PagedBatch b, const QueryRows q) {
  __shared__ float2 cs[kRopeMaxTokens][kRopeMaxPairs];
  rotate_queries<T>(L, tab, b, q, blockIdx.x, cs);
}

// scale * code + zero, each operation rounded once.  EXACT: the product is (a compact scale has at most 11 bits, a code
// four), and one multiply-add gives the same number.
template <bool EXACT>
__device__ __forceinline__ float dequantized(float code, float2 pair) {
#pragma clang fp contract(off)
  if constexpr (EXACT) {
    return __builtin_fmaf(pair.x, code, pair.y);
  } else {
    const float p = pair.x * code;
    return p + pair.y;
  }
}
// Eight codes of a dword into a parked row at their offsets; element(n): which of them nibble n is, and its pair.
template <bool EXACT, class T, class Element, class Pair>
__device__ __forceinline__ void scatter_codes(unsigned w, T *row, unsigned long long offsets, Element element, Pair pair) {
  const unsigned even = w & 0x0f0f0f0fu, odd = (w >> 4) & 0x0f0f0f0fu;
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    const float code = (float)(((n % 2 ? odd : even) >> (8 * (n / 2))) & 0xffu);
    at_offset(row, offsets, element(n)) = (T)dequantized<EXACT>(code, pair(n));
  }
}

// The i-th (scale, zero) pair, converted by the chip's instruction.
__device__ __forceinline__ float2 load_pair(const uint8_t *pairs, int i, int fmt) {
  if (fmt == SKVQ_META_F32) return reinterpret_cast<const float2 *>(pairs)[i];
  if (fmt == SKVQ_META_F16) {
    typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
    const half2_t h = reinterpret_cast<const half2_t *>(pairs)[i];
    return make_float2((float)h[0], (float)h[1]);
  }
  const int w = reinterpret_cast<const unsigned short *>(pairs)[i];
  return make_float2(__builtin_amdgcn_cvt_f32_fp8(w, 0), __builtin_amdgcn_cvt_f32_fp8(w, 1));
}

// Bound by its writes and vector instructions: 8 sequences of up to 16k tokens, 20 MB of codes to 121 MB of rows, 42 us with
// pairs converted by integer arithmetic, 39 with the chip's instruction, 28 with streaming stores too (a
// fill of 121 MB takes 20).  Two rows of a lane side by side, half as many writes to LDS of twice the width: 33.
template <class T, int NG>
__global__ __launch_bounds__(kRopeThreads) void paged_read_kernel(const PagedLayout L, const PagedBatch b, T *k, long long k_stride,
                                                                  T *v, long long v_stride, int heads_per_group) {
  __shared__ __align__(16) T parked[4][kEight][kRowStride];
  int i;
  const Sequence s = locate(b, L, blockIdx.x, kReadDeal, i);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane >> 3, m = lane & 7;
  const long long unit = blockIdx.x - unit_start(kReadDeal, s.row0, i);
  const int f = b.first ? b.first[i] : s.total - s.n_new;
  const bool range_ok = f >= 0 && f <= s.total - s.n_new;
  if (!s.counts_ok || !s.slot_ok || !range_ok) {
    if (threadIdx.x == 0)
      atomicOr(L.errors, !s.counts_ok ? SKVQ_PAGED_BAD_COUNTS : !s.slot_ok ? SKVQ_PAGED_BAD_SLOT : SKVQ_PAGED_BAD_RANGE);
    return;
  }
  if (unit < 0 || unit >= read_eights(f, s.n_new, L.S)) return;
  const int a = read_token(f, L.S, (int)unit, r);
  bool valid = a >= f && a < f + s.n_new;
  const TokenPlace place = token_place(a, s.total, L.W, L.S);
  const bool full = place.full;
  const uint8_t *page = nullptr;
  if (valid && !full) {
    page = page_of(L, b, i, place.row);
    valid = page != nullptr;
  }
  const int rp = place.row & ((1 << L.page_log2) - 1);
  const bool keys = wave < 2;
  T *to = keys ? k : v;
  if (!to) return;
  to += (s.row0 + (long long)(a - f)) * (keys ? k_stride : v_stride);
  const T *rows = reinterpret_cast<const T *>(keys ? L.k_rows : L.v_rows) + (long long)s.slot * L.Hk * (L.W + L.S) * kD;
  T *row = parked[wave][r];
  const LanePieces at = {8 * m, kD / 2 + 8 * m, false};  // (whole lines per instruction)
  const int h1 = min(L.Hk, (int)(blockIdx.y + 1) * heads_per_group);
  const bool exact = L.meta_fmt != SKVQ_META_F32;
  for (int h = blockIdx.y * heads_per_group + (wave & 1); h < h1; h += 2) {
    Pieces<T> x = {};
    if (valid && full) x = load_pieces(rows + ((long long)h * (L.W + L.S) + place.row) * kD, at);
    if (valid && !full) {
      const uint8_t *part = page + (long long)h * L.part_bytes, *order = (keys ? L.k_offset : L.v_offset) + h * kD;
      unsigned w[2];
      unsigned long long offsets[2];
      float2 pair[NG];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int dword = keys ? key_dword(m, e) : value_piece(m, e);
        offsets[e] = lane_bytes(order + 8 * dword);
        if (keys) {
          w[e] = reinterpret_cast<const unsigned *>(part + rp * (kD / 2))[dword];
        } else {  // the row's halves of two dwords
          const uint2 two = *reinterpret_cast<const uint2 *>(part + L.v_at + (rp >> 2) * (2 * kD) + 16 * dword + 8 * ((rp & 3) >> 1));
          w[e] = __builtin_amdgcn_perm(two.y, two.x, rp & 1 ? 0x07060302u : 0x05040100u);
        }
      }
      if (keys) {
        pair[0] = load_pair(part + L.km_at, rp * NG + (m >> 1) * NG / 4, L.meta_fmt);
      } else {
#pragma unroll
        for (int g = 0; g < NG; ++g) pair[g] = load_pair(part + L.vm_at, rp * NG + g, L.meta_fmt);
      }
      auto key_pair = [&](int) { return pair[0]; };
      auto value_pair = [&](int n) { return pair[n * NG / 8]; };
      auto same = [](int n) { return n; };
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (keys && exact) scatter_codes<true>(w[e], row, offsets[e], key_element, key_pair);
        if (keys && !exact) scatter_codes<false>(w[e], row, offsets[e], key_element, key_pair);
        if (!keys && exact) scatter_codes<true>(w[e], row, offsets[e], same, value_pair);
        if (!keys && !exact) scatter_codes<false>(w[e], row, offsets[e], same, value_pair);
      }
    }
    wave_lds_sync();
    if (!full) x = load_pieces((const T *)row, at);
    if (valid) {
      __builtin_nontemporal_store(x.a, reinterpret_cast<Piece<T, 8> *>(to + h * kD + at.a));
      __builtin_nontemporal_store(x.b, reinterpret_cast<Piece<T, 8> *>(to + h * kD + at.b));
    }
    wave_lds_sync();
  }
}

// kv heads per workgroup: two (a wavefront each for keys and values) while workgroups are few, more where
// they are many: the sequence, its page and the cosines are then found once for all of them.
int heads_per_group(int Hk, long long units, int n_cus) {
  int n = 2;
  while (n < Hk && units * ((Hk + 2 * n - 1) / (2 * n)) >= 8ll * n_cus) n *= 2;
  return n;
}

template <class T, bool WHOLE, bool QUERIES>
void launch_append_as(const PagedLayout &L, const RopeTable &tab, const PagedBatch &b, TokenRows k, TokenRows v, QueryRows q, unsigned units,
                      dim3 grid, int heads, hipStream_t s) {
  switch (L.NG) {
    case 1: paged_append_kernel<T, 1, WHOLE, QUERIES><<<grid, kRopeThreads, 0, s>>>(L, tab, b, k, v, q, units, heads); break;
    case 2: paged_append_kernel<T, 2, WHOLE, QUERIES><<<grid, kRopeThreads, 0, s>>>(L, tab, b, k, v, q, units, heads); break;
    default: paged_append_kernel<T, 4, WHOLE, QUERIES><<<grid, kRopeThreads, 0, s>>>(L, tab, b, k, v, q, units, heads); break;
  }
}
template <class T>
hipError_t launch_append(const PagedLayout &L, const RopeTable &tab, const PagedBatch &b, TokenRows k, TokenRows v, QueryRows q,
                         unsigned units, unsigned query_groups, int heads, hipStream_t s) {
  // One launch for both while a launch is much of the call; large batches take two (25143 tokens of 32 query and 8 kv heads
  // 147 us in one launch, 128 in two).
  const bool apart = query_groups && b.n_tokens >= 2048;
  if (apart) {
    paged_queries_kernel<T><<<query_groups, kRopeThreads, 0, s>>>(L, tab, b, q);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const bool queries = query_groups && !apart;
  const dim3 grid(units + (queries ? query_groups : 0), (L.Hk + heads - 1) / heads);
  if (tab.half % 8 == 0)
    queries ? launch_append_as<T, true, true>(L, tab, b, k, v, q, units, grid, heads, s) : launch_append_as<T, true, false>(L, tab, b, k, v, q, units, grid, heads, s);
  else
    queries ? launch_append_as<T, false, true>(L, tab, b, k, v, q, units, grid, heads, s) : launch_append_as<T, false, false>(L, tab, b, k, v, q, units, grid, heads, s);
  return hipGetLastError();
}

template <class T>
hipError_t launch_read(const PagedLayout &L, const PagedBatch &b, void *k, long long k_stride, void *v, long long v_stride,
                       unsigned units, int heads, hipStream_t s) {
  const dim3 grid(units, (L.Hk + heads - 1) / heads);
  switch (L.NG) {
    case 1: paged_read_kernel<T, 1><<<grid, kRopeThreads, 0, s>>>(L, b, (T *)k, k_stride, (T *)v, v_stride, heads); break;
    case 2: paged_read_kernel<T, 2><<<grid, kRopeThreads, 0, s>>>(L, b, (T *)k, k_stride, (T *)v, v_stride, heads); break;
    default: paged_read_kernel<T, 4><<<grid, kRopeThreads, 0, s>>>(L, b, (T *)k, k_stride, (T *)v, v_stride, heads); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append(const PagedLayout &L, const RopeTable &tab, const skvq_batch &batch, TokenRows k, TokenRows v,
                               TokenRows q, void *q_out, long long q_out_stride, int n_cus, hipStream_t s) {
  const PagedBatch b = batch_of(batch);
  const long long units = units_of(batch, kAppendDeal);
  const int pieces = (q.p != q_out ? kD : 2 * tab.half) / (tab.half % 8 ? 1 : 8) / 2;
  const QueryRows query{q.p, q_out, q.stride, q_out_stride, rope_tokens_per_group(b.n_tokens, pieces > 0 ? pieces : 1, L.Hq)};
  const unsigned groups = q.p && (tab.half || q.p != q_out) ? (b.n_tokens + query.tokens_per_group - 1) / query.tokens_per_group : 0;
  const int heads = heads_per_group(L.Hk, units, n_cus);
  return L.dtype == SKVQ_DTYPE_BF16 ? launch_append<__bf16>(L, tab, b, k, v, query, (unsigned)units, groups, heads, s)
                                    : launch_append<_Float16>(L, tab, b, k, v, query, (unsigned)units, groups, heads, s);
}

hipError_t launch_paged_read(const PagedLayout &L, const skvq_batch &batch, void *k, long long k_stride, void *v,
                             long long v_stride, int n_cus, hipStream_t s) {
  const PagedBatch b = batch_of(batch);
  const long long units = units_of(batch, kReadDeal);
  const int heads = heads_per_group(L.Hk, units, n_cus);
  return L.dtype == SKVQ_DTYPE_BF16 ? launch_read<__bf16>(L, b, k, k_stride, v, v_stride, (unsigned)units, heads, s)
                                    : launch_read<_Float16>(L, b, k, k_stride, v, v_stride, (unsigned)units, heads, s);
}

}  // namespace skvq
