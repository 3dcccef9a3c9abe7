// skvq_paged_append and skvq_paged_read: tokens into the paged cache and back out (Section 3.2, Eq. 2).
//
// Both work on fours of packed rows (four rows share their value codes' 256 bytes): one workgroup takes a
// four of one sequence and some kv heads, one wavefront one head's keys or values at a time.  Lane (r, m) =
// (lane / 16, lane % 16) holds row r's channels 8m .. 8m+7 as they come and go, 16 bytes; as codes it holds
// dword m of a key row, or row r's part of value piece m, eight reordered positions either way.  The reorder
// goes through LDS, a row of halves per (wavefront, r).
//
// Bound by memory for prompts (a row's 512 bytes in, 140 out), by the chain of dependent loads for decode
// steps: sequence, its counts, its page, its ring row.
#include <hip/hip_runtime.h>

#include "skvq_append_device.h"
#include "skvq_paged.h"

namespace skvq {
namespace {

constexpr int kRowStride = 136;  // values per parked row: 272 B, so the rows' channels fall in different banks
constexpr int kRor4 = 0x124, kRor8 = 0x128;

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
      const int i = sequence_of_unit(b, token, kTokenDeal);
      const Sequence s = sequence_of(b, L, i);
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
  if (tab.half % 8 == 0)
    rope_walk<T, 8>(tab, cs, q.tokens_per_group, kD, copy, L.Hq, rows);
  else
    rope_walk<T, 1>(tab, cs, q.tokens_per_group, kD, copy, L.Hq, rows);
}

// What a lane's eight rotated channels need: its own cosines and sines (1 and 0 behind the rotated part).
struct LaneRotation {
  float c[8], s[8];
};
__device__ __forceinline__ LaneRotation lane_rotation(const RopeTable &tab, const float2 *cs, int m) {
  LaneRotation t;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int ch = 8 * m + e;
    t.c[e] = 1.0f;
    t.s[e] = 0.0f;
    if (ch < 2 * tab.half) {
      const bool first = tab.interleaved ? !(ch & 1) : ch < tab.half;
      const float2 f = cs[tab.interleaved ? ch >> 1 : first ? ch : ch - tab.half];
      t.c[e] = f.x;
      t.s[e] = first ? -f.y : f.y;
    }
  }
  return t;
}
// row: this row's place in LDS (kRowStride values), used on the way
template <class T>
__device__ __forceinline__ Piece<T, 8> rotated(const RopeTable &tab, const LaneRotation &t, const Piece<T, 8> &x, T *row, int m) {
  Piece<T, 8> other, y;
  if (tab.interleaved) {
#pragma unroll
    for (int e = 0; e < 8; ++e) other[e] = x[e ^ 1];
  } else {
    *reinterpret_cast<Piece<T, 8> *>(row + 8 * m) = x;
    wave_lds_sync();
    const int ch = 8 * m, half = tab.half;
    if (half % 8 == 0) {
      const int at = ch < half ? ch + half : ch < 2 * half ? ch - half : ch;
      other = *reinterpret_cast<const Piece<T, 8> *>(row + at);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = ch + e;
        other[e] = row[c < half ? c + half : c < 2 * half ? c - half : c];
      }
    }
    wave_lds_sync();
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int ch = 8 * m + e;
    const T z = (T)rope_turned((float)x[e], (float)other[e], t.c[e], t.s[e]);
    y[e] = ch < 2 * tab.half ? z : x[e];
  }
  return y;
}

__device__ __forceinline__ unsigned long long lane_bytes(const uint8_t *p) { return *reinterpret_cast<const unsigned long long *>(p); }
__device__ __forceinline__ int byte_of(unsigned long long w, int e) { return (int)((w >> (8 * e)) & 0xffu); }
constexpr int key_nibble(int e) { return e % 2 ? 4 + e / 2 : e / 2; }

// Quantizes a four's key rows of one head (parked in LDS) and stores codes and pairs.  part: the head's part
// of the page, or null; rp: the row's place in it.
template <class T, int NG>
__device__ __forceinline__ void pack_keys(const PagedLayout &L, const T *row, unsigned long long channels, const float *clip,
                                          uint8_t *part, int rp, int m) {
  float x[8], mn, mx;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[e] = (float)row[byte_of(channels, e)];
    mn = e ? fminf(mn, x[e]) : x[e];
    mx = e ? fmaxf(mx, x[e]) : x[e];
  }
  // dword m = 4g + j holds positions 32j + 8g ..: a group is the lanes of one j (NG = 4), of a pair, or all
  minmax_with<kRor8>(mn, mx);
  minmax_with<kRor4>(mn, mx);
  if (NG <= 2) minmax_with<kLaneXor1>(mn, mx);
  if (NG == 1) minmax_with<kLaneXor2>(mn, mx);
  const int g = (m & 3) * NG / 4;
  const GroupParams gp = group_params(mn, mx, clip[g], 15.0f, L.meta_fmt);
  unsigned w = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) w |= encode(x[e], gp, 15.0f) << (4 * key_nibble(e));
  if (part) {
    reinterpret_cast<unsigned *>(part + rp * (kD / 2))[m] = w;
    if (m < 4 && m % (4 / NG) == 0)
      meta_store_pair(part + L.km_at, rp * NG + g, MetaPair{gp.scale, gp.lo, gp.stored}, L.meta_fmt);
  }
}

// ... its value rows: lane (r, m) holds positions 16n + m, n = 0 .. 7, some of every group.
template <class T, int NG>
__device__ __forceinline__ void pack_values(const PagedLayout &L, const T *row, unsigned long long channels, const float *clip,
                                            uint8_t *part, int rp, int m) {
  unsigned w[2] = {0u, 0u};
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    float x[8 / NG], mn, mx;
#pragma unroll
    for (int e = 0; e < 8 / NG; ++e) {
      x[e] = (float)row[byte_of(channels, g * (8 / NG) + e)];
      mn = e ? fminf(mn, x[e]) : x[e];
      mx = e ? fmaxf(mx, x[e]) : x[e];
    }
    minmax_with<kLaneXor1>(mn, mx);
    minmax_with<kLaneXor2>(mn, mx);
    minmax_with<kMirror8>(mn, mx);
    minmax_with<kMirror16>(mn, mx);
    const GroupParams gp = group_params(mn, mx, clip[g], 15.0f, L.meta_fmt);
#pragma unroll
    for (int e = 0; e < 8 / NG; ++e) {
      const int n = g * (8 / NG) + e;
      w[n / 4] |= encode(x[e], gp, 15.0f) << (4 * (n % 4));
    }
    if (part && m == g) meta_store_pair(part + L.vm_at, rp * NG + g, MetaPair{gp.scale, gp.lo, gp.stored}, L.meta_fmt);
  }
  if (part) {
    const int r = rp & 3;
    unsigned short *to = reinterpret_cast<unsigned short *>(part + L.v_at + (rp >> 2) * (2 * kD) + 16 * m + 8 * (r >> 1) + 2 * (r & 1));
    to[0] = (unsigned short)w[0];
    to[2] = (unsigned short)w[1];
  }
}

// Append: see AppendPlan for which lanes do what.
template <class T, int NG>
__global__ __launch_bounds__(kRopeThreads) void paged_append_kernel(const PagedLayout L, const RopeTable tab, const PagedBatch b,
                                                                    const TokenRows k, const TokenRows v, const QueryRows q,
                                                                    unsigned n_units, int heads_per_group) {
  __shared__ float2 cs[kRopeMaxTokens][kRopeMaxPairs];
  __shared__ __align__(16) T parked[4][4][kRowStride];
  if (blockIdx.x >= n_units) {
    if (blockIdx.y == 0) rotate_queries<T>(L, tab, b, q, blockIdx.x - n_units, cs);
    return;
  }
  typedef Piece<T, 8> P;
  const int i = sequence_of_unit(b, blockIdx.x, kAppendDeal);
  const Sequence s = sequence_of(b, L, i);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane >> 4, m = lane & 15;
  const long long unit = blockIdx.x - unit_start(kAppendDeal, s.row0, i);
  if (!s.counts_ok || !s.slot_ok) {
    if (threadIdx.x == 0) atomicOr(L.errors, s.counts_ok ? SKVQ_PAGED_BAD_SLOT : SKVQ_PAGED_BAD_COUNTS);
    return;
  }
  const AppendPlan plan = append_plan(s.total, s.n_new, L.W, L.S);
  if (unit < 0 || unit >= plan.leaving_fours + plan.vacant_fours) return;
  const AppendRow x = append_row(plan, (int)unit, r);  // this lane's row
  const long long token = s.row0 + (x.fresh - plan.len);  // (of valid rows: a row of k and v)
  if (x.valid && tab.half) {
    // (sixteen lanes of each wavefront per row, all wavefronts together: 64 threads)
    const int position = b.positions ? b.positions[token] : x.fresh;
    for (int p = 16 * wave + m; p < tab.half; p += 64) cs[r][p] = rope_cos_sin(tab.turn[p], position, tab.amplitude);
  }
  uint8_t *page = nullptr;
  if (x.valid && x.leaving && !x.sink) page = page_of(L, b, i, x.te);
  __syncthreads();
  const bool keys = wave < 2;  // wavefronts 0, 1: keys; 2, 3: values
  LaneRotation turn;
  if (keys) turn = lane_rotation(tab, cs[r], m);
  const TokenRows src = keys ? k : v;
  T *rows = reinterpret_cast<T *>(keys ? L.k_rows : L.v_rows) + (long long)s.slot * L.Hk * (L.W + L.S) * kD;
  T *row = parked[wave][r];
  const int h1 = min(L.Hk, (int)(blockIdx.y + 1) * heads_per_group);
  for (int h = blockIdx.y * heads_per_group + (wave & 1); h < h1; h += 2) {
    T *head_rows = rows + (long long)h * (L.W + L.S) * kD + 8 * m;
    P fresh = {}, gone = {};
    if (x.valid) {
      fresh = *reinterpret_cast<const P *>((const T *)src.p + token * src.stride + h * kD + 8 * m);
      if (x.old) gone = *reinterpret_cast<const P *>(head_rows + (long long)x.ring * kD);
    }
    if (keys && tab.half) fresh = rotated(tab, turn, fresh, row, m);
    if (x.valid && x.ring >= 0) *reinterpret_cast<P *>(head_rows + (long long)x.ring * kD) = fresh;
    if (!x.leaving) continue;
    if (!x.old) gone = fresh;
    if (x.valid && x.sink) *reinterpret_cast<P *>(head_rows + (long long)(L.W + x.token) * kD) = gone;
    *reinterpret_cast<P *>(row + 8 * m) = gone;
    wave_lds_sync();
    uint8_t *part = page ? page + (long long)h * L.part_bytes : nullptr;
    const int rp = x.te & ((1 << L.page_log2) - 1);
    if (keys)
      pack_keys<T, NG>(L, row, lane_bytes(L.k_channel + h * kD + 8 * m), L.clip_k + h * NG, part, rp, m);
    else
      pack_values<T, NG>(L, row, lane_bytes(L.v_channel + h * kD + 8 * m), L.clip_v + h * NG, part, rp, m);
    wave_lds_sync();
  }
}

// scale * code + zero, each operation rounded once
__device__ __forceinline__ float dequantized(unsigned code, float2 pair) {
#pragma clang fp contract(off)
  const float p = pair.x * (float)code;
  return p + pair.y;
}

template <class T, int NG>
__global__ __launch_bounds__(kRopeThreads) void paged_read_kernel(const PagedLayout L, const PagedBatch b, T *k, long long k_stride,
                                                                  T *v, long long v_stride, int heads_per_group) {
  __shared__ __align__(16) T parked[4][4][kRowStride];
  typedef Piece<T, 8> P;
  const int i = sequence_of_unit(b, blockIdx.x, kReadDeal);
  const Sequence s = sequence_of(b, L, i);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane >> 4, m = lane & 15;
  const long long unit = blockIdx.x - unit_start(kReadDeal, s.row0, i);
  const int f = b.first ? b.first[i] : s.total - s.n_new;
  const bool range_ok = f >= 0 && f <= s.total - s.n_new;
  if (!s.counts_ok || !s.slot_ok || !range_ok) {
    if (threadIdx.x == 0)
      atomicOr(L.errors, !s.counts_ok ? SKVQ_PAGED_BAD_COUNTS : !s.slot_ok ? SKVQ_PAGED_BAD_SLOT : SKVQ_PAGED_BAD_RANGE);
    return;
  }
  if (unit < 0 || unit >= read_fours(f, s.n_new, L.S)) return;
  const int a = read_token(f, L.S, (int)unit, r);
  bool valid = a >= f && a < f + s.n_new;
  const TokenPlace at = token_place(a, s.total, L.W, L.S);
  const bool full = at.full;
  const uint8_t *page = nullptr;
  if (valid && !full) {
    page = page_of(L, b, i, at.row);
    valid = page != nullptr;
  }
  const int rp = at.row & ((1 << L.page_log2) - 1);
  const bool keys = wave < 2;
  T *to = keys ? k : v;
  if (!to) return;
  to += (s.row0 + (long long)(a - f)) * (keys ? k_stride : v_stride) + 8 * m;
  const T *rows = reinterpret_cast<const T *>(keys ? L.k_rows : L.v_rows) + (long long)s.slot * L.Hk * (L.W + L.S) * kD;
  T *row = parked[wave][r];
  const int h1 = min(L.Hk, (int)(blockIdx.y + 1) * heads_per_group);
  for (int h = blockIdx.y * heads_per_group + (wave & 1); h < h1; h += 2) {
    P x = {};
    if (valid && full) x = *reinterpret_cast<const P *>(rows + ((long long)h * (L.W + L.S) + at.row) * kD + 8 * m);
    if (valid && !full) {
      const uint8_t *part = page + (long long)h * L.part_bytes;
      if (keys) {
        const unsigned w = reinterpret_cast<const unsigned *>(part + rp * (kD / 2))[m];
        const float2 pair = meta_load_pair(part + L.km_at, rp * NG + (m & 3) * NG / 4, L.meta_fmt);
        const unsigned long long ch = lane_bytes(L.k_channel + h * kD + 8 * m);
#pragma unroll
        for (int e = 0; e < 8; ++e) row[byte_of(ch, e)] = (T)dequantized((w >> (4 * key_nibble(e))) & 15u, pair);
      } else {
        const unsigned short *halves = reinterpret_cast<const unsigned short *>(part + L.v_at + (rp >> 2) * (2 * kD) + 16 * m + 8 * ((rp & 3) >> 1) + 2 * (rp & 1));
        const unsigned w = halves[0] | ((unsigned)halves[2] << 16);
        const unsigned long long ch = lane_bytes(L.v_channel + h * kD + 8 * m);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const float2 pair = meta_load_pair(part + L.vm_at, rp * NG + g, L.meta_fmt);
#pragma unroll
          for (int e = 0; e < 8 / NG; ++e) {
            const int n = g * (8 / NG) + e;
            row[byte_of(ch, n)] = (T)dequantized((w >> (4 * n)) & 15u, pair);
          }
        }
      }
    }
    wave_lds_sync();
    if (!full) x = *reinterpret_cast<const P *>(row + 8 * m);
    if (valid) *reinterpret_cast<P *>(to + h * kD) = x;
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

template <class T>
hipError_t launch_append(const PagedLayout &L, const RopeTable &tab, const PagedBatch &b, TokenRows k, TokenRows v, QueryRows q,
                         unsigned units, unsigned query_groups, int heads, hipStream_t s) {
  const dim3 grid(units + query_groups, (L.Hk + heads - 1) / heads);
  switch (L.NG) {
    case 1: paged_append_kernel<T, 1><<<grid, kRopeThreads, 0, s>>>(L, tab, b, k, v, q, units, heads); break;
    case 2: paged_append_kernel<T, 2><<<grid, kRopeThreads, 0, s>>>(L, tab, b, k, v, q, units, heads); break;
    default: paged_append_kernel<T, 4><<<grid, kRopeThreads, 0, s>>>(L, tab, b, k, v, q, units, heads); break;
  }
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
  // (as in skvq_rope_apply: four tokens a workgroup once that leaves enough of them)
  const QueryRows query{q.p, q_out, q.stride, q_out_stride, b.n_tokens >= 4096 ? kRopeMaxTokens : 1};
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
