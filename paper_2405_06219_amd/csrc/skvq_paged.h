// Internal declarations of rotary positions and of the paged 4-bit cache.  Not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "skvq.h"
#include "skvq_internal.h"
#include "skvq_paged_plan.h"
#include "skvq_rope_device.h"

namespace skvq {

// Everything a kernel of the paged cache needs to find its data; passed by value.
struct PagedLayout {
  int Hq, Hk, R;      // R = Hq / Hk
  unsigned recip_R;   // recip_of(R)
  int G, NG;
  int W, S;
  int meta_fmt, meta_size;  // skvq_meta_format, bytes of a scale or zero
  int page_log2;            // P = 1 << page_log2
  int n_pages, max_seqs;
  int dtype;                       // skvq_dtype
  unsigned part_bytes;             // a kv head's part of a page
  unsigned v_at, km_at, vm_at;     // its sections (key codes at 0)
  float sm_scale;
  uint8_t *pages;
  void *k_rows, *v_rows;
  float *workspace;
  // device constants: twice the channel (the offset of its 16-bit value) of key code e of a row's dword m, at
  // [head][8 m + e]; of value code n of piece m, at [head][8 m + n]; and the place 8 m + e of a key channel
  const uint8_t *k_offset, *v_offset, *k_place;
  const float *clip_k, *clip_v;  // [Hk][NG]
  int *errors;                   // SKVQ_PAGED_BAD_*
};

struct PagedBatch {
  int n_seqs, n_tokens, table_stride;
  const int *cu, *lens, *table, *slots, *positions, *first;
};

inline PagedBatch batch_of(const skvq_batch &b) {
  return PagedBatch{b.n_seqs, b.n_tokens, b.table_stride, b.cu_tokens, b.seq_lens, b.page_table, b.slots, b.positions, b.first};
}

// A sequence of a batch as a kernel sees it.
struct Sequence {
  int row0, n_new;   // its rows of the token arrays
  int total;         // tokens cached, the new ones among them
  int slot;
  bool counts_ok, slot_ok;
};

__device__ __forceinline__ Sequence sequence_of(const PagedBatch &b, const PagedLayout &L, int i) {
  Sequence s;
  const int c0 = b.cu[i], c1 = b.cu[i + 1];
  s.total = b.lens[i];
  s.slot = b.slots ? b.slots[i] : i;
  s.row0 = c0;
  s.n_new = c1 - c0;
  // (lengths near 2^31 would wrap the row numbers of a four or a tile)
  s.counts_ok = c0 >= 0 && c1 >= c0 && c1 <= b.n_tokens && s.total >= s.n_new && s.total <= SKVQ_MAX_QUANT_TOKENS;
  s.slot_ok = s.slot >= 0 && s.slot < L.max_seqs;
  return s;
}

// Finds the sequence of a unit (see UnitDeal): the last one that starts at or before it.  Every lane of the wavefront
// takes part; 64 starts are compared at a time (a search by halves costs a memory round trip per bit).  Whatever cu
// holds, the answer lies in [0, n_seqs).
__device__ __forceinline__ int sequence_of_unit(const PagedBatch &b, long long unit, const UnitDeal &d) {
  int lo = 0, n = b.n_seqs;
  const int lane = threadIdx.x & 63;
  while (n > 1) {
    const int step = (n + 63) >> 6, at = lane * step;
    const bool starts = at < n && unit_start(d, b.cu[lo + at], lo + at) <= unit;
    const int count = __popcll(__ballot(starts));
    const int k = count > 0 ? count - 1 : 0;
    lo += k * step;
    if (step == 1) break;
    n = n - k * step < step ? n - k * step : step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}
// The unit's sequence.  Up to 64 sequences: every lane reads one, all at once.
__device__ __forceinline__ Sequence locate(const PagedBatch &b, const PagedLayout &L, long long unit, const UnitDeal &d, int &i) {
  if (b.n_seqs > 64) {
    i = sequence_of_unit(b, unit, d);
    return sequence_of(b, L, i);
  }
  const int lane = threadIdx.x & 63;
  Sequence s = sequence_of(b, L, lane < b.n_seqs ? lane : b.n_seqs - 1);
  const unsigned long long started = __ballot(lane < b.n_seqs && unit_start(d, s.row0, lane) <= unit);
  i = __builtin_amdgcn_readfirstlane(started ? 63 - __builtin_clzll(started) : 0);
  auto of_it = [&](int v) { return __builtin_amdgcn_readlane(v, i); };
  return Sequence{of_it(s.row0), of_it(s.n_new), of_it(s.total), of_it(s.slot), (bool)of_it(s.counts_ok), (bool)of_it(s.slot_ok)};
}
inline long long units_of(const skvq_batch &b, const UnitDeal &d) {
  return (((long long)b.n_tokens * d.mul) >> d.div_log2) + (long long)b.n_seqs * d.pad;
}

hipError_t launch_rope(const RopeTable &tab, int head_dim, const skvq_rope_tensor *tensors, int n_tensors, int dtype,
                       int batch, unsigned n_tokens, const int *positions, long long positions_batch, int start,
                       bool transpose, hipStream_t s);

struct TokenRows {  // rows of tokens: element stride between tokens, a token's heads in a row
  const void *p;
  long long stride;
};
hipError_t launch_paged_append(const PagedLayout &L, const RopeTable &tab, const skvq_batch &b, TokenRows k, TokenRows v,
                               TokenRows q, void *q_out, long long q_out_stride, int n_cus, hipStream_t s);
hipError_t launch_paged_read(const PagedLayout &L, const skvq_batch &b, void *k, long long k_stride, void *v,
                             long long v_stride, int n_cus, hipStream_t s);

// The most work (see plan) that a call can have.
long long paged_most_work(const PagedLayout &L, const skvq_batch &b);
hipError_t launch_paged_attention(const PagedLayout &L, const skvq_batch &b, TokenRows q, void *out, long long out_stride,
                                  float *out_f32, int n_cus, hipStream_t s);

}  // namespace skvq
