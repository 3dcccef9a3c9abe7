// How the paged cache's kernels deal a batch out: which workgroup has which rows of which sequence, and where a row
// goes.  Plain constexpr arithmetic without device types, so that the host can check it at every length.
#pragma once

namespace skvq {

// Workgroups are dealt to sequences without a prefix sum: sequence i, whose new tokens begin at row0, has the units from
// unit_start(row0, i) on, and at most n_new * mul / 2^div_log2 + pad (rounded down) of them, for which the next
// sequence's start leaves room: floor(x + y) >= floor(x) + floor(y).
struct UnitDeal {
  int mul, div_log2, pad;
};
constexpr UnitDeal kAppendDeal{1, 3, 3};
constexpr UnitDeal kReadDeal{1, 3, 2};
constexpr UnitDeal kTokenDeal{1, 0, 0};
constexpr long long unit_start(const UnitDeal &d, int row0, int i) {
  return (((long long)row0 * d.mul) >> d.div_log2) + (long long)i * d.pad;
}

// Token a is packed row a - S.  Kernels take packed rows by eights (two fours, which share their value codes' bytes; an
// eight lies in one page, whose size is a multiple of 16): tokens with the same (a + lead) / 8.
constexpr int kEight = 8;
constexpr int lead_of(int S) { return (kEight - S % kEight) % kEight; }

// Append, with `len` tokens cached before and `total` after: the tokens that leave the window are [lo, hi) =
// [max(0, len - W), total - W): ring rows and, of a long prompt, new tokens that never were in the ring.  A ring row is
// overwritten by the lanes that have read it: those that pack old token a also write its successor, the newest token
// of the same row.  Rows that held nothing (len < W) are eights of their own.
struct AppendPlan {
  int W, S, total, len, lo, hi, lead, eight0, leaving, vacant_end, vacant;
};
constexpr AppendPlan append_plan(int total, int n_new, int W, int S) {
  AppendPlan p{W, S, total, total - n_new, 0, 0, lead_of(S), 0, 0, 0, 0};
  p.lo = p.len > W ? p.len - W : 0;
  p.hi = total - W > p.lo ? total - W : p.lo;
  p.eight0 = (p.lo + p.lead) / kEight;
  p.leaving = p.hi > p.lo ? (p.hi + p.lead + kEight - 1) / kEight - p.eight0 : 0;
  p.vacant_end = total < W ? total : W;
  p.vacant = p.len < p.vacant_end ? (p.vacant_end - p.len + kEight - 1) / kEight : 0;
  return p;
}
struct AppendRow {
  bool valid;    // there is something to do
  bool leaving;  // token `token` leaves: to its sink row (sink) or packed row te
  bool old;      // ... from ring row `ring`
  bool sink;
  int token, te;
  int fresh;     // the new token to load: the leaving one itself, or what enters ring row `ring` (-1: none)
  int ring;
};
constexpr AppendRow append_row(const AppendPlan &p, int unit, int r) {
  AppendRow x{false, unit < p.leaving, false, false, -1, -1, 0, -1};
  if (x.leaving) {
    const int a = kEight * (p.eight0 + unit) + r - p.lead;
    x.valid = a >= p.lo && a < p.hi;
    x.token = a;
    x.old = a < p.len;
    x.sink = a < p.S;
    x.te = a - p.S;
    x.fresh = x.old ? a + (p.total - 1 - a) / p.W * p.W : a;
    if (x.old) x.ring = a % p.W;
  } else {
    x.ring = p.len + kEight * (unit - p.leaving) + r;
    x.valid = x.ring < p.vacant_end;
    x.fresh = x.ring + (p.total - 1 - x.ring) / p.W * p.W;
  }
  return x;
}

// Read of tokens [first, first + n): eights, and where a token is.
constexpr int read_eights(int first, int n, int S) {
  return n > 0 ? (first + n + lead_of(S) + kEight - 1) / kEight - (first + lead_of(S)) / kEight : 0;
}
constexpr int read_token(int first, int S, int unit, int r) { return kEight * ((first + lead_of(S)) / kEight + unit) + r - lead_of(S); }
struct TokenPlace {
  bool full;  // in a row of k_rows / v_rows, else packed row `row`
  int row;
};
constexpr TokenPlace token_place(int token, int total, int W, int S) {
  return token >= total - W ? TokenPlace{true, token % W} : token < S ? TokenPlace{true, W + token} : TokenPlace{false, token - S};
}

// Attention: the rows of a sequence are cut into chunks of full-precision rows and chunks of packed rows, each read by a
// workgroup per (block of 16 query rows, kv head): a unit.  A workgroup's wavefronts take every kPagedWaves-th tile of a
// chunk of packed rows; chunks are whole tiles for each of them, at least two.
constexpr int kPagedWaves = 4, kPagedTile = 32;
constexpr int kPagedStep = kPagedTile * kPagedWaves;
constexpr int kPagedMinChunk = 2 * kPagedStep;
constexpr int kPagedMaxSplits = 128;     // chunks of packed rows of a sequence
constexpr int kPagedRowsPerChunk = 512;  // rows of k_rows / v_rows per chunk
constexpr int paged_row_chunks(int W, int S) { return (W + S + kPagedRowsPerChunk - 1) / kPagedRowsPerChunk; }
constexpr int whole_steps(int rows) { return (rows / kPagedStep + (rows % kPagedStep > 0)) * kPagedStep; }
// Lengths are known on the device only, so every workgroup, of `groups` per kv head, finds the batch's chunk size from two
// sums over the batch: `work`, packed rows times blocks, and `extra`, units beyond work / chunk at most (a last, shorter
// chunk per block).  The units of packed rows fit `rounds` rounds over the groups of a head: as few as keep a chunk within
// 4096 rows, more where the extra units would fill half of them.  (The units of full rows, short ones, come after them.
// Numbers of 24 bits do: units are counted exactly from the chunk size, which is the same in every workgroup.)
constexpr int chunk_for(float work, float extra, int groups) {
  const float least = work / (4096.0f * groups), full = 2.0f * extra / groups;
  const float most = least > full ? least : full;
  const float rounds = (float)(int)(most < 1e6f ? most : 1e6f) + 1.0f;
  const float rows = work / (rounds * groups - extra);  // (positive: rounds > full)
  const int chunk = whole_steps(rows < 1e9f ? (int)rows + 1 : 1000000000);
  return chunk < kPagedMinChunk ? kPagedMinChunk : chunk;
}
// Quotient by a number of 1 .. 16 (recip_of it) of y < 2^27.
constexpr unsigned recip_of(int divisor) { return ((1u << 31) + divisor - 1) / divisor; }
constexpr int quotient(int y, unsigned recip) { return (int)(((unsigned long long)(2u * (unsigned)y) * recip) >> 32); }
struct Chunks {
  int n_kept, n_win, nq;    // sink rows, ring rows, packed rows
  int rows, packed, chunk;  // chunks of full rows, of packed rows; packed rows per chunk
};
constexpr Chunks chunks_of(int total, int W, int S, int chunk) {
  Chunks c{0, total < W ? total : W, 0, 0, 0, chunk};
  const int before = total - c.n_win;
  c.n_kept = before < S ? before : S;
  c.nq = before - c.n_kept;
  c.rows = (c.n_win + c.n_kept + kPagedRowsPerChunk - 1) / kPagedRowsPerChunk;
  const int least = whole_steps(c.nq / kPagedMaxSplits + (c.nq % kPagedMaxSplits > 0));  // (partials have room for so many)
  if (least > c.chunk) c.chunk = least;
  c.packed = c.nq / c.chunk + (c.nq % c.chunk > 0);
  return c;
}

// Whether a sequence's entry x of the page table can be followed.
constexpr bool page_known(int x, int table_stride) { return x >= 0 && x < table_stride; }
constexpr bool page_valid(int id, int n_pages) { return id >= 0 && id < n_pages; }

}  // namespace skvq
