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

// Attention: work is counted in steps of packed rows (a tile for each of a workgroup's wavefronts) and dealt out in equal
// shares.  A run, one unit's query rows of a sequence against all it sees, is its chunks of full-precision rows (each taken
// whole by the workgroup in whose share it begins; 128 rows count as four steps, by their bytes) and then its steps of
// packed rows.  Runs follow one another; a share may end in one run and begin in another, and what each workgroup finds of
// a run is a partial result.
constexpr int kPagedWaves = 4, kPagedTile = 32;
constexpr int kPagedStep = kPagedTile * kPagedWaves;
constexpr int kPagedMaxSplits = 128;     // partial results of packed rows of a run
constexpr int kPagedRowsPerChunk = 512;  // rows of k_rows / v_rows per chunk
constexpr int kRowStep = 128, kRowStepWeight = 4, kRowChunkWeight = kPagedRowsPerChunk / kRowStep * kRowStepWeight;
constexpr unsigned kPagedMostWork = 1u << 30;  // of a call: work is counted in 32 bits
constexpr int paged_row_chunks(int W, int S) { return (W + S + kPagedRowsPerChunk - 1) / kPagedRowsPerChunk; }
constexpr int steps_of(int rows, int step) { return rows / step + (rows % step > 0); }
constexpr int row_weight_of(int rows) { return kRowStepWeight * steps_of(rows, kRowStep); }
struct Run {
  int n_kept, n_win, nq;  // sink rows, ring rows, packed rows
  int rows, row_weight;   // chunks of full rows, their work
  int steps;              // of packed rows
};
// capacity: packed rows that a row of the page table has room for (a longer sequence is an error, found elsewhere).
constexpr Run run_of(int total, int W, int S, int capacity) {
  Run r{0, total < W ? total : W, 0, 0, 0, 0};
  const int before = total - r.n_win;
  r.n_kept = before < S ? before : S;
  r.nq = before - r.n_kept;
  r.rows = (r.n_win + r.n_kept + kPagedRowsPerChunk - 1) / kPagedRowsPerChunk;
  r.row_weight = row_weight_of(r.n_win + r.n_kept);
  r.steps = steps_of(r.nq < capacity ? r.nq : capacity, kPagedStep);
  return r;
}
// The share of each of `groups` workgroups (of a kv head), with room for a run's partial results.
constexpr int share_of(int work, int most_steps, int groups) {
  int share = steps_of(work, groups);
  const int least = steps_of(most_steps, kPagedMaxSplits - 2);
  if (least > share) share = least;
  return share > 0 ? share : 1;
}
// What a workgroup does next: its share ends at `stop`, it is at `at`, which is `done` into the run.
struct Portion {
  int work;                 // how far it goes, at least 1
  bool there, packed;       // !there: the rest of a chunk that another workgroup has
  int begin, end;           // rows
  int partial, n_partials;  // which of the run's partial results, of how many
};
constexpr Portion portion_of(const Run &r, int done, int at, int stop, int share) {
  const int packed_at = at - done + r.row_weight, first = packed_at / share;
  Portion p{1, true, done >= r.row_weight, 0, 0, 0, r.rows + (r.steps > 0 ? (packed_at + r.steps - 1) / share - first + 1 : 0)};
  if (p.packed) {
    const int step = done - r.row_weight, left = r.steps - step, n = stop - at < left ? stop - at : left;
    if (n > 0) p.work = n;
    p.begin = step * kPagedStep;
    const long long end = (long long)(step + p.work) * kPagedStep;
    p.end = end < r.nq ? (int)end : r.nq;
    p.partial = r.rows + at / share - first;
  } else {
    p.partial = done / kRowChunkWeight;
    p.there = done % kRowChunkWeight == 0;
    const int next = (p.partial + 1) * kRowChunkWeight;
    p.work = (next < r.row_weight ? next : r.row_weight) - done;
    p.begin = p.partial * kPagedRowsPerChunk;
    p.end = p.begin + kPagedRowsPerChunk < r.n_kept + r.n_win ? p.begin + kPagedRowsPerChunk : r.n_kept + r.n_win;
  }
  return p;
}
// Quotient by a number of 1 .. 16 (recip_of it) of y < 2^27.
constexpr unsigned recip_of(int divisor) { return ((1u << 31) + divisor - 1) / divisor; }
constexpr int quotient(int y, unsigned recip) { return (int)(((unsigned long long)(2u * (unsigned)y) * recip) >> 32); }
// Whether a sequence's entry x of the page table can be followed.
constexpr bool page_known(int x, int table_stride) { return x >= 0 && x < table_stride; }
constexpr bool page_valid(int id, int n_pages) { return id >= 0 && id < n_pages; }

}  // namespace skvq
