"""The paged cache and rotary positions without a GPU: the kernels' own dealing arithmetic (csrc/skvq_paged_plan.h)
compiled for the host, rotary frequencies against their formulas, and what the entry points refuse."""
import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
D = 128

SOURCE = """
#include "skvq_paged_plan.h"
using namespace skvq;
extern "C" int append_rows(int total, int n_new, int W, int S, int *out, int most) {
  const AppendPlan p = append_plan(total, n_new, W, S);
  int n = 0;
  for (int u = 0; u < p.leaving + p.vacant; ++u)
    for (int r = 0; r < 8; ++r) {
      const AppendRow x = append_row(p, u, r);
      if (!x.valid) continue;
      if (n == most) return -1;
      int *o = out + 8 * n++;
      o[0] = u; o[1] = r; o[2] = x.leaving; o[3] = x.old; o[4] = x.token; o[5] = x.te; o[6] = x.fresh; o[7] = x.ring;
    }
  return n;
}
extern "C" int append_units(int total, int n_new, int W, int S) {
  const AppendPlan p = append_plan(total, n_new, W, S);
  return p.leaving + p.vacant;
}
extern "C" long long start_of(int kind, int row0, int i) {
  return unit_start(kind == 0 ? kAppendDeal : kind == 1 ? kReadDeal : kTokenDeal, row0, i);
}
extern "C" int eights_to_read(int first, int n, int S) { return read_eights(first, n, S); }
extern "C" int token_to_read(int first, int S, int unit, int r) { return read_token(first, S, unit, r); }
extern "C" int place(int token, int total, int W, int S) {
  const TokenPlace p = token_place(token, total, W, S);
  return p.full ? -1 - p.row : p.row;
}
extern "C" int divided(int y, int by) { return quotient(y, recip_of(by)); }
extern "C" void run(int total, int W, int S, int capacity, int *out) {
  const Run r = run_of(total, W, S, capacity);
  out[0] = r.n_kept; out[1] = r.n_win; out[2] = r.nq; out[3] = r.rows; out[4] = r.row_weight; out[5] = r.steps;
}
extern "C" int share(int work, int most_steps, int groups) { return share_of(work, most_steps, groups); }
// The portions of workgroups 0 .. groups - 1 in runs one after another: {run, work, there, packed, begin, end, partial, n_partials}.
extern "C" int portions(int n, const int *totals, int W, int S, int groups, int share, int *out, int most) {
  long long work = 0;
  for (int i = 0; i < n; ++i) { const Run r = run_of(totals[i], W, S, 0x7fffffff); work += r.row_weight + r.steps; }
  int k = 0;
  for (int g = 0; g < groups; ++g) {
    const long long from = (long long)g * share;
    const int stop = (int)(work < from + share ? work : from + share);
    for (int at = (int)(work < from ? work : from); at < stop;) {
      int i = 0, done = at;
      Run r = run_of(totals[0], W, S, 0x7fffffff);
      while (done >= r.row_weight + r.steps) { done -= r.row_weight + r.steps; r = run_of(totals[++i], W, S, 0x7fffffff); }
      const Portion p = portion_of(r, done, at, stop, share);
      if (k == most) return -1;
      int *o = out + 8 * k++;
      o[0] = i; o[1] = p.work; o[2] = p.there; o[3] = p.packed; o[4] = p.begin; o[5] = p.end; o[6] = p.partial; o[7] = p.n_partials;
      at += p.work;
    }
  }
  return k;
}
extern "C" int page_ok(int x, int stride, int id, int n_pages) { return page_known(x, stride) && page_valid(id, n_pages); }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged_plan")
    (d / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-fsanitize=undefined", "-fno-sanitize-recover",
                    "-static-libubsan", "-I", os.path.join(ROOT, "paper_2405_06219_amd", "csrc"), str(d / "plan.cpp"),
                    "-o", str(d / "plan.so")], check=True)
    lib = C.CDLL(str(d / "plan.so"))
    lib.start_of.restype = C.c_longlong
    return lib


@pytest.fixture(scope="module")
def B():
    from paper_2405_06219_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2405_06219_amd import build
        build.build()
    return binding


def rows_of(plan, total, n_new, W, S):
    out = np.zeros((8 * (n_new + 16), 8), np.int32)
    n = plan.append_rows(total, n_new, W, S, out.ctypes.data_as(C.c_void_p), len(out))
    assert n >= 0
    return out[:n]


@pytest.mark.parametrize("W", [1, 2, 3, 4, 7, 16])
@pytest.mark.parametrize("S", [0, 1, 4, 5])
def test_append_puts_every_token_in_its_place_once(plan, W, S):
    for total in range(1, 3 * W + 12):
        for n_new in range(0, total + 1):
            length = total - n_new
            ring = {a % W: a for a in range(max(length - W, 0), length)}      # what the rows hold before
            left, writers = [], {}
            for u, r, leaving, old, token, te, fresh, row in rows_of(plan, total, n_new, W, S):
                if leaving:
                    left.append(token)
                    assert te == token - S and (te < 0 or te % 8 == r)        # the eights of a page
                    assert old == (token < length)
                    if old:
                        assert row == token % W and ring[row] == token        # read where it is ...
                    else:
                        assert fresh == token and row == -1
                if row >= 0:                                                  # ... by whom overwrites it
                    assert row not in writers and fresh >= length
                    assert fresh % W == row and fresh >= total - W and fresh < total
                    writers[row] = fresh
            assert left == list(range(max(length - W, 0), max(total - W, 0)))
            assert sorted(writers.values()) == list(range(max(length, total - W), total))


@pytest.mark.parametrize("W,S", [(1, 0), (7, 3), (128, 5), (1 << 20, 1 << 20)])
def test_units_of_sequences_do_not_overlap(plan, W, S):
    rng = np.random.default_rng(W)
    for trial in range(60):
        news = [int(n) for n in rng.integers(0, [2, 9, 5000][trial % 3], size=rng.integers(1, 70))]
        row0 = np.concatenate([[0], np.cumsum(news)])
        for i, n in enumerate(news):
            extra = int(rng.choice([0, 1, W - 1, W, 2 * W + 3]))
            most = {0: plan.append_units(n + extra, n, W, S),
                    1: max(plan.eights_to_read(extra, n, S), plan.eights_to_read(0, n, S)), 2: n}
            for kind, units in most.items():
                gap = plan.start_of(kind, int(row0[i + 1]), i + 1) - plan.start_of(kind, int(row0[i]), i)
                assert units <= gap, (kind, n, extra)


def test_read_covers_its_tokens_once(plan):
    for S in (0, 1, 2, 3, 5):
        for first in range(0, 9):
            for n in range(0, 12):
                got = [plan.token_to_read(first, S, u, r) for u in range(plan.eights_to_read(first, n, S)) for r in range(8)]
                assert [a for a in got if first <= a < first + n] == list(range(first, first + n))
                assert len(got) <= 8 * (n // 8 + 2)
    for total, W, S in [(5, 8, 2), (8, 8, 2), (9, 8, 2), (30, 8, 3), (30, 1, 0), (2 ** 31 - 65, 128, 5)]:
        for a in {0, 1, 2, 3, total // 2, max(total - W - 1, 0), max(total - W, 0), total - 1}:
            want = -1 - a % W if a >= total - W else -1 - (W + a) if a < S else a - S
            assert plan.place(a, total, W, S) == want


def test_runs(plan):
    out = np.zeros(6, np.int32)
    for total in [1, 2, 127, 128, 129, 133, 134, 384, 385, 700, 4000, 131072, 2 ** 24 + 7, 2 ** 31 - 65]:
        for W, S in [(1, 0), (128, 0), (128, 5), (600, 1000), (1 << 20, 1 << 20)]:
            for capacity in [0, 256, 4096, 2 ** 31 - 1]:
                plan.run(total, W, S, capacity, out.ctypes.data_as(C.c_void_p))
                kept, win, nq, rows, weight, steps = (int(x) for x in out)
                assert win == min(total, W) and kept == min(total - win, S) and kept + win + nq == total
                assert rows == -(-(kept + win) // 512) and weight == 4 * -(-(kept + win) // 128)
                assert steps == -(-min(nq, capacity) // 128)


@pytest.mark.parametrize("groups", [1, 24, 96, 768])
def test_shares_cover_every_run_once(plan, groups):
    """Every row of every run is in one portion, partial results are numbered without gaps and fit the workspace, and no
    workgroup has more than its share and what a chunk of full rows goes past its end."""
    rng = np.random.default_rng(groups)
    room = np.zeros((100000, 8), np.int32)
    for trial in range(120):
        W, S = int(rng.choice([1, 128, 700, 3000])), int(rng.choice([0, 5, 900]))
        lens = [int(10 ** rng.uniform(0, rng.uniform(1, 5.5))) for _ in range(rng.integers(1, 80))]
        runs = []
        for t in lens:
            out = np.zeros(6, np.int32)
            plan.run(t, W, S, 2 ** 31 - 1, out.ctypes.data_as(C.c_void_p))
            runs.append([int(x) for x in out])
        work = sum(r[4] + r[5] for r in runs)
        share = plan.share(work, max(r[5] for r in runs), groups)
        assert share >= 1 and share * groups >= work
        totals = np.array(lens, np.int32)
        n = plan.portions(len(lens), totals.ctypes.data_as(C.c_void_p), W, S, groups, share, room.ctypes.data_as(C.c_void_p), len(room))
        assert n > 0
        got = room[:n].copy()
        assert got[:, 1].min() >= 1 and got[got[:, 3] == 1][:, 1].max(initial=0) <= share
        for i, (kept, win, nq, rows, weight, steps) in enumerate(runs):
            mine = got[(got[:, 0] == i) & (got[:, 2] == 1)]
            packed, full = mine[mine[:, 3] == 1], mine[mine[:, 3] == 0]
            for part, count in ((packed, nq), (full, kept + win)):
                assert sorted(map(tuple, part[:, 4:6])) == list(map(tuple, part[:, 4:6]))
                ends = np.concatenate([[0], part[:, 5]])
                assert (part[:, 4] == ends[:-1]).all() and ends[-1] == count
            assert sorted(mine[:, 6]) == list(range(len(mine))) and (mine[:, 7] == len(mine)).all()
            assert (full[:, 6] < rows).all() and len(packed) <= 127 and (packed[:, 4] % 128 == 0).all()
    assert plan.share(0, 0, groups) == 1
    assert plan.share(2 ** 30 - 1, 2 ** 24, groups) >= 2 ** 24 // 126


def test_quotients(plan):
    for by in range(1, 17):
        for y in [0, 1, by - 1, by, by + 1, 12345, *range(2 ** 27 - 40, 2 ** 27), *(by * (2 ** 23 + k) - 1 for k in range(3))]:
            assert plan.divided(y, by) == y // by


def test_append_plan_at_the_longest_sequence(plan):
    # (built with -fsanitize=undefined: a sum past 2^31 ends the process)
    for total in (2 ** 31 - 65, 2 ** 31 - 66):
        for W, S, n in [(1, 0, 1), (128, 5, 3), (1 << 20, 1 << 20, 9)]:
            got = rows_of(plan, total, n, W, S)
            assert [int(x) for x in got[:, 4]] == list(range(total - n - W, total - W))


def test_pages_that_cannot_be_followed(plan):
    for x, stride, page, n, want in [(0, 1, 0, 1, 1), (1, 1, 0, 1, 0), (0, 1, 1, 1, 0), (0, 1, -1, 1, 0), (-1, 4, 0, 9, 0),
                                     (3, 4, 8, 9, 1), (3, 4, 9, 9, 0), (2 ** 31 - 1, 4, 0, 9, 0), (0, 4, -2 ** 31, 9, 0)]:
        assert plan.page_ok(x, stride, page, n) == want


# ---- rotary frequencies ------------------------------------------------------------------------------------

def plain_frequencies(r, base, scaling, factor, original, low, high):
    """The formulas of skvq_rope_scaling, pair by pair."""
    f = [base ** (-2.0 * i / r) for i in range(r // 2)]
    amplitude = 1.0
    if scaling == "linear":
        f = [x / factor for x in f]
    elif scaling == "ntk":
        f = [(base * factor ** (r / (r - 2.0))) ** (-2.0 * i / r) for i in range(r // 2)]
    elif scaling == "yarn":
        def pair_of(turns):
            return r * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
        a, b = max(math.floor(pair_of(high)), 0), min(math.ceil(pair_of(low)), r - 1)
        ramp = [min(max((i - a) / max(b - a, 1e-3), 0.0), 1.0) for i in range(r // 2)]
        f = [x / factor * t + x * (1 - t) for x, t in zip(f, ramp)]
        amplitude = 0.1 * math.log(factor) + 1.0
    elif scaling == "bands":
        out = []
        for x in f:
            turns = original * x / (2 * math.pi)
            s = min(max((turns - low) / (high - low), 0.0), 1.0)
            out.append((1 - s) * x / factor + s * x)
        f = out
    return np.array(f), amplitude


@pytest.mark.parametrize("r,base", [(128, 10000.0), (64, 500000.0), (20, 1e6), (4, 10000.0)])
@pytest.mark.parametrize("scaling,factor,original,low,high", [("none", 0.0, 0.0, 0.0, 0.0), ("linear", 8.0, 0.0, 0.0, 0.0),
                                                              ("ntk", 2.5, 0.0, 0.0, 0.0), ("yarn", 16.0, 4096.0, 1.0, 32.0),
                                                              ("bands", 8.0, 8192.0, 1.0, 4.0)])
def test_frequencies_follow_their_formulas(B, r, base, scaling, factor, original, low, high):
    rope = B.SkvqRope(D, r, "half", base, scaling, factor, original, low, high)
    got, amplitude = rope.skvq_rope_frequencies()
    want, a = plain_frequencies(r, base, scaling, factor, original, low, high)
    assert np.allclose(got, want, rtol=1e-13, atol=0) and abs(amplitude - a) < 1e-15
    assert B.SkvqRope(D, r, "half", base, scaling, factor, original, low, high, amplitude=1.25).skvq_rope_frequencies()[1] == 1.25


def test_own_frequencies(B):
    f = np.array([0.5, -3.0, 0.0, 7.25])
    got, amplitude = B.SkvqRope(16, 8, "interleaved", frequencies=f).skvq_rope_frequencies()
    assert np.array_equal(got, f) and amplitude == 1.0
    with pytest.raises(ValueError):
        B.SkvqRope(16, 8, frequencies=f[:3])


def test_rope_refusals(B):
    for kw, status in [(dict(head_dim=128, rotary_dim=130), B.SKVQ_ERR_INVALID_ARG), (dict(rotary_dim=7), B.SKVQ_ERR_INVALID_ARG),
                       (dict(rotary_dim=0), B.SKVQ_ERR_INVALID_ARG), (dict(head_dim=258), B.SKVQ_ERR_UNSUPPORTED),
                       (dict(base=0.0), B.SKVQ_ERR_INVALID_ARG), (dict(base=math.inf), B.SKVQ_ERR_INVALID_ARG),
                       (dict(scaling="linear"), B.SKVQ_ERR_INVALID_ARG), (dict(scaling="ntk", factor=-1.0), B.SKVQ_ERR_INVALID_ARG),
                       (dict(scaling="yarn", factor=1.0, original_context=4096, low=1, high=32), B.SKVQ_ERR_INVALID_ARG),
                       (dict(scaling="yarn", factor=4.0, low=1, high=32), B.SKVQ_ERR_INVALID_ARG),
                       (dict(scaling="bands", factor=4.0, original_context=4096, low=4, high=4), B.SKVQ_ERR_INVALID_ARG),
                       (dict(amplitude=-1.0), B.SKVQ_ERR_INVALID_ARG), (dict(amplitude=math.nan), B.SKVQ_ERR_INVALID_ARG),
                       (dict(frequencies=np.full(64, math.nan)), B.SKVQ_ERR_INVALID_ARG)]:
        with pytest.raises(B.SkvqError) as e:
            B.SkvqRope(**kw)
        assert e.value.status == status, kw
    L, rope = B.lib(), B.SkvqRope()
    one = B.skvq_rope_tensor(64, 64, 0, 0, 0, 0, 0, 0, 1)
    two = (B.skvq_rope_tensor * 2)(one, B.skvq_rope_tensor(64, 64, 0, 0, 0, 0, 0, 8, 1))   # in place, other strides

    def call(rope=rope._h, tensors=C.pointer(one), n=1, dtype=0, batch=1, tokens=1, start=0):
        return L.skvq_rope_apply(rope, tensors, n, dtype, batch, tokens, None, 0, start, 0, None)

    assert L.skvq_rope_create(None, C.byref(C.c_void_p())) == B.SKVQ_ERR_INVALID_ARG
    assert L.skvq_rope_frequencies(None, None, None) == B.SKVQ_ERR_INVALID_ARG
    for kw, want in [(dict(rope=None), B.SKVQ_ERR_INVALID_ARG), (dict(tensors=None), B.SKVQ_ERR_INVALID_ARG),
                     (dict(n=3), B.SKVQ_ERR_INVALID_ARG), (dict(n=0), B.SKVQ_ERR_INVALID_ARG), (dict(dtype=3), B.SKVQ_ERR_UNSUPPORTED),
                     (dict(batch=-1), B.SKVQ_ERR_INVALID_ARG), (dict(tokens=-1), B.SKVQ_ERR_INVALID_ARG),
                     (dict(tokens=2 ** 31), B.SKVQ_ERR_UNSUPPORTED), (dict(batch=2 ** 16, tokens=2 ** 15), B.SKVQ_ERR_UNSUPPORTED),
                     (dict(start=2 ** 31), B.SKVQ_ERR_INVALID_ARG), (dict(start=-2 ** 31 - 1), B.SKVQ_ERR_INVALID_ARG),
                     (dict(tensors=two, n=2), B.SKVQ_ERR_INVALID_ARG),
                     (dict(tensors=C.pointer(B.skvq_rope_tensor(None, 64, 0, 0, 0, 0, 0, 0, 1))), B.SKVQ_ERR_INVALID_ARG),
                     (dict(tensors=C.pointer(B.skvq_rope_tensor(65, 64, 0, 0, 0, 0, 0, 0, 1))), B.SKVQ_ERR_INVALID_ARG),
                     # nothing to do: nothing is launched
                     (dict(batch=0), B.SKVQ_OK), (dict(tokens=0), B.SKVQ_OK),
                     (dict(tensors=C.pointer(B.skvq_rope_tensor(None, None, 0, 0, 0, 0, 0, 0, 0))), B.SKVQ_OK)]:
        assert call(**kw) == want, kw
    B.lib().skvq_rope_destroy(None)


# ---- the paged cache's configuration -------------------------------------------------------------------------

def paged_config(B, **kw):
    hk, g = kw.get("n_kv_heads", 8), kw.get("group_size", 128)
    perm = kw.pop("perm", np.tile(np.arange(D, dtype=np.int32), (hk, 1)))
    clip = kw.pop("clip", np.ones((hk, D // g), np.float32))
    args = dict(n_q_heads=32, n_kv_heads=hk, group_size=g, window=128, page_size=64, n_pages=10, max_seqs=3, max_tokens=7,
                perm_k=perm, perm_v=perm, clip_k=clip, clip_v=clip)
    args.update(kw)
    return B.make_paged_config(**args)


def test_sizes(B):
    for hk, hq, g, meta, size, P, pages, seqs, tokens, W, S in [(8, 32, 128, "f16", 2, 64, 10, 3, 7, 128, 0),
                                                                (2, 32, 32, "e4m3", 1, 16, 1, 1, 1, 1, 5), (1, 1, 64, "f32", 4, 256, 99, 64, 300, 600, 9)]:
        cfg, keep = paged_config(B, n_kv_heads=hk, n_q_heads=hq, group_size=g, meta=meta, page_size=P, n_pages=pages, max_seqs=seqs,
                                 max_tokens=tokens, window=W, n_sink=S)
        rows = seqs * hk * (W + S) * D * 2
        assert B.skvq_paged_sizes(cfg) == [pages * hk * P * (D + 4 * (D // g) * size), rows, rows,
                                           tokens * hq * (128 + -(-(W + S) // 512)) * 132 * 4]


def test_paged_refusals(B):
    bad_perm = np.tile(np.arange(D, dtype=np.int32), (8, 1))
    bad_perm[3, 5] = 6
    I, U = B.SKVQ_ERR_INVALID_ARG, B.SKVQ_ERR_UNSUPPORTED
    for kw, want in [(dict(perm=bad_perm), I), (dict(clip=np.full((8, 1), 1.5)), I), (dict(clip=np.zeros((8, 1))), I),
                     (dict(clip=np.full((8, 1), np.nan)), I), (dict(n_q_heads=30), I), (dict(window=0), I), (dict(n_sink=-1), I),
                     (dict(n_pages=0), I), (dict(max_seqs=0), I), (dict(max_tokens=0), I), (dict(sm_scale=-1.0), I),
                     (dict(sm_scale=math.nan), I), (dict(window=2 ** 20 + 1), I), (dict(n_sink=2 ** 20 + 1), I),
                     (dict(n_q_heads=8 * 17), U), (dict(k_bits=2.0), U), (dict(v_bits=1.5), U), (dict(dtype=torch.float32), U),
                     (dict(page_size=8), U), (dict(page_size=48), U), (dict(page_size=512), U), (dict(page_size=0), U),
                     (dict(max_tokens=2 ** 27), U)]:
        cfg, keep = paged_config(B, **kw)
        assert B.skvq_paged_validate_config(cfg) == want, kw
        with pytest.raises(B.SkvqError):
            B.skvq_paged_sizes(cfg)
    for kw in (dict(head_dim=64), dict(group_size=16)):
        ok, keep = paged_config(B)
        for name, value in kw.items():
            setattr(ok, name, value)
        assert B.skvq_paged_validate_config(ok) == U
    for name in ("perm_k", "perm_v", "clip_k", "clip_v"):
        ok, keep = paged_config(B)
        setattr(ok, name, None)
        assert B.skvq_paged_validate_config(ok) == I
    ok, keep = paged_config(B)
    assert B.skvq_paged_validate_config(ok) == B.SKVQ_OK
    L, h = B.lib(), C.c_void_p()
    # refused before the device is touched
    assert L.skvq_paged_create(C.byref(ok), None, C.byref(h)) == I
    for bufs in ([0, 16, 16, 16], [16, 16, 8, 16]):
        assert L.skvq_paged_create(C.byref(ok), C.byref(B.skvq_paged_buffers(*bufs)), C.byref(h)) == I and not h.value
    assert L.skvq_paged_create(C.byref(ok), C.byref(B.skvq_paged_buffers(16, 16, 16, 16)), None) == I
    batch = B.skvq_batch(1, 1, 64, 64, 64, 1, None, None, None)
    assert L.skvq_paged_append(None, None, C.byref(batch), 64, 1024, 64, 1024, None, 0, None, 0, None) == I
    assert L.skvq_paged_read(None, C.byref(batch), 64, 1024, 64, 1024, None) == I
    assert L.skvq_paged_attention(None, C.byref(batch), 64, 4096, 64, 4096, None, None) == I
    assert L.skvq_paged_errors(None, C.byref(C.c_int32()), None) == I
    assert L.skvq_paged_last_error(None) == b""
    L.skvq_paged_destroy(None)
    with pytest.raises(ValueError):
        paged_config(B, clip=np.ones((8, 2), np.float32))
