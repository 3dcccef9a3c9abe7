"""The operators of serving many sequences from one pool of 4-bit pages, as cases that can be timed and compared.

A case is one attention layer's shape and format, the batch of sequences, and one of these kinds of pass:

  rope     skvq_rope_apply: rotary positions of queries and keys (or the gradient's way back through them)
  append   skvq_paged_append: the batch's new tokens rotated and put into the paged cache, and
           skvq_paged_read of the rows that this packed, as a program reads them that hands them on
  read     skvq_paged_read: cached tokens of every sequence back as rows, to move a sequence elsewhere
  attend   skvq_paged_attention: the batch's query tokens attend over their sequences' cached tokens

The plain forms work on the same buffers.  A page holds, per kv head, P tokens in four sections:

  key codes    P rows of 16 dwords: position p = 32 j + 8 g + e of the reordered head is in dword 4 g + j,
               nibble e / 2 for an even e, 4 + e / 2 for an odd one
  value codes  for every four tokens 16 pieces of 16 bytes: position p = 16 n + m of token r of the four is in
               piece m, byte 8 (r / 2) + 4 (n / 4) + 2 (r % 2) + (n % 4) / 2, the low nibble for an even n
  key pairs    (scale, zero) of every group, P x D / G pairs
  value pairs  likewise

and a token beyond the window is packed row (token - sinks) of its sequence, in page_table[row / P]; the last
`window` tokens are rows token % window of the sequence's fp16 (bf16) rows, the first `sinks` ones, once they
have left the window, the rows after those.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

D = 128
CLIP = 0.95
META = {"f32": (torch.float32, 4), "f16": (torch.float16, 2), "e4m3": (torch.float8_e4m3fn, 1)}
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
DEVICE = "cuda:0"


def _rope_case(name, batch, tokens, q_heads, kv_heads, dtype, head_dim=D, rotary=D, layout="half", scaling="none", start=0,
               transpose=False):
    return {"name": name, "kind": "rope", "batch": batch, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads,
            "dtype": dtype, "head_dim": head_dim, "rotary": rotary, "layout": layout, "scaling": scaling, "start": start,
            "transpose": transpose}


def _paged_case(name, kind, seqs, context, q_heads, kv_heads, dtype="f16", group=128, meta="f16", page=64, window=128,
                sinks=0, new=1, ragged=False, rotary=D, layout="half", scaling="none"):
    return {"name": name, "kind": kind, "seqs": seqs, "context": context, "q_heads": q_heads, "kv_heads": kv_heads,
            "dtype": dtype, "group": group, "meta": meta, "page": page, "window": window, "sinks": sinks, "new": new,
            "ragged": ragged, "rotary": rotary, "layout": layout, "scaling": scaling}


def listed():
    return [
        # a decode step's rotation of one token: one small launch, nothing but latency
        _rope_case("rope_step", 1, 1, 32, 8, "f16", start=4095),
        # the rotation of a long prompt, with frequencies stretched for long contexts
        _rope_case("rope_prompt_32k_yarn", 1, 32768, 32, 8, "bf16", scaling="yarn"),
        # the gradient's way back in 32 bits: neighbouring pairs, half of an odd head turned, odd lengths
        _rope_case("rope_backward_partial", 3, 1913, 32, 32, "f32", head_dim=96, rotary=48, layout="interleaved",
                   transpose=True),
        # a batched decode step's new tokens: each sequence packs the token that leaves its window
        _paged_case("append_step_batch64", "append", 64, 16384, 32, 8, page=16, ragged=True),
        # a batch of prompts of all lengths enters empty slots, in the setting of the 4-bit accuracy figures
        # (groups of 64, FP8 scale and zero, five sinks)
        _paged_case("append_prompts_batch16", "append", 16, 8192, 32, 8, "bf16", group=64, meta="e4m3", sinks=5, new=0,
                    ragged=True, scaling="bands"),
        # a short sequence leaves the pool
        _paged_case("read_short", "read", 1, 700, 4, 4, page=16),
        # a batch of long ones does
        _paged_case("read_batch8_16k", "read", 8, 16384, 32, 8, "bf16", group=64, meta="e4m3", sinks=5, ragged=True),
        # the smallest decode call: a small model at 2k tokens of context
        _paged_case("attend_4heads_2k", "attend", 1, 2048, 4, 4, page=16),
        # one long document with grouped queries
        _paged_case("attend_gqa_128k", "attend", 1, 131072, 32, 8),
        # continuous batching: 64 sequences of all lengths, small pages
        _paged_case("attend_ragged64_16k", "attend", 64, 16384, 32, 8, "bf16", group=64, meta="e4m3", page=16, sinks=5,
                    ragged=True),
        # the largest: a batch of long sequences with a kv head per query head
        _paged_case("attend_batch16_32k", "attend", 16, 32768, 32, 32),
        # speculated tokens checked: up to eight query tokens per sequence, eight query heads per kv head
        _paged_case("attend_verify8_40k", "attend", 8, 40011, 64, 8, "bf16", group=32, meta="f32", new=8, ragged=True),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """One more case: types, heads, groups, formats, pages and windows that the operators take, lengths from a
    few tokens to those of the listed cases, no more work than the largest of its kind."""
    kind = rng.choice(["rope", "append", "append", "read", "attend", "attend", "attend"])
    q_heads, kv_heads = rng.choice([(4, 4), (8, 1), (16, 4), (24, 8), (32, 8), (32, 32), (64, 8)])
    scaling = rng.choice(["none", "linear", "ntk", "yarn", "bands"])
    if kind == "rope":
        head_dim, rotary = rng.choice([(128, 128), (128, 64), (64, 64), (96, 48), (80, 20), (256, 64), (192, 192)])
        batch = _log_int(rng, 1, 8)
        tokens = max(1, min(_log_int(rng, 1, 32768), 32768 * 40 * 128 // (batch * (q_heads + kv_heads) * head_dim)))
        case = _rope_case("", batch, tokens, q_heads, kv_heads, rng.choice(["f16", "bf16", "f32"]), head_dim, rotary,
                          rng.choice(["half", "interleaved"]), scaling, rng.choice([0, 17, 99991, 1000003]),
                          rng.random() < 0.3)
    else:
        context = _log_int(rng, 3, {"append": 8192, "read": 16384, "attend": 131072}[kind])
        most = {"append": 16 * 8 * 8192, "read": 8 * 8 * 16384, "attend": 16 * 32 * 32768 // 4}[kind]
        seqs = _log_int(rng, 1, max(1, min(64, most // (kv_heads * context))))
        context = max(3, min(context, most // (kv_heads * seqs)))
        new = rng.choice([1, 1, 2, 5, 8]) if kind == "attend" else rng.choice([0, 1, 7, 300]) if kind == "append" else 1
        group, meta = rng.choice([(128, "f16"), (128, "f32"), (64, "e4m3"), (64, "f16"), (32, "e4m3"), (32, "f32")])
        case = _paged_case("", kind, seqs, context, q_heads, kv_heads, rng.choice(["f16", "bf16"]), group, meta,
                           rng.choice([16, 32, 64, 128, 256]), rng.choice([1, 16, 100, 128, 512]), rng.choice([0, 0, 4, 5]),
                           min(new, context), rng.random() < 0.7, rng.choice([128, 64]), rng.choice(["half", "interleaved"]),
                           scaling)
    del case["name"]
    return case


def _lengths(case):
    """(tokens cached after the pass, new tokens) of every sequence, from the case alone: the first has the
    case's context, the others of a ragged batch anything down to a 64th of it."""
    rng = random.Random(case["seqs"] * 1_000_003 + case["context"])
    low = max(1, case["context"] // 64)
    total = [case["context"] if i == 0 or not case["ragged"] else _log_int(rng, low, case["context"])
             for i in range(case["seqs"])]
    if case["kind"] == "read":
        new = total
    elif case["new"] == 0:
        new = total
    else:
        new = [min(t, case["new"] if i == 0 or not case["ragged"] else rng.randint(1, case["new"])) for i, t in enumerate(total)]
    return total, new


# ---- frequencies ----------------------------------------------------------------------------------------

BASE, FACTOR, ORIGINAL = 10000.0, 4.0, 8192
SCALING_ARGS = {"none": {}, "linear": {"factor": FACTOR}, "ntk": {"factor": FACTOR},
                "yarn": {"factor": FACTOR, "original_context": ORIGINAL, "low": 1.0, "high": 32.0},
                "bands": {"factor": FACTOR, "original_context": ORIGINAL, "low": 1.0, "high": 4.0}}


def _frequencies(rotary, scaling):
    """Radians per token of every pair in 64 bits, and the factor on cosine and sine."""
    i = np.arange(rotary // 2, dtype=np.float64)
    f = BASE ** (-2.0 * i / rotary)
    if scaling == "linear":
        return f / FACTOR, 1.0
    if scaling == "ntk":
        return (BASE * FACTOR ** (rotary / max(rotary - 2.0, 1.0))) ** (-2.0 * i / rotary), 1.0
    if scaling == "yarn":  # turns over the original context: 32 and more keep their frequency, one and fewer are stretched
        def pair_of(turns):
            return rotary * math.log(ORIGINAL / (turns * 2.0 * math.pi)) / (2.0 * math.log(BASE))
        low, high = max(math.floor(pair_of(32.0)), 0), min(math.ceil(pair_of(1.0)), rotary - 1)
        ramp = np.clip((i - low) / max(high - low, 1e-3), 0.0, 1.0)
        return f / FACTOR * ramp + f * (1.0 - ramp), 0.1 * math.log(FACTOR) + 1.0
    if scaling == "bands":
        turns = ORIGINAL * f / (2.0 * math.pi)
        s = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return (1.0 - s) * f / FACTOR + s * f, 1.0
    return f, 1.0


# ---- inputs -----------------------------------------------------------------------------------------------

def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE)


def _channel_order(gen, kv_heads):
    """Channels by their magnitude (spread over a decade), as the reorder of a calibrated cache is."""
    size = 10.0 ** (torch.rand((kv_heads, D), generator=gen, device=DEVICE) - 0.5)
    return size, torch.argsort(size, dim=-1)


def _page_bytes(case):
    return case["page"] * (D + 4 * (D // case["group"]) * META[case["meta"]][1])


def _pairs(gen, case, pages, centre):
    """(scale, zero) pairs of a section of every page, as normal values of about unit size lead to."""
    hk, ng = case["kv_heads"], D // case["group"]
    spread = (0.25 + 0.3 * torch.rand((pages, hk, case["page"], ng), generator=gen, device=DEVICE)) * CLIP
    zero = -spread * 7.5 * (0.9 + 0.2 * torch.rand(spread.shape, generator=gen, device=DEVICE)) + centre
    return torch.stack((spread, zero), -1).to(META[case["meta"]][0])


def _filled_pages(gen, case, pages):
    hk, P = case["kv_heads"], case["page"]
    codes = torch.randint(0, 256, (pages, hk, P * D), generator=gen, device=DEVICE, dtype=torch.uint8)
    parts = [codes] + [_pairs(gen, case, pages, c).view(torch.uint8).reshape(pages, hk, -1) for c in (0.0, 0.1)]
    return torch.cat(parts, -1).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    dtype = TYPES[case["dtype"]]
    hq, hk = case["q_heads"], case["kv_heads"]
    state = {"case": case}
    if case["kind"] == "rope":
        # queries and keys as the layer's projection leaves them: one row per token, queries, keys and values in turn
        b, t, d = case["batch"], case["tokens"], case["head_dim"]
        rows = _normal(gen, b, t, hq + 2 * hk, d).to(dtype)
        state["q"], state["k"] = rows[:, :, :hq], rows[:, :, hq:hq + hk]
        # outputs as the prompt's attention takes them: a head's tokens in a row
        state["out"] = [torch.empty((b, h, t, d), dtype=dtype, device=DEVICE).transpose(1, 2) for h in (hq, hk)]
        if own:
            from paper_2405_06219_amd import binding
            state["rope"] = binding.SkvqRope(d, case["rotary"], case["layout"], BASE, case["scaling"],
                                             **SCALING_ARGS[case["scaling"]])
        return state
    total, new = _lengths(case)
    P, W, S = case["page"], case["window"], case["sinks"]
    stride = max(1, -(-max(max(total) - W - S, 0) // P))
    per_seq = [-(-max(t - W - S, 0) // P) for t in total]
    pages = sum(per_seq) + 1
    order = torch.randperm(pages, generator=gen, device=DEVICE).to(torch.int32).cpu().numpy()
    table, at = np.full((len(total), stride), -1, np.int32), 0
    for i, n in enumerate(per_seq):
        table[i, :n] = order[at:at + n]
        at += n
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    leaves = [max(t - W, 0) - max(t - n - W, 0) for t, n in zip(total, new)]  # tokens that this pass packs or keeps
    state.update(n_tokens=int(cu[-1]), cu=torch.from_numpy(cu).to(DEVICE),
                 lens=torch.tensor(total, dtype=torch.int32, device=DEVICE), table=torch.from_numpy(table).to(DEVICE),
                 slots=torch.randperm(len(total), generator=gen, device=DEVICE).to(torch.int32))
    state["size_k"], state["perm_k"] = _channel_order(gen, hk)
    state["size_v"], state["perm_v"] = _channel_order(gen, hk)
    if case["kind"] == "append":
        state["pages"] = torch.zeros((pages, hk, _page_bytes(case)), dtype=torch.uint8, device=DEVICE)
    else:
        state["pages"] = _filled_pages(gen, case, pages)
    shape = (len(total), hk, W + S, D)
    state["k_rows"] = _normal(gen, *shape).to(dtype)
    state["v_rows"] = _normal(gen, *shape).to(dtype)
    n = state["n_tokens"]
    if case["kind"] == "append":
        state["k_rows"], state["v_rows"] = ((x.float() * state[s][None, :, None]).to(dtype) for x, s in
                                            ((state["k_rows"], "size_k"), (state["v_rows"], "size_v")))
        rows = _normal(gen, n, (hq + 2 * hk), D)
        rows[:, hq:hq + hk] *= state["size_k"]
        rows[:, hq + hk:] *= state["size_v"]
        rows = rows.to(dtype)
        state["q"], state["k"], state["v"] = rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:]
        state["out"] = torch.empty((n, hq, D), dtype=dtype, device=DEVICE)
        cu2 = np.concatenate([[0], np.cumsum(leaves)]).astype(np.int32)
        first = [max(t - x - W, 0) for t, x in zip(total, new)]
    else:
        cu2, first = cu, [0] * len(total)
    if case["kind"] != "attend":
        state["read_n"], state["read_cu"] = int(cu2[-1]), torch.from_numpy(cu2).to(DEVICE)
        state["read_first"] = torch.tensor(first, dtype=torch.int32, device=DEVICE)
        state["read_out"] = [torch.empty((int(cu2[-1]), hk, D), dtype=dtype, device=DEVICE) for _ in range(2)]
    else:
        state["q"] = _normal(gen, n, hq, D).to(dtype)
        state["out"] = torch.empty((n, hq, D), dtype=dtype, device=DEVICE)
    if own:
        from paper_2405_06219_amd import binding
        clip = np.full((hk, D // case["group"]), CLIP, np.float32)
        perm_k, perm_v = (state[p].to(torch.int32).cpu().numpy() for p in ("perm_k", "perm_v"))
        state["cache"] = binding.SkvqPagedCache(
            hq, hk, case["group"], W, P, pages, len(total), n, perm_k, perm_v, clip, clip, n_sink=S, meta=case["meta"],
            dtype=dtype, device=DEVICE,
            buffers={"pages": state["pages"], "k_rows": state["k_rows"], "v_rows": state["v_rows"]})
        state["rope"] = binding.SkvqRope(D, case["rotary"], case["layout"], BASE, case["scaling"],
                                         **SCALING_ARGS[case["scaling"]])
        state["batch"] = binding.SkvqBatch(state["cu"], state["lens"], state["table"], slots=state["slots"], n_tokens=n)
        if case["kind"] != "attend":
            state["read"] = binding.SkvqBatch(state["read_cu"], state["lens"], state["table"], slots=state["slots"],
                                              first=state["read_first"], n_tokens=state["read_n"])
    return state


# ---- the plain forms ----------------------------------------------------------------------------------------

def _rotate(x, position, case, transpose=False):
    """x [..., heads, d] with position [...]: each pair of the first `rotary` channels turned, cosine and sine
    from 64-bit angles and rounded to 32 bits, products and sums in 32, rounded to x's type."""
    r = case["rotary"]
    freq, amplitude = _frequencies(r, case["scaling"])
    angle = position[..., None].double() * torch.from_numpy(freq).to(x.device)
    cos = (torch.cos(angle) * amplitude).float()[..., None, :]
    sin = (torch.sin(angle) * amplitude).float()[..., None, :] * (-1.0 if transpose else 1.0)
    part = x[..., :r].float()
    if case["layout"] == "half":
        a, b = part[..., :r // 2], part[..., r // 2:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((turned.to(x.dtype), x[..., r:]), -1)


def _key_places(device):
    """Nibble of a key row that holds reordered position p."""
    p = torch.arange(D, device=device)
    j, g, e = p // 32, p % 32 // 8, p % 8
    return 8 * (4 * g + j) + torch.where(e % 2 == 0, e // 2, 4 + e // 2)


def _value_places(device):
    """Nibble of four tokens' 256 value bytes that holds position p of token r: [4][D]."""
    r, p = torch.arange(4, device=device)[:, None], torch.arange(D, device=device)[None, :]
    n, m = p // 16, p % 16
    return 2 * (16 * m + 8 * (r // 2) + 4 * (n // 4) + 2 * (r % 2) + n % 4 // 2) + n % 2


def _nibbles(b):
    return torch.stack((b & 15, b >> 4), -1).flatten(-2)


def _unpacked(state, pages):
    """Keys and values of whole pages [..., hk, bytes] as 32-bit numbers, reordered positions: two of [..., hk, P, D]."""
    case = state["case"]
    P, G, lead = case["page"], case["group"], pages.shape[:-1]
    kind, size = META[case["meta"]]
    half, pairs = P * D // 2, 2 * P * (D // G) * size
    k, v, mk, mv = torch.split(pages, (half, half, pairs, pairs), -1)
    k = _nibbles(k.reshape(*lead, P, D // 2))[..., _key_places(pages.device)]
    v = _nibbles(v.reshape(*lead, P // 4, 2 * D))[..., _value_places(pages.device).flatten()].reshape(*lead, P, D)

    def values(codes, pair):
        pair = pair.contiguous().view(kind).reshape(*lead, P, D // G, 1, 2).float()
        return (codes.reshape(*lead, P, D // G, G).float() * pair[..., 0] + pair[..., 1]).flatten(-2)

    return values(k, mk), values(v, mv)


def _in_channels(x, perm):
    """x [..., hk, n, D] from reordered positions to channels; perm [hk, D]."""
    return torch.gather(x, -1, torch.argsort(perm, -1)[:, None, :].expand_as(x))


def _members(cu, n):
    """For each of the n tokens that cu counts: its sequence, and its number there."""
    counts = (cu[1:] - cu[:-1]).long()
    seq = torch.repeat_interleave(torch.arange(counts.numel(), device=cu.device), counts, output_size=n)
    return seq, torch.arange(n, device=cu.device) - cu.long()[seq]


def _places(case, t):
    """Bytes of a page's part of one kv head that hold packed row t [n] of the page: key codes, value codes, key
    pairs, value pairs, each [n, count]; and the positions of a row's key nibbles [D] and value nibbles [n, D]."""
    P, ng, size, device = case["page"], D // case["group"], META[case["meta"]][1], t.device
    half, pair = P * D // 2, ng * 2 * size
    order = torch.argsort(_value_places(device), -1)
    value_bytes = torch.gather(_value_places(device), -1, order)[:, ::2] // 2
    pairs = 2 * half + (t * pair)[:, None] + torch.arange(pair, device=device)
    return ((t * (D // 2))[:, None] + torch.arange(D // 2, device=device), half + (t // 4 * 2 * D)[:, None] + value_bytes[t % 4],
            pairs, pairs + P * pair, torch.argsort(_key_places(device)), order[t % 4])


def _tokens_as_rows(state, seq, token):
    """Cached tokens (sequence, number) as K and V rows [n, hk, D] in the cache's type."""
    case = state["case"]
    P, W, S, G, hk = case["page"], case["window"], case["sinks"], case["group"], case["kv_heads"]
    kind = META[case["meta"]][0]
    total, slot = state["lens"].long()[seq], state["slots"].long()[seq]
    kept, recent = token < S, token >= total - W
    row = torch.where(recent, token % W, W + torch.clamp(token, max=max(S - 1, 0)))
    row = torch.clamp(row, max=W + S - 1)
    te = torch.clamp(token - S, min=0)
    packed = ~(kept | recent)
    page = state["table"].long()[seq, torch.clamp(te // P, max=state["table"].shape[1] - 1)]
    page = torch.where(packed, page, 0)[:, None, None]
    head = torch.arange(hk, device=token.device)
    k_at, v_at, mk_at, mv_at, k_order, v_order = _places(case, te % P)

    def values(at, pair_at, order, perm):
        codes = _nibbles(state["pages"][page, head[:, None], at[:, None]])
        codes = torch.gather(codes, -1, torch.argsort(order, -1)[:, None].expand_as(codes)).reshape(-1, hk, D // G, G)
        pair = state["pages"][page, head[:, None], pair_at[:, None]].view(kind).reshape(-1, hk, D // G, 2).float()
        x = (codes.float() * pair[..., :1] + pair[..., 1:]).flatten(-2)
        return torch.gather(x, -1, torch.argsort(perm, -1).expand_as(x))

    k = values(k_at, mk_at, k_order.expand(te.shape[0], D), state["perm_k"])
    v = values(v_at, mv_at, v_order, state["perm_v"])
    return [torch.where(packed[:, None, None], x.to(rows.dtype), rows[slot[:, None], head, row[:, None]])
            for x, rows in ((k, state["k_rows"]), (v, state["v_rows"]))]


def _pack(state, seq, token, k, v):
    """Rows k, v [n, hk, D] of tokens that leave the window into pages (or the sinks' rows): Eq. 2."""
    case = state["case"]
    P, W, S, G, hk = case["page"], case["window"], case["sinks"], case["group"], case["kv_heads"]
    kind, ng = META[case["meta"]][0], D // case["group"]
    head = torch.arange(hk, device=token.device)
    kept = token < S
    slot = state["slots"].long()[seq][kept][:, None]
    state["k_rows"][slot, head, (W + token[kept])[:, None]] = k[kept]
    state["v_rows"][slot, head, (W + token[kept])[:, None]] = v[kept]
    seq, te, k, v = seq[~kept], token[~kept] - S, k[~kept], v[~kept]
    page = state["table"].long()[seq, te // P][:, None, None]
    k_at, v_at, mk_at, mv_at, k_order, v_order = _places(case, te % P)

    def store(x, perm, at, pair_at, order):
        x = torch.gather(x.float(), -1, perm.expand(x.shape)).reshape(-1, hk, ng, G)
        low, high = (x.amin(-1) + 0.0) * CLIP, (x.amax(-1) + 0.0) * CLIP
        pair = torch.stack(((high - low) / torch.full_like(high, 15.0), low), -1)
        pair = (pair.clamp(-448.0, 448.0) if kind == torch.float8_e4m3fn else pair).to(kind)
        scale, zero = pair.float().unbind(-1)
        inverse = torch.where(scale > 0, 1.0 / scale, 0.0)
        codes = torch.clamp(torch.round((x - zero[..., None]) * inverse[..., None]), 0, 15)
        codes = codes.reshape(-1, hk, D).to(torch.uint8)
        codes = torch.gather(codes, -1, order[:, None].expand_as(codes)).reshape(-1, hk, D // 2, 2)
        state["pages"][page, head[:, None], at[:, None]] = codes[..., 0] | (codes[..., 1] << 4)
        state["pages"][page, head[:, None], pair_at[:, None]] = pair.reshape(-1, hk, ng * 2).view(torch.uint8)

    store(k, state["perm_k"], k_at, mk_at, k_order.expand(te.shape[0], D))
    store(v, state["perm_v"], v_at, mv_at, v_order)


def _append(state):
    case = state["case"]
    W, hk = case["window"], case["kv_heads"]
    head = torch.arange(hk, device=state["cu"].device)
    seq, j = _members(state["cu"], state["n_tokens"])
    total = state["lens"].long()
    before = total - (state["cu"][1:] - state["cu"][:-1]).long()
    token = before[seq] + j
    q, k = _rotate(state["q"], token, case), _rotate(state["k"], token, case)
    v = state["v"]
    state["out"].copy_(q)
    # the tokens that leave: from the ring, or new ones that never get there
    lseq, x = _members(state["read_cu"], state["read_n"])
    leaving = torch.clamp(before - W, min=0)[lseq] + x
    fresh = leaving >= before[lseq]
    slot = state["slots"].long()[lseq]
    at = torch.where(fresh, state["cu"].long()[lseq] + leaving - before[lseq], 0)
    rows = [torch.where(fresh[:, None, None], new[at], ring[slot[:, None], head, (leaving % W)[:, None]])
            for new, ring in ((k, state["k_rows"]), (v, state["v_rows"]))]
    _pack(state, lseq, leaving, *rows)
    stay = token >= total[seq] - W
    slot, row = state["slots"].long()[seq][stay][:, None], (token[stay] % W)[:, None]
    state["k_rows"][slot, head, row] = k[stay]
    state["v_rows"][slot, head, row] = v[stay]


def _attend(state):
    case = state["case"]
    P, W, S, hk = case["page"], case["window"], case["sinks"], case["kv_heads"]
    R = case["q_heads"] // hk
    total, seqs = state["lens"].long(), case["seqs"]
    seq, j = _members(state["cu"], state["n_tokens"])
    new = (state["cu"][1:] - state["cu"][:-1]).long()
    most = case["new"]
    # queries [seqs, hk, most * R, D]
    q = torch.zeros((seqs, most, case["q_heads"], D), dtype=torch.float32, device=seq.device)
    q[seq, j] = state["q"].float()
    q = q.reshape(seqs, most, hk, R, D).permute(0, 2, 1, 3, 4).reshape(seqs, hk, most * R, D) / math.sqrt(D)
    last = total[:, None] - new[:, None] + torch.arange(most, device=seq.device)  # the last token a query sees
    # packed rows, then the fp16 (bf16) rows
    table = torch.clamp(state["table"].long(), min=0)
    k, v = (x[table].transpose(1, 2).flatten(2, 3) for x in _unpacked(state, state["pages"]))
    row = torch.arange(table.shape[1] * P, device=seq.device)[None] + S
    row = torch.where(row < total[:, None] - W, row, 1 << 40)
    ring = torch.arange(W, device=seq.device)[None]
    ring = total[:, None] - 1 - (total[:, None] - 1 - ring) % W
    ring = torch.where(ring >= 0, ring, 1 << 40)
    sink = torch.arange(S, device=seq.device)[None].expand(seqs, S)
    sink = torch.where(sink < total[:, None] - W, sink, 1 << 40)
    slots = state["slots"].long()
    here = torch.cat((row, ring, sink), 1)
    k_rows, v_rows = state["k_rows"][slots].float(), state["v_rows"][slots].float()
    scores = torch.cat((torch.matmul(torch.gather(q, -1, state["perm_k"][:, None, :].expand_as(q)), k.transpose(-1, -2)),
                        torch.matmul(q, k_rows.transpose(-1, -2))), -1)
    del k
    seen = here[:, None, :] <= last[:, :, None]
    scores.masked_fill_(~seen.repeat_interleave(R, 1)[:, None], -math.inf)
    scores -= torch.clamp(scores.amax(-1, keepdim=True), min=-1e30)
    weights = torch.exp_(scores)
    sums = weights.sum(-1, keepdim=True)
    n = row.shape[1]
    out = _in_channels(torch.matmul(weights[..., :n], v), state["perm_v"]) + torch.matmul(
        weights[..., n:], torch.where((here[:, n:] < 1 << 40)[:, None, :, None], v_rows, 0.0))
    out = (out / sums).reshape(seqs, hk, most, R, D).permute(0, 2, 1, 3, 4).reshape(seqs, most, case["q_heads"], D)
    return out[seq, j].to(state["q"].dtype)


def _plain(state):
    case = state["case"]
    if case["kind"] == "rope":
        position = torch.arange(case["tokens"], device=DEVICE) + case["start"]
        position = position[None].expand(case["batch"], -1)
        state["out"][0].copy_(_rotate(state["q"], position, case, case["transpose"]))
        state["out"][1].copy_(_rotate(state["k"], position, case, case["transpose"]))
        return {"q": state["out"][0], "k": state["out"][1]}
    if case["kind"] == "attend":
        return {"out": _attend(state)}
    if case["kind"] == "append":
        _append(state)
    seq, x = _members(state["read_cu"], state["read_n"])
    k, v = _tokens_as_rows(state, seq, state["read_first"].long()[seq] + x)
    if case["kind"] == "read":
        return {"k": k, "v": v}
    return {"q": state["out"], "k": k, "v": v, "k_rows": state["k_rows"], "v_rows": state["v_rows"]}


def run(state):
    """One pass through the case's operator, and its outputs."""
    if not own:
        return _plain(state)
    case = state["case"]
    if case["kind"] == "rope":
        q, k = state["rope"].skvq_rope_apply(state["q"], state["k"], start=case["start"], out_q=state["out"][0],
                                             out_k=state["out"][1], transpose=case["transpose"])
        return {"q": q, "k": k}
    if case["kind"] == "attend":
        return {"out": state["cache"].skvq_paged_attention(state["batch"], state["q"], out=state["out"])}
    if case["kind"] == "append":
        state["cache"].skvq_paged_append(state["batch"], state["k"], state["v"], rope=state["rope"], q=state["q"],
                                         out_q=state["out"])
    k, v = state["cache"].skvq_paged_read(state["read"], out_k=state["read_out"][0], out_v=state["read_out"][1])
    if case["kind"] == "read":
        return {"k": k, "v": v}
    return {"q": state["out"], "k": k, "v": v, "k_rows": state["k_rows"], "v_rows": state["v_rows"]}


# ---- what a pass cannot do without ---------------------------------------------------------------------------

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    hq, hk = case["q_heads"], case["kv_heads"]
    if case["kind"] == "rope":
        n = case["batch"] * case["tokens"] * (hq + hk)
        return {"bytes": 2 * n * case["head_dim"] * size, "flops": 3 * n * case["rotary"]}
    total, new = _lengths(case)
    W, S = case["window"], case["sinks"]
    row = hk * (D + 4 * (D // case["group"]) * META[case["meta"]][1])   # a packed token
    full = hk * 2 * D * size                                            # a token in fp16 or bf16
    packed = sum(max(t - W - S, 0) for t in total)
    rows = sum(min(t, W + S) for t in total)
    if case["kind"] == "attend":
        pairs = sum(hq * n * t - hq * (n * (n - 1) // 2) for t, n in zip(total, new))
        return {"bytes": packed * row + rows * full + 2 * sum(new) * hq * D * size, "flops": 4 * D * pairs}
    if case["kind"] == "read":
        return {"bytes": packed * row + rows * full + sum(total) * full, "flops": 4 * D * hk * packed}
    leaves = [max(t - W, 0) - max(t - n - W, 0) for t, n in zip(total, new)]
    old = sum(min(x, t - n) for x, t, n in zip(leaves, total, new))     # of them, from the ring
    out = sum(leaves)
    # the new rows read, the ones that stay written, the leaving ones read and packed; then those read back
    rows_in = sum(new) * (hq * D * 2 * size + full) + sum(min(n, W) for n in new) * full + old * full + out * row
    return {"bytes": rows_in + out * (row + full), "flops": (sum(new) * (hq + hk) * 3 * case["rotary"] + out * hk * D * 12)}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------

def _turned64(x, position, case, transpose=False):
    freq, amplitude = _frequencies(case["rotary"], case["scaling"])
    half = case["rotary"] // 2
    pairs = [(c, c + half) if case["layout"] == "half" else (2 * c, 2 * c + 1) for c in range(half)]
    first, second = (torch.tensor([p[i] for p in pairs], device=x.device) for i in (0, 1))
    theta = position.double()[..., None, None] * torch.from_numpy(freq).to(x.device)
    turn = torch.polar(torch.full_like(theta, amplitude), -theta if transpose else theta)
    y = x.double().clone()
    z = torch.complex(y[..., first], y[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _stored_pair64(case, low, high):
    pair = torch.stack(((high - low) / 15.0, low), -1)
    if case["meta"] == "e4m3":
        pair = pair.clamp(-448.0, 448.0)
    return pair.float().to(META[case["meta"]][0]).double().unbind(-1)


def _stored64(case, x, perm):
    """What rows x [n, hk, D] stand for once packed, a group at a time.  Values lie on borders between codes (short
    numbers meet short scales), so the three operations that choose a code round to 32 bits, as Eq. 2 has it here."""
    out = torch.empty_like(x)
    for h in range(case["kv_heads"]):
        for g in range(D // case["group"]):
            channels = perm[h, g * case["group"]:(g + 1) * case["group"]]
            y = x[:, h][:, channels]
            clip = float(np.float32(CLIP))
            scale, zero = _stored_pair64(case, clip * y.min(1).values, clip * y.max(1).values)
            step = torch.where(scale > 0, 1.0 / scale, 0.0).float().double()
            above = (y - zero[:, None]).float().double()
            code = torch.round((above * step[:, None]).float().double()).clamp(0, 15)
            out[:, h, channels] = zero[:, None] + scale[:, None] * code
    return out


def _packed64(state, i, h, count, section):
    """The first `count` packed rows of sequence i, kv head h, reordered positions: nibble by nibble from the bytes."""
    case = state["case"]
    P, G = case["page"], case["group"]
    kind, size = META[case["meta"]]
    n_pages = -(-count // P)
    raw = state["pages"][state["table"][i, :n_pages].long(), h]
    half, pairs = P * D // 2, 2 * P * (D // G) * size
    code = torch.empty((n_pages, P, D), dtype=torch.float64, device=raw.device)
    body = raw[:, section * half:(section + 1) * half]
    for p in range(D):
        if section == 0:
            j, g, e = p // 32, p % 32 // 8, p % 8
            nibble = e // 2 if e % 2 == 0 else 4 + e // 2
            b = body.reshape(n_pages, P, D // 2)[:, :, 4 * (4 * g + j) + nibble // 2]
            code[:, :, p] = ((b >> 4) if nibble % 2 else (b & 15)).double()
        else:
            n, m = p // 16, p % 16
            four = body.reshape(n_pages, P // 4, 16, 16)[:, :, m]
            for r in range(4):
                b = four[:, :, 8 * (r // 2) + 4 * (n // 4) + 2 * (r % 2) + n % 4 // 2]
                code[:, r::4, p] = ((b >> 4) if n % 2 else (b & 15)).double()
    at = 2 * half + section * pairs
    pair = raw[:, at:at + pairs].contiguous().view(kind).double().reshape(n_pages, P, D // G, 2)
    pair = pair.repeat_interleave(G, 2)
    return (code * pair[..., 0] + pair[..., 1]).reshape(-1, D)[:count]


def _cached64(state, i, h):
    """All cached tokens of sequence i, kv head h: K and V [tokens, D] in channel order."""
    case = state["case"]
    T, W, S = int(state["lens"][i]), case["window"], case["sinks"]
    old = max(T - W, 0)
    sinks = min(old, S)
    slot = int(state["slots"][i])
    got = []
    for section, (perm, rows) in enumerate(((state["perm_k"], state["k_rows"]), (state["perm_v"], state["v_rows"]))):
        x = torch.empty((T, D), dtype=torch.float64, device=rows.device)
        x[:sinks] = rows[slot, h, W:W + sinks].double()
        if old > sinks:
            x[sinks:old, perm[h]] = _packed64(state, i, h, old - sinks, section)
        x[old:] = rows[slot, h, torch.arange(old, T, device=rows.device) % W].double()
        got.append(x)
    return got


def exact(case, seed):
    """What run() returns, in 64 bits from the definitions, a head of a sequence at a time; None where that takes long."""
    if case["kind"] != "rope" and case["seqs"] * case["kv_heads"] > 512:
        return None
    state = prepare(case, seed)
    if case["kind"] == "rope":
        position = (torch.arange(case["tokens"], device=DEVICE) + case["start"])[None].expand(case["batch"], -1)
        return {"q": _turned64(state["q"], position, case, case["transpose"]),
                "k": _turned64(state["k"], position, case, case["transpose"])}
    total, new = _lengths(case)
    hk, hq, W, S = case["kv_heads"], case["q_heads"], case["window"], case["sinks"]
    if case["kind"] == "read":
        parts = [[torch.stack(x, 1) for x in zip(*[_cached64(state, i, h) for h in range(hk)])] for i in range(len(total))]
        return {"k": torch.cat([p[0] for p in parts]), "v": torch.cat([p[1] for p in parts])}
    if case["kind"] == "append":
        position = torch.cat([torch.arange(t - n, t, device=DEVICE) for t, n in zip(total, new)])
        q = _turned64(state["q"], position, case)
        k, v = _turned64(state["k"], position, case).to(state["k"].dtype).double(), state["v"].double()
        k_rows, v_rows = state["k_rows"].double(), state["v_rows"].double()
        read, at = {"k": [], "v": []}, 0
        for i, (t, n) in enumerate(zip(total, new)):
            slot, before = int(state["slots"][i]), t - n
            for x, rows, perm, name in ((k, k_rows, state["perm_k"], "k"), (v, v_rows, state["perm_v"], "v")):
                first = max(before - W, 0)
                ring = rows[slot, :, torch.arange(first, before, device=DEVICE) % W].transpose(0, 1)
                every = torch.cat((ring, x[at:at + n]))          # tokens first .. t-1
                left = max(t - W, 0) - first
                gone = every[:left]
                stored = _stored64(case, gone, perm)
                kept = max(0, min(S, first + left) - first)
                stored[:kept] = gone[:kept]
                rows[slot, :, W + first:W + first + kept] = gone[:kept].transpose(0, 1)
                # the values as rows of the cache's type
                read[name].append(stored.float().to(TYPES[case["dtype"]]).double())
                rows[slot, :, torch.arange(first + left, t, device=DEVICE) % W] = every[left:].transpose(0, 1)
            at += n
        return {"q": q, "k": torch.cat(read["k"]), "v": torch.cat(read["v"]), "k_rows": k_rows, "v_rows": v_rows}
    R = hq // hk
    out = torch.empty((sum(new), hq, D), dtype=torch.float64, device=DEVICE)
    at = 0
    for i, (t, n) in enumerate(zip(total, new)):
        for h in range(hk):
            k, v = _cached64(state, i, h)
            q = state["q"][at:at + n, h * R:(h + 1) * R].double()
            for x in range(n):
                s = torch.softmax(q[x] @ k[:t - n + x + 1].T / math.sqrt(D), -1)
                out[at + x, h * R:(h + 1) * R] = s @ v[:t - n + x + 1]
        at += n
    return {"out": out}
