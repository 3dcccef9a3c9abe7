"""A plain paged cache on the host: tokens in lists, rows quantized one by one with Eq. 2's single-rounding fp32 steps,
pages written byte by byte from the format statement, attention in 64 bits, and how far a kernel may be from it."""
from __future__ import annotations

import numpy as np
import torch

D = 128
META_NUMPY = {"f32": np.float32, "f16": np.float16}
META_SIZE = {"f32": 4, "f16": 2, "e4m3": 1}


def stored_pair(x: np.ndarray, meta: str):
    """(values as they read back, bytes) of fp32 scales or zeros in the pair format."""
    if meta == "e4m3":
        t = torch.from_numpy(np.clip(x.astype(np.float32), -448, 448)).to(torch.float8_e4m3fn)
        return t.float().numpy(), t.view(torch.uint8).numpy()
    y = x.astype(META_NUMPY[meta])
    return y.astype(np.float32), y


def quantize(row: np.ndarray, perm, clip, group: int, meta: str):
    """Eq. 2 of one row [D] (fp32 values): codes in reordered order, scale and zero per group, their stored bytes."""
    x = row.astype(np.float32)[perm].reshape(-1, group)
    mn, mx = x.min(1) + np.float32(0), x.max(1) + np.float32(0)
    clip = clip.astype(np.float32)
    lo, hi = clip * mn, clip * mx
    pair = np.stack(((hi - lo) / np.float32(15), lo), -1)
    values, raw = stored_pair(pair, meta)
    scale, zero = values[:, :1], values[:, 1:]
    with np.errstate(divide="ignore"):
        inv = np.where(scale > 0, np.float32(1) / scale, np.float32(0)).astype(np.float32)
    codes = np.clip(np.rint((x - zero) * inv), 0, 15).astype(np.uint8)
    return codes.reshape(D), scale[:, 0], zero[:, 0], np.ascontiguousarray(raw).view(np.uint8).reshape(-1)


def rounded(x: np.ndarray, dtype: torch.dtype) -> np.ndarray:
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(dtype).float().numpy()


class PlainPaged:
    """Sequences by slot; every token's rows are kept as they came and as they are stored."""

    def __init__(self, hk, group, window, page, n_pages, max_seqs, perm_k, perm_v, clip_k, clip_v, sinks=0, meta="f16",
                 dtype=torch.float16, fill=0xAB):
        self.hk, self.group, self.W, self.S, self.P, self.meta, self.dtype = hk, group, window, sinks, page, meta, dtype
        self.ng = D // group
        self.perm, self.clip = (perm_k, perm_v), (clip_k, clip_v)
        self.part = page * (D + 4 * self.ng * META_SIZE[meta])
        self.pages = np.full((n_pages, hk, self.part), fill, np.uint8)
        self.tokens = {}   # slot: [K rows [n][hk][D], V rows]
        self.rows = [np.zeros((max_seqs, hk, window + sinks, D), np.float32) for _ in range(2)]
        self.written = np.zeros((max_seqs, window + sinks), bool)

    def place(self, page, h, te, which, codes, raw):
        at, t = self.pages[page, h], te % self.P
        half, pairs = self.P * D // 2, self.P * self.ng * 2 * META_SIZE[self.meta]
        for p in range(D):
            if which == 0:
                j, g, e = p // 32, p % 32 // 8, p % 8
                nibble = e // 2 if e % 2 == 0 else 4 + e // 2
                byte, high = t * (D // 2) + 4 * (4 * g + j) + nibble // 2, nibble % 2
            else:
                n, m, r = p // 16, p % 16, t % 4
                byte, high = half + t // 4 * 2 * D + 16 * m + 8 * (r // 2) + 4 * (n // 4) + 2 * (r % 2) + n % 4 // 2, n % 2
            at[byte] = (at[byte] & (0x0F if high else 0xF0)) | (int(codes[p]) << (4 if high else 0))
        start = 2 * half + which * pairs + t * len(raw)
        at[start:start + len(raw)] = raw

    def append(self, slot, table, k, v):
        """k, v [n][hk][D] (fp32 values of the cache's type): new tokens of the sequence in `slot`."""
        have = self.tokens.setdefault(slot, [np.zeros((0, self.hk, D), np.float32) for _ in range(2)])
        before = have[0].shape[0]
        for which, x in enumerate((k, v)):
            have[which] = np.concatenate([have[which], np.asarray(x, np.float32)])
        total = have[0].shape[0]
        for a in range(max(before - self.W, 0), max(total - self.W, 0)):
            for which in range(2):
                for h in range(self.hk):
                    row = have[which][a, h]
                    if a < self.S:
                        self.rows[which][slot, h, self.W + a] = row
                    elif 0 <= (page := int(table[(a - self.S) // self.P])) < self.pages.shape[0]:
                        codes, _, _, raw = quantize(row, self.perm[which][h], self.clip[which][h], self.group, self.meta)
                        self.place(page, h, a - self.S, which, codes, raw)
            if a < self.S:
                self.written[slot, self.W + a] = True
        for a in range(max(before, total - self.W), total):
            for which in range(2):
                self.rows[which][slot, :, a % self.W] = have[which][a]
            self.written[slot, a % self.W] = True

    def stored(self, slot, which, h):
        """What attention reads: values [T][D] in channel order, and per packed token (codes, scales, zeros)."""
        x = self.tokens[slot][which][:, h].astype(np.float64).copy()
        parts = {}
        for a in range(self.S, max(x.shape[0] - self.W, 0)):
            codes, scale, zero, _ = quantize(self.tokens[slot][which][a, h], self.perm[which][h], self.clip[which][h],
                                             self.group, self.meta)
            s, z = np.repeat(scale, self.group), np.repeat(zero, self.group)
            parts[a] = (codes, s, z)
            x[a, self.perm[which][h]] = s.astype(np.float64) * codes + z
        return x, parts

    def read(self, slot, first, n):
        """Rows [n][hk][D] of K and V as skvq_paged_read gives them (fp32 values of the cache's type)."""
        out = []
        for which in range(2):
            rows = self.tokens[slot][which]
            got = rows[first:first + n].copy()
            for a in range(first, first + n):
                if self.S <= a < rows.shape[0] - self.W:
                    for h in range(self.hk):
                        codes, scale, zero, _ = quantize(rows[a, h], self.perm[which][h], self.clip[which][h], self.group, self.meta)
                        s, z = np.repeat(scale, self.group), np.repeat(zero, self.group)
                        got[a - first, h, self.perm[which][h]] = rounded(s * codes.astype(np.float32) + z, self.dtype)
            out.append(got)
        return out

    def attend(self, slot, q, scale=None):
        """q [n][Hq][D] (fp32 values), the sequence's last n tokens' queries: (outputs in 64 bits [n][Hq][D], bounds).

        The bound, term by term (fp32 sums: 2^-24 a step; u = half a step of the outputs' type relative to the value):
          outputs     u |out|
          scores      codes enter the matrix core as fp16 subnormals code 2^-20, aligned as 2^-14: 64 code units of 2^-24
                      each; the fp32 sums and products around it 2^-22 of their terms' sizes; a bf16 query brought to
                      fp16's range 2^-25 of its row's largest.  An error d of a token's score moves the output by at most
                      p d |v - out|, and its logarithms' own rounding adds 2^-22 |score|
          weights     weight x scale rounded to fp16: 2^-11 of weight x scale x |code - 7.5|; full rows: 2^-11 of weight x |v|
          sums        the value product's alignment again: 2^-18 of the largest weight x scale per token, 2^-20 of all of it
        """
        n, hq, _ = q.shape
        R = hq // self.hk
        T = self.tokens[slot][0].shape[0]
        sm = 1.0 / np.sqrt(D) if scale is None else scale
        u = torch.finfo(self.dtype).eps / 2
        out, bound = np.zeros((n, hq, D)), np.zeros((n, hq, D))
        for h in range(self.hk):
            k, kp = self.stored(slot, 0, h)
            v, vp = self.stored(slot, 1, h)
            for j in range(n):
                t = T - n + j + 1
                for r in range(R):
                    x = q[j, h * R + r].astype(np.float64)
                    s = k[:t] @ x * sm
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    o = p @ v[:t]
                    d = 2.0 ** -22 * (np.abs(s) + np.abs(k[:t]) @ np.abs(x) * sm)
                    w_err = p[:, None] * np.abs(v[:t]) * 2.0 ** -11
                    top = 0.0
                    for a in kp:
                        if a >= t:
                            continue
                        codes, sc, z = kp[a]
                        xp = np.abs(x[self.perm[0][h]])
                        d[a] += sm * (sc.sum() * 64 * 2.0 ** -24 * xp.max() + 2.0 ** -22 * (sc * codes * xp + np.abs(z) * xp).sum()
                                      + 2.0 ** -25 * xp.max() * (sc * codes).sum())
                        codes, sc, z = vp[a]
                        w_err[a, self.perm[1][h]] = p[a] * sc * (np.abs(codes - 7.5) * 2.0 ** -11 + codes * 2.0 ** -20)
                        top = max(top, p[a] * sc.max())
                    e = (p * d) @ np.abs(v[:t]) + np.abs(o) * (p @ d) + w_err.sum(0) + len(kp) * top * 2.0 ** -18
                    e += 2.0 ** -20 * (p @ np.abs(v[:t]))
                    out[j, h * R + r] = o
                    bound[j, h * R + r] = 1.01 * e + u * (np.abs(o) + e) + 1e-7
        return out, bound
