"""float64 oracle of the paged K/V cache, from the definitions.

Rotary pairs are complex numbers times a unit phase; tables are Python lists
changed one row after another; attention is a softmax over the listed tokens.
"""

from __future__ import annotations

import math

import numpy as np

PAGE = 64
OK, FULL, BAD = range(3)


def kv_rope_frequencies(d_rot, base=10000.0, scaling="none", factor=1.0, original=4096.0, beta_fast=32.0,
                        beta_slow=1.0):
    """(angles per position [d_rot/2], magnitude)."""
    half = d_rot // 2
    if scaling == "ntk":
        base = base * factor ** (d_rot / (d_rot - 2))
    plain = np.array([base ** (-2 * i / d_rot) for i in range(half)])
    if scaling == "linear":
        return plain / factor, 1.0
    if scaling != "yarn":
        return plain, 1.0

    def index(turns):  # pair whose angle reaches 2 pi turns at `original`
        return d_rot * math.log(original / (2 * math.pi * turns)) / (2 * math.log(base))

    low, high = max(math.floor(index(beta_fast)), 0), min(math.ceil(index(beta_slow)), d_rot - 1)
    out = np.empty(half)
    for i in range(half):
        ramp = min(max((i - low) / max(high - low, 1e-3), 0.0), 1.0)
        out[i] = plain[i] * (1 - ramp) + plain[i] / factor * ramp
    return out, 0.1 * math.log(factor) + 1.0


def kv_rope(x, pos, freq, interleaved=False, magnitude=1.0, transpose=False):
    """x [..., width] at positions pos (broadcast over the leading dimensions)."""
    x = np.asarray(x, dtype=np.float64)
    n = len(freq)
    pos = np.asarray(pos, dtype=np.float64)
    phase = np.exp(1j * np.multiply.outer(pos, np.asarray(freq)) * (-1 if transpose else 1)) * magnitude
    y = x.copy()
    if interleaved:
        z = (x[..., 0:2 * n:2] + 1j * x[..., 1:2 * n:2]) * phase
        y[..., 0:2 * n:2], y[..., 1:2 * n:2] = z.real, z.imag
    else:
        z = (x[..., :n] + 1j * x[..., n:2 * n]) * phase
        y[..., :n], y[..., n:2 * n] = z.real, z.imag
    return y


def kv_seen(n, sink=0, window=0):
    """Positions of an n-token sequence that a decode attends."""
    return [t for t in range(n) if not window or t < sink or t >= n - window]


def kv_decode_attn(q, k_pages, v_pages, table, length, rows=None, scale=None, sink=0, window=0):
    """(out [B, H, d], lse [B, H]) over pools k [P, Hkv, 64, d], v [P, Hkv, d, 64]."""
    B, H, d = q.shape
    group = H // k_pages.shape[1]
    out, lse = np.zeros((B, H, d)), np.full((B, H), -np.inf)
    scale = 1 / math.sqrt(d) if scale is None else scale
    for b in range(B):
        row = b if rows is None else rows[b]
        at = kv_seen(length[row], sink, window) if row >= 0 else []
        if not at:
            continue
        pages, slots = np.array([table[row][t // PAGE] for t in at]), np.array([t % PAGE for t in at])
        for h in range(H):
            k, v = k_pages[pages, h // group, slots], v_pages[pages, h // group, :, slots]
            s = k @ q[b, h] * scale
            p = np.exp(s - s.max())
            out[b, h] = p @ v / p.sum()
            lse[b, h] = s.max() + math.log(p.sum())
    return out, lse


class KvTables:
    """Tables as lists, changed one row after another; rows of -1 are passed over."""

    def __init__(self, n_seqs, max_pages, n_pages):
        self.table = [[-1] * max_pages for _ in range(n_seqs)]
        self.length = [0] * n_seqs
        self.refs = [0] * n_pages
        self.free = list(range(n_pages - 1, -1, -1))
        self.max_pages, self.n_pages = max_pages, n_pages

    def _bad(self, rows):
        rows = [r for r in rows if r != -1]
        return len(set(rows)) < len(rows) or any(not 0 <= r < len(self.length) for r in rows)

    def reserve(self, rows, add):
        """(status, start, pairs)"""
        none = [-1] * len(rows)
        if self._bad(rows) or any(r != -1 and (a < 0 or self.length[r] + a > PAGE * self.max_pages) for r, a in zip(rows, add)):
            return BAD, none, []
        before = ([list(t) for t in self.table], list(self.length), list(self.refs), list(self.free))
        start, pairs = [], []
        try:
            for r, a in zip(rows, add):
                if r == -1:
                    start.append(-1)
                    continue
                n = self.length[r]
                last = n // PAGE
                if n % PAGE and a and self.refs[self.table[r][last]] > 1:
                    old, new = self.table[r][last], self.free.pop()
                    self.refs[old] -= 1
                    self.refs[new] = 1
                    self.table[r][last] = new
                    pairs.append((old, new))
                for i in range(-(-n // PAGE), -(-(n + a) // PAGE)):
                    self.table[r][i] = self.free.pop()
                    self.refs[self.table[r][i]] = 1
                start.append(n)
                self.length[r] = n + a
        except IndexError:
            self.table, self.length, self.refs, self.free = before
            return FULL, none, []
        return OK, start, pairs

    def fork(self, src, dst):
        pairs = [(s, r) for s, r in zip(src, dst) if r != -1]
        if (self._bad(dst) or any(not 0 <= s < len(self.length) or s in dst for s, _ in pairs)
                or any(self.length[r] for _, r in pairs)):
            return BAD
        for s, r in pairs:
            n = -(-self.length[s] // PAGE)
            self.table[r][:n] = self.table[s][:n]
            self.length[r] = self.length[s]
            for page in self.table[s][:n]:
                self.refs[page] += 1
        return OK

    def free_rows(self, rows):
        if self._bad(rows):
            return BAD
        rows = [r for r in rows if r != -1]
        back = []
        held = [(r, i) for r in rows for i in range(-(-self.length[r] // PAGE))]
        for r, i in held:
            self.refs[self.table[r][i]] -= 1
        for r, i in held:  # a page without holders, where it is met first
            page = self.table[r][i]
            if self.refs[page] == 0 and page not in back:
                back.append(page)
        for r, i in held:
            self.table[r][i] = -1
        for r in rows:
            self.length[r] = 0
        self.free += back[::-1]
        return OK


# ---------------------------------------------------------------------------
# packed batches and shared prompts
# ---------------------------------------------------------------------------

def kv_slots(table, start, n_new, total, n_pages, rows=None, pos0=None):
    """(offset, entry, pos, slot) of packed tokens, one token after another."""
    offset, entry, pos, slot = [0], [-1] * total, [-1] * total, [-1] * total
    t = 0
    for b, n in enumerate(n_new):
        row = b if rows is None else rows[b]
        for i in range(max(0, n)):
            if t == total:
                break
            entry[t] = b
            if start[b] >= 0:
                place, turned = start[b] + i, (start[b] if pos0 is None else pos0[b]) + i
                if 0 <= turned < 2 ** 31:
                    pos[t] = turned
                if 0 <= row < len(table) and place < PAGE * len(table[0]) and 0 <= table[row][place // PAGE] < n_pages:
                    slot[t] = PAGE * table[row][place // PAGE] + place % PAGE
            t += 1
        offset.append(t)
    return offset, entry, pos, slot


def kv_shared_prefix(table, length, n_pages, rows=None, least=1):
    """(lead, shared): runs of neighbours with the same leading pages."""
    rows = list(range(len(table))) if rows is None else rows
    lead, shared, groups = [], [], []

    def held(r):
        return min(length[r], PAGE * len(table[r])) if 0 <= r < len(table) else 0

    for b, r in enumerate(rows):
        c = 0
        if b and held(r) and held(rows[b - 1]):
            x, y = table[r], table[rows[b - 1]]
            c = min(held(r), held(rows[b - 1]))
            if r != rows[b - 1]:
                for i in range(-(-c // PAGE)):
                    if x[i] != y[i] or not 0 <= x[i] < n_pages:
                        c = min(c, PAGE * i)
                        break
        if c >= least:
            groups[-1].append(c)
        else:
            groups.append([b])
    for g in groups:
        lead += [g[0]] * len(g)
        shared += [min(g[1:], default=0)] * len(g)
    return lead, shared


def kv_prefill_seen(p, sink=0, window=0):
    """Places that the token at place p attends."""
    return [n for n in range(p + 1) if not window or n < sink or n > p - window]


def kv_prefill_attn(q, k_pages, v_pages, table, offset, start, rows=None, scale=None, sink=0, window=0):
    """(out [total, H, d], lse [total, H]) of packed tokens; NaN in rows that are no
    entry's, zeros and -inf in those of padding."""
    total, H, d = q.shape
    group = H // k_pages.shape[1]
    out, lse = np.full((total, H, d), np.nan), np.full((total, H), np.nan)
    scale = 1 / math.sqrt(d) if scale is None else scale
    for b in range(len(start)):
        row = b if rows is None else rows[b]
        for t in range(offset[b], offset[b + 1]):
            if row < 0 or start[b] < 0:
                out[t], lse[t] = 0.0, -np.inf
                continue
            at = kv_prefill_seen(start[b] + t - offset[b], sink, window)
            pages, slots = np.array([table[row][n // PAGE] for n in at]), np.array([n % PAGE for n in at])
            for g in range(k_pages.shape[1]):
                k, v = k_pages[pages, g, slots], v_pages[pages, g, :, slots]
                hs = slice(g * group, (g + 1) * group)
                s = q[t, hs] @ k.T * scale
                m = s.max(axis=1, keepdims=True)
                p = np.exp(s - m)
                out[t, hs] = p @ v / p.sum(axis=1, keepdims=True)
                lse[t, hs] = m[:, 0] + np.log(p.sum(axis=1))
    return out, lse
