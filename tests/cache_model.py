"""The paged key/value cache written out in plain numpy and 64 bits: one request, one position, one element after the other.
Shares no code with the library; the tests compare the GPU calls with it."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 16
BAD, NO_PAGES = 1, 4


def e4m3_value(code: np.ndarray) -> np.ndarray:
    code = np.asarray(code, dtype=np.int64)
    expo, mant = (code >> 3) & 15, code & 7
    v = np.where(expo == 0, mant * 2.0 ** -9, (8 + mant) * 2.0 ** (expo - 10.0))
    v = np.where((code & 127) == 127, np.nan, v)
    return np.where(code >= 128, -v, v)


def e4m3_round(x: np.ndarray) -> np.ndarray:
    """Nearest e4m3 value, ties to the even mantissa, at most 448; NaN for what is not finite."""
    x = np.asarray(x, dtype=np.float64)
    mag = np.minimum(np.where(np.isfinite(x), np.abs(x), 0.0), 448.0)
    step = 2.0 ** (np.floor(np.log2(np.maximum(mag, 2.0 ** -6))) - 3)
    return np.where(np.isfinite(x), np.copysign(np.rint(mag / step) * step, x), np.nan)


def block_exponent(x: np.ndarray) -> int:
    amax = float(np.max(np.abs(x[np.isfinite(x)]), initial=0.0))
    if amax == 0.0:
        return -100
    m, e = math.frexp(amax)                  # amax = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    return min(max(e - 9 if m <= 0.875 else e - 8, -100), 119)


class Rows:
    """Cached values of one sequence and head matrix ([position, heads, d]) as storing in order leaves them."""

    def __init__(self, heads: int, d: int):
        self.heads, self.d = heads, d
        self.values = np.zeros((0, heads, d))
        self.exps: dict = {}                 # (block, head) -> exponent

    def store(self, first: int, x: np.ndarray) -> None:
        """x [n, heads, d]: positions first .. first + n - 1 (first <= what is stored)."""
        n = len(x)
        v = np.concatenate([self.values[:first], np.zeros((n, self.heads, self.d))])
        for b in range(first // BLOCK, (first + n - 1) // BLOCK + 1 if n else 0):
            lo, hi = max(first, b * BLOCK), min(first + n, (b + 1) * BLOCK)
            for h in range(self.heads):
                new = x[lo - first:hi - first, h]
                e = block_exponent(new)
                if first > b * BLOCK:
                    e = max(e, self.exps[b, h])
                    old = v[b * BLOCK:first, h]
                    v[b * BLOCK:first, h] = e4m3_round(old * 2.0 ** -e) * 2.0 ** e
                self.exps[b, h] = e
                v[lo:hi, h] = e4m3_round(new * 2.0 ** -e) * 2.0 ** e
        self.values = v


def attention(q: np.ndarray, K: np.ndarray, V: np.ndarray, first: int, scale: float, usable=None):
    """q [n, heads, d] at positions first ..; K, V [positions, kv heads, d].  Returns (out, sum of p |v|, largest error factor of the
    scores in fp32) with out zero where nothing is seen.  usable: truth value per position."""
    n, heads, d = q.shape
    G = heads // K.shape[1]
    out, mag, slack = np.zeros((n, heads, d)), np.zeros((n, heads, d)), np.zeros((n, heads, 1))
    for i in range(n):
        seen = np.arange(len(K)) <= first + i
        if usable is not None:
            seen &= usable
        if not seen.any():
            continue
        for h in range(heads):
            k, v = K[seen, h // G], V[seen, h // G]
            s = scale * (k @ q[i, h])
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h], mag[i, h] = p @ v, p @ np.abs(v)
            slack[i, h] = abs(scale) * np.max(np.abs(k) @ np.abs(q[i, h]))
    return out, mag, slack


class Pages:
    """Table, lengths, reference counts, and the contents of every pool's pages as one number each."""

    def __init__(self, n_pages: int, n_slots: int, max_pages: int, page_tokens: int):
        self.T, self.max_pages = page_tokens, max_pages
        self.table = np.full((n_slots, max_pages), -1, np.int64)
        self.lens, self.refs = np.zeros(n_slots, np.int64), np.zeros(n_pages, np.int64)
        self.content = np.arange(n_pages)
        self.error = 0

    def _held(self, n: int) -> int:
        return -(-n // self.T)

    def _serve(self, wants):
        """wants: per entry the number of pages, or None for one that cannot be used.  Pages per entry; None behind the first that does not fit."""
        free = [p for p in range(len(self.refs)) if self.refs[p] == 0]
        got, full = [], False
        for w in wants:
            if w is None:
                self.error |= BAD
                got.append(None)
                continue
            full = full or w > len(free)
            if full:
                self.error |= NO_PAGES
                got.append(None)
                continue
            got.append(free[:w])
            free = free[w:]
        return got

    def reserve(self, slots, add):
        wants, seen = [], set()
        for s, a in zip(slots, add):
            ok = 0 <= s < len(self.lens) and s not in seen and a >= 0 and self.lens[s] + a <= self.max_pages * self.T
            seen.add(s)
            wants.append(self._held(self.lens[s] + a) - self._held(self.lens[s]) if ok else None)
        for s, a, got in zip(slots, add, self._serve(wants)):
            if got is not None:
                h = self._held(self.lens[s])
                self.table[s, h:h + len(got)] = got
                self.refs[got] = 1
                self.lens[s] += a

    def fork(self, src, dst, keep=None):
        lens = self.lens.copy()
        keep = [lens[s] if 0 <= s < len(lens) else 0 for s in src] if keep is None else keep
        wants, seen = [], set()
        for s, t, k in zip(src, dst, keep):
            ok = 0 <= s < len(lens) and 0 <= t < len(lens) and t not in seen and lens[t] == 0 and 0 <= k <= lens[s]
            seen.add(t)
            wants.append(int(k % self.T != 0) if ok else None)
        table = self.table.copy()
        for s, t, k, got in zip(src, dst, keep, self._serve(wants)):
            if got is None:
                continue
            full = k // self.T
            self.table[t, :full] = table[s, :full]
            np.add.at(self.refs, table[s, :full], 1)
            if got:
                self.table[t, full] = got[0]
                self.refs[got[0]] = 1
                self.content[got[0]] = self.content[table[s, full]]
            self.lens[t] = k

    def free(self, slots):
        for s in slots:
            if not 0 <= s < len(self.lens):
                self.error |= BAD
                continue
            h = self._held(self.lens[s])
            np.add.at(self.refs, self.table[s, :h], -1)
            self.table[s, :h] = -1
            self.lens[s] = 0

    def compact(self) -> int:
        live = [p for p in range(len(self.refs)) if self.refs[p] > 0]
        n = len(live)
        src = [p for p in live if p >= n]
        dst = [p for p in range(n) if self.refs[p] == 0]
        to = dict(zip(src, dst))
        for a, b in to.items():
            self.refs[b], self.refs[a], self.content[b] = self.refs[a], 0, self.content[a]
        for s in range(len(self.lens)):
            for j in range(self._held(self.lens[s])):
                self.table[s, j] = to.get(self.table[s, j], self.table[s, j])
        return n
