"""A plain cache in numpy, float64: what the calls of the paged 8-bit cache are defined to do, without blocking, fusion
or any code of the package.  Used by the cache tests only."""
import math

import numpy as np

PAGE = 128


def e4m3_values():
    """The value of each byte, from the definition of the format (no infinities; 0x7f and 0xff are NaN)."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = (1 + m / 8) * 2.0 ** (e - 7) if e else (m / 8) * 2.0 ** -6
        out[c] = (math.nan if c & 127 == 127 else v) * (-1 if c & 128 else 1)
    return out


E4M3 = e4m3_values()
INT8 = np.concatenate([np.arange(128), np.arange(-128, 0)]).astype(np.float64)
LARGEST = {"e4m3": 448.0, "int8": 127.0}


def values(codes, fmt):
    return (E4M3 if fmt == "e4m3" else INT8)[codes]


def encode(x, fmt):
    """Bytes of the codes nearest to x (float64, in units of the scale), ties to the even code."""
    x = np.asarray(x, dtype=np.float64)
    if fmt == "int8":
        y = np.where(np.isnan(x), 0.0, np.clip(x, -127, 127))
        return np.rint(y).astype(np.int8).view(np.uint8)
    grid = E4M3[:127]                       # ascending: 0 .. 448
    a = np.minimum(np.abs(np.where(np.isnan(x), 0.0, x)), 448.0)
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    lo = hi - 1
    up, down = grid[hi] - a, a - grid[lo]
    pick = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    code = (pick + 128 * np.signbit(x)).astype(np.uint8)
    return np.where(np.isnan(x), 0x7f, code).astype(np.uint8)


def exponent(amax, fmt):
    """Smallest e >= -126 with amax <= LARGEST 2^e."""
    e = -126
    if amax > 0:
        e = max(e, math.floor(math.log2(amax / LARGEST[fmt])) - 2)
        while amax > LARGEST[fmt] * 2.0 ** e:
            e += 1
    return e


def pages_of(n):
    return -(-n // PAGE)


class Refused(Exception):
    pass


class RefCache:
    def __init__(self, layers, pages, heads, max_seqs, max_pages, fmt):
        self.fmt, self.layers, self.pages, self.heads = fmt, layers, pages, heads
        self.max_pages, self.max_seqs = max_pages, max_seqs
        self.codes = {x: np.zeros((layers, pages, heads, PAGE, 128), np.uint8) for x in "kv"}
        self.exps = {x: np.zeros((layers, pages, heads), np.int64) for x in "kv"}
        self.table = np.full((max_seqs, max_pages), -1, np.int64)
        self.lens = np.zeros(max_seqs, np.int64)
        self.refs = np.zeros(pages, np.int64)

    def _take(self, n):
        free = np.nonzero(self.refs == 0)[0]
        if len(free) < n:
            raise Refused("no pages")
        return [int(p) for p in free[:n]]

    def reserve(self, ids, n_new):
        pairs = [(s, n) for s, n in zip(ids, n_new) if s >= 0]
        if len({s for s, _ in pairs}) < len(pairs):
            raise Refused("listed twice")
        need = []
        for s, n in pairs:
            if pages_of(self.lens[s] + n) > self.max_pages:
                raise Refused("no room")
            need.append(pages_of(self.lens[s] + n) - pages_of(self.lens[s]))
        got = self._take(sum(need))
        for (s, n), k in zip(pairs, need):
            at = pages_of(self.lens[s])
            for j in range(k):
                self.table[s, at + j] = got.pop(0)
                self.refs[self.table[s, at + j]] = 1
            self.lens[s] += n

    def append(self, k, v, ids, cu, layer=0):
        for i, s in enumerate(ids):
            if s < 0:
                continue
            n = cu[i + 1] - cu[i]
            pos = self.lens[s] - n
            t = cu[i]
            while pos < self.lens[s]:
                held = pos % PAGE
                rows = min(PAGE - held, self.lens[s] - pos)
                page = self.table[s, pos // PAGE]
                assert self.refs[page] == 1
                for name, x in (("k", k), ("v", v)):
                    for h in range(self.heads):
                        y = np.asarray(x[t:t + rows, h], np.float64)
                        fin = np.abs(y[np.isfinite(y)])
                        e = exponent(fin.max() if fin.size else 0.0, self.fmt)
                        codes = self.codes[name][layer, page, h]
                        if held:
                            old = self.exps[name][layer, page, h]
                            e = max(e, old)
                            codes[:held] = encode(values(codes[:held], self.fmt) * 2.0 ** (old - e), self.fmt)
                        with np.errstate(invalid="ignore"):
                            codes[held:held + rows] = encode(y * 2.0 ** -e, self.fmt)
                        self.exps[name][layer, page, h] = e
                t, pos = t + rows, pos + rows

    def fork(self, src, dst, n_tokens=None, share=True):
        todo = []
        for i, (a, b) in enumerate(zip(src, dst)):
            if a < 0 or b < 0:
                continue
            n = self.lens[a] if n_tokens is None else n_tokens[i]
            if self.lens[b] != 0 or not 0 <= n <= self.lens[a] or sum(d == b and c >= 0 for c, d in zip(src, dst)) > 1:
                raise Refused("bad fork")
            todo.append((a, b, int(n)))
        own = [pages_of(n) - (n // PAGE if share else 0) for _, _, n in todo]
        got = self._take(sum(own))
        for a, b, n in todo:
            for j in range(pages_of(n)):
                p = self.table[a, j]
                if share and j < n // PAGE:
                    self.refs[p] += 1
                    self.table[b, j] = p
                else:
                    q = got.pop(0)
                    self.refs[q] = 1
                    self.table[b, j] = q
                    rows = min(PAGE, n - j * PAGE)
                    for x in "kv":
                        self.codes[x][:, q, :, :rows] = self.codes[x][:, p, :, :rows]
                        self.exps[x][:, q] = self.exps[x][:, p]
            self.lens[b] = n

    def free(self, ids):
        for s in ids:
            if s < 0:
                continue
            for j in range(pages_of(self.lens[s])):
                self.refs[self.table[s, j]] -= 1
                self.table[s, j] = -1
            self.lens[s] = 0

    def compact(self):
        left = int((self.refs > 0).sum())
        src = [int(p) for p in np.nonzero(self.refs)[0] if p >= left]
        dst = [int(p) for p in np.nonzero(self.refs == 0)[0] if p < left]
        for a, b in zip(src, dst):
            for x in "kv":
                self.codes[x][:, b] = self.codes[x][:, a]
                self.exps[x][:, b] = self.exps[x][:, a]
            self.refs[b], self.refs[a] = self.refs[a], 0
            for s in range(self.max_seqs):
                row = self.table[s, :pages_of(self.lens[s])]
                row[row == a] = b
        return left

    def states(self, x, s, layer=0):
        """K or V of a sequence as stored, float64 [len, heads, 128]."""
        n = self.lens[s]
        if n == 0:
            return np.zeros((0, self.heads, 128))
        pages = self.table[s, :pages_of(n)]
        y = values(self.codes[x][layer, pages], self.fmt) * (2.0 ** self.exps[x][layer, pages])[..., None, None]
        return y.transpose(0, 2, 1, 3).reshape(-1, self.heads, 128)[:n]

    def attention(self, q, ids, cu, layer=0, scale=None):
        return attention(lambda s: (self.states("k", s, layer), self.states("v", s, layer)), q, ids, cu, scale)


def attention(states, q, ids, cu, scale=None):
    """(o, lse, slack, dot) in float64; rows of no item are NaN.  slack and dot go into the tolerances below."""
    q = np.asarray(q, np.float64)
    n, hq, _ = q.shape
    scale = 1 / math.sqrt(128) if scale is None else scale
    o, lse = np.full(q.shape, np.nan), np.full((hq, n), np.nan)
    slack, dots = np.full(q.shape, np.nan), np.zeros((hq, n))
    for i, s in enumerate(ids):
        if s < 0:
            continue
        k, v = states(s)
        new = cu[i + 1] - cu[i]
        for t in range(cu[i], cu[i + 1]):
            seen = len(k) - new + (t - cu[i]) + 1
            for h in range(hq):
                if seen <= 0:
                    o[t, h], lse[h, t], slack[t, h] = 0.0, -np.inf, 0.0
                    continue
                kh, vh = k[:seen, h * k.shape[1] // hq], v[:seen, h * k.shape[1] // hq]
                x = kh @ q[t, h] * scale
                top = x.max()
                p = np.exp(x - top)
                lse[h, t] = top + math.log(p.sum())
                p /= p.sum()
                o[t, h] = p @ vh
                # error budget of a row
                dot = (np.abs(kh) @ np.abs(q[t, h])).max() * scale
                slack[t, h], dots[h, t] = (p @ np.abs(vh)) * (1.0 + dot), dot
    return o, lse, slack, dots


def tolerance(o, slack, p_eps, terms):
    """How far an output may be off, element by element.  bf16 output: 2^-8 of the value.  With A = sum p |v|: each
    weight is rounded once (relative p_eps) and its exponential and the fp32 sums are off by at most terms 2^-23
    relative; a logit is a fp32 sum of 128 exact products and off by at most 128 2^-23 of sum |q k| scale (tensor cores
    may truncate), which moves a normalised weight by at most twice that.  slack = A (1 + max sum |q k| scale)."""
    return 2.0 ** -8 * np.abs(o) + slack * (p_eps + 2.0 ** -23 * (terms + 2 * 128)) + 1e-30


def lse_tolerance(lse, dots, terms):
    """The logits' error (dots = max sum |q k| scale, see tolerance) and the exponentials' and sums', absolute."""
    return 2.0 ** -23 * (128 * dots + terms + 4 * np.abs(lse))
