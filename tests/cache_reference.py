"""The 8-bit cache's definitions in 64 bits, one sequence, token and head after the other (numpy, no library code), and
helpers that lay out test caches.  Code arrays are uint8 bit patterns."""
import math

import numpy as np
import torch

from paper_2411_17686_b200 import binding

E4M3 = np.zeros(256)
for _c in range(256):
    _e, _m = (_c >> 3) & 15, _c & 7
    _v = math.ldexp(_m, -9) if _e == 0 else math.ldexp(8 + _m, _e - 10)
    E4M3[_c] = (math.nan if (_c & 127) == 127 else _v) * (-1 if _c & 128 else 1)
_POS = E4M3[:127]


def to_codes(x):
    """Nearest code, ties to the even one, beyond 448 to 448, NaN to 0x7F (sign aside)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(x), 448.0)
    a = np.where(np.isnan(a), 0.0, a)
    hi = np.clip(np.searchsorted(_POS, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POS[lo], _POS[hi] - a
    pick = np.where(dl < dh, lo, np.where(dl > dh, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.where(np.isnan(x), 127, pick + np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_of(amax):
    s = 2.0 ** -64
    while 448.0 * s < amax:
        s *= 2.0
    return s


class Cache:
    """Host image of a cache; pages of a sequence are taken in a shuffled order."""

    def __init__(self, rng, lengths, page, kv, dim, spare=3, garbage=True, max_pages=None, fill=1.0):
        self.page, self.kv, self.dim, self.lengths = page, kv, dim, list(lengths)
        per = [-(-n // page) for n in lengths]
        n_pages = sum(per) + spare
        order = rng.permutation(n_pages)
        width = max_pages or max(max(per), 1) + 1
        self.table = np.full((len(lengths), width), -7, dtype=np.int32)      # never to be read behind the last page
        at = 0
        for b, p in enumerate(per):
            self.table[b, :p] = order[at:at + p]
            at += p
        self.spare = order[at:]
        shape = (n_pages, kv, page, dim)
        # what no sequence holds is NaN: codes and scales
        self.kc = np.full(shape, 0x7F if garbage else 0, dtype=np.uint8)
        self.vc = np.full(shape, 0xFF if garbage else 0, dtype=np.uint8)
        self.ks = np.full((n_pages, kv), math.nan if garbage else 1.0, dtype=np.float32)
        self.vs = self.ks.copy()
        for b, n in enumerate(lengths):
            if n:
                self.write(b, 0, fill * rng.standard_normal((n, kv, dim)), rng.standard_normal((n, kv, dim)) * 0.5)

    def write(self, b, start, k, v):
        """Append's definition: rows k, v at positions start.. of sequence b."""
        n = k.shape[0]
        P = self.page
        for pi in range(start // P, -(-(start + n) // P) if n else 0):
            lo, hi = max(start, pi * P), min(start + n, (pi + 1) * P)
            page, s0 = self.table[b, pi], lo - pi * P
            for h in range(self.kv):
                x = [k[lo - start:hi - start, h], v[lo - start:hi - start, h]]
                bad = ~(np.isfinite(x[0]).all(1) & np.isfinite(x[1]).all(1))
                for w, codes, scales in ((0, self.kc, self.ks), (1, self.vc, self.vs)):
                    good = np.abs(x[w][~bad])
                    s = scale_of(good.max() if good.size else 0.0)
                    if s0:
                        old = float(scales[page, h])
                        s = max(s, old)
                        if s > old:
                            codes[page, h, :s0] = to_codes(E4M3[codes[page, h, :s0]] * (old / s))
                    scales[page, h] = s
                    c = to_codes(np.where(bad[:, None], 0.0, x[w]) / s)
                    codes[page, h, s0:s0 + hi - lo] = np.where(bad[:, None], 127 if w == 0 else 0, c)

    def tokens(self, b, h, n=None):
        n = self.lengths[b] if n is None else n
        j = np.arange(n)
        pages, slots = self.table[b, j // self.page], j % self.page
        k = E4M3[self.kc[pages, h, slots]] * self.ks[pages, h].astype(np.float64)[:, None]
        v = E4M3[self.vc[pages, h, slots]] * self.vs[pages, h].astype(np.float64)[:, None]
        return k, v, self.vs[pages, h].astype(np.float64)

    def device(self, dev="cuda:0"):
        t = lambda a: torch.from_numpy(a.copy()).to(dev)      # noqa: E731
        return binding.PagedCache(t(self.kc).view(torch.float8_e4m3fn), t(self.vc).view(torch.float8_e4m3fn), t(self.ks), t(self.vs),
                                  t(self.table), t(np.array(self.lengths, dtype=np.int32)))


def visible(n, pos, causal, window, sinks):
    j = np.arange(n)
    see = j <= pos if causal else np.ones(n, dtype=bool)
    return see & ((j > pos - window) | (j < sinks)) if window else see


def attention(cache, q, rows, causal=True, window=0, sinks=0, scale=None):
    """(out, lse, tolerance of out per element, of lse) for rows q [sum(rows), heads, dim], the last ones of each sequence.

    Tolerances, bf16 rows.  A softmax weight (times its page's value scale) is held as two e4m3 terms: each is off by at most
    2^-4 of what it stands for, together 2^-8; the second one's smallest step puts another 2^-22 of the largest weight on
    every token.  A query row is two such terms of the row scaled to between 224 and 448: exact for bf16 elements down to 2^-10
    of the row's largest, below that off by half of the second term's smallest step, 2^-10 where both terms have one scale (many
    rows per sequence), hence by at most 2^-10 / 224 < 2^-17 of the largest element, which moves a score by at most ds and every
    weight by 2 ds (numerator and denominator).  With many rows weights are fp16 (2^-12, smallest step 2^-24 of the largest).  fp32 sums of 128 exact products: 2^-21 of the sum of magnitudes (measured 2^-22), exponentials and the
    other operations a few 2^-22 more.  The result is rounded to half a bf16 step, 2^-8 of it at most.
    fp32 rows: six terms, 2^-24 of the weight or better; the rest as above, and 2^-24 for the result."""
    heads, dim = q.shape[1], q.shape[2]
    scale = dim ** -0.5 if scale is None else scale
    bf16 = q.dtype == torch.bfloat16
    qn = q.double().cpu().numpy()
    out, lse = np.zeros(qn.shape), np.full(qn.shape[:2], -math.inf)
    tol, ltol = np.zeros(qn.shape), np.zeros(qn.shape[:2])
    r0 = 0
    for b, m in enumerate(rows):
        n = cache.lengths[b]
        see = np.array([visible(n, n - m + i, causal, window, sinks) for i in range(m)]).reshape(m, n)
        some = see.any(1)                                # rows that see nothing: zeros, -inf
        for h in range(heads):
            k, v, sv = cache.tokens(b, h // (heads // cache.kv))
            x = qn[r0:r0 + m, h]
            if not some.any():
                continue
            s = np.where(see, x @ k.T * scale, -math.inf)[some]
            on = see[some]
            top = s.max(1, keepdims=True)
            p = np.exp(s - top)
            l = p.sum(1, keepdims=True)
            p /= l
            o = p @ v
            e = top[:, 0] + np.log(l[:, 0])
            size = np.where(on, s, 0.0)
            ds = 2.0 ** -21 * scale * np.where(on, np.abs(x[some]) @ np.abs(k).T, 0.0).max(1) + 2.0 ** -21 * (1 + np.abs(size).max(1))
            if bf16:
                ds += scale * np.abs(x[some]).max(1) * np.where(on, np.abs(k).sum(1)[None], 0.0).max(1) * 2.0 ** -17
            t = (p @ np.abs(v)) * ((2.0 ** -8 if bf16 else 2.0 ** -22) + 2 * ds)[:, None]
            t += (2.0 ** -22 if bf16 else 2.0 ** -27) * (p * sv).max(1)[:, None] * (on @ (np.abs(v) / sv[:, None]))
            t += (2.0 ** -8 if bf16 else 2.0 ** -23) * np.abs(o) + 1e-38
            at = np.nonzero(some)[0] + r0
            out[at, h], lse[at, h], tol[at, h] = o, e, t
            ltol[at, h] = ds + 2.0 ** -22 * (4 + np.abs(e))
        r0 += m
    return out, lse, tol, ltol


def weights(cache, q, lse, rows, n_text, first, count, causal=True, window=0, sinks=0, scale=None):
    """(weights [batch, heads, n_text, count], tolerance): relative 2 ds of the scores, ds as in attention()."""
    heads, dim = q.shape[1], q.shape[2]
    scale = dim ** -0.5 if scale is None else scale
    bf16 = q.dtype == torch.bfloat16
    qn, ln = q.double().cpu().numpy(), lse.double().cpu().numpy()
    out = np.zeros((len(rows), heads, n_text, count))
    tol = np.zeros_like(out)
    r0 = 0
    for b, m in enumerate(rows):
        n = cache.lengths[b]
        for h in range(heads):
            k = cache.tokens(b, h // (heads // cache.kv))[0]
            for t in range(n_text):
                i = m - n_text + t
                if i < 0:
                    continue
                see = np.nonzero(visible(n, n - m + i, causal, window, sinks))[0]
                see = see[(see >= first) & (see < first + count)]
                x = qn[r0 + i, h]
                s = k[see] @ x * scale
                out[b, h, t, see - first] = np.exp(s - ln[r0 + i, h])
                s1 = scale * (np.abs(k[see]) @ np.abs(x))
                ds = 2.0 ** -21 * s1 + 2.0 ** -21 * (2 + np.abs(s) + abs(ln[r0 + i, h]))
                if bf16:
                    ds += scale * np.abs(x).max() * np.abs(k[see]).sum(1) * 2.0 ** -18
                tol[b, h, t, see - first] = out[b, h, t, see - first] * ds * 1.5 + 1e-38
        r0 += m
    return out, tol


def cu(rows, extra=0):
    return torch.tensor(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32), device="cuda:0")
