"""Plain references of a prompt's pass and its pages: packed attention row by row in 64 bits
(bounds as in model_ref.py), a write's row, and a pool of pages as Python lists."""
import numpy as np

import model_ref as ref
from model_ref import f64


def sequences(starts, N):
    """(first row, end) of each sequence of packed rows."""
    return [(a, b) for a, b in zip(starts[:-1], starts[1:])]


def check_attn(q, k, v, starts, out, lse, softcap=0.0, window=0, scale=None, rows=None, fill=7.0, poisoned=()):
    """out and lse against 64 bits at `rows` (all); rows of no sequence hold `fill`.  poisoned: rows
    whose key or value is not finite: what sees one is not checked but for reaching the output."""
    N, Hq, D = q.shape
    heads = k.shape[1]
    G = Hq // heads
    scale = D ** -0.5 if scale is None else scale
    out, lse = f64(out), None if lse is None else lse.cpu().numpy()
    k, v, q = f64(k), f64(v), f64(q)
    inside = np.zeros(N, bool)
    checked = 0
    for a, b in sequences(starts, N):
        inside[a:b] = True
        for r in range(a, b):
            if rows is not None and r not in rows:
                continue
            lo = max(a, r + 1 - window) if window else a
            if any(lo <= p <= r for p in poisoned):
                continue
            for h in range(Hq):
                kk, vv = k[lo:r + 1, h // G], v[lo:r + 1, h // G]
                _, o, want, tol, spread = ref.attn_row(q[r, h], kk, vv, r - lo, scale, softcap, 0)
                off = np.abs(out[r, h] - o) - ref.out_bound(o, spread, tol)
                assert off.max() <= 0, (r, h, off.max())
                if lse is not None:
                    assert abs(lse[r, h] - want) <= ref.lse_bound(tol, want, r + 1 - lo), (r, h, lse[r, h], want)
                checked += 1
    assert np.all(out[~inside] == fill) and (lse is None or np.all(lse[~inside] == fill))
    return checked


def turned(x, rope, positions, pair_axis, halves):
    """A head's row x fp64 with each pair at its axis' position."""
    r = rope.shape[1]
    at = np.asarray([positions[a] for a in pair_axis])
    t = np.arange(r // 2)
    c, s = rope[at, t], rope[at, r // 2 + t]
    y = x.copy()
    i, j = (t, t + r // 2) if halves else (2 * t, 2 * t + 1)
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    return y


class Pool:
    """The integers of a pool, and what each position of each sequence holds: calls as documented."""

    def __init__(self, seqs, max_pages, num_pages, page_size):
        self.table = np.full((seqs, max_pages), -1, np.int64)
        self.refs = np.zeros(num_pages, np.int64)
        self.ps, self.P = page_size, num_pages

    def is_page(self, x):
        return 0 <= x < self.P

    def lowest(self):
        free = np.flatnonzero(self.refs <= 0)
        return int(free[0]) if len(free) else None

    def take(self, seq, need):
        status, short = [], False
        lists = []
        for i, (s, n) in enumerate(zip(seq, need)):
            pages = -(-max(n, 0) // self.ps)
            if not 0 <= s < len(self.table) or pages > self.table.shape[1] or seq.count(s) > 1:
                lists.append(None)
            else:
                lists.append([p for p in range(pages) if not self.is_page(self.table[s, p])])
        for s, lacks in zip(seq, lists):
            if lacks is None:
                status.append(-1)
                continue
            if lacks and (short or len(lacks) > int((self.refs <= 0).sum())):
                short = True
                status.append(len(lacks))
                continue
            for p in lacks:
                x = self.lowest()
                self.table[s, p], self.refs[x] = x, 1
            status.append(0)
        return status

    def free(self, seq, keep=None):
        for i, s in enumerate(seq):
            if not 0 <= s < len(self.table):
                continue
            first = -(-max(keep[i], 0) // self.ps) if keep is not None else 0
            for p in range(first, self.table.shape[1]):
                if self.is_page(self.table[s, p]):
                    self.refs[self.table[s, p]] -= 1
                self.table[s, p] = -1

    def fork(self, src, dst, lens):
        """Status and the copies (from, to, slots)."""
        good = []
        for i, (s, d, T) in enumerate(zip(src, dst, lens)):
            ok = 0 <= s < len(self.table) and 0 <= d < len(self.table) and d not in src and dst.count(d) == 1 and T >= 0
            last = (T - 1) // self.ps
            ok = ok and (T == 0 or (last < self.table.shape[1] and self.is_page(self.table[s, last])))
            good.append(ok)
        for i, (s, d, T) in enumerate(zip(src, dst, lens)):
            if not good[i]:
                continue
            self.free([d])
            for p in range(max(T - 1, 0) // self.ps):
                x = self.table[s, p]
                if self.is_page(x):
                    self.table[d, p] = x
                    self.refs[x] += 1
        status, copies, short = [], [], False
        for i, (s, d, T) in enumerate(zip(src, dst, lens)):
            if not good[i]:
                status.append(-1)
                continue
            x = self.lowest() if T else None
            if T and x is None:
                short = True
            elif T:
                last = (T - 1) // self.ps
                copies.append((int(self.table[s, last]), x, T - last * self.ps))
                self.table[d, last], self.refs[x] = x, 1
            status.append(-2 if T and x is None else 0)
        for d, st in zip(dst, status):
            if st == -2:
                self.free([d])
        return status, copies

    def compact(self):
        """(map, used, moves): the pool's own numbers change."""
        used = self.refs > 0
        n = int(used.sum())
        holes = [x for x in range(n) if not used[x]]
        high = [x for x in range(n, self.P) if used[x]]
        new = np.where(used, np.arange(self.P), -1)
        new[high] = holes
        refs = np.zeros_like(self.refs)
        refs[new[used]] = self.refs[used]
        self.refs = refs
        named = (self.table >= 0) & (self.table < self.P)
        self.table[named] = new[self.table[named]]
        return new, n, list(zip(high, holes))
