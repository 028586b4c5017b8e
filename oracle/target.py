"""Target side of a round: a paged key/value cache, attention over it and
acceptance from given probabilities (Sec. 2.1, Eq. acceptance, Eq. residual).

Plain loops over sequences and pages.  Attention is computed in fp64 from the
stored values; the page operators move values and count; acceptance compares
and divides in fp32, the precision the decision is defined in.
"""
from __future__ import annotations

import numpy as np


class PagedCache:
    """k, v [layers][pages][nkv][page][d]; table [seqs][max_pages] (-1: none); len [seqs]; refs [pages]."""

    def __init__(self, k, v, table, lens, refs):
        self.k, self.v = np.array(k), np.array(v)
        self.table, self.len, self.refs = np.array(table), np.array(lens), np.array(refs)
        self.page = self.k.shape[3]

    def held(self, s):
        return -(-int(self.len[s]) // self.page)

    def usable(self, s):
        """A sequence of the cache, of a length that its row of the table can hold."""
        return 0 <= s < len(self.len) and 0 <= self.len[s] <= self.table.shape[1] * self.page

    def stray(self, s, first=0):
        """Whether one of the sequence's pages, from column `first` on, is none of the pool."""
        return any(not 0 <= pg < len(self.refs) for pg in self.table[s, first:self.held(s)])

    def fork(self, src, dst):
        """-> indices of the pairs that were refused."""
        bad = []
        for i, (s, d) in enumerate(zip(src, dst)):
            if not (self.usable(s) and self.usable(d)) or d in dst[:i] or d in src or self.stray(s) or self.stray(d):
                bad.append(i)
                continue
            self._cut(d, 0)
            n = self.held(s)
            self.table[d, :n] = self.table[s, :n]
            for pg in self.table[s, :n]:
                self.refs[pg] += 1
            self.len[d] = self.len[s]
        return bad

    def _cut(self, s, new_len):
        for col in range(-(-new_len // self.page), self.held(s)):
            self.refs[self.table[s, col]] -= 1
            self.table[s, col] = -1
        self.len[s] = min(self.len[s], new_len)

    def trim(self, seqs, new_len):
        bad = []
        for i, (s, n) in enumerate(zip(seqs, new_len)):
            if not self.usable(s) or n < 0 or s in seqs[:i] or self.stray(s, -(-n // self.page)):
                bad.append(i)
            elif n < self.len[s]:
                self._cut(s, n)
        return bad

    def reserve(self, seqs, add):
        """-> (indices refused, indices left without pages)."""
        bad, short = [], []
        free = [int(x) for x in np.flatnonzero(self.refs == 0)]
        refs0, copies, used = self.refs.copy(), {}, 0
        for i, (s, a) in enumerate(zip(seqs, add)):
            if not self.usable(s) or a < 0 or s in seqs[:i] or self.len[s] + a > self.table.shape[1] * self.page:
                bad.append(i)
                continue
            n = int(self.len[s])
            part = n % self.page
            last = int(self.table[s, self.held(s) - 1]) if part and a else -1
            if part and a and not 0 <= last < len(self.refs):
                bad.append(i)
                continue
            copy = last >= 0 and copies.get(last, 0) < refs0[last] - 1
            if last >= 0:
                copies[last] = copies.get(last, 0) + 1
            need = -(-(n + a) // self.page) - self.held(s) + int(copy)
            used += need
            if used > len(free):
                short.append(i)
                continue
            new = free[used - need:used]
            col = self.held(s)
            if copy:
                pg = new.pop(0)
                self.k[:, pg, :, :part] = self.k[:, last, :, :part]
                self.v[:, pg, :, :part] = self.v[:, last, :, :part]
                self.table[s, col - 1] = pg
                self.refs[pg] = 1
                self.refs[last] -= 1
            for pg in new:
                self.table[s, col] = pg
                self.refs[pg] = 1
                col += 1
            self.len[s] = n + a
        return bad, short

    def write(self, layer, seqs, start, k_new, v_new):
        for i, s in enumerate(seqs):
            if not self.usable(s):
                continue
            for r in range(start[i], start[i + 1]):
                pos = int(self.len[s]) - int(start[i + 1]) + r
                if pos < 0 or not 0 <= self.table[s, pos // self.page] < len(self.refs):
                    continue
                pg, slot = self.table[s, pos // self.page], pos % self.page
                self.k[layer, pg, :, slot], self.v[layer, pg, :, slot] = k_new[r], v_new[r]

    def compact(self):
        live = int((self.refs > 0).sum())
        holes = [x for x in range(live) if self.refs[x] == 0]
        movers = [x for x in range(live, len(self.refs)) if self.refs[x] > 0]
        to = dict(zip(movers, holes))
        for a, b in to.items():
            self.k[:, b], self.v[:, b] = self.k[:, a], self.v[:, a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        for row in self.table:
            row[:] = [to.get(int(pg), pg) for pg in row]
        return live

    def tokens(self, layer, s):
        """(k, v) [len][nkv][d] of a sequence, fp64; a page outside the pool reads as zeros."""
        n, out = int(self.len[s]), []
        for pool in (self.k, self.v):
            rows = []
            for pg in self.table[s, :self.held(s)]:
                x = pool[layer, pg] if 0 <= pg < pool.shape[1] else np.zeros_like(pool[layer, 0])
                rows.append(np.moveaxis(x, 0, 1).astype(np.float64))
            out.append(np.concatenate(rows)[:n] if rows else np.zeros((0,) + pool.shape[2:3] + pool.shape[4:]))
        return out


def cache_attention(cache, layer, q, seqs, start, scale):
    """Rows [start[i], start[i+1]) of q [total][nq][d] are the last tokens of sequence seqs[i] and see
    what is not after them: (out, lse, softmax(..) |V|, the scale of out's rounding errors), fp64.
    Rows that see nothing: 0, -inf."""
    total, nq, d = q.shape
    out, size = np.zeros((total, nq, d)), np.zeros((total, nq, d))
    lse = np.full((total, nq), -np.inf)
    for i, s in enumerate(seqs):
        if not cache.usable(s):
            continue
        k, v = cache.tokens(layer, s)
        rep = nq // k.shape[1]
        rows = start[i + 1] - start[i]
        for r in range(start[i], start[i + 1]):
            n = int(cache.len[s]) - rows + (r - start[i]) + 1
            if n <= 0:
                continue
            for h in range(nq):
                x = scale * (k[:n, h // rep] @ q[r, h].astype(np.float64))
                m = x.max()
                w = np.exp(x - m)
                z = w.sum()
                lse[r, h] = m + np.log(z)
                out[r, h] = w @ v[:n, h // rep] / z
                size[r, h] = w @ np.abs(v[:n, h // rep]) / z
    return out, lse, size


def verify_probs(p, q, y, n, u, e):
    """One request: p [B+1][V], q [B][V] or None, y [B], u [B], e [V] fp32 -> (accepted, next token)."""
    p, u, e = np.float32(p), np.float32(u), np.float32(e)
    V, r = p.shape[1], 0
    while r < n:
        t = int(y[r])
        if not 0 <= t < V:
            break
        qy = np.float32(q[r, t]) if q is not None else np.float32(1)
        if not np.float32(u[r] * qy) < p[r, t]:
            break
        r += 1
    w = p[r].copy()
    if r < n:
        if q is not None:
            w = p[r] - np.float32(q[r])
        elif 0 <= y[r] < V:
            w[y[r]] = 0
        if not (w > 0).any():
            w = p[r]
    with np.errstate(all="ignore"):
        score = np.where(w > 0, w / e, np.float32(-1))
    return r, int(np.argmax(score)) if (w > 0).any() else -1
