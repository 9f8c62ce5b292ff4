"""Plain definitions of the paged-cache operations and of the attention over a cache, one request after another and
in 64 bits; nothing of the library is used."""
import math

import torch


class Pool:
    """Tables as lists, rows of the cache as (layer, page, offset) copies."""

    def __init__(self, k, v, ref, table, length):
        self.k, self.v = k.cpu().clone(), v.cpu().clone()
        self.ref, self.table, self.length = ref.tolist(), table.tolist(), length.tolist()
        self.page = k.shape[2]
        self.n_free = None

    def begin(self):
        self.free = [p for p, x in enumerate(self.ref) if x == 0]
        self.n_free, self.asked = len(self.free), 0

    def grant(self, need):
        self.asked += need
        return need == 0 or self.asked <= self.n_free

    def take(self, s, c):
        p = self.free.pop(0)
        self.table[s][c] = p
        self.ref[p] += 1
        return p

    def release(self, s):
        for p in self.table[s]:
            if p >= 0:
                self.ref[p] -= 1
        self.table[s], self.length[s] = [-1] * len(self.table[s]), 0

    def fork(self, src, dst, keep=None):
        self.begin()
        old_table, old_len, old_ref = [list(r) for r in self.table], list(self.length), list(self.ref)
        named, ok, moves = {}, [], []
        for i, d in enumerate(dst):
            named.setdefault(d, i)
        for i, (a, d) in enumerate(zip(src, dst)):
            n = len(self.table)
            if not (0 <= a < n and 0 <= d < n) or named[d] != i or (a != d and a in named):
                ok.append(0)
                continue
            tokens = old_len[a] if keep is None else keep[i]
            if not 0 <= tokens <= old_len[a]:
                ok.append(0)
                continue
            tail, full = tokens % self.page, tokens // self.page
            own = a == d and tail and old_ref[old_table[a][full]] <= 1
            if not self.grant(int(tail > 0 and not own)):
                ok.append(0)
                continue
            ok.append(1)
            row = old_table[a][:full + (1 if own else 0)]
            for p in row:
                self.ref[p] += 1
            fresh = None
            if tail and not own:
                fresh = self.free.pop(0)
                self.ref[fresh] += 1
                moves.append((fresh, old_table[a][full], tail))
                row = row + [fresh]
            self.release(d)
            self.table[d][:len(row)], self.length[d] = row, tokens
        for to, at, tail in moves:
            self.k[:, to, :tail], self.v[:, to, :tail] = self.k[:, at, :tail].clone(), self.v[:, at, :tail].clone()
        return ok

    def drop(self, seqs):
        for s in dict.fromkeys(seqs):
            if 0 <= s < len(self.table):
                self.release(s)

    def grow(self, seqs, counts):
        self.begin()
        ok, seen = [], set()
        for s, more in zip(seqs, counts):
            bad = not 0 <= s < len(self.table) or s in seen or more < 0
            if not bad:
                seen.add(s)
                bad = self.length[s] + more > len(self.table[s]) * self.page
            if bad:
                ok.append(0)
                continue
            have, want = -(-self.length[s] // self.page), -(-(self.length[s] + more) // self.page)
            if not self.grant(want - have):
                ok.append(0)
                continue
            ok.append(1)
            for c in range(have, want):
                self.take(s, c)
            self.length[s] += more
        return ok

    def write(self, layer, seqs, cu, k, v, rows=None, ok=None):
        for i, s in enumerate(seqs):
            for t in range(cu[i], cu[i + 1]):
                if ok is None or ok[i]:
                    at = self.length[s] - (cu[i + 1] - t)
                    p, row = self.table[s][at // self.page], t if rows is None else rows[t]
                    self.k[layer, p, at % self.page], self.v[layer, p, at % self.page] = k[row], v[row]

    def copy(self, other, src, dst):
        self.begin()
        ok, seen = [], set()
        for a, d in zip(src, dst):
            if not (0 <= a < len(other.table) and 0 <= d < len(self.table)) or d in seen:
                ok.append(0)
                continue
            seen.add(d)
            tokens = other.length[a]
            if tokens > len(self.table[d]) * self.page or not self.grant(-(-tokens // self.page)):
                ok.append(0)
                continue
            ok.append(1)
            self.release(d)
            for c in range(-(-tokens // self.page)):
                self.take(d, c)
            self.length[d] = tokens
            for t in range(tokens):
                p, q = self.table[d][t // self.page], other.table[a][t // other.page]
                self.k[:, p, t % self.page], self.v[:, p, t % self.page] = other.k[:, q, t % other.page], other.v[:, q, t % other.page]
        return ok

    def compact(self):
        used = [p for p, x in enumerate(self.ref) if x]
        goes = [p if self.ref[p] else -1 for p in range(len(self.ref))]
        holes = [p for p in range(len(used)) if not self.ref[p]]
        for p, to in zip([p for p in used if p >= len(used)], holes):
            goes[p] = to
            self.ref[to], self.ref[p] = self.ref[p], 0
            self.k[:, to], self.v[:, to] = self.k[:, p].clone(), self.v[:, p].clone()
        self.table = [[goes[p] if p >= 0 else -1 for p in row] for row in self.table]
        return goes

    def rows(self, layer, s):
        n = self.length[s]
        at = [(self.table[s][t // self.page], t % self.page) for t in range(n)]
        if not at:
            return self.k[layer, 0, :0], self.v[layer, 0, :0]
        p, o = zip(*at)
        return self.k[layer, list(p), list(o)], self.v[layer, list(p), list(o)]


def attend(q, k, v, mask, scale):
    """q [rows, heads, dim], k and v [keys, kv heads, dim], mask [rows, keys], all in 64 bits.  Returns the result, the
    logarithm of the sums, the weighted mean of |v|, the largest scale * sum |q||k| and the largest |v| seen."""
    rows, heads, dim = q.shape
    out, mean = torch.zeros(rows, heads, dim, dtype=torch.float64), torch.zeros(rows, heads, dim, dtype=torch.float64)
    log = torch.full((rows, heads), -math.inf, dtype=torch.float64)
    size = 0.0
    for h in range(heads):
        g = h * k.shape[1] // heads
        for r in range(rows):
            seen = mask[r].nonzero()[:, 0]
            if not len(seen):
                continue
            kk, vv = k[seen, g], v[seen, g]
            x = scale * (kk @ q[r, h])
            log[r, h] = torch.logsumexp(x, 0)
            w = torch.exp(x - log[r, h])
            out[r, h] = (w[:, None] * vv).sum(0)
            mean[r, h] = (w[:, None] * vv.abs()).sum(0)
            parts = scale * (kk.abs() @ q[r, h].abs())
            size = max(size, float(parts[torch.isfinite(parts)].max()) if torch.isfinite(parts).any() else 0.0)
    return out, log, mean, size


def bounds(dtype, dim, keys, out, log, mean, size, v_max):
    """How far results may be from the definition.  A score is a sum of `dim` products in 24 bits, each addition off by
    2^-23 of the partial sum at most (the matrix unit may cut instead of round): (dim + 8) 2^-23 size, and with it the exponent; exp2 and the scaling add
    2^-21.  A weight is rounded to the type (half a step), the sums over the keys are in 24 bits, the result is rounded
    once more.  float16 has steps of 2^-24 below 2^-14: each weight, at most 1 beside a sum of at least 1 where the
    largest weight is 1, is off by 2^-25 at most there."""
    half = torch.finfo(dtype).eps / 2
    delta = (dim + 8) * 2.0 ** -23 * size + 2.0 ** -21 + (keys / 16 + 64) * 2.0 ** -23
    tol = half * out.abs() * 1.01 + (half + 2.5 * delta) * mean * 1.01
    if dtype == torch.float16:
        tol = tol + keys * 2.0 ** -25 * v_max + 2.0 ** -25
    return tol + 1e-30, delta + 2.0 ** -22 * log.abs().nan_to_num(posinf=0.0) + 2.0 ** -22


def window_mask(length, num, window, sinks):
    p = torch.arange(length - num, length)[:, None]
    j = torch.arange(length)
    return (j <= p) & ((j > p - window) | (j < sinks))


def tree_mask(length, parents):
    t = len(parents)
    mask = torch.zeros(t, length + t, dtype=torch.bool)
    for r in range(t):
        a, chain = r, []
        while a >= 0:
            chain.append(a)
            p = parents[a]
            a = p if -2 <= p < a else -2
        if a == -1:
            mask[r, :length] = True
            mask[r, [length + c for c in chain]] = True
    return mask
