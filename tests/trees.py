"""Plain forms of trees of drafted tokens over the paged cache and of page tables, for the tests: loops, 64 bits, one statement per definition."""
from __future__ import annotations

import math

import torch

import paged
from paged import PAGE


def random_parents(n, gen, roots=0.1, back=8, order=None):
    """the token that each of n tokens continues, -1: the context; order: "any": children may stand in front of their parents"""
    p = [-1 if i == 0 or float(torch.rand((), generator=gen)) < roots else i - 1 - int(torch.randint(0, min(i, back), (1,), generator=gen)) for i in range(n)]
    if order == "any":
        to = torch.randperm(n, generator=gen).tolist()
        q = [0] * n
        for i in range(n):
            q[to[i]] = -1 if p[i] < 0 else to[p[i]]
        p = q
    return p


def ancestors(parents):
    """for each token the set of it and what leads to it"""
    out = []
    for i in range(len(parents)):
        s, j = set(), i
        while 0 <= j < len(parents) and j not in s:
            s.add(j)
            j = parents[j]
        out.append(s)
    return out


def to_words(sets, words):
    """int32 bit patterns [tokens, words]"""
    rows = [[sum(1 << j % 32 for j in s if j // 32 == w) for w in range(words)] for s in sets]
    return torch.tensor([[x - (1 << 32) if x >> 31 else x for x in r] for r in rows], dtype=torch.int32).reshape(len(sets), words)


def to_sets(words, n):
    return [{j for j in range(n) if int(r[j // 32]) >> (j % 32) & 1} for r in words.tolist()]


def attention(q, k, v, scales, table, news, ctxs, sets, softmax_scale, lists=None, dense_below=0):
    """(out [T, hq, d], lse [T, hq], sum of weights times |v|) in float64.  sets: for each token the drafted tokens that it attends to; lists [B][hkv]: blocks"""
    T, hq, d = q.shape
    hkv = k.shape[1]
    G = hq // hkv
    out = torch.zeros((T, hq, d), dtype=torch.float64, device=q.device)
    mass, lse = torch.zeros_like(out), torch.full((T, hq), -math.inf, dtype=torch.float64, device=q.device)
    t0 = 0
    for b, (n, L) in enumerate(zip(news, ctxs)):
        for h in range(hkv if n else 0):
            K, there = paged.rows_of(k, scales and scales[0], table, b, L, h)
            V, _ = paged.rows_of(v, scales and scales[1], table, b, L, h)
            front = torch.ones(L - n, dtype=torch.bool)
            if lists is not None and L >= dense_below:
                front[:] = False
                for j in lists[b][h]:
                    if j >= 0:
                        front[j * PAGE:(j + 1) * PAGE] = True
            for i in range(n):
                own = torch.zeros(n, dtype=torch.bool)
                own[sorted(sets[t0 + i])] = True
                u = torch.nonzero(torch.cat([front, own]).to(q.device) & there)[:, 0]
                if len(u) == 0:
                    continue
                z = q[t0 + i, h * G:(h + 1) * G].double() @ K[u].T * softmax_scale
                p = torch.softmax(z, -1)
                out[t0 + i, h * G:(h + 1) * G] = p @ V[u]
                mass[t0 + i, h * G:(h + 1) * G] = p @ V[u].abs()
                lse[t0 + i, h * G:(h + 1) * G] = torch.logsumexp(z, -1)
        t0 += n
    return out, lse, mass


def accept(k, v, scales, table, news, ctxs, paths):
    """The pages after the rows of paths[b] have been brought together, in place; returns the new lengths.  scales: (k_scale, v_scale) or None"""
    lens = []
    for b, (n, L) in enumerate(zip(news, ctxs)):
        path = []
        for j in paths[b]:
            if not (path[-1] if path else -1) < j < n:
                break
            path.append(j)
        start = L - n
        lens.append(start + len(path))
        at = lambda t: (int(table[b, t // PAGE]), t % PAGE)  # noqa: E731
        for pool, scale in ((k, scales and scales[0]), (v, scales and scales[1])):
            was_pool, was_scale = pool.clone(), None if scale is None else scale.clone()
            raw, was_raw = (x.view(torch.uint8) if scale is not None else x for x in (pool, was_pool))
            good = lambda t: 0 <= at(t)[0] < pool.shape[0]  # noqa: E731
            moved = [(start + i, start + j) for i, j in enumerate(path) if i != j and good(start + i) and good(start + j)]
            for block in sorted({t // PAGE for t, _ in moved}):
                page = int(table[b, block])
                rows = [(t % PAGE, at(f)) for t, f in moved if t // PAGE == block]
                for h in range(pool.shape[1]):
                    if scale is None:
                        for to, (fp, fr) in rows:
                            raw[page, h, to] = was_raw[fp, h, fr]
                        continue
                    vals = [was_pool[fp, h, fr].double() * was_scale[fp, h].double() for _, (fp, fr) in rows]
                    mag = torch.stack(vals).abs()
                    top = float(mag[torch.isfinite(mag)].max()) if torch.isfinite(mag).any() else 0.0
                    s, old = max(paged.scale_for(top), float(was_scale[page, h])), float(was_scale[page, h])
                    if s != old:
                        raw[page, h] = paged.to_codes(was_pool[page, h].double() * (old / s)).view(torch.uint8)
                        scale[page, h] = s
                    for (to, (fp, fr)), x in zip(rows, vals):
                        same = float(was_scale[fp, h]) == s
                        raw[page, h, to] = was_raw[fp, h, fr] if same else paged.to_codes(x / s).view(torch.uint8)
    return lens


class Pool:
    """page tables as lists"""

    def __init__(self, refs, table):
        self.refs, self.table = list(refs), [list(r) for r in table]

    @staticmethod
    def blocks(n):
        return (n + PAGE - 1) // PAGE

    def give(self, row, block):
        page = self.table[row][block]
        if 0 <= page < len(self.refs):
            self.refs[page] -= 1
        self.table[row][block] = -1

    def take(self):
        for g, r in enumerate(self.refs):
            if r <= 0:
                self.refs[g] = 1
                return g
        return -1

    def resize(self, old, new):
        short = 0
        for b, (x, y) in enumerate(zip(old, new)):
            for j in range(self.blocks(y), self.blocks(x)):
                self.give(b, j)
        for b, (x, y) in enumerate(zip(old, new)):
            for j in range(self.blocks(x), self.blocks(y)):
                self.table[b][j] = self.take()
                short += self.table[b][j] < 0
        return short

    def fork(self, src, dst, tokens, old):
        copies, short = [], 0
        for d, o in zip(dst, old):
            for j in range(self.blocks(o)):
                self.give(d, j)
        for s, d, n in zip(src, dst, tokens):
            for j in range(n // PAGE):
                page = self.table[s][j]
                good = 0 <= page < len(self.refs)
                self.table[d][j] = page if good else -1
                if good:
                    self.refs[page] += 1
        for s, d, n in zip(src, dst, tokens):
            pair = [-1, -1]
            if n % PAGE:
                page = self.table[s][n // PAGE]
                self.table[d][n // PAGE] = -1
                if 0 <= page < len(self.refs):
                    new = self.take()
                    self.table[d][n // PAGE] = new
                    short += new < 0
                    if new >= 0:
                        pair = [page, new]
            copies.append(pair)
        return copies, short

    def compact(self, lens):
        live = sum(r > 0 for r in self.refs)
        frm = [g for g, r in enumerate(self.refs) if r > 0 and g >= live]
        to = [g for g, r in enumerate(self.refs) if r <= 0 and g < live]
        place = dict(zip(frm, to))
        refs = [0] * len(self.refs)
        for g, r in enumerate(self.refs):
            if r > 0:
                refs[place.get(g, g)] = r
        for b, n in enumerate(lens):
            for j, page in enumerate(self.table[b]):
                self.table[b][j] = place.get(page, page) if j < self.blocks(n) and 0 <= page < len(refs) else -1
        self.refs = refs
        return list(map(list, zip(frm, to))), live
