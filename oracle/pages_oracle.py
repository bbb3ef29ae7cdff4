"""CPU oracle of the latent cache in pages (definitions of include/cca.h, "Cache in pages").

TEST INFRASTRUCTURE ONLY, like cca_oracle.py: plain definitions on Python lists, one loop per index, nothing shared with the CUDA path.

Pins: tests/test_pages_oracle.py.
"""
from __future__ import annotations

import math

import torch

F64 = torch.float64
MISSING, SHORT = 122, 123


class Pool:
    """refs, table and len as lists; k, v bf16 [n_pages, h_k, P, d_h] on the CPU.  Every operation returns the status it would leave."""

    def __init__(self, k, v, refs, table, lens):
        self.k, self.v, self.refs, self.table, self.len = k.clone(), v.clone(), list(refs), [list(r) for r in table], list(lens)
        self.n_pages, _, self.P, _ = k.shape
        self.wide = len(self.table[0])

    @staticmethod
    def of(pages):
        return Pool(*(pages[n].cpu() for n in ("k", "v")), *(pages[n].tolist() for n in ("refs", "table", "len")))

    def page(self, b, i):
        e = self.table[b][i]
        return e if 0 <= e < self.n_pages else None

    def place(self, b, row):
        """(page, place) of a row, or None."""
        if row < 0 or row >= self.wide * self.P:
            return None
        page = self.page(b, row // self.P)
        return None if page is None else (page, row % self.P)

    def append(self, k, v, count=None):
        status = 0
        for b in range(len(self.table)):
            n = k.shape[1] if count is None else min(max(count[b], 0), k.shape[1])
            for i in range(n if self.len[b] >= 0 else 0):
                at = self.place(b, self.len[b] + i)
                if at is None or self.refs[at[0]] != 1:
                    status = MISSING
                else:
                    self.k[at[0], :, at[1]], self.v[at[0], :, at[1]] = k[b, i], v[b, i]
        return status

    def read(self, n, first=None):
        out = torch.zeros(2, len(self.table), n, self.k.shape[1], self.k.shape[3], dtype=torch.bfloat16)
        for b in range(len(self.table)):
            for i in range(n if first is not None or self.len[b] >= 0 else 0):       # (not in use: zeros)
                at = self.place(b, (self.len if first is None else first)[b] + i)
                if at is not None:
                    out[0, b, i], out[1, b, i] = self.k[at[0], :, at[1]], self.v[at[0], :, at[1]]
        return out[0], out[1]

    def reserve(self, n, count=None, first=None):
        status, window = 0, []
        for b in range(len(self.table)):
            m = n if count is None else min(max(count[b], 0), n)
            r = (self.len if first is None else first)[b]
            if m and first is None and r < 0:
                m = 0
            if m and (r < 0 or r + m > self.wide * self.P):
                status, m = MISSING, 0
            window.append(range(r // self.P, (r + m - 1) // self.P + 1) if m else range(0))
        holders = {}
        for b, w in enumerate(window):
            for i in w:
                holders.setdefault(self.page(b, i), []).append(b)
        need = []
        for b, w in enumerate(window):
            for i in w:
                p = self.page(b, i)
                if p is None or (self.refs[p] > 1 and not (len(holders[p]) == self.refs[p] and holders[p][-1] == b)):
                    need.append((b, i, p))
        free = [p for p in range(self.n_pages) if self.refs[p] <= 0]
        if len(need) > len(free):
            return SHORT if status == 0 else status
        for (b, i, p), new in zip(need, free):
            self.table[b][i] = new
            self.refs[new] = 1
            if p is not None:
                self.k[new], self.v[new] = self.k[p], self.v[p]
                self.refs[p] -= 1
        return status

    def let_go(self, page):
        if self.refs[page] <= 0:
            return MISSING
        self.refs[page] -= 1
        return 0

    def fork(self, parent, child):
        status, B, todo = 0, len(self.table), {}
        for p, c in zip(parent, child):
            if not (0 <= p < B and 0 <= c < B):
                status = MISSING
                continue
            if not 0 <= self.len[p] <= self.wide * self.P:
                status = MISSING
                continue
            todo[c] = p if p != c else None
        held = {p: [e if i * self.P < self.len[p] and 0 <= e < self.n_pages else -1 for i, e in enumerate(self.table[p])]
                for p in todo.values() if p is not None}
        rows = {c: (held[p], self.len[p]) for c, p in todo.items() if p is not None}
        for c, (row, _) in rows.items():
            for e in row:
                if e >= 0:
                    self.refs[e] += 1
        for c, (row, n) in rows.items():
            for i in range(self.wide):
                p = self.page(c, i)
                if p is not None:
                    status = self.let_go(p) or status
            self.table[c], self.len[c] = list(row), n
        return status

    def free(self, keep):
        status = 0
        for b, m in enumerate(keep):
            if m < 0:
                continue
            left = min(m, max(self.len[b], 0))
            self.len[b] = left if self.len[b] >= 0 else self.len[b]
            for i in range(-(-left // self.P), self.wide):
                p = self.page(b, i)
                self.table[b][i] = -1
                if p is not None:
                    status = self.let_go(p) or status
        return status

    def compact(self):
        held = [p for p in range(self.n_pages) if self.refs[p] > 0]
        used = len(held)
        place = dict(zip([p for p in held if p >= used], [p for p in range(used) if self.refs[p] <= 0]))
        for p, to in place.items():
            self.k[to], self.v[to] = self.k[p], self.v[p]
            self.refs[to], self.refs[p] = self.refs[p], 0
        self.table = [[place.get(e, e) for e in row] for row in self.table]
        return used

    def rows(self, b, n):
        """(k, v) F64 [h_k, rows, d_h] of the first n rows, those without a page left out."""
        at = [self.place(b, r) for r in range(n)]
        at = [a for a in at if a is not None]
        if not at:
            return torch.zeros(2, self.k.shape[1], 0, self.k.shape[3], dtype=F64)
        page, place = (torch.tensor(x) for x in zip(*at))
        return torch.stack([x[page, :, place].transpose(0, 1).to(F64) for x in (self.k, self.v)])


def attention(q, k, v, g):
    """One sequence: q [h_q, d], k, v F64 [h_k, n, d] -> (o F64 [h_q, d], lse F64 [h_q], p F64 [h_q, n])."""
    hq, d = q.shape
    o, lse, p = torch.zeros(hq, d, dtype=F64), torch.full((hq,), -math.inf, dtype=F64), torch.zeros(hq, k.shape[1], dtype=F64)
    for i in range(hq if k.shape[1] else 0):
        s = (k[i // g] @ q[i].to(F64)) / math.sqrt(d)
        lse[i] = torch.logsumexp(s, 0)
        p[i] = torch.softmax(s, 0)
        o[i] = p[i] @ v[i // g]
    return o, lse, p
