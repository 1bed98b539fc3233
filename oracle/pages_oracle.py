"""Reference of the paged cache (numpy, integers exact, attention in float64): what the calls leave in table, lengths and
counts, where rows lie, and attention over a slot's tokens.  Written from the definitions, slot by slot."""
from __future__ import annotations

import numpy as np


class OutOfPages(Exception):
    def __init__(self, missing: int):
        super().__init__(f"{missing} pages missing")
        self.missing = missing


class Pages:
    """Pools k, v: arrays [n_layers][n_pages][H_k][page][d] of any element type."""

    def __init__(self, k, v, max_seqs: int, max_pages: int):
        self.k, self.v = k, v
        self.page = k.shape[3]
        self.table = np.zeros((max_seqs, max_pages), dtype=np.int64)
        self.len = np.zeros(max_seqs, dtype=np.int64)
        self.refs = np.zeros(k.shape[1], dtype=np.int64)

    def pages(self, slot: int):
        return [int(x) for x in self.table[slot, :-(-int(self.len[slot]) // self.page)]]

    def reserve(self, want) -> None:
        """Lowest free pages, in the order of slots and positions; a shared last page that is not full is copied.  Pages
        count as they stand before the call."""
        before = self.refs.copy()
        free = [p for p in range(len(before)) if before[p] == 0]
        jobs, need = [], 0
        for s, w in enumerate(want):
            n = int(self.len[s])
            if w <= n:
                continue
            if w > self.table.shape[1] * self.page:
                raise ValueError(s)
            copies = n % self.page != 0 and before[self.table[s, n // self.page]] > 1
            fresh = -(-int(w) // self.page) - -(-n // self.page)
            jobs.append((s, int(w), copies, fresh))
            need += fresh + copies
        if need > len(free):
            raise OutOfPages(need - len(free))
        at = 0
        for s, w, copies, fresh in jobs:
            n = int(self.len[s])
            if copies:
                old, new = self.table[s, n // self.page], free[at]
                at += 1
                held = n % self.page
                self.k[:, new, :, :held] = self.k[:, old, :, :held]
                self.v[:, new, :, :held] = self.v[:, old, :, :held]
                self.refs[old] -= 1
                self.refs[new] = 1
                self.table[s, n // self.page] = new
            first = -(-n // self.page)
            for j in range(fresh):
                self.table[s, first + j] = free[at]
                self.refs[free[at]] = 1
                at += 1
            self.len[s] = w

    def fork(self, parent) -> None:
        lens, table = self.len.copy(), self.table.copy()
        for s, p in enumerate(parent):
            if p < 0 or p >= len(parent) or p == s or parent[p] >= 0 or lens[s] != 0:
                continue
            m = -(-int(lens[p]) // self.page)
            self.table[s, :m] = table[p, :m]
            np.add.at(self.refs, table[p, :m], 1)
            self.len[s] = lens[p]

    def trim(self, to) -> None:
        for s, t in enumerate(to):
            n = int(self.len[s])
            if t < 0 or t >= n:
                continue
            np.subtract.at(self.refs, self.table[s, -(-int(t) // self.page):-(-n // self.page)], 1)
            self.len[s] = t

    def put(self, layer: int, slot: int, pos: int, h: int, k, v) -> None:
        p = self.table[slot, pos // self.page]
        self.k[layer, p, h, pos % self.page] = k
        self.v[layer, p, h, pos % self.page] = v

    def rows(self, pool, layer: int, slot: int, h: int):
        """A slot's rows of one kv head, in order."""
        n = int(self.len[slot])
        return np.concatenate([pool[layer, p, h] for p in self.pages(slot)] or [pool[layer, 0, h, :0]])[:n]


def attend(q, k, v):
    """q [n_q][rows][d], k, v [n][d] in float64, the n_q tokens being the sequence's last: (out, lse, A, E) where A is the sum
    of weight x |v| and E the largest sum of |q_i k_i| / sqrt(d) over the keys seen, per row: what errors scale with."""
    nq, rows, d = q.shape
    n = k.shape[0]
    out, lse = np.zeros(q.shape), np.full((nq, rows), -np.inf)
    weight, most = np.zeros(q.shape), np.zeros((nq, rows))
    for t in range(nq):
        see = n - nq + t + 1
        if see <= 0:
            continue
        x = q[t] @ k[:see].T / np.sqrt(d)
        top = x.max(axis=1, keepdims=True)
        e = np.exp(x - top)
        s = e.sum(axis=1, keepdims=True)
        lse[t] = (top + np.log(s))[:, 0]
        out[t] = (e / s) @ v[:see]
        weight[t] = (e / s) @ np.abs(v[:see])
        most[t] = (np.abs(q[t]) @ np.abs(k[:see]).T / np.sqrt(d)).max(axis=1)
    return out, lse, weight, most
