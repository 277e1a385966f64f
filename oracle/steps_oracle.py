"""Oracles of what stands around the chunk attention: verification of proposed tokens in fp64, and the books of paged caches, each
written step by step from its definition.  They share nothing with the product."""
from __future__ import annotations

import numpy as np


def distribution(scores, temperature, probabilities: bool):
    """One row of scores (float) as (p, log p at the temperature, or at 1 where it is greedy), fp64."""
    x = np.asarray(scores, np.float64)
    if probabilities:
        p = np.where(np.isfinite(x) & (x > 0), x, 0.0)
        with np.errstate(divide="ignore"):
            return p, np.log(p)
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if top == -np.inf:
        return np.zeros_like(x), np.full_like(x, -np.inf)
    greedy = not temperature > 0
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        if top == np.inf:
            free = np.where(x == np.inf, 0.0, -np.inf)
        else:
            free = (x - top) / (1.0 if greedy else min(np.float64(temperature), float(np.float32(1e30))))
            free = np.where(x == -np.inf, -np.inf, free)
        free = free - np.log(np.exp(free).sum())
        if not greedy:
            return np.exp(free), free
    p = np.zeros_like(x)
    p[int(np.argmax(x == top))] = 1.0  # (the first)
    return p, free


def pick(w, uniform):
    """First i whose running sum passes uniform times the whole; behind the last, the last that has any; -1 if none has."""
    c = np.cumsum(w)
    if not c[-1] > 0:
        return -1
    more = np.nonzero((c > uniform * c[-1]) & (w > 0))[0]
    return int(more[0]) if len(more) else int(np.nonzero(w > 0)[0][-1])


def draft_verify(target, tokens, cu_qlens, uniform, draft=None, temperature=None, probabilities=False):
    """-> dict(out, accepted, logp).  target [sum T, V], draft [B, steps, V] or None, temperature [B] or None."""
    n, vocab = target.shape
    b = len(cu_qlens) - 1
    out, logp, accepted = np.full(n, -1, np.int64), np.zeros(n), np.zeros(b, np.int64)
    for u in range(b):
        lo, hi = int(cu_qlens[u]), int(cu_qlens[u + 1])
        heat = 1.0 if temperature is None else float(temperature[u])
        for a in range(hi - lo):
            row = lo + a
            p, free = distribution(target[row], heat, probabilities)
            x = int(tokens[row + 1]) if row + 1 < hi else -1
            w = p
            if 0 <= x < vocab and (draft is None or a < draft.shape[1]):
                q = np.zeros(vocab)
                q[x] = 1.0
                if draft is not None:
                    q = distribution(draft[u, a], heat, probabilities)[0]
                if not probabilities and not heat > 0:
                    stands = p[x] == 1.0
                else:
                    stands = float(uniform[row]) * q[x] < p[x]
                if stands:
                    out[row], logp[row] = x, free[x]
                    accepted[u] += 1
                    continue
                w = np.maximum(p - q, 0.0)
                if not w.sum() > 0:
                    w = p
            out[row] = pick(w, float(uniform[hi - 1]))
            logp[row] = free[out[row]] if out[row] >= 0 else 0.0
            break
    return dict(out=out, accepted=accepted, logp=logp)


class Books:
    """Page table, counts and lengths, changed one question after the other."""

    def __init__(self, table, refs, self_len, page_tokens: int):
        self.table, self.refs, self.self_len = (np.array(x, np.int64) for x in (table, refs, self_len))
        self.page = page_tokens

    def _is_page(self, e):
        return 0 <= e < len(self.refs)

    def _used(self, n):
        return -(-min(max(int(n), 0), self.table.shape[1] * self.page) // self.page)

    def fork(self, source):
        table, length = self.table.copy(), self.self_len.copy()
        for u, s in enumerate(int(x) for x in source):
            if s == u or not 0 <= s < len(table):
                continue
            for c in range(table.shape[1]):
                now = table[s, c] if c < self._used(length[s]) and self._is_page(table[s, c]) else -1
                if self._is_page(table[u, c]):
                    self.refs[table[u, c]] -= 1
                if now >= 0:
                    self.refs[now] += 1
                self.table[u, c] = now
            self.self_len[u] = length[s]

    def _asks(self, u, more):
        """Whether question u can be served at all, and the columns its new tokens reach into behind its last page in use."""
        n = max(int(self.self_len[u]), 0)
        if more <= 0 or n + more > self.table.shape[1] * self.page:
            return False, range(0)
        if n % self.page and not self._is_page(int(self.table[u, n // self.page])):
            return False, range(0)
        return True, range(self._used(n), self._used(n + more))

    def reserve(self, add):
        """-> (got, copies)"""
        # what lies behind the tokens holds nothing: entries that share their page go back before anything is handed out
        before = self.refs.copy()
        for u, more in enumerate(int(x) for x in add):
            for c in self._asks(u, more)[1]:
                if self._is_page(self.table[u, c]) and before[self.table[u, c]] > 1:
                    self.refs[self.table[u, c]] -= 1
                    self.table[u, c] = -1
        free = [p for p in range(len(self.refs)) if self.refs[p] <= 0]
        got, copies, stopped = np.zeros(len(add), np.int64), [], False
        for u, more in enumerate(int(x) for x in add):
            n = max(int(self.self_len[u]), 0)
            asks, reached = self._asks(u, more)
            if stopped or not asks:
                continue
            rows = n % self.page
            tail = int(self.table[u, n // self.page]) if rows else -1
            replace = tail >= 0 and self.refs[tail] > 1
            lacks = [c for c in reached if not self._is_page(self.table[u, c])]
            if replace + len(lacks) > len(free):
                stopped = True
                continue
            if replace:
                page = free.pop(0)
                copies.append((tail, page, rows))
                self.refs[tail] -= 1
                self.refs[page] = 1
                self.table[u, n // self.page] = page
            for c in lacks:
                page = free.pop(0)
                self.refs[page] = 1
                self.table[u, c] = page
            got[u] = more
            self.self_len[u] = n + more
        return got, copies

    def trim(self):
        for u in range(len(self.table)):
            for c in range(self._used(self.self_len[u]), self.table.shape[1]):
                if self._is_page(self.table[u, c]):
                    self.refs[self.table[u, c]] -= 1
                    self.table[u, c] = -1

    def compact(self):
        """-> (copies, pages in use, where each page is)"""
        live = int((self.refs > 0).sum())
        holes = [p for p in range(live) if self.refs[p] <= 0]
        come = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        place = np.where(self.refs > 0, np.arange(len(self.refs)), -1)
        for a, b in zip(come, holes):
            place[a] = b
            self.refs[b], self.refs[a] = self.refs[a], 0
        for u in range(self.table.shape[0]):
            for c in range(self.table.shape[1]):
                if self._is_page(self.table[u, c]):
                    self.table[u, c] = place[self.table[u, c]]
        return [(a, b, self.page) for a, b in zip(come, holes)], live, place


def copy_rows(pages, copies):
    """pages [layers, pages, page tokens, ...], in place."""
    for a, b, rows in copies:
        pages[:, b, :rows] = pages[:, a, :rows]
