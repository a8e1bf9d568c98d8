"""Plain models of the paged cache, on the CPU: the table as lists, pools built row
by row, and the pages that a kv head's queries choose, by 64-bit scores."""
import math

import torch

from rows_reference import row


def attend(q, k, v, dtype):
    """Rows q [heads, d] over keys and values [n, d]: (o, bound).  fp32: the bound that
    rows_reference.py derives.  bf16: the output is rounded, half a step, 2^-8 of it; a
    weight is cut off after 8 bits, which leaves less than 2^-7 of it, and what is left is
    rounded in its turn, 2^-8 of that: 2^-15 of sum_j p_j |v_j|."""
    o, bound = row(q, k, v, torch.zeros(len(k), dtype=torch.float64), torch.float32)
    if dtype == torch.bfloat16:
        p = torch.softmax(q.double() @ k.T / math.sqrt(q.shape[-1]), -1)
        bound = bound + 2.0 ** -8 * o.abs() + 2.0 ** -15 * (p @ v.abs())
    return o, bound


class Table:
    """eva.PageTable as lists; `stack` holds the free pages, its last one on top."""

    def __init__(self, B, P, n_pages, max_pages):
        self.P, self.max_pages = P, max_pages
        self.n = [0] * B
        self.rows = [[] for _ in range(B)]
        self.stack = list(range(n_pages - 1, -1, -1))

    def held(self, n):
        return -(-n // self.P)

    def extend(self, T, counts=None):
        slots, start, granted, asked, free = [], [], [], 0, len(self.stack)
        for b, n in enumerate(self.n):
            c = T if counts is None else min(max(counts[b], 0), T)
            if n + c > self.max_pages * self.P:
                c = 0
            need = self.held(n + c) - self.held(n)
            asked += need
            if need and asked > free:
                c = need = 0
            for _ in range(need):
                self.rows[b].append(self.stack.pop())
            slots.append([self.rows[b][p // self.P] * self.P + p % self.P for p in range(n, n + c)] + [-1] * (T - c))
            start.append(n)
            granted.append(c)
            self.n[b] = n + c
        return slots, start, granted

    def truncate(self, lens):
        for b in range(len(self.n) - 1, -1, -1):
            n = min(self.n[b], max(lens[b], 0))
            while len(self.rows[b]) > self.held(n):
                self.stack.append(self.rows[b].pop())
            self.n[b] = n

    def check(self, t):
        """Holds what the device's arrays do."""
        assert t.n_tok.tolist() == self.n
        assert t.n_free.item() == len(self.stack)
        assert t.free_pages[:len(self.stack)].tolist() == self.stack
        table = t.table.cpu()
        for b, row in enumerate(self.rows):
            assert table[b].tolist() == row + [-1] * (self.max_pages - len(row)), f"sequence {b}"


def choice(q, mean, held, S, first, last):
    """Pages that queries q [G, d] choose from pages of these mean keys [held, d]."""
    if held <= S:
        return list(range(held)) + [-1] * (S - held)
    score = (mean.double() @ q.double().T).amax(-1)   # a NaN is carried
    key = [float("inf") if s != s else s for s in score.tolist()]
    nan = [0 if s != s else 1 for s in score.tolist()]
    inner = sorted(range(first, held - last), key=lambda j: (nan[j], -key[j], j))[:S - first - last]
    return list(range(first)) + sorted(inner) + list(range(held - last, held))


def keys_of(pages, P, n):
    """Positions that a list of pages attends, of a sequence of n tokens."""
    held = -(-n // P)
    return [p for j in pages[:held] if 0 <= j < held for p in range(j * P, min(n, j * P + P))]


def tiles(v):
    """Values [..., P, d] as the pool holds them: [..., P / 8, d, 8]."""
    *lead, P, d = v.shape
    return v.reshape(*lead, P // 8, 8, d).transpose(-1, -2).contiguous()


def mean_bound(k):
    """Error of a mean of P fp32 additions over rows k [P, d]: each partial sum is
    rounded once, P of them at most, and the division by P (a power of two) is exact."""
    return (k.shape[0] + 1) * 2.0 ** -24 * k.double().abs().mean(0) + 1e-45


def random_pages(B, P, lens, n_pages, max_pages, gen):
    """A table that gives sequences of these lengths pages in any order: (table, free, n_free)."""
    order = torch.randperm(n_pages, generator=gen)
    table, at = torch.full((B, max_pages), -1, dtype=torch.int32), 0
    for b, n in enumerate(lens):
        m = -(-n // P)
        table[b, :m] = order[at:at + m].int()
        at += m
    return table, order[at:].flip(0).int(), n_pages - at
