"""The paged cache from its definitions, in 64 bits and plain loops, on the CPU: what the GPU tests compare with.  Shares no
code with the library."""
from __future__ import annotations

import math

import torch

E4M3_MAX = 448.0


def pages_of(n, page):
    return -(-n // page)


class Allocator:
    """Block tables and free pages as lists."""

    def __init__(self, batch, num_pages, max_pages, page, ring, head, count, table, lens):
        self.batch, self.num_pages, self.max_pages, self.page = batch, num_pages, max_pages, page
        self.ring, self.head, self.count = list(ring), head, count
        self.table = [list(r) for r in table]
        self.lens = list(lens)

    def step(self, keep, new, max_tokens):
        """(status, q_start, slots); the state moves on where status is 0."""
        nothing = [0] * (self.batch + 1), [-1] * max_tokens
        held = [pages_of(n, self.page) for n in self.lens]
        if any(k < 0 or k > n or x < 0 or k + x > self.max_pages * self.page for k, n, x in zip(keep, self.lens, new)):
            return (2, *nothing)
        if sum(new) > max_tokens:
            return (3, *nothing)
        want = [pages_of(k + x, self.page) for k, x in zip(keep, new)]
        if sum(max(0, w - h) for w, h in zip(want, held)) > self.count:
            return (1, *nothing)
        head, tail = self.head, self.head + self.count
        for b in range(self.batch):
            for i in range(held[b], want[b]):
                self.table[b][i] = self.ring[head % self.num_pages]
                head += 1
        for b in range(self.batch):
            for i in range(want[b], held[b]):
                self.ring[tail % self.num_pages] = self.table[b][i]
                tail += 1
        self.head, self.count = head % self.num_pages, tail - head
        q_start, slots = [0], []
        for b in range(self.batch):
            q_start.append(q_start[-1] + new[b])
            for x in range(keep[b], keep[b] + new[b]):
                slots.append(self.table[b][x // self.page] * self.page + x % self.page)
        self.lens = [k + x for k, x in zip(keep, new)]
        return 0, q_start, slots + [-1] * (max_tokens - len(slots))


def to_store(x, fp8):
    """Values as the cache holds them."""
    if not fp8:
        return x
    return torch.where(x.isnan(), x.float(), x.float().clamp(-E4M3_MAX, E4M3_MAX)).to(torch.float8_e4m3fn)


def _least_exponent(amax):
    """Least e >= -100 with amax <= 127 * 2^e."""
    e = -100
    while amax > 127.0 * 2.0 ** e:
        e += 1
    return e


def _number(x):
    x = x.double()
    return torch.where(x.isnan(), 0.0, x).clamp(-2.0 ** 127, 2.0 ** 127)


def bounds_of(rows):
    """rows [n, d] -> ([2, d] whole numbers, power of two)."""
    x = _number(rows)
    both = torch.stack([x.amax(0), (-x).amax(0)])
    scale = 2.0 ** _least_exponent(float(both.abs().max()))
    return torch.ceil(both / scale).to(torch.int8), scale


def select(q, bounds, scales, table, q_start, lens, page, first, last, top, causal):
    """[tokens][kv heads] lists of pages; None for tokens of no request.  q [tokens, Hq, d]."""
    tokens, Hq, d = q.shape
    H = bounds.shape[1]
    G = Hq // H
    out = [None] * tokens
    for b in range(len(lens)):
        n = q_start[b + 1] - q_start[b]
        for j in range(n):
            t = q_start[b] + j
            sees = max(0, lens[b] - n + j + 1) if causal else lens[b]
            k = pages_of(sees, page)
            out[t] = []
            for h in range(H):
                x = _number(q[t, h * G:(h + 1) * G])
                code = torch.round(x / 2.0 ** _least_exponent(float(x.abs().max())))
                a, c = code.clamp(min=0).sum(0), (-code).clamp(min=0).sum(0)
                ids = table[b][:k]
                w = bounds[ids, h].double()
                dots = (w[:, 0] * a + w[:, 1] * c).sum(1)
                score = (dots.float() * scales[ids, h].float()).tolist()
                fixed = {i for i in range(k) if i < first or i >= k - last}
                rest = sorted((i for i in range(k) if i not in fixed), key=lambda i: (-score[i], i))
                out[t].append(sorted(list(fixed) + rest[:max(0, top - len(fixed))]))
    return out


def attend(q, k_pages, v_pages, table, q_start, lens, page, sm, causal, chosen=None):
    """out, lse, and A = sum p |v| / sum p (what a relative error of the probabilities is multiplied by), all in 64 bits; rows of
    tokens of no request are NaN.  Pages as stored; chosen [tokens][kv heads] of page lists, or None."""
    tokens, Hq, d = q.shape
    H = k_pages.shape[1]
    G = Hq // H
    out = torch.full((tokens, Hq, d), math.nan, dtype=torch.float64)
    mag = out.clone()
    lse = torch.full((tokens, Hq), math.nan, dtype=torch.float64)
    for b in range(len(lens)):
        n, size = q_start[b + 1] - q_start[b], lens[b]
        if n == 0:
            continue
        ids = table[b][:pages_of(size, page)]
        for h in range(H):
            k = k_pages[ids, h].double().reshape(-1, d)[:size] if ids else torch.zeros(0, d, dtype=torch.float64)
            v = v_pages[ids, h].double().reshape(-1, d)[:size] if ids else torch.zeros(0, d, dtype=torch.float64)
            for j in range(n):
                t = q_start[b] + j
                sees = torch.zeros(size, dtype=torch.bool)
                sees[:max(0, size - n + j + 1) if causal else size] = True
                if chosen is not None:
                    of = torch.zeros(size, dtype=torch.bool)
                    for x in chosen[t][h]:
                        if x >= 0:
                            of[x * page:(x + 1) * page] = True
                    sees &= of
                for g in range(G):
                    hq = h * G + g
                    s = k[sees] @ q[t, hq].double() * sm
                    top = s.max() if s.numel() else torch.tensor(-math.inf)
                    if not s.numel() or top == -math.inf:
                        out[t, hq], mag[t, hq], lse[t, hq] = 0.0, 0.0, -math.inf
                        continue
                    e = torch.exp(s - top)
                    out[t, hq] = e @ v[sees] / e.sum()
                    mag[t, hq] = e @ v[sees].abs() / e.sum()
                    lse[t, hq] = torch.log(e.sum()) + top
    return out, lse, mag
