"""4-bit cache rows and pages that several requests hold, from their definitions, in 64 bits and plain loops, on the CPU: what the
GPU tests compare with.  Shares no code with the library."""
from __future__ import annotations

import torch

from tests.paged_reference import pages_of

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def fp4_encode(x):
    """[..., d] -> (codes [..., d] of 0 to 15, scale bytes [..., d / 32]); the codes of a block with a NaN are 0."""
    b = x.double().unflatten(-1, (-1, 32))
    nan = b.isnan().any(-1)
    b = torch.where(nan[..., None], 0.0, b).clamp(-2.0 ** 140, 2.0 ** 140)
    top = b.abs().amax(-1)
    e = torch.full_like(top, -100)
    for n in range(-99, 126):
        e = torch.where(top > 7 * 2.0 ** (n - 1), float(n), e)
    y = b.abs() * torch.exp2(-e)[..., None]
    code = torch.zeros(y.shape, dtype=torch.int64)
    for i in range(7):
        middle = (E2M1[i] + E2M1[i + 1]) / 2
        code += (y > middle) | ((y == middle) & (i % 2 == 1))
    code += 8 * torch.signbit(b)
    return torch.where(nan[..., None], 0, code).flatten(-2), torch.where(nan, 255, e.long() + 127)


def fp4_decode(codes, scales):
    values = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=torch.float64)[codes]
    power = torch.where(scales == 255, torch.nan, torch.exp2(scales.double() - 127))
    return (values.unflatten(-1, (-1, 32)) * power[..., None]).flatten(-2)


def fp4_pack(codes, scales):
    """codes [pages, H, page, d], scales [pages, H, page, d / 32] -> uint8 [pages, H, bytes of a page]."""
    n, H, page, d = codes.shape
    half = (codes[..., ::2] + 16 * codes[..., 1::2]).view(n, H, page // 16, 16 * d // 2)
    tail = scales.view(n, H, page // 16, 16 * d // 32)
    return torch.cat([half, tail], -1).flatten(2).to(torch.uint8)


def fp4_unpack(pages, page, d):
    """The other way."""
    n, H = pages.shape[:2]
    x = pages.long().view(n, H, page // 16, 16 * (d // 2 + d // 32))
    half, tail = x[..., :8 * d].reshape(n, H, page, d // 2), x[..., 8 * d:].reshape(n, H, page, d // 32)
    return torch.stack([half % 16, half // 16], -1).flatten(-2), tail


class Sharing:
    """Block table, holders and ring of free pages as lists; in place, as the library has them."""

    def __init__(self, num_pages, max_pages, page, ring, head, count, table, lens):
        self.num_pages, self.max_pages, self.page = num_pages, max_pages, page
        self.ring, self.head, self.count = list(ring), head, count
        self.table, self.lens = [list(r) for r in table], list(lens)
        self.holders = [0] * num_pages
        for row, n in zip(self.table, self.lens):
            for p in row[:pages_of(n, page)]:
                self.holders[p] += 1

    def _rows(self):
        return [row[:pages_of(n, self.page)] for row, n in zip(self.table, self.lens)]

    def _settle(self, before, lens, tail):
        """Holders from the rows; what nobody holds any more, ascending, from ring place `tail` on."""
        self.lens = lens
        now = [0] * self.num_pages
        for row in self._rows():
            for p in row:
                now[p] += 1
        for p in range(self.num_pages):
            if before[p] and not now[p]:
                self.ring[tail % self.num_pages] = p
                tail += 1
                self.count += 1
        self.holders = now

    def _bad(self):
        return any(n < 0 or n > self.max_pages * self.page for n in self.lens)

    def fork(self, parent):
        if self._bad():
            return 2
        if any(p < -1 or p >= len(self.lens) for p in parent):
            return 5
        rows, lens, before = self._rows(), list(self.lens), list(self.holders)
        for b, p in enumerate(parent):
            if p >= 0:
                self.table[b][:len(rows[p])] = rows[p]
        self._settle(before, [lens[p] if p >= 0 else 0 for p in parent], self.head + self.count)
        return 0

    def assign(self, keep, new, max_tokens):
        """(status, q_start, slots, copies [batch][page] of (from, to) or (-1, -1))."""
        page, B = self.page, len(self.lens)
        nothing = [0] * (B + 1), [-1] * max_tokens, [[(-1, -1)] * page for _ in range(B)]
        if self._bad() or any(k < 0 or k > n or x < 0 or k + x > self.max_pages * page for k, n, x in zip(keep, self.lens, new)):
            return (2, *nothing)
        if sum(new) > max_tokens:
            return (3, *nothing)
        shared = [x > 0 and k % page > 0 and self.holders[row[k // page]] > 1 for k, x, row in zip(keep, new, self.table)]
        first = [pages_of(k, page) - s for k, s in zip(keep, shared)]
        takes = [pages_of(k + x, page) - f for k, x, f in zip(keep, new, first)]
        if sum(takes) > self.count:
            return (1, *nothing)
        before, tail = list(self.holders), self.head + self.count
        q_start, slots, copies = [0], [], nothing[2]
        for b in range(B):
            old = self.table[b][first[b]] if shared[b] else None
            for c in range(first[b], first[b] + takes[b]):
                self.table[b][c] = self.ring[self.head]
                self.head = (self.head + 1) % self.num_pages
                self.count -= 1
            if shared[b]:
                for r in range(keep[b] % page):
                    copies[b][r] = (old * page + r, self.table[b][first[b]] * page + r)
            q_start.append(q_start[-1] + new[b])
            slots += [self.table[b][x // page] * page + x % page for x in range(keep[b], keep[b] + new[b])]
        self._settle(before, [k + x for k, x in zip(keep, new)], tail)
        return 0, q_start, slots + [-1] * (max_tokens - len(slots)), copies

    def compact(self, kept, max_moves):
        """(status, moves [max_moves] of (from, to) or (-1, -1))."""
        page = self.page
        nothing = [(-1, -1)] * max_moves
        if self._bad():
            return 2, nothing
        plans, moves_all, takes_all = [], 0, 0
        for n, marks in zip(self.lens, kept):
            stay = [x for x in range(n) if marks[x]]
            lead = next((x for x in range(n) if not marks[x]), n)
            cut = len(stay) == lead
            first = pages_of(len(stay), page) if cut else lead // page
            takes = pages_of(len(stay), page) - first
            plans.append((stay, first, takes, cut))
            moves_all += 0 if cut else len(stay) - first * page
            takes_all += takes
        if moves_all > max_moves:
            return 3, nothing
        if takes_all > self.count:
            return 1, nothing
        before, tail, moves = list(self.holders), self.head + self.count, []
        for row, (stay, first, takes, cut) in zip(self.table, plans):
            old = list(row)
            for c in range(first, first + takes):
                row[c] = self.ring[self.head]
                self.head = (self.head + 1) % self.num_pages
                self.count -= 1
            if not cut:
                for y in range(first * page, len(stay)):
                    x = stay[y]
                    moves.append((old[x // page] * page + x % page, row[y // page] * page + y % page))
        self._settle(before, [len(p[0]) for p in plans], tail)
        return 0, moves + [(-1, -1)] * (max_moves - len(moves))
