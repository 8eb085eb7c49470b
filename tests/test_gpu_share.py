"""Pages that several requests hold, on the GPU against lists (tests/share_reference.py): rows of the table that continue others, the
allocator's step that copies on write, requests that lose tokens, and a server's steps with the rows of the cache and attention."""
import math
import random

import pytest
import torch

import paper_2605_14877_amd as hk
from tests import paged_reference as ref
from tests import share_reference as sref
from tests.paged_reference import pages_of

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _numbers(rng, n, most):
    return [rng.randrange(most) for _ in range(n)]


class Server:
    """The arrays of one cache's tables on the GPU, and the reference beside them."""

    def __init__(self, batch, num_pages, max_pages, page, seed=0, kv=(1, 1, 64, "bf16", hk.KV_NATIVE), apart=False):
        self.rng = random.Random(seed)
        self.batch, self.page, self.apart = batch, page, apart
        q, h, d, dtype, fmt = kv
        self.shape = hk.PagedShape(q, h, d, page, num_pages, batch, max_pages, dtype, fmt)
        ring = list(range(num_pages))
        self.rng.shuffle(ring)
        head = self.rng.randrange(num_pages)
        table = [_numbers(self.rng, max_pages, 2 ** 31 - 1) for _ in range(batch)]  # entries of pages that a row lacks are anything
        self.ref = sref.Sharing(num_pages, max_pages, page, ring, head, num_pages, table, [0] * batch)
        self.lens, self.span = _ints([0] * batch), _ints([head, num_pages])
        self.ring, self.table, self.holders = _ints(ring), _ints(table), _ints([0] * num_pages)
        self.status = _ints([9])
        n = hk.paged_tables_workspace_bytes(self.shape)
        self.ws = torch.full((n + 64,), 255, dtype=torch.uint8, device="cuda")

    def call(self, name, *args, tail=()):
        """One of the three calls; with `apart` lengths and span go to arrays of their own, and the old ones stay."""
        more = {}
        if self.apart:
            more = dict(lens_out=torch.full_like(self.lens, 77), free_span_out=torch.full_like(self.span, 77))
            old = self.lens.clone(), self.span.clone()
        getattr(hk, "heatkv_paged_" + name)(self.shape, *args, self.lens, self.holders, self.ring, self.span, self.table, *tail,
                                            self.status, self.ws[:-64], **more)
        if self.apart:
            assert torch.equal(self.lens, old[0]) and torch.equal(self.span, old[1])
            self.lens, self.span = more["lens_out"], more["free_span_out"]
        assert torch.all(self.ws[-64:] == 255)

    def fork(self, parent):
        self.call("fork", _ints(parent))
        self.check(self.ref.fork(parent))

    def assign(self, keep, new, max_tokens=None):
        max_tokens = sum(new) + 5 if max_tokens is None else max_tokens
        q_start, slots = _ints([77] * (self.batch + 1)), _ints([77] * max_tokens)
        copies = [torch.full((self.batch, self.page), 77, dtype=torch.int32, device="cuda") for _ in range(2)]
        self.call("assign_shared", _ints(keep), _ints(new), tail=(q_start, slots, *copies))
        status, want_q, want_slots, want = self.ref.assign(keep, new, max_tokens)
        self.check(status)
        assert q_start.tolist() == want_q and slots.tolist() == want_slots
        assert [[tuple(x) for x in row] for row in torch.stack(copies, -1).tolist()] == want
        return q_start, slots, *copies

    def compact(self, kept, max_moves, dtype=torch.bool):
        marks = torch.tensor(kept).to(dtype)
        if dtype == torch.uint8:
            marks *= 0x80
        moves = [torch.full((max_moves,), 77, dtype=torch.int32, device="cuda") for _ in range(2)]
        self.call("compact", marks.cuda(), tail=tuple(moves))
        status, want = self.ref.compact(kept, max_moves)
        self.check(status)
        assert list(zip(*(m.tolist() for m in moves))) == want
        return moves

    def check(self, status):
        r = self.ref
        assert self.status.item() == status
        assert self.lens.tolist() == r.lens and self.span.tolist() == [r.head, r.count]
        assert self.holders.tolist() == r.holders
        assert self.ring.tolist() == r.ring
        assert self.table.tolist() == r.table
        if status == 0:  # every page is held or free, once
            free = [r.ring[(r.head + i) % r.num_pages] for i in range(r.count)]
            assert sorted(free + [p for p, n in enumerate(r.holders) if n]) == list(range(r.num_pages))

    # random arguments
    def parents(self):
        B = self.batch
        out = []
        for b in range(B):
            u = self.rng.random()
            out.append(b if u < 0.4 else -1 if u < 0.5 else self.rng.randrange(B))
        return out

    def step_sizes(self, most_new):
        keep, new = [], []
        room = self.shape.max_pages * self.page
        for n in self.ref.lens:
            u = self.rng.random()
            k = n if u < 0.6 else self.rng.randint(0, n) if u < 0.8 else max(0, n - self.rng.randint(0, 5)) if u < 0.9 else 0
            keep.append(k)
            new.append(min(room - k, self.rng.randint(0, most_new)) if self.rng.random() < 0.8 else 0)
        return keep, new

    def marks(self):
        width = self.shape.max_pages * self.page
        out = []
        for n in self.ref.lens:
            share = self.rng.choice((0.0, 0.1, 0.5, 0.9, 1.0))
            lead = self.rng.choice((0, 0, n // 2, n))
            tail = self.rng.choice((0, 0, n // 3))
            out.append([x < lead or (self.rng.random() < share and x < n - tail) for x in range(width)])
        return out


SIZES = [(1, 9, 4, 16), (4, 40, 6, 16), (5, 60, 8, 32), (16, 200, 9, 16), (3, 30, 5, 256), (70, 900, 10, 16), (150, 2500, 12, 64)]


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_random_steps(size, apart):
    s = Server(*size, seed=sum(size), apart=apart)
    most = size[2] * size[3] // 4
    s.assign([0] * s.batch, [s.rng.randint(0, most) for _ in range(s.batch)])
    for step in range(12):
        what = step % 4
        if what in (0, 2):
            s.fork(s.parents())
        if what in (1, 2):
            s.assign(*s.step_sizes(s.rng.choice((1, 1, 3, most))))
        if what == 3:
            s.compact(s.marks(), s.rng.choice((sum(s.ref.lens), sum(s.ref.lens) + 9, sum(s.ref.lens) // 8)), s.rng.choice((torch.bool, torch.uint8)))


def test_rows_that_swap_and_rows_that_follow_one_another():
    s = Server(5, 50, 6, 16, seed=1)
    s.assign([0] * 5, [16, 33, 1, 0, 96])
    for parent in ([1, 0, 2, 3, 4], [1, 2, 3, 4, 0], [4, 4, 4, 4, 4], [-1, 0, 1, 2, 3], [-1] * 5, [0, 1, 2, 3, 4]):
        s.fork(parent)
        s.assign(list(s.ref.lens), [min(1, 96 - n) for n in s.ref.lens])


@pytest.mark.parametrize("beams", [2, 4, 64])
def test_beams_write_to_pages_of_their_own(beams):
    s = Server(beams, 40 * beams, 12, 16, seed=beams)
    s.assign([0] * beams, [37] + [0] * (beams - 1))
    s.fork([0] * beams)
    assert sorted(set(s.holders.tolist())) == [0, beams]
    _, _, copies, _ = s.assign([37] * beams, [1] * beams)
    assert int((copies >= 0).sum()) == 5 * beams  # all of them, also the last one: its page is free then
    s.fork([b // 2 for b in range(beams)])
    s.assign(list(s.ref.lens), [1] * beams)
    # on the border of a page nothing is copied
    s.assign([32] * beams, [0] * beams)
    s.fork([0] * beams)
    _, _, copies, _ = s.assign([32] * beams, [1] * beams)
    assert torch.all(copies == -1)


def test_cut_back_into_pages_that_others_hold():
    s = Server(3, 40, 8, 16, seed=3)
    s.assign([0] * 3, [70, 0, 0])
    s.fork([0, 0, 0])
    s.assign([70, 40, 32], [0, 3, 20])  # the second copies 8 rows of its third page, the third none
    s.assign([5, 43, 52], [1, 1, 0])    # the first copies 5 rows of its first page
    s.assign([5, 0, 52], [0, 0, 0])     # nothing new: nothing is copied, even on a page of several
    s.assign([5, 0, 7], [1, 0, 9])


@pytest.mark.parametrize("seed", range(3))
def test_steps_that_cannot_be_made_change_nothing(seed):
    s = Server(4, 20, 6, 16, seed=seed)
    s.assign([0] * 4, [70, 20, 30, 1])
    s.fork([0, 0, 2, 3])
    s.fork([0, 1, 4, 3])
    assert s.status.item() == hk.PAGED_BAD_PARENT
    s.fork([0, -2, 2, 3])
    s.assign([70, 70, 30, 1], [26, 26, 60, 80])
    assert s.status.item() == hk.PAGED_NO_PAGES
    s.assign([70, 71, 30, 1], [1, 1, 1, 1])
    assert s.status.item() == hk.PAGED_BAD_LENGTH
    s.assign([70, 70, 30, 1], [1, -1, 1, 1])
    s.assign([70, 70, 30, 1], [27, 1, 1, 1])
    s.assign([70, 70, 30, 1], [1, 1, 1, 1], max_tokens=3)
    assert s.status.item() == hk.PAGED_TOO_MANY_TOKENS
    every = [[x % 2 == 0 for x in range(96)]] * 4
    s.compact(every, 50)
    assert s.status.item() == hk.PAGED_TOO_MANY_TOKENS
    s.compact(every, 0)
    good = s.lens.clone()
    for bad in (-1, 97, 2 ** 31 - 1, -2 ** 31):
        s.lens[1] = bad
        s.ref.lens[1] = bad
        s.fork([0, 1, 2, 3])
        s.assign([0, 0, 0, 0], [1, 1, 1, 1])
        s.compact(every, 500)
        assert s.status.item() == hk.PAGED_BAD_LENGTH
    s.lens.copy_(good)
    s.ref.lens = good.tolist()
    span = s.span.clone()
    for bad in ([-1, 4], [20, 4], [0, 21], [0, -1], [2 ** 31 - 1, 2 ** 31 - 1]):
        s.span.copy_(_ints(bad))
        before = [x.clone() for x in (s.lens, s.ring, s.holders, s.table)]
        s.call("fork", _ints([0, 0, 0, 0]))
        assert s.status.item() == hk.PAGED_BAD_FREE_LIST
        s.call("compact", torch.zeros(4, 96, dtype=torch.bool, device="cuda"), tail=(_ints([5] * 7), _ints([5] * 7)))
        assert s.status.item() == hk.PAGED_BAD_FREE_LIST
        assert all(torch.equal(x, y) for x, y in zip(before, (s.lens, s.ring, s.holders, s.table))) and s.span.tolist() == bad
    s.span.copy_(span)
    s.assign(list(s.ref.lens), [1, 1, 1, 1])


def test_no_pages_for_what_stays():
    # the ring is empty: a request may lose its last tokens, but not one out of its middle
    s = Server(2, 6, 4, 16, seed=5)
    s.assign([0, 0], [64, 32])
    s.compact([[x != 10 for x in range(64)], [True] * 64], 200)
    assert s.status.item() == hk.PAGED_NO_PAGES
    s.compact([[x < 20 for x in range(64)], [True] * 64], 0)
    assert s.status.item() == hk.PAGED_OK and s.ref.count == 2
    s.compact([[True] * 64, [x != 20 for x in range(64)]], 15)
    assert s.status.item() == hk.PAGED_OK


def test_arrays_that_do_not_fit_touch_nothing_outside():
    # holders, ring and table hold anything: the call may do nonsense, but only within its arrays
    for seed in range(4):
        s = Server(6, 37, 5, 16, seed=seed)
        g = torch.Generator().manual_seed(seed)
        guard = torch.full((37 + 200,), 123456, dtype=torch.int32, device="cuda")
        s.holders, s.ring = guard[:37], torch.full((237,), 654321, dtype=torch.int32, device="cuda")[200:]
        table = torch.full((36, 5), 999, dtype=torch.int32, device="cuda")
        s.table = table[10:16]
        s.holders.copy_(torch.randint(-3, 4, (37,), generator=g))
        s.ring.copy_(torch.randint(-2 ** 31, 2 ** 31 - 1, (37,), generator=g))
        s.table.copy_(torch.randint(-2 ** 31, 2 ** 31 - 1, (6, 5), generator=g))
        s.lens.copy_(_ints([80, 16, 33, 0, 50, 7]))
        s.span.copy_(_ints([30, 30]))
        for _ in range(3):
            s.call("fork", _ints([1, 1, 0, 4, 4, -1]))
            q_start, slots = _ints([0] * 7), _ints([0] * 20)
            copies = [torch.zeros(6, 16, dtype=torch.int32, device="cuda") for _ in range(2)]
            keep = s.lens.clamp(max=30)
            s.call("assign_shared", keep, _ints([1, 2, 1, 0, 3, 1]), tail=(q_start, slots, *copies))
            s.call("compact", torch.rand(6, 80, device="cuda") < 0.7, tail=(_ints([0] * 500), _ints([0] * 500)))
            head, count = s.span.tolist()
            assert 0 <= head < 37 and 0 <= count <= 37
        torch.cuda.synchronize()
        assert torch.all(guard[37:] == 123456) and torch.all(table[:10] == 999) and torch.all(table[16:] == 999)


@pytest.mark.parametrize("what", ["fork", "assign_shared", "compact"])
@pytest.mark.parametrize("batch", [4, 1100])  # one workgroup, several launches
def test_holders_that_do_not_fit_are_reported(batch, what):
    def server():
        s = Server(batch, 6 * batch, 4, 16, seed=batch)
        s.assign([0] * batch, [20] * batch)
        return s

    def call(s, ends):
        """Row 1 loses all of its tokens, or nothing changes."""
        B, lens = s.batch, s.lens.tolist()
        if what == "fork":
            s.call("fork", _ints([-1 if b == 1 and ends else b for b in range(B)]))
        elif what == "assign_shared":
            copies = [torch.zeros(B, 16, dtype=torch.int32, device="cuda") for _ in range(2)]
            s.call("assign_shared", _ints([0 if b == 1 and ends else n for b, n in enumerate(lens)]), _ints([0] * B),
                   tail=(_ints([0] * (B + 1)), _ints([0] * 5), *copies))
        else:
            kept = torch.ones(B, 64, dtype=torch.bool, device="cuda")
            kept[1] = not ends
            s.call("compact", kept, tail=(_ints([0] * 5), _ints([0] * 5)))
        return s.status.item(), s.lens.tolist(), s.span.tolist()

    # a count below 0: the page is not given back
    s = server()
    head, count = s.span.tolist()
    lost, other = s.table[1, :2].tolist()
    s.holders[lost] = 0
    lens = [0 if b == 1 else 20 for b in range(batch)]
    assert call(s, True) == (hk.PAGED_BAD_HOLDERS, lens, [head, count + 1])
    assert s.holders[lost].item() == -1 and s.ring[(head + count) % s.shape.num_pages].item() == other
    s.holders[lost] = 0
    assert call(s, False) == (hk.PAGED_OK, lens, [head, count + 1])  # nothing of it stays
    # more pages than the ring has room for, by its span
    s = server()
    ring, full = s.ring.clone(), s.shape.num_pages - 1
    s.span[1] = full
    assert call(s, True) == (hk.PAGED_BAD_HOLDERS, lens, [head, full + 1])
    first = s.ring[(head + full) % s.shape.num_pages].item()
    ring[(head + full) % s.shape.num_pages] = first
    assert first == min(s.table[1, :2].tolist()) and torch.equal(s.ring, ring)  # one of the two, and nothing else
    # as many as there is room for
    s = server()
    s.span[1] = full - 1
    assert call(s, True) == (hk.PAGED_OK, lens, [head, full + 1])


def test_long_requests_and_many_of_them():
    # stretches and chunks of tokens with borders everywhere; more than one workgroup's words of the bitmap
    s = Server(3, 5000, 1700, 16, seed=7)
    s.assign([0] * 3, [27000, 9000, 4096])
    s.fork([0, 1, 0])
    width = 1700 * 16
    rng = random.Random(8)
    a, b = ([rng.random() < p for _ in range(width)] for p in (0.6, 0.02))
    s.compact([a, [x < 4100 or x % 3 == 0 for x in range(width)], b], 40000)
    s.compact([[x >= 4095 for x in range(width)], [x != 4096 for x in range(width)], [False] * width], 40000)
    s = Server(1100, 200000, 30, 16, seed=9)
    s.assign([0] * 1100, [s.rng.randint(0, 300) for _ in range(1100)])
    s.fork(s.parents())
    s.assign(*s.step_sizes(20))
    s.fork([-1 if b % 3 else b for b in range(1100)])
    s.compact([[(x + b) % 5 > 1 for x in range(480)] for b in range(1100)], 300000)


def test_the_largest_batch():
    s = Server(4096, 30000, 5, 16, seed=11)
    s.assign([0] * 4096, [s.rng.randint(0, 60) for _ in range(4096)])
    s.fork(s.parents())
    s.assign(*s.step_sizes(2))
    s.compact([[(x + b) % 4 > 0 for x in range(80)] for b in range(4096)], 300000)


def test_requests_of_more_tokens_than_a_stretch():
    # a table so wide that a workgroup looks at 8192 tokens of a request
    s = Server(2, 5000, 70000, 16, seed=12)
    s.assign([0, 0], [30000, 20001])
    keep = [True] * (70000 * 16)
    other = list(keep)
    for x in range(8000, 30000, 7):
        keep[x] = False
    other[16384] = other[20000] = False
    s.compact([keep, other], 40000)


# ---- captured, on other streams -----------------------------------------------------------------------------------------

def test_a_captured_step_is_replayed_for_other_requests():
    s = Server(8, 300, 12, 16, seed=13)
    s.assign([0] * 8, [s.rng.randint(1, 90) for _ in range(8)])
    parent, keep, new = _ints([0] * 8), _ints([0] * 8), _ints([0] * 8)
    q_start, slots = _ints([0] * 9), _ints([0] * 40)
    copies = [torch.zeros(8, 16, dtype=torch.int32, device="cuda") for _ in range(2)]
    kept = torch.zeros(8, 192, dtype=torch.bool, device="cuda")
    moves = [_ints([0] * 900) for _ in range(2)]
    ws = [s.ws[:-64].clone() for _ in range(3)]
    status = [_ints([9]) for _ in range(3)]

    def step():
        t = (s.lens, s.holders, s.ring, s.span, s.table)
        hk.heatkv_paged_fork(s.shape, parent, *t, status[0], ws[0])
        hk.heatkv_paged_assign_shared(s.shape, keep, new, *t, q_start, slots, *copies, status[1], ws[1])
        hk.heatkv_paged_compact(s.shape, kept, *t, *moves, status[2], ws[2])

    stream = torch.cuda.Stream()
    state = [x.clone() for x in (s.lens, s.holders, s.ring, s.span, s.table)]
    parent.copy_(_ints(list(range(8))))
    keep.copy_(s.lens)
    kept.fill_(True)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for x, y in zip((s.lens, s.holders, s.ring, s.span, s.table), state):
        assert torch.equal(x, y)  # nothing has run
    for _ in range(6):
        parents = s.parents()
        lens = [s.ref.lens[p] if p >= 0 else 0 for p in parents]
        keeps = [n - min(n, s.rng.randint(0, 3)) for n in lens]
        news = [min(192 - k, s.rng.randint(0, 4)) for k in keeps]
        parent.copy_(_ints(parents))
        keep.copy_(_ints(keeps))
        new.copy_(_ints(news))
        marks = torch.rand(8, 192, generator=torch.Generator().manual_seed(sum(lens))) < 0.9
        kept.copy_(marks)
        graph.replay()
        torch.cuda.synchronize()
        want = [s.ref.fork(parents), *s.ref.assign(keeps, news, 40)]
        last = s.ref.compact(marks.tolist(), 900)
        assert [x.item() for x in status] == [want[0], want[1], last[0]] == [0, 0, 0]
        assert q_start.tolist() == want[2] and slots.tolist() == want[3]
        assert list(zip(*(m.tolist() for m in moves))) == last[1]
        s.status.fill_(0)
        s.check(0)


def test_two_caches_on_two_streams():
    servers = [Server(40, 600, 12, 16, seed=20 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    plans = []
    for s in servers:
        plans.append([(s.rng.randint(0, 100), s.parents()) for _ in range(40)])
    new = [[s.rng.randint(0, 60) for _ in range(40)] for s in servers]
    args = [(_ints([0] * 40), _ints(n)) for n in new]
    outs = [(_ints([0] * 41), _ints([0] * 3000), *[torch.zeros(40, 16, dtype=torch.int32, device="cuda") for _ in range(2)]) for _ in servers]
    parents = [_ints(s.parents()) for s in servers]
    torch.cuda.synchronize()
    for s, stream, a, o, p in zip(servers, streams, args, outs, parents):
        with torch.cuda.stream(stream):
            s.call("assign_shared", *a, tail=o)
            s.call("fork", p)
    torch.cuda.synchronize()
    for s, n, p in zip(servers, new, parents):
        s.ref.assign([0] * 40, n, 3000)
        s.check(s.ref.fork(p.tolist()))


# The same where calls are several launches, which pass what they have found through the workspace: all of them by the number of rows, or
# of pages; fork and compact by the width of the table.
LAUNCHES = [(1100, 9000, 12, 16), (5, 131200, 30, 16), (64, 9000, 193, 16)]


@pytest.mark.parametrize("size", [(1100, 9000, 6, 16), (300, 6000, 60, 16), (5, 131200, 70, 16)], ids=str)
def test_random_steps_of_several_launches_into_arrays_of_their_own(size):
    test_random_steps(size, True)


class Steps:
    """Steps of a server, each a fork, an allocator's step and a compaction, without a look at any result."""

    def __init__(self, size, seed, max_moves):
        self.s = s = Server(*size, seed=seed)
        self.width, self.max_moves = s.shape.max_pages * s.page, max_moves
        s.assign([0] * s.batch, [s.rng.randint(1, 90) for _ in range(s.batch)])
        B = s.batch
        self.parent, self.keep, self.new = _ints(list(range(B))), s.lens.clone(), _ints([0] * B)
        self.q_start, self.slots = _ints([0] * (B + 1)), _ints([0] * (4 * B + 9))
        self.copies = [torch.zeros(B, s.page, dtype=torch.int32, device="cuda") for _ in range(2)]
        self.kept = torch.ones(B, self.width, dtype=torch.bool, device="cuda")
        self.moves = [_ints([0] * max_moves) for _ in range(2)]
        self.ws = [torch.full_like(s.ws, 255) for _ in range(3)]
        self.status = [_ints([9]) for _ in range(3)]

    def draw(self):
        """Arguments of a step into the arrays; what it comes to."""
        s = self.s
        parents = s.parents()
        lens = [s.ref.lens[p] if p >= 0 else 0 for p in parents]
        keeps = [n - min(n, s.rng.randint(0, 3)) for n in lens]
        news = [min(self.width - k, s.rng.randint(0, 4)) for k in keeps]
        marks = torch.rand(s.batch, self.width, generator=torch.Generator().manual_seed(sum(lens))) < 0.9
        for x, y in ((self.parent, _ints(parents)), (self.keep, _ints(keeps)), (self.new, _ints(news)), (self.kept, marks)):
            x.copy_(y)
        return [s.ref.fork(parents), *s.ref.assign(keeps, news, self.slots.numel()), *s.ref.compact(marks.tolist(), self.max_moves)]

    def run(self):
        s = self.s
        t = (s.lens, s.holders, s.ring, s.span, s.table)
        hk.heatkv_paged_fork(s.shape, self.parent, *t, self.status[0], self.ws[0][:-64])
        hk.heatkv_paged_assign_shared(s.shape, self.keep, self.new, *t, self.q_start, self.slots, *self.copies, self.status[1], self.ws[1][:-64])
        hk.heatkv_paged_compact(s.shape, self.kept, *t, *self.moves, self.status[2], self.ws[2][:-64])

    def check(self, want):
        assert [x.item() for x in self.status] == [want[0], want[1], want[5]]
        assert self.q_start.tolist() == want[2] and self.slots.tolist() == want[3]
        assert [[tuple(x) for x in row] for row in torch.stack(self.copies, -1).tolist()] == want[4]
        assert list(zip(*(m.tolist() for m in self.moves))) == want[6]
        assert all(torch.all(w[-64:] == 255) for w in self.ws)
        self.s.status.fill_(want[5])
        self.s.check(want[5])


@pytest.mark.parametrize("size", LAUNCHES, ids=str)
def test_captured_steps_of_several_launches_are_replayed(size):
    p = Steps(size, 31, max_moves=100 * size[0])
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    state = [x.clone() for x in (p.s.lens, p.s.holders, p.s.ring, p.s.span, p.s.table)]
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        p.run()
    for x, y in zip((p.s.lens, p.s.holders, p.s.ring, p.s.span, p.s.table), state):
        assert torch.equal(x, y)  # nothing has run
    for i in range(6):
        want = p.draw()
        graph.replay()
        torch.cuda.synchronize()
        assert want[0] == want[1] == want[5] == 0
        p.check(want)
        if i % 2:  # eager steps of the same cache and workspaces between the replays
            want = p.draw()
            p.run()
            p.check(want)


@pytest.mark.parametrize("size", LAUNCHES, ids=str)
def test_steps_of_several_launches_on_two_streams(size):
    pairs = [(Steps(size, 41 + i, max_moves=100 * size[0]), torch.cuda.Stream()) for i in range(2)]
    for _ in range(3):
        wants = [p.draw() for p, _ in pairs]
        torch.cuda.synchronize()
        for p, stream in pairs:
            with torch.cuda.stream(stream):
                p.run()
        torch.cuda.synchronize()
        for (p, _), want in zip(pairs, wants):
            p.check(want)


# ---- with the rows of the cache -----------------------------------------------------------------------------------------

KINDS = [("bf16", "NATIVE", 64, 16), ("bf16", "FP8_E4M3", 128, 32), ("bf16", "FP4_E2M1", 128, 16), ("f32", "NATIVE", 128, 16),
         ("bf16", "FP4_E2M1", 64, 64)]


def _held(x, fmt):
    if fmt == "FP4_E2M1":
        return sref.fp4_decode(*sref.fp4_encode(x))
    return ref.to_store(x, fmt == "FP8_E4M3").double()


@pytest.mark.parametrize("dtype,fmt,d,page", KINDS, ids=str)
def test_a_servers_steps(dtype, fmt, d, page):
    """Requests that continue others, drop tokens and go on, with rows, bounds and attention, against each request's own list of
    rows: what is shared, copied or moved makes no difference."""
    B, H, G = 6, 2, 2
    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    s = Server(B, 60 * 16 // page + 60, 200 // page + 2, page, seed=d, kv=(H * G, H, d, dtype, getattr(hk, "KV_" + fmt)))
    g = torch.Generator().manual_seed(d)
    store = torch.uint8 if fmt != "NATIVE" else t
    k, v = (torch.full(s.shape.pages_shape, 255 if store is torch.uint8 else math.nan, dtype=store, device="cuda") for _ in range(2))
    bounds = torch.zeros(s.shape.num_pages, H, 2, d, dtype=torch.int8, device="cuda")
    scales = torch.zeros(s.shape.num_pages, H, device="cuda")
    rows = [(torch.zeros(0, H, d, dtype=torch.float64), torch.zeros(0, H, d, dtype=torch.float64)) for _ in range(B)]
    sm = 1 / math.sqrt(d)

    def append(keep, new):
        q_start, slots, frm, to = s.assign(keep, new)
        assert s.status.item() == 0
        n = slots.numel()
        kv = torch.randn(n, 2, H, d, generator=g).to(t)
        dev = kv.cuda()
        hk.heatkv_paged_move(s.shape, frm, to, k, v, bounds, scales)
        hk.heatkv_paged_append(s.shape, slots, dev[:, 0], dev[:, 1], k, v, bounds, scales)
        at = 0
        for b in range(B):
            mine = [_held(kv[at:at + new[b], i], fmt) for i in range(2)]
            rows[b] = tuple(torch.cat([x[:keep[b]], y]) for x, y in zip(rows[b], mine))
            at += new[b]
        q = torch.randn(n, H * G, d, generator=g).to(t)
        out = torch.full((n, H * G, d), 7.0, dtype=t, device="cuda")
        ws = torch.zeros(max(hk.paged_attend_workspace_bytes(s.shape, n), 16), dtype=torch.uint8, device="cuda")
        hk.heatkv_paged_attend(s.shape, q.cuda(), k, v, s.table, q_start, s.lens, sm, out, ws)
        out = out.cpu().double()
        starts = q_start.tolist()
        for b in range(B):
            if not new[b]:
                continue
            ks, vs = rows[b]
            one = [x.transpose(0, 1)[:, None].reshape(H, -1, 1, d).transpose(0, 1).contiguous() for x in (ks, vs)]  # [rows, H, 1, d]
            want, _, mag = ref.attend(q[starts[b]:starts[b + 1]], *one, [list(range(len(ks)))], [0, new[b]], [len(ks)], 1, sm, True)
            S = float(q.double().abs().amax((0, 1)) @ ks.abs().amax((0, 1))) * sm
            e = 2.0 ** -24 * (d * S + 2 * 1.443 * 2 * S + len(ks) + 64)  # as in test_gpu_paged.py
            r, w = (2.0 ** -8, 2.0 ** -8) if dtype == "bf16" else (0.0, 2.0 ** -24)
            off = (out[starts[b]:starts[b + 1]] - want).abs() - (mag * (2 * e + r) * (1 + 1e-6) + w * (want.abs() + mag * (2 * e + r)) + 1e-30)
            assert float(off.max()) <= 0, (b, float(off.max()))
        check_rows()

    def check_rows():
        b_h, s_h = bounds.cpu(), scales.cpu()
        for b in range(B):
            n = s.ref.lens[b]
            assert n == len(rows[b][0])
            if not n:
                continue
            ids = _ints([s.ref.table[b][x // page] * page + x % page for x in range(n)])
            got = [torch.zeros(n, H, d, dtype=t, device="cuda") for _ in range(2)]
            hk.heatkv_paged_read(s.shape, ids, k, v, *got)
            for x, y in zip(got, rows[b]):
                assert torch.equal(x.cpu().double(), y)
            for i, p in enumerate(s.ref.table[b][:pages_of(n, page)]):  # bounds hold for every key (older ones of the page may widen them)
                keys = rows[b][0][i * page:min(n, (i + 1) * page)]
                top = b_h[p].double() * s_h[p][:, None, None].double()
                assert torch.all(keys <= top[:, 0]) and torch.all(-keys <= top[:, 1])

    append([0] * B, [50, 0, 17, 90, 0, 16])
    for step in range(4):
        parent = [0, 0, 2, 3, 3, 5] if step == 0 else s.parents()
        s.fork(parent)
        rows[:] = [rows[p] if p >= 0 else (rows[0][0][:0], rows[0][1][:0]) for p in parent]
        check_rows()
        keep = [n - min(n, s.rng.randint(0, 2)) for n in s.ref.lens]
        append(keep, [s.rng.randint(0, 3) for _ in range(B)])
        marks = [[s.rng.random() < 0.8 or x < 5 for x in range(s.shape.max_pages * page)] for _ in range(B)]
        before = list(s.ref.lens)
        frm, to = s.compact(marks, sum(before))
        assert s.status.item() == 0
        hk.heatkv_paged_move(s.shape, frm, to, k, v, bounds, scales)
        for b in range(B):
            stay = [x for x in range(before[b]) if marks[b][x]]
            rows[b] = tuple(x[stay] for x in rows[b])
        check_rows()
        append(list(s.ref.lens), [1] * B)


# ---- one workgroup or a few launches: both sides of the rules (paged_share.hip) ------------------------------------------

@pytest.mark.parametrize("batch,num_pages,max_pages,page", [(64, 3000, 192, 16), (64, 3000, 193, 16), (768, 5000, 16, 16), (769, 5000, 16, 16), (1024, 5000, 8, 16), (1025, 5000, 8, 16),
                                                            (4, 131072, 8, 16), (4, 131073, 8, 16), (1024, 5000, 32, 16)], ids=str)
def test_forks_and_steps_on_both_sides_of_one_workgroup(batch, num_pages, max_pages, page):
    s = Server(batch, num_pages, max_pages, page, seed=batch + max_pages)
    most = min(max_pages * page, 60 if batch > 100 else 700)
    s.assign([0] * batch, [s.rng.randint(0, most) for _ in range(batch)])
    for tokens in (4096, 4097):
        s.fork(s.parents())
        keep, new = s.step_sizes(2)
        s.assign(keep, new, tokens)
    s.fork([-1] * batch)


@pytest.mark.parametrize("batch,num_pages,max_pages,page", [(1, 3000, 1024, 16), (1, 3000, 1025, 16), (256, 5000, 4, 16), (257, 5000, 3, 16),
                                                            (8, 65536, 8, 256), (8, 65537, 8, 256), (3, 5000, 21, 256), (7, 5000, 18, 128)], ids=str)
def test_requests_thinned_out_on_both_sides_of_one_workgroup(batch, num_pages, max_pages, page):
    s = Server(batch, num_pages, max_pages, page, seed=batch + max_pages)
    room = max_pages * page
    for _ in range(3):
        s.assign(list(s.ref.lens), [s.rng.randint(0, max(0, min(room, 40000 // batch) - n)) for n in s.ref.lens])
        s.fork([s.rng.randrange(batch) if s.rng.random() < 0.3 else b for b in range(batch)])
        s.compact(s.marks(), sum(s.ref.lens) + 3, s.rng.choice((torch.bool, torch.uint8)))
