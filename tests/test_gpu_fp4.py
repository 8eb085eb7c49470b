"""4-bit cache rows (E2M1 codes, a power of two for 32 channels) on the GPU against their definitions in 64 bits: rows written, read
back and moved, page bounds, attention, attention over chosen pages.  What the cache holds is exact in bf16, so attention has the
tolerances of the bf16 cache (test_gpu_paged.py) against the values that are held."""
import math
import random

import pytest
import torch

import paper_2605_14877_amd as hk
from tests import paged_reference as ref
from tests import share_reference as sref
from tests.test_gpu_paged import FEW, MANY, Problem, _check_with_nan, _ints, _spoil

pytestmark = pytest.mark.gpu


def _pack(x):
    """bf16 or fp32 pages [n, H, page, d] -> 4-bit pages and the values that they hold."""
    codes, scales = sref.fp4_encode(x)
    return sref.fp4_pack(codes, scales), sref.fp4_decode(codes, scales)


class Fp4Problem(Problem):
    """Problem with 4-bit pages; k and v are the values that they hold."""

    def __init__(self, q_heads, kv_heads, d, page, lens, new, **more):
        super().__init__("bf16", q_heads, kv_heads, d, page, lens, new, **more)
        self.shape = hk.PagedShape(q_heads, kv_heads, d, page, self.num_pages, len(lens), self.max_pages, "bf16", hk.KV_FP4_E2M1)
        self.store()

    def store(self):
        for name in "kv":
            pages, values = _pack(getattr(self, name))
            setattr(self, name, values.to(torch.bfloat16))
            assert torch.equal(getattr(self, name).double().nan_to_num(7.0), values.nan_to_num(7.0))  # bf16 has them all
            self.dev[name] = pages.cuda()


def _score_error(q, k, sm, keys):
    """e of test_gpu_paged.py's tolerances."""
    d = q.shape[-1]
    S = float(q.abs().double().amax((0, 1)) @ k.double().nan_to_num(0.0).abs().amax((0, 1, 2))) * sm
    return 2.0 ** -24 * (d * S + 2 * 1.443 * 2 * S + keys + 64)


CASES = [c[1:] for c in FEW + MANY if c[0] == "bf16"]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_attention(case, causal):
    p = Fp4Problem(*case, seed=1)
    p.check(causal, p.run(causal))


@pytest.mark.parametrize("new", [[9, 0, 70, 2, 1], [3, 1, 2, 2, 1]])
def test_rows_that_see_nothing_are_zeros(new):
    p = Fp4Problem(2, 1, 64, 16, [4, 0, 20, 0, 0], new, seed=2)
    for causal in (True, False):
        p.check(causal, p.run(causal))


@pytest.mark.parametrize("new", [1, 80])
def test_the_same_call_gives_the_same_bits_and_those_of_the_values_in_bf16(new):
    p = Fp4Problem(8, 2, 128, 16, [2000, 900], [new, 1], seed=4)
    first = p.run(True)
    again = p.run(True)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    # The same products but for the order of the channels within a score: probabilities and their sum differ by e each (as in
    # test_gpu_paged.py), which may turn the rounding of a probability (2^-8) and of the output (a step of 2^-7).
    q = Problem("bf16", 8, 2, 128, 16, [2000, 900], [new, 1], seed=4)
    q.dev.update(k=p.k.cuda(), v=p.v.cuda())
    other = q.run(True)
    real = p.q_start[-1]
    mag, e = float(p.v.double().nan_to_num(0.0).abs().max()), _score_error(p.q[:real], p.k, p.sm, max(p.lens))
    assert float((first[0] - other[0])[:real].double().abs().max()) <= (2.0 ** -8 + 2.0 ** -7 + 4 * e) * mag
    assert float((first[1] - other[1])[:real].abs().max()) <= 2 * e + 2.0 ** -22 * float(other[1][:real].abs().max())


@pytest.mark.parametrize("new", [1, 70])
def test_scores_far_apart_and_rising(new):
    p = Fp4Problem(2, 1, 64, 16, [400], [new], seed=5, scale=3.0)
    for i, page in enumerate(p.table[0]):
        p.k[page] = (p.k[page].float() * (0.2 + 0.1 * i)).to(p.k.dtype)
    p.store()
    p.check(True, p.run(True))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [2, 70])
def test_blocks_of_very_different_sizes(d, new):
    # powers of two from 2^-100 to 2^8 next to one another in a row, zeros, and V up to the largest that there is
    p = Fp4Problem(4, 2, d, 16, [300, 40], [new, 1], seed=6)
    g = torch.Generator().manual_seed(7)
    n = p.k.shape
    power = torch.exp2(torch.randint(-40, 3, (n[0], n[1], n[2], d // 32), generator=g).float()).repeat_interleave(32, -1)
    p.k = (p.k.float() * power).to(torch.bfloat16)
    p.k[:, :, ::3, :32] = p.k[:, :, ::3, :32] * 0.0
    power = torch.exp2(torch.randint(-110, 100, (n[0], n[1], 1, d // 32), generator=g).float()).repeat_interleave(32, -1)
    p.v = (p.v.float() * power).to(torch.bfloat16)
    p.store()
    p.check(True, p.run(True))


@pytest.mark.parametrize("new", [1, 40, 100])
@pytest.mark.parametrize("what", ["k", "v"])
def test_nan_blocks_behind_what_a_row_sees_do_not_reach_it(new, what):
    # the last tokens' blocks are NaN: rows before them do not see them, rows from them on are NaN
    p = Fp4Problem(4, 2, 128, 32, [200, 90], [new, 1], seed=8)
    own = getattr(p, what)
    last = p.lens[0] - 1
    own[p.table[0][last // 32], 1, last % 32, 64:96] = math.nan
    p.store()
    out, lse = p.run(True)
    clean = Fp4Problem(4, 2, 128, 32, [200, 90], [new, 1], seed=8)
    want = clean.run(True)
    t = p.q_start[1] - 1  # the one token that sees it, and its heads
    seen = torch.zeros(p.tokens, 4, dtype=torch.bool, device="cuda")
    seen[t, 2:] = True
    assert torch.equal(lse[~seen], want[1][~seen])
    # A row that shares a tile with the NaN has those columns computed anew, with probabilities that are not rounded to bf16.  Either
    # result is off by A 2 e and half a step of the output (2^-8), the clean one by A 2^-8 as well (test_gpu_paged.py), A <= max |v|.
    e, A = _score_error(p.q, clean.k, p.sm, 200), float(clean.v.double().nan_to_num(0.0).abs().max())
    a, b = out[~seen].double(), want[0][~seen].double()
    assert torch.all((a - b).abs() <= A * (4 * e + 2.0 ** -8) + 2.0 ** -8 * (a.abs() + b.abs()))
    if what == "k":
        assert out[t, 2:].isnan().all() and lse[t, 2:].isnan().all()
    else:
        assert out[t, 2:, 64:96].isnan().all() and not out[t, 2:, :64].isnan().any() and not out[t, 2:, 96:].isnan().any()
        assert torch.equal(lse, want[1])


@pytest.mark.parametrize("d,page,G,new", [(128, 32, 4, 1), (64, 16, 3, 2), (128, 16, 2, 90), (64, 64, 4, 100)])
def test_chosen_pages(d, page, G, new):
    H, lens = 2, [700, 300]
    p = Fp4Problem(G * H, H, d, page, lens, [new, 1], seed=9)
    bounds = torch.zeros(p.num_pages, H, 2, d, dtype=torch.int8)
    scales = torch.zeros(p.num_pages, H)
    for n, ids in zip(lens, p.table):
        for i, x in enumerate(ids):
            for h in range(H):
                b, s = ref.bounds_of(p.k[x, h, :min(page, n - i * page)])
                bounds[x, h], scales[x, h] = b, s
    top = 5
    selected = torch.full((p.tokens, H, top), -7, dtype=torch.int32, device="cuda")
    d_ = p.dev
    hk.heatkv_paged_select(p.shape, d_["q"], bounds.cuda(), scales.cuda(), d_["table"], d_["q_start"], d_["lens"], 1, 2, selected)
    want = ref.select(p.q, bounds, scales, p.table, p.q_start, lens, page, 1, 2, top, True)
    got = selected.cpu()
    for t in range(p.q_start[-1]):
        for h in range(H):
            assert [x for x in got[t, h].tolist() if x >= 0] == want[t][h]
    p.check(True, p.run(True, selected=selected), chosen=got.tolist())


# ---- rows ---------------------------------------------------------------------------------------------------------------

def _values(shape, seed):
    """bf16 values with everything that a block can have."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    b = x.unflatten(-1, (-1, 32))
    n = b.shape[:-1]
    b *= torch.exp2(torch.randint(-20, 20, n, generator=g).float())[..., None]
    kind = torch.randint(0, 14, n, generator=g)
    b[kind == 0] = 0.0
    b[kind == 1] *= 2.0 ** -110                       # under the least power
    b[kind == 2] *= 2.0 ** 110                        # over the largest
    b[kind == 3] = torch.round(b[kind == 3] * 4) / 4 * 0.25  # many in the middle between two codes
    quarters = torch.randint(-28, 29, b[kind == 4].shape, generator=g).float() / 4
    b[kind == 4] = quarters
    k = torch.nonzero(kind == 5)
    for i, at in enumerate(k[:40]):
        b[tuple(at)][i % 32] = [math.inf, -math.inf, math.nan, 3.3895e38][i % 4]
    k = torch.nonzero(kind == 6)
    b[kind == 6] = 0.01
    for i, at in enumerate(k):                       # around 7 times a power of two
        b[tuple(at)][3] = [7.0, 7.03125, 6.96875, -7.0][i % 4] * 2.0 ** (i % 9 - 4)
    return b.flatten(-2).to(torch.bfloat16)


def _cache(H, d, page, num_pages, batch=1, max_pages=1):
    shape = hk.PagedShape(H, H, d, page, num_pages, batch, max_pages, "bf16", hk.KV_FP4_E2M1)
    k, v = (torch.randint(0, 200, shape.pages_shape, dtype=torch.uint8, generator=torch.Generator().manual_seed(i)).cuda() for i in (1, 2))
    return shape, k, v


def _same(got, want):
    return torch.equal(got.double().cpu().nan_to_num(7e300), want.nan_to_num(7e300)) and torch.equal(got.isnan().cpu(), want.isnan())


@pytest.mark.parametrize("bounds", [False, True])
@pytest.mark.parametrize("H,d,page,tokens", [(1, 64, 16, 1), (3, 128, 16, 70), (2, 64, 32, 300), (2, 128, 256, 400), (5, 64, 128, 999),
                                             (8, 128, 64, 700)])
def test_rows_are_written_and_read_back(H, d, page, tokens, bounds):
    num_pages = ref.pages_of(tokens, page) + 2
    shape, k, v = _cache(H, d, page, num_pages)
    before = [k.cpu().clone(), v.cpu().clone()]
    order = torch.randperm(num_pages, generator=torch.Generator().manual_seed(5)).tolist()
    start = 5 if tokens > 5 else 0  # the first page's older rows stay, and are in its bounds
    slots = [order[x // page] * page + x % page for x in range(start, start + tokens)]
    qkv = _values((tokens + 3, 2 * H + 1, d), seed=tokens)
    dev = qkv.cuda()
    b = torch.full((num_pages, H, 2, d), 77, dtype=torch.int8, device="cuda") if bounds else None
    s = torch.full((num_pages, H), 77.0, device="cuda") if bounds else None
    ids = _ints(slots + [-1, num_pages * page, -5])
    hk.heatkv_paged_append(shape, ids, dev[:, :H], dev[:, H:2 * H], k, v, b, s)
    want = []
    for name, pages, x in (("k", before[0], qkv[:tokens, :H]), ("v", before[1], qkv[:tokens, H:2 * H])):
        codes, scales = sref.fp4_unpack(pages, page, d)
        c, e = sref.fp4_encode(x)
        at, r = torch.tensor(slots) // page, torch.tensor(slots) % page
        codes[at, :, r], scales[at, :, r] = c, e
        got_c, got_e = sref.fp4_unpack((k if name == "k" else v).cpu(), page, d)
        assert torch.equal(got_e, scales)
        number = (scales != 255).repeat_interleave(32, -1)
        assert torch.equal(got_c[number], codes[number])
        want.append(sref.fp4_decode(codes, scales))
    out = torch.full((tokens + 3, 2 * H + 1, d), 5.0, dtype=torch.bfloat16, device="cuda")
    hk.heatkv_paged_read(shape, ids, k, v, out[:, :H], out[:, H:2 * H])
    at, r = torch.tensor(slots) // page, torch.tensor(slots) % page
    assert _same(out[:tokens, :H], want[0][at, :, r]) and _same(out[:tokens, H:2 * H], want[1][at, :, r])
    assert torch.all(out[tokens:] == 5.0) and torch.all(out[:, 2 * H:] == 5.0)
    if bounds:
        b, s = b.cpu(), s.cpu()
        last = {}
        for x in slots:
            last[x // page] = max(last.get(x // page, 0), x % page + 1)
        for p in range(num_pages):
            for h in range(H):
                if p not in last:
                    assert torch.all(b[p, h] == 77) and s[p, h] == 77
                    continue
                codes, scale = ref.bounds_of(want[0][p, h, :last[p]])
                assert torch.equal(b[p, h], codes) and s[p, h] == scale, (p, h)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 60])  # the 16-row kernel, the 128-row kernel
def test_every_code_under_every_scale_byte(d, new):
    """Pages from elsewhere: numbers of the bf16 range are exact, its smallest ones among them, those beyond are infinite.  One key of
    a request is seen by its first token: the output is its V."""
    H, page, blocks = 8, 64, d // 32
    B = 256 // (H * blocks)
    codes = (torch.arange(d) % 16).expand(B, H, page, d).contiguous()
    scales = torch.arange(256).view(B, H, 1, blocks).expand(B, H, page, blocks).contiguous()
    v = sref.fp4_pack(codes, scales).cuda()
    shape = hk.PagedShape(H, H, d, page, B, B, 1, "bf16", hk.KV_FP4_E2M1)
    k = torch.zeros_like(v)
    want = sref.fp4_decode(codes, scales)
    want = torch.where(want.abs() >= 2.0 ** 128, torch.copysign(torch.tensor(math.inf, dtype=torch.float64), want), want)
    assert torch.equal(want.to(torch.bfloat16).double().nan_to_num(7e300), want.nan_to_num(7e300))  # bf16 has them all
    rows = [torch.zeros(B * page, H, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    hk.heatkv_paged_read(shape, _ints(list(range(B * page))), k, v, *rows)
    assert _same(rows[1].view(B, page, H, d).transpose(1, 2), want)
    out = torch.full((B * new, H, d), 5.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(max(hk.paged_attend_workspace_bytes(shape, B * new), 16), dtype=torch.uint8, device="cuda")
    q = torch.randn(B * new, H, d, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    hk.heatkv_paged_attend(shape, q, k, v, _ints([[b] for b in range(B)]), _ints([b * new for b in range(B + 1)]), _ints([new] * B), 0.1,
                           out, ws)
    assert _same(out.view(B, new, H, d)[:, 0], want[:, :, 0])


@pytest.mark.parametrize("dtype,fmt", [("f32", "NATIVE"), ("bf16", "NATIVE"), ("bf16", "FP8_E4M3"), ("bf16", "FP4_E2M1")])
@pytest.mark.parametrize("d,page,bounds", [(64, 16, False), (128, 32, False), (64, 32, True), (128, 256, True), (128, 16, True)])
def test_rows_are_moved_as_they_are(dtype, fmt, d, page, bounds):
    H, num_pages = 3, 40
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    shape = hk.PagedShape(H, H, d, page, num_pages, 1, 1, dtype, getattr(hk, "KV_" + fmt))
    g = torch.Generator().manual_seed(3)
    store = t if fmt == "NATIVE" else torch.uint8
    bytes_ = torch.randint(0, 120, (*shape.pages_shape[:-1], shape.pages_shape[-1] * (t.itemsize if store is t else 1)),
                           dtype=torch.uint8, generator=g)
    k = bytes_.view(store).cuda().contiguous()
    v = bytes_.flip(0).contiguous().view(store).cuda()
    # runs of rows, single rows, whole pages, in the order of their new places
    half = num_pages // 2 * page
    to, frm = [], []
    for p in range(num_pages // 2, num_pages, 2):
        n = [1, page, page // 2 + 1, 3][p // 2 % 4]
        to += [p * page + i for i in range(n)]
        frm += torch.randint(0, half, (n,), generator=g).tolist()
    to += [-1, num_pages * page, -9]
    frm += [0, 1, 2]
    b = torch.full((num_pages, H, 2, d), 77, dtype=torch.int8, device="cuda") if bounds else None
    s = torch.full((num_pages, H), 77.0, device="cuda") if bounds else None
    read = [torch.zeros(num_pages * page, H, d, dtype=t, device="cuda") for _ in range(2)]
    every = torch.arange(num_pages * page, dtype=torch.int32, device="cuda")
    hk.heatkv_paged_read(shape, every, k, v, *read)
    want = [x.clone() for x in read]
    for x in want:
        x[to[:-3]] = x[frm[:-3]]
    hk.heatkv_paged_move(shape, _ints(frm), _ints(to), k, v, b, s)
    hk.heatkv_paged_read(shape, every, k, v, *read)
    for x, y in zip(read, want):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    if bounds:
        values = want[0].cpu().view(num_pages, page, H, d)
        last = {}
        for x in to[:-3]:
            last[x // page] = max(last.get(x // page, 0), x % page + 1)
        for p in range(num_pages):
            for h in range(H):
                if p in last:
                    codes, scale = ref.bounds_of(values[p, :last[p], h])
                    assert torch.equal(b[p, h].cpu(), codes) and s[p, h] == scale, (p, h)
                else:
                    assert torch.all(b[p, h] == 77) and s[p, h] == 77


@pytest.mark.parametrize("dtype,fmt", [("f32", "NATIVE"), ("bf16", "FP8_E4M3")])
def test_rows_of_other_formats_are_read_as_values(dtype, fmt):
    H, d, page, n = 2, 64, 32, 3
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    shape = hk.PagedShape(H, H, d, page, n, 1, 1, dtype, getattr(hk, "KV_" + fmt))
    x = torch.randn(shape.pages_shape, generator=torch.Generator().manual_seed(1)).to(t)
    pages = ref.to_store(x, fmt != "NATIVE")
    out = torch.zeros(n * page, 2, H, d, dtype=t, device="cuda")
    ids = torch.randperm(n * page, generator=torch.Generator().manual_seed(2)).to(torch.int32)
    hk.heatkv_paged_read(shape, ids.cuda(), pages.cuda(), pages.cuda(), out[:, 0], out[:, 1])
    want = pages.to(t).transpose(1, 2).reshape(n * page, H, d)[ids.long()]
    assert torch.equal(out[:, 0].cpu(), want) and torch.equal(out[:, 1].cpu(), want)


@pytest.mark.parametrize("bounds", [False, True])
def test_a_list_of_more_rows_than_a_call_takes_is_moved_in_pieces(bounds):
    H, d, page, rows = 64, 64, 256, (1 << 23) // 64 + 300
    half = ref.pages_of(rows, page)
    shape = hk.PagedShape(H, H, d, page, 2 * half, 1, 1, "bf16", hk.KV_FP4_E2M1)
    g = torch.Generator(device="cuda").manual_seed(4)
    first = [torch.randint(0, 252, shape.pages_shape, dtype=torch.uint8, device="cuda", generator=g) for _ in range(2)]
    to = _ints(list(range(half * page, half * page + rows)))
    frm = torch.randperm(rows, device="cuda", generator=g).int()

    def moved(cuts):
        k, v = (x.clone() for x in first)
        b, s = (torch.full(n, 77, dtype=t, device="cuda") for n, t in (((2 * half, H, 2, d), torch.int8), ((2 * half, H), torch.float32)))
        for i, j in zip([0, *cuts], [*cuts, rows]):
            hk.heatkv_paged_move(shape, frm[i:j], to[i:j], k, v, *((b, s) if bounds else ()))
        return k, v, b, s

    with pytest.raises(hk.HeatKVError, match="2\\^23"):
        moved([])
    want = moved([half // 2 * page])  # cut between two pages
    for cuts in ([300], [1 << 17], [half // 2 * page - 131, half // 2 * page - 126, half // 2 * page + 7]):  # within; a few rows alone
        assert all(torch.equal(x, y) for x, y in zip(moved(cuts), want))
    ids = torch.tensor([0, 1, 255, 256, half // 2 * page - 1, rows - 301, rows - 1], device="cuda")
    got, old = ([torch.zeros(len(ids), H, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2))
    hk.heatkv_paged_read(shape, to[ids], *want[:2], *got)
    hk.heatkv_paged_read(shape, frm[ids], *first, *old)
    assert all(torch.equal(x, y) for x, y in zip(got, old))


def test_addresses_beyond_32_bits():
    # 4-bit pages of more than 4 GiB each; the request's tokens on the last of them
    H, d, page = 8, 128, 256
    num_pages = (1 << 32) // (H * page * 68) + 40
    shape = hk.PagedShape(H, H, d, page, num_pages, 1, 4, "bf16", hk.KV_FP4_E2M1)
    k, v = (torch.zeros(shape.pages_shape, dtype=torch.uint8, device="cuda") for _ in range(2))
    assert k.numel() > 1 << 32
    n = 700
    x = torch.randn(2, n, H, d, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    ids = [num_pages - 1, num_pages - 9, num_pages - 4]
    slots = _ints([ids[i // page] * page + i % page for i in range(n)])
    hk.heatkv_paged_append(shape, slots, x[0].cuda(), x[1].cuda(), k, v)
    got = torch.zeros(2, n, H, d, dtype=torch.bfloat16, device="cuda")
    hk.heatkv_paged_read(shape, slots, k, v, got[0], got[1])
    held = [sref.fp4_decode(*sref.fp4_encode(y)) for y in x]
    assert _same(got[0], held[0]) and _same(got[1], held[1])
    small = [torch.zeros(3 * page, H, d).index_copy_(0, torch.arange(n), y.float()).view(3, page, H, d).transpose(1, 2) for y in held]
    for new in (1, 90):
        q = torch.randn(new, H, d, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
        out = torch.zeros(new, H, d, dtype=torch.bfloat16, device="cuda")
        ws = torch.zeros(max(hk.paged_attend_workspace_bytes(shape, new), 16), dtype=torch.uint8, device="cuda")
        hk.heatkv_paged_attend(shape, q.cuda(), k, v, _ints([ids + [0]]), _ints([0, new]), _ints([n]), 0.09, out, ws)
        want, _, mag = ref.attend(q, *small, [[0, 1, 2]], [0, new], [n], page, 0.09, True)
        r = 2.0 ** -8 + 2 * _score_error(q, small[0], 0.09, n)
        off = (out.cpu().double() - want).abs() - (mag * r * (1 + 1e-6) + 2.0 ** -8 * (want.abs() + mag * r))
        assert float(off.max()) <= 0
    frm, to = slots[:3], _ints([5, 6, 7])
    hk.heatkv_paged_move(shape, frm, to, k, v)
    hk.heatkv_paged_read(shape, to, k, v, got[0, :3], got[1, :3])
    assert _same(got[0, :3], held[0][:3]) and _same(got[1, :3], held[1][:3])


# ---- what tiles have in common, calls of any content, graphs ------------------------------------------------------------

def _spoiled(case, seed, last_only):
    p = Fp4Problem(*case, seed=seed)
    p.dtype = "fp8"  # of values that are not finite only NaN: 4 bits have no infinity
    _spoil(p, seed, last_only)
    p.store()
    return p


@pytest.mark.parametrize("case", [(4, 2, 128, 16, [50, 33], [20, 5]), (2, 1, 64, 32, [400], [90]), (6, 1, 128, 64, [700, 65], [40, 30]),
                                  (4, 2, 64, 16, [50, 300], [20, 70]), (8, 1, 128, 16, [2000], [4])], ids=str)
def test_values_that_a_row_does_not_see_do_not_reach_it(case):
    p = _spoiled(case, 11, True)
    fine = _check_with_nan(p, True, p.run(True))
    last = [s - 1 for s in p.q_start[1:]]
    assert fine[[t for t in range(p.q_start[-1]) if t not in last]].all() and not fine[last].all()
    p = _spoiled(case, 12, False)
    for causal in (True, False):
        _check_with_nan(p, causal, p.run(causal))


@pytest.mark.parametrize("case,top", [((4, 2, 128, 16, [300, 33], [6, 5]), 4), ((4, 1, 64, 32, [400], [90]), 4),
                                      ((4, 2, 128, 16, [50, 300], [20, 70]), 4), ((4, 1, 128, 64, [3000, 900], [90, 70]), 9),
                                      ((4, 2, 64, 128, [2600], [200]), 2)], ids=str)
def test_pages_that_a_token_has_not_chosen_do_not_reach_it(case, top):
    p = _spoiled(case, 13, False)
    r = random.Random(5)
    pages = max(p.lens) // p.page + 1
    sel = [[[r.randrange(0, pages) for _ in range(top)] for _ in range(p.H)] for _ in range(p.tokens)]
    for causal in (True, False):
        fine = _check_with_nan(p, causal, p.run(causal, _ints(sel)), sel)
        assert fine.any() and not fine.all()


@pytest.mark.parametrize("new", [[4, 19, 1], [150, 70, 1]])
@pytest.mark.parametrize("group,d", [(1, 64), (3, 128), (16, 64), (16, 128)])
def test_selections_of_any_content(group, d, new):
    p = Fp4Problem(2 * group, 2, d, 16, [333, 100, 5], new, seed=9)
    top, r = 6, random.Random(3)
    sel = [[[r.choice([-1, -7, 2 ** 31 - 1, r.randrange(0, 25), r.randrange(0, 25), r.randrange(0, 8)]) for _ in range(top)]
            for _ in range(2)] for _ in range(p.tokens)]
    sel[0][0], sel[1][1], sel[2][0] = [-1] * top, [3] * top, [24, 23, 22, 21, 20, 0]
    for t in range(20, min(150, p.tokens)):
        sel[t][1] = [-1] * top  # a tile without any page
    for causal in (True, False):
        p.check(causal, p.run(causal, _ints(sel)), sel)


@pytest.mark.parametrize("heads,top", [((4, 2), 0), ((3, 1), 0), ((4, 2), 3)])
@pytest.mark.parametrize("batch", [64, 65, 1000])
def test_many_requests(heads, top, batch):
    r = random.Random(batch)
    lens = [r.choice((0, 1, 15, 16, 17, 40, 90)) for _ in range(batch)]
    new = [min(n, r.choice((0, 1, 1, 1, 20))) for n in lens]
    p = Fp4Problem(*heads, 64, 16, lens, new, seed=batch)
    sel = [[[r.randrange(0, 6) for _ in range(top)] for _ in range(p.H)] for _ in range(p.tokens)] if top else None
    p.check(True, p.run(True, _ints(sel) if top else None), sel)


@pytest.mark.parametrize("dtype", ["fp4", "fp8", "bf16"])
@pytest.mark.parametrize("d,group", [(64, 1), (128, 4)])
@pytest.mark.parametrize("batch", [2, 32, 33, 130])
def test_few_and_many_rows_in_one_call(dtype, d, group, batch):
    # one launch has both, in either order (up to 32 requests and beyond): tokens that decode, drafts, prompts, requests without work
    r = random.Random(batch)
    lens = [r.choice((1, 30, 300, 1200)) for _ in range(batch)]
    new = [min(n, r.choice((0, 1, 1, 1, 5, 20))) for n in lens]
    lens[-1], new[-1] = 500, 170
    case = (2 * group, 2, d, 16, lens, new)
    p = Fp4Problem(*case, seed=batch) if dtype == "fp4" else Problem(dtype, *case, seed=batch)
    for causal in (True, False):
        first, again = p.run(causal), p.run(causal)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
        p.check(causal, first)
    sel = [[[r.randrange(0, 60) for _ in range(4)] for _ in range(p.H)] for _ in range(p.tokens)]
    p.check(True, p.run(True, _ints(sel)), sel)


@pytest.mark.parametrize("dtype", ["fp4", "fp8", "bf16"])
@pytest.mark.parametrize("d,max_pages,top", [(128, 1000, 8), (64, 3000, 24)])
@pytest.mark.parametrize("batch", [5, 40])
def test_few_and_many_rows_beside_a_large_union(dtype, d, max_pages, top, batch):
    # the union of a tile's pages leaves room for one workgroup on a compute unit: two launches, or one with few rows first
    r = random.Random(batch)
    lens = [r.choice((1, 30, 300, 1200)) for _ in range(batch)]
    new = [min(n, r.choice((0, 1, 1, 1, 5, 20))) for n in lens]
    lens[-1], new[-1] = 500, 170
    case = (2, 2, d, 16, lens, new)
    p = Fp4Problem(*case, seed=batch, max_pages=max_pages) if dtype == "fp4" else Problem(dtype, *case, seed=batch, max_pages=max_pages)
    sel = [[[r.randrange(0, 60) for _ in range(top)] for _ in range(p.H)] for _ in range(p.tokens)]
    first, again = p.run(True, _ints(sel)), p.run(True, _ints(sel))
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    p.check(True, first, sel)


@pytest.mark.parametrize("dtype", ["fp4", "fp8", "bf16", "f32"])
@pytest.mark.parametrize("batch,heads,new", [(1, 8, 240), (3, 8, 256), (10, 8, 240), (64, 8, 1), (64, 21, 1), (63, 20, 2), (64, 1, 17), (65, 8, 1),
                                             (8, 64, 30)])
def test_short_caches_of_many_segments(dtype, batch, heads, new):
    # none is cut: a workgroup to a segment up to 64 requests and 2560 segments, else up to 512 of them
    r = random.Random(batch)
    lens = [r.randint(new, 256) for _ in range(batch)]
    case = (2 * heads, heads, 64, 16, lens, [r.choice((new, new, max(new // 2, 1), 0)) for _ in range(batch)])
    p = Fp4Problem(*case, seed=batch, max_pages=16) if dtype == "fp4" else Problem(dtype, *case, seed=batch, max_pages=16)
    for causal in (True, False):
        p.check(causal, p.run(causal))


@pytest.mark.parametrize("case,top", [(c, 0) for c in CASES[3:9] + CASES[-4:]] + [
    ((4, 2, 64, 16, [n for n in (900, 300, 40) for _ in range(30)], [n for n in (1, 2, 70) for _ in range(30)]), 0),
    ((8, 8, 64, 32, [2000] * 40, [1] * 40), 6), ((4, 2, 128, 64, [3000, 900], [90, 70]), 9)], ids=lambda x: str(x)[:50])
def test_nothing_is_written_behind_the_workspace(case, top):
    p = Fp4Problem(*case, seed=35)
    d, n, guard = p.dev, hk.paged_attend_workspace_bytes(p.shape, p.tokens, top), 1 << 16
    ws = torch.full((n + guard,), 165, dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(d["q"])
    args = (p.shape, d["q"], d["k"], d["v"], d["table"], d["q_start"], d["lens"])
    r = random.Random(35)
    for causal in (True, False):
        if top:
            sel = _ints([[[r.randrange(0, p.max_pages) for _ in range(top)] for _ in range(p.H)] for _ in range(p.tokens)])
            hk.heatkv_paged_attend_selected(*args, sel, p.sm, out, ws[:n], causal=causal)
        else:
            hk.heatkv_paged_attend(*args, p.sm, out, ws[:n], causal=causal)
    torch.cuda.synchronize()
    assert torch.all(ws[n:] == 165)


@pytest.mark.parametrize("new", [2, 70])
def test_rows_may_be_slices_with_any_stride(new):
    p = Fp4Problem(4, 2, 64, 16, [90, 33], [new, 1], seed=3)
    want = p.run(True)
    wide = torch.full((p.tokens, 7, 80), 9.0, dtype=p.q.dtype, device="cuda")
    q = wide[:, 2:6, 8:72]
    q.copy_(p.dev["q"])
    by_head = torch.full((6, p.tokens + 1, 64), 7.0, dtype=p.q.dtype, device="cuda")
    got = p.run(True, out=by_head.transpose(0, 1)[:p.tokens, 1:5], q=q)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.all(by_head[0] == 7.0) and torch.all(by_head[5] == 7.0) and torch.all(by_head[:, p.tokens:] == 7.0)


@pytest.mark.parametrize("new", [1, 60])
def test_a_captured_step_is_replayed(new):
    """Rows in, bounds, read back, the choice, attention over all and over chosen pages, rows moved: one graph, replayed for new rows
    with eager calls in between."""
    p = Fp4Problem(4, 2, 128, 16, [300, 90], [new, 1], seed=20)
    d, n = p.dev, p.q_start[-1]
    slots = [p.table[b][x // 16] * 16 + x % 16 for b in range(2) for x in range(p.lens[b] - p.new[b], p.lens[b])]
    slots = _ints(slots + [-1] * (p.tokens - n))
    kv = torch.zeros(p.tokens, 4, 128, dtype=torch.bfloat16, device="cuda")
    bounds = torch.zeros(p.num_pages, 2, 2, 128, dtype=torch.int8, device="cuda")
    scales = torch.zeros(p.num_pages, 2, device="cuda")
    spare = [x for x in range(p.num_pages) if not any(x in r for r in p.table)]
    to = _ints([spare[0] * 16 + i for i in range(7)])

    def state():
        return dict(k=d["k"].clone(), v=d["v"].clone(), bounds=bounds.clone(), scales=scales.clone(),
                    read=[torch.zeros(p.tokens, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)],
                    sel=torch.zeros(p.tokens, 2, 5, dtype=torch.int32, device="cuda"), out=[torch.zeros_like(d["q"]) for _ in range(2)],
                    ws=torch.zeros(max(hk.paged_attend_workspace_bytes(p.shape, p.tokens, t) for t in (0, 5)) + 16, dtype=torch.uint8,
                                   device="cuda"))

    def step(s):
        more = (d["table"], d["q_start"], d["lens"])
        hk.heatkv_paged_append(p.shape, slots, kv[:, :2], kv[:, 2:], s["k"], s["v"], s["bounds"], s["scales"])
        hk.heatkv_paged_read(p.shape, slots, s["k"], s["v"], *s["read"])
        hk.heatkv_paged_attend(p.shape, d["q"], s["k"], s["v"], *more, p.sm, s["out"][0], s["ws"])
        hk.heatkv_paged_select(p.shape, d["q"], s["bounds"], s["scales"], *more, 1, 1, s["sel"])
        hk.heatkv_paged_attend_selected(p.shape, d["q"], s["k"], s["v"], *more, s["sel"], p.sm, s["out"][1], s["ws"])
        hk.heatkv_paged_move(p.shape, slots[:1].expand(7).contiguous(), to, s["k"], s["v"], s["bounds"], s["scales"])
    captured, eager = state(), state()
    step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step(captured)
    for turn in range(4):
        kv.copy_(torch.randn(kv.shape, generator=torch.Generator().manual_seed(turn)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        for name in ("k", "v", "bounds", "scales", "sel"):
            assert torch.equal(captured[name], eager[name]), name
        for name in ("read", "out"):
            assert all(torch.equal(x, y) for x, y in zip(captured[name], eager[name])), name


def test_the_native_path_makes_the_calls(monkeypatch):
    """Plain calls do not reach the Python checks; malformed ones do, and are named there."""
    from paper_2605_14877_amd import paged
    H, d, page, n, B = 2, 64, 16, 40, 3
    shape = hk.PagedShape(2 * H, H, d, page, n, B, 8, "bf16", hk.KV_FP4_E2M1)
    k, v = (torch.zeros(shape.pages_shape, dtype=torch.uint8, device="cuda") for _ in range(2))
    rows = torch.zeros(4, H, d, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros(4, 2, H, d, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(4, 2 * H, d, dtype=torch.bfloat16, device="cuda")
    bounds, scales = torch.zeros(n, H, 2, d, dtype=torch.int8, device="cuda"), torch.zeros(n, H, device="cuda")
    tables = [_ints([0] * B), _ints([0] * n), _ints(list(range(n))), _ints([0, n]), _ints([[0] * 8] * B)]  # lens, holders, ring, span, table
    ws = torch.zeros(hk.paged_tables_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    status, some, moves = _ints([0]), _ints([0] * B), _ints([-1] * 9)
    copies = [_ints([[0] * page] * B) for _ in range(2)]
    kept = torch.ones(B, 8 * page, dtype=torch.bool, device="cuda")
    kept_bytes = kept.to(torch.uint8)
    att = torch.zeros(max(hk.paged_attend_workspace_bytes(shape, 4), 16), dtype=torch.uint8, device="cuda")
    calls = {
        "append": lambda k=k: hk.heatkv_paged_append(shape, moves[:4], rows, rows, k, v, bounds, scales),
        "read": lambda k=k: hk.heatkv_paged_read(shape, moves[:4], k, v, out[:, 0], out[:, 1]),
        "attend": lambda k=k: hk.heatkv_paged_attend(shape, q, k, v, tables[4], _ints([0] * 4), tables[0], 0.1, torch.zeros_like(q), att),
        "move": lambda k=k: hk.heatkv_paged_move(shape, moves, moves.clone(), k, v, bounds, scales),
        "move of copies": lambda k=k: hk.heatkv_paged_move(shape, *copies, k, v),
        "fork": lambda k=some: hk.heatkv_paged_fork(shape, k, *tables, status, ws),
        "assign_shared": lambda k=some: hk.heatkv_paged_assign_shared(shape, some, k, *tables, _ints([0] * (B + 1)), moves.clone(), *copies, status, ws),
        "compact": lambda k=kept: hk.heatkv_paged_compact(shape, k, *tables, moves, moves.clone(), status, ws,
                                                          lens_out=_ints([0] * B), free_span_out=_ints([0, 0])),
    }
    for call in calls.values():  # by the native path or the other, they are made
        call()

    def reached(*_):
        raise AssertionError("the call went through the Python checks")
    monkeypatch.setattr(paged, "_Call", reached)
    for call in calls.values():
        call()
    calls["compact"](kept_bytes)
    monkeypatch.undo()
    torch.cuda.synchronize()
    wrong = {"append": k[:-1], "read": k.view(torch.int8), "attend": k.cpu(), "move": k.view(n, H, -1, 68), "move of copies": k[:, :1],
             "fork": some.long(), "assign_shared": some[:2], "compact": kept[:, :-1]}
    for name, x in wrong.items():
        with pytest.raises((ValueError, TypeError)):
            calls[name](x)


def test_a_value_that_is_not_a_number_does_not_stall_a_call():
    # NaN in V of a key that all rows see: their results are NaN as they stand (as for the other formats: test_gpu_paged.py)
    p = Fp4Problem(4, 1, 128, 64, [4096], [300], seed=31)
    d, out = p.dev, torch.empty_like(p.dev["q"])
    ws = torch.zeros(max(hk.paged_attend_workspace_bytes(p.shape, p.tokens), 16), dtype=torch.uint8, device="cuda")
    clean = d["v"]
    p.v[p.table[0][32], :, 3, 5] = math.nan
    p.store()

    def least(v):
        times = []
        for _ in range(20):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            torch.cuda.synchronize()
            a.record()
            hk.heatkv_paged_attend(p.shape, d["q"], d["k"], v, d["table"], d["q_start"], d["lens"], p.sm, out, ws)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)
    usual = least(clean)
    assert least(d["v"]) < 3 * usual
    real = p.q_start[-1]
    assert out[:real, :, :32].isnan().all() and out[:real, :, 32:].isfinite().all()
