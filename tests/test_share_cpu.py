"""CPU-side checks of 4-bit rows and of pages that several requests hold: refusals of the C ABI before any GPU work, the binding's
messages, and the references of the GPU tests against closed forms.  No GPU needed."""
import math
import random

import pytest
import torch

import paper_2605_14877_amd as hk
from paper_2605_14877_amd import paged
from tests import share_reference as sref
from tests.test_paged_cpu import BAD_SHAPES, _fail, _shape, rules  # noqa: F401

at = lambda i: (i + 1) << 36  # noqa: E731  addresses are never followed: every call is refused
TOKENS, MOVES = 4, 9
TABLES = ("lens", "lens_out", "holders", "free_ring", "free_span", "free_span_out", "table")
# name: arrays in the order of the C entry, those that it writes, its call
CALLS = {
    "fork": (("parent", *TABLES, "status", "ws"), ("lens_out", "holders", "free_ring", "free_span_out", "table", "status", "ws"),
             lambda L, sh, a, n: L.heatkv_paged_fork(sh.ref, *[a[x] for x in ("parent", *TABLES, "status", "ws")], n, None)),
    "assign_shared": (("keep", "new_tokens", *TABLES, "q_start", "slots", "copy_from", "copy_to", "status", "ws"),
                      ("lens_out", "holders", "free_ring", "free_span_out", "table", "q_start", "slots", "copy_from", "copy_to",
                       "status", "ws"),
                      lambda L, sh, a, n: L.heatkv_paged_assign_shared(
                          sh.ref, *[a[x] for x in ("keep", "new_tokens", *TABLES, "q_start", "slots")], TOKENS, a["copy_from"],
                          a["copy_to"], a["status"], a["ws"], n, None)),
    "compact": (("kept", *TABLES, "move_from", "move_to", "status", "ws"),
                ("lens_out", "holders", "free_ring", "free_span_out", "table", "move_from", "move_to", "status", "ws"),
                lambda L, sh, a, n: L.heatkv_paged_compact(sh.ref, *[a[x] for x in ("kept", *TABLES, "move_from", "move_to")], MOVES,
                                                           a["status"], a["ws"], n, None)),
    "move": (("move_from", "move_to", "k_pages", "v_pages", "bounds", "bound_scales"), ("k_pages", "v_pages", "bounds", "bound_scales"),
             lambda L, sh, a, n: L.heatkv_paged_move(sh.ref, a["move_from"], a["move_to"], MOVES, a["k_pages"], a["v_pages"],
                                                     a["bounds"], a["bound_scales"], None)),
    "read": (("slots", "k_pages", "v_pages", "k_out", "v_out"), ("k_out", "v_out"),
             lambda L, sh, a, n: L.heatkv_paged_read(sh.ref, a["slots"], TOKENS, a["k_pages"], a["v_pages"],
                                                     paged._CRows(a["k_out"], 512, 128), paged._CRows(a["v_out"], 512, 128), None)),
}


def _sizes(sh):
    row, heads = 4 * sh.batch, sh.num_pages * sh.kv_heads
    pages = math.prod(sh.pages_shape) * (1 if sh.kv_format else 2)
    rows = ((TOKENS - 1) * 512 + 128 + 128) * 2
    return dict(parent=row, keep=row, new_tokens=row, lens=row, lens_out=row, holders=4 * sh.num_pages, free_ring=4 * sh.num_pages,
                free_span=8, free_span_out=8, table=row * sh.max_pages, status=4, q_start=row + 4, slots=4 * TOKENS,
                copy_from=row * sh.page_size, copy_to=row * sh.page_size, kept=sh.batch * sh.max_pages * sh.page_size,
                move_from=4 * MOVES, move_to=4 * MOVES, k_pages=pages, v_pages=pages, bounds=heads * 2 * sh.d, bound_scales=heads * 4,
                k_out=rows, v_out=rows, ws=hk.paged_tables_workspace_bytes(sh))


def _apart(names):
    return {n: at(i) for i, n in enumerate(names)}


@pytest.mark.parametrize("change,match", [x for x in BAD_SHAPES if "kv_format" not in x[0]] + [
    (dict(kv_format=hk.KV_FP4_E2M1, dtype="f32"), "FP4_E2M1 needs a bf16 shape"), (dict(kv_format=3), "storage format"),
    (dict(kv_format=5), "storage format")], ids=str)
def test_shapes_that_do_not_fit_are_refused(change, match):
    L, sh = paged._lib(), _shape(**change)
    assert hk.paged_tables_workspace_bytes(sh) == 0
    for names, _, call in CALLS.values():
        _fail(call(L, sh, _apart(names), 1 << 40), match)


def test_only_the_paged_cache_has_4_bit_rows():
    import numpy as np
    shape = hk.Shape(1, 2, 128, [1, 4, 16], 1, "bf16")
    with pytest.raises(hk.HeatKVError, match="storage format"):
        hk.heatkv_build_schedule(shape, np.ones((1, 2, 3, 3), np.float32), 1 << 20, 1, kv_format=hk.KV_FP4_E2M1)


def test_pages_of_4_bit_rows():
    for d, page in ((64, 16), (128, 16), (128, 256)):
        sh = _shape(d=d, page_size=page, kv_format=hk.KV_FP4_E2M1)
        assert sh.pages_shape == (100, 2, page * (d // 2 + d // 32))


@pytest.mark.parametrize("kv_format", [hk.KV_NATIVE, hk.KV_FP4_E2M1])
@pytest.mark.parametrize("name", CALLS)
def test_arguments_that_do_not_fit_are_refused(name, kv_format):
    L, sh = paged._lib(), _shape(kv_format=kv_format)
    names, written, call = CALLS[name]
    size = _sizes(sh)
    good = _apart(names)
    for x in names:
        if x in ("bounds", "bound_scales"):
            _fail(call(L, sh, {**good, x: None}, size["ws"]), "go together")
            _fail(call(L, sh, {**good, x: good[x] + 2}, size["ws"]), "aligned")
            continue
        match = {"ws": "workspace", "kept": "kept", "k_pages": "page pointer", "v_pages": "page pointer", "k_out": "k_out is null",
                 "v_out": "v_out is null"}.get(x, "integer array")
        _fail(call(L, sh, {**good, x: None}, size["ws"]), match)
        _fail(call(L, sh, {**good, x: good[x] + 2}, size["ws"]), "aligned|multiples of 16")
    if "ws" in names:
        _fail(call(L, sh, good, size["ws"] - 1), "workspace")
        _fail(call(L, _shape(max_pages=2 ** 22, page_size=16, batch=4096), good, 1 << 60), "2\\^30")


@pytest.mark.parametrize("kv_format", [hk.KV_NATIVE, hk.KV_FP4_E2M1])
@pytest.mark.parametrize("name", CALLS)
def test_arrays_that_overlap_are_refused(name, kv_format):
    L, sh = paged._lib(), _shape(kv_format=kv_format)
    names, written, call = CALLS[name]
    size, apart = _sizes(sh), _apart(names)
    for w in written:
        for other in names:
            if other == w or {w, other} in ({"lens_out", "lens"}, {"free_span_out", "free_span"}):
                continue
            for where in (apart[w], apart[w] + (size[w] - 1) // 16 * 16, apart[w] - (size[other] - 1) // 16 * 16):
                _fail(call(L, sh, {**apart, other: where}, size["ws"]), f"{w} overlaps {other}|{other} overlaps {w}")
    for w, other in (("lens_out", "lens"), ("free_span_out", "free_span")):
        if w in names:
            _fail(call(L, sh, {**apart, other: apart[w] + 4}, size["ws"]), "in part")


def test_numbers_that_do_not_fit_are_refused():
    L, sh, a = paged._lib(), _shape(), _apart(CALLS["assign_shared"][0] + ("kept", "move_from", "move_to"))
    assign = lambda n: L.heatkv_paged_assign_shared(sh.ref, *[a[x] for x in ("keep", "new_tokens", *TABLES, "q_start", "slots")], n,  # noqa: E731
                                                    a["copy_from"], a["copy_to"], a["status"], a["ws"], 1 << 40, None)
    compact = lambda n: L.heatkv_paged_compact(sh.ref, *[a[x] for x in ("kept", *TABLES, "move_from", "move_to")], n, a["status"],  # noqa: E731
                                               a["ws"], 1 << 40, None)
    rows = paged._CRows(at(50), 512, 128)
    move = lambda n, s=sh: L.heatkv_paged_move(s.ref, at(60), at(61), n, at(62), at(63), None, None, None)  # noqa: E731
    read = lambda n, k=rows, v=rows, s=sh: L.heatkv_paged_read(s.ref, at(60), n, at(62), at(63), k, v, None)  # noqa: E731
    for n in (-1, 2 ** 22 + 1):
        for call in (assign, compact, move, read):
            _fail(call(n), "tokens")
    wide = _shape(q_heads=1024, kv_heads=1024)
    _fail(move(2 ** 13 + 1, wide), "2\\^23")
    _fail(read(2 ** 13 + 1, s=wide), "2\\^23")
    assert move(0) == 0 and read(0) == 0
    _fail(read(4), "k_out overlaps v_out")
    _fail(read(4, v=paged._CRows(at(50) + 256, 512, 64)), "v_out: rows overlap")
    _fail(read(4, k=paged._CRows(at(50), 128, 128)), "k_out: rows overlap")
    _fail(read(4, k=paged._CRows(at(50), 500, 128)), "k_out: address")


def test_binding_names_what_does_not_fit():
    sh = _shape()
    x = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: hk.heatkv_paged_fork(sh, *[x] * 8), lambda: hk.heatkv_paged_assign_shared(sh, *[x] * 13),
                 lambda: hk.heatkv_paged_compact(sh, *[x] * 10), lambda: hk.heatkv_paged_move(sh, *[x] * 4),
                 lambda: hk.heatkv_paged_read(sh, *[x] * 5)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(TypeError, match="PagedShape"):
        hk.heatkv_paged_fork(None, *[x] * 8)
    with pytest.raises(TypeError, match="torch tensor"):
        hk.heatkv_paged_move(sh, None, None, x, x)


# ---- the references ----------------------------------------------------------------------------------------------------

def test_reference_codes():
    x = torch.zeros(1, 32, dtype=torch.float64)
    x[0, :9] = torch.tensor([6.0, 0.25, 0.75, 1.25, -1.75, 2.5, 3.5, 5.0, -0.2])
    codes, scales = sref.fp4_encode(x)
    assert scales.tolist() == [[127]] and codes[0, :9].tolist() == [7, 0, 2, 2, 12, 4, 6, 6, 8]
    for top, byte in ((7.0, 127), (7.01, 128), (3.5, 126), (3.4, 126), (3.51, 127), (0.0, 27), (1e-40, 27), (math.inf, 252), (1e38, 251),
                      (math.nan, 255)):
        x[0, 3] = top
        x[0, [0, 1, 2, 4, 5, 6, 7, 8]] = 0.0
        assert sref.fp4_encode(x)[1].tolist() == [[byte]], (top, byte)
    # every value is off by at most half a step: 1/4 of its own size above one, of the block's largest value 1/7
    y = torch.randn(200, 128, generator=torch.Generator().manual_seed(1), dtype=torch.float64) * 3
    held = sref.fp4_decode(*sref.fp4_encode(y))
    most = y.unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True)
    assert torch.all((held - y).unflatten(-1, (-1, 32)).abs() <= most * (2 / 7))
    again = sref.fp4_decode(*sref.fp4_encode(held))
    assert torch.equal(again, held)


def test_reference_tables_keep_every_page_once():
    for seed in range(60):
        rng = random.Random(seed)
        B, page, most = rng.randint(1, 6), 16, 6
        R = rng.randint(B * most, 3 * B * most)
        ring = list(range(R))
        rng.shuffle(ring)
        s = sref.Sharing(R, most, page, ring, rng.randrange(R), R, [[0] * most for _ in range(B)], [0] * B)
        content = {}  # what the rows of the cache hold: tokens are numbers
        rows, number = [[] for _ in range(B)], 0
        for _ in range(15):
            what = rng.randrange(3)
            if what == 0:
                parent = [rng.randrange(-1, B) for _ in range(B)]
                assert s.fork(parent) == 0
                rows = [list(rows[p]) if p >= 0 else [] for p in parent]
            elif what == 1:
                keep = [rng.randint(0, n) for n in s.lens]
                new = [min(96 - k, rng.randint(0, 30)) for k in keep]
                status, q_start, slots, copies = s.assign(keep, new, 200)
                if status == 0:
                    old = dict(content)
                    for f, t in (x for row in copies for x in row if x[0] >= 0):
                        content[t] = old[f]
                    for b in range(B):
                        mine = list(range(number, number + new[b]))
                        number += new[b]
                        rows[b] = rows[b][:keep[b]] + mine
                        content.update(zip(slots[q_start[b]:q_start[b + 1]], mine))
            else:
                kept = [[rng.random() < 0.7 for _ in range(96)] for _ in range(B)]
                status, moves = s.compact(kept, 1000)
                if status == 0:
                    old = dict(content)
                    for f, t in moves:
                        if f >= 0:
                            content[t] = old[f]
                    rows = [[x for x, k in zip(r, marks) if k] for r, marks in zip(rows, kept)]
            free = [s.ring[(s.head + i) % R] for i in range(s.count)]
            assert sorted(free + [p for p, n in enumerate(s.holders) if n]) == list(range(R))
            for b in range(B):
                assert [content[s.table[b][x // page] * page + x % page] for x in range(s.lens[b])] == rows[b]


def test_short_caches_have_a_workgroup_for_each_segment(rules):  # noqa: F811
    # where nothing is cut and there are few segments they are whole pieces: as many workgroups as segments there may be
    for bf16, batch, heads, group, new, grid in (
            (True, 1, 8, 4, 1, 512), (True, 16, 8, 2, 1, 512), (True, 64, 8, 2, 1, 576), (True, 64, 32, 1, 1, 2176), (True, 64, 38, 1, 1, 512), (True, 64, 20, 1, 1, 1360),
            (True, 1, 8, 2, 40, 512), (False, 1, 8, 2, 240, 512), (False, 4, 8, 2, 240, 992), (False, 64, 1, 16, 30, 1984),
            (False, 64, 2, 16, 30, 512), (True, 4, 8, 2, 240, 512)):
        few, many, _ = rules(bf16, batch, heads, group, batch * new, 16, 16)
        assert few["parts"] == 0 and few["grid"] == grid and few["whole_from"] == grid + 1
        assert bool(many["workgroups"]) == (bf16 and new == 240)
    for batch in (65, 300):  # more requests than lanes
        few, _, _ = rules(True, batch, 8, 2, batch, 16, 16)
        assert few["whole_from"] == 128 and few["grid"] == 512 and few["parts"] == 0
    for batch in (1, 16, 64, 65, 300):  # a cache whose segments may be cut
        few, _, _ = rules(True, batch, 8, 2, batch, 17, 16)
        assert few["whole_from"] == 128 and few["grid"] == 512 and few["parts"] == 1024


def test_no_segment_of_a_short_cache_is_left_out(rules):  # noqa: F811
    import random
    r = random.Random(4)
    for _ in range(2000):
        group, heads, batch = r.choice([1, 2, 3, 5, 16]), r.choice([1, 2, 8, 20, 64]), r.choice([1, 2, 5, 40, 64, 65, 300])
        new = [r.choice([0, 1, 1, 2, 5, 16, 17, 100, 240]) if r.random() < 0.7 else 1 for _ in range(batch)]
        few, _, _ = rules(r.random() < 0.5, batch, heads, group, sum(new) + r.choice([0, 1, 9]), 16, 16)
        segments = heads * sum(-(-n * group // 16) for n in new if n * group <= few["most_rows"])
        assert segments >= few["whole_from"] or segments <= few["grid"]
