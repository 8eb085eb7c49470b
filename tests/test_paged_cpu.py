"""CPU-side checks of the paged cache: refusals of the C ABI before any GPU work, the launch rules, the compiled kernels' tile
copies, and the reference of the GPU tests against closed forms.  No GPU needed."""
import ctypes as C
import math
import os
import subprocess
import tempfile

import pytest
import torch

import paper_2605_14877_amd as hk
from paper_2605_14877_amd import build as hb
from paper_2605_14877_amd import paged
from tests import paged_reference as ref
from tests.test_isa_hazards import scan

GOOD = dict(q_heads=8, kv_heads=2, d=128, page_size=64, num_pages=100, batch=4, max_pages=30, dtype="bf16")


def _shape(**change):
    return hk.PagedShape(**{**GOOD, **change})


BAD_SHAPES = [
    (dict(q_heads=7), "multiple"), (dict(q_heads=0), ">= 1"), (dict(kv_heads=0), ">= 1"), (dict(q_heads=34), "more than 16"),
    (dict(q_heads=2048, kv_heads=2048), "1024 kv heads"), (dict(d=96), "64 or 128"), (dict(d=256), "64 or 128"), (dict(dtype=2), "dtype"),
    (dict(kv_format=2), "storage format"), (dict(kv_format=hk.KV_FP8_E4M3, dtype="f32"), "bf16 shape"), (dict(page_size=8), "page_size"),
    (dict(page_size=48), "page_size"), (dict(page_size=512), "page_size"), (dict(batch=0), "batch"), (dict(batch=4097), "batch"),
    (dict(num_pages=0), "num_pages"), (dict(num_pages=2 ** 24 + 1), "2\\^30"), (dict(max_pages=0), "max_pages"),
    (dict(max_pages=2 ** 24 + 1), "2\\^30"), (dict(num_pages=2 ** 24, kv_heads=32, q_heads=32), "2\\^34"),
]


def _fail(rc, match):
    with pytest.raises(hk.HeatKVError, match=match) as e:
        paged._check(rc)
    assert e.value.code == -1


ROWS = paged._CRows(1 << 20, 1024, 128)


def _calls(L, sh):
    """Every call with that shape, its other arguments in order (addresses that are never followed: the shape is refused)."""
    a = 1 << 20
    return [lambda: L.heatkv_paged_assign(sh.ref, *[a] * 10, 4, a, None),
            lambda: L.heatkv_paged_append(sh.ref, a, 4, ROWS, ROWS, a, a, None, None, None),
            lambda: L.heatkv_paged_attend(sh.ref, 4, ROWS, a, a, a, a, a, 0.1, 1, ROWS, None, a, 1 << 40, None),
            lambda: L.heatkv_paged_select(sh.ref, 4, ROWS, a, a, a, a, a, 1, 1, 4, 1, a, None),
            lambda: L.heatkv_paged_attend_selected(sh.ref, 4, ROWS, a, a, a, a, a, a, 4, 0.1, 1, ROWS, None, a, 1 << 40, None)]


@pytest.mark.parametrize("change,match", BAD_SHAPES, ids=str)
def test_shapes_that_do_not_fit_are_refused(change, match):
    L, sh = paged._lib(), _shape(**change)
    assert hk.paged_attend_workspace_bytes(sh, 4) == 0
    for call in _calls(L, sh):
        _fail(call(), match)


def test_arguments_that_do_not_fit_are_refused():
    L, sh, a = paged._lib(), _shape(), 1 << 20
    attend = lambda tokens=4, q=ROWS, k=a, ints=(a, a, a), sm=0.1, out=ROWS, lse=None, ws=a, n=1 << 40: L.heatkv_paged_attend(  # noqa: E731
        sh.ref, tokens, q, k, a, *ints, sm, 1, out, lse, ws, n, None)
    _fail(attend(tokens=-1), "tokens")
    _fail(attend(tokens=2 ** 22 + 1), "tokens")
    _fail(attend(q=paged._CRows(None, 1024, 128)), "q is null")
    _fail(attend(q=paged._CRows(a + 8, 1024, 128)), "q: address")
    _fail(attend(q=paged._CRows(a, 1020, 128)), "q: address")
    _fail(attend(out=paged._CRows(a, 1024, 4)), "out: address")
    _fail(attend(out=paged._CRows(a, 0, 128)), "overlap")
    _fail(attend(out=paged._CRows(a, 512, 128)), "overlap")
    _fail(attend(k=0), "page pointer")
    _fail(attend(k=a + 4), "16-byte")
    _fail(attend(ints=(a, 0, a)), "integer array")
    _fail(attend(ints=(a, a, a + 2)), "4-byte")
    for sm in (0.0, -1.0, math.inf, math.nan):
        _fail(attend(sm=sm), "sm_scale")
    _fail(attend(lse=a + 1), "lse")
    assert hk.paged_attend_workspace_bytes(sh, 4) > 0
    _fail(attend(ws=0), "workspace")
    _fail(attend(n=hk.paged_attend_workspace_bytes(sh, 4) - 1), "workspace")
    _fail(attend(ws=a + 8), "16-byte")
    assert attend(tokens=0, q=paged._CRows(), ints=(0, 0, 0), ws=0, n=0) == 0

    append = lambda slots=a, tokens=4, k=ROWS, pages=a, b=None, s=None: L.heatkv_paged_append(  # noqa: E731
        sh.ref, slots, tokens, k, ROWS, pages, a, b, s, None)
    _fail(append(slots=0), "integer array")
    _fail(append(k=paged._CRows(a, 1024, 3)), "k_new")
    _fail(append(pages=0), "page pointer")
    _fail(append(b=a), "go together")
    _fail(append(s=a), "go together")
    _fail(append(b=a + 8, s=a), "16-byte")
    assert append(tokens=0, slots=0) == 0

    select = lambda sh=sh, first=1, last=1, top=4, bounds=a, out=a: L.heatkv_paged_select(  # noqa: E731
        sh.ref, 4, ROWS, bounds, a, a, a, a, first, last, top, 1, out, None)
    for first, last, top in ((0, 1, 0), (0, 1, 513), (-1, 1, 4), (1, 0, 4), (3, 2, 4), (2 ** 31 - 1, 2 ** 31 - 1, 4)):
        _fail(select(first=first, last=last, top=top), "top|first")
    _fail(select(bounds=a + 4), "bounds")
    _fail(select(out=0), "integer array")
    _fail(select(sh=_shape(max_pages=32769)), "32768")
    chosen = lambda sh=sh, sel=a, top=4: L.heatkv_paged_attend_selected(  # noqa: E731
        sh.ref, 4, ROWS, a, a, a, a, a, sel, top, 0.1, 1, ROWS, None, a, 1 << 40, None)
    _fail(chosen(sel=0), "integer array")
    _fail(chosen(top=0), "top")
    _fail(chosen(top=513), "top")
    _fail(chosen(sh=_shape(max_pages=32769)), "32768")

    assign = lambda **c: L.heatkv_paged_assign(sh.ref, *[c.get(n, d) for n, d in (  # noqa: E731
        ("keep", a), ("new", a + 64), ("lens", a + 128), ("lens_out", a + 128), ("ring", a), ("span", a), ("span_out", a), ("table", a),
        ("q_start", a), ("slots", a), ("tokens", 4), ("status", a))], None)
    for name in ("keep", "new", "lens", "lens_out", "ring", "span", "span_out", "table", "q_start", "slots", "status"):
        _fail(assign(**{name: 0}), "integer array")
    _fail(assign(tokens=-1), "tokens")
    _fail(assign(lens_out=a + 132), "in part")
    _fail(assign(span_out=a + 4), "in part")
    _fail(assign(lens_out=a), "overlap")


def test_calls_of_more_tokens_and_heads_than_a_launch_has_lanes_are_refused():
    sh = _shape(q_heads=1024, kv_heads=1024)
    rows, n = paged._CRows(1 << 20, 1024 * 128, 128), 2 ** 13 + 1
    L, a = paged._lib(), 1 << 20
    for call in (lambda: L.heatkv_paged_append(sh.ref, a, n, rows, rows, a, a, None, None, None),
                 lambda: L.heatkv_paged_attend(sh.ref, n, rows, a, a, a, a, a, 0.1, 1, rows, None, a, 1 << 40, None),
                 lambda: L.heatkv_paged_select(sh.ref, n, rows, a, a, a, a, a, 1, 1, 4, 1, a, None),
                 lambda: L.heatkv_paged_attend_selected(sh.ref, n, rows, a, a, a, a, a, a, 4, 0.1, 1, rows, None, a, 1 << 40, None)):
        _fail(call(), "2\\^23")
    assert hk.paged_attend_workspace_bytes(sh, n) == 0 and hk.paged_attend_workspace_bytes(sh, n - 1) > 0


def test_binding_names_tensors_that_are_not_on_a_device():
    sh = _shape()
    q = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        hk.heatkv_paged_attend(sh, q, q, q, q, q, q, 0.1, q)
    with pytest.raises(ValueError, match="device tensor"):
        hk.heatkv_paged_append(sh, torch.zeros(4, dtype=torch.int32), q, q, q, q)
    with pytest.raises(ValueError, match="device tensor"):
        hk.heatkv_paged_assign(sh, *[torch.zeros(4, dtype=torch.int32)] * 9)
    with pytest.raises(ValueError, match="device tensor"):
        hk.heatkv_paged_select(sh, q, q, q, q, q, q, 1, 1, q)
    with pytest.raises(TypeError, match="PagedShape"):
        hk.heatkv_paged_attend(hk.Shape(1, 1, 64, [1, 2], 1, "f32"), q, q, q, q, q, q, 0.1, q)
    with pytest.raises(TypeError, match="torch tensor"):
        hk.heatkv_paged_attend(sh, None, q, q, q, q, q, 0.1, q)


RULES = r"""
#include "paged_rules.h"
extern "C" void plan(int bf16, int batch, int kv, int group, long long tokens, long long pages, int page, long long top, long long* out) {
  const auto p = heatkv::paged::plan_launches(bf16, batch, kv, group, tokens, pages, page, top);
  int i = 0;
  for (const auto& l : {p.few, p.many}) {
    out[i++] = l.workgroups; out[i++] = l.grid; out[i++] = l.parts; out[i++] = l.whole_from; out[i++] = l.least_steps;
    out[i++] = l.least_rows; out[i++] = l.most_rows;
  }
  out[i] = static_cast<long long>(heatkv::paged::many_union_bytes(group, pages, top));
}
"""
FIELDS = ("workgroups", "grid", "parts", "whole_from", "least_steps", "least_rows", "most_rows")


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    src, lib = d / "rules.cpp", d / "librules.so"
    src.write_text(RULES)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", hb.CSRC, str(src), "-o", str(lib)], check=True)
    L = C.CDLL(str(lib))

    def plan(bf16, batch, kv, group, tokens, pages, page, top=0):
        out = (C.c_longlong * 15)()
        L.plan(*[C.c_longlong(x) if i in (4, 5, 7) else C.c_int(x) for i, x in enumerate((int(bf16), batch, kv, group, tokens, pages, page, top))],
               out)
        return dict(zip(FIELDS, out[:7])), dict(zip(FIELDS, out[7:14])), out[14]
    return plan


def test_launch_rules_on_both_sides(rules):
    for pages, top, extra, least in ((512, 0, 40, 16), (1023, 0, 40, 16), (1024, 0, 16, 16), (1024, 8, 40, 64)):
        few, many, _ = rules(True, 64, 8, 4, 64 + extra, pages, 16, top)  # a decoding step and padding
        assert many["workgroups"] == 0 and few["most_rows"] > 10 ** 6 and few["parts"] > 0
        few, many, _ = rules(True, 64, 8, 4, 64 + extra + 1, pages, 16, top)
        assert many["workgroups"] and few["most_rows"] == many["least_rows"] == least
    assert rules(False, 1, 8, 4, 5000, 512, 16)[1]["workgroups"] == 0  # fp32 has one kernel
    assert rules(True, 1, 1, 1, 41, 512, 16)[1]["workgroups"] == 0 and rules(True, 1, 1, 1, 42, 512, 16)[1]["workgroups"]
    assert rules(True, 1, 1, 1, 64, 512, 16, 4)[1]["workgroups"] == 0 and rules(True, 1, 1, 1, 65, 512, 16, 4)[1]["workgroups"]
    assert rules(True, 1, 8, 4, 1, 16, 16)[0]["parts"] == 0 and rules(True, 1, 8, 4, 1, 17, 16)[0]["parts"] > 0
    few, many, size = rules(True, 1, 8, 1, 4000, 32768, 16, 512)  # a union too large for the LDS
    assert size > 92 * 1024 and many["workgroups"] == 0
    few, many, size = rules(True, 1, 8, 4, 4000, 512, 64, 32)
    assert size < 92 * 1024 and many["workgroups"]


def _pieces(many, requests, heads, group, causal, top_keys):
    """What the 128-row launch deals, as the kernel counts it, and how many places it needs."""
    def load(n_new, length):
        rows = n_new * group
        if not many["least_rows"] < rows <= many["most_rows"]:
            return 0, 0
        tiles, dw = -(-rows // 128), 0
        if top_keys:
            length = min(length, top_keys)
        elif causal:
            dw = 128 * 32 // 64 // group
            length = max(length - n_new + min(n_new, 128 // group), 0)
        w0 = max(-(-length // 64), 1) * 32
        return tiles, tiles * w0 + tiles * (tiles - 1) // 2 * dw
    loads = [load(*r) for r in requests]
    total, count = sum(w for _, w in loads) * heads, sum(t for t, _ in loads) * heads
    if count >= many["whole_from"] or not many["parts"]:
        return count, 0
    share = max(-(-total // many["workgroups"]), many["least_steps"] * 32)
    n = sum(t * -(-(w // t) // share) for t, w in loads if t) * heads
    return n, n


def test_pieces_fit_the_grid_and_the_workspace(rules):
    import random
    r = random.Random(2)
    for _ in range(400):
        group, heads, batch = r.choice([1, 2, 3, 4, 7, 16]), r.choice([1, 2, 8, 16, 64]), r.choice([1, 2, 5, 40, 300])
        causal, longest = r.random() < 0.5, r.choice([16, 512, 513, 4096, 70000])
        new = [r.choice([0, 1, 5, 64 // group, 64 // group + 1, r.randint(0, 3000)]) for _ in range(batch)]
        tokens = sum(new) + r.choice([0, 3])
        requests = [(n, r.randint(min(n, longest), longest)) for n in new]
        few, many, _ = rules(True, batch, heads, group, tokens, -(-longest // 16), 16)
        if not many["workgroups"]:
            continue
        grid, places = _pieces(many, requests, heads, group, causal, 0)
        assert grid <= many["grid"] and places <= many["parts"]


def test_pieces_of_the_16_row_launch_fit_the_grid_and_the_workspace(rules):
    import random
    r = random.Random(3)
    some = 0
    for _ in range(400):
        group, heads, batch = r.choice([1, 2, 4, 16]), r.choice([1, 2, 8, 64]), r.choice([1, 2, 5, 40, 255])
        longest = r.choice([16, 256, 257, 4096, 70000])
        new = [r.choice([0, 1, 1, 5]) for _ in range(batch)]
        few, many, _ = rules(True, batch, heads, group, max(sum(new), 1), -(-longest // 16), 16)
        # segments of any weights, one row of keys each at the least
        segments = [(-(-n * group // 16), max(-(-r.randint(1, longest) // 32), 1) * 32) for n in new if n]
        count, total = heads * sum(t for t, _ in segments), heads * sum(t * w for t, w in segments)
        if not few["parts"] or not 0 < count < few["whole_from"]:
            continue
        shares = few["workgroups"] - count
        share = max(-(-total // shares), few["least_steps"] * 32)
        pieces = heads * sum(t * -(-w // share) for t, w in segments)
        assert pieces <= few["grid"] <= few["parts"]
        some += 1
    assert some > 50


def test_tile_copies_do_not_depend_on_scalars_from_the_vector_alu():
    with tempfile.TemporaryDirectory() as tmp:
        for src in ("paged_attend_long.hip", "paged_attend_f32.hip"):
            out = os.path.join(tmp, src + ".s")
            subprocess.run(["hipcc", *hb.HIP_FLAGS, "-S", "--cuda-device-only", os.path.join(hb.CSRC, src), "-o", out], check=True,
                           capture_output=True)
            with open(out) as f:
                copies, hazards = scan(f.read())
            assert copies > 0 and not hazards, (src, hazards[:5])


# ---- the reference -----------------------------------------------------------------------------------------------------

def test_reference_attention_against_torch():
    g = torch.Generator().manual_seed(1)
    page, lens, new = 4, [13, 6], [5, 6]
    k, v = (torch.randn(10, 2, page, 8, generator=g, dtype=torch.float64) for _ in range(2))
    q = torch.randn(12, 4, 8, generator=g, dtype=torch.float64)
    table, q_start = [[3, 1, 7, 0], [9, 2]], [0, 5, 11]
    for causal in (True, False):
        out, lse, mag = ref.attend(q, k, v, table, q_start, lens, page, 0.3, causal)
        assert out[11].isnan().all()
        for b in range(2):
            ks, vs = (x[table[b]].transpose(0, 1).reshape(2, -1, 8)[:, :lens[b]].repeat_interleave(2, 0) for x in (k, v))
            qs = q[q_start[b]:q_start[b + 1]].transpose(0, 1)
            seen = torch.ones(new[b], lens[b], dtype=torch.bool)
            if causal:
                seen = seen.tril(lens[b] - new[b])
            want = torch.nn.functional.scaled_dot_product_attention(qs, ks, vs, seen, scale=0.3)
            assert (out[q_start[b]:q_start[b + 1]].transpose(0, 1) - want).abs().max() < 1e-12
    assert (mag[:11] >= out[:11].abs() - 1e-12).all()
    everything = [[list(range(4))] * 2 for _ in range(12)]
    assert torch.equal(ref.attend(q, k, v, table, q_start, lens, page, 0.3, True, everything)[0][:11],
                       ref.attend(q, k, v, table, q_start, lens, page, 0.3, True)[0][:11])


def test_reference_bounds_bound_the_scores():
    g = torch.Generator().manual_seed(2)
    rows = torch.randn(16, 64, generator=g).bfloat16()
    b, scale = ref.bounds_of(rows)
    assert (b[0].double() * scale >= rows.double().amax(0)).all() and (b[1].double() * scale >= -rows.double().amin(0)).all()
    assert math.log2(scale) == int(math.log2(scale)) and b.abs().max() <= 127
    code = torch.randint(-127, 128, (64,), generator=g).double()  # a query on its grid
    bound = scale * (code.clamp(min=0) @ b[0].double() + (-code).clamp(min=0) @ b[1].double())
    assert bound >= (rows.double() @ code).max()


def test_reference_allocator_keeps_every_page_once():
    import random
    r = random.Random(1)
    a = ref.Allocator(5, 30, 8, 16, list(range(30)), 7, 30, [[-1] * 8 for _ in range(5)], [0] * 5)
    for _ in range(200):
        keep = [r.randint(0, n) for n in a.lens]
        new = [r.randint(0, 40) for _ in a.lens]
        status, q_start, slots = a.step(keep, new, 150)
        used = [x for row, n in zip(a.table, a.lens) for x in row[:ref.pages_of(n, 16)]]
        free = [a.ring[(a.head + i) % 30] for i in range(a.count)]
        assert sorted(used + free) == list(range(30))
        assert status == 0 or set(slots) == {-1}


JOIN_RULES = r"""
#include "paged_rules.h"
extern "C" void launches(int bf16, int batch, int kv, int group, long long tokens, long long pages, int page, long long top, long long* out) {
  const auto p = heatkv::paged::plan_launches(bf16, batch, kv, group, tokens, pages, page, top);
  int i = 0;
  for (const auto& l : {p.few, p.many}) {
    out[i++] = l.grid;
    out[i++] = heatkv::paged::join_workgroups(l);
  }
}
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    d = tmp_path_factory.mktemp("launches")
    src, lib = d / "launches.cpp", d / "liblaunches.so"
    src.write_text(JOIN_RULES)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", hb.CSRC, str(src), "-o", str(lib)], check=True)
    L = C.CDLL(str(lib))

    def call(bf16, batch, kv, group, tokens, pages, page, top=0):
        out = (C.c_longlong * 4)()
        L.launches(*[C.c_longlong(x) if i in (4, 5, 7) else C.c_int(x)
                     for i, x in enumerate((int(bf16), batch, kv, group, tokens, pages, page, top))], out)
        return dict(zip(("few", "few_join", "many", "many_join"), out))
    return call


@pytest.mark.parametrize("top", [0, 4])
@pytest.mark.parametrize("kv", [1, 3, 128, 1024])
@pytest.mark.parametrize("batch", [1, 300, 1024, 4096])
def test_no_launch_has_more_lanes_than_there_can_be(launches, kv, batch, top):
    # at the limits of tokens, heads and requests; the join has 4 workgroups of 256 lanes for one of few rows, 8 for one of many
    for group in (1, 16):
        for tokens in {min(2 ** 22, 2 ** 23 // kv), min(2 ** 22, 2 ** 23 // kv) // 2, batch + 41}:
            n = launches(True, batch, kv, group, tokens, 64, 256, top)
            assert n["few"] * 256 < 2 ** 32 and n["many"] * 256 < 2 ** 32
            assert (4 * n["few_join"] + 8 * n["many_join"]) * 256 < 2 ** 32


def test_the_join_looks_at_every_piece(rules, launches):
    import random
    r, some = random.Random(4), 0
    for _ in range(400):
        group, heads, batch = r.choice([1, 2, 4, 16]), r.choice([1, 2, 8, 64]), r.choice([1, 2, 40, 300])
        longest = r.choice([513, 4096, 70000])
        new = [r.choice([0, 1, 5, 64 // group + 1, r.randint(0, 3000)]) for _ in range(batch)]
        args = (True, batch, heads, group, sum(new), -(-longest // 16), 16)
        many, n = rules(*args)[1], launches(*args)
        if not many["workgroups"]:
            continue
        assert n["few_join"] == n["few"] and n["many_join"] <= many["parts"]
        _, places = _pieces(many, [(x, r.randint(min(x, longest), longest)) for x in new], heads, group, True, 0)
        assert places <= n["many_join"]
        some += places > 0
    assert some > 50


def test_arrays_that_overlap_are_refused():
    # addresses are never followed: every call is refused
    L, sh, tokens = paged._lib(), _shape(), 4
    at = lambda i: (i + 1) << 36  # noqa: E731
    requests, rows_bytes = 4 * sh.batch, ((tokens - 1) * 1024 + 7 * 128 + 128) * 2
    pages = sh.num_pages * sh.page_size * sh.kv_heads * sh.d * 2
    size = dict(q=rows_bytes, out=rows_bytes, k_new=rows_bytes // 2, v_new=rows_bytes // 2, k_pages=pages, v_pages=pages,
                table=requests * sh.max_pages, q_start=requests + 4, lens=requests, keep=requests, new_tokens=requests,
                lens_out=requests, free_ring=4 * sh.num_pages, free_span=8, free_span_out=8, slots=4 * tokens, status=4,
                bounds=sh.num_pages * sh.kv_heads * 2 * sh.d, bound_scales=sh.num_pages * sh.kv_heads * 4,
                selected=tokens * sh.kv_heads * 4 * 4, lse=tokens * sh.q_heads * 4)
    rows = lambda a: paged._CRows(a, 1024, 128)  # noqa: E731
    kv_rows = lambda a: paged._CRows(a, 512, 128)  # noqa: E731
    size["k_new"] = size["v_new"] = (3 * 512 + 128 + 128) * 2

    def attend(a, top=0):
        size["ws"] = hk.paged_attend_workspace_bytes(sh, tokens, top)
        more = (a["selected"], top) if top else ()
        call = L.heatkv_paged_attend_selected if top else L.heatkv_paged_attend
        return lambda: call(sh.ref, tokens, rows(a["q"]), a["k_pages"], a["v_pages"], a["table"], a["q_start"], a["lens"], *more, 0.1, 1,
                            rows(a["out"]), a["lse"], a["ws"], 1 << 40, None)
    calls = {
        "assign": (("keep", "new_tokens", "lens", "lens_out", "free_ring", "free_span", "free_span_out", "table", "q_start", "slots", "status"),
                   ("lens_out", "free_ring", "free_span_out", "table", "q_start", "slots", "status"),
                   lambda a: lambda: L.heatkv_paged_assign(
                       sh.ref, *[a[x] for x in ("keep", "new_tokens", "lens", "lens_out", "free_ring", "free_span", "free_span_out",
                                                "table", "q_start", "slots")], tokens, a["status"], None), ()),
        "append": (("slots", "k_new", "v_new", "k_pages", "v_pages", "bounds", "bound_scales"), ("k_pages", "v_pages", "bounds", "bound_scales"),
                   lambda a: lambda: L.heatkv_paged_append(sh.ref, a["slots"], tokens, kv_rows(a["k_new"]), kv_rows(a["v_new"]),
                                                           a["k_pages"], a["v_pages"], a["bounds"], a["bound_scales"], None),
                   {("k_pages", "k_new"), ("k_pages", "v_new"), ("v_pages", "k_new"), ("v_pages", "v_new")}),
        "attend": (("q", "k_pages", "v_pages", "table", "q_start", "lens", "out", "lse", "ws"), ("out", "lse", "ws"), attend, ()),
        "attend_selected": (("q", "k_pages", "v_pages", "table", "q_start", "lens", "out", "lse", "ws", "selected"), ("out", "lse", "ws"),
                            lambda a: attend(a, 4), ()),
        "select": (("q", "bounds", "bound_scales", "table", "q_start", "lens", "selected"), ("selected",),
                   lambda a: lambda: L.heatkv_paged_select(sh.ref, tokens, rows(a["q"]), a["bounds"], a["bound_scales"], a["table"],
                                                           a["q_start"], a["lens"], 1, 1, 4, 1, a["selected"], None), ()),
    }
    for names, written, call, allowed in calls.values():
        apart = {n: at(i) for i, n in enumerate((*names, "ws"))}
        call(apart)  # sets the workspace's size; not called
        for w in written:
            for other in names:
                if other == w or (w, other) in allowed or {w, other} in ({"lens_out", "lens"}, {"free_span_out", "free_span"}):
                    continue
                # the same first byte; the other's last 16 bytes or less; the other lies within, or begins at the last bytes
                for where in (apart[w], apart[w] + (size[w] - 1) // 16 * 16, apart[w] - (size[other] - 1) // 16 * 16):
                    _fail(call({**apart, other: where})(), f"{w} overlaps {other}|{other} overlaps {w}|must not overlap")


def test_outputs_among_the_queries_are_refused():
    L, sh, a = paged._lib(), _shape(kv_heads=2, q_heads=4, d=64), 1 << 36
    call = lambda q, out, tokens=5: L.heatkv_paged_attend(  # noqa: E731
        sh.ref, tokens, paged._CRows(*q), 1 << 37, 1 << 38, 1 << 39, 1 << 40, 1 << 41, 0.1, 1, paged._CRows(*out), None, 1 << 42, 1 << 40, None)
    for q, out in (((a, 256, 64), (a, 256, 64)), ((a, 512, 64), (a + 2 * 248, 512, 64)), ((a, 512, 64), (a + 2 * (2048 + 192), 512, 64)),
                   ((a + 2 * (2048 + 192), 512, 64), (a, 512, 64)), ((a, 64, 320), (a + 2 * 256, 64, 320)),
                   ((a, 512, 128), (a + 2 * 8, 512, 128)), ((a, 512, 128), (a + 2 * (512 + 128), 512, 128)), ((a, 512, 64), (a + 512, 768, 64)),
                   ((a, 0, 0), (a, 256, 64))):
        _fail(call(q, out), "out overlaps q")
    _fail(call((a, 1 << 61, 1 << 60), (a, 1 << 61, 1 << 60)), "overlaps")  # everything
    _fail(call((a, 8, 64), (a, 16, 64), 1), "out overlaps q")


def test_pieces_of_chosen_pages_fit_the_grid_and_the_workspace(rules, launches):
    # a segment is as heavy as the pages that its tile's tokens can have chosen between them
    import random
    r, some = random.Random(5), {"few": 0, "many": 0}
    for _ in range(1500):
        group, heads, batch = r.choice([1, 2, 3, 4, 16]), r.choice([1, 2, 8, 64]), r.choice([1, 2, 5, 40, 300])
        page, top = r.choice([16, 64, 256]), r.choice([1, 3, 32, 512])
        longest = r.choice([16, 513, 4096, 70000])
        new = [r.choice([0, 1, 5, 64 // group, 64 // group + 1, r.randint(0, 3000 if batch < 40 else 100)]) for _ in range(batch)]
        requests = [(n, r.randint(min(n, longest), longest)) for n in new]
        args = (True, batch, heads, group, sum(new) + r.choice([0, 3]), -(-longest // page), page, top)
        few, many, _ = rules(*args)
        for name, launch, rows, keys in (("few", few, 16, 32), ("many", many, 128, 64)):
            if not launch["workgroups"]:
                continue
            loads = []
            for n_new, length in requests:
                if launch["least_rows"] < n_new * group <= launch["most_rows"]:
                    tokens = min(rows, (rows - 1) // group + 2, n_new)
                    loads.append((-(-n_new * group // rows), max(-(-min(length, tokens * top * page) // keys), 1) * 32))
            count, total = heads * sum(t for t, _ in loads), heads * sum(t * w for t, w in loads)
            if name == "few" and count >= launch["whole_from"]:
                continue  # dealt along the line: two places for each workgroup
            if name == "many" and (count >= launch["whole_from"] or not launch["parts"]):
                assert count <= launch["grid"]
                continue
            if not launch["parts"]:
                assert count <= launch["grid"]
                continue
            shares = launch["workgroups"] - (count if name == "few" else 0)
            share = max(-(-total // shares), launch["least_steps"] * 32)
            pieces = heads * sum(t * -(-w // share) for t, w in loads)
            assert pieces <= launch["grid"] and pieces <= launch["parts"] and pieces <= launches(*args)[name + "_join"]
            some[name] += pieces > count
    assert min(some.values()) > 50, some
