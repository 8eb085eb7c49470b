"""Performance cases of the paged cache: many requests of different lengths, their rows on fixed-size pages.

A case is a dict of plain values.  `what` says which operator a pass runs:

  tables   one step of the page allocator: block tables, slots of the new tokens, pages taken and given back
  append   the new tokens' rows into their slots; `bounds`: with the 8-bit key bounds of every page that they touch
  attend   attention of the new tokens over their requests' pages
  sparse   the choice of `top` pages for each new token by their bounds, and attention over these

`dtype` is f32, bf16, or fp8 for bf16 operands over cache rows of FP8 E4M3 codes.  A case has `batch` requests of up to
`ctx` cached tokens, to which up to `new` come in this step; `ragged` spreads both downwards and leaves the token tensors
a little longer than what the requests fill, as a program does that replays one captured step for many.  Lengths follow
from the case, values from the seed.
"""
import math
import random

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.bfloat16}
_E4M3_MAX = 448.0
_CLAMP = 2.0 ** 127       # key and query values enter the bounds within +-2^127, NaN as 0
_LEAST_EXPONENT = -100    # of the bounds' and the query codes' powers of two


def _case(name, what, **fields):
    case = dict(what=what, dtype="bf16", q_heads=32, kv_heads=8, d=128, page=64, batch=1, ctx=0, new=1, ragged=True,
                causal=True, bounds=False, top=0, first=1, last=2)
    case.update(fields)
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # Every request of a small server gets its next token: what the allocator does between two decoding steps.
        _case("tables_decode_step", "tables", batch=64, ctx=8192, page=16, ragged=False),
        # A large server after a wave of finished requests: new prompts in their places, drafts cut back, pages both ways.
        _case("tables_admission", "tables", batch=1024, ctx=8192, new=512, page=64),
        # One new token of 128 requests into the cache, page bounds kept for the sparse attention.
        _case("append_decode_bounds", "append", batch=128, ctx=4096, bounds=True),
        # Prompts into an 8-bit cache, ragged, with bounds.
        _case("append_prompts_fp8", "append", dtype="fp8", batch=12, ctx=500, new=2048, page=32, bounds=True),
        # Decoding, 64 requests of ragged lengths, small pages, grouped heads: the bulk of serving.
        _case("attend_decode", "attend", batch=64, ctx=8192, page=16),
        # One long document, one token, 8-bit cache: latency of a lone user.
        _case("attend_decode_one_fp8", "attend", dtype="fp8", batch=1, ctx=65536, ragged=False),
        # Prefill in chunks behind a cached prefix.
        _case("attend_chunk", "attend", batch=2, ctx=4096, new=2048, ragged=False),
        # Image generators at different scales of their token maps: every new token sees all of its scale, no grouped heads.
        _case("attend_scales_d64", "attend", q_heads=16, kv_heads=16, d=64, page=32, batch=8, ctx=2000, new=1024,
              causal=False),
        # Reference outputs in fp32, a few short requests: latency.
        _case("attend_f32", "attend", dtype="f32", q_heads=8, kv_heads=4, page=16, batch=3, ctx=700, new=37),
        # Decoding at long contexts, each token over 32 of up to 512 pages.
        _case("sparse_decode", "sparse", batch=16, ctx=32768, top=32),
        # A chunk of a long prompt, each token with a choice of its own.
        _case("sparse_chunk", "sparse", q_heads=16, kv_heads=4, ctx=16384, new=1024, top=32, ragged=False),
        # Drafted tokens of a few requests in fp32, small heads, odd sizes.
        _case("sparse_f32", "sparse", dtype="f32", q_heads=6, kv_heads=2, d=64, page=16, batch=5, ctx=900, new=3, top=7),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(("tables", "append", "attend", "attend", "attend", "sparse", "sparse"))
    kv = rng.choice((1, 2, 3, 4, 8, 8, 16))
    group = rng.choice((1, 1, 2, 3, 4, 4, 6, 8, 16))
    dtype = rng.choice(("bf16", "bf16", "bf16", "fp8", "f32"))
    case = _case(None, what, dtype=dtype, kv_heads=kv, q_heads=kv * group, d=rng.choice((64, 128, 128)),
                 page=rng.choice((16, 32, 64, 64, 128, 256)), batch=_log_uniform(rng, 1, 96),
                 ctx=_log_uniform(rng, 1, 40000), new=rng.choice((1, 1, 1, rng.randint(2, 9), _log_uniform(rng, 10, 2500))),
                 ragged=rng.random() < 0.75, causal=rng.random() < 0.7)
    if what == "tables":
        case.update(batch=_log_uniform(rng, 1, 1500), ctx=min(case["ctx"], 8192), new=min(case["new"], 600), dtype="bf16",
                    kv_heads=8, q_heads=32, d=128)
    if what == "append":
        case["bounds"] = rng.random() < 0.6
        case["ctx"] = min(case["ctx"], 4096)
    if what == "sparse":
        case.update(top=rng.randint(3, 64), first=rng.randint(0, 1), last=rng.randint(1, 2))
    while _cost(case) > 1.0:  # no drawn case costs more than the largest listed one
        if case["batch"] > 1:
            case["batch"] //= 2
        elif case["new"] > 64:
            case["new"] //= 2
        else:
            case["ctx"] //= 2
    return case


def _cost(case):
    """Share of the largest listed case's work and memory, from the sizes alone."""
    rows = case["batch"] * (case["ctx"] + case["new"])
    if case["what"] == "tables":
        return max(rows / 8e6, case["batch"] * case["new"] / 5e5)
    pairs = case["batch"] * case["new"] * (case["ctx"] + case["new"]) * case["q_heads"]
    slow = 4 if case["dtype"] == "f32" else 1
    return max(rows * case["kv_heads"] * case["d"] / 5e8, slow * pairs * case["d"] / 8e10, pairs / 8e8,
               case["batch"] * case["new"] * case["kv_heads"] * case["d"] / 2.5e7)


def _lengths(case):
    """(cached, new) tokens of every request."""
    r = random.Random(1000003 * case["batch"] + 1009 * case["ctx"] + 13 * case["new"] + case["page"])
    cached, new = [], []
    for b in range(case["batch"]):
        if not case["ragged"]:
            cached.append(case["ctx"])
            new.append(case["new"])
            continue
        cached.append(case["ctx"] if b == 0 else r.randint(case["ctx"] // 8, case["ctx"]))
        n = case["new"] if b == 0 else r.randint(0 if case["new"] > 1 else 1, case["new"])
        if b and case["new"] > 16 and r.random() < 0.3:
            n = 1  # a decoding request among prompts
        new.append(n)
    return cached, new


def _table_lengths(case):
    """(held before, kept of it, new) tokens of every request of an allocator step."""
    cached, new = _lengths(case)
    if not case["ragged"]:
        return cached, list(cached), new
    r = random.Random(case["batch"] + 7 * case["ctx"])
    before, keep, come = [], [], []
    for c, n in zip(cached, new):
        u = r.random()
        if u < 0.25:  # finished, a new prompt in its place
            before.append(c)
            keep.append(0)
            come.append(n)
        elif u < 0.35:  # finished, the place stays empty
            before.append(c)
            keep.append(0)
            come.append(0)
        elif u < 0.6:  # some drafted tokens were rejected
            before.append(c)
            keep.append(c - min(c, r.randint(0, 8)))
            come.append(min(n, r.randint(1, 9)))
        else:
            before.append(c)
            keep.append(c)
            come.append(min(n, 1))
    return before, keep, come


def _pages(n, page):
    return -(-n // page)


def _ints(v, dev):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def _rows(gen, case, tokens, heads, drift, dtype):
    """[tokens, heads, d] rows; `drift`: neighbouring tokens have something in common, as keys and queries do."""
    dev = gen.device
    x = torch.randn(tokens, heads, case["d"], generator=gen, device=dev, dtype=torch.float32)
    if drift:
        slow = torch.randn(_pages(tokens, 48) + 1, heads, case["d"], generator=gen, device=dev, dtype=torch.float32)
        at = torch.arange(tokens, device=dev) // 48
        x = 0.8 * x + 0.6 * slow[at]
    return x.to(dtype)


def _to_store(x, case):
    """Rows as the cache holds them."""
    if case["dtype"] != "fp8":
        return x
    return x.float().clamp(-_E4M3_MAX, _E4M3_MAX).to(torch.float8_e4m3fn)


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 7919 + 31)
    page, B = case["page"], case["batch"]
    st = {"case": case}
    if case["what"] == "tables":
        before, keep, new = _table_lengths(case)
        held = [_pages(n, page) for n in before]
        max_pages = _pages(case["ctx"] + case["new"], page) + 1
        num_pages = sum(held) + sum(max(0, _pages(k + n, page) - h) for k, n, h in zip(keep, new, held)) + 17
        order = torch.randperm(num_pages, generator=gen, device=dev).to(torch.int32)
        cols = torch.arange(max_pages, device=dev)
        h = torch.tensor(held, device=dev)
        at = (torch.cumsum(h, 0) - h)[:, None] + cols
        table = torch.where(cols < h[:, None], order[at.clamp(max=num_pages - 1)], 0).to(torch.int32)
        free = num_pages - sum(held)
        head = int(seed) % num_pages  # the ring has been round a few times
        ring = torch.roll(torch.cat([order[sum(held):], order[:sum(held)]]), head).contiguous()
        tokens = sum(new) + (37 if case["ragged"] else 0)
        st.update(num_pages=num_pages, max_pages=max_pages, lens=_ints(before, dev), keep=_ints(keep, dev),
                  new=_ints(new, dev), ring=ring, span=_ints([head, free], dev), table=table,
                  lens_out=_ints([0] * B, dev), span_out=_ints([0, 0], dev), q_start=_ints([0] * (B + 1), dev),
                  slots=_ints([0] * max(tokens, 1), dev), status=_ints([0], dev))
        return _with_shape(st)
    cached, new = _lengths(case)
    lens = [c + n for c, n in zip(cached, new)]
    held = [_pages(n, page) for n in lens]
    max_pages = max(max(held), 1)
    num_pages = sum(held) + 3
    total = sum(new)
    tokens = max(total + (5 if case["ragged"] and B > 1 else 0), 1)
    order = torch.randperm(num_pages, generator=gen, device=dev).to(torch.int32)
    cols = torch.arange(max_pages, device=dev)
    h = torch.tensor(held, device=dev)
    at = (torch.cumsum(h, 0) - h)[:, None] + cols
    table = torch.where(cols < h[:, None], order[at.clamp(max=num_pages - 1)], 0).to(torch.int32)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    dt = _TORCH[case["dtype"]]
    drift = case["what"] == "sparse" or case["bounds"]
    # Rows in request order, scattered to their pages; the rest of a page holds zeros.
    shape = (num_pages, case["kv_heads"], page, case["d"])
    n_rows = sum(held) * page
    k_rows = _rows(gen, case, n_rows, case["kv_heads"], drift, dt).view(sum(held), page, case["kv_heads"], case["d"])
    v_rows = _rows(gen, case, n_rows, case["kv_heads"], False, dt).view(sum(held), page, case["kv_heads"], case["d"])
    # valid rows of every page, in the order of the requests' pages
    owner = torch.repeat_interleave(torch.arange(B, device=dev), h)
    nth = torch.arange(sum(held), device=dev) - (torch.cumsum(h, 0) - h)[owner]
    after = (torch.tensor(lens, device=dev)[owner] - nth * page).clamp(0, page)
    valid = (torch.arange(page, device=dev) < after[:, None])[:, :, None, None]
    store = torch.float8_e4m3fn if case["dtype"] == "fp8" else dt
    k_pages, v_pages = torch.zeros(shape, device=dev, dtype=store), torch.zeros(shape, device=dev, dtype=store)
    phys = order[:sum(held)].long()
    for rows, pages in ((k_rows, k_pages), (v_rows, v_pages)):
        r = _to_store(torch.where(valid, rows, 0), case).transpose(1, 2).contiguous()
        pages.view(torch.uint8).index_copy_(0, phys, r.view(torch.uint8))
    st.update(num_pages=num_pages, max_pages=max_pages, lens=_ints(lens, dev), table=table, q_start=_ints(starts, dev),
              k_pages=k_pages, v_pages=v_pages, total=total, tokens=tokens, max_new=max(max(new), 1),
              sm=1.0 / math.sqrt(case["d"]))
    if case["what"] == "append" or case["what"] == "sparse":
        fill = torch.zeros(num_pages, dtype=torch.int64, device=dev)
        fill[phys] = after
        bounds, scales = _page_bounds(k_pages, fill)
        st.update(bounds=bounds, scales=scales)
    if case["what"] == "append":
        flat = torch.repeat_interleave(torch.arange(B, device=dev), torch.tensor(new, device=dev))
        j = torch.arange(total, device=dev) - torch.tensor(starts, device=dev)[flat]
        pos = torch.tensor(cached, device=dev)[flat] + j
        slots = torch.full((tokens,), -1, dtype=torch.int32, device=dev)
        slots[:total] = table[flat, pos // page] * page + (pos % page).to(torch.int32)
        # keys and values are slices of one fused projection of the tokens
        heads = case["q_heads"] + 2 * case["kv_heads"]
        qkv = _rows(gen, case, tokens, heads, drift, dt)
        st.update(slots=slots, k_new=qkv[:, case["q_heads"]:case["q_heads"] + case["kv_heads"]],
                  v_new=qkv[:, case["q_heads"] + case["kv_heads"]:])
        if not case["bounds"]:
            st.update(bounds=None, scales=None)
        return _with_shape(st)
    q = _rows(gen, case, tokens, case["q_heads"], drift, dt)
    st.update(q=q, out=torch.zeros(tokens, case["q_heads"], case["d"], dtype=dt, device=dev),
              lse=torch.zeros(tokens, case["q_heads"], dtype=torch.float32, device=dev))
    if case["what"] == "sparse":
        st["selected"] = torch.full((tokens, case["kv_heads"], case["top"]), -1, dtype=torch.int32, device=dev)
    return _with_shape(st)


def _with_shape(st):
    st["shape"] = None
    st["ws"] = None
    return st


# ---- plain forms ------------------------------------------------------------------------------------------------------

def _power_of_two(amax):
    """The least power of two that amax fits 127 times, no less than 2^_LEAST_EXPONENT."""
    m, x = torch.frexp(amax)
    e = torch.where(m <= 127.0 / 128.0, x - 7, x - 6)
    e = torch.where(amax > 0, e, _LEAST_EXPONENT).clamp(min=_LEAST_EXPONENT)
    return torch.ldexp(torch.ones_like(amax), e)


def _finite(x):
    return torch.nan_to_num(x.float(), nan=0.0, posinf=_CLAMP, neginf=-_CLAMP).clamp(-_CLAMP, _CLAMP)


def _page_bounds(k_pages, fill):
    """8-bit bounds of the keys on every page: codes [pages, heads, 2, d] of the largest and of minus the smallest value of
    each channel over the page's first `fill` rows, and their power of two [pages, heads]; zeros for an empty page."""
    x = _finite(k_pages)
    rows = torch.arange(x.shape[2], device=x.device)
    valid = (rows < fill[:, None])[:, None, :, None]
    top = torch.where(valid, x, -math.inf).amax(2)
    low = torch.where(valid, -x, -math.inf).amax(2)
    some = (fill > 0)[:, None, None]
    both = torch.where(some[..., None], torch.stack([top, low], 2), 0.0)
    scale = _power_of_two(both.abs().amax((2, 3)))
    codes = torch.ceil(both.double() / scale[..., None, None].double())  # in 32 bits a small channel next to a huge one underflows
    return codes.to(torch.int8), torch.where(some[..., 0], scale, 0.0)


def _query_codes(q, kv_heads):
    """[tokens, kv_heads, 2 d]: sums over a group's queries of their positive and of their negative parts, as whole numbers."""
    x = _finite(q).view(q.shape[0], kv_heads, -1, q.shape[2])
    code = torch.round(x / _power_of_two(x.abs().amax((2, 3)))[:, :, None, None])
    return torch.cat([code.clamp(min=0).sum(2), (-code).clamp(min=0).sum(2)], -1)


def _requests_of(st):
    """Request of every token (the last one's for those behind the end) and its place in it."""
    q_start = st["q_start"].long()
    t = torch.arange(st["tokens"], device=q_start.device)
    b = torch.searchsorted(q_start[1:].contiguous(), t, right=True).clamp(max=q_start.numel() - 2)
    return t, b, t - q_start[b]


def _limits(st, b, j):
    """Keys that each token sees."""
    q_start, lens = st["q_start"].long(), st["lens"].long()
    n_new = (q_start[1:] - q_start[:-1])[b]
    return (lens[b] - n_new + j + 1 if st["case"]["causal"] else lens[b]).clamp(min=0)


def _plain_tables(st):
    page, ring, table = st["case"]["page"], st["ring"].long(), st["table"].long()
    lens, keep, new = st["lens"].long(), st["keep"].long(), st["new"].long()
    head, count = st["span"].long()[0], st["span"].long()[1]
    held, want = (lens + page - 1) // page, (keep + new + page - 1) // page
    takes, gives = (want - held).clamp(min=0), (held - want).clamp(min=0)
    q_start = torch.cat([torch.zeros_like(new[:1]), torch.cumsum(new, 0)])
    bad = (keep < 0) | (keep > lens) | (new < 0) | (want > table.shape[1])
    status = torch.where(bad.any(), 2, torch.where(q_start[-1] > st["slots"].numel(), 3,
                                                   torch.where(takes.sum() > count, 1, 0)))
    ok = status == 0
    cols = torch.arange(table.shape[1], device=table.device)
    r = ring.numel()
    nth = (torch.cumsum(takes, 0) - takes)[:, None] + cols - held[:, None]
    is_taken = (cols >= held[:, None]) & (cols < want[:, None]) & ok
    table_out = torch.where(is_taken, ring[(head + nth) % r], table)
    nth = (torch.cumsum(gives, 0) - gives)[:, None] + cols - want[:, None]
    is_given = (cols >= want[:, None]) & (cols < held[:, None]) & ok
    at = torch.where(is_given, (head + count + nth) % r, r)
    ring_out = torch.cat([ring, ring[:1]]).scatter(0, at.flatten(), table.flatten())[:r]
    t = torch.arange(st["slots"].numel(), device=table.device)
    b = torch.searchsorted(q_start[1:].contiguous(), t, right=True).clamp(max=new.numel() - 1)
    pos = keep[b] + t - q_start[b]
    entry = table_out[b, (pos // page).clamp(0, table.shape[1] - 1)]
    slots = torch.where((t < q_start[-1]) & ok, entry * page + pos % page, -1)
    span = torch.stack([(head + takes.sum()) % r, count - takes.sum() + gives.sum()])
    out = [torch.where(ok, keep + new, lens), torch.where(ok, span, st["span"].long()), table_out, ring_out,
           torch.where(ok, q_start, 0), slots, status[None]]
    return [x.to(torch.int32) for x in out]


def _plain_append(st):
    case = st["case"]
    slots = st["slots"][:st["total"]].long()
    page, off = slots // case["page"], slots % case["page"]
    for new, pages in ((st["k_new"], st["k_pages"]), (st["v_new"], st["v_pages"])):
        rows = _to_store(new[:st["total"]], case)
        pages.view(torch.uint8)[page, :, off] = rows.contiguous().view(torch.uint8)
    if not case["bounds"]:
        return [st["k_pages"], st["v_pages"]]
    fill = torch.zeros(st["num_pages"], dtype=torch.int64, device=slots.device)
    fill = fill.scatter_reduce(0, page, off + 1, "amax")
    bounds, scales = _page_bounds(st["k_pages"], fill)
    touched = (fill > 0)[:, None]
    st["bounds"].copy_(torch.where(touched[..., None, None], bounds, st["bounds"]))
    st["scales"].copy_(torch.where(touched, scales, st["scales"]))
    return [st["k_pages"], st["v_pages"], st["bounds"], st["scales"]]


def _plain_select(st):
    case = st["case"]
    t, b, j = _requests_of(st)
    page, top = case["page"], case["top"]
    visible = (_limits(st, b, j) + page - 1) // page
    codes = _query_codes(st["q"], case["kv_heads"]).double()
    at = st["table"].long()                                                # [batch, pages]
    rows = st["bounds"].flatten(2)[at].double().permute(0, 2, 3, 1)        # [batch, heads, 2 d, pages]
    pad_t = (st["q_start"].long()[:-1, None] + torch.arange(st["max_new"], device=t.device)).clamp(max=st["tokens"] - 1)
    dots = torch.matmul(codes[pad_t].transpose(1, 2), rows.contiguous())   # [batch, heads, tokens, pages], exact
    scores = (dots.float() * st["scales"][at].transpose(1, 2)[:, :, None]).transpose(1, 2)
    scores = scores[b, j.clamp(max=st["max_new"] - 1)]                     # [tokens, heads, pages]
    n = torch.arange(scores.shape[2], device=t.device)
    seen = n < visible[:, None]
    forced = seen & ((n < case["first"]) | (n >= visible[:, None] - case["last"]))
    # Forced pages first, then by score, ties to the lowest index; those that a token does not see come last.
    scores = torch.where(forced[:, None], math.inf, torch.where(seen[:, None], scores.clamp(max=3e38), -math.inf))
    order = torch.argsort(scores, dim=2, descending=True, stable=True)[:, :, :top]
    chosen = torch.where(order < visible[:, None, None], order, scores.shape[2])
    chosen = torch.sort(chosen, dim=2).values
    chosen = torch.where(chosen < scores.shape[2], chosen, -1)
    out = st["selected"].clone()
    out[:, :, :chosen.shape[2]] = torch.where(t[:, None, None] < st["q_start"].long()[-1], chosen.to(torch.int32),
                                              out[:, :, :chosen.shape[2]])
    return out


def _plain_attend(st, selected=None):
    case = st["case"]
    t, b, j = _requests_of(st)
    B, H, G = case["batch"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    d, page, n_max = case["d"], case["page"], st["max_new"]
    at = st["table"].long()
    S = at.shape[1] * page
    k = st["k_pages"][at].float().transpose(1, 2).reshape(B, H, S, d)
    v = st["v_pages"][at].float().transpose(1, 2).reshape(B, H, S, d)
    pad_t = (st["q_start"].long()[:-1, None] + torch.arange(n_max, device=t.device)).clamp(max=st["tokens"] - 1)
    q = st["q"].float()[pad_t].view(B, n_max, H, G, d).permute(0, 2, 1, 3, 4).reshape(B, H, n_max * G, d)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).view(B, H, n_max, G, S) * st["sm"]
    pos = torch.arange(S, device=t.device)
    seen = (pos < _limits(st, b, j)[pad_t][..., None])[:, None]            # [B, 1, n_max, S]
    if selected is not None:
        pages = torch.zeros(st["tokens"], H, at.shape[1] + 1, dtype=torch.bool, device=t.device)
        pages = pages.scatter(2, torch.where(selected >= 0, selected, at.shape[1]).long(), True)[..., :-1]
        seen = seen & pages[pad_t].transpose(1, 2).repeat_interleave(page, 3)
    s = torch.where(seen[:, :, :, None], s, -math.inf)
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(s - m)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, H, n_max * G, S), v).view(B, H, n_max, G, d)
    o = torch.where(total > 0, o / total, 0.0)
    lse = torch.log(total) + m
    at_row = j.clamp(max=n_max - 1)
    o = o.permute(0, 2, 1, 3, 4)[b, at_row].reshape(st["tokens"], H * G, d)
    lse = torch.where(total > 0, lse, -math.inf)[..., 0].permute(0, 2, 1, 3)[b, at_row].reshape(st["tokens"], H * G)
    real = (t < st["q_start"].long()[-1])[:, None]
    return [torch.where(real[..., None], o.to(st["out"].dtype), st["out"]), torch.where(real, lse, st["lse"])]


# ---- one pass ---------------------------------------------------------------------------------------------------------

def _own_shape(st):
    """The shape object and workspace that a program makes once."""
    import paper_2605_14877_amd as hk
    case = st["case"]
    st["shape"] = hk.PagedShape(case["q_heads"], case["kv_heads"], case["d"], case["page"], st["num_pages"], case["batch"],
                                st["max_pages"], "f32" if case["dtype"] == "f32" else "bf16",
                                hk.KV_FP8_E4M3 if case["dtype"] == "fp8" else hk.KV_NATIVE)
    if case["what"] in ("attend", "sparse"):
        n = hk.paged_attend_workspace_bytes(st["shape"], st["tokens"], case["top"])
        st["ws"] = torch.empty(max(n, 16), dtype=torch.uint8, device=st["q"].device)


def _own_pass(st):
    import paper_2605_14877_amd as hk
    if st["shape"] is None:
        _own_shape(st)
    case, shape = st["case"], st["shape"]
    if case["what"] == "tables":
        hk.heatkv_paged_assign(shape, st["keep"], st["new"], st["lens"], st["ring"], st["span"], st["table"], st["q_start"],
                               st["slots"], st["status"], lens_out=st["lens_out"], free_span_out=st["span_out"])
        return [st["lens_out"], st["span_out"], st["table"], st["ring"], st["q_start"], st["slots"], st["status"]]
    if case["what"] == "append":
        hk.heatkv_paged_append(shape, st["slots"], st["k_new"], st["v_new"], st["k_pages"], st["v_pages"], st["bounds"],
                               st["scales"])
        return [st["k_pages"], st["v_pages"]] + ([st["bounds"], st["scales"]] if case["bounds"] else [])
    if case["what"] == "attend":
        hk.heatkv_paged_attend(shape, st["q"], st["k_pages"], st["v_pages"], st["table"], st["q_start"], st["lens"], st["sm"],
                               st["out"], st["ws"], causal=case["causal"], lse=st["lse"])
        return [st["out"], st["lse"]]
    hk.heatkv_paged_select(shape, st["q"], st["bounds"], st["scales"], st["table"], st["q_start"], st["lens"], case["first"],
                           case["last"], st["selected"], causal=case["causal"])
    hk.heatkv_paged_attend_selected(shape, st["q"], st["k_pages"], st["v_pages"], st["table"], st["q_start"], st["lens"],
                                    st["selected"], st["sm"], st["out"], st["ws"], causal=case["causal"], lse=st["lse"])
    return [st["selected"], st["out"], st["lse"]]


def run(st):
    if own:
        return _own_pass(st)
    what = st["case"]["what"]
    if what == "tables":
        return _plain_tables(st)
    if what == "append":
        return _plain_append(st)
    if what == "attend":
        return _plain_attend(st)
    selected = _plain_select(st)
    return [selected] + _plain_attend(st, selected)


# ---- bytes and operations ---------------------------------------------------------------------------------------------

def work(case):
    """Bytes and operations of one pass: every input read once, every output written once."""
    page, d, H, Hq = case["page"], case["d"], case["kv_heads"], case["q_heads"]
    esz = 4 if case["dtype"] == "f32" else 2
    kv = {"f32": 4, "bf16": 2, "fp8": 1}[case["dtype"]]
    if case["what"] == "tables":
        before, keep, new = _table_lengths(case)
        moved = sum(abs(_pages(k + n, page) - _pages(c, page)) for c, k, n in zip(before, keep, new))
        tokens = sum(new) + (37 if case["ragged"] else 0)
        return {"bytes": 4.0 * (5 * case["batch"] + 2 * moved + tokens + sum(_pages(n, page) for n in new)),
                "flops": 4.0 * case["batch"] + 4.0 * tokens}
    cached, new = _lengths(case)
    total = sum(new)
    if case["what"] == "append":
        byts, flops = 2.0 * total * H * d * (esz + kv) + 4.0 * total, 0.0
        if case["bounds"]:
            touched = sum(_pages(c + n, page) - c // page for c, n in zip(cached, new) if n)
            older = sum(c % page for c, n in zip(cached, new) if n)
            byts += H * (older * d * kv + touched * (2.0 * d + 4))
            flops = 2.0 * H * d * (older + total)
        return {"bytes": byts, "flops": flops}
    byts, flops = total * Hq * (2.0 * d * esz + 4), 0.0
    for c, n in zip(cached, new):
        if not n:
            continue
        seen = [c + i + 1 if case["causal"] else c + n for i in range(n)]
        if case["what"] == "attend":
            byts += 2.0 * (c + n) * H * d * kv
            flops += 4.0 * d * Hq * sum(seen)
        else:
            chosen = [min(s, case["top"] * page) for s in seen]
            pages = [_pages(s, page) for s in seen]
            byts += 2.0 * min(c + n, sum(chosen)) * H * d * kv + pages[-1] * H * (2.0 * d + 4)
            byts += 4.0 * n * H * case["top"]
            flops += 4.0 * d * Hq * sum(chosen) + 4.0 * d * H * sum(pages)
    return {"bytes": byts, "flops": flops}


# ---- from the definitions, in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    if case["what"] == "tables":
        return None
    st = prepare(case, seed)
    cached, new = _lengths(case)
    page, H, G = case["page"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    table = st["table"].tolist()
    if case["what"] == "append":
        pages = [st["k_pages"].double(), st["v_pages"].double()]
        scales, t = (st["scales"].double() if case["bounds"] else None), 0
        for b, (c, n) in enumerate(zip(cached, new)):
            for first in range(c // page, _pages(c + n, page) if n else 0):
                lo, hi = max(c, first * page), min(c + n, (first + 1) * page)
                p = table[b][first]
                for x, rows in zip(pages, (st["k_new"], st["v_new"])):
                    r = rows[t + lo - c:t + hi - c].double()
                    r = r.clamp(-_E4M3_MAX, _E4M3_MAX) if case["dtype"] == "fp8" else r
                    x[p, :, lo - first * page:hi - first * page] = r.transpose(0, 1)
                if scales is not None:
                    k = pages[0][p, :, :hi - first * page]
                    k = k.to(torch.float8_e4m3fn).double() if case["dtype"] == "fp8" else k
                    least = torch.ceil(torch.log2(k.abs().amax((1, 2)) / 127.0)).clamp(min=_LEAST_EXPONENT)
                    scales[p] = torch.exp2(least)
            t += n
        return pages + ([None, scales] if case["bounds"] else [])
    sparse = case["what"] == "sparse"
    out, lse = st["out"].double(), st["lse"].double()
    t = 0
    for b, (c, n) in enumerate(zip(cached, new)):
        if not n:
            continue
        ids = torch.tensor(table[b][:_pages(c + n, page)], device=out.device)
        for h in range(H):
            unseen = _exact_unselected(st, b, t, c, n, h, ids) if sparse else None
            k = st["k_pages"][ids, h].double().reshape(-1, case["d"])[:c + n]
            v = st["v_pages"][ids, h].double().reshape(-1, case["d"])[:c + n]
            for j in range(0, n, 256):
                m = min(256, n - j)
                q = st["q"][t + j:t + j + m, h * G:(h + 1) * G].double()
                s = torch.tensordot(q, k, ([2], [1])) * st["sm"]
                hidden = torch.zeros(m, c + n, dtype=torch.bool, device=out.device)
                if case["causal"]:
                    hidden |= torch.arange(c + n, device=out.device) > c + j + torch.arange(m, device=out.device)[:, None]
                if sparse:
                    hidden |= unseen[j:j + m].repeat_interleave(page, 1)[:, :c + n]
                s = s.masked_fill(hidden[:, None], -math.inf)
                out[t + j:t + j + m, h * G:(h + 1) * G] = torch.tensordot(torch.softmax(s, -1), v, 1)
                lse[t + j:t + j + m, h * G:(h + 1) * G] = torch.logsumexp(s, -1)
        t += n
    return ([None] if sparse else []) + [out, lse]


def _exact_unselected(st, b, t, c, n, h, ids):
    """[n, pages] of request b: the pages that a token's queries of head group h do not take."""
    case = st["case"]
    G = case["q_heads"] // case["kv_heads"]
    q = st["q"][t:t + n, h * G:(h + 1) * G].double()
    e = torch.ceil(torch.log2(q.abs().amax((1, 2)) / 127.0)).clamp(min=_LEAST_EXPONENT)
    code = torch.round(q * torch.exp2(-e)[:, None, None]).long()
    ups, downs = (code * (code > 0)).sum(1).double(), (-code * (code < 0)).sum(1).double()
    top, low = st["bounds"][ids, h, 0].double(), st["bounds"][ids, h, 1].double()
    score = (ups @ top.T.contiguous() + downs @ low.T.contiguous()).float() * st["scales"][ids, h]
    unseen = torch.ones(n, len(ids), dtype=torch.bool, device=q.device)
    for i in range(n):
        k = _pages(c + i + 1 if case["causal"] else c + n, case["page"])
        fixed = set(range(min(case["first"], k))) | set(range(max(0, k - case["last"]), k))
        rank = torch.sort(score[i, :k], descending=True, stable=True).indices
        free = torch.tensor([p not in fixed for p in range(k)], device=q.device)
        take = rank[free[rank]][:max(0, case["top"] - len(fixed))].tolist()
        unseen[i, sorted(fixed) + take] = False
    return unseen
