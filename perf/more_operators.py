"""Performance cases of the paged cache's 4-bit rows, and of pages that requests share, copy, thin out and give back.

A case is a dict of plain values.  `what` says which operators a pass runs:

  append   the new tokens' rows into 4-bit pages; `bounds`: with the 8-bit key bounds of every page that they touch.  The rows
           are then read back as the values that the cache holds, which is what a prompt's own attention goes on with
  attend   attention of the new tokens over their requests' 4-bit pages
  sparse   the choice of `top` pages for each new token by their bounds, and attention over these, 4-bit pages
  share    requests continue others (beams, samples of one prompt) or end; the next step of the allocator, which replaces the
           partly filled pages that several requests hold; and the rows of these pages, for one layer
  compact  every request loses the tokens that a policy has marked: tables, and the rows that move up, for one layer

`dtype` is f32, bf16, fp8 or fp4: the cache rows (the last two are E4M3 and E2M1 codes of bf16 operands).  A case has `batch`
requests of up to `ctx` cached tokens, to which up to `new` come in this step; `ragged` spreads both downwards and leaves the
token tensors a little longer than what the requests fill, as a program does that replays one captured step for many.
Lengths follow from the case, values from the seed.

4-bit rows: a block of 32 channels is E2M1 codes and one E8M0 byte, the power of two 2^e with the least e >= -100 for which no
value is more than 7 times 2^e (at most 125).  16 rows lie together: their codes, d / 2 bytes each, channel 2 i in the low
half of byte i, then their scale bytes, d / 32 each.
"""
import math
import random

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.bfloat16, "fp4": torch.bfloat16}
_CLAMP = 2.0 ** 127       # key and query values enter the bounds within +-2^127
_LEAST_EXPONENT = -100    # of the bounds', the query codes' and the 4-bit blocks' powers of two
_MOST_EXPONENT = 125      # of the 4-bit blocks'
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_EDGE = 64                # first and last tokens that no policy drops


def _case(name, what, **fields):
    case = dict(what=what, dtype="fp4", q_heads=32, kv_heads=8, d=128, page=64, batch=1, ctx=0, new=1, ragged=True, causal=True,
                bounds=False, top=0, first=1, last=2, beams=1, percent=50, runs=1)
    case.update(fields)
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # One new token of 128 requests into the 4-bit cache, page bounds kept for the sparse attention.
        _case("append_decode_bounds", "append", batch=128, ctx=4096, bounds=True),
        # Ragged prompts into the 4-bit cache.
        _case("append_prompts", "append", batch=12, ctx=500, new=2048, page=32),
        # Decoding, 64 requests of long ragged contexts, grouped heads: what the 4-bit cache is for.
        _case("attend_decode", "attend", batch=64, ctx=16384, page=32),
        # One long document, one token: latency of a lone user.
        _case("attend_decode_one", "attend", ctx=131072, ragged=False),
        # A chunk of a prompt behind a cached prefix.
        _case("attend_chunk", "attend", batch=2, ctx=4096, new=2048, ragged=False),
        # Image generators at different scales of their token maps: every new token sees all of its scale, no grouped heads.
        _case("attend_scales_d64", "attend", q_heads=16, kv_heads=16, d=64, page=32, batch=8, ctx=2000, new=1024, causal=False),
        # Decoding at long contexts, each token over 32 of up to 512 pages.
        _case("sparse_decode", "sparse", batch=16, ctx=32768, top=32),
        # Drafted tokens of a few requests, small heads, odd sizes: latency.
        _case("sparse_drafts", "sparse", q_heads=6, kv_heads=2, d=64, page=16, batch=5, ctx=900, new=3, top=7),
        # 16 beam searches of 4 beams: the surviving beams of a step, their next slots, the page that each writes to.
        _case("share_beams", "share", dtype="bf16", batch=64, ctx=4075, page=32, beams=4, ragged=False),
        # A large server: samples of common prompts start and end, drafts are cut back, pages both ways.
        _case("share_samples", "share", dtype="fp8", kv_heads=4, batch=512, ctx=8192, new=64, beams=8),
        # One request drops every other token of its past, one by one.
        _case("compact_one", "compact", dtype="bf16", ctx=3000, page=16, ragged=False),
        # Requests drop the scales or passages that their heads do not read, long runs of tokens.
        _case("compact_runs", "compact", dtype="bf16", batch=32, ctx=8192, runs=256, percent=60),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(("append", "attend", "attend", "attend", "sparse", "sparse", "share", "share", "compact", "compact"))
    kv = rng.choice((1, 2, 3, 4, 8, 8, 16))
    group = rng.choice((1, 1, 2, 3, 4, 4, 6, 8, 16))
    case = _case(None, what, kv_heads=kv, q_heads=kv * group, d=rng.choice((64, 128, 128)),
                 page=rng.choice((16, 32, 64, 64, 128, 256)), batch=_log_uniform(rng, 1, 96), ctx=_log_uniform(rng, 1, 60000),
                 new=rng.choice((1, 1, 1, rng.randint(2, 9), _log_uniform(rng, 10, 2500))), ragged=rng.random() < 0.75,
                 causal=rng.random() < 0.7)
    if what == "append":
        case["bounds"] = rng.random() < 0.6
        case["ctx"] = min(case["ctx"], 4096)
    if what == "sparse":
        case.update(top=rng.randint(3, 64), first=rng.randint(0, 1), last=rng.randint(1, 2))
    if what in ("share", "compact"):
        case.update(dtype=rng.choice(("bf16", "bf16", "fp8", "fp4", "f32")), bounds=rng.random() < 0.4)
    if what == "share":
        case.update(beams=rng.randint(2, 8), batch=_log_uniform(rng, 2, 800), ctx=min(case["ctx"], 8192), new=min(case["new"], 100))
    if what == "compact":
        case.update(percent=rng.randint(5, 95), runs=_log_uniform(rng, 1, 600), new=1)
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
    if case["what"] in ("share", "compact"):
        return rows * case["kv_heads"] * case["d"] * (2 if case["dtype"] == "f32" else 1) / 5e8
    pairs = case["batch"] * case["new"] * (case["ctx"] + case["new"]) * case["q_heads"]
    return max(rows * case["kv_heads"] * case["d"] / 1e9, pairs * case["d"] / 8e10, pairs / 8e8,
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


# ---- 4-bit rows -------------------------------------------------------------------------------------------------------

def _encode(x):
    """[..., d] -> E2M1 codes [..., d / 2] and scale bytes [..., d / 32]."""
    blocks = x.float().unflatten(-1, (-1, 32))
    m, e = torch.frexp(blocks.abs().amax(-1))
    e = torch.where(m > 0, torch.where(m <= 0.875, e - 3, e - 2), _LEAST_EXPONENT).clamp(_LEAST_EXPONENT, _MOST_EXPONENT)
    y = torch.ldexp(blocks, -e[..., None])
    a = y.abs()
    # steps of a half up to 2, of 1 up to 4, of 2 beyond; ties to even
    code = torch.where(a < 2, torch.round(2 * a), torch.where(a < 4, 2 + torch.round(a), 4 + torch.round(a / 2)))
    code = code.clamp(max=7).to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)
    code = code.flatten(-2)
    return code[..., ::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _decode(codes, scales):
    """fp32 values [..., d] of codes [..., d / 2] and scale bytes [..., d / 32]."""
    both = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()
    x = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=codes.device)[both]
    return torch.ldexp(x.unflatten(-1, (-1, 32)), scales.int()[..., None] - 127).flatten(-2)


def _pack(rows, page):
    """[pages, heads, page, d] values -> 4-bit pages [pages, heads, bytes]."""
    codes, scales = (x.unflatten(2, (page // 16, 16)).flatten(3) for x in _encode(rows))
    return torch.cat([codes, scales], -1).flatten(2)


def _unpack(pages, case):
    """4-bit pages [..., bytes] -> fp32 values [..., page, d]."""
    d, page = case["d"], case["page"]
    x = pages.unflatten(-1, (page // 16, 16 * (d // 2 + d // 32)))
    codes, scales = x[..., :8 * d].unflatten(-1, (16, d // 2)), x[..., 8 * d:].unflatten(-1, (16, d // 32))
    return _decode(codes, scales).flatten(-3, -2)


def _row_bytes(case):
    """Where the bytes of each of a page's rows lie within the page, codes before scale bytes: [page, d / 2 + d / 32]."""
    d = case["d"]
    r = torch.arange(case["page"], device="cuda:0")[:, None]
    start = r // 16 * (16 * (d // 2 + d // 32))
    return torch.cat([start + r % 16 * (d // 2) + torch.arange(d // 2, device=r.device),
                      start + 8 * d + r % 16 * (d // 32) + torch.arange(d // 32, device=r.device)], 1)


def _page_values(pages, case):
    """fp32 values [pages, heads, page, d] of the cache."""
    return _unpack(pages, case) if case["dtype"] == "fp4" else pages.float()


def _bytes_of(pages, case):
    """A view [pages, heads, page, bytes of a row] of pages whose rows are contiguous (not the 4-bit ones)."""
    return pages.view(torch.uint8).view(*pages.shape[:3], -1)


# ---- what a program has in hand ---------------------------------------------------------------------------------------

def _key_bounds(st, case, pages, fill):
    if not (case["bounds"] or case["what"] == "sparse"):
        st.update(bounds=None, scales=None)
        return
    st["bounds"], st["scales"] = _page_bounds(_page_values(pages, case), fill)


def _filled(gen, case, num_pages, phys, fill, drift):
    """K and V pages whose pages `phys` hold rows, the first `fill` of each; the rest zeros."""
    page, H, d = case["page"], case["kv_heads"], case["d"]
    dev = gen.device
    valid = (torch.arange(page, device=dev) < fill[:, None])[:, None, :, None]
    out = []
    for drifts in (drift, False):
        rows = _rows(gen, case, phys.numel() * page, H, drifts, _TORCH[case["dtype"]]).view(phys.numel(), page, H, d)
        rows = torch.where(valid, rows.transpose(1, 2), 0).contiguous()
        if case["dtype"] == "fp4":
            pages = torch.zeros(num_pages, H, page * (d // 2 + d // 32), dtype=torch.uint8, device=dev)
            pages.index_copy_(0, phys, _pack(rows, page))
        else:
            store = torch.float8_e4m3fn if case["dtype"] == "fp8" else rows.dtype
            pages = torch.zeros(num_pages, H, page, d, dtype=store, device=dev)
            pages.view(torch.uint8).index_copy_(0, phys, rows.to(store).view(torch.uint8))
        out.append(pages)
    return out


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 7919 + 37)
    if case["what"] in ("share", "compact"):
        return _prepare_tables(case, int(seed), gen)
    page, B = case["page"], case["batch"]
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
    owner = torch.repeat_interleave(torch.arange(B, device=dev), h)
    nth = torch.arange(sum(held), device=dev) - (torch.cumsum(h, 0) - h)[owner]
    fill = (torch.tensor(lens, device=dev)[owner] - nth * page).clamp(0, page)
    phys = order[:sum(held)].long()
    drift = case["what"] == "sparse" or case["bounds"]
    k_pages, v_pages = _filled(gen, case, num_pages, phys, fill, drift)
    st = dict(case=case, num_pages=num_pages, max_pages=max_pages, lens=_ints(lens, dev), table=table, q_start=_ints(starts, dev),
              k_pages=k_pages, v_pages=v_pages, total=total, tokens=tokens, max_new=max(max(new), 1),
              sm=1.0 / math.sqrt(case["d"]), shape=None, ws=None)
    every = torch.zeros(num_pages, dtype=torch.int64, device=dev)
    every[phys] = fill
    _key_bounds(st, case, k_pages, every)
    if case["what"] == "append":
        flat = torch.repeat_interleave(torch.arange(B, device=dev), torch.tensor(new, device=dev))
        j = torch.arange(total, device=dev) - torch.tensor(starts, device=dev)[flat]
        pos = torch.tensor(cached, device=dev)[flat] + j
        slots = torch.full((tokens,), -1, dtype=torch.int32, device=dev)
        slots[:total] = table[flat, pos // page] * page + (pos % page).to(torch.int32)
        # keys and values are slices of one fused projection of the tokens
        heads = case["q_heads"] + 2 * case["kv_heads"]
        qkv = _rows(gen, case, tokens, heads, drift, torch.bfloat16)
        st.update(slots=slots, k_new=qkv[:, case["q_heads"]:case["q_heads"] + case["kv_heads"]],
                  v_new=qkv[:, case["q_heads"] + case["kv_heads"]:])
        _read_into(st, tokens)
        return st
    q = _rows(gen, case, tokens, case["q_heads"], drift, torch.bfloat16)
    st.update(q=q, out=torch.zeros_like(q), lse=torch.zeros(tokens, case["q_heads"], dtype=torch.float32, device=dev))
    if case["what"] == "sparse":
        st["selected"] = torch.full((tokens, case["kv_heads"], case["top"]), -1, dtype=torch.int32, device=dev)
    return st


def _read_into(st, rows):
    """Places for the values of rows that are read back."""
    case = st["case"]
    for name in ("k_read", "v_read"):
        st[name] = torch.zeros(rows, case["kv_heads"], case["d"], dtype=_TORCH[case["dtype"]], device="cuda:0")


def _table_lengths(case):
    """Cached tokens of every request; those of a group of `beams` are alike."""
    cached, _ = _lengths(case)
    return [cached[b - b % case["beams"]] for b in range(case["batch"])] if case["what"] == "share" else cached


def _kept_of(n, percent):
    """How many of n tokens a policy keeps."""
    inner = max(0, n - 2 * _EDGE)
    return n - inner * percent // 100


def _prepare_tables(case, seed, gen):
    dev = gen.device
    page, B, beams = case["page"], case["batch"], case["beams"]
    r, by_seed = random.Random(7919 * B + 13 * case["ctx"] + page), random.Random(seed * 104729 + 11)
    lens = _table_lengths(case)
    held = [_pages(n, page) for n in lens]
    st = dict(case=case, shape=None, ws=None)
    # Full pages of a group's common beginning are one request's, held by all of them; what follows is each one's own.
    ids, start, common, spent = [], {}, [], 0
    for b in range(B):
        if case["what"] == "share" and b % beams:
            n = common[-1]
        else:
            n = 0
            start[b] = spent
            common.append(lens[b] // page * r.randint(50, 100) // 100)
        first = start[b - b % beams] if case["what"] == "share" else spent
        ids.append((first, n, spent))
        spent += held[b] - n
    if case["what"] == "share":
        # rows that end, rows that continue another one of their group; a draft is cut back, or a whole prompt's part comes
        parent, keep, new = [], [], []
        for b in range(B):
            group = b - b % beams
            p = by_seed.randrange(group, min(group + beams, B))
            if case["ragged"] and r.random() < 0.15:
                p = -1
            n = 0 if p < 0 else lens[p]
            parent.append(p)
            keep.append(n - min(n, r.randint(0, 8)) if case["ragged"] and r.random() < 0.3 else n)
            new.append(r.randint(1, case["new"]) if p >= 0 else 0)
        most = max(lens) + case["new"]
        spare = sum(_pages(k + n, page) - k // page for k, n in zip(keep, new))
        tokens = sum(new) + (37 if case["ragged"] else 0)
        st.update(parent=_ints(parent, dev), keep=_ints(keep, dev), new=_ints(new, dev), tokens=tokens,
                  q_start=_ints([0] * (B + 1), dev), slots=_ints([0] * max(tokens, 1), dev))
    else:
        most = max(lens)
        spare = sum(_pages(_kept_of(n, case["percent"]), page) for n in lens)
    max_pages = _pages(most, page) + 1
    num_pages = spent + spare + 17
    order = torch.randperm(num_pages, generator=gen, device=dev).to(torch.int32)
    cols = torch.arange(max_pages, device=dev)
    first, n, rest = (torch.tensor(x, device=dev)[:, None] for x in zip(*ids))
    at = torch.where(cols < n, first + cols, rest + cols - n).clamp(max=num_pages - 1)
    is_held = cols < torch.tensor(held, device=dev)[:, None]
    table = torch.where(is_held, order[at], 0)
    holders = torch.bincount(table[is_held].long(), minlength=num_pages).to(torch.int32)
    head = seed % num_pages  # the ring has been round a few times
    ring = torch.roll(torch.cat([order[spent:], order[:spent]]), head)
    # lens, head and length of the ring, ring, holders and table one behind the other, so that a pass can start from them anew
    parts = [_ints(lens, dev), _ints([head, num_pages - spent], dev), ring, holders, table.flatten().to(torch.int32)]
    st.update(num_pages=num_pages, max_pages=max_pages, before=torch.cat(parts), sizes=[x.numel() for x in parts])
    st["now"] = torch.empty_like(st["before"])
    st["status"] = torch.zeros(2, dtype=torch.int32, device=dev)
    phys = order[:spent].long()
    fill = torch.zeros(num_pages, dtype=torch.int64, device=dev)
    rows = (torch.tensor(lens, device=dev)[:, None] - cols * page).clamp(0, page)
    fill[table[is_held].long()] = rows[is_held]
    st["k_pages"], st["v_pages"] = _filled(gen, case, num_pages, phys, fill[phys], case["bounds"])
    _key_bounds(st, case, st["k_pages"], fill)
    if case["what"] == "share":
        moves = (B, page)
    else:
        # A policy that drops a fixed share of what lies between the first and last tokens, in runs of about `runs` tokens.
        kept = torch.zeros(B, max_pages * page, dtype=torch.bool, device=dev)
        for b, m in enumerate(lens):
            inner = max(0, m - 2 * _EDGE)
            score = torch.rand(_pages(max(inner, 1), case["runs"]), generator=gen, device=dev)
            score = score.repeat_interleave(case["runs"])[:inner]
            kept[b, :m] = True
            drop = torch.argsort(score, stable=True)[:inner * case["percent"] // 100]
            kept[b, _EDGE + drop] = False
        st["kept"] = kept
        moves = (sum(_kept_of(m, case["percent"]) for m in lens) + 37,)
    st["move_from"] = torch.zeros(moves, dtype=torch.int32, device=dev)
    st["move_to"] = torch.zeros(moves, dtype=torch.int32, device=dev)
    if case["dtype"] == "fp4":
        _read_into(st, st["move_to"].numel())
    return st


def _parts(st, x):
    """lens, ring's span, ring, holders, table out of a state's one array of integers."""
    lens, span, ring, holders, table = torch.split(x, st["sizes"])
    return lens, span, ring, holders, table.view(-1, st["max_pages"])


# ---- plain forms ------------------------------------------------------------------------------------------------------

def _power_of_two(amax):
    """The least power of two that amax fits 127 times, no less than 2^_LEAST_EXPONENT."""
    m, x = torch.frexp(amax)
    e = torch.where(m <= 127.0 / 128.0, x - 7, x - 6)
    e = torch.where(amax > 0, e, _LEAST_EXPONENT).clamp(min=_LEAST_EXPONENT)
    return torch.ldexp(torch.ones_like(amax), e)


def _finite(x):
    return torch.nan_to_num(x.float(), nan=0.0, posinf=_CLAMP, neginf=-_CLAMP).clamp(-_CLAMP, _CLAMP)


def _page_bounds(values, fill):
    """8-bit bounds of the keys on every page: codes [pages, heads, 2, d] of the largest and of minus the smallest value of
    each channel over the page's first `fill` rows, and their power of two [pages, heads]; zeros for an empty page."""
    x = _finite(values)
    rows = torch.arange(x.shape[2], device=x.device)
    valid = (rows < fill[:, None])[:, None, :, None]
    top = torch.where(valid, x, -math.inf).amax(2)
    low = torch.where(valid, -x, -math.inf).amax(2)
    some = (fill > 0)[:, None, None]
    both = torch.where(some[..., None], torch.stack([top, low], 2), 0.0)
    scale = _power_of_two(both.abs().amax((2, 3)))
    codes = torch.ceil(both.double() / scale[..., None, None].double())  # in 32 bits a small channel next to a huge one underflows
    return codes.to(torch.int8), torch.where(some[..., 0], scale, 0.0)


def _renew_bounds(st, slots):
    """Of the pages that `slots` are on, up to the last of them."""
    case = st["case"]
    if not case["bounds"]:
        return []
    page = slots // case["page"]
    fill = torch.zeros(st["num_pages"], dtype=torch.int64, device=slots.device)
    fill = fill.scatter_reduce(0, page, slots % case["page"] + 1, "amax")
    bounds, scales = _page_bounds(_page_values(st["k_pages"], case), fill)
    touched = (fill > 0)[:, None]
    st["bounds"].copy_(torch.where(touched[..., None, None], bounds, st["bounds"]))
    st["scales"].copy_(torch.where(touched, scales, st["scales"]))
    return [st["bounds"], st["scales"]]


def _plain_read(st, slots, real):
    """The values of rows; where `real` does not hold, what was there."""
    case, out = st["case"], []
    at = torch.where(real, slots.long(), 0)
    where = _row_bytes(case)[at % case["page"]]
    for pages, name in ((st["k_pages"], "k_read"), (st["v_pages"], "v_read")):
        raw = torch.gather(pages[at // case["page"]], 2, where[:, None].expand(-1, case["kv_heads"], -1))
        x = _decode(raw[..., :case["d"] // 2], raw[..., case["d"] // 2:])
        out.append(torch.where(real[:, None, None], x.to(st[name].dtype), st[name]))
    return out


def _plain_append(st):
    case = st["case"]
    slots = st["slots"][:st["total"]].long()
    page, off = slots // case["page"], slots % case["page"]
    where = _row_bytes(case)[off][:, None]
    heads = torch.arange(case["kv_heads"], device=slots.device)[None, :, None]
    for new, pages in ((st["k_new"], st["k_pages"]), (st["v_new"], st["v_pages"])):
        pages[page[:, None, None], heads, where] = torch.cat(_encode(new[:st["total"]]), -1)
    bounds = _renew_bounds(st, slots)
    return _plain_read(st, st["slots"], torch.arange(st["tokens"], device=slots.device) < st["total"]) + bounds


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


def _query_codes(q, kv_heads):
    """[tokens, kv_heads, 2 d]: sums over a group's queries of their positive and of their negative parts, as whole numbers."""
    x = _finite(q).view(q.shape[0], kv_heads, -1, q.shape[2])
    code = torch.round(x / _power_of_two(x.abs().amax((2, 3)))[:, :, None, None])
    return torch.cat([code.clamp(min=0).sum(2), (-code).clamp(min=0).sum(2)], -1)


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
    k = _unpack(st["k_pages"][at], case).transpose(1, 2).reshape(B, H, S, d)
    pad_t = (st["q_start"].long()[:-1, None] + torch.arange(n_max, device=t.device)).clamp(max=st["tokens"] - 1)
    q = st["q"].float()[pad_t].view(B, n_max, H, G, d).permute(0, 2, 1, 3, 4).reshape(B, H, n_max * G, d)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).view(B, H, n_max, G, S) * st["sm"]
    del k
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
    v = _unpack(st["v_pages"][at], case).transpose(1, 2).reshape(B, H, S, d)
    o = torch.matmul(p.view(B, H, n_max * G, S), v).view(B, H, n_max, G, d)
    o = torch.where(total > 0, o / total, 0.0)
    lse = torch.log(total) + m
    at_row = j.clamp(max=n_max - 1)
    o = o.permute(0, 2, 1, 3, 4)[b, at_row].reshape(st["tokens"], H * G, d)
    lse = torch.where(total > 0, lse, -math.inf)[..., 0].permute(0, 2, 1, 3)[b, at_row].reshape(st["tokens"], H * G)
    real = (t < st["q_start"].long()[-1])[:, None]
    return [torch.where(real[..., None], o.to(st["out"].dtype), st["out"]), torch.where(real, lse, st["lse"])]


def _count(holders, pages, by):
    """holders, with `by` added for every entry of `pages` (those behind the last page count for nothing)."""
    more = torch.cat([holders, holders[:1]])
    return more.scatter_add(0, pages.flatten(), torch.full_like(pages.flatten(), by))[:-1]


def _give_back(ring, head, count, before, after):
    """The pages that had holders and have none any more behind the ring's tail, in ascending order."""
    r = ring.numel()
    gone = (before > 0) & (after == 0)
    nth = torch.cumsum(gone, 0) - 1
    at = torch.where(gone, (head + count + nth) % r, r)
    ring = torch.cat([ring, ring[:1]]).scatter(0, at, torch.arange(r, device=ring.device))[:r]
    return ring, count + gone.sum()


def _plain_share(st):
    page, R = st["case"]["page"], st["num_pages"]
    lens, span, ring, holders, table = (x.long() for x in _parts(st, st["before"]))
    head, count = span[0], span[1]
    cols = torch.arange(table.shape[1], device=table.device)
    rows = torch.arange(lens.numel(), device=table.device)
    # Rows of the table that continue others
    parent = st["parent"].long()
    p = parent.clamp(min=0)
    held = (lens + page - 1) // page
    status = torch.where(((parent < -1) | (parent >= lens.numel())).any(), 5, 0)
    lens = torch.where(parent < 0, 0, lens[p])
    changed = (parent != rows)[:, None]
    gains, loses = changed & (cols < ((lens + page - 1) // page)[:, None]), changed & (cols < held[:, None])
    counted = _count(_count(holders, torch.where(gains, table[p], R), 1), torch.where(loses, table, R), -1)
    ring, count = _give_back(ring, head, count, holders, counted)
    table, holders = torch.where(gains, table[p], table), counted
    # The allocator's step
    keep, new = st["keep"].long(), st["new"].long()
    k, f, held = (keep + page - 1) // page, (keep + new + page - 1) // page, (lens + page - 1) // page
    last = table.gather(1, (keep // page)[:, None].clamp(max=table.shape[1] - 1))[:, 0]
    shared = (keep % page > 0) & (new > 0) & (holders[last] > 1)
    takes = f - k + shared
    q_start = torch.cat([torch.zeros_like(new[:1]), torch.cumsum(new, 0)])
    bad = (keep < 0) | (keep > lens) | (new < 0) | (f > table.shape[1])
    status2 = torch.where(bad.any(), 2, torch.where(q_start[-1] > st["slots"].numel(), 3, torch.where(takes.sum() > count, 1, 0)))
    first = (k - shared.long())[:, None]
    fresh = (cols >= first) & (cols < f[:, None])
    loses = ((cols >= k[:, None]) & (cols < held[:, None])) | (shared[:, None] & (cols == first))
    nth = (torch.cumsum(takes, 0) - takes)[:, None] + cols - first
    taken = torch.where(fresh, ring[(head + nth) % R], R)
    counted = _count(_count(holders, torch.where(loses, table, R), -1), taken, 1)
    ring, count = _give_back(ring, head, count, holders, torch.where(_count(torch.zeros_like(holders), taken, 1) > 0, 1, counted))
    table, holders = torch.where(fresh, taken, table), counted
    t = torch.arange(st["slots"].numel(), device=table.device)
    b = torch.searchsorted(q_start[1:].contiguous(), t, right=True).clamp(max=new.numel() - 1)
    pos = keep[b] + t - q_start[b]
    entry = table[b, (pos // page).clamp(0, table.shape[1] - 1)]
    slots = torch.where(t < q_start[-1], entry * page + pos % page, -1)
    off = torch.arange(page, device=table.device)
    copied = shared[:, None] & (off < (keep % page)[:, None])
    to = table.gather(1, first.clamp(min=0, max=table.shape[1] - 1))
    move_from = torch.where(copied, last[:, None] * page + off, -1)
    move_to = torch.where(copied, to * page + off, -1)
    span = torch.stack([(head + takes.sum()) % R, count - takes.sum()])
    out = [keep + new, span, ring, holders, table, q_start, slots, move_from, move_to, torch.stack([status, status2])]
    return [x.to(torch.int32) for x in out] + _plain_move(st, move_from.flatten(), move_to.flatten())


def _plain_compact(st):
    page, R = st["case"]["page"], st["num_pages"]
    lens, span, ring, holders, table = (x.long() for x in _parts(st, st["before"]))
    head, count = span[0], span[1]
    B = lens.numel()
    cols = torch.arange(table.shape[1], device=table.device)
    pos = torch.arange(table.shape[1] * page, device=table.device)
    real = pos < lens[:, None]
    kept = st["kept"] & real
    dropped = real & ~st["kept"]
    total = kept.sum(1)
    lead = torch.where(dropped.any(1), dropped.to(torch.uint8).argmax(1), lens)  # tokens in front of the first that is dropped
    cut = total == lead                                                          # nothing behind it stays: nothing moves
    first = torch.where(cut, (total + page - 1) // page, lead // page)
    want, held = (total + page - 1) // page, (lens + page - 1) // page
    takes = want - first
    starts, ends = first[:, None] * page, torch.where(cut, 0, lens)[:, None]
    moves = kept & (pos >= starts) & (pos < ends)
    status = torch.where(moves.sum() > st["move_to"].numel(), 3, torch.where(takes.sum() > count, 1, 0))
    fresh = (cols >= first[:, None]) & (cols < want[:, None])
    loses = (cols >= first[:, None]) & (cols < held[:, None])
    nth = (torch.cumsum(takes, 0) - takes)[:, None] + cols - first[:, None]
    taken = torch.where(fresh, ring[(head + nth) % R], R)
    counted = _count(_count(holders, torch.where(loses, table, R), -1), taken, 1)
    ring, count = _give_back(ring, head, count, holders, torch.where(_count(torch.zeros_like(holders), taken, 1) > 0, 1, counted))
    after = torch.where(fresh, taken, table)
    to_pos = (torch.cumsum(kept, 1) - 1).clamp(min=0)
    move_from = (table.repeat_interleave(page, 1) * page + pos % page)[moves]
    move_to = (after.gather(1, to_pos // page) * page + to_pos % page)[moves]
    pad = torch.full((st["move_to"].numel() - move_to.numel(),), -1, dtype=torch.int64, device=pos.device)
    move_from, move_to = torch.cat([move_from, pad]), torch.cat([move_to, pad])
    span = torch.stack([(head + takes.sum()) % R, count - takes.sum()])
    out = [total, span, ring, counted, after, move_from, move_to, status[None]]
    return [x.to(torch.int32) for x in out] + _plain_move(st, move_from, move_to)


def _plain_move(st, move_from, move_to):
    case, page = st["case"], st["case"]["page"]
    real = move_to >= 0
    f, t = move_from[real], move_to[real]
    heads = torch.arange(case["kv_heads"], device=f.device)[None, :, None]
    for pages in (st["k_pages"], st["v_pages"]):
        if case["dtype"] == "fp4":
            where = _row_bytes(case)
            pages[t[:, None, None] // page, heads, where[t % page][:, None]] = \
                pages[f[:, None, None] // page, heads, where[f % page][:, None]]
        else:
            rows = _bytes_of(pages, case)
            rows[t // page, :, t % page] = rows[f // page, :, f % page]
    bounds = _renew_bounds(st, t)
    if case["dtype"] == "fp4":
        return _plain_read(st, move_to, real) + bounds
    return [st["k_pages"], st["v_pages"]] + bounds


# ---- one pass ---------------------------------------------------------------------------------------------------------

def _own_shape(st):
    """The shape object and workspace that a program makes once."""
    import paper_2605_14877_amd as hk
    case = st["case"]
    formats = {"fp8": hk.KV_FP8_E4M3, "fp4": hk.KV_FP4_E2M1}
    st["shape"] = hk.PagedShape(case["q_heads"], case["kv_heads"], case["d"], case["page"], st["num_pages"], case["batch"],
                                st["max_pages"], "f32" if case["dtype"] == "f32" else "bf16",
                                formats.get(case["dtype"], hk.KV_NATIVE))
    n = 0
    if case["what"] in ("attend", "sparse"):
        n = hk.paged_attend_workspace_bytes(st["shape"], st["tokens"], case["top"])
    elif case["what"] in ("share", "compact"):
        n = hk.paged_tables_workspace_bytes(st["shape"])
    st["ws"] = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda:0")


def _own_tables(st):
    import paper_2605_14877_amd as hk
    case, shape = st["case"], st["shape"]
    st["now"].copy_(st["before"])  # a pass starts from the same tables each time
    lens, span, ring, holders, table = _parts(st, st["now"])
    if case["what"] == "share":
        hk.heatkv_paged_fork(shape, st["parent"], lens, holders, ring, span, table, st["status"][:1], st["ws"])
        hk.heatkv_paged_assign_shared(shape, st["keep"], st["new"], lens, holders, ring, span, table, st["q_start"], st["slots"],
                                      st["move_from"], st["move_to"], st["status"][1:], st["ws"])
        out = [lens, span, ring, holders, table, st["q_start"], st["slots"], st["move_from"], st["move_to"], st["status"]]
    else:
        hk.heatkv_paged_compact(shape, st["kept"], lens, holders, ring, span, table, st["move_from"], st["move_to"],
                                st["status"][:1], st["ws"])
        out = [lens, span, ring, holders, table, st["move_from"], st["move_to"], st["status"][:1]]
    hk.heatkv_paged_move(shape, st["move_from"], st["move_to"], st["k_pages"], st["v_pages"], st["bounds"], st["scales"])
    bounds = [st["bounds"], st["scales"]] if case["bounds"] else []
    if case["dtype"] != "fp4":
        return out + [st["k_pages"], st["v_pages"]] + bounds
    hk.heatkv_paged_read(shape, st["move_to"].view(-1), st["k_pages"], st["v_pages"], st["k_read"], st["v_read"])
    return out + [st["k_read"], st["v_read"]] + bounds


def _own_pass(st):
    import paper_2605_14877_amd as hk
    if st["shape"] is None:
        _own_shape(st)
    case, shape = st["case"], st["shape"]
    if case["what"] in ("share", "compact"):
        return _own_tables(st)
    if case["what"] == "append":
        hk.heatkv_paged_append(shape, st["slots"], st["k_new"], st["v_new"], st["k_pages"], st["v_pages"], st["bounds"],
                               st["scales"])
        hk.heatkv_paged_read(shape, st["slots"], st["k_pages"], st["v_pages"], st["k_read"], st["v_read"])
        return [st["k_read"], st["v_read"]] + ([st["bounds"], st["scales"]] if case["bounds"] else [])
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
    if what == "share":
        return _plain_share(st)
    if what == "compact":
        return _plain_compact(st)
    if what == "append":
        return _plain_append(st)
    if what == "attend":
        return _plain_attend(st)
    selected = _plain_select(st)
    return [selected] + _plain_attend(st, selected)


# ---- bytes and operations ---------------------------------------------------------------------------------------------

def work(case):
    """Bytes and operations of one pass: every input read once, every output written once."""
    page, d, H, Hq, B = case["page"], case["d"], case["kv_heads"], case["q_heads"], case["batch"]
    row = d * {"f32": 4.0, "bf16": 2.0, "fp8": 1.0, "fp4": 0.5 + 1 / 32}[case["dtype"]]
    if case["what"] == "share":
        lens = _table_lengths(case)
        held = sum(_pages(n, page) for n in lens)
        tokens = B * (1 + case["new"]) / 2
        copied = 0.5 * B * page * H if case["new"] else 0.0  # half a page of most requests
        return {"bytes": 4.0 * (8 * B + 4 * held + tokens + 2 * B * page) + 4 * row * copied, "flops": 4.0 * (B + held)}
    if case["what"] == "compact":
        lens = _table_lengths(case)
        moved = sum(max(0, _kept_of(n, case["percent"]) - _EDGE) for n in lens)
        pages = sum(_pages(n, page) for n in lens)
        byts = sum(lens) + 8.0 * moved + 4.0 * (6 * B + 5 * pages) + 4 * moved * H * row
        if case["dtype"] == "fp4":
            byts += 2 * moved * H * d * 2.0
        return {"bytes": byts, "flops": 2.0 * sum(lens)}
    cached, new = _lengths(case)
    total = sum(new)
    if case["what"] == "append":
        byts, flops = 2.0 * total * H * (2 * 2 * d + row) + 4.0 * total, 4.0 * total * H * d
        if case["bounds"]:
            touched = sum(_pages(c + n, page) - c // page for c, n in zip(cached, new) if n)
            older = sum(c % page for c, n in zip(cached, new) if n)
            byts += H * (older * row + touched * (2.0 * d + 4))
            flops += 2.0 * H * d * (older + total)
        return {"bytes": byts, "flops": flops}
    byts, flops = total * Hq * (2.0 * d * 2 + 4), 0.0
    for c, n in zip(cached, new):
        if not n:
            continue
        seen = [c + i + 1 if case["causal"] else c + n for i in range(n)]
        if case["what"] == "attend":
            byts += 2.0 * (c + n) * H * row
            flops += 4.0 * d * Hq * sum(seen)
        else:
            chosen = [min(s, case["top"] * page) for s in seen]
            pages = [_pages(s, page) for s in seen]
            byts += 2.0 * min(c + n, sum(chosen)) * H * row + pages[-1] * H * (2.0 * d + 4)
            byts += 4.0 * n * H * case["top"]
            flops += 4.0 * d * Hq * sum(chosen) + 4.0 * d * H * sum(pages)
    return {"bytes": byts, "flops": flops}


# ---- from the definitions, in 64 bits ---------------------------------------------------------------------------------

def _exact_rows(x):
    """[..., d] -> the values that 4 bits hold: of each block the nearest multiples of its power of two."""
    b = x.double().unflatten(-1, (-1, 32))
    e = torch.ceil(torch.log2(b.abs().amax(-1, keepdim=True) / 7)).clamp(_LEAST_EXPONENT, _MOST_EXPONENT)
    grid = torch.tensor([(1 + f / 2) * 2.0 ** g for g in (0, 1, 2) for f in (0, 1)], dtype=torch.float64, device=x.device)
    grid = torch.cat([torch.tensor([0.0, 0.5], dtype=torch.float64, device=x.device), grid])
    y = b.abs() * torch.exp2(-e)
    # above the middle of two neighbours the larger one; in the middle the one with an even number
    code = torch.zeros(y.shape, dtype=torch.int64, device=x.device)
    for i, middle in enumerate(((grid[1:] + grid[:-1]) / 2).tolist()):
        code += (y > middle) | ((y == middle) & (i % 2 == 1))
    return (grid[code] * torch.exp2(e) * torch.sign(b)).flatten(-2)


def _exact_values(pages, ids, h, case):
    """[rows, d] of kv head h on the pages `ids`, byte by byte."""
    d = case["d"]
    g = pages[ids, h].reshape(-1, 16 * (d // 2 + d // 32)).long()
    codes, scales = g[:, :8 * d].reshape(-1, d // 2), g[:, 8 * d:].reshape(-1, d // 32)
    nibbles = torch.stack([codes % 16, codes // 16], 2).reshape(-1, d)
    m = nibbles % 8
    mag = torch.where(m < 2, m / 2.0, (1 + (m % 2) / 2.0) * torch.exp2((m // 2 - 1).double()))
    return mag.double() * (1 - 2 * (nibbles // 8)) * torch.exp2(scales.double() - 127).repeat_interleave(32, 1)


def _exact_moves(st):
    """(from, to, rows) of every run of rows that a pass moves, from lists of pages."""
    case, page = st["case"], st["case"]["page"]
    lens, span, ring, _, table = (x.tolist() for x in _parts(st, st["before"]))
    free = [ring[(span[0] + i) % len(ring)] for i in range(span[1])]
    held = [row[:_pages(n, page)] for n, row in zip(lens, table)]
    moves = []
    if case["what"] == "share":
        # The ring is long enough for the step without the pages that come back in it.
        parent, keep, new = st["parent"].tolist(), st["keep"].tolist(), st["new"].tolist()
        held = [[] if p < 0 else held[p] for p in parent]
        count = {}
        for p in sum(held, []):
            count[p] = count.get(p, 0) + 1
        for pages, k, n in zip(held, keep, new):
            if k % page and n and count[pages[k // page]] > 1:
                moves.append((pages[k // page] * page, free.pop(0) * page, k % page))
            del free[:_pages(k + n, page) - _pages(k, page)]
        return moves
    for pages, n, kept in zip(held, lens, st["kept"].tolist()):
        stay = [i for i in range(n) if kept[i]]
        lead = next((i for i in range(n) if not kept[i]), n)
        if len(stay) == lead:
            continue
        first = lead // page
        fresh = [free.pop(0) for _ in range(_pages(len(stay), page) - first)]
        for j in range(first * page, len(stay)):
            moves.append((pages[stay[j] // page] * page + stay[j] % page, fresh[j // page - first] * page + j % page, 1))
    return moves


def _exact_pages(st):
    case, page = st["case"], st["case"]["page"]
    moves = _exact_moves(st)
    f = torch.tensor([a + i for a, _, n in moves for i in range(n)], dtype=torch.int64, device="cuda:0")
    t = torch.tensor([b + i for _, b, n in moves for i in range(n)], dtype=torch.int64, device="cuda:0")
    out = []
    for pages in (st["k_pages"], st["v_pages"]):
        x = pages.double().transpose(1, 2).flatten(0, 1)
        x[t] = x[f]
        out.append(x.unflatten(0, (-1, page)).transpose(1, 2))
    return out


def exact(case, seed):
    tables = case["what"] in ("share", "compact")
    if tables and case["dtype"] == "fp4":
        return None  # integers, and values that other cases form
    st = prepare(case, seed)
    if tables:
        whole = [None] * (10 if case["what"] == "share" else 8)
        return whole + _exact_pages(st) + ([None, None] if case["bounds"] else [])
    cached, new = _lengths(case)
    page, H, G = case["page"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    if case["what"] == "append":
        out = []
        for x, y in ((st["k_new"], st["k_read"]), (st["v_new"], st["v_read"])):
            z = y.double()
            z[:st["total"]] = _exact_rows(x[:st["total"]])
            out.append(z)
        return out + ([None, None] if case["bounds"] else [])
    table = st["table"].tolist()
    sparse = case["what"] == "sparse"
    out, lse = st["out"].double(), st["lse"].double()
    t = 0
    for b, (c, n) in enumerate(zip(cached, new)):
        if not n:
            continue
        ids = torch.tensor(table[b][:_pages(c + n, page)], device=out.device)
        for h in range(H):
            unseen = _exact_unselected(st, b, t, c, n, h, ids) if sparse else None
            k = _exact_values(st["k_pages"], ids, h, case)[:c + n]
            v = _exact_values(st["v_pages"], ids, h, case)[:c + n]
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
