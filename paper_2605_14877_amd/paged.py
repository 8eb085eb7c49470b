"""Binding of the paged cache's calls (include/heatkv.h, "Paged cache"): same names, argument marshalling and checks only.

Token tensors are [tokens, heads, d] with any token and head stride; pages [num_pages, kv_heads, page_size, d] in the shape's
dtype, or E4M3 codes as torch.float8_e4m3fn or torch.uint8; 4-bit pages [num_pages, kv_heads, bytes of a page] are torch.uint8.
Integer arrays are int32 device tensors.

Calls go through the module _heatkv_call first (csrc/call_path.cpp: the same checks without the interpreter); it declines
whatever is not plainly in order, and the ctypes path below it names the mistake."""
from __future__ import annotations

import ctypes as C

from . import binding
from .binding import BF16, KV_FP4_E2M1, KV_FP8_E4M3, KV_NATIVE, _check, _DTYPES, lib

PAGED_OK, PAGED_NO_PAGES, PAGED_BAD_LENGTH, PAGED_TOO_MANY_TOKENS, PAGED_BAD_FREE_LIST = 0, 1, 2, 3, 4
PAGED_BAD_PARENT, PAGED_BAD_HOLDERS = 5, 6


class _CPagedShape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("q_heads", "kv_heads", "d", "dtype", "kv_format", "page_size", "num_pages", "batch",
                                         "max_pages")]


class _CRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


_bound = False


def _lib():
    global _bound
    L = lib()
    if not _bound:
        vp, sp, i64, f32 = C.c_void_p, C.POINTER(_CPagedShape), C.c_int64, C.c_float
        L.heatkv_paged_assign.restype = C.c_int
        L.heatkv_paged_assign.argtypes = [sp] + [vp] * 10 + [i64, vp, vp]
        L.heatkv_paged_append.restype = C.c_int
        L.heatkv_paged_append.argtypes = [sp, vp, i64, _CRows, _CRows, vp, vp, vp, vp, vp]
        L.heatkv_paged_attend_workspace_bytes.restype = C.c_size_t
        L.heatkv_paged_attend_workspace_bytes.argtypes = [sp, i64, C.c_int]
        L.heatkv_paged_attend.restype = C.c_int
        L.heatkv_paged_attend.argtypes = [sp, i64, _CRows, vp, vp, vp, vp, vp, f32, C.c_int, _CRows, vp, vp, C.c_size_t, vp]
        L.heatkv_paged_select.restype = C.c_int
        L.heatkv_paged_select.argtypes = [sp, i64, _CRows, vp, vp, vp, vp, vp] + [C.c_int] * 4 + [vp, vp]
        L.heatkv_paged_attend_selected.restype = C.c_int
        L.heatkv_paged_attend_selected.argtypes = [sp, i64, _CRows, vp, vp, vp, vp, vp, vp, C.c_int, f32, C.c_int, _CRows, vp,
                                                   vp, C.c_size_t, vp]
        n = C.c_size_t
        L.heatkv_paged_read.restype = C.c_int
        L.heatkv_paged_read.argtypes = [sp, vp, i64, vp, vp, _CRows, _CRows, vp]
        L.heatkv_paged_tables_workspace_bytes.restype = n
        L.heatkv_paged_tables_workspace_bytes.argtypes = [sp]
        L.heatkv_paged_fork.restype = C.c_int
        L.heatkv_paged_fork.argtypes = [sp] + [vp] * 10 + [n, vp]
        L.heatkv_paged_assign_shared.restype = C.c_int
        L.heatkv_paged_assign_shared.argtypes = [sp] + [vp] * 11 + [i64] + [vp] * 4 + [n, vp]
        L.heatkv_paged_compact.restype = C.c_int
        L.heatkv_paged_compact.argtypes = [sp] + [vp] * 10 + [i64] + [vp] * 2 + [n, vp]
        L.heatkv_paged_move.restype = C.c_int
        L.heatkv_paged_move.argtypes = [sp, vp, vp, i64] + [vp] * 5
        _bound = True
    return L


class PagedShape:
    """Heads, head dimension and types, the cache's pages, and the block table's rows (batch) and columns (max_pages)."""

    def __init__(self, q_heads, kv_heads, d, page_size, num_pages, batch, max_pages, dtype, kv_format=KV_NATIVE):
        self.q_heads, self.kv_heads, self.d = int(q_heads), int(kv_heads), int(d)
        self.page_size, self.num_pages = int(page_size), int(num_pages)
        self.batch, self.max_pages = int(batch), int(max_pages)
        self.dtype = _DTYPES[dtype] if isinstance(dtype, str) else int(dtype)
        self.kv_format = int(kv_format)
        self.c_struct = _CPagedShape(self.q_heads, self.kv_heads, self.d, self.dtype, self.kv_format, self.page_size,
                                     self.num_pages, self.batch, self.max_pages)
        self.pages_shape = (self.num_pages, self.kv_heads, self.page_size, self.d)
        if self.kv_format == KV_FP4_E2M1:
            self.pages_shape = (self.num_pages, self.kv_heads, self.page_size * (self.d // 2 + self.d // 32))
        self.address = C.addressof(self.c_struct)

    @property
    def ref(self):
        return C.byref(self.c_struct)


def _native(name, shape, *args):
    """True if the module _heatkv_call has made the call; it declines whatever is not plainly in order."""
    if type(shape) is not PagedShape:
        return False
    if binding._call is None:
        lib()
    rc = getattr(binding._call, name)(shape.address, *args)
    if rc is None:
        return False
    if rc:
        _check(rc)
    return True


class _Call:
    """Checks of one call's tensors.  The kernels trust sizes, so every operand is checked here, on the host: a wrong tensor
    becomes a Python error, not a memory fault on the GPU.  Tensors that overlap are refused by the C entries."""

    def __init__(self, shape):
        if not isinstance(shape, PagedShape):
            raise TypeError("shape: expected a PagedShape")
        self.lib = _lib()
        self.shape = shape
        self.torch = binding._torch
        self.device = None

    def tensor(self, x, name):
        torch = self.torch
        if not isinstance(x, torch.Tensor):
            raise TypeError(f"{name}: expected a torch tensor")
        if not x.is_cuda:
            raise ValueError(f"{name}: expected a device tensor")
        if self.device is None:
            self.device = x.device
            if x.device.index != torch.cuda.current_device():
                raise ValueError(f"{name} is on {x.device}, the current device is cuda:{torch.cuda.current_device()}")
        elif x.device != self.device:
            raise ValueError(f"{name} is on {x.device}, other tensors on {self.device}")

    def dense(self, x, name, dtypes, size=None):
        self.tensor(x, name)
        if x.dtype not in dtypes:
            raise ValueError(f"{name}: dtype {x.dtype}, expected {' or '.join(str(d) for d in dtypes)}")
        if not x.is_contiguous():
            raise ValueError(f"{name}: tensor must be contiguous")
        if size is not None and tuple(x.shape) != tuple(size):
            raise ValueError(f"{name}: shape {tuple(x.shape)} does not match {tuple(size)}")
        return x.data_ptr()

    def ints(self, x, name, *size):
        return self.dense(x, name, (self.torch.int32,), size)

    def rows(self, x, name, tokens, heads):
        self.tensor(x, name)
        sh = self.shape
        if x.dtype is not (self.torch.bfloat16 if sh.dtype == BF16 else self.torch.float32):
            raise ValueError(f"{name}: dtype {x.dtype} does not match the shape's")
        if x.dim() != 3 or (tokens is not None and x.shape[0] != tokens) or x.shape[1] != heads or x.shape[2] != sh.d:
            raise ValueError(f"{name}: shape {tuple(x.shape)} does not match {('tokens' if tokens is None else tokens, heads, sh.d)}")
        if x.stride(2) != 1 and x.numel():
            raise ValueError(f"{name}: rows must be contiguous")
        return _CRows(x.data_ptr(), x.stride(0), x.stride(1))

    def pages(self, x, name):
        torch, sh = self.torch, self.shape
        if sh.kv_format == KV_FP4_E2M1:
            types = (torch.uint8,)
        elif sh.kv_format == KV_FP8_E4M3:
            types = (torch.float8_e4m3fn, torch.uint8)
        else:
            types = (torch.bfloat16 if sh.dtype == BF16 else torch.float32,)
        return self.dense(x, name, types, sh.pages_shape)

    def requests(self, table, q_start, lens):
        sh = self.shape
        return (self.ints(table, "table", sh.batch, sh.max_pages), self.ints(q_start, "q_start", sh.batch + 1),
                self.ints(lens, "lens", sh.batch))

    def workspace(self, ws):
        if ws is None:
            return None, 0
        self.tensor(ws, "ws")
        if not ws.is_contiguous():
            raise ValueError("ws: tensor must be contiguous")
        return ws.data_ptr(), ws.numel() * ws.element_size()

    def bounds(self, bounds, bound_scales):
        sh = self.shape
        bp = sp = None
        if bounds is not None:
            bp = self.dense(bounds, "bounds", (self.torch.int8,), (sh.num_pages, sh.kv_heads, 2, sh.d))
        if bound_scales is not None:
            sp = self.dense(bound_scales, "bound_scales", (self.torch.float32,), (sh.num_pages, sh.kv_heads))
        return bp, sp

    def tables(self, lens, lens_out, holders, free_ring, free_span, free_span_out, table):
        """Addresses in the order of the C entries."""
        sh = self.shape
        return (self.ints(lens, "lens", sh.batch), self.ints(lens if lens_out is None else lens_out, "lens_out", sh.batch),
                self.ints(holders, "holders", sh.num_pages), self.ints(free_ring, "free_ring", sh.num_pages),
                self.ints(free_span, "free_span", 2),
                self.ints(free_span if free_span_out is None else free_span_out, "free_span_out", 2),
                self.ints(table, "table", sh.batch, sh.max_pages))

    def stream(self, stream):
        return self.torch.cuda.current_stream().cuda_stream if stream is None else stream


def heatkv_paged_assign(shape, keep, new_tokens, lens, free_ring, free_span, table, q_start, slots, status, lens_out=None,
                        free_span_out=None, stream=None):
    """One step of the page allocator.  lens_out, free_span_out: None for in place."""
    if _native("paged_assign", shape, keep, new_tokens, lens, free_ring, free_span, table, q_start, slots, status, lens_out,
               free_span_out, stream):
        return
    c, sh = _Call(shape), shape
    lens_out = lens if lens_out is None else lens_out
    free_span_out = free_span if free_span_out is None else free_span_out
    args = [c.ints(keep, "keep", sh.batch), c.ints(new_tokens, "new_tokens", sh.batch), c.ints(lens, "lens", sh.batch),
            c.ints(lens_out, "lens_out", sh.batch), c.ints(free_ring, "free_ring", sh.num_pages),
            c.ints(free_span, "free_span", 2), c.ints(free_span_out, "free_span_out", 2),
            c.ints(table, "table", sh.batch, sh.max_pages), c.ints(q_start, "q_start", sh.batch + 1)]
    c.dense(slots, "slots", (c.torch.int32,))
    if slots.dim() != 1:
        raise ValueError("slots: expected one dimension")
    _check(c.lib.heatkv_paged_assign(sh.ref, *args, slots.data_ptr(), slots.shape[0], c.ints(status, "status", 1),
                                     c.stream(stream)))


def heatkv_paged_append(shape, slots, k_new, v_new, k_pages, v_pages, bounds=None, bound_scales=None, stream=None):
    """The new tokens' rows into their slots; with bounds and bound_scales also the bounds of the pages that they touch."""
    if _native("paged_append", shape, slots, k_new, v_new, k_pages, v_pages, bounds, bound_scales, stream):
        return
    c, sh = _Call(shape), shape
    c.dense(slots, "slots", (c.torch.int32,))
    if slots.dim() != 1:
        raise ValueError("slots: expected one dimension")
    tokens = slots.shape[0]
    k, v = c.rows(k_new, "k_new", tokens, sh.kv_heads), c.rows(v_new, "v_new", tokens, sh.kv_heads)
    kp, vp = c.pages(k_pages, "k_pages"), c.pages(v_pages, "v_pages")
    bp, sp = c.bounds(bounds, bound_scales)
    _check(c.lib.heatkv_paged_append(sh.ref, slots.data_ptr(), tokens, k, v, kp, vp, bp, sp, c.stream(stream)))


def paged_attend_workspace_bytes(shape, tokens, top=0):
    return int(_lib().heatkv_paged_attend_workspace_bytes(shape.ref, int(tokens), int(top)))


def _attend_operands(c, q, k_pages, v_pages, table, q_start, lens, out, ws, lse):
    sh = c.shape
    qr = c.rows(q, "q", None, sh.q_heads)
    tokens = q.shape[0]
    operands = [tokens, qr, c.pages(k_pages, "k_pages"), c.pages(v_pages, "v_pages"), *c.requests(table, q_start, lens)]
    outr = c.rows(out, "out", tokens, sh.q_heads)
    lp = None if lse is None else c.dense(lse, "lse", (c.torch.float32,), (tokens, sh.q_heads))
    return operands, outr, lp, *c.workspace(ws)


def heatkv_paged_attend(shape, q, k_pages, v_pages, table, q_start, lens, sm_scale, out, ws=None, causal=True, lse=None,
                        stream=None):
    """Attention of the new tokens over all tokens of their requests, or (causal) those up to themselves."""
    if _native("paged_attend", shape, q, k_pages, v_pages, table, q_start, lens, None, sm_scale, out, ws, causal, lse, stream):
        return
    c = _Call(shape)
    operands, outr, lp, wp, n = _attend_operands(c, q, k_pages, v_pages, table, q_start, lens, out, ws, lse)
    _check(c.lib.heatkv_paged_attend(shape.ref, *operands, float(sm_scale), int(bool(causal)), outr, lp, wp, n, c.stream(stream)))


def heatkv_paged_select(shape, q, bounds, bound_scales, table, q_start, lens, first, last, selected, causal=True, stream=None):
    """The pages with the best scores for every new token and kv head, ascending, -1 behind the last; their number is
    selected's last dimension."""
    if _native("paged_select", shape, q, bounds, bound_scales, table, q_start, lens, first, last, selected, causal, stream):
        return
    c, sh = _Call(shape), shape
    if not 0 <= first < 2 ** 31 or not 1 <= last < 2 ** 31:
        raise ValueError("first must be at least 0, last at least 1, both below 2^31")
    qr = c.rows(q, "q", None, sh.q_heads)
    tokens = q.shape[0]
    bp = c.dense(bounds, "bounds", (c.torch.int8,), (sh.num_pages, sh.kv_heads, 2, sh.d))
    sp = c.dense(bound_scales, "bound_scales", (c.torch.float32,), (sh.num_pages, sh.kv_heads))
    requests = c.requests(table, q_start, lens)
    top = selected.shape[-1] if isinstance(selected, c.torch.Tensor) and selected.dim() == 3 else 0
    out = c.ints(selected, "selected", tokens, sh.kv_heads, top)
    _check(c.lib.heatkv_paged_select(sh.ref, tokens, qr, bp, sp, *requests, int(first), int(last), top, int(bool(causal)), out,
                                     c.stream(stream)))


def heatkv_paged_attend_selected(shape, q, k_pages, v_pages, table, q_start, lens, selected, sm_scale, out, ws=None,
                                 causal=True, lse=None, stream=None):
    """heatkv_paged_attend over the pages selected [tokens, kv_heads, top] of each token only."""
    if selected is not None and _native("paged_attend", shape, q, k_pages, v_pages, table, q_start, lens, selected, sm_scale, out,
                                        ws, causal, lse, stream):
        return
    c, sh = _Call(shape), shape
    operands, outr, lp, wp, n = _attend_operands(c, q, k_pages, v_pages, table, q_start, lens, out, ws, lse)
    top = selected.shape[-1] if isinstance(selected, c.torch.Tensor) and selected.dim() == 3 else 0
    sel = c.ints(selected, "selected", q.shape[0], sh.kv_heads, top)
    _check(c.lib.heatkv_paged_attend_selected(sh.ref, *operands, sel, top, float(sm_scale), int(bool(causal)), outr, lp, wp, n,
                                              c.stream(stream)))


def heatkv_paged_read(shape, slots, k_pages, v_pages, k_out, v_out, stream=None):
    """Rows of the cache by their slots, as values of the shape's dtype; rows of slots out of range are left as they are."""
    if _native("paged_read", shape, slots, k_pages, v_pages, k_out, v_out, stream):
        return
    c, sh = _Call(shape), shape
    c.dense(slots, "slots", (c.torch.int32,))
    if slots.dim() != 1:
        raise ValueError("slots: expected one dimension")
    tokens = slots.shape[0]
    kp, vp = c.pages(k_pages, "k_pages"), c.pages(v_pages, "v_pages")
    k, v = c.rows(k_out, "k_out", tokens, sh.kv_heads), c.rows(v_out, "v_out", tokens, sh.kv_heads)
    _check(c.lib.heatkv_paged_read(sh.ref, slots.data_ptr(), tokens, kp, vp, k, v, c.stream(stream)))


def paged_tables_workspace_bytes(shape):
    return int(_lib().heatkv_paged_tables_workspace_bytes(shape.ref))


def heatkv_paged_fork(shape, parent, lens, holders, free_ring, free_span, table, status, ws, lens_out=None, free_span_out=None,
                      stream=None):
    """Row b of the table continues row parent[b]; -1 ends it.  lens_out, free_span_out: None for in place."""
    if _native("paged_fork", shape, parent, lens, holders, free_ring, free_span, table, status, ws, lens_out, free_span_out, stream):
        return
    c, sh = _Call(shape), shape
    _check(c.lib.heatkv_paged_fork(sh.ref, c.ints(parent, "parent", sh.batch),
                                   *c.tables(lens, lens_out, holders, free_ring, free_span, free_span_out, table),
                                   c.ints(status, "status", 1), *c.workspace(ws), c.stream(stream)))


def heatkv_paged_assign_shared(shape, keep, new_tokens, lens, holders, free_ring, free_span, table, q_start, slots, copy_from,
                               copy_to, status, ws, lens_out=None, free_span_out=None, stream=None):
    """One step of the allocator that leaves pages alone which several rows hold.  copy_from, copy_to [batch, page_size] list the
    rows of such pages for heatkv_paged_move.  lens_out, free_span_out: None for in place."""
    if _native("paged_assign_shared", shape, keep, new_tokens, lens, holders, free_ring, free_span, table, q_start, slots, copy_from,
               copy_to, status, ws, lens_out, free_span_out, stream):
        return
    c, sh = _Call(shape), shape
    args = [c.ints(keep, "keep", sh.batch), c.ints(new_tokens, "new_tokens", sh.batch),
            *c.tables(lens, lens_out, holders, free_ring, free_span, free_span_out, table), c.ints(q_start, "q_start", sh.batch + 1)]
    c.dense(slots, "slots", (c.torch.int32,))
    if slots.dim() != 1:
        raise ValueError("slots: expected one dimension")
    _check(c.lib.heatkv_paged_assign_shared(sh.ref, *args, slots.data_ptr(), slots.shape[0],
                                            c.ints(copy_from, "copy_from", sh.batch, sh.page_size),
                                            c.ints(copy_to, "copy_to", sh.batch, sh.page_size), c.ints(status, "status", 1),
                                            *c.workspace(ws), c.stream(stream)))


def heatkv_paged_compact(shape, kept, lens, holders, free_ring, free_span, table, move_from, move_to, status, ws, lens_out=None,
                         free_span_out=None, stream=None):
    """Every request keeps the tokens that are marked in kept [batch, max_pages * page_size] (bool or uint8).  move_from, move_to list
    the rows that move for heatkv_paged_move.  lens_out, free_span_out: None for in place."""
    if _native("paged_compact", shape, kept, lens, holders, free_ring, free_span, table, move_from, move_to, status, ws, lens_out,
               free_span_out, stream):
        return
    c, sh = _Call(shape), shape
    kp = c.dense(kept, "kept", (c.torch.bool, c.torch.uint8), (sh.batch, sh.max_pages * sh.page_size))
    tables = c.tables(lens, lens_out, holders, free_ring, free_span, free_span_out, table)
    c.dense(move_to, "move_to", (c.torch.int32,))
    if move_to.dim() != 1:
        raise ValueError("move_to: expected one dimension")
    _check(c.lib.heatkv_paged_compact(sh.ref, kp, *tables, c.ints(move_from, "move_from", move_to.shape[0]), move_to.data_ptr(),
                                      move_to.shape[0], c.ints(status, "status", 1), *c.workspace(ws), c.stream(stream)))


def heatkv_paged_move(shape, move_from, move_to, k_pages, v_pages, bounds=None, bound_scales=None, stream=None):
    """Rows move_to of the cache become what rows move_from are (int32 arrays of one shape, of one or two dimensions); with bounds
    and bound_scales also the bounds of the pages that they touch.  A list of more than 2^23 / kv_heads rows is moved in pieces, by a
    call for each: cut anywhere, rows and bounds are the same."""
    if _native("paged_move", shape, move_from, move_to, k_pages, v_pages, bounds, bound_scales, stream):
        return
    c, sh = _Call(shape), shape
    c.dense(move_to, "move_to", (c.torch.int32,))
    if move_to.dim() not in (1, 2):
        raise ValueError("move_to: expected one or two dimensions")
    fp = c.ints(move_from, "move_from", *move_to.shape)
    kp, vp = c.pages(k_pages, "k_pages"), c.pages(v_pages, "v_pages")
    bp, sp = c.bounds(bounds, bound_scales)
    _check(c.lib.heatkv_paged_move(sh.ref, fp, move_to.data_ptr(), move_to.numel(), kp, vp, bp, sp, c.stream(stream)))
