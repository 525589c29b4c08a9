"""ctypes front end of the paged 8-bit cache (include/lessdec.h, "Paged cache in 8 bits"): argument marshalling only.

Everything runs in the HIP kernels; torch is used for device memory and streams.
"""
from __future__ import annotations

import ctypes as C

from .binding import DTYPE_BF16, DTYPE_F16, LessdecError, PagesDesc, _check, _p, _stream, lib

BLOCK = 16


def lessdec_pages_workspace_bytes(desc: PagesDesc, max_rows: int) -> int:
    return int(lib().lessdec_pages_workspace_bytes(C.byref(desc), int(max_rows)))


def lessdec_pages_reset(desc: PagesDesc, stream=None):
    _check(lib().lessdec_pages_reset(C.byref(desc), _stream(stream)), "lessdec_pages_reset")


def lessdec_pages_reserve(desc: PagesDesc, n_new, granted, plan, stream=None):
    _check(lib().lessdec_pages_reserve(C.byref(desc), _p(n_new), _p(granted), _p(plan), _stream(stream)), "lessdec_pages_reserve")


def lessdec_pages_select(desc: PagesDesc, source, stream=None):
    _check(lib().lessdec_pages_select(C.byref(desc), _p(source), _stream(stream)), "lessdec_pages_select")


def lessdec_pages_compact(desc: PagesDesc, plan, stream=None):
    _check(lib().lessdec_pages_compact(C.byref(desc), _p(plan), _stream(stream)), "lessdec_pages_compact")


def lessdec_pages_copy(desc: PagesDesc, plan, max_pairs: int, stream=None):
    _check(lib().lessdec_pages_copy(C.byref(desc), _p(plan), int(max_pairs), _stream(stream)), "lessdec_pages_copy")


def lessdec_pages_append(desc: PagesDesc, layer: int, k, v, row_stride: int, start, rows: int, stream=None):
    _check(lib().lessdec_pages_append(C.byref(desc), layer, _p(k), _p(v), row_stride, _p(start), rows, _stream(stream)),
           "lessdec_pages_append")


def lessdec_pages_attend(desc: PagesDesc, layer: int, q, q_stride: int, out, lse, start, rows: int, max_new: int, stream=None):
    _check(lib().lessdec_pages_attend(C.byref(desc), layer, _p(q), q_stride, _p(out), _p(lse), _p(start), rows, max_new, _stream(stream)),
           "lessdec_pages_attend")


def lessdec_pages_share_ints(desc: PagesDesc, max_rows: int) -> int:
    return int(lib().lessdec_pages_share_ints(C.byref(desc), int(max_rows)))


def lessdec_pages_shared_workspace_bytes(desc: PagesDesc, max_rows: int) -> int:
    return int(lib().lessdec_pages_shared_workspace_bytes(C.byref(desc), int(max_rows)))


def lessdec_pages_share(desc: PagesDesc, start, rows: int, least_bytes: int, plan, stream=None):
    _check(lib().lessdec_pages_share(C.byref(desc), _p(start), rows, least_bytes, _p(plan), _stream(stream)), "lessdec_pages_share")


def lessdec_pages_attend_shared(desc: PagesDesc, layer: int, q, q_stride: int, out, lse, start, rows: int, max_new: int, plan, stream=None):
    _check(lib().lessdec_pages_attend_shared(C.byref(desc), layer, _p(q), q_stride, _p(out), _p(lse), _p(start), rows, max_new, _p(plan),
                                             _stream(stream)), "lessdec_pages_attend_shared")


def lessdec_pages_read(desc: PagesDesc, layer: int, slots, n: int, first: int, count: int, K, V, stream=None):
    _check(lib().lessdec_pages_read(C.byref(desc), layer, _p(slots), n, first, count, _p(K), _p(V), _stream(stream)),
           "lessdec_pages_read")


class PagedCache:
    """Owns the device buffers of a paged cache (or takes a program's own, `buffers`) and its descriptor.

    Plumbing only: allocation with torch, checks of tensors, pointer marshalling, no arithmetic.  dtype: "f16" or "bf16", of the
    rows that go in and come out.  max_rows: the most rows that an attend() gets in one call.  shared: whether there is scratch for
    attend_shared(), too.  Calls run on the cache's device, on its current stream if none is given.
    """

    # every buffer that makes up the cache (a checkpoint copies these)
    STATE = ("k_codes", "v_codes", "exps", "table", "length", "refs")

    def __init__(self, slots, pages, page_tokens, table_len, heads, head_dim, dtype, layers=1, q_per_kv=1, sinks=0, window=0,
                 scale=0.0, max_rows=0, device="cuda:0", buffers=None, shared=False):
        import torch
        if not torch.cuda.is_available():
            raise LessdecError("no GPU visible: lessdec has no CPU path")
        if dtype not in ("f16", "bf16"):
            raise LessdecError("PagedCache: dtype is 'f16' or 'bf16'")
        lib()
        self.torch = torch
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.tdtype = torch.float16 if dtype == "f16" else torch.bfloat16
        self.slots, self.pages, self.page_tokens, self.table_len = slots, pages, page_tokens, table_len
        self.heads, self.D, self.layers, self.G, self.max_rows = heads, head_dim, layers, max(1, int(q_per_kv)), max_rows
        d = PagesDesc()
        d.slots, d.pages, d.page_tokens, d.table_len = slots, pages, page_tokens, table_len
        d.heads, d.head_dim, d.q_per_kv, d.layers = heads, head_dim, q_per_kv, layers
        d.dtype = DTYPE_F16 if dtype == "f16" else DTYPE_BF16
        d.sinks, d.window, d.scale = sinks, window, scale
        self.shared = shared
        need = lessdec_pages_shared_workspace_bytes(d, max_rows) if shared else lessdec_pages_workspace_bytes(d, max_rows)
        if need == 0:
            raise LessdecError("lessdec_pages_workspace_bytes: invalid shape")
        blocks = layers * pages * heads * (page_tokens // BLOCK)
        sizes = {"k_codes": (blocks * BLOCK * head_dim, 1), "v_codes": (blocks * BLOCK * head_dim, 1), "exps": (2 * blocks, 1),
                 "table": (slots * table_len, 4), "length": (slots, 4), "refs": (pages, 4)}
        types = {"k_codes": torch.uint8, "v_codes": torch.uint8, "exps": torch.int8}
        for name, (count, size) in sizes.items():
            if buffers is None:
                t = torch.empty(count, dtype=types.get(name, torch.int32), device=self.device)
            else:
                t = buffers[name]
                if t.numel() != count or t.element_size() != size or t.device != self.device or not t.is_contiguous():
                    raise LessdecError(f"PagedCache: {name} must be {count} contiguous elements of {size} bytes on {self.device}")
            setattr(self, name, t)
            setattr(d, name, t.data_ptr())
        if buffers is None:
            self.table, self.exps = self.table.view(slots, table_len), self.exps.view(layers, pages, heads, page_tokens // BLOCK, 2)
        self.workspace = torch.zeros(need, dtype=torch.uint8, device=self.device)   # (zeros: lessdec.h)
        d.workspace, d.workspace_bytes = self.workspace.data_ptr(), need
        self.desc = d
        # torch.cuda.current_stream and current_device, by what they call: 0.2 us of a call's 5.6, 1.4 by the public names
        self._pointer, self._lib, self._current = C.pointer(d), lib(), (torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice)
        if buffers is None:
            self.reset()

    def _call(self, name, stream, *args):
        index, (raw_stream, device) = self.device.index, self._current
        s = raw_stream(index) if stream is None else stream.cuda_stream
        f = getattr(self._lib, name)
        if device() == index:
            rc = f(self._pointer, *args, s)
        else:
            with self.torch.cuda.device(index):
                rc = f(self._pointer, *args, s)
        if rc:
            _check(rc, name)

    def _ints(self, t, count, what):
        if t.dtype != self.torch.int32 or t.numel() < count or not t.is_contiguous() or t.device != self.device:
            raise LessdecError(f"{what} must be {count} contiguous int32 on {self.device}")
        return t.data_ptr()

    def _rows(self, t, heads, what):
        """(rows, elements from a row to the next) of a [rows, heads, D] tensor whose rows may lie apart."""
        shape, d = t.shape, self.D
        if len(shape) != 3 or shape[1] != heads or shape[2] != d or t.dtype != self.tdtype or t.device != self.device:
            raise LessdecError(f"{what} must be [rows, {heads}, {d}] {self.tdtype} on {self.device}")
        rows, (a, b, c) = shape[0], t.stride()
        if rows and (c != 1 or (b != d and heads > 1) or (rows > 1 and (a < heads * d or a % 8)) or t.data_ptr() % 16):
            raise LessdecError(f"{what}: heads of a row must be packed, rows 16-byte aligned and not overlap")
        return rows, a if rows > 1 else 0

    def reset(self, stream=None):
        """Every slot empty, every page free."""
        self._call("lessdec_pages_reset", stream)

    def reserve(self, n_new, granted, plan, stream=None):
        """Room for n_new int32 [slots] more tokens; granted int32 [slots] or None; plan int32 [1 + 2 slots], for copy()."""
        self._call("lessdec_pages_reserve", stream, self._ints(n_new, self.slots, "n_new"),
                   None if granted is None else self._ints(granted, self.slots, "granted"), self._ints(plan, 1 + 2 * self.slots, "plan"))

    def select(self, source, stream=None):
        """Slot s becomes a copy of slot source[s] (int32 [slots]; -1: becomes empty)."""
        self._call("lessdec_pages_select", stream, self._ints(source, self.slots, "source"))

    def compact(self, plan, stream=None):
        """Pages in use to the front of the pool; plan int32 [1 + 2 (pages // 2)], for copy()."""
        self._call("lessdec_pages_compact", stream, self._ints(plan, 1 + 2 * (self.pages // 2), "plan"))

    def copy(self, plan, max_pairs, stream=None):
        """Carries out a plan of at most max_pairs pairs of pages, in all layers."""
        self._call("lessdec_pages_copy", stream, self._ints(plan, 1 + 2 * max_pairs, "plan"), max_pairs)

    def append(self, layer, k, v, start, stream=None):
        """k, v [rows, heads, D] of the slots' last tokens; start int32 [slots + 1]."""
        n, step = self._rows(k, self.heads, "k")
        if self._rows(v, self.heads, "v") != (n, step):
            raise LessdecError("append: k and v must have the same rows and row stride")
        self._call("lessdec_pages_append", stream, layer, k.data_ptr(), v.data_ptr(), step, self._ints(start, self.slots + 1, "start"), n)

    def attend(self, layer, q, out, start, max_new, lse=None, stream=None):
        """q [rows, heads * q_per_kv, D] of the slots' last tokens, at most max_new of a slot; out the same, contiguous; lse fp32
        [rows, heads * q_per_kv] or None."""
        n, args = self._attention(layer, q, out, start, max_new, lse)
        self._call("lessdec_pages_attend", stream, *args, n, max_new)

    def _attention(self, layer, q, out, start, max_new, lse):
        n, step = self._rows(q, self.heads * self.G, "q")
        if out.dtype != self.tdtype or out.device != self.device or out.shape != q.shape or not out.is_contiguous():
            raise LessdecError("attend: out must be contiguous, like q")
        if lse is not None and (lse.dtype != self.torch.float32 or lse.device != self.device or not lse.is_contiguous() or
                                lse.numel() != n * self.heads * self.G):
            raise LessdecError("attend: lse must be contiguous fp32 [rows, heads * q_per_kv]")
        if n > self.max_rows:
            raise LessdecError(f"attend: {n} rows exceed max_rows={self.max_rows} the workspace was sized for")
        return n, (layer, q.data_ptr(), step, out.data_ptr(), None if lse is None else lse.data_ptr(), self._ints(start, self.slots + 1, "start"))

    def share_plan(self):
        """An int32 tensor for share(), for up to max_rows rows."""
        return self.torch.zeros(lessdec_pages_share_ints(self.desc, self.max_rows), dtype=self.torch.int32, device=self.device)

    def _plan(self, plan, rows):
        if rows > self.max_rows:
            raise LessdecError(f"share: {rows} rows exceed max_rows={self.max_rows} the workspace was sized for")
        return self._ints(plan, lessdec_pages_share_ints(self.desc, rows), "plan")

    def share(self, start, rows, plan, least_bytes=-1, stream=None):
        """What neighbouring slots have in common, for attend_shared() calls of `rows` rows; holds until slots, lengths or start change.
        Nothing is shared if that saves less than least_bytes of a layer's reading (-1: than has been measured to pay)."""
        self._call("lessdec_pages_share", stream, self._ints(start, self.slots + 1, "start"), rows, least_bytes,
                   self._plan(plan, rows))

    def attend_shared(self, layer, q, out, start, max_new, plan, lse=None, stream=None):
        """attend() that reads what slots share once for all of them; plan: of share() for these rows (with one for another number of rows, or slots, out is
        left as it is)."""
        if not self.shared:
            raise LessdecError("attend_shared: the cache was made without shared=True")
        n, args = self._attention(layer, q, out, start, max_new, lse)
        self._call("lessdec_pages_attend_shared", stream, *args, n, max_new, self._plan(plan, n))

    def read(self, layer, slots, first, K, V, stream=None):
        """K, V [n, heads, count, D]: tokens first .. first + count - 1 of slots (int32 [n]), from a slot's end if first < 0."""
        for t in (K, V):
            if t.dim() != 4 or t.dtype != self.tdtype or t.device != self.device or not t.is_contiguous() or t.shape != K.shape or \
                    t.shape[1] != self.heads or t.shape[3] != self.D:
                raise LessdecError(f"read: K and V must be contiguous [n, {self.heads}, count, {self.D}] {self.tdtype}")
        self._call("lessdec_pages_read", stream, layer, self._ints(slots, K.shape[0], "slots"), K.shape[0], first, K.shape[2],
                   K.data_ptr(), V.data_ptr())
