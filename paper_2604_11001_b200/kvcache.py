"""ctypes binding of the paged key-value cache (include/fcsim_kv.h): append, attend, prefill, evict, read.

Argument checks and marshalling only -- the work is done by the CUDA library, on the current stream of the cache's
device.  PyTorch provides device memory and streams; there is no CPU fallback.

    cache = PagedKV.allocate(n_pages=1024, page_size=16, n_kv_heads=8, head_dim=128, weight=True)
    q = cache.append(q, k, v, positions, slots, rope=table, q_norm=w_q, k_norm=w_k)   # a slot's new tokens
    out = cache.attend(q, table, lengths, add_weight=True)                            # one query per request
    out = cache.prefill(q, starts, table, lengths)                                    # several, as of a prompt
    new_lengths, kept = cache.evict(table, lengths, budget, new_table, max_budget=512, recent=64, first=4)
    k, v = cache.read(slots)                                                          # what stands there
    cache.check()                                                                     # synchronises
"""
from __future__ import annotations

import ctypes as C
import math
import struct
import threading
import weakref

import torch

from . import binding as _fb

F16, BF16, E4M3 = 0, 1, 2
BAD_PAGE, BAD_LENGTH, BAD_POSITION, BAD_BUDGET, STUCK = 1, 2, 4, 8, 16
_TYPES = {torch.float16: F16, torch.bfloat16: BF16, torch.float8_e4m3fn: E4M3}
_I32, _I64 = torch.int32, torch.int64
_WIDE = frozenset((torch.float16, torch.bfloat16))
_ESIZE = -3
# device -> stream -> workspace of that stream's calls, whichever cache they are of (a stream's calls follow one another; the lock
# keeps the launches of one call together where threads share a stream)
_WORKSPACES = {}
_LOCK = threading.Lock()
# device -> (cache, its status word) of every cache whose word may hold something, also of those that are gone; and how often a wait was given up
# there: what that has left wrong is in the workspaces, which are all caches'
_STATUS, _GIVEN_UP = {}, {}
_NO_FIT = struct.error   # of a number that an argument struct has no room for
_MOST = 2 ** 31 - 2 ** 16   # tokens of a request or a budget, at most
_grad_enabled = torch.is_grad_enabled
# the current device's number and a device's current stream as plain integers, without the objects around them
_current_device, _current_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


class fcsim_kv_cache(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("k", "v", "weight", "k_scale", "v_scale")]
                + [(n, C.c_int64) for n in ("stride_page", "stride_slot", "stride_head")]
                + [(n, C.c_int32) for n in ("dtype", "n_pages", "page_size", "n_kv_heads", "head_dim", "reserved")])


class fcsim_kv_append_args(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("q", "k", "v", "q_out", "q_norm", "k_norm", "rope", "positions", "slots",
                                           "status")]
                + [(n, C.c_int64) for n in ("q_row", "q_head", "k_row", "k_head", "v_row", "v_head")]
                + [(n, C.c_int32) for n in ("n_tokens", "n_heads", "dtype", "rope_dim", "n_positions",
                                            "interleaved")]
                + [("eps", C.c_float), ("reserved", C.c_int32)])


class fcsim_kv_attend_args(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("q", "out", "lse", "table", "lengths", "status")]
                + [(n, C.c_int64) for n in ("q_row", "q_head", "table_row")]
                + [(n, C.c_int32) for n in ("n_requests", "n_heads", "dtype", "table_cols", "max_length", "window",
                                            "add_weight")]
                + [("scale", C.c_float), ("first", C.c_int32), ("reserved", C.c_int32)])


class fcsim_kv_prefill_args(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("q", "out", "lse", "starts", "table", "lengths", "status")]
                + [(n, C.c_int64) for n in ("q_row", "q_head", "table_row")]
                + [(n, C.c_int32) for n in ("n_rows", "n_requests", "n_heads", "dtype", "table_cols", "max_length", "window",
                                            "first")]
                + [("scale", C.c_float), ("reserved", C.c_int32)])


class fcsim_kv_evict_args(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("table", "lengths", "budget", "new_table", "new_lengths", "kept",
                                           "status")]
                + [(n, C.c_int64) for n in ("table_row", "new_row")]
                + [(n, C.c_int32) for n in ("n_requests", "table_cols", "new_cols", "max_length", "max_budget",
                                            "recent", "first", "reserved")])


class fcsim_kv_read_args(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("slots", "k_out", "v_out", "status")] + [("n_tokens", C.c_int32), ("dtype", C.c_int32)]


class fcsim_kv_workspace(C.Structure):
    _fields_ = [("bytes", C.c_size_t), ("zeroed", C.c_size_t)]


# the argument structs as one packing each (native sizes and alignment, as the compiler's)
_APPEND, _ATTEND, _EVICT = struct.Struct("10P6q6ifi"), struct.Struct("6P3q7if2i"), struct.Struct("7P2q8i")
_READ, _PREFILL = struct.Struct("4P2i"), struct.Struct("7P3q8ifi")
assert (_APPEND.size, _ATTEND.size, _EVICT.size) == (C.sizeof(fcsim_kv_append_args), C.sizeof(fcsim_kv_attend_args),
                                                     C.sizeof(fcsim_kv_evict_args))
assert (_READ.size, _PREFILL.size) == (C.sizeof(fcsim_kv_read_args), C.sizeof(fcsim_kv_prefill_args))

EXPORTS = ("fcsim_kv_append", "fcsim_kv_attend_workspace", "fcsim_kv_attend", "fcsim_kv_prefill_workspace", "fcsim_kv_prefill",
           "fcsim_kv_evict_workspace",
           "fcsim_kv_evict", "fcsim_kv_read", "fcsim_kv_last_cuda_error")

_lib = None


def load():
    """The CUDA library with the signatures of this module's entry points."""
    global _lib
    if _lib is None:
        lib = _fb.load()
        vp = C.c_void_p
        lib.fcsim_kv_append.argtypes = lib.fcsim_kv_read.argtypes = [vp, vp, vp]
        for name in ("attend", "prefill", "evict"):
            getattr(lib, f"fcsim_kv_{name}_workspace").argtypes = [vp, vp, C.POINTER(fcsim_kv_workspace)]
            getattr(lib, f"fcsim_kv_{name}").argtypes = [vp, vp, vp, C.c_size_t, vp]
        lib.fcsim_kv_last_cuda_error.argtypes = []
        for name in EXPORTS:
            getattr(lib, name).restype = C.c_int
        _lib = lib
    return _lib


def _raise(code, where):
    e = _fb.FcsimError(code, where)
    if code == -5:
        e.args = (f"{e.args[0]} [cudaError {load().fcsim_kv_last_cuda_error()}]",)
    raise e


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _refuse_gradient():
    raise ValueError("a tensor requires a gradient, and there is no backward pass: detach it, or call under no_grad()")


def _pointer(t):
    return 0 if t is None else t.data_ptr()


class PagedKV:
    """One layer's cache: ``k`` and ``v`` as [n_pages, page_size, n_kv_heads, head_dim] views of either memory order
    (head_dim contiguous), and what belongs to them.

    ``weight``: [n_pages, n_kv_heads, page_size] float32, the attention each cached token has received.
    ``k_scale``, ``v_scale``: [n_kv_heads] float32 for 8-bit caches: a stored x stands for x * scale.

    There is no backward pass: tensors that require a gradient are refused, unless gradients are off.
    Calls run on the current stream; calls on different streams that touch the same pages are the caller's to order.
    All caches of a device share one workspace per stream, kept for good.
    The object is not thread-safe."""

    def __init__(self, k, v, weight=None, k_scale=None, v_scale=None):
        _need(k.dim() == 4 and k.dtype in _TYPES and k.is_cuda, "k: a CUDA tensor [n_pages, page_size, n_kv_heads, "
              "head_dim] of float16, bfloat16 or float8_e4m3fn")
        _need(v.shape == k.shape and v.dtype == k.dtype and v.device == k.device and v.stride() == k.stride(),
              "v: shape, strides, type and device of k")
        n_pages, page_size, n_kv, head_dim = k.shape
        _need(k.stride(3) == 1 or head_dim == 1, "k, v: head_dim has to be contiguous")
        if weight is not None:
            _need(tuple(weight.shape) == (n_pages, n_kv, page_size) and weight.dtype == torch.float32
                  and weight.is_contiguous() and weight.device == k.device,
                  "weight: contiguous float32 [n_pages, n_kv_heads, page_size] on k's device")
        wide = k.dtype != torch.float8_e4m3fn
        for s in (k_scale, v_scale):
            _need(s is None if wide else (s is not None and tuple(s.shape) == (n_kv,) and s.dtype == torch.float32
                                          and s.is_contiguous() and s.device == k.device),
                  "k_scale, v_scale: None for 16-bit caches, contiguous float32 [n_kv_heads] for 8-bit ones")
        self.k, self.v, self.weight, self.k_scale, self.v_scale = k, v, weight, k_scale, v_scale
        self.n_pages, self.page_size, self.n_kv_heads, self.head_dim = n_pages, page_size, n_kv, head_dim
        self.device, self._index = k.device, k.get_device()
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self._status = self.status.data_ptr()
        torch.cuda.current_stream(k.device).synchronize()   # cleared, whatever stream the calls come on
        self._workspaces = _WORKSPACES.setdefault(self._index, {})   # of the device
        with _LOCK:
            _STATUS.setdefault(self._index, []).append((weakref.ref(self), self.status))
            self._given_up = _GIVEN_UP.setdefault(self._index, 0)   # what this cache's check() has told of
        self._c = fcsim_kv_cache(k.data_ptr(), v.data_ptr(), _pointer(weight), _pointer(k_scale), _pointer(v_scale),
                                 k.stride(0), k.stride(1), k.stride(2), _TYPES[k.dtype], n_pages, page_size, n_kv,
                                 head_dim, 0)
        self._c_ref = C.byref(self._c)
        load()

    @classmethod
    def allocate(cls, n_pages, page_size, n_kv_heads, head_dim, dtype=torch.bfloat16, *, heads_first=False,
                 weight=False, k_scale=None, v_scale=None, device="cuda:0"):
        """A zeroed cache.  ``heads_first``: pages laid out [n_kv_heads, page_size, head_dim] in memory."""
        def pool():
            if heads_first:
                return torch.zeros(n_pages, n_kv_heads, page_size, head_dim, dtype=dtype, device=device).transpose(1, 2)
            return torch.zeros(n_pages, page_size, n_kv_heads, head_dim, dtype=dtype, device=device)
        w = torch.zeros(n_pages, n_kv_heads, page_size, device=device) if weight else None
        if dtype == torch.float8_e4m3fn:
            one = torch.ones(n_kv_heads, device=device)
            k_scale = one if k_scale is None else k_scale
            v_scale = one.clone() if v_scale is None else v_scale
        return cls(pool(), pool(), w, k_scale, v_scale)

    # ------------------------------------------------------------------------------------------ helpers
    # A slot's calls take a few microseconds on the device: checks are plain comparisons, the argument struct is packed
    # in one go, and messages are only made when they are needed.
    def _refuse(self, name, what, x):
        raise ValueError(f"{name}: {what} on {self.device}, got {x.dtype} {list(x.shape)} on {x.device}")

    def _table(self, table, name, n):
        """Columns of a page table."""
        shape = table.shape
        if len(shape) != 2 or shape[0] != n or table.dtype != _I32 or table.get_device() != self._index \
                or not (shape[1] <= 1 or table.stride(1) == 1):
            self._refuse(name, f"int32 [{n}, pages], rows contiguous", table)
        return shape[1]

    def _call(self, entry, args, size=None):
        """Run an entry point on the current stream of the cache's device.  ``size``: the entry point that tells the size
        of its workspace, asked when the one at hand is too small."""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self._call(entry, args, size)
        stream = _current_stream(self._index)
        if size is None:
            code = entry(self._c_ref, args, stream)
        else:
            with _LOCK:
                buf = None if torch.cuda.is_current_stream_capturing() else self._workspaces.get(stream)
                if buf is None:  # (enough for the calls that need none)
                    code = entry(self._c_ref, args, None, 0, stream)
                else:
                    code = entry(self._c_ref, args, buf.data_ptr(), buf.numel(), stream)
                if code == _ESIZE:
                    need = fcsim_kv_workspace()
                    code = size(self._c_ref, args, C.byref(need))
                    if code == 0:
                        buf = self._workspace(stream, need.bytes, need.zeroed)
                        code = entry(self._c_ref, args, buf.data_ptr(), buf.numel(), stream)
        if code != 0:
            _raise(code, entry.__name__)

    def _workspace(self, stream, size, zeroed):
        """A new workspace, kept for the stream's later calls.  Its first `zeroed` bytes are cleared; every call leaves them
        as it found them, and the rest does not matter.  One that replaces a smaller one grows by half of it at least.  A graph
        under capture gets its own for each call, whose clearing is part of the graph."""
        capturing = torch.cuda.is_current_stream_capturing()
        old = None if capturing else self._workspaces.get(stream)
        if old is not None:
            size = max(size, old.numel() * 3 // 2)
        buf = torch.empty(max(size, 16), dtype=torch.uint8, device=self.device)
        buf[:zeroed].zero_()
        if not capturing:
            self._workspaces[stream] = buf
        return buf

    # ------------------------------------------------------------------------------------------ operators
    def append(self, q, k, v, positions, slots, *, rope=None, interleaved=False, q_norm=None, k_norm=None, eps=1e-6):
        """Normalise and rotate the heads of ``q`` [n, heads, head_dim] and ``k`` [n, n_kv_heads, head_dim], store k
        and ``v`` at ``slots`` (int64 [n], page * page_size + place, negative = not stored) and return q.

        ``rope``: float32 [positions, rope_dim], cosines then sines; ``positions``: int32 [n].  ``q_norm``,
        ``k_norm``: [head_dim] weights of the norms over each head.  ``q`` may be None (nothing is returned)."""
        if (k.requires_grad or v.requires_grad or (q is not None and q.requires_grad) or (rope is not None and rope.requires_grad)
                or (q_norm is not None and q_norm.requires_grad) or (k_norm is not None and k_norm.requires_grad)) and _grad_enabled():
            _refuse_gradient()
        dtype, shape, index = k.dtype, k.shape, self._index
        if dtype not in _WIDE or len(shape) != 3 or shape[1] != self.n_kv_heads or shape[2] != self.head_dim \
                or k.get_device() != index:
            self._refuse("k", f"float16 or bfloat16 [tokens, {self.n_kv_heads}, {self.head_dim}]", k)
        if v.shape != shape or v.dtype != dtype or v.get_device() != index:
            self._refuse("v", f"{dtype} {list(shape)}", v)
        n = shape[0]
        k_row, k_head, k_one = k.stride()
        v_row, v_head, v_one = v.stride()
        if slots.dtype != _I64 or slots.numel() != n or slots.get_device() != index or not slots.is_contiguous():
            self._refuse("slots", f"contiguous int64 [{n}]", slots)
        out, heads, q_row, q_head, q_one, q_at, out_at = None, 0, 0, 0, 1, 0, 0
        if q is not None:
            q_shape = q.shape
            if len(q_shape) != 3 or q_shape[0] != n or q_shape[2] != self.head_dim or q.dtype != dtype or q.get_device() != index:
                self._refuse("q", f"{dtype} [{n}, heads, {self.head_dim}]", q)
            heads = q_shape[1]
            q_row, q_head, q_one = q.stride()
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            q_at, out_at = q.data_ptr(), out.data_ptr()
        if k_one != 1 or v_one != 1 or q_one != 1:
            raise ValueError("q, k, v: head_dim has to be contiguous")
        rope_at = positions_at = rope_dim = n_positions = 0
        if rope is not None:
            if rope.dim() != 2 or rope.dtype != torch.float32 or rope.get_device() != index or not rope.is_contiguous():
                self._refuse("rope", "contiguous float32 [positions, rope_dim]", rope)
            if positions is None or positions.dtype != _I32 or positions.numel() != n or positions.get_device() != index \
                    or not positions.is_contiguous():
                raise ValueError(f"positions: contiguous int32 [{n}] on {self.device}")
            n_positions, rope_dim = rope.shape
            rope_at, positions_at = rope.data_ptr(), positions.data_ptr()
        q_norm_at = k_norm_at = 0
        if q_norm is not None:
            if q_norm.dtype != dtype or q_norm.numel() != self.head_dim or q_norm.get_device() != index or not q_norm.is_contiguous():
                self._refuse("q_norm", f"contiguous {dtype} [{self.head_dim}]", q_norm)
            q_norm_at = q_norm.data_ptr()
        if k_norm is not None:
            if k_norm.dtype != dtype or k_norm.numel() != self.head_dim or k_norm.get_device() != index or not k_norm.is_contiguous():
                self._refuse("k_norm", f"contiguous {dtype} [{self.head_dim}]", k_norm)
            k_norm_at = k_norm.data_ptr()
        try:
            args = _APPEND.pack(
                q_at, k.data_ptr(), v.data_ptr(), out_at, q_norm_at, k_norm_at, rope_at, positions_at, slots.data_ptr(),
                self._status, q_row, q_head, k_row, k_head, v_row, v_head, n, heads, _TYPES[dtype], rope_dim, n_positions,
                1 if interleaved else 0, eps, 0)
        except _NO_FIT as e:
            raise ValueError(f"append: {e}") from None
        self._call(_lib.fcsim_kv_append, args)
        return out

    def attend(self, q, table, lengths, *, max_length=None, scale=None, window=0, first=0, add_weight=False,
               return_lse=False):
        """Attention of one token per request: ``q`` [requests, heads, head_dim] over the ``lengths`` (int32) tokens
        that the rows of ``table`` (int32 [requests, pages]) hold; returns [requests, heads, head_dim], with
        ``return_lse`` also the float32 [requests, heads] log-sum-exp.

        ``max_length`` bounds the lengths (default: what the table's width holds).  ``window`` > 0: the newest tokens
        only, and the ``first`` oldest.  ``add_weight``: the cache's weights grow by each token's share (requests must not share pages)."""
        if q.requires_grad and _grad_enabled():
            _refuse_gradient()
        dtype, shape, index = q.dtype, q.shape, self._index
        if dtype not in _WIDE or len(shape) != 3 or shape[2] != self.head_dim or q.get_device() != index:
            self._refuse("q", f"float16 or bfloat16 [requests, heads, {self.head_dim}]", q)
        n, heads, _ = shape
        q_row, q_head, q_one = q.stride()
        if q_one != 1:
            raise ValueError("q: head_dim has to be contiguous")
        cols = self._table(table, "table", n)
        if lengths.dtype != _I32 or lengths.numel() != n or lengths.get_device() != index or not lengths.is_contiguous():
            self._refuse("lengths", f"contiguous int32 [{n}]", lengths)
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        lse = q.new_empty((n, heads), dtype=torch.float32) if return_lse else None
        try:
            args = _ATTEND.pack(
                q.data_ptr(), out.data_ptr(), _pointer(lse), table.data_ptr(), lengths.data_ptr(), self._status, q_row,
                q_head, table.stride(0), n, heads, _TYPES[dtype], cols,
                min(cols * self.page_size, _MOST) if max_length is None else max_length, window, 1 if add_weight else 0,
                1.0 / math.sqrt(self.head_dim) if scale is None else scale, first, 0)
        except _NO_FIT as e:
            raise ValueError(f"attend: {e}") from None
        self._call(_lib.fcsim_kv_attend, args, _lib.fcsim_kv_attend_workspace)
        return (out, lse) if return_lse else out

    def prefill(self, q, starts, table, lengths, *, max_length=None, scale=None, window=0, first=0, return_lse=False):
        """Attention of several tokens per request, such as those of a prompt or of a chunk of one: the rows ``starts[r]`` ..
        ``starts[r + 1] - 1`` (``starts``: int32 [requests + 1]) of ``q`` [n, heads, head_dim] are the newest of the ``lengths`` (int32)
        tokens of request r, which the rows of ``table`` (int32 [requests, pages]) hold already.  Each sees the tokens up to its own, with
        ``window`` > 0 only the newest so many of these and the ``first`` oldest.  Returns [n, heads, head_dim], with ``return_lse``
        also the float32 [n, heads] log-sum-exp; rows of no request are zeros.  The cache's weights, by which ``evict`` ranks, do not
        grow by it: only those tokens' shares count that ``attend`` adds."""
        if q.requires_grad and _grad_enabled():
            _refuse_gradient()
        dtype, shape, index = q.dtype, q.shape, self._index
        if dtype not in _WIDE or len(shape) != 3 or shape[2] != self.head_dim or q.get_device() != index:
            self._refuse("q", f"float16 or bfloat16 [tokens, heads, {self.head_dim}]", q)
        n, heads, _ = shape
        q_row, q_head, q_one = q.stride()
        if q_one != 1:
            raise ValueError("q: head_dim has to be contiguous")
        requests = lengths.numel()
        cols = self._table(table, "table", requests)
        if lengths.dtype != _I32 or lengths.get_device() != index or not lengths.is_contiguous():
            self._refuse("lengths", "contiguous int32 [requests]", lengths)
        if starts.dtype != _I32 or starts.numel() != requests + 1 or starts.get_device() != index or not starts.is_contiguous():
            self._refuse("starts", f"contiguous int32 [{requests + 1}]", starts)
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        lse = q.new_empty((n, heads), dtype=torch.float32) if return_lse else None
        try:
            args = _PREFILL.pack(
                q.data_ptr(), out.data_ptr(), _pointer(lse), starts.data_ptr(), table.data_ptr(), lengths.data_ptr(), self._status,
                q_row, q_head, table.stride(0), n, requests, heads, _TYPES[dtype], cols,
                min(cols * self.page_size, _MOST) if max_length is None else max_length, window, first,
                1.0 / math.sqrt(self.head_dim) if scale is None else scale, 0)
        except _NO_FIT as e:
            raise ValueError(f"prefill: {e}") from None
        self._call(_lib.fcsim_kv_prefill, args, _lib.fcsim_kv_prefill_workspace)
        return (out, lse) if return_lse else out

    def evict(self, table, lengths, budget, new_table, *, max_budget=None, recent=0, first=0, max_length=None):
        """Cut every request to its ``budget`` (int32 [requests]) of tokens per kv head: the ``recent`` newest, the
        ``first`` oldest and the largest weights, copied in order to the pages of ``new_table`` (none of which the
        call may read).  Returns the new lengths (int32 [requests]) and the old index of every kept token (int32
        [requests, n_kv_heads, max_budget], -1 beyond).  Weights are what ``attend`` has added: a prompt that ``prefill`` has loaded ranks
        by the tokens that followed it."""
        n, index = lengths.numel(), self._index
        cols, new_cols = self._table(table, "table", n), self._table(new_table, "new_table", n)
        if lengths.dtype != _I32 or lengths.get_device() != index or not lengths.is_contiguous():
            self._refuse("lengths", "contiguous int32", lengths)
        if budget.dtype != _I32 or budget.numel() != n or budget.get_device() != index or not budget.is_contiguous():
            self._refuse("budget", f"contiguous int32 [{n}]", budget)
        if max_budget is None:
            max_budget = min(new_cols * self.page_size, _MOST)
        if max_budget < 0:
            raise ValueError("max_budget: 0 or more")
        new_lengths = torch.empty_like(lengths)
        kept = lengths.new_empty((n, self.n_kv_heads, max_budget))
        try:
            args = _EVICT.pack(
                table.data_ptr(), lengths.data_ptr(), budget.data_ptr(), new_table.data_ptr(), new_lengths.data_ptr(),
                kept.data_ptr(), self._status, table.stride(0), new_table.stride(0), n, cols, new_cols,
                min(cols * self.page_size, _MOST) if max_length is None else max_length, max_budget, recent, first, 0)
        except _NO_FIT as e:
            raise ValueError(f"evict: {e}") from None
        self._call(_lib.fcsim_kv_evict, args, _lib.fcsim_kv_evict_workspace)
        return new_lengths, kept

    def read(self, slots, *, dtype=None):
        """What stands at ``slots`` (int64 [n], page * page_size + place, negative = zeros): k and v as [n, n_kv_heads, head_dim]
        of ``dtype`` (float16 or bfloat16; default: the cache's own, of an 8-bit cache bfloat16), 8-bit values times their scales (the float32 product, rounded)."""
        if dtype is None:
            dtype = torch.bfloat16 if self.k_scale is not None else self.k.dtype
        if dtype not in _WIDE:
            raise ValueError(f"dtype: float16 or bfloat16, got {dtype}")
        n = slots.numel()
        if slots.dtype != _I64 or slots.get_device() != self._index or not slots.is_contiguous():
            self._refuse("slots", "contiguous int64", slots)
        k = slots.new_empty((n, self.n_kv_heads, self.head_dim), dtype=dtype)
        v = torch.empty_like(k)
        try:
            args = _READ.pack(slots.data_ptr(), k.data_ptr(), v.data_ptr(), self._status, n, _TYPES[dtype])
        except _NO_FIT as e:
            raise ValueError(f"read: {e}") from None
        self._call(_lib.fcsim_kv_read, args)
        return k, v

    def check(self):
        """Wait for all calls, on every stream, read and clear the device status; raise when a call met a bad page, length, position
        or budget, or when a wait inside a kernel was given up, in a call of this cache or of another one on its device (all share the
        workspaces that it leaves wrong: each of them tells of it once)."""
        torch.cuda.synchronize(self.device)
        with _LOCK:
            words = torch.cat([word for _, word in _STATUS[self._index]]).tolist()
            if any(bits & STUCK for bits in words):
                _GIVEN_UP[self._index] += 1
                self._workspaces.clear()   # what has to be zero in them may not be
                for _, word in _STATUS[self._index]:
                    word.bitwise_and_(~STUCK)
            _STATUS[self._index] = [entry for entry in _STATUS[self._index] if entry[0]() is not None]
            told, self._given_up = self._given_up, _GIVEN_UP[self._index]
        bits = int(self.status.item())
        if bits:
            self.status.zero_()
        if told != self._given_up:
            raise RuntimeError("a wait inside a kernel was given up: results since the last check() are wrong (graphs captured before have to be "
                               "captured again)")
        if bits:
            names = [s for b, s in ((BAD_PAGE, "page or slot outside the pool"),
                                    (BAD_LENGTH, "length outside 0 .. max_length"),
                                    (BAD_POSITION, "position outside the rope table"),
                                    (BAD_BUDGET, "budget outside 0 .. max_budget")) if bits & b]
            raise ValueError("; ".join(names))
