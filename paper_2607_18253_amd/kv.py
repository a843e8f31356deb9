"""Python binding of the paged key/value cache (lar_kv_* in include/lar.h): a token batch's
K and V rows into and out of the pages, its attention over them, with trees of drafted tokens,
the weights that it gives to the rows, and which rows stay within a budget.  Argument marshalling
only, as in ``lar``; every step runs in the HIP kernels behind the C ABI.
"""

from __future__ import annotations

import ctypes as C
import math

import numpy as np

from .lar import LAR_E_STATE, LAR_OK, LarError, _dev, load_library

KV_F16, KV_BF16, KV_E4M3 = 0, 1, 2


def _raw_stream(index):
    """hipStream_t of the current stream of a device; from the first call on, torch's short way
    to it where it has one."""
    global _raw_stream
    import torch
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                          lambda i: torch.cuda.current_stream(i).cuda_stream)
    return _raw_stream(index)


def _int32s(x, name):
    """One-dimensional int32 array of integers, none of which is cut."""
    a = np.asarray(x)
    if a.ndim != 1 or (a.size and (a.dtype.kind not in "iu" or a.max() > 2 ** 31 - 1 or a.min() < -2 ** 31)):
        raise ValueError(f"{name} must be one-dimensional 32-bit integers")
    return np.ascontiguousarray(a, np.int32)


def _int32(x, name):
    """A number as an int that 32 bits hold, nothing cut off."""
    if not -2 ** 31 <= x < 2 ** 31 or int(x) != x:
        raise ValueError(f"{name} must be a 32-bit integer")
    return int(x)


def _on(index, t, dtype, name, numel=None):
    """_dev of a tensor on GPU `index`."""
    p = _dev(t, dtype, name, numel)
    if t is not None and t.get_device() != index:
        raise ValueError(f"{name} must be on cuda:{index}")
    return p


class KvConfig(C.Structure):
    _fields_ = [("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32), ("cache_dtype", C.c_int32), ("block_size", C.c_int32),
                ("max_seqs", C.c_int32), ("max_tokens", C.c_int32), ("reserved", C.c_int32),
                ("stream", C.c_void_p)]


class KvPagesArg(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_exp", C.c_void_p), ("v_exp", C.c_void_p),
                ("n_blocks", C.c_int64)]


class KvRowsArg(C.Structure):
    _fields_ = [("data", C.c_void_p), ("tok_stride", C.c_int64), ("head_stride", C.c_int64)]


class KvPages:
    """The pages of one layer: GPU tensors k and v [n_blocks][n_kv_heads][block_size][head_dim]
    (16-bit, or float8_e4m3fn with k_exp and v_exp uint8 [n_blocks][n_kv_heads][block_size]).
    Make new ones with PagedKV.new_pages.  Which tensors they are is fixed; where these are is
    looked up by every call."""

    __slots__ = ("_tensors", "_ptr", "_at", "_arg", "_ref", "_kind")
    k, v, k_exp, v_exp = (property(lambda self, i=i: self._tensors[i]) for i in range(4))

    def __init__(self, k, v, k_exp=None, v_exp=None):
        self._tensors = (k, v, k_exp, v_exp)
        self._look()

    def _look(self):
        """Checks the tensors and takes their places down."""
        import torch
        k, v, k_exp, v_exp = self._tensors
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype:
            raise ValueError("k and v must be [n_blocks][n_kv_heads][block_size][head_dim] of one dtype")
        e4m3 = k.dtype == torch.float8_e4m3fn
        for e in (k_exp, v_exp):
            if (e is not None) != e4m3 or (e4m3 and e.shape != k.shape[:3]):
                raise ValueError("float8_e4m3fn pages, and only they, have k_exp and v_exp "
                                 "[n_blocks][n_kv_heads][block_size]")
        index = k.get_device()
        self._arg = KvPagesArg(_on(index, k, k.dtype, "k"), _on(index, v, v.dtype, "v"),
                               _on(index, k_exp, torch.uint8, "k_exp"), _on(index, v_exp, torch.uint8, "v_exp"),
                               int(k.shape[0]))
        self._ref = C.byref(self._arg)
        self._kind = (k.dtype, *k.shape[1:], index)
        self._ptr = [None if t is None else t.data_ptr for t in self._tensors]
        self._at = [p and p() for p in self._ptr]

    def tensors(self):
        return [t for t in self._tensors if t is not None]


class PagedKV:
    """A paged key/value cache's geometry and the plan of the current token batch; see
    lar_kv_config and lar_kv_plan.  The pages of each layer are KvPages.

    Work runs on ``stream`` (the current one when the handle is made) and its device,
    whichever device is current when a call is made.  A call made while another stream is
    current is ordered after that stream's work, and that stream after the call; a graph is
    captured on the handle's own stream (which then is not the default one).  A captured
    call belongs to the plan it was captured with: replayed while a batch of other lengths is
    planned it does nothing, and ``sync`` raises.  There are no gradients: under autograd a
    tensor that requires one is refused."""

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, *, block_size: int,
                 dtype=None, cache_dtype=None, max_seqs: int, max_tokens: int, stream=None):
        import torch
        self._torch = torch
        self._L = load_library()
        self.stream = torch.cuda.current_stream() if stream is None else stream
        self._sid = self.stream.cuda_stream
        self.device = self.stream.device
        self.dtype = torch.bfloat16 if dtype is None else dtype
        self.cache_dtype = self.dtype if cache_dtype is None else cache_dtype
        kinds = {torch.float16: KV_F16, torch.bfloat16: KV_BF16, torch.float8_e4m3fn: KV_E4M3}
        if self.dtype not in kinds or self.cache_dtype not in kinds:
            raise ValueError("dtype must be float16 or bfloat16, cache_dtype dtype or float8_e4m3fn")
        self.n_q, self.n_kv = _int32(n_q_heads, "n_q_heads"), _int32(n_kv_heads, "n_kv_heads")
        self.head_dim, self.block_size = _int32(head_dim, "head_dim"), _int32(block_size, "block_size")
        cfg = KvConfig(self.n_q, self.n_kv, self.head_dim, kinds[self.dtype], kinds[self.cache_dtype],
                       self.block_size, _int32(max_seqs, "max_seqs"), _int32(max_tokens, "max_tokens"), 0,
                       C.c_void_p(self._sid))
        h = C.c_void_p()
        with torch.cuda.device(self.device):
            st = self._L.lar_kv_create(C.byref(h), C.byref(cfg))
        if st != LAR_OK:
            raise LarError(st, "lar_kv_create failed")
        self._h = h
        self._int32, self._index = torch.int32, self.device.index
        self._none = torch.empty(0, dtype=self.dtype, device=self.device)
        self._scale = 1.0 / math.sqrt(self.head_dim)
        self._batch(0, 0)
        self._kind = (self.cache_dtype, self.n_kv, self.block_size, self.head_dim, self._index)
        # the arguments of a call are read before it returns: one record each will do
        args = {n: KvRowsArg() for n in ("q", "k", "v")}
        self._args = {n: (a, C.byref(a)) for n, a in args.items()}

    # ------------------------------------------------------------------ plumbing
    def _check(self, st: int):
        if st != LAR_OK:
            raise LarError(st, self._L.lar_kv_error_string(self._h).decode())

    def close(self):
        if getattr(self, "_h", None):
            self._L.lar_kv_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _pages(self, pages):
        k, v, ke, ve = pages._ptr
        at = pages._at
        if k() != at[0] or v() != at[1] or (ke is not None and (ke() != at[2] or ve() != at[3])):
            pages._look()
        if pages._kind != self._kind:
            raise ValueError(f"pages must be [n_blocks][{self.n_kv}][{self.block_size}][{self.head_dim}] "
                             f"of {self.cache_dtype} on {self.device}")
        return pages._ref

    def _rows(self, t, shape, name):
        if t.dtype is not self.dtype or t.get_device() != self._index:
            raise ValueError(f"{name} must be a tensor of {self.dtype} on {self.device}")
        if t.requires_grad:
            self._no_gradient(name)
        if t.shape != shape:
            raise ValueError(f"{name} must be [{shape[0]}][{shape[1]}][{shape[2]}]")
        a, ref = self._args[name]
        a.tok_stride, a.head_stride, last = t.stride()
        if last != 1:
            raise ValueError(f"{name} must have contiguous rows")
        a.data = t.data_ptr()
        return ref

    def _no_gradient(self, name):
        if self._torch.is_grad_enabled():
            raise ValueError(f"{name} requires a gradient, and these calls have none: detach it, or use torch.no_grad()")

    def _table(self, table):
        shape = table.shape
        if len(shape) != 2 or shape[0] < self._n_seq:
            raise ValueError(f"table must have {self._n_seq} rows")
        if table.dtype is not self._int32 or table.get_device() != self._index or not table.is_contiguous():
            _on(self._index, table, self._int32, "table")
        return table.data_ptr(), shape[1]

    def _weights(self, t, name, n_blocks=None):
        p = _on(self._index, t, self._torch.float32, name)
        if t.dim() != 3 or t.shape[1:] != (self.n_kv, self.block_size) or n_blocks not in (None, t.shape[0]):
            n = "n_blocks" if n_blocks is None else n_blocks
            raise ValueError(f"{name} must be [{n}][{self.n_kv}][{self.block_size}]")
        if t.requires_grad:
            self._no_gradient(name)
        return p

    def _call(self, f, pages, tensors, *args):
        """f(handle, *args) in order with the current stream."""
        if _raw_stream(self._index) == self._sid:
            st = f(self._h, *args)
            if st != LAR_OK:
                self._check(st)
            return
        with self._torch.cuda.device(self.device):
            if self._torch.cuda.is_current_stream_capturing():
                raise ValueError("capture a graph on the handle's own stream")
            now = self._torch.cuda.current_stream()
        self.stream.wait_stream(now)
        try:
            self._check(f(self._h, *args))
        finally:
            for t in (*tensors, *(pages.tensors() if pages else ())):
                if t is not None:
                    t.record_stream(self.stream)
            now.wait_stream(self.stream)

    def _batch(self, n_seq, n_tok):
        self._n_seq, self._n_tok = n_seq, n_tok
        self._q_shape = (n_tok, self.n_q, self.head_dim)
        self._kv_shape = (n_tok, self.n_kv, self.head_dim)

    # ------------------------------------------------------------------ calls
    def new_pages(self, n_blocks: int) -> KvPages:
        """Pages of one layer, not initialised."""
        torch = self._torch
        shape = (int(n_blocks), self.n_kv, self.block_size, self.head_dim)
        kv = [torch.empty(shape, dtype=self.cache_dtype, device=self.device) for _ in range(2)]
        if self.cache_dtype == torch.float8_e4m3fn:
            kv += [torch.empty(shape[:3], dtype=torch.uint8, device=self.device) for _ in range(2)]
        return KvPages(*kv)

    def new_weights(self, n_blocks: int):
        """Weights of the rows of one layer's pages (weigh), all 0."""
        return self._torch.zeros((int(n_blocks), self.n_kv, self.block_size), dtype=self._torch.float32,
                                 device=self.device)

    def plan(self, q_len, ctx_len, window: int = 0, sinks: int = 0, parents=None):
        """The token batch of the calls that follow: new tokens per sequence and context
        with them (host integers).  parents, for sequences whose new tokens are a tree of drafted
        ones: of each new token of the batch the number of its parent among the sequence's new
        tokens, or -1 for the context."""
        q, c = _int32s(q_len, "q_len"), _int32s(ctx_len, "ctx_len")
        if q.shape != c.shape:
            raise ValueError("q_len and ctx_len must be of one length")
        _int32s([window, sinks], "window and sinks")
        if _raw_stream(self._index) != self._sid:   # else the library sees to it
            with self._torch.cuda.device(self.device):
                if self._torch.cuda.is_current_stream_capturing():
                    raise LarError(LAR_E_STATE, "no plan under stream capture")
        if parents is None:
            st = self._L.lar_kv_plan(self._h, len(q), q.ctypes.data, c.ctypes.data, int(window), int(sinks))
        else:
            up = _int32s(parents, "parents")
            if (q < 0).any() or len(up) != q.sum(dtype=np.int64):
                raise ValueError("parents must be one for each new token")
            st = self._L.lar_kv_plan_tree(self._h, len(q), q.ctypes.data, c.ctypes.data, up.ctypes.data,
                                          int(window), int(sinks))
        self._check(st)
        self._batch(len(q), int(q.sum()))

    def append(self, pages: KvPages, k, v, table):
        """The batch's K and V rows [T][n_kv][head_dim] into the pages."""
        t, cols = self._table(table)
        self._call(self._L.lar_kv_append, pages, (k, v, table), self._pages(pages),
                   self._rows(k, self._kv_shape, "k"), self._rows(v, self._kv_shape, "v"), t, cols)

    def read(self, pages: KvPages, table, k=None, v=None):
        """The rows of the batch's tokens back from the pages: (k, v), each
        [T][n_kv][head_dim] of dtype."""
        if k is None:
            k = self._none.new_empty(self._kv_shape)
        if v is None:
            v = self._none.new_empty(self._kv_shape)
        t, cols = self._table(table)
        self._call(self._L.lar_kv_read, pages, (k, v, table), self._pages(pages), t, cols,
                   self._rows(k, self._kv_shape, "k"), self._rows(v, self._kv_shape, "v"))
        return k, v

    def attend(self, pages: KvPages, q, table, scale=None, out=None, lse=None):
        """Attention of the batch's queries [T][n_q][head_dim] over the pages; scale
        defaults to head_dim ** -0.5.  Returns out [T][n_q][head_dim]; lse, when given, is
        a float32 tensor [T][n_q] that takes the log of each row's sum."""
        n = self._n_tok * self.n_q
        qa = self._rows(q, self._q_shape, "q")
        if out is None:
            out = self._none.new_empty(self._q_shape)
            to = out.data_ptr()
        else:
            to = _on(self._index, out, self.dtype, "out", n * self.head_dim)
            if out.requires_grad:
                self._no_gradient("out")
        t, cols = self._table(table)
        self._call(self._L.lar_kv_attend, pages, (q, out, lse, table), self._pages(pages), qa, t, cols,
                   self._scale if scale is None else float(scale), to,
                   None if lse is None else _on(self._index, lse, self._torch.float32, "lse", n))
        return out

    def weigh(self, pages: KvPages, q, lse, table, weights, before=None, scale=None):
        """Adds to the weights of the cache's rows what each gets of the attention of the batch's
        queries [T][n_q][head_dim], whose log-sums attend() gave as lse.  weights is a float32
        tensor [n_blocks][n_kv][block_size] (new_weights), updated in place, or made of `before`;
        the batch's new tokens start with 0."""
        pg, qa = self._pages(pages), self._rows(q, self._q_shape, "q")
        z = _on(self._index, lse, self._torch.float32, "lse", self._n_tok * self.n_q)
        if lse is not None and lse.requires_grad:
            self._no_gradient("lse")
        w = self._weights(weights, "weights", pages.k.shape[0])
        b = w if before is None else self._weights(before, "before", pages.k.shape[0])
        t, cols = self._table(table)
        self._call(self._L.lar_kv_weigh, pages, (q, lse, table, weights, before), pg, qa, t, cols,
                   self._scale if scale is None else float(scale), z, b, w)
        return weights

    def select(self, weights, table, budget: int, first: int = 0, last: int = 0, rows=None):
        """Which rows of each planned context stay within a budget: the first and last ones and
        those of the largest weights.  Returns rows, int32 [n_seqs][n_kv][budget], the positions
        in ascending order, then -1."""
        torch = self._torch
        budget, first, last = _int32(budget, "budget"), _int32(first, "first"), _int32(last, "last")
        w = self._weights(weights, "weights")
        shape = (self._n_seq, self.n_kv, budget)
        if budget < 1:
            raise ValueError("budget must be positive")
        if rows is None:
            rows = torch.empty(shape, dtype=torch.int32, device=self.device)
        elif rows.shape != shape:
            raise ValueError(f"rows must be [{shape[0]}][{shape[1]}][{shape[2]}]")
        to = _on(self._index, rows, torch.int32, "rows")
        t, cols = self._table(table)
        self._call(self._L.lar_kv_select, None, (weights, table, rows), w, weights.shape[0], t, cols, budget, first,
                   last, to)
        return rows

    def keep(self, pages: KvPages, table, rows, *, new: bool = False, to=None, weights=None):
        """Moves the rows that lists name, int32 [n_seqs][n_kv][n] or for all heads [n_seqs][n] (in
        ascending order, ended by -1), to the front of each planned context, with `new` to where
        its new tokens start, from which the lists count then: an accepted path of a tree.  Into
        the pages of the table `to`, if given.  weights go along."""
        pg = self._pages(pages)
        if rows.dim() not in (2, 3) or rows.shape[0] != self._n_seq or (rows.dim() == 3 and rows.shape[1] != self.n_kv):
            raise ValueError(f"rows must be [{self._n_seq}][{self.n_kv}][n] or [{self._n_seq}][n]")
        r = _on(self._index, rows, self._torch.int32, "rows")
        w = None if weights is None else self._weights(weights, "weights", pages.k.shape[0])
        t, cols = self._table(table)
        t2, cols2 = (None, 0) if to is None else self._table(to)
        self._call(self._L.lar_kv_keep, pages, (table, rows, to, weights), pg, t, cols, t2, cols2, r,
                   _int32(rows.shape[-1], "n"), int(rows.dim() == 3), int(bool(new)), w)

    def sync(self):
        """Synchronise; raises the sticky device error, if any."""
        self._check(self._L.lar_kv_sync(self._h))
