"""The cache in pages: ctypes binding of the rkv_paged_* calls.  Argument marshalling only."""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass, replace

from .binding import _check, _CPagedBatch, _CPagedConfig, _dev, _device, _stream, load_library


def _int32(**values):
    """Whole numbers that the library's 32-bit fields hold (ctypes would cut others off)."""
    for name, x in values.items():
        if not isinstance(x, int) or not -(2**31) <= x < 2**31:
            raise ValueError(f"{name} must be an int of 32 bits, not {x!r}")


@dataclass
class RkvPagedConfig:
    """rkv_paged_config: bits 16, 8 (E4M3 codes) or 4 (E2M1 codes); dtype 0 fp16, 1 bf16."""
    n_q_heads: int
    n_kv_heads: int
    n_pages: int
    head_dim: int = 128
    page_tokens: int = 64
    bits: int = 8
    dtype: int = 0

    def to_c(self) -> _CPagedConfig:
        _int32(**vars(self))
        return _CPagedConfig(self.n_q_heads, self.n_kv_heads, self.head_dim, self.page_tokens, self.n_pages, self.bits, self.dtype)


def paged_sizes(cfg: RkvPagedConfig) -> int:
    """rkv_paged_sizes: bytes of the pool."""
    n, cc = C.c_size_t(0), cfg.to_c()
    _check(load_library().rkv_paged_sizes(C.byref(cc), C.byref(n)), "rkv_paged_sizes")
    return n.value


class RkvPagedBatch:
    """rkv_paged_batch: the sequences of a call and their new rows.

    page_table [n_seqs, max_pages], row_start [n_seqs + 1] and lengths [n_seqs] are int32 tensors on the device, read by every
    call anew (and by every replay of a captured one); n_rows, max_new and max_len are the host's bounds on them (n_rows
    and the tables' capacity where not given: close bounds choose the better launch, max_new = 1 for single tokens).  The object is fixed: a batch of other bounds or tensors is another object."""

    __slots__ = ("page_table", "row_start", "lengths", "device", "n_rows", "_c", "_defaults")

    def __init__(self, page_table, row_start, lengths, n_rows: int, max_new: int = None, max_len: int = None):
        import torch
        if page_table is None or row_start is None or lengths is None:
            raise TypeError("page_table, row_start and lengths are needed")
        page_table, row_start = _dev(page_table, torch.int32, "page_table"), _dev(row_start, torch.int32, "row_start")
        lengths = _dev(lengths, torch.int32, "lengths")
        if page_table.dim() != 2 or row_start.shape != (page_table.shape[0] + 1,) or lengths.shape != page_table.shape[:1]:
            raise ValueError("page_table must be [n_seqs, max_pages], row_start [n_seqs + 1], lengths [n_seqs]")
        if row_start.device != page_table.device or lengths.device != page_table.device:
            raise ValueError("page_table, row_start and lengths must be on one device")
        self.page_table, self.row_start, self.lengths = page_table, row_start, lengths
        self.device, self.n_rows = page_table.device, n_rows
        n_seqs, max_pages = page_table.shape
        max_new = n_rows if max_new is None else max_new
        _int32(n_rows=n_rows, max_new=max_new, max_len=0 if max_len is None else max_len, n_seqs=n_seqs, max_pages=max_pages)
        self._defaults = max_len is None
        self._c = _CPagedBatch(page_table.data_ptr(), row_start.data_ptr(), lengths.data_ptr(), n_seqs, max_pages, n_rows, max_new, max_len or 0)

    def to_c(self, cfg: RkvPagedConfig) -> _CPagedBatch:
        """The C structure, for a cache of this configuration."""
        c = self._c
        if not self._defaults:
            return c
        return _CPagedBatch(c.dev_page_table, c.dev_row_start, c.dev_lengths, c.n_seqs, c.max_pages, c.n_rows, c.max_new,
                            min(c.max_pages * cfg.page_tokens, 1 << 30))


class RkvPagedCache:
    """One layer's pool of pages.  The page tables and lengths are the caller's (RkvPagedBatch); `mem` is memory of the
    caller's for the pool, as it is (uint8, paged_sizes bytes), or None for a cleared pool of its own."""

    def __init__(self, cfg: RkvPagedConfig, device="cuda:0", mem=None):
        import torch
        self.cfg, self.lib = replace(cfg), load_library()
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        n = paged_sizes(cfg)
        if mem is None:
            mem = torch.zeros(n, dtype=torch.uint8, device=self.device)
        self.mem = _dev(mem, torch.uint8, "mem")
        if mem.device != self.device or mem.numel() < n:
            raise ValueError(f"mem must hold {n} bytes on {self.device}")
        self.dtype = torch.bfloat16 if cfg.dtype else torch.float16
        self._c = cfg.to_c()
        # (what every call needs again; a call's own time is a few microseconds)
        self._at, self._mem_at = C.byref(self._c), mem.data_ptr()
        self._torch, self._index = torch, self.device.index

    def _rows(self, t, heads: int, n_rows: int, what: str):
        """Pointer and row stride of a tensor [n_rows, heads, head_dim] whose heads are dense."""
        D = self.cfg.head_dim
        if not isinstance(t, self._torch.Tensor) or t.dtype is not self.dtype or t.device != self.device:
            raise TypeError(f"{what} must be a tensor of dtype {self.dtype} on {self.device}")
        if t.shape != (n_rows, heads, D):
            raise ValueError(f"{what} must be [{n_rows}, {heads}, {D}]")
        s = t.stride()
        if s[2] != 1 or (s[1] != D and heads > 1):
            raise ValueError(f"{what} must have its heads side by side")
        return t.data_ptr(), s[0] if n_rows > 1 else heads * D

    def _call(self, function, name, *args):
        """One call of the library with the cache's device current."""
        if _device() == self._index:
            rc = function(self._at, self._mem_at, *args, _stream())
        else:
            with self._torch.cuda.device(self.device):
                rc = function(self._at, self._mem_at, *args, _stream())
        if rc:
            _check(rc, name)

    def _batch(self, batch):
        if batch.device != self.device:
            raise ValueError(f"the batch must be on {self.device}")
        return C.byref(batch.to_c(self.cfg))

    def append(self, k, v, batch: RkvPagedBatch):
        """rkv_paged_append: k, v [n_rows, n_kv_heads, head_dim] of the cache's type (rows may be strided)."""
        h, n = self.cfg.n_kv_heads, batch.n_rows
        kp, ks = self._rows(k, h, n, "k")
        vp, vs = self._rows(v, h, n, "v")
        self._call(self.lib.rkv_paged_append, "rkv_paged_append", self._batch(batch), kp, ks, vp, vs)

    def read(self, batch: RkvPagedBatch, k=None, v=None):
        """rkv_paged_read: the rows' keys and values as the cache holds them, into k and v where given."""
        empty, n, h, D = self._torch.empty, batch.n_rows, self.cfg.n_kv_heads, self.cfg.head_dim
        k = empty((n, h, D), dtype=self.dtype, device=self.device) if k is None else k
        v = empty((n, h, D), dtype=self.dtype, device=self.device) if v is None else v
        kp, ks = self._rows(k, h, n, "k")
        vp, vs = self._rows(v, h, n, "v")
        self._call(self.lib.rkv_paged_read, "rkv_paged_read", self._batch(batch), kp, ks, vp, vs)
        return k, v

    def attention(self, q, batch: RkvPagedBatch, causal: bool = True, window: int = 0, scale: float = None, out=None, lse=None,
                  want_lse: bool = False):
        """rkv_paged_attention: q [n_rows, n_q_heads, head_dim] -> out of the same shape and type (and lse [n_rows, n_q_heads]
        fp32).  Work space is allocated for each call on its stream, so that calls may overlap."""
        torch, cfg, n, dev = self._torch, self.cfg, batch.n_rows, self.device
        qp, qs = self._rows(q, cfg.n_q_heads, n, "q")
        if out is None:
            out = torch.empty((n, cfg.n_q_heads, cfg.head_dim), dtype=self.dtype, device=dev)
        elif _dev(out, self.dtype, "out").shape != q.shape or out.device != dev:
            raise ValueError("out must be a tensor like q")
        if lse is None:
            lse = torch.empty((n, cfg.n_q_heads), dtype=torch.float32, device=dev) if want_lse else None
        elif _dev(lse, torch.float32, "lse").shape != (n, cfg.n_q_heads) or lse.device != dev:
            raise ValueError("lse must be [n_rows, n_q_heads]")
        if not 0 <= window < 2**31:
            raise ValueError("window must be an int of 32 bits, 0 for none")
        cb, need = self._batch(batch), C.c_size_t()
        rc = self.lib.rkv_paged_scratch(self._at, cb, C.byref(need))
        if rc:
            _check(rc, "rkv_paged_scratch")
        need = need.value
        scratch = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
        self._call(self.lib.rkv_paged_attention, "rkv_paged_attention", cb, qp, qs, 1 if causal else 0, window,
                   cfg.head_dim ** -0.5 if scale is None else scale, out.data_ptr(), None if lse is None else lse.data_ptr(),
                   scratch.data_ptr() if need else None, need)
        return (out, lse) if want_lse else out
