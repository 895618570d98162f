"""Device buffers of one paged cache and convenience wrappers over the binding.

Allocation and bookkeeping only (torch owns the memory); all work is done by libsparq.
"""
from __future__ import annotations

from contextlib import nullcontext
from typing import Optional, Union

import torch

from . import binding as B
from .cache import DecodeCache

PAGE_TYPES = {"16": B.SPARQ_PAGES_16, "i8": B.SPARQ_PAGES_I8, "e4m3": B.SPARQ_PAGES_E4M3}
CODE_TYPES = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}


def on_stream(stream):
    """What a call makes for itself belongs to its stream: torch fills it in order with the call's kernels."""
    return nullcontext() if stream is None else torch.cuda.stream(stream)


class PagedCache:
    """A pool of pages for K and V, a page table and lengths: K, V [n_pages, H_kv, page_size, d_h], page_table [B, max_pages],
    seq_lens [B] (int32, the caller's: which page a sequence gets and how long it is are decided by whoever schedules the batch).

    seq_lens counts the rows of the call that is made: raise it first, then append the new rows and attend with their queries.
    Rows are [B, heads, n, d_h] in any order with contiguous channels ([B, heads, d_h] for one row each), of which sequence b has
    n_new_per_seq[b] (all n without it); or packed [n_rows, heads, d_h] with row_start [B + 1] and n_new, the most rows of a sequence.
    """

    def __init__(self, Bsz: int, H: int, H_kv: int, d_h: int, page_size: int, n_pages: int, max_pages: int, dtype, pages: str = "16",
                 device="cuda", causal: bool = True, window: int = 0):
        if pages not in PAGE_TYPES:
            raise ValueError(f"pages must be one of {sorted(PAGE_TYPES)}, got {pages!r}")
        mk = lambda *size, dtype: torch.zeros(size, dtype=dtype, device=device)   # noqa: E731
        pool = CODE_TYPES.get(pages, dtype)
        scale = (lambda: mk(n_pages, H_kv, page_size, dtype=torch.float32)) if pages != "16" else (lambda: None)
        self._hold(mk(n_pages, H_kv, page_size, d_h, dtype=pool), mk(n_pages, H_kv, page_size, d_h, dtype=pool), mk(Bsz, max_pages, dtype=torch.int32),
                   mk(Bsz, dtype=torch.int32), H, dtype, scale(), scale(), causal, window)

    @classmethod
    def over(cls, K: torch.Tensor, V: torch.Tensor, page_table: torch.Tensor, seq_lens: torch.Tensor, H: int, dtype,
             K_scale: Optional[torch.Tensor] = None, V_scale: Optional[torch.Tensor] = None, causal: bool = True, window: int = 0) -> "PagedCache":
        """The same over buffers that exist already; the pools' dtype says what the pages hold."""
        c = cls.__new__(cls)
        c._hold(K, V, page_table, seq_lens, H, dtype, K_scale, V_scale, causal, window)
        return c

    def _hold(self, K, V, page_table, seq_lens, H, dtype, K_scale, V_scale, causal, window):
        kinds = {dtype: "16", torch.int8: "i8", torch.float8_e4m3fn: "e4m3"}
        if K.dim() != 4 or K.shape != V.shape or K.dtype != V.dtype or K.dtype not in kinds:
            raise ValueError("K and V must be pools [n_pages, H_kv, page_size, d_h] of the rows' dtype, int8 or float8_e4m3fn")
        n_pages, H_kv, page_size, d_h = K.shape
        Bsz, max_pages = page_table.shape
        if seq_lens.shape != (Bsz,):
            raise ValueError("seq_lens must be [B], page_table [B, max_pages]")
        self.pages = kinds[K.dtype]
        for name, s in (("K_scale", K_scale), ("V_scale", V_scale)):
            if self.pages != "16" and (s is None or s.shape != (n_pages, H_kv, page_size)):
                raise ValueError(f"{name} must be [n_pages, H_kv, page_size] for 8-bit pages")
        if self.pages == "16":
            K_scale = V_scale = None
        for t in (K, V, page_table, seq_lens, K_scale, V_scale):
            if t is not None and t.device != K.device:
                raise ValueError("all buffers of a cache must live on one device")
        self.K, self.V, self.K_scale, self.V_scale, self.page_table, self.seq_lens = K, V, K_scale, V_scale, page_table, seq_lens
        self.B, self.H, self.H_kv, self.d_h, self.page_size, self.n_pages, self.max_pages = Bsz, H, H_kv, d_h, page_size, n_pages, max_pages
        self.dtype, self.device, self._index = dtype, K.device, K.device.index
        self.cache = B.make_paged_cache(K, V, K_scale, V_scale, page_table, seq_lens)
        self.shape = B.make_paged_shape(Bsz, H, H_kv, d_h, page_size, n_pages, max_pages, dtype, PAGE_TYPES[self.pages],
                                        0 if causal else B.SPARQ_FLAG_PAGED_ALL, window)
        need = B.sparq_paged_workspace_bytes(self.shape, 1)
        self._rows_room, self._outgrown = 1, []
        with torch.cuda.device(self.device):
            self.workspace = self._new_workspace(need, None)

    def _new_workspace(self, need: int, stream) -> torch.Tensor:
        with on_stream(stream):
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("a cache's workspace cannot be made during a capture: make a call of this size before it")
            w = torch.empty((need,), dtype=torch.uint8, device=self.device)
            B.sparq_workspace_init(w, stream)
            return w

    def with_bound(self, S_bound: int) -> "PagedCache":
        """Promise that no sequence is longer than S_bound (0: what the page table has room for)."""
        self.shape.S_bound = S_bound
        self._rows_room = 0
        return self

    def with_lengths(self, seq_lens: torch.Tensor) -> "PagedCache":
        """The same pages with another tensor of lengths."""
        if seq_lens.shape != (self.B,) or seq_lens.device != self.device:
            raise ValueError(f"seq_lens must be [B] on {self.device}")
        if seq_lens is not self.seq_lens:
            self.seq_lens = seq_lens
            self.cache = B.make_paged_cache(self.K, self.V, self.K_scale, self.V_scale, self.page_table, seq_lens)
        return self

    # ---- the calls ----
    def _rows(self, t: torch.Tensor, heads: int, n_new, n_new_per_seq, row_start, stream) -> "B.SparqRows":
        """Checks the rows of a call; what says which they are; a workspace that is large enough."""
        if t.dtype is not self.dtype or t.device != self.device:
            raise ValueError(f"rows must be {self.dtype} on {self.device}, got {t.dtype} on {t.device}")
        size = t.shape
        if row_start is None:
            if len(size) != 4 or size[0] != self.B or size[1] != heads or size[3] != self.d_h:
                raise ValueError(f"rows must be [{self.B}, {heads}, n, {self.d_h}], got {tuple(size)}")
            n, n_rows = size[2], 0
            if n_new is not None and n_new != n:
                raise ValueError("n_new is the rows' third size where they are not packed")
        else:
            if len(size) != 3 or size[1] != heads or size[2] != self.d_h:
                raise ValueError(f"packed rows must be [n_rows, {heads}, {self.d_h}], got {tuple(size)}")
            if n_new is None:
                raise ValueError("packed rows need n_new, the most rows of a sequence")
            if row_start.shape != (self.B + 1,) or row_start.device != self.device:
                raise ValueError(f"row_start must be [B + 1] on {self.device}")
            n, n_rows = n_new, size[0]
        if n_new_per_seq is not None and (n_new_per_seq.shape != (self.B,) or n_new_per_seq.device != self.device):
            raise ValueError(f"n_new_per_seq must be [B] on {self.device}")
        if n > self._rows_room:
            self._grow(n, stream)
        return B.make_rows(n, n_new_per_seq, row_start, n_rows)

    def _grow(self, n: int, stream) -> None:
        """Room for calls of n rows per sequence.  The old workspace stays: calls in flight and captured ones go on using it."""
        need = B.sparq_paged_workspace_bytes(self.shape, n)
        if need > self.workspace.numel():
            w = self._new_workspace(need, stream)
            self._outgrown.append(self.workspace)
            self.workspace = w
        self._rows_room = n

    def _elsewhere(self, stream) -> bool:
        """Whether the current device is another one than the cache's (the calls go to the current one)."""
        if stream is not None and stream.device != self.device:
            raise ValueError(f"the stream must be one of {self.device}")
        return torch.cuda.current_device() != self._index

    def append(self, k_new: torch.Tensor, v_new: torch.Tensor, n_new_per_seq: Optional[torch.Tensor] = None,
               row_start: Optional[torch.Tensor] = None, n_new: Optional[int] = None, stream=None) -> None:
        """Write the rows at the last positions of every sequence (heads: H_kv)."""
        if self._elsewhere(stream):
            with torch.cuda.device(self.device):
                return self.append(k_new, v_new, n_new_per_seq, row_start, n_new, stream)
        if row_start is None and k_new.dim() == 3:
            k_new, v_new = k_new.unsqueeze(2), v_new.unsqueeze(2)
        rows = self._rows(k_new, self.H_kv, n_new, n_new_per_seq, row_start, stream)
        B.sparq_paged_append(self.shape, self.cache, rows, k_new, v_new, self.workspace, stream)

    def attend(self, q: torch.Tensor, n_new_per_seq: Optional[torch.Tensor] = None, row_start: Optional[torch.Tensor] = None,
               n_new: Optional[int] = None, out: Optional[torch.Tensor] = None, lse: Union[None, bool, torch.Tensor] = None, stream=None):
        """Attention of the last rows of every sequence (heads: H).  lse: True, or a float32 tensor for the logarithms of the
        denominators, [B, H, n] or packed [H, n_rows]; (out, lse) is returned if it is True."""
        if self._elsewhere(stream):
            with torch.cuda.device(self.device):
                return self.attend(q, n_new_per_seq, row_start, n_new, out, lse, stream)
        if out is None:          # rows that belong to no sequence are not written
            with on_stream(stream):
                out = torch.empty_like(q) if n_new_per_seq is None and row_start is None else torch.zeros_like(q)
        elif out.shape != q.shape or out.dtype is not q.dtype or out.device != q.device:
            raise ValueError("out must have q's shape, type and device")
        q4, o4 = (q.unsqueeze(2), out.unsqueeze(2)) if row_start is None and q.dim() == 3 else (q, out)
        rows = self._rows(q4, self.H, n_new, n_new_per_seq, row_start, stream)
        lse_out = None
        if lse is not None and lse is not False:
            size = (self.H, q.shape[0]) if row_start is not None else (self.B, self.H, q4.shape[2])
            with on_stream(stream):
                lse_out = torch.full(size, -float("inf"), dtype=torch.float32, device=self.device) if lse is True else lse
            if lse_out.shape != size or lse_out.device != self.device:
                raise ValueError(f"lse must be {size} on {self.device}")
        B.sparq_paged_attention(self.shape, self.cache, rows, q4, o4, lse_out, self.workspace, stream)
        return (out, lse_out) if lse is True else out

    def read(self, K_out: torch.Tensor, V_out: torch.Tensor, first: Optional[torch.Tensor] = None, n_per_seq: Optional[torch.Tensor] = None,
             row_start: Optional[torch.Tensor] = None, n_new: Optional[int] = None, stream=None):
        """Rows first[b] .. (0 .. without it) of every sequence as 16-bit rows, into K_out and V_out (heads: H_kv); they are returned."""
        if self._elsewhere(stream):
            with torch.cuda.device(self.device):
                return self.read(K_out, V_out, first, n_per_seq, row_start, n_new, stream)
        k, v = (K_out.unsqueeze(2), V_out.unsqueeze(2)) if row_start is None and K_out.dim() == 3 else (K_out, V_out)
        rows = self._rows(k, self.H_kv, n_new, n_per_seq, row_start, stream)
        if first is not None and (first.shape != (self.B,) or first.device != self.device):
            raise ValueError(f"first must be [B] on {self.device}")
        B.sparq_paged_read(self.shape, self.cache, rows, first, k, v, self.workspace, stream)
        return K_out, V_out

    def to_decode_cache(self, n: int, S_max: int, r: int, k: int, flags: int = 0) -> DecodeCache:
        """A SparQ cache with the rows of these pages (n: the most positions of a sequence): read back, then appended."""
        c = DecodeCache(self.B, self.H, self.H_kv, S_max, self.d_h, r, k, self.dtype, device=self.device, flags=flags)
        K, V = (torch.empty((self.B, self.H_kv, n, self.d_h), dtype=self.dtype, device=self.device) for _ in range(2))
        self.read(K, V, n_per_seq=self.seq_lens)
        c.append(K, V, self.seq_lens)
        return c

    def error_flags(self) -> int:
        """The SPARQ_ERR_* bits of the calls so far (waits for the current stream), which are cleared."""
        with torch.cuda.device(self.device):
            flags = 0
            for w in self._outgrown + [self.workspace]:
                flags |= B.sparq_async_error(w)
            return flags
