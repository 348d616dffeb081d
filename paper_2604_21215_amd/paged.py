"""Pages of a stack's key-value caches: the pools of all layers, one page table, and which pages are free.

A sequence has a place (a row of the table).  Pages are given out on the host, one number for the same page of every layer's pool; the
rows in them are written and read by the library's kernels only.  reserve and release copy the table to the device on torch's current
stream and return when it is there: that is the stream of the context that reads it, or one that the caller orders after the calls that
still read it (a step in flight may lose the pages that release takes from it).  The pools are whole when __init__ returns."""
from __future__ import annotations

import torch

from . import binding
from .torch_io import torch_dtype


class PagedCaches:
    """layers pools of `pages` pages of `page_len` positions, `places` sequences of at most `max_len` positions; bits 0 (storage dtype) or 8."""

    def __init__(self, layers: int, n_heads: int, places: int, max_len: int, pages: int, *, page_len: int = 64, bits: int = 0,
                 dtype: str = "bf16", device="cuda:0"):
        if bits not in (0, 8):
            raise ValueError("bits is 0 (the storage dtype) or 8")
        per = -(-max_len // page_len)
        self.page_len, self.max_len, self.bits, self.n_heads, self.dtype = page_len, max_len, bits, n_heads, dtype
        self.host_table = torch.full((places, per), -1, dtype=torch.int32)   # -1: no page
        self.table = self.host_table.to(device)
        self.free = list(range(pages - 1, -1, -1))
        self.held = [0] * places                                             # pages of each place
        shape = (pages, n_heads, page_len, 64)
        td = torch.int8 if bits else torch_dtype(dtype)
        self.K = [torch.zeros(shape, dtype=td, device=device) for _ in range(layers)]
        self.V = [torch.zeros(shape, dtype=td, device=device) for _ in range(layers)]
        self.K_exp = [torch.zeros(shape[:3], dtype=torch.uint8, device=device) if bits else None for _ in range(layers)]
        self.V_exp = [torch.zeros(shape[:3], dtype=torch.uint8, device=device) if bits else None for _ in range(layers)]
        self.layer = [binding.make_cache(self.K[l], self.V[l], self.table, self.K_exp[l], self.V_exp[l]) for l in range(layers)]
        if self.table.is_cuda:
            torch.cuda.current_stream(self.table.device).synchronize()   # the fills: any stream's context may use the pools from here on

    def reserve(self, lengths) -> None:
        """Pages for positions 0 .. lengths[s] - 1 of every place s (a length below what a place holds changes nothing; places past the
        last length keep what they hold).  Raises before anything is given out if there are not enough."""
        lengths = [int(n) for n in lengths]
        if len(lengths) > len(self.held):
            raise ValueError("%d lengths for %d places" % (len(lengths), len(self.held)))
        if any(n > self.max_len for n in lengths):
            raise ValueError("a sequence is longer than max_len")
        need = [max(0, -(-n // self.page_len) - self.held[s]) for s, n in enumerate(lengths)]
        if sum(need) > len(self.free):
            raise MemoryError("%d pages are wanted and %d are free" % (sum(need), len(self.free)))
        if not any(need):
            return
        for s, n in enumerate(need):
            for _ in range(n):
                self.host_table[s, self.held[s]] = self.free.pop()
                self.held[s] += 1
        self.table.copy_(self.host_table)

    def release(self, place: int) -> None:
        """The pages of a place are free again; its line of the table names none."""
        if not 0 <= place < len(self.held):
            raise ValueError("place %d of %d" % (place, len(self.held)))
        self.free.extend(int(p) for p in self.host_table[place, :self.held[place]])
        self.host_table[place] = -1
        self.held[place] = 0
        self.table.copy_(self.host_table)
