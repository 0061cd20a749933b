"""One layer's paged key/value cache as a serving program holds it: the pool, page tables of the running sequences, and the
calls on it (binding.tkphi_kv_append, tkphi_paged_attention, tkphi_block_attention; with normed heads tkphi_norm_append; over a cache in 8 bits
tkphi_quant_append and so on).  Bookkeeping only: which page is whose is decided here, on the host; all arithmetic is in the library's kernels."""
from __future__ import annotations

import torch

from . import binding as B


class PagedCache:
    """heads_first: pages are [KV head][token][channel] in memory, else [token][KV head][channel].  block: tokens per block whose
    mean keys are kept (0: none, no attend_blocks).  max_rows, max_len: bounds of one step that the workspace is sized for.
    codes: the cache holds e4m3 codes and scales (bf16 rows only).  norms: (weights of q, of k, eps[, offset]) as for binding.make_head_norms: query and key
    heads are normed before they are rotated."""

    def __init__(self, n_q_heads, n_kv_heads, d_head, n_pages, page_tokens, max_seqs, max_rows, max_len, dtype="bf16", heads_first=True,
                 score_scale=None, window=0, rot_dim=None, rot_adjacent=False, rot_base=500000.0, block=0, first_blocks=0, last_blocks=0,
                 top_blocks=0, device="cuda", codes=False, norms=None):
        t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
        self.dtype, self.codes, mean_type = t, codes, t
        if codes:
            if dtype != "bf16":
                raise ValueError("a cache in 8 bits takes bf16 rows")
            t = torch.uint8
        shape = (n_pages, n_kv_heads, page_tokens, d_head) if heads_first else (n_pages, page_tokens, n_kv_heads, d_head)
        self.K, self.V = (torch.zeros(shape, dtype=t, device=device) for _ in range(2))
        if codes:
            self.K, self.V = self.K.view(torch.float8_e4m3fn), self.V.view(torch.float8_e4m3fn)
            self.scales = torch.full((n_pages, n_kv_heads, page_tokens, 2), 127, dtype=torch.uint8, device=device)
        if not heads_first:
            self.K, self.V = self.K.transpose(1, 2), self.V.transpose(1, 2)
        self.M = torch.zeros(n_pages, n_kv_heads, page_tokens // block, d_head, dtype=mean_type, device=device) if block else None
        rot_dim = d_head if rot_dim is None else rot_dim
        self.inv_freq = rot_base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device) / max(rot_dim, 1))
        scale = d_head ** -0.5 if score_scale is None else score_scale
        cfg = dict(rot_dim=rot_dim, rot_adjacent=rot_adjacent, block=block, first_blocks=first_blocks, last_blocks=last_blocks, top_blocks=top_blocks)
        self.cfg = B.make_paged_config(n_q_heads, n_kv_heads, d_head, dtype, scale, self.K, self.V, window=window, **cfg)
        self.block_cfg = B.make_paged_config(n_q_heads, n_kv_heads, d_head, dtype, scale, self.K, self.V, **cfg) if window else self.cfg
        self.pool = B.make_quant_pool(self.K, self.V, self.scales, self.M) if codes else B.make_pool(self.K, self.V, self.M)
        self.norm_weights = None if norms is None else tuple(norms[:2])      # (the struct holds their addresses)
        self.norms = None if norms is None else B.make_head_norms(*norms)
        self.page_tokens, self.device = page_tokens, device
        self.free = list(range(n_pages - 1, -1, -1))
        self.pages: dict = {}                  # sequence -> its page ids
        self.length: dict = {}                 # sequence -> tokens in the cache
        self._new: dict = {}                   # sequence -> new tokens of the step that has begun
        bound = B.tkphi_step(0, 0, max_seqs, 1, max_rows, max_rows, max_len, 0)
        self.bounds = (max_seqs, max_rows, max_len)
        self.ws_bytes = max(B.tkphi_paged_workspace_bytes(c, bound) for c in (self.cfg, self.block_cfg))
        if self.ws_bytes == 0:
            raise B.TkphiError(B.TKPHI_ESHAPE, B.tkphi_last_error())
        self.ws = B.alloc_paged_workspace(self.ws_bytes, device)

    def begin_step(self, new_tokens: dict) -> B.tkphi_step:
        """new_tokens: {sequence: number of new tokens}, in the order of their rows.  Takes the pages they need from the pool."""
        seqs, row = [], 0
        need = {s: -(-(self.length.get(s, 0) + m) // self.page_tokens) for s, m in new_tokens.items()}
        lengths = [self.length.get(s, 0) + m for s, m in new_tokens.items()]
        if min(new_tokens.values(), default=0) < 0:
            raise ValueError(f"negative numbers of new tokens: {new_tokens}")
        if len(new_tokens) > self.bounds[0] or sum(new_tokens.values()) > self.bounds[1] or max(lengths, default=0) > self.bounds[2]:
            raise ValueError(f"step beyond the bounds {self.bounds}")
        if sum(max(0, n - len(self.pages.get(s, ()))) for s, n in need.items()) > len(self.free):
            raise MemoryError("no free pages")
        for s, m in new_tokens.items():
            pages = self.pages.setdefault(s, [])
            while len(pages) < need[s]:
                pages.append(self.free.pop())
            seqs.append([self.length.get(s, 0), m, row, 0])
            row += m
        width = max([len(self.pages[s]) for s in new_tokens] + [1])
        table = [self.pages[s] + [-1] * (width - len(self.pages[s])) for s in new_tokens]
        # (the caller's program would keep these on the device and update them there)
        self._seqs = torch.tensor(seqs, dtype=torch.int32).reshape(-1, 4).to(self.device)
        self._table = torch.tensor(table, dtype=torch.int32).reshape(-1, width).to(self.device)
        self._new = dict(new_tokens)
        self._tables_on = B.current_stream_ptr() if self._seqs.is_cuda else 0
        self.step = B.make_step(self._seqs, self._table, row, max(new_tokens.values(), default=0), max(lengths, default=0))
        return self.step

    def _stream(self) -> int:
        """The current stream's handle.  The step's tables, which the next step replaces, keep their memory until the work on it is done, also where
        begin_step ran on another stream."""
        stream = B.current_stream_ptr()
        if stream != self._tables_on:
            for t in (self._seqs, self._table):
                t.record_stream(torch.cuda.current_stream())
        return stream

    def append(self, q, k, v, q_rot) -> None:
        """Rotates q into q_rot and k into the pages, copies v: rows of the step's new tokens, [rows][heads][channels]."""
        io, tail = B.make_new_rows(q, k, v, q_rot, inv_freq=self.inv_freq), (self.ws.data_ptr(), self.ws_bytes, self._stream())
        if self.codes:
            B.tkphi_quant_append(self.cfg, self.step, self.pool, io, self.norms, *tail)
        elif self.norms is not None:
            B.tkphi_norm_append(self.cfg, self.step, self.pool, io, self.norms, *tail)
        else:
            B.tkphi_kv_append(self.cfg, self.step, self.pool, io, *tail)

    def attend(self, q_rot, out, lse=None) -> None:
        call = B.tkphi_quant_attention if self.codes else B.tkphi_paged_attention
        call(self.cfg, self.step, self.pool, B.make_attention_rows(q_rot, out, lse), self.ws.data_ptr(), self.ws_bytes, self._stream())

    def attend_blocks(self, q_rot, out) -> None:
        call = B.tkphi_quant_block_attention if self.codes else B.tkphi_block_attention
        call(self.block_cfg, self.step, self.pool, B.make_attention_rows(q_rot, out), self.ws.data_ptr(), self.ws_bytes, self._stream())

    def read(self, seq, k, v) -> None:
        """The sequence's cached keys and values (of a cache in 8 bits) to the first rows of k and v, [rows][KV heads][channels] in any layout; either may
        be None.  What the calls on contiguous caches read is [KV heads][rows][channels], transposed.  In calls of at most max_rows rows."""
        if not self.codes:
            raise ValueError("a cache of codes is read back; others hold the rows themselves")
        length = self.length.get(seq, 0)
        for name, x in (("k", k), ("v", v)):
            if x is not None and x.shape[0] < length:
                raise ValueError(f"{name}: {x.shape[0]} rows for a sequence of {length}")
        pages = torch.tensor([self.pages.get(seq, []) or [-1]], dtype=torch.int32).to(self.device)
        for start in range(0, length, self.bounds[1]):
            n = min(self.bounds[1], length - start)
            seqs = torch.tensor([[start, n, 0, 0]], dtype=torch.int32).to(self.device)
            io = B.make_read_rows(*(None if x is None else x[start:start + n] for x in (k, v)))
            B.tkphi_quant_read(self.cfg, B.make_step(seqs, pages, n, n, start + n), self.pool, io, self.ws.data_ptr(), self.ws_bytes, B.current_stream_ptr())

    def end_step(self) -> None:
        """The step's tokens are in the cache (once; sequences released since begin_step stay away)."""
        for s, m in self._new.items():
            self.length[s] = self.length.get(s, 0) + m
        self._new = {}

    def release(self, seq) -> None:
        """Gives the sequence's pages back, within a step too."""
        self.free += reversed(self.pages.pop(seq, []))
        self.length.pop(seq, None)
        self._new.pop(seq, None)

    def status(self) -> int:
        return B.tkphi_read_device_status(self.ws.data_ptr(), B.current_stream_ptr())
