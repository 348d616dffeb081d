"""A stack of RT layers on the device: embedding -> L x rt_layer_prefill -> final norm + output projection,
and the same per decoding step over the per-layer caches (Sec. 2: the layers of one model are stacked,
each with its own key-value memory; Sec. 7.3: decoding).  Sequencing and pointer marshalling only: every
arithmetic step is a call into the C library.

Everything that a call enqueues, torch's fills and copies included, goes to the stream of the context, whatever torch's current stream
is: the caller orders that stream after the work that makes a call's inputs, and before its own work on what a call returns."""
from __future__ import annotations

from contextlib import contextmanager

import torch

from . import binding
from .paged import PagedCaches
from .torch_io import DeviceLayer, to_device, torch_dtype


class DeviceStack:
    def __init__(self, ctx: binding.RTContext, layers: list[DeviceLayer], embedding, lm_head, g_final, dtype: str,
                 device="cuda:0"):
        self.ctx, self.layers, self.dtype, self.device = ctx, layers, dtype, device
        self.embedding = to_device(embedding, dtype, device)
        self.lm_head = to_device(lm_head, dtype, device)
        self.g_final = None if g_final is None else to_device(g_final, dtype, device)
        self.vocab, self.d = self.embedding.shape
        self.H = ctx.cfg.n_heads
        self.K = self.V = self.y = None
        self.head4 = None

    @contextmanager
    def _on_context_stream(self, *given: torch.Tensor):
        """Torch allocates, fills and copies on the context's stream inside.  Yields what is called on each tensor that is handed out: its
        memory, like that of the tensors given, is not used again before the other stream is done with it."""
        device = self.embedding.device
        if device.type == "cpu":
            yield lambda t: t
            return
        here, address = torch.cuda.current_stream(device), self.ctx.cfg.stream or 0
        if here.cuda_stream == address:
            yield lambda t: t
            return
        stream = torch.cuda.ExternalStream(address, device) if address else torch.cuda.default_stream(device)
        for t in given:
            t.record_stream(stream)

        def out(t):
            t.record_stream(here)
            return t
        with torch.cuda.stream(stream):
            yield out

    def prefill(self, ids: torch.Tensor, N: int, kv_cap: int, keep_outputs: bool = True, wavefront: bool = False,
                chunk: int = 0):
        """ids [B, >= N] int32 on the device.  Runs positions 0..N-1 through every layer; returns the
        logits [B, vocab] (fp32) of position N-1.  Layer outputs stay in self.y[l] ([B, N, d]) and the
        caches in self.K[l], self.V[l] ([kv_cap, B, H, 64]).  wavefront: one rt_stack_prefill call (layers
        run concurrently, `chunk` positions apart) instead of one rt_layer_prefill per layer."""
        with self._on_context_stream(ids) as out:
            B = ids.shape[0]
            td = torch_dtype(self.dtype)
            x = torch.empty((B, N, self.d), dtype=td, device=self.device)
            self.ctx.rt_embed_rows(self.embedding, ids, 0, x)
            self.x0 = x
            self.K, self.V, self.y = [], [], []
            if wavefront:
                for _ in self.layers:
                    self.y.append(torch.empty_like(x))
                    self.K.append(torch.zeros((kv_cap, B, self.H, self.d // self.H), dtype=td, device=self.device))
                    self.V.append(torch.zeros_like(self.K[-1]))
                self.ctx.rt_stack_prefill([lay.struct for lay in self.layers], x, self.y, self.K, self.V, chunk)
                x = self.y[-1]
            else:
                for lay in self.layers:
                    y = torch.empty_like(x)
                    K = torch.zeros((kv_cap, B, self.H, self.d // self.H), dtype=td, device=self.device)
                    V = torch.zeros_like(K)
                    self.ctx.rt_layer_prefill(lay.struct, x, y, K, V)
                    self.K.append(K); self.V.append(V)
                    if keep_outputs:
                        self.y.append(y)
                    x = y
            self.last = x
            logits = torch.empty((B, self.vocab), dtype=torch.float32, device=self.device)
            self.ctx.rt_lm_head(self.lm_head, self.g_final, x[:, N - 1], x.stride(0), B, logits)
            return out(logits)

    def decode_step(self, ids: torch.Tensor, t: int):
        """One position t (0-based) for all sequences: ids[:, t] is the input token.  Returns
        (logits [B, vocab] fp32, per-layer outputs [L, B, d])."""
        with self._on_context_stream(ids) as out:
            B = ids.shape[0]
            td = torch_dtype(self.dtype)
            L = len(self.layers)
            rows = torch.empty((L + 1, B, 1, self.d), dtype=td, device=self.device)
            self.ctx.rt_embed_rows(self.embedding, ids, t, rows[0])
            for l, lay in enumerate(self.layers):
                self.ctx.rt_decode_step(lay.struct, rows[l, :, 0], t, rows[l + 1, :, 0], self.K[l], self.V[l])
            logits = torch.empty((B, self.vocab), dtype=torch.float32, device=self.device)
            self.ctx.rt_lm_head(self.lm_head, self.g_final, rows[L], self.d, B, logits)
            return out(logits), out(rows)[1:, :, 0]

    def pack_lm_head(self):
        """The output projection in 4 bits beside the stored one (rt_mx4_pack on the host); decode_step_paged(head4=True) reads it."""
        w = self.lm_head.view(torch.int16).cpu().numpy().view("uint16") if self.dtype == "bf16" else self.lm_head.cpu().numpy()
        self.head4 = tuple(torch.from_numpy(a).to(self.device) for a in binding.rt_mx4_pack(w))

    def _check_caches(self, caches: PagedCaches, S: int):
        if len(caches.layer) != len(self.layers) or S > len(caches.held):
            raise ValueError("caches of %d layers and at least %d places are required" % (len(self.layers), S))
        # the kernels address the pools by the stack's heads and type
        if caches.n_heads != self.H or (not caches.bits and torch_dtype(caches.dtype) != torch_dtype(self.dtype)) \
                or caches.table.device != self.embedding.device:
            raise ValueError("the caches hold %d heads in %s on %s, the stack has %d in %s on %s" % (
                caches.n_heads, "8 bits" if caches.bits else caches.dtype, caches.table.device, self.H, self.dtype, self.embedding.device))

    def into_pages(self, caches: PagedCaches, lens):
        """The pairs that the last prefill (and the decode_steps behind it) left in self.K, self.V, rows 0 .. lens[b] - 1 of sequence b, into
        the pages of place b (which are reserved here, with room for the next token where max_len has it).  One length for each sequence of the prefill;
        lens[b] < 0: nothing of sequence b."""
        lens = [int(n) for n in lens]
        if self.K is None or len(lens) != self.K[0].shape[1] or max(lens) > self.K[0].shape[0]:
            raise ValueError("one length, of at most kv_cap, for each sequence of a prefill")
        self._check_caches(caches, len(lens))
        with self._on_context_stream():
            caches.reserve([max(n, min(n + 1, caches.max_len)) if n >= 0 else 0 for n in lens])
            count = torch.tensor([max(n, 0) for n in lens], dtype=torch.int32, device=self.device)
            first = torch.tensor([0 if n >= 0 else -1 for n in lens], dtype=torch.int32, device=self.device)
            N = max(max(lens), 1)
            for l in range(len(self.layers)):
                self.ctx.rt_cache_write(caches.layer[l], first, count, self.K[l][:N].transpose(0, 1), self.V[l][:N].transpose(0, 1))

    def decode_step_paged(self, caches: PagedCaches, ids: torch.Tensor, pos: torch.Tensor, max_pos: int, head4: bool = False):
        """One token of every sequence: ids [S] int32 on the device, sequence s at its own position pos[s] (int32 on the device, at most
        max_pos; negative: an idle place, whose rows hold nothing).  The pages have been reserved for pos[s] + 1 positions.  Returns (logits
        [S, vocab] fp32, per-layer outputs [L, S, d]); head4: the read-out with the 4-bit weights of pack_lm_head."""
        S, L = ids.shape[0], len(self.layers)
        for t in (ids, pos):   # the kernels follow their addresses
            if t.dtype != torch.int32 or t.shape != (S,) or not t.is_contiguous() or t.device != self.embedding.device:
                raise ValueError("ids and pos are contiguous int32 [S] on the stack's device")
        if head4 and self.head4 is None:
            raise ValueError("pack_lm_head comes first")
        self._check_caches(caches, S)
        with self._on_context_stream(ids, pos) as out:
            rows = torch.zeros((L + 1, S, 1, self.d), dtype=torch_dtype(self.dtype), device=self.device)
            self.ctx.rt_embed_rows(self.embedding, ids.view(S, 1), 0, rows[0])
            for l, lay in enumerate(self.layers):
                self.ctx.rt_decode_step_paged(lay.struct, caches.layer[l], rows[l, :, 0], pos, max_pos, rows[l + 1, :, 0])
            logits = torch.empty((S, self.vocab), dtype=torch.float32, device=self.device)
            if head4:
                self.ctx.rt_lm_head_mx4(self.head4[0], self.head4[1], self.g_final, rows[L], self.d, S, logits)
            else:
                self.ctx.rt_lm_head(self.lm_head, self.g_final, rows[L], self.d, S, logits)
            return out(logits), out(rows)[1:, :, 0]
