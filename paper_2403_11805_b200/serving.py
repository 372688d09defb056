"""Serving the resident contexts of a MultiApp between Load and Reclaim (Sec. 3.1: inference runs on the resident chunks).

A Serving is a batch of contexts whose working sets are locked in the pool: their chunk table and lengths on the device, an
accumulator of attention weights per layer, KV head and token, and the calls that a decoding step makes.  A model
calls `decode` once per layer with the step's query, key and value rows; `shrink` drops the tokens that attention weighed
least and gives the slots they no longer need back to the pool.  The accumulator belongs to the batch: it starts at zero, so
`shrink` ranks by what the `decode` calls of this step have added (of tokens with equal weight the first stay).

Lengths follow rules that the host knows as well (one more token a step, min(budget, length) after a shrink), so no length is
read back from the device.  `decode` and an `advance` within the last chunk wait for nothing; growth into a new chunk and
`shrink` copy the changed table from pageable memory, which waits for the stream.

The calls run on the pool's stream, in order with its Reclaim and Load.  Made on another stream they come after what was queued
there, and what is queued there next comes after them.  Only a `decode` that is being captured into a graph stays on the
capturing stream; its replays are ordered by the stream that they, `advance` and `shrink` are called on.
"""
import contextlib

import numpy as np
import torch

from . import binding as B


class Serving:
    def __init__(self, app, ctxs):
        self.app, self.ctxs = app, list(ctxs)
        sh = app.shape
        n, self.capacity = len(self.ctxs), app.cpc * sh.chunk_len
        self._main = app.main.cuda_stream
        self.closed = False
        self.lengths = np.array([app.lengths[c] for c in self.ctxs], dtype=np.int64)
        self.host_table = np.full((n, app.cpc), -1, dtype=np.int32)
        for i, c in enumerate(self.ctxs):
            rows = app.rows(c)
            assert (app.slot[rows] >= 0).all()
            self.host_table[i, :len(rows)] = app.slot[rows]
        self.table = torch.from_numpy(self.host_table).cuda()
        self.lens = torch.from_numpy(self.lengths.astype(np.int32)).cuda()
        self.mass = torch.zeros(sh.n_layers, n, sh.n_kv_heads, self.capacity, dtype=torch.float32, device="cuda")
        self.new_lens = torch.empty_like(self.lens)
        self.workspace = torch.empty(B.decode_workspace_bytes(app.desc_pool, n, self.capacity, True), dtype=torch.uint8, device="cuda")

    @contextlib.contextmanager
    def _on_another_stream(self):
        """The body's calls go to the pool's stream, between what the current stream has and what it gets."""
        here = torch.cuda.current_stream()
        self.app.main.wait_stream(here)
        try:
            with torch.cuda.stream(self.app.main):
                yield
        finally:
            here.wait_stream(self.app.main)

    def _on_pool_stream(self):
        return contextlib.nullcontext() if B.current_stream() == self._main else self._on_another_stream()

    def _check_open(self):
        if self.closed:
            raise RuntimeError("the step that this batch was served in has ended: its chunks may be others' by now")

    def advance(self):
        """Room for one more token per context: its length grows by one, by a new chunk where the last one is full."""
        self._check_open()
        app = self.app
        if (self.lengths >= self.capacity).any():
            raise RuntimeError("a context is full: shrink it before it takes more tokens")
        grown = [i for i in range(len(self.ctxs)) if self.lengths[i] % app.shape.chunk_len == 0]
        with self._on_pool_stream():
            slots = app.take_slots(len(grown))
            for i, s in zip(grown, slots):
                chunk = int(self.lengths[i]) // app.shape.chunk_len
                app.occupy(self.ctxs[i] * app.cpc + chunk, s)
                self.host_table[i, chunk] = s
            if grown:
                self.table.copy_(torch.from_numpy(self.host_table))
            self.lengths += 1
            self.lens += 1

    def decode(self, layer, q, k_new, v_new, out=None):
        """Attention of the newest token of every context in one layer: q [n, n_q_heads, head_dim], k_new and v_new
        [n, n_kv_heads, head_dim], fp16 (views of one projection's output will do).  Stores k_new and v_new as the newest
        token's rows, adds the attention weights to self.mass, returns the output rows."""
        self._check_open()
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
        if B.current_stream() != self._main and not torch.cuda.is_current_stream_capturing():
            with self._on_another_stream():
                self._decode(layer, q, k_new, v_new, out)
        else:
            self._decode(layer, q, k_new, v_new, out)
        return out

    def _decode(self, layer, q, k_new, v_new, out):
        B.decode_attention(self.app.desc_pool, layer, self.app.pool, q, self.table, self.lens, self.capacity, out, self.workspace,
                           k_new=k_new, v_new=v_new, mass_in=self.mass[layer], mass_out=self.mass[layer])

    def shrink(self, budget, recent):
        """Every context longer than `budget` keeps, per layer and KV head, that many tokens: the last `recent` ones and those
        with the largest accumulated weight.  Returns the kept positions [n_layers, n, n_kv_heads, budget] (device)."""
        self._check_open()
        app = self.app
        sh = app.shape
        kept = torch.empty(sh.n_layers, len(self.ctxs), sh.n_kv_heads, budget, dtype=torch.int32, device="cuda")
        with self._on_pool_stream():
            B.evict_tokens(app.desc_pool, app.pool, self.mass, self.table, self.lens, self.capacity, budget, recent, kept, self.new_lens)
            self.lens.copy_(self.new_lens)
            self.lengths = np.minimum(self.lengths, budget)
            for i, c in enumerate(self.ctxs):
                first = -(-int(self.lengths[i]) // sh.chunk_len)
                gone = self.host_table[i, first:]
                app.vacate(c * app.cpc + first + np.flatnonzero(gone >= 0))
                gone[:] = -1
            self.table.copy_(torch.from_numpy(self.host_table))
        return kept

    def close(self):
        """The end of the step: the contexts' lengths are what the pool's bookkeeping goes by from now on, and the batch is no
        longer to be used (nor graphs captured from it)."""
        self.closed = True
        for i, c in enumerate(self.ctxs):
            self.app.lengths[c] = int(self.lengths[i])
