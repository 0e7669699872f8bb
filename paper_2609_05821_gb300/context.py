"""Contexts of a serving batch kept in a 4-bit paged cache.

``PackedContexts`` ties the calls together as a serving loop uses them: prompts
(image patches with their time, height and width positions, then text) are
appended with the rotation applied on the way, decoding steps append one token
per request and attend over everything cached so far, and a context that is to
be scored and refreshed is taken up into a plain cache.

    ctx = PackedContexts(num_requests, max_len, num_layers, num_q_heads, num_kv_heads, head_dim, rope)
    q_rot = ctx.append(rows, k, v, pos, q)            # rows: new tokens per request
    out = ctx.attend(rows, q_rot)                     # [L, T, Hq, d], causal at the end of each context
    step = ctx.decoder(dtype)                         # buffers of a one-token step
    out = step(q, k, v, pos)                          # append and attend, capturable in a CUDA graph
    ctx.take_up(batch, kv)                            # values into a cache that conduit_score reads

The lengths live on the device (``ctx.lens``) and advance in place, so a captured
step can be replayed while the contexts grow. A request whose new rows do not fit into
max_len keeps its tokens and its length, none of the rows is written and ``check`` says so; what
the same step's attention returns for such rows is not theirs. A context ends by setting
its length (``ctx.lens[r] = 0``). Every buffer belongs to the object;
its calls run on the caller's current stream.
"""

from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import conduit as C


_NO_SLOT = 2 ** 31 - 1  # a length whose rows all lie past any context: flagged, and not written


class PackedContexts:
    def __init__(self, num_requests: int, max_len: int, num_layers: int, num_q_heads: int, num_kv_heads: int,
                 head_dim: int, rope: Optional[C.Rope] = None, page_size: int = 16, device="cuda"):
        pages = -(-max_len // page_size)
        table = torch.arange(num_requests * pages, dtype=torch.int32, device=device).view(num_requests, pages)
        self.kv = C.PackedKv.empty(num_layers, num_requests * pages, num_q_heads, num_kv_heads, head_dim, page_size,
                                   table, device)
        self.rope, self.max_len, self.num_requests = rope, max_len, num_requests
        self.lens = torch.zeros(num_requests, dtype=torch.int32, device=device)
        self._grown = torch.zeros_like(self.lens)  # the lengths with a call's rows, until the call is accepted
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def _seqs(self, rows: Sequence[int], lens: torch.Tensor) -> C.Seqs:
        if len(rows) != self.num_requests or min(rows, default=0) < 0:
            raise C.ConduitError(C.ERR_INVALID_ARG, f"rows needs a count >= 0 for each of {self.num_requests} requests")
        off = [0]
        for n in rows:
            off.append(off[-1] + int(n))
        return C.Seqs(off, lens, self.max_len)

    def append(self, rows: Sequence[int], k, v, pos=None, q=None):
        """New tokens, rows[r] of request r: keys turned and packed, queries turned. Returns the turned
        queries (None without q). Rows k, v [L, T, Hkv, d], q [L, T, Hq, d], pos int32 [A, T]. A call that
        raises leaves the contexts as they were."""
        seqs = self._seqs(rows, self._grown)
        more = torch.tensor([int(n) for n in rows], dtype=torch.int32, device=self.lens.device)
        fits = more <= self.max_len - self.lens
        self._grown.copy_(torch.where(fits, self.lens + more, _NO_SLOT))
        q_rot = C.conduit_packed_append(self.kv, seqs, k, v, self.rope, pos, q, status=self.status)
        self.lens.copy_(torch.where(fits, self._grown, self.lens))
        return q_rot

    def attend(self, rows: Sequence[int], q, limits=None, lse=None):
        """Attention of the newest rows[r] tokens of each request over its context."""
        return C.conduit_packed_attn(self.kv, self._seqs(rows, self.lens), q, limits=limits, lse=lse, status=self.status)

    def decoder(self, dtype: torch.dtype = torch.bfloat16):
        """A one-token step: step(q, k, v, pos) appends a row per request and returns their attention
        [L, R, Hq, d]. Its buffers are allocated here, so that it can be captured."""
        kv, R = self.kv, self.num_requests
        seqs, grown = self._seqs([1] * R, self.lens), self._seqs([1] * R, self._grown)
        shape = (kv.num_layers, R, kv.num_q_heads, kv.head_dim)
        q_rot, out = (torch.empty(shape, dtype=dtype, device=self.lens.device) for _ in range(2))
        need = C.conduit_packed_attn_workspace_size(kv, seqs, dtype)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=self.lens.device)

        def step(q, k, v, pos=None):
            torch.add(self.lens, 1, out=self._grown)
            C.conduit_packed_append(kv, grown, k, v, self.rope, pos, q, q_rot, status=self.status)
            torch.clamp(self._grown, max=self.max_len, out=self.lens)
            return C.conduit_packed_attn(kv, seqs, q_rot, out=out, workspace=workspace, status=self.status)

        return step

    def take_up(self, batch: C.Batch, dst: C.KvCache, first=None):
        """The values of tokens first[r] .. of every request into a plain cache, as the batch lays it out."""
        C.conduit_packed_read(self.kv, batch, dst, first, status=self.status)
        return dst

    def check(self) -> int:
        """Synchronises; C.OK, or what the device found since the last check."""
        code = C.conduit_read_status(self.status)
        C.conduit_clear_status(self.status)
        return code
