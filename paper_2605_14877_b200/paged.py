"""A paged cache of requests of any length: its buffers, and the library's calls in the order in which a model's step makes them (pages
and slots of the new tokens; then per layer the store of their K and V and their attention).  Pure call sequencing; every computation
happens inside the library."""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import heatkv as hk


class Step:
    """The new tokens of one model step: `positions` for the position encoding, `batch` and `slots` for the calls, and `kv_len`, the tokens
    that every row attends to (int32, on the device): 0 for a row whose new tokens were refused."""

    def __init__(self, batch: hk.PagedBatch, slots: torch.Tensor, positions: torch.Tensor, kv_len: torch.Tensor):
        self.batch, self.slots, self.positions, self.kv_len = batch, slots, positions, kv_len


class PagedCache:
    """`rows` requests at a time, each with up to `max_pages` pages of 64 tokens out of `n_pages`, which all layers use alike.

    A row is free while its length is 0.  `begin(new)` takes the number of new tokens of every row (host integers: they size the step's
    buffers); per layer, `attend` stores K and V and attends; `keep` cuts requests back (drafted tokens that were turned down) or ends them."""

    def __init__(self, layers: int, n_heads: int, n_kv_heads: int, d: int, n_pages: int, rows: int, max_pages: int,
                 dtype: torch.dtype = torch.bfloat16, summaries: bool = False, device: str = "cuda:0"):
        self.n_heads, self.rows = n_heads, rows
        self.device = torch.device(device)
        new = lambda *shape, dt=torch.int32: torch.zeros(shape, dtype=dt, device=self.device)      # noqa: E731
        self.pools = []
        for _ in range(layers):
            k, v = new(n_pages, n_kv_heads, hk.PAGE_TOKENS, d, dt=dtype), new(n_pages, n_kv_heads, hk.PAGE_TOKENS, d, dt=dtype)
            codes = (new(n_pages, n_kv_heads, d, dt=torch.int8), new(n_pages, n_kv_heads, dt=torch.float32)) if summaries else (None, None)
            self.pools.append(hk.PagedPool.make(k, v, *codes))
        self.table = new(rows, max_pages)
        self.free = torch.arange(n_pages, dtype=torch.int32, device=self.device)
        self.state = torch.tensor([0, n_pages, 0, 0], dtype=torch.int32, device=self.device)
        self.other_state = new(4)
        self.lengths = new(rows)                       # tokens of every row
        self.at_most = [0] * rows                      # ... as far as the host knows: more where rows sat a step out
        self.workspace: Optional[torch.Tensor] = None

    def begin(self, new: Sequence[int]) -> Step:
        """Pages and slots of a step with new[i] new tokens in row i (0: none).  Pages are wanted in row order, and from the first row that the free
        ones do not suffice for, every row that needs one is refused; a row that would outgrow `max_pages` is refused alone.  Refused rows
        sit the step out: their new tokens are stored nowhere, their rows of the attention are zero, their length stays.  The step's `kv_len` is
        0 for them, and `state[2]` counts them: their tokens have to come again."""
        if len(new) != self.rows or min(new) < 0 or sum(new) == 0:
            raise ValueError(f"new: expected {self.rows} numbers of tokens, none below 0 and not all 0, got {list(new)}")
        tokens, longest = sum(new), max(new)
        count = torch.tensor(list(new), dtype=torch.int32, device=self.device)
        q_begin, kv_len = torch.empty(self.rows + 1, dtype=torch.int32, device=self.device), torch.empty_like(count)
        slots, positions = (torch.empty(tokens, dtype=torch.int32, device=self.device) for _ in range(2))
        hk.heatkv_paged_tables(count, self.lengths, self.free, self.state, self.other_state, self.table, q_begin, kv_len, slots, positions)
        self.state, self.other_state = self.other_state, self.state
        self.lengths = torch.where(kv_len > 0, kv_len, self.lengths)
        self.at_most = [a + n for a, n in zip(self.at_most, new)]
        # the calls get no more of the table than may be in use: its width is what they know of lengths beforehand
        pages = min(max(-(-max(self.at_most) // hk.PAGE_TOKENS), 1), self.table.shape[1])
        step = Step(hk.PagedBatch.make(q_begin, kv_len, self.table[:, :pages], tokens, longest), slots, positions, kv_len)
        need = hk.heatkv_paged_workspace_bytes(self.pools[0], step.batch, self.n_heads)
        if self.workspace is None or self.workspace.numel() < need:
            grown = torch.zeros(need, dtype=torch.uint8, device=self.device)
            if self.workspace is not None:
                grown[:4] = self.workspace[:4]         # (the status, for the next `check`)
            self.workspace = grown
        return step

    def attend(self, layer: int, step: Step, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
               lse: Optional[torch.Tensor] = None, causal: bool = True, sm_scale: float = 0.0, pages: int = 0, sink: int = 1,
               local: int = 2) -> None:
        """Stores k, v [tokens, n_kv_heads, d] and writes to out the attention of q [tokens, n_heads, d]: over everything, or (pages > 0, always
        causal) over that many pages of each token's choice."""
        if pages > 0 and not causal:
            raise ValueError("attention over selected pages is causal: a token's choice ends with its own page")
        pool = self.pools[layer]
        hk.heatkv_paged_store(pool, k, v, step.slots)
        if pages == 0:
            hk.heatkv_paged_attention(pool, step.batch, q, out, lse, self.workspace, causal, sm_scale)
            return
        sel = torch.empty(step.batch.n_tokens, pool.n_kv_heads, pages, dtype=torch.int32, device=self.device)
        hk.heatkv_paged_select(pool, step.batch, q, sel, sink, local)
        hk.heatkv_paged_sparse_attention(pool, step.batch, q, sel, out, lse, self.workspace, sm_scale)

    def check(self) -> None:
        """Raises HeatKVError if a bounded wait inside a kernel ran out since the last look: what `attend` wrote since then is not to be used.  The
        workspace is zeroed, so that the steps can be attended to again (K and V are stored whatever happens there).  Waits for the device."""
        status = hk.heatkv_paged_status(self.workspace) if self.workspace is not None else 0
        if status != 0:
            if status == -7:                           # HEATKV_ERR_DEVICE_TIMEOUT
                self.workspace.zero_()
            raise hk.HeatKVError(status, "PagedCache.check")

    def keep(self, lengths: Sequence[int]) -> None:
        """Cuts row i back to lengths[i] tokens (0: the request is over, its row and pages are free; more than it has: it stays as it is)."""
        if len(lengths) != self.rows or min(lengths) < 0:
            raise ValueError(f"lengths: expected {self.rows} numbers of tokens, none below 0, got {list(lengths)}")
        keep = torch.tensor(list(lengths), dtype=torch.int32, device=self.device)
        hk.heatkv_paged_release(self.lengths, keep, self.table, self.free, self.state, self.other_state)
        self.state, self.other_state = self.other_state, self.state
        self.lengths = torch.minimum(self.lengths, keep)
        self.at_most = [min(a, n) for a, n in zip(self.at_most, lengths)]
