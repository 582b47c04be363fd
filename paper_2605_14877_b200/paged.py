"""A paged cache of requests of any length: its buffers, and the library's calls in the order in which a model's step makes them (pages
and slots of the new tokens; then per layer the store of their K and V and their attention).  Pure call sequencing; every computation
happens inside the library."""
from __future__ import annotations

from typing import Optional, Sequence, Tuple

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
    buffers); per layer, `attend` stores K and V and attends; `keep` cuts requests back (drafted tokens that were turned down) or ends them;
    `fork` makes rows copies of others (beams, several answers to one prompt), whose full pages they share; `compact` takes tokens out of the cache.
    With bits=4 the pages hold 4-bit codes (values code * scale * 2^k_exp, 2^v_exp), 3.6 times as many tokens in the same memory."""

    def __init__(self, layers: int, n_heads: int, n_kv_heads: int, d: int, n_pages: int, rows: int, max_pages: int,
                 dtype: torch.dtype = torch.bfloat16, summaries: bool = False, device: str = "cuda:0", bits: int = 16, k_exp: int = 0, v_exp: int = 0):
        if bits not in (4, 16) or (bits == 16 and (k_exp or v_exp)):
            raise ValueError(f"bits: expected 4 or 16 (k_exp and v_exp are for 4), got {bits}")
        if bits == 4 and summaries:
            raise ValueError("page summaries are for a cache of 16 bits")
        self.n_heads, self.rows, self.bits = n_heads, rows, bits
        self.device = torch.device(device)
        new = lambda *shape, dt=torch.int32: torch.zeros(shape, dtype=dt, device=self.device)      # noqa: E731
        self.pools = []
        for _ in range(layers):
            if bits == 4:
                blocks = new(n_pages, n_kv_heads, hk.PagedPool4.block_bytes(d), dt=torch.uint8)
                self.pools.append(hk.PagedPool4.make(blocks, d, dtype, k_exp, v_exp))
                continue
            k, v = new(n_pages, n_kv_heads, hk.PAGE_TOKENS, d, dt=dtype), new(n_pages, n_kv_heads, hk.PAGE_TOKENS, d, dt=dtype)
            codes = (new(n_pages, n_kv_heads, d, dt=torch.int8), new(n_pages, n_kv_heads, dt=torch.float32)) if summaries else (None, None)
            self.pools.append(hk.PagedPool.make(k, v, *codes))
        self.table = new(rows, max_pages)
        self.free = torch.arange(n_pages, dtype=torch.int32, device=self.device)
        self.state = torch.tensor([0, n_pages, 0, 0], dtype=torch.int32, device=self.device)
        self.other_state = new(4)
        self.lengths = new(rows)                       # tokens of every row
        self.at_most = [0] * rows                      # ... as far as the host knows: more where rows sat a step out, or tokens left
        self.workspace: Optional[torch.Tensor] = None
        # what `fork` and `compact` need, from their first use on: the other table and lengths, moves, a workspace
        self.other: Optional[Tuple[torch.Tensor, torch.Tensor]] = None
        self.moves = new(2, 0)
        self.rows_workspace: Optional[torch.Tensor] = None
        self.shared = False                            # may rows list the same pages
        # tokens that `compact` took out of every row, and in front of each of its first `upto` places
        self.gone: Optional[torch.Tensor] = None
        self.left, self.upto, self.places = new(rows, 0, dt=torch.int64), new(rows), new(0, dt=torch.int64)

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
        if self.gone is not None:                      # places in the cache are not the positions any more
            positions += torch.repeat_interleave(self.gone, count, output_size=tokens)
        self.at_most = [a + n for a, n in zip(self.at_most, new)]
        # the calls get no more of the table than may be in use: its width is what they know of lengths beforehand
        pages = min(max(-(-max(self.at_most) // hk.PAGE_TOKENS), 1), self.table.shape[1])
        step = Step(hk.PagedBatch.make(q_begin, kv_len, self.table[:, :pages], tokens, longest), slots, positions, kv_len)
        need = (hk.heatkv_paged_workspace_bytes if self.bits == 16 else hk.heatkv_paged4_workspace_bytes)(self.pools[0], step.batch, self.n_heads)
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
        if self.bits == 4:
            if pages > 0:
                raise ValueError("attention over selected pages is for a cache of 16 bits")
            hk.heatkv_paged4_store(pool, k, v, step.slots)
            hk.heatkv_paged4_attention(pool, step.batch, q, out, lse, self.workspace, causal, sm_scale)
            return
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
        """Cuts row i back to lengths[i] tokens (0: the request is over, its row and pages are free; more than it has: it stays as it is).  Where rows share
        pages, a row that is cut to a place inside a page which another row has whole gets a copy of it, from a free page or one that this
        call frees.  Where there is none it loses that page's tokens, too, and goes on at the position of the first of them: `lengths` says what it has, and
        `state[2]` counts such rows."""
        if len(lengths) != self.rows or min(lengths) < 0:
            raise ValueError(f"lengths: expected {self.rows} numbers of tokens, none below 0, got {list(lengths)}")
        keep = torch.tensor(list(lengths), dtype=torch.int32, device=self.device)
        if self.shared:
            own = torch.arange(self.rows, dtype=torch.int32, device=self.device)
            asked = torch.minimum(self.lengths, keep) if self._may_run_out() else None
            if any(n < a and n % hk.PAGE_TOKENS for a, n in zip(self.at_most, lengths)):
                # whole pages first: that takes none, moves nothing, and what it frees is there for the copies
                most = self.table.shape[1]
                whole = torch.tensor([min(-(-n // hk.PAGE_TOKENS), most) * hk.PAGE_TOKENS for n in lengths], dtype=torch.int32, device=self.device)
                self._rearrange(hk.heatkv_paged_fork, (own, whole), self.rows * hk.PAGE_TOKENS, moves=False)
            self._rearrange(hk.heatkv_paged_fork, (own, keep), self.rows * hk.PAGE_TOKENS)
            self.at_most = [min(a, n) for a, n in zip(self.at_most, lengths)]
            self.shared = sum(n > 0 for n in self.at_most) > 1
            self._forget(asked)
            return
        hk.heatkv_paged_release(self.lengths, keep, self.table, self.free, self.state, self.other_state)
        self.state, self.other_state = self.other_state, self.state
        self.lengths = torch.minimum(self.lengths, keep)
        self.at_most = [min(a, n) for a, n in zip(self.at_most, lengths)]
        self._forget()

    def fork(self, parents: Sequence[Optional[int]]) -> None:
        """Row i goes on as a copy of row parents[i] (its own number: as it is; None: it is over).  Full pages are shared; of a page that is not full every
        row but one gets a copy, from a free page each.  Where those end, rows lose that page's tokens and go on at the position of the first of them: `lengths`
        says what they have, and `state[2]` counts them."""
        if len(parents) != self.rows or any(p is not None and not 0 <= p < self.rows for p in parents):
            raise ValueError(f"parents: expected {self.rows} rows or None, got {list(parents)}")
        of = torch.tensor([-1 if p is None else p for p in parents], dtype=torch.int32, device=self.device)
        before, short = self.lengths, self._may_run_out()
        self._rearrange(hk.heatkv_paged_fork, (of, None), self.rows * hk.PAGE_TOKENS)
        self.at_most = [0 if p is None else self.at_most[p] for p in parents]
        parents = [p for p, n in zip(parents, self.at_most) if n]
        self.shared = (self.shared or len(set(parents)) < len(parents)) and len(parents) > 1
        if self.gone is not None:
            row = of.clamp(min=0).long()
            self.gone, self.left, self.upto = self.gone[row], self.left[row], self.upto[row]
            self._forget(torch.where(of >= 0, before[row], 0) if short else None)

    def compact(self, stays: torch.Tensor) -> None:
        """Token t of row i leaves the cache where stays[i, t] (bool, on the device) is False; tokens past its width stay.  The others keep their
        order and the positions that they were encoded with, and `begin` goes on counting positions as if nothing had left (so `keep` is to cut such a
        row behind its last token that left).  Tokens move into free pages: rows for which those do not suffice stay as they are (`state[2]` counts
        them).  The host does not learn how many tokens are left, which steps and further compactions are sized by: `keep` with a number that no row exceeds
        tells it."""
        if stays.dtype is not torch.bool or stays.dim() != 2 or stays.shape[0] != self.rows:
            raise ValueError(f"stays: expected bool [{self.rows}, tokens], got {stays.dtype} {tuple(stays.shape)}")
        before = self.lengths
        self._rearrange(hk.heatkv_paged_compact, (stays,), min(max(sum(self.at_most), 1), self.free.numel() * hk.PAGE_TOKENS))
        self._count_out(stays, before)
        self._forget()

    def _count_out(self, stays: torch.Tensor, before: torch.Tensor) -> None:
        """What left in front of every place of the rows that a compaction changed (it leaves the lengths of the others as they were)."""
        changed = self.lengths < before
        if self.gone is None:
            self.gone = torch.zeros_like(before)
        if stays.shape[1] < self.left.shape[1]:        # (what the mask does not reach stays)
            stays = torch.nn.functional.pad(stays, (0, self.left.shape[1] - stays.shape[1]), value=True)
        width = stays.shape[1]
        if self.places.numel() < width:
            self.places = torch.arange(width, device=self.device)
        place = self.places[:width]
        leaves = (place < torch.where(changed, before, 0)[:, None]) > stays
        in_front = leaves.cumsum(1)
        left = in_front + self.gone[:, None]
        known = self.left.shape[1]
        if known > 0:
            left[:, :known] = torch.where(place[:known] < self.upto[:, None], self.left + in_front[:, :known], left[:, :known])
        # (those that left are written behind the others, to a column that is dropped)
        self.left = left.new_empty(self.rows, width + 1).scatter_(1, (place - in_front).masked_fill_(leaves, width), left)[:, :width]
        went = before - self.lengths
        self.upto, self.gone = torch.minimum(self.lengths, width - went), self.gone + went

    def _rearrange(self, call, what, n_moves: int, moves: bool = True) -> None:
        """One of the two calls that write new lengths and a new table, and the moves of K and V that it asks for (moves False: it asks for none)."""
        if self.rows_workspace is None:
            need = hk.heatkv_paged_rows_workspace_bytes(self.rows, self.table.shape[1], self.free.numel())
            self.rows_workspace = torch.zeros(need, dtype=torch.uint8, device=self.device)
        if self.other is None:
            self.other = torch.zeros_like(self.lengths), torch.zeros_like(self.table)
        if self.moves.shape[1] < n_moves:
            self.moves = torch.empty(2, n_moves, dtype=torch.int32, device=self.device)
        (lengths, table), (source, target) = self.other, (m[:n_moves] for m in self.moves)
        call(*what, self.lengths, self.table, self.free, self.state, lengths, table, self.other_state, source, target, self.rows_workspace)
        self.other = torch.empty_like(lengths), self.table         # (the old lengths may still be somebody's)
        self.lengths, self.table = lengths, table
        self.state, self.other_state = self.other_state, self.state
        move = hk.heatkv_paged_move if self.bits == 16 else hk.heatkv_paged4_move
        for pool in self.pools if moves else ():
            move(pool, source, target)

    def _may_run_out(self) -> bool:
        """May a call that gives every row a page find too few, for rows of which tokens left?"""
        return self.gone is not None and self.free.numel() < self.rows + sum(min(-(-n // hk.PAGE_TOKENS), self.table.shape[1]) for n in self.at_most)

    def _forget(self, asked: Optional[torch.Tensor] = None) -> None:
        """A row that is over has nothing that left it; one that was cut deeper than `asked` goes on at the position of the first token that it was not to lose."""
        if self.gone is None:
            return
        if self.left.shape[1] > 0:
            if asked is not None:
                in_front = lambda n: torch.where(n < self.upto, self.left.gather(1, n.clamp(max=self.left.shape[1] - 1).long()[:, None])[:, 0],      # noqa: E731
                                                 self.gone)
                self.gone = self.gone - in_front(asked) + in_front(self.lengths)
            self.upto = torch.minimum(self.upto, self.lengths)
        self.gone = torch.where(self.lengths > 0, self.gone, 0)
