"""PagedCache's own part of the work, on the CPU: the library's calls are played by the plain oracle, and what lies in every slot is a token's number, so that a
row's tokens, their order and the positions of those to come are compared with a plain list of them."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from paper_2605_14877_b200 import heatkv as H
from paper_2605_14877_b200.paged import PagedCache

PAGE = 64


class Server:
    """A cache of one layer, the oracle behind its calls, and the lists: `held` has (number, position) of every token of a row, `next` the position of the one
    to come."""

    def __init__(self, monkeypatch, n_pages, rows, max_pages, bits=4):
        self.slots, self.tokens, self.calls = np.full(n_pages * PAGE, -1), 0, []
        for name in ("tables", "release", "fork", "compact"):
            monkeypatch.setattr(H, f"heatkv_paged_{name}", getattr(self, f"_{name}"))
        for name in ("paged", "paged4"):
            monkeypatch.setattr(H, f"heatkv_{name}_workspace_bytes", lambda *a: 256)
            monkeypatch.setattr(H, f"heatkv_{name}_move", self._move)
        self.cache = PagedCache(1, 2, 1, 64, n_pages=n_pages, rows=rows, max_pages=max_pages, device="cpu", bits=bits)
        self.held, self.next = [[] for _ in range(rows)], [0] * rows

    # ---- the library's calls
    @staticmethod
    def _ring(free, state):
        head, count = state.tolist()[:2]
        return [int(free[(head + j) % len(free)]) for j in range(count)]

    def _tables(self, new, past, free, state, state_out, table, q_begin, kv_len, slots, positions):
        self.calls.append("tables")
        fifo = self._ring(free, state)
        made, begin, kv, slot, pos, taken, refused = P.tables(new.tolist(), past.tolist(), fifo, table.numpy(), len(slots))
        for out, x in ((table, made), (q_begin, begin), (kv_len, kv), (slots, slot), (positions, pos)):
            out.copy_(torch.from_numpy(np.asarray(x)))
        state_out.copy_(torch.tensor([(int(state[0]) + taken) % len(free), len(fifo) - taken, refused, int(new.sum())]))

    def _back(self, free, state, state_out, taken, back, third, fourth):
        head, count = state.tolist()[:2]
        for j, page in enumerate(back):
            free[(head + count + j) % len(free)] = page
        state_out.copy_(torch.tensor([(head + taken) % len(free), count - taken + len(back), third, fourth]))

    def _release(self, kv_len, keep_len, table, free, state, state_out):
        self.calls.append("release")
        back = [int(page) for row, n, k in zip(table, kv_len.tolist(), keep_len.tolist()) for page in row[-(-min(n, k) // PAGE): -(-n // PAGE)]]
        assert len(set(back)) == len(back) and not set(back) & set(self._ring(free, state))            # (no page for two rows)
        self._back(free, state, state_out, 0, back, 0, len(back))

    def _fork(self, parents, keep, lengths, table, free, state, lengths_out, table_out, state_out, source, target, workspace):
        self.calls.append("fork")
        new, made, a, b, taken, cut, back = P.fork(parents.tolist(), [10**9] * len(parents) if keep is None else keep.tolist(), lengths.tolist(), table.numpy(),
                                                   self._ring(free, state))
        for out, x in ((lengths_out, new), (table_out, made), (source, a), (target, b)):
            out.copy_(torch.from_numpy(x))
        self._back(free, state, state_out, taken, back, cut, len(back))

    def _compact(self, stays, lengths, table, free, state, lengths_out, table_out, state_out, source, target, workspace):
        self.calls.append("compact")
        new, made, a, b, taken, refused, back, done = P.compact(stays.numpy(), lengths.tolist(), table.numpy(), self._ring(free, state), len(source))
        for out, x in ((lengths_out, new), (table_out, made), (source, a), (target, b)):
            out.copy_(torch.from_numpy(np.asarray(x)))
        self._back(free, state, state_out, taken, back, refused, done)

    def _move(self, pool, source, target):
        self.calls.append("move")
        pairs = [(a, b) for a, b in zip(source.tolist(), target.tolist()) if a >= 0 and b >= 0]
        for b, x in [(b, self.slots[a]) for a, b in pairs]:
            self.slots[b] = x

    # ---- what a server does
    def check(self):
        lengths, table = self.cache.lengths.tolist(), self.cache.table
        assert lengths == [len(x) for x in self.held]
        assert all(a >= n for a, n in zip(self.cache.at_most, lengths))
        for i, row in enumerate(self.held):
            assert [int(self.slots[int(table[i][t // PAGE]) * PAGE + t % PAGE]) for t in range(len(row))] == [number for number, _ in row], i
        listed = {int(table[i][j]) for i, n in enumerate(lengths) for j in range(-(-n // PAGE))}
        ring = self._ring(self.cache.free, self.cache.state)
        assert sorted(listed | set(ring)) == list(range(len(self.cache.free))) and len(listed) + len(ring) == len(self.cache.free)

    def begin(self, new):
        step = self.cache.begin(new)
        slots, positions, at = step.slots.tolist(), step.positions.tolist(), 0
        for i, n in enumerate(new):
            if step.kv_len[i] > 0:
                assert positions[at: at + n] == list(range(self.next[i], self.next[i] + n)), i
                for slot in slots[at: at + n]:
                    self.slots[slot] = self.tokens
                    self.held[i].append((self.tokens, self.next[i]))
                    self.tokens += 1
                    self.next[i] += 1
            at += n
        self.check()

    @staticmethod
    def _in_front(row, to_come, n):
        """How many tokens left in front of place n of a row."""
        return row[n][1] - n if n < len(row) else to_come - len(row)

    def _cut(self, wanted):
        """Rows cut to the numbers of tokens that were wanted, which go on as many positions behind those as before, or to that number's whole pages: then
        they go on at the first token that they were not to lose.  How many those are."""
        short = 0
        for i, (n, want) in enumerate(zip(self.cache.lengths.tolist(), wanted)):
            row, to_come = self.held[i], self.next[i]
            assert n in (want, want // PAGE * PAGE)
            short += n != want
            left = to_come - len(row) - self._in_front(row, to_come, want) + self._in_front(row, to_come, n)
            self.held[i], self.next[i] = row[:n], n + left if n else 0
        assert self.cache.state.tolist()[2] == short
        self.check()
        return short

    def fork(self, parents):
        self.cache.fork(parents)
        self.held = [[] if p is None else list(self.held[p]) for p in parents]
        self.next = [0 if p is None else self.next[p] for p in parents]
        return self._cut([len(x) for x in self.held])

    def keep(self, lengths):
        self.cache.keep(lengths)
        return self._cut([min(len(x), n) for x, n in zip(self.held, lengths)])

    def compact(self, stays):
        stays = torch.as_tensor(stays, dtype=torch.bool)
        before = [len(x) for x in self.held]
        self.cache.compact(stays)
        for i, n in enumerate(self.cache.lengths.tolist()):
            kept = [x for t, x in enumerate(self.held[i]) if t >= stays.shape[1] or stays[i, t]]
            if n == len(kept):
                self.held[i] = kept
                self.next[i] = self.next[i] if kept else 0
            else:
                assert n == before[i] and self.cache.state[2] > 0
        self.check()


def test_a_row_that_lost_its_tokens_to_a_fork_begins_anew(monkeypatch):
    """No page is free: a copy of a row of less than a page has nothing, and whoever comes next in its place starts at position 0."""
    s = Server(monkeypatch, n_pages=4, rows=3, max_pages=4)
    s.begin([192, 0, 40])
    stays = np.ones((3, 40), dtype=bool)
    stays[2, 5:25] = False
    s.keep([128, 0, 40])
    s.compact(stays)
    s.begin([64, 0, 0])
    assert s.cache.lengths.tolist() == [192, 0, 20] and s.cache.state.tolist()[1] == 0
    assert s.fork([0, 2, 2]) == 1 and s.cache.lengths.tolist() == [192, 0, 20]
    s.fork([None, 1, 2])
    s.begin([0, 5, 3])


def test_a_cut_into_a_shared_page_takes_a_page_that_the_same_call_frees(monkeypatch):
    """Row 0 is cut to a place inside a page that row 1 has whole, and no page is free before row 2 ends in the same call."""
    s = Server(monkeypatch, n_pages=3, rows=3, max_pages=4)
    s.begin([128, 0, 10])
    s.fork([0, 0, 2])
    assert s.cache.state.tolist()[1] == 0
    assert s.keep([100, 128, 0]) == 0 and s.cache.lengths.tolist() == [100, 128, 0]
    assert s.cache.state.tolist()[1] == 0
    # nothing is freed: then the page's tokens are lost, and the call says so
    s.fork([1, 1, None])
    s.begin([0, 0, 1])
    assert s.keep([100, 2**31 - 1, 1000]) == 1 and s.cache.lengths.tolist() == [64, 128, 1]
    # one row's pages are enough for another's copy, whatever their order
    s = Server(monkeypatch, n_pages=5, rows=3, max_pages=4)
    s.begin([128, 0, 192])
    s.fork([0, 0, 2])
    assert s.cache.state.tolist()[1] == 0
    assert s.keep([1000, 65, 150]) == 1                    # (the third row keeps its third page)
    assert s.keep([30, 1000, 64]) == 0 and s.cache.lengths.tolist() == [30, 64, 64]


def test_a_cut_of_whole_rows_is_one_call(monkeypatch):
    """Only a place inside a page may want a page: rows that end, or that are not cut, take no second call."""
    s = Server(monkeypatch, n_pages=9, rows=3, max_pages=4)
    s.begin([128, 0, 10])
    s.fork([0, 0, 2])
    s.calls.clear()
    s.keep([1000, 0, 1000])
    assert s.calls.count("fork") == 1


def test_positions_of_a_row_that_lost_tokens_among_which_some_had_left(monkeypatch):
    """A call that has no page for a copy cuts a row where nobody asked it to: the next token takes the position of the first one that was lost."""
    s = Server(monkeypatch, n_pages=4, rows=2, max_pages=4)
    s.begin([150, 0])
    stays = np.ones((2, 150), dtype=bool)
    stays[0, 140:145] = False
    s.compact(stays)
    s.begin([0, 64])
    assert s.fork([0, 0]) == 1 and s.cache.lengths.tolist() == [145, 128] and s.next == [150, 128]
    s.fork([None, 1])
    s.begin([0, 30])
    s.begin([60, 0])
    # the same by a cut, in front of which others had left
    s = Server(monkeypatch, n_pages=5, rows=3, max_pages=4)
    s.begin([150, 0, 0])
    stays = np.ones((3, 150), dtype=bool)
    stays[0, 70:77] = stays[0, 141] = False
    s.compact(stays)
    s.begin([50, 0, 0])
    s.fork([0, 0, 2])
    s.begin([0, 0, 64])
    assert s.cache.lengths.tolist() == [192, 192, 64] and s.cache.state.tolist()[1] == 1 and s.next == [200, 200, 64]
    s.begin([0, 0, 1])
    assert s.keep([180, 1000, 1000]) == 1 and s.cache.lengths.tolist() == [128, 192, 65] and s.next == [135, 200, 65]


@pytest.mark.parametrize("seed", range(30))
def test_a_server_at_random(monkeypatch, seed):
    """Steps, forks, cuts and compactions in any order, with and without enough pages: tokens, positions and pages as the lists have them."""
    rng = np.random.default_rng(seed)
    rows = int(rng.integers(1, 6))
    s = Server(monkeypatch, n_pages=int(rng.integers(3, 25)), rows=rows, max_pages=int(rng.integers(2, 7)), bits=4 if seed % 2 else 16)
    for _ in range(60):
        length = lambda i: len(s.held[i])                                      # noqa: E731
        kind = rng.choice(["begin", "begin", "begin", "fork", "keep", "compact"])
        if kind == "begin":
            new = [int(rng.choice([0, 1, 3, 40, 64, 100])) for _ in range(rows)]
            if sum(new):
                s.begin(new)
        elif kind == "fork":
            s.fork([None if rng.random() < 0.15 else int(rng.integers(rows)) if rng.random() < 0.5 else i for i in range(rows)])
        elif kind == "keep":
            s.keep([int(rng.choice([0, length(i), 10**6, rng.integers(length(i) + 1), rng.integers(length(i) + 1)])) for i in range(rows)])
        else:
            s.compact(rng.random((rows, int(rng.integers(1, 300)))) < rng.choice([0.1, 0.6, 0.97, 1.0]))


def test_rows_that_share_no_page_are_cut_without_a_fork(monkeypatch):
    """A cache knows when rows list no page together any more: rows that only move share none, nor does the last row that is left."""
    s = Server(monkeypatch, n_pages=12, rows=3, max_pages=4)
    s.begin([130, 70, 0])
    s.fork([1, 0, None])
    s.calls.clear()
    s.keep([60, 100, 0])
    assert s.calls == ["release"]
    s.fork([0, 1, 0])
    s.keep([10, 100, 1000])
    assert "fork" in s.calls
    s.keep([0, 0, 1000])
    s.calls.clear()
    s.keep([0, 0, 30])
    assert s.calls == ["release"]
    s.begin([5, 0, 200])
    s.fork([0, None, 2])
    s.keep([0, 0, 130])
    assert s.calls == ["release", "tables", "fork", "move", "release"]
    s.fork([2, 2, 2])                                      # (from now on they do, whoever ends)
    s.keep([1000, 0, 1000])
    s.calls.clear()
    s.keep([100, 0, 1000])
    assert "release" not in s.calls


def test_a_mask_of_no_width(monkeypatch):
    s = Server(monkeypatch, n_pages=8, rows=2, max_pages=4)
    s.begin([150, 3])
    s.compact(np.ones((2, 0)))
    s.begin([1, 1])
    stays = np.ones((2, 100))
    stays[:, 1:60:2] = 0
    s.compact(stays)
    s.compact(np.ones((2, 0)))
    s.keep([5, 1000])
    s.begin([1, 1])
