"""Edges of the paged cache in 4 bits and of rows between steps that the other tests do not reach."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as P

pytestmark = pytest.mark.gpu
PAGE = 64
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


def _np(x):
    return x.detach().double().cpu().numpy()


@pytest.fixture(scope="module")
def hk():
    import paper_2605_14877_b200 as hk
    return hk


def _cache(**more):
    from paper_2605_14877_b200.paged import PagedCache
    return PagedCache(1, 2, 2, 64, **more)


def _begin(cache, new):
    """A step whose tokens are stored; the positions of its tokens, row by row."""
    step, n = cache.begin(new), sum(new)
    x = torch.zeros(n, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache.attend(0, step, x, x, x, torch.empty_like(x))
    at = np.concatenate([[0], np.cumsum(new)])
    return [step.positions.tolist()[a:b] for a, b in zip(at, at[1:])]


@pytest.mark.parametrize("bits", [4, 16])
def test_a_row_that_lost_its_tokens_to_a_fork_begins_anew(hk, bits):
    """No page is free: a copy of a row of less than a page has nothing, and whoever comes next in its place starts at position 0."""
    cache = _cache(n_pages=4, rows=3, max_pages=4, bits=bits)
    _begin(cache, [128, 0, 40])
    stays = torch.ones(3, 40, dtype=torch.bool, device="cuda")
    stays[2, 5:25] = False
    cache.compact(stays)
    _begin(cache, [64, 0, 0])
    assert cache.lengths.tolist() == [192, 0, 20] and cache.state.tolist()[1] == 0
    cache.fork([0, 2, 2])
    assert cache.lengths.tolist() == [192, 0, 20] and cache.state.tolist()[2] == 1
    cache.fork([None, 1, 2])
    assert _begin(cache, [0, 5, 3]) == [[], [0, 1, 2, 3, 4], [40, 41, 42]]


def test_a_cut_into_a_shared_page_takes_a_page_that_the_same_call_frees(hk):
    """Row 0 is cut to a place inside a page that row 1 has whole, no page is free before row 2 ends in the same call: its tokens, too, are there."""
    cache = _cache(n_pages=3, rows=3, max_pages=4, bits=16)
    k, v = (torch.arange(138, device="cuda").remainder(101)[:, None, None].expand(138, 2, 64).bfloat16().contiguous() for _ in "kv")
    cache.attend(0, cache.begin([128, 0, 10]), k, k, v, torch.empty_like(k))
    cache.fork([0, 0, 2])
    cache.keep([100, 128, 0])
    assert cache.lengths.tolist() == [100, 128, 0] and cache.state.tolist()[1:3] == [0, 0]
    pages = cache.table[:, :2].long()
    assert len({*pages[0].tolist(), int(pages[1, 1])}) == 3 and pages[0, 0] == pages[1, 0]
    for i, n in ((0, 100), (1, 128)):
        for x, new in zip(cache.pools[0].tensors, (k, v)):
            assert torch.equal(x[pages[i]].transpose(1, 2).reshape(128, 2, 64)[:n], new[:n])


@pytest.mark.parametrize("bits", [4, 16])
def test_positions_of_a_row_that_lost_tokens_among_which_some_had_left(hk, bits):
    """A fork that has no page for a copy cuts a row where nobody asked it to: the next token takes the position of the first one that was lost."""
    cache = _cache(n_pages=4, rows=2, max_pages=4, bits=bits)
    _begin(cache, [150, 0])
    stays = torch.ones(2, 150, dtype=torch.bool, device="cuda")
    stays[0, 140:145] = False
    cache.compact(stays)
    _begin(cache, [0, 64])
    cache.fork([0, 0])
    assert cache.lengths.tolist() == [145, 128]
    cache.fork([None, 1])
    assert _begin(cache, [0, 2]) == [[], [128, 129]]


@pytest.mark.parametrize("bits", [4, 16])
def test_a_mask_of_no_width(hk, bits):
    """Tokens past a mask's width stay: all of them, of a mask that has none."""
    cache = _cache(n_pages=8, rows=2, max_pages=4, bits=bits)
    _begin(cache, [150, 3])
    table = cache.table[:, :3].clone()
    for stays in (torch.ones(2, 0, dtype=torch.bool, device="cuda"), torch.zeros(2, 9, dtype=torch.bool, device="cuda")[:, :0]):
        cache.compact(stays)
        assert cache.lengths.tolist() == [150, 3] and cache.state.tolist()[1:] == [4, 0, 0]
        assert torch.equal(cache.table[0, :3], table[0]) and cache.table[1, 0] == table[1, 0]
    assert _begin(cache, [1, 1]) == [[150], [3]]
