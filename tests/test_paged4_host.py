"""Refusals of the calls of the 4-bit cache and of those that rearrange rows, through the C ABI: every check comes before anything touches the device, so
the addresses here are numbers.  And the plain oracle's format and rows against hand-worked cases."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2605_14877_b200 as hk
from oracle import paged_oracle as P
from paper_2605_14877_b200 import heatkv as H

INVALID, SHAPE, LARGE = -1, -2, -10
A = 1 << 20                                                # an aligned address that nothing follows


def _pool(**change):
    p = hk.PagedPool4()
    for name, value in {**dict(blocks=A, page_stride=8 * 9216, head_stride=9216, n_pages=10, n_kv_heads=8, d=128, dtype=hk.DTYPE_BF16), **change}.items():
        setattr(p, name, value)
    return p


def _batch(**change):
    b = hk.PagedBatch()
    for name, value in {**dict(q_begin=A, kv_len=A, block_table=A, table_stride=5, n_seq=3, table_pages=5, n_tokens=7, max_new=2), **change}.items():
        setattr(b, name, value)
    return b


def _attention(pool=None, batch=None, heads=16, q=A, st=None, scale=0.0, out=A, ws=A, size=1 << 40):
    pool, batch = pool or _pool(), batch or _batch()
    return H._lib.heatkv_paged4_attention(C.addressof(pool), C.addressof(batch), heads, q, C.byref(st) if st else None, 1, scale, out, None, ws, size, None)


@pytest.mark.parametrize("change,status", [
    (dict(blocks=None), INVALID), (dict(blocks=A + 8), INVALID), (dict(d=96), INVALID), (dict(dtype=2), INVALID), (dict(n_pages=0), INVALID),
    (dict(n_kv_heads=0), INVALID), (dict(head_stride=9208), INVALID), (dict(head_stride=9200), INVALID), (dict(page_stride=4608), INVALID),
    (dict(k_exp=65), INVALID), (dict(v_exp=-65), INVALID), (dict(n_pages=(1 << 25) + 1), LARGE), (dict(n_kv_heads=4097), LARGE)])
def test_a_pool_that_is_none(change, status):
    pool = _pool(**change)
    at, size = C.addressof(pool), C.c_uint64()
    assert _attention(pool=pool) == status
    assert H._lib.heatkv_paged4_store(at, A, A, 1024, 128, A, 7, None) == status
    assert H._lib.heatkv_paged4_load(at, A, 7, A, A + 4096, 1024, 128, None) == status
    assert H._lib.heatkv_paged4_move(at, A, A, 7, None) == status
    assert H._lib.heatkv_paged4_workspace_bytes(at, C.addressof(_batch()), 16, C.byref(size)) == status


def test_arguments_of_attention():
    assert _attention(heads=12) == SHAPE and _attention(heads=8 * 129) == SHAPE
    assert _attention(q=None) == INVALID and _attention(out=None) == INVALID and _attention(q=A + 8) == INVALID and _attention(out=A + 2) == INVALID
    assert _attention(scale=float("nan")) == INVALID and _attention(st=hk.TokenStrides(2048, 132, 2048, 128)) == INVALID
    assert _attention(batch=_batch(n_seq=4097)) == LARGE and _attention(batch=_batch(max_new=0)) == INVALID


def test_arguments_of_rows():
    at = C.addressof(_pool())
    pool = _pool()
    at = C.addressof(pool)
    store = lambda k=A, v=A, tok=1024, head=128, slots=A, n=7: H._lib.heatkv_paged4_store(at, k, v, tok, head, slots, n, None)    # noqa: E731
    assert store(k=None) == store(v=None) == store(slots=None) == store(n=0) == store(k=A + 4) == store(tok=1020) == store(head=-128) == INVALID
    load = lambda k=A, v=2 * A, tok=1024, head=128, slots=A, n=7: H._lib.heatkv_paged4_load(at, slots, n, k, v, tok, head, None)  # noqa: E731
    assert load(k=None) == load(v=A) == load(slots=None) == load(n=0) == load(tok=0) == load(head=64) == load(v=A + 8) == INVALID
    move = lambda a=A, b=A, n=7: H._lib.heatkv_paged4_move(at, a, b, n, None)                                                     # noqa: E731
    assert move(a=None) == move(b=None) == move(n=0) == INVALID


def test_scales_of_logits_that_32_bits_do_not_hold():
    for k_exp, scale in ((-64, 1e-20), (64, 1e10), (0, 1e-30), (0, 1e25)):
        assert _attention(_pool(k_exp=k_exp), scale=scale) == INVALID


def test_arguments_of_fork_and_compact():
    size = C.c_uint64()
    assert H._lib.heatkv_paged_rows_workspace_bytes(3, 5, 10, C.byref(size)) == 0 and size.value % 4 == 0
    for bad, status in (((0, 5, 10), INVALID), ((3, 0, 10), INVALID), ((3, 5, 0), INVALID), ((4097, 5, 10), LARGE), ((3, 5, (1 << 25) + 1), LARGE)):
        assert H._lib.heatkv_paged_rows_workspace_bytes(*bad, C.byref(size)) == status
    assert H._lib.heatkv_paged_rows_workspace_bytes(3, 5, 10, None) == INVALID
    # parents, keep, lengths, n, table, stride, pages, free, n_pages, state, lengths_out, table_out, stride, state_out, from, to, workspace, bytes
    ok = [A, A, A, 3, A, 5, 5, A, 10, A, 2 * A, 2 * A, 5, 2 * A, A, 2 * A, A, 1 << 40]
    fork = lambda args: H._lib.heatkv_paged_fork(*args, None)                       # noqa: E731
    for i in (0, 2, 4, 7, 9, 10, 11, 13, 14, 15, 16):
        assert fork(ok[:i] + [None] + ok[i + 1:]) == INVALID, i
    for i, value, status in ((3, 0, INVALID), (3, 4097, LARGE), (5, 4, INVALID), (6, 0, INVALID), (8, 0, INVALID), (8, (1 << 25) + 1, LARGE), (10, A, INVALID),
                             (11, A, INVALID), (12, 4, INVALID), (13, A, INVALID), (15, A, INVALID), (16, A + 8, INVALID), (17, 1000, LARGE)):
        assert fork(ok[:i] + [value] + ok[i + 1:]) == status, (i, value)
    # stays, stride, width, then as above up to the moves, their number, workspace, bytes
    ok = [A, 300, 300] + ok[2:16] + [900, A, 1 << 40]
    compact = lambda args: H._lib.heatkv_paged_compact(*args, None)                 # noqa: E731
    for i in (0, 3, 5, 8, 10, 11, 12, 14, 15, 16, 18):
        assert compact(ok[:i] + [None] + ok[i + 1:]) == INVALID, i
    for i, value, status in ((1, 299, INVALID), (2, -1, INVALID), (4, 0, INVALID), (17, 0, INVALID), (19, 1000, LARGE)):
        assert compact(ok[:i] + [value] + ok[i + 1:]) == status, (i, value)


def test_the_binding_says_what_is_wrong():
    blocks = torch.zeros(4, 2, 64 * 72, dtype=torch.uint8)
    pool = hk.PagedPool4.make(blocks, 64, torch.float16)
    with pytest.raises(ValueError, match="blocks"):
        hk.PagedPool4.make(blocks, 128, torch.float16)
    with pytest.raises(ValueError, match="dtype"):
        hk.PagedPool4.make(blocks, 64, torch.float32)
    i = lambda *n: torch.zeros(*n, dtype=torch.int32)                                # noqa: E731
    rows = torch.zeros(3, 2, 64, dtype=torch.float16)
    with pytest.raises(ValueError, match="PagedPool4"):
        hk.heatkv_paged4_store(hk.PagedPool.make(torch.zeros(4, 2, 64, 64).bfloat16(), torch.zeros(4, 2, 64, 64).bfloat16()), rows, rows, i(3))
    with pytest.raises(ValueError, match="expected a PagedPool, got PagedPool4"):
        hk.heatkv_paged_move(pool, i(3), i(3))
    with pytest.raises(ValueError, match="k_new"):
        hk.heatkv_paged4_store(pool, rows.bfloat16(), rows, i(3))
    with pytest.raises(ValueError, match="k_out, v_out"):
        hk.heatkv_paged4_load(pool, i(3), rows, rows.transpose(0, 1).contiguous().transpose(0, 1))
    with pytest.raises(ValueError, match="current CUDA device"):
        hk.heatkv_paged4_move(pool, i(3), i(3))
    new = [i(3), i(3, 5), i(4), i(128), i(128), torch.zeros(1 << 20, dtype=torch.uint8)]
    with pytest.raises(ValueError, match="move_from"):
        hk.heatkv_paged_fork(i(3), None, i(3), i(3, 5), i(10), i(4), *new)
    with pytest.raises(ValueError, match="table_out"):
        hk.heatkv_paged_fork(i(3), None, i(3), i(3, 4), i(10), i(4), *new)
    with pytest.raises(ValueError, match="stays"):
        hk.heatkv_paged_compact(torch.zeros(3, 7), i(3), i(3, 5), i(10), i(4), *new)
    # a pool of 4 bits is none for the calls over 16, nor the other way round
    with pytest.raises(AttributeError):
        hk.heatkv_paged_store(pool, rows, rows, i(3))


def test_the_cache_refuses_what_it_cannot_do():
    from paper_2605_14877_b200.paged import PagedCache
    make = lambda **more: PagedCache(1, 4, 2, 64, n_pages=4, rows=2, max_pages=4, device="cpu", **more)      # noqa: E731
    for bad in (dict(bits=8), dict(bits=16, k_exp=1), dict(bits=4, summaries=True)):
        with pytest.raises(ValueError):
            make(**bad)
    cache = make(bits=4)
    for bad in ([0], [0, 2], [0, -1]):
        with pytest.raises(ValueError, match="parents"):
            cache.fork(bad)
    for bad in (torch.ones(2, 5), torch.ones(3, 5, dtype=torch.bool), torch.ones(2, dtype=torch.bool)):
        with pytest.raises(ValueError, match="stays"):
            cache.compact(bad)


def test_the_oracles_numbers():
    numbers = P._e4m3()
    assert numbers[0] == 0 and numbers[1] == 2.0**-9 and numbers[8] == 2.0**-6 and numbers[126] == 448 and (np.diff(numbers) > 0).all()
    x = np.zeros((1, 16))
    x[0, :6] = [7, 0.5, 1.5, -2.5, 6.5, -7]                # scale 1: halves go to the even code
    code, byte = P.quantise(x)
    assert numbers[byte[0, 0]] == 1 and code[0, :6].tolist() == [7, 0, 2, -2, 6, -7]
    assert P.quantise(np.full((1, 16), 5000.0))[0].max() == 7 and P.quantise(np.full((1, 16), 1e-5))[1][0, 0] == 0
    assert np.array_equal(P.quantise(x * 32, 5)[0], code)
    page = np.arange(64 * 64).reshape(64, 64) % 15 - 7
    data = P.block((page, np.arange(256).reshape(64, 4) % 127), (page[::-1], np.zeros((64, 4), int)))
    assert len(data) == 64 * 72 and data[0] == (page[0, 0] + 8) | (page[0, 2] + 8) << 4 and data[2] == (page[0, 1] + 8) | (page[0, 3] + 8) << 4
    (a, s), (b, _) = P.unblock(data, 64)
    assert np.array_equal(a, page) and np.array_equal(b, page[::-1]) and s[1, 2] == 6


def test_the_oracles_rows():
    table = np.array([[5, 7, -1], [-1, -1, -1], [-1, -1, -1]])
    lengths, new, source, target, taken, cut, back = P.fork([0, 0, -1], [99, 70, 9], [100, 0, 0], table, [2, 3])
    assert lengths.tolist() == [99, 70, 0] and new.tolist() == [[5, 7, -1], [5, 2, -1], [-1, -1, -1]] and (taken, cut, back) == (1, 0, [])
    assert source[64:71].tolist() == [448, 449, 450, 451, 452, 453, -1] and target[64:70].tolist() == [128, 129, 130, 131, 132, 133]
    stays = np.ones((3, 100), dtype=bool)
    stays[0, [70, 80]] = False
    lengths, new, source, target, taken, refused, back, done = P.compact(stays, [100, 0, 0], table, [2, 3], 40)
    assert lengths.tolist() == [98, 0, 0] and new[0].tolist() == [5, 2, -1] and (taken, refused, back, done) == (1, 0, [7], 34)
    assert source[:8].tolist() == [448, 449, 450, 451, 452, 453, 455, 456] and target[33] == 2 * 64 + 33 and source[34] == -1
