"""Refusals of the paged cache's calls, through the C ABI: every check comes before anything touches the device, so the addresses here are
numbers.  And the plain oracle's page choice against a hand-worked case."""
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
    p = hk.PagedPool()
    values = dict(k=A, v=A, k_code=A, k_scale=A, page_stride=8 * 64 * 128, head_stride=64 * 128, row_stride=128, n_pages=10, n_kv_heads=8, d=128,
                  dtype=hk.DTYPE_BF16)
    for name, value in {**values, **change}.items():
        setattr(p, name, value)
    return p


def _batch(**change):
    b = hk.PagedBatch()
    values = dict(q_begin=A, kv_len=A, block_table=A, table_stride=5, n_seq=3, table_pages=5, n_tokens=7, max_new=2)
    for name, value in {**values, **change}.items():
        setattr(b, name, value)
    return b


def _attention(pool=None, batch=None, heads=16, q=A, st=None, scale=0.0, out=A, ws=A, size=1 << 40):
    pool, batch = pool or _pool(), batch or _batch()
    return H._lib.heatkv_paged_attention(C.addressof(pool), C.addressof(batch), heads, q, C.byref(st) if st else None, 1, scale, out, None, ws, size, None)


def _sparse(pool=None, batch=None, heads=16, sel=A, n=4):
    pool, batch = pool or _pool(), batch or _batch()
    return H._lib.heatkv_paged_sparse_attention(C.addressof(pool), C.addressof(batch), heads, A, None, sel, n, 0.0, A, None, A, 1 << 40, None)


def _select(pool=None, batch=None, heads=16, sink=1, local=1, n=4, sel=A):
    pool, batch = pool or _pool(), batch or _batch()
    return H._lib.heatkv_paged_select(C.addressof(pool), C.addressof(batch), heads, A, None, sink, local, n, sel, None)


@pytest.mark.parametrize("change,status", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=A + 8), INVALID), (dict(d=96), INVALID), (dict(d=0), INVALID), (dict(dtype=2), INVALID),
    (dict(n_pages=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(row_stride=132), INVALID), (dict(head_stride=64), INVALID),
    (dict(page_stride=0), INVALID), (dict(k_code=None), INVALID), (dict(k_code=A + 4), INVALID), (dict(n_pages=(1 << 25) + 1), LARGE)])
def test_a_pool_that_is_none(change, status):
    assert _attention(pool=_pool(**change)) == status
    pool = _pool(**change)
    assert H._lib.heatkv_paged_store(C.addressof(pool), A, A, 1024, 128, A, 7, None) == status
    size = C.c_uint64()
    assert H._lib.heatkv_paged_workspace_bytes(C.addressof(pool), C.addressof(_batch()), 16, C.byref(size)) == status
    assert _select(pool=pool) == status and _sparse(pool=pool) == status


@pytest.mark.parametrize("change,status", [
    (dict(q_begin=None), INVALID), (dict(kv_len=None), INVALID), (dict(block_table=None), INVALID), (dict(n_seq=0), INVALID), (dict(n_tokens=0), INVALID),
    (dict(max_new=0), INVALID), (dict(table_pages=0), INVALID), (dict(table_stride=4), INVALID), (dict(n_seq=4097), LARGE),
    (dict(table_pages=(1 << 19) + 1, table_stride=1 << 20), LARGE), (dict(n_tokens=1 << 28), LARGE)])
def test_a_batch_that_is_none(change, status):
    assert _attention(batch=_batch(**change)) == status
    assert _select(batch=_batch(**change)) == status and _sparse(batch=_batch(**change)) == status


def test_arguments_of_attention():
    assert _attention(heads=12) == SHAPE and _attention(heads=0) == SHAPE and _attention(heads=8 * 129) == SHAPE
    assert _attention(q=None) == INVALID and _attention(out=None) == INVALID and _attention(q=A + 8) == INVALID and _attention(out=A + 2) == INVALID
    for bad in ((2048, 120, 2048, 128), (2048, 132, 2048, 128), (0, 128, 2048, 128), (2048, 128, 2052, 128), (2048, 128, 2048, 64), (2048, 128, -2048, 128)):
        assert _attention(st=hk.TokenStrides(*bad)) == INVALID, bad
    assert _attention(scale=float("nan")) == INVALID and _attention(scale=float("inf")) == INVALID
    assert H._lib.heatkv_paged_status(None, None) == INVALID


def test_arguments_of_selection():
    assert _select(pool=_pool(k_code=None, k_scale=None)) == INVALID
    assert _select(sink=-1) == INVALID and _select(local=0) == INVALID and _select(n=0) == INVALID and _select(sel=None) == INVALID
    assert _select(sink=2, local=3, n=4) == INVALID and _select(heads=9) == SHAPE
    assert _select(batch=_batch(table_pages=32769, table_stride=32769)) == LARGE
    assert _sparse(sel=None) == INVALID and _sparse(n=0) == INVALID and _sparse(heads=8 * 65) == SHAPE
    assert _sparse(batch=_batch(n_tokens=1 << 20), n=1 << 10) == LARGE


def test_arguments_of_tables_release_and_store():
    ok = [A, A, 3, A, 10, A, A + 64, A, 5, 5, A, A, A, None, 7]
    call = lambda args: H._lib.heatkv_paged_tables(*args, None)                     # noqa: E731
    for at in (0, 1, 3, 5, 6, 7, 10, 11, 12):
        assert call(ok[:at] + [None] + ok[at + 1:]) == INVALID, at
    for at, value, status in ((2, 0, INVALID), (2, 4097, LARGE), (4, 0, INVALID), (4, (1 << 25) + 1, LARGE), (6, A, INVALID), (8, 4, INVALID), (9, 0, INVALID),
                              (14, 0, INVALID)):
        assert call(ok[:at] + [value] + ok[at + 1:]) == status, (at, value)
    assert call(ok) == INVALID and call([A + 64] + ok[1:]) == INVALID                # lengths written where they are read
    ok = [A, A, 3, A, 5, 5, A, 10, A, A + 64]
    call = lambda args: H._lib.heatkv_paged_release(*args, None)                    # noqa: E731
    for at in (0, 1, 3, 6, 8, 9):
        assert call(ok[:at] + [None] + ok[at + 1:]) == INVALID, at
    assert call(ok[:9] + [A]) == INVALID and call(ok[:4] + [4] + ok[5:]) == INVALID and call(ok[:2] + [5000] + ok[3:]) == LARGE
    pool = _pool()
    store = lambda k=A, v=A, tok=1024, head=128, slots=A, n=7: H._lib.heatkv_paged_store(C.addressof(pool), k, v, tok, head, slots, n, None)    # noqa: E731
    assert store(k=None) == store(v=None) == store(slots=None) == store(n=0) == store(k=A + 4) == store(tok=1020) == store(head=-128) == INVALID


def test_the_binding_says_what_is_wrong():
    k = torch.zeros(4, 2, 64, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="float32"):
        hk.PagedPool.make(k.float(), k.float())
    with pytest.raises(ValueError, match="equal strides"):
        hk.PagedPool.make(k, torch.zeros(4, 64, 2, 64, dtype=torch.bfloat16).transpose(1, 2))
    with pytest.raises(ValueError, match="k_code"):
        hk.PagedPool.make(k, k.clone(), torch.zeros(4, 2, 63, dtype=torch.int8), torch.zeros(4, 2))
    with pytest.raises(ValueError, match="expected"):
        hk.PagedPool.make(k[:, :, :32], k[:, :, :32])
    i = lambda *n: torch.zeros(*n, dtype=torch.int32)                                # noqa: E731
    with pytest.raises(ValueError, match="q_begin"):
        hk.PagedBatch.make(i(3), i(3), i(3, 5), 7, 2)
    pool, batch = hk.PagedPool.make(k, k.clone()), hk.PagedBatch.make(i(4), i(3), i(3, 5), 7, 2)
    q, ws = torch.zeros(7, 4, 64, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.uint8)
    for bad, what in ((dict(q=q[:6]), "q"), (dict(q=q.half()), "q"), (dict(out=q[:, :2]), "out"), (dict(lse=torch.zeros(7, 2)), "lse")):
        args = {**dict(q=q, out=q.clone(), lse=None), **bad}
        with pytest.raises(ValueError, match=what):
            hk.heatkv_paged_attention(pool, batch, args["q"], args["out"], args["lse"], ws)
    with pytest.raises(ValueError, match="sel"):
        hk.heatkv_paged_sparse_attention(pool, batch, q, i(7, 4, 3), q.clone(), None, ws)
    with pytest.raises(ValueError, match="slot_map"):
        hk.heatkv_paged_store(pool, q[:, :2], q[:, :2], i(7).long())
    with pytest.raises(ValueError, match="v_new"):
        hk.heatkv_paged_store(pool, q[:, :2], q, i(7))
    with pytest.raises(ValueError, match="state"):
        hk.heatkv_paged_tables(i(2), i(2), i(9), i(3), i(4), i(2, 5), i(3), i(2), i(4))
    with pytest.raises(ValueError, match="block_table"):
        hk.heatkv_paged_release(i(2), i(2), i(3, 5), i(9), i(4), i(4))


def test_host_memory_never_reaches_a_kernel():
    i = lambda *n: torch.zeros(*n, dtype=torch.int32)                                # noqa: E731
    k, q = torch.zeros(4, 2, 64, 64, dtype=torch.bfloat16), torch.zeros(7, 4, 64, dtype=torch.bfloat16)
    pool = hk.PagedPool.make(k, k.clone(), torch.zeros(4, 2, 64, dtype=torch.int8), torch.zeros(4, 2))
    batch, ws = hk.PagedBatch.make(i(4), i(3), i(3, 5), 7, 2), torch.zeros(1 << 20, dtype=torch.uint8)
    for call in (lambda: hk.heatkv_paged_tables(i(2), i(2), i(9), i(4), i(4), i(2, 5), i(3), i(2), i(4)),
                 lambda: hk.heatkv_paged_release(i(2), i(2), i(2, 5), i(9), i(4), i(4)),
                 lambda: hk.heatkv_paged_store(pool, q[:, :2], q[:, :2], i(7)),
                 lambda: hk.heatkv_paged_attention(pool, batch, q, q.clone(), None, ws),
                 lambda: hk.heatkv_paged_select(pool, batch, q, i(7, 2, 4), 1, 1),
                 lambda: hk.heatkv_paged_sparse_attention(pool, batch, q, i(7, 2, 4), q.clone(), None, ws),
                 lambda: hk.heatkv_paged_status(ws)):
        with pytest.raises(ValueError, match="not on the current CUDA device"):
            call()
    with pytest.raises(ValueError, match="contiguous"):
        hk.heatkv_paged_attention(pool, batch, q, q.clone(), None, ws[::2])


def test_page_choice_by_hand():
    """Two heads of one group, d = 2: sums 3 and -1, codes 127 and -42."""
    q = np.array([[1.0, 0.0], [2.0, -1.0]], dtype=np.float32)
    codes = np.array([[1, 0], [2, 0], [0, -3], [2, 0], [0, 5], [9, 9]], dtype=np.int64)       # 127, 254, 126, 254, -210, (own page)
    scales = np.array([1, 1, 4, 1, 1, 1], dtype=np.float32)                                   # .., 504, ..
    assert P.select(q, codes, scales, 5 * 64 + 7, 0, 1, 2) == [2, 5]
    assert P.select(q, codes, scales, 5 * 64 + 7, 0, 1, 3) == [1, 2, 5]                       # 1 and 3 are equal: the lower page
    assert P.select(q, codes, scales, 5 * 64 + 7, 1, 2, 4) == [0, 2, 4, 5]
    assert P.select(q, codes, scales, 63, 0, 1, 4) == [0]
    c, s = P.summary(np.tile(np.array([[1.0, -0.5, 0.0]], dtype=np.float32), (64, 1)))
    assert c.tolist() == [127, -64, 0] and s == np.float32(1) / np.float32(127)


def test_the_cache_refuses_selected_pages_that_see_what_is_behind():
    """Attention over selected pages is causal; asked for without, it is refused and nothing is stored."""
    from paper_2605_14877_b200.paged import PagedCache
    cache = PagedCache(1, 4, 2, 64, n_pages=4, rows=1, max_pages=4, summaries=True, device="cpu")
    q, kv = torch.ones(3, 4, 64, dtype=torch.bfloat16), torch.ones(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="causal"):
        cache.attend(0, None, q, kv, kv, torch.empty_like(q), causal=False, pages=2)
    assert (cache.pools[0].tensors[0] == 0).all()


def test_the_cache_refuses_numbers_of_tokens_that_are_none():
    """Negative numbers would shorten the step's tensors, or a row's length, silently."""
    from paper_2605_14877_b200.paged import PagedCache
    cache = PagedCache(1, 4, 2, 64, n_pages=4, rows=2, max_pages=4, device="cpu")
    for bad in ([3, -1], [0, 0], [1], [1, 2, 3]):
        with pytest.raises(ValueError, match="new: expected 2 numbers"):
            cache.begin(bad)
    for bad in ([3, -1], [1], [1, 2, 3]):
        with pytest.raises(ValueError, match="lengths: expected 2 numbers"):
            cache.keep(bad)
    assert cache.at_most == [0, 0] and cache.lengths.tolist() == [0, 0]


def test_arguments_of_the_waits_self_test():
    assert H._lib.heatkv_paged_selftest_wait_expiry(None, None) == INVALID and H._lib.heatkv_paged_selftest_wait_expiry(A + 16, None) == INVALID
    with pytest.raises(ValueError, match="256"):
        hk.heatkv_paged_selftest_wait_expiry(torch.zeros(255, dtype=torch.uint8))
    with pytest.raises(ValueError, match="not on the current CUDA device"):
        hk.heatkv_paged_selftest_wait_expiry(torch.zeros(256, dtype=torch.uint8))
