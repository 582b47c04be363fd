"""The paged cache in 4 bits, and rows of block tables between steps, against plain numpy: codes, scales, tables and moves bit for bit, attention in 64 bits.

Tolerances of attention.  With u = 2^-8 (bf16) or 2^-11 (fp16): the output is rounded once (u |out|), the probabilities once, to 16 bits of either
type (u sum p |v|, and in fp16 at most 2^-25 of the largest value each where they are subnormal); what is multiplied are the values that the codes stand for,
exactly.  A query row may be scaled to fp16's range: numbers 2^29 times smaller than its largest lose bits, 2^-30 of the largest each, which is inside the
2^-24 of the logits' sums.  Those are sums of d products in 32 bits and one scaling, off by at most (d + 8) 2^-24 of sum |q k| scale, which moves a
probability by twice that and the logarithm of the sum by once that; exponentials and sums of 32 bits add 2^-18."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as P

pytestmark = pytest.mark.gpu
PAGE = 64
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def hk():
    import paper_2605_14877_b200 as hk
    return hk


def _i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


def _np(x):
    return x.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------------------------ store and load

def _garbage(g, n_pages, Hkv, d):
    """Blocks whose every byte may be anything, scales that are no numbers among them."""
    return torch.randint(0, 256, (n_pages, Hkv, PAGE * (d + d // 8)), dtype=torch.uint8, generator=g, device="cuda")


def _hard_rows(g, T, Hkv, d, dt):
    """Rows of every size: zeros, numbers so small that scales are subnormal or zero, ties between codes, numbers past the largest scale."""
    x = torch.empty(T, Hkv, d, device="cuda").normal_(generator=g)
    size = torch.tensor([0.0, 2.0**-12, 2.0**-9, 2.0**-7, 0.05, 1.0, 3.0, 40.0, 900.0, 4000.0, 30000.0], device="cuda")
    x *= size[torch.randint(0, len(size), (T, Hkv, d // 16), generator=g, device="cuda")].repeat_interleave(16, -1)
    x[T // 2:, :, ::16] = 7.0                              # scale 1: halves are ties
    x[T // 2:, :, 1::2] = (x[T // 2:, :, 1::2].clamp(-13, 13) * 2).round() / 2
    return x.to(dt)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,Hkv,exps", [(128, 8, (0, 0)), (128, 1, (-3, 5)), (64, 5, (0, 0)), (64, 16, (7, -9))])
def test_store_and_load(hk, dtype, d, Hkv, exps):
    g = torch.Generator("cuda").manual_seed(d + Hkv)
    n_pages, T = 9, 150
    blocks = _garbage(g, n_pages, Hkv, d)
    before = blocks.cpu().numpy()
    pool = hk.PagedPool4.make(blocks, d, DTYPES[dtype], *exps)
    slots = torch.randperm(n_pages * PAGE, generator=g, device="cuda")[:T].int()
    slots[5], slots[9], slots[77] = -1, n_pages * PAGE, 2**31 - 1
    qkv = torch.stack([_hard_rows(g, T, Hkv, d, DTYPES[dtype]) for _ in range(3)], 1)
    hk.heatkv_paged4_store(pool, qkv[:, 1], qkv[:, 2], slots)
    after = blocks.cpu().numpy()
    got, was = P.unblock(after, d), P.unblock(before, d)
    wide = torch.full((T, Hkv + 1, 2, d), 5.0, dtype=DTYPES[dtype], device="cuda")
    back = wide[:, :Hkv, 0], wide[:, :Hkv, 1]
    hk.heatkv_paged4_load(pool, slots, *back)
    untouched = np.ones((n_pages, PAGE), dtype=bool)
    for part in range(2):
        code, byte = P.quantise(_np(qkv[:, 1 + part]), exps[part])
        want = P.values(code, byte, exps[part])
        for t, s in enumerate(slots.tolist()):
            if not 0 <= s < n_pages * PAGE:
                want[t] = 0
                continue
            untouched[s // PAGE, s % PAGE] = False
            assert np.array_equal(got[part][0][s // PAGE, :, s % PAGE], code[t]) and np.array_equal(got[part][1][s // PAGE, :, s % PAGE], byte[t]), (part, t)
        assert np.array_equal(_np(back[part]), _np(torch.from_numpy(want).to(DTYPES[dtype])))
    for x, y in zip(got, was):
        for i in range(2):
            assert np.array_equal(x[i].swapaxes(1, 2)[untouched], y[i].swapaxes(1, 2)[untouched])
    assert (wide[:, Hkv] == 5.0).all()


def test_blocks_are_laid_out_as_documented(hk):
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.empty(2, PAGE, 1, 64, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    wide = torch.zeros(3, 2, PAGE * 72 + 16, dtype=torch.uint8, device="cuda")
    pool = hk.PagedPool4.make(wide[:, 1:, : PAGE * 72], 64, torch.bfloat16)
    hk.heatkv_paged4_store(pool, x[0], x[1], _i32(range(PAGE, 2 * PAGE)))
    want = P.block(*(P.quantise(_np(y[:, 0])) for y in x))
    assert np.array_equal(wide[1, 1, : PAGE * 72].cpu().numpy(), want)
    assert not wide[0].any() and not wide[2].any() and not wide[1, 0].any() and not wide[:, :, PAGE * 72:].any()


# ------------------------------------------------------------------------------------------------ attention

LENS = {                                                   # (new tokens, tokens in all) per request
    "one_key": [(1, 1)],
    "one_of_each": [(1, 2), (1, 63), (1, 64), (1, 65), (1, 128), (1, 129)],
    "no_keys": [(1, 0), (1, 70), (0, 0), (2, 0), (0, 100)],
    "decode": [(1, 1000), (1, 17), (1, 3), (1, 517), (1, 64)],
    "long_one": [(1, 20011)],
    "many": [(1, 1 + (i * 97) % 700) for i in range(150)],
    "drafts": [(5, 130), (1, 40), (3, 64), (5, 5), (4, 66)],
    "more_new_than_tokens": [(4, 2), (3, 0), (2, 65)],
    "short_prompts": [(1, 1), (33, 33), (64, 64), (65, 65), (127, 127)],
    "prompt": [(300, 300)],
    "chunk_behind": [(130, 700), (257, 260), (128, 128 * 3)],
    "mixed": [(1, 900), (200, 450), (1, 5), (70, 1000)],
}


def _batch(hk, rng, lens, n_pages, spare=0):
    """lens: (new, kv) per request; pages in random order.  Returns (batch, table, q_begin)."""
    width = max(max(-(-kv // PAGE) for _, kv in lens), 1) + 1
    order = rng.permutation(n_pages)
    table = np.full((len(lens), width), -1)
    at = 0
    for i, (_, kv) in enumerate(lens):
        h = -(-kv // PAGE)
        table[i, :h] = order[at: at + h]
        at += h
    q_begin = np.concatenate([[0], np.cumsum([n for n, _ in lens])])
    b = hk.PagedBatch.make(_i32(q_begin), _i32([kv for _, kv in lens]), _i32(table), int(q_begin[-1]) + spare, max(max(n for n, _ in lens), 1))
    return b, table, q_begin


def _filled(hk, g, rng, lens, Hkv, d, dt, exps=(0, 0), spare_pages=2, size=1.0, **more):
    """A pool whose requests' rows are random and every other byte anything; K and V as 64-bit numbers [pages, heads, 64, d]."""
    n_pages = sum(-(-kv // PAGE) for _, kv in lens) + spare_pages
    blocks = _garbage(g, n_pages, Hkv, d)
    pool = hk.PagedPool4.make(blocks, d, dt, *exps)
    b, table, q_begin = _batch(hk, rng, lens, n_pages, **more)
    slots = np.concatenate([np.zeros(0, int)] + [table[i][np.arange(kv) // PAGE] * PAGE + np.arange(kv) % PAGE for i, (_, kv) in enumerate(lens)])
    if len(slots):
        k, v = (torch.empty(len(slots), Hkv, d, device="cuda").normal_(generator=g).mul_(size).to(dt) for _ in "kv")
        hk.heatkv_paged4_store(pool, k, v, _i32(slots))
    known = np.zeros((n_pages, PAGE), dtype=bool)
    known[slots // PAGE, slots % PAGE] = True
    kv = [np.where(known[:, None, :, None], P.values(c, np.minimum(s, 126), e), np.nan) for (c, s), e in zip(P.unblock(blocks.cpu().numpy(), d), exps)]
    return pool, b, table, q_begin, kv


def _check(out, lse, q, kv, lens, table, q_begin, Hkv, causal, scale, dtype):
    G, d = q.shape[1] // Hkv, q.shape[2]
    u = 2.0**-8 if dtype == "bf16" else 2.0**-11
    out, q = _np(out), _np(q)
    lse = None if lse is None else _np(lse)
    for i, (n, length) in enumerate(lens):
        pages = table[i, : -(-length // PAGE)]
        for h in range(Hkv):
            keys, values = (x[pages, h].reshape(-1, d) for x in kv)
            rows, at, j = slice(q_begin[i], q_begin[i] + n), np.arange(length - n, length), np.arange(len(keys))
            seen = np.broadcast_to(j < length, (n, len(keys)))
            if causal:
                seen = seen & (j <= at[:, None])
            big = np.abs(np.where(np.isfinite(values), values, 0.0)).max(initial=0.0)
            for g in range(G):
                o, l, pv, reach = P.attention(q[rows, h * G + g], keys, values, seen, scale)
                off = (d + 8) * 2.0**-24 * reach + 2.0**-18
                tol = u * np.abs(o) + (u + 2 * off)[:, None] * pv + len(keys) * 2.0**-25 * big + 1e-30
                got = out[rows, h * G + g]
                assert np.isfinite(got).all(), (i, h, g)
                assert (np.abs(got - o) <= tol).all(), (i, h, g, float((np.abs(got - o) / tol).max()))
                if lse is not None:
                    gl = lse[rows, h * G + g]
                    assert np.array_equal(np.isinf(gl), np.isinf(l)), (i, h, g)
                    fin = np.isfinite(l)
                    assert (np.abs(gl[fin] - l[fin]) <= (off + 2.0**-22 * np.abs(l))[fin]).all(), (i, h, g)


def _workspace(hk, pool, b, H):
    return torch.zeros(hk.heatkv_paged4_workspace_bytes(pool, b, H), dtype=torch.uint8, device="cuda")


def _attend(hk, pool, b, q, lens, table, q_begin, kv, Hkv, causal=True, scale=0.0, dtype="bf16"):
    T, H, d = q.shape
    out, lse = torch.full_like(q, 7.0), torch.full((T, H), 7.0, device="cuda")
    ws = _workspace(hk, pool, b, H)
    hk.heatkv_paged4_attention(pool, b, q, out, lse, ws, causal=causal, sm_scale=scale)
    assert hk.heatkv_paged_status(ws) == 0
    _check(out, lse, q, kv, lens, table, q_begin, Hkv, causal, scale or 1 / math.sqrt(d), dtype)
    end = q_begin[-1]
    assert (out[end:] == 7.0).all() and (lse[end:] == 7.0).all()
    again = torch.zeros_like(out)
    hk.heatkv_paged4_attention(pool, b, q, again, None, ws, causal=causal, sm_scale=scale)
    assert torch.equal(again[:end], out[:end])             # and the same bits again, without the logarithms
    return out, lse


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("H,Hkv,d,dtype", [(16, 16, 128, "bf16"), (32, 8, 128, "fp16"), (28, 4, 64, "bf16"), (5, 5, 64, "fp16"), (8, 1, 128, "bf16")])
@pytest.mark.parametrize("name", LENS)
def test_attention(hk, name, H, Hkv, d, dtype, causal):
    lens = LENS[name]
    rng, g = np.random.default_rng(len(name) + H), torch.Generator("cuda").manual_seed(len(name) + H)
    pool, b, table, q_begin, kv = _filled(hk, g, rng, lens, Hkv, d, DTYPES[dtype], spare=3)
    q = torch.empty(b.n_tokens, H, d, dtype=DTYPES[dtype], device="cuda").normal_(generator=g)
    _attend(hk, pool, b, q, lens, table, q_begin, kv, Hkv, causal, dtype=dtype)


@pytest.mark.parametrize("n,d", [(341, 128), (400, 64), (3300, 64), (4096, 128)])
def test_attention_of_many_requests(hk, n, d):
    """So many that their lengths take the place of pages under way."""
    lens = [(1 + i % 2 * (i % 3 == 0), (i * 37) % 150) for i in range(n)]
    rng, g = np.random.default_rng(n), torch.Generator("cuda").manual_seed(n)
    pool, b, table, q_begin, kv = _filled(hk, g, rng, lens, 1, d, torch.bfloat16)
    q = torch.empty(b.n_tokens, 2, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    _attend(hk, pool, b, q, lens, table, q_begin, kv, 1)


@pytest.mark.parametrize("lens,Hkv", [([(1, 3000 + 500 * (i % 5)) for i in range(40)], 8), ([(1, 9000), (1, 64 * 100), (1, 7)], 2)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_of_much(hk, lens, Hkv, dtype):
    """Units cut by many borders."""
    rng, g = np.random.default_rng(Hkv), torch.Generator("cuda").manual_seed(Hkv)
    pool, b, table, q_begin, kv = _filled(hk, g, rng, lens, Hkv, 128, DTYPES[dtype])
    q = torch.empty(b.n_tokens, 3 * Hkv, 128, dtype=DTYPES[dtype], device="cuda").normal_(generator=g)
    _attend(hk, pool, b, q, lens, table, q_begin, kv, Hkv, dtype=dtype)


@pytest.mark.parametrize("G", [1, 3, 8, 9, 16, 17, 32, 33, 64, 128])
def test_attention_any_group(hk, G):
    """Query heads per kv head, from one to 128."""
    lens = [(1, 200), (2, 64), (1, 1)]
    rng, g = np.random.default_rng(G), torch.Generator("cuda").manual_seed(G)
    pool, b, table, q_begin, kv = _filled(hk, g, rng, lens, 2, 128, torch.bfloat16)
    q = torch.empty(b.n_tokens, 2 * G, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    _attend(hk, pool, b, q, lens, table, q_begin, kv, 2, scale=0.05)


@pytest.mark.parametrize("max_new", [1, 4, 1000])
@pytest.mark.parametrize("name", ["decode", "drafts", "mixed", "no_keys", "more_new_than_tokens"])
def test_attention_with_a_wrong_longest_request(hk, name, max_new):
    """max_new picks the kernel and nothing else."""
    lens = LENS[name]
    rng, g = np.random.default_rng(3), torch.Generator("cuda").manual_seed(3)
    pool, b, table, q_begin, kv = _filled(hk, g, rng, lens, 4, 128, torch.bfloat16)
    b.max_new = max_new
    q = torch.empty(b.n_tokens, 16, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    _attend(hk, pool, b, q, lens, table, q_begin, kv, 4)


@pytest.mark.parametrize("dtype,exps", [("bf16", (20, -30)), ("fp16", (-6, 4)), ("bf16", (-40, 35))])
@pytest.mark.parametrize("name", ["decode", "mixed"])
def test_attention_with_powers_of_two(hk, name, dtype, exps):
    """Pools of very small and very large numbers, and queries to match."""
    lens = LENS[name]
    rng, g = np.random.default_rng(5), torch.Generator("cuda").manual_seed(5)
    pool, b, table, q_begin, kv = _filled(hk, g, rng, lens, 4, 128, DTYPES[dtype], exps, size=2.0 ** min(exps) if dtype == "fp16" else 1.0)
    q = (torch.empty(b.n_tokens, 8, 128, device="cuda").normal_(generator=g) / max(np.nanmax(np.abs(kv[0])), 1e-6)).to(DTYPES[dtype])
    _attend(hk, pool, b, q, lens, table, q_begin, kv, 4, dtype=dtype)


@pytest.mark.parametrize("name", ["decode", "drafts", "chunk_behind"])
def test_attention_strides_streams_and_shifted_maxima(hk, name):
    """q inside a QKV tensor, out with a gap between heads, another stream than the tensors', and logits whose maximum rises by hundreds along
    the keys (every reference moves) or sits on the first key."""
    lens, H, Hkv, d = LENS[name], 12, 4, 128
    rng, g = np.random.default_rng(7), torch.Generator("cuda").manual_seed(7)
    n_pages = sum(-(-kv // PAGE) for _, kv in lens)
    for rising in (True, False):
        blocks = _garbage(g, n_pages, Hkv, d)
        pool = hk.PagedPool4.make(blocks, d, torch.bfloat16)
        b, table, q_begin = _batch(hk, rng, lens, n_pages)
        known = np.zeros((n_pages, PAGE), dtype=bool)
        for i, (_, kv) in enumerate(lens):
            slots = table[i][np.arange(kv) // PAGE] * PAGE + np.arange(kv) % PAGE
            known[slots // PAGE, slots % PAGE] = True
            k = torch.empty(kv, Hkv, d, device="cuda").normal_(generator=g)
            size = torch.arange(kv, device="cuda") / kv if rising else torch.where(torch.arange(kv, device="cuda") == 0, 1.0, 0.0)
            k[:, :, 0] = size[:, None] * 300
            hk.heatkv_paged4_store(pool, k.bfloat16(), k.bfloat16().roll(1, 0).contiguous(), _i32(slots))
        kv = [np.where(known[:, None, :, None], P.values(c, np.minimum(s, 126)), np.nan) for c, s in P.unblock(blocks.cpu().numpy(), d)]
        qkv = torch.empty(b.n_tokens, H + 2 * Hkv, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        q = qkv[:, :H]
        q[..., 0] = 20.0
        wide = torch.zeros(b.n_tokens, H, 2, d, dtype=torch.bfloat16, device="cuda")
        out, ws = wide[:, :, 1], _workspace(hk, pool, b, H)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        hk.heatkv_paged4_attention(pool, b, q, out, None, ws, stream=side)
        side.synchronize()
        _check(out, None, q, kv, lens, table, q_begin, Hkv, True, 1 / math.sqrt(d), "bf16")
        assert not wide[:, :, 0].any()


@pytest.mark.parametrize("name", ["decode", "chunk_behind"])
def test_attention_of_pages_outside_of_the_pool_and_of_nan(hk, name):
    """Entries that name no page read as zeros; NaN in a query row shows in that row and its logarithm, and nowhere else."""
    lens, H, Hkv, d = LENS[name], 8, 4, 64
    rng, g = np.random.default_rng(9), torch.Generator("cuda").manual_seed(9)
    pool, b, table, q_begin, kv = _filled(hk, g, rng, lens, Hkv, d, torch.float16)
    wrong = table.copy()
    n_pages = pool.n_pages
    zero = [np.concatenate([x, np.zeros((1, *x.shape[1:]))]) for x in kv]
    wrong[0, 1], wrong[0, 3] = n_pages, -5
    b.tensors[2].copy_(_i32(wrong))
    wrong[0, 1] = wrong[0, 3] = n_pages                    # where the oracle has its zeros
    q = torch.empty(b.n_tokens, H, d, dtype=torch.float16, device="cuda").normal_(generator=g)
    out, _ = _attend(hk, pool, b, q, lens, wrong, q_begin, zero, Hkv, dtype="fp16")
    bad = q.clone()
    bad[-1, 2, 5] = math.nan
    got, lse = torch.zeros_like(out), torch.zeros(q.shape[:2], device="cuda")
    hk.heatkv_paged4_attention(pool, b, bad, got, lse, _workspace(hk, pool, b, H))
    assert got[-1, 2].isnan().all() and lse[-1, 2].isnan()
    got[-1, 2], lse[-1, 2] = out[-1, 2], 0.0
    assert torch.equal(got, out) and not lse.isnan().any()


@pytest.mark.parametrize("name", ["decode", "mixed"])
def test_attention_captured_and_replayed(hk, name):
    """One graph, lengths and rows changed between its replays; a workspace that calls of all kinds share."""
    lens, H, Hkv, d = LENS[name], 16, 4, 128
    rng, g = np.random.default_rng(11), torch.Generator("cuda").manual_seed(11)
    pool, b, table, q_begin, kv = _filled(hk, g, rng, lens, Hkv, d, torch.bfloat16)
    q = torch.empty(b.n_tokens, H, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out, ws = torch.zeros_like(q), _workspace(hk, pool, b, H)
    hk.heatkv_paged4_attention(pool, b, q, out, None, ws)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        hk.heatkv_paged4_attention(pool, b, q, out, None, ws)
    for cut in (0, 1, 40):
        shorter = [(n, max(kv - cut, 0)) for n, kv in lens]
        b.tensors[1].copy_(_i32([kv for _, kv in shorter]))
        q.normal_(generator=g)
        graph.replay()
        _check(out, None, q, kv, shorter, table, q_begin, Hkv, True, 1 / math.sqrt(d), "bf16")
        b.max_new = 1 if cut else 1 << 16                  # another kernel on the same workspace
        hk.heatkv_paged4_attention(pool, b, q, out.zero_(), None, ws)
        _check(out, None, q, kv, shorter, table, q_begin, Hkv, True, 1 / math.sqrt(d), "bf16")


@pytest.mark.parametrize("max_new", [1, 400])
def test_attention_on_a_workspace_whose_status_is_set(hk, max_new):
    """As after a wait that ran out: calls end at once whatever the workspace holds; zeroed, it serves again."""
    lens, H, Hkv = [(1, 3000), (3, 700), (1, 64 * 40)], 8, 2
    rng, g = np.random.default_rng(12), torch.Generator("cuda").manual_seed(12)
    pool, b, table, q_begin, kv = _filled(hk, g, rng, lens, Hkv, 128, torch.bfloat16)
    b.max_new = max_new
    q = torch.empty(b.n_tokens, H, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    ws = _workspace(hk, pool, b, H)
    words, head = ws.view(torch.int32), 64 + 8192          # status and counters; behind them what kernels hand to one another
    for _ in range(3):
        words[head:] = torch.randint(-2**31, 2**31 - 1, (len(words) - head,), generator=g, device="cuda").int()
        words[0] = 1
        hk.heatkv_paged4_attention(pool, b, q, torch.zeros_like(q), None, ws)
        assert hk.heatkv_paged_status(ws) == -7
    words.zero_()
    out = torch.zeros_like(q)
    hk.heatkv_paged4_attention(pool, b, q, out, None, ws)
    assert hk.heatkv_paged_status(ws) == 0
    _check(out, None, q, kv, lens, table, q_begin, Hkv, True, 1 / math.sqrt(128), "bf16")


@pytest.mark.parametrize("new", [1, 5, 70])
@pytest.mark.parametrize("k_exp,of_q", [(-64, 2.0**-110), (-64, 2.0**68), (64, 2.0**-64)])
def test_attention_at_the_ends_of_the_exponents(hk, k_exp, of_q, new):
    """Keys and values of 2^-64 and 2^64, query rows that make their logits nothing, or large, or ordinary."""
    lens, H, Hkv = [(new, 300), (new, 64), (1, 1)], 8, 2
    rng, g = np.random.default_rng(new), torch.Generator("cuda").manual_seed(new)
    pool, b, table, q_begin, kv = _filled(hk, g, rng, lens, Hkv, 128, torch.bfloat16, (k_exp, k_exp), size=2.0**k_exp)
    q = torch.empty(b.n_tokens, H, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=g).mul_(of_q)
    _attend(hk, pool, b, q, lens, table, q_begin, kv, Hkv)


@pytest.mark.parametrize("new", [1, 70])
def test_pages_behind_two_gigabytes(hk, new):
    """A pool whose last pages lie past 2^31 bytes: stored to, moved, attended to, read back."""
    n_pages, kv, H, d = 250000, 300, 2, 128
    blocks = torch.zeros(n_pages, 1, PAGE * (d + d // 8), dtype=torch.uint8, device="cuda")
    pool = hk.PagedPool4.make(blocks, d, torch.bfloat16)
    g = torch.Generator("cuda").manual_seed(new)
    k, v, q = (torch.empty(n, h, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for n, h in ((kv, 1), (kv, 1), (new, H)))
    first, last = np.arange(kv) + 5 * PAGE, np.arange(kv) + (n_pages - 5) * PAGE
    hk.heatkv_paged4_store(pool, k, v, _i32(first))
    hk.heatkv_paged4_move(pool, _i32(first), _i32(last))
    back = torch.zeros_like(k), torch.zeros_like(v)
    hk.heatkv_paged4_load(pool, _i32(last), *back)
    want = [P.values(*P.quantise(_np(x))) for x in (k, v)]
    for x, w in zip(back, want):
        assert np.array_equal(_np(x), w)
    table = np.arange(n_pages - 5, n_pages)[None]
    b = hk.PagedBatch.make(_i32([0, new]), _i32([kv]), _i32(table), new, new)
    full = np.full((2, 5, 1, PAGE, d), np.nan)
    for x, w in zip(full, want):
        for t in range(kv):
            x[t // PAGE, :, t % PAGE] = w[t]
    _attend(hk, pool, b, q, [(new, kv)], np.arange(5)[None], np.array([0, new]), full, 1)


def test_calls_from_two_threads(hk):
    """Each with a pool, a workspace and a stream of its own, calls of several kinds at once: the bits of one after another."""
    import threading
    lens = [[(1, 900), (1, 5000)], [(40, 300), (1, 700), (65, 65)]]
    jobs = []
    for n, l in enumerate(lens):
        rng, g = np.random.default_rng(n), torch.Generator("cuda").manual_seed(n)
        pool, b, _, q_begin, _ = _filled(hk, g, rng, l, 4, 128, torch.bfloat16)
        q = torch.empty(b.n_tokens, 16, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        ws, want = _workspace(hk, pool, b, 16), torch.zeros_like(q)
        hk.heatkv_paged4_attention(pool, b, q, want, None, ws)
        jobs.append((pool, b, q, ws, want))
    torch.cuda.synchronize()
    wrong = []

    def work(pool, b, q, ws, want):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(50):
                out = torch.zeros_like(q)
                hk.heatkv_paged4_attention(pool, b, q, out, None, ws)
                if not torch.equal(out, want):
                    wrong.append(b.n_tokens)

    threads = [threading.Thread(target=work, args=job) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_graphs_that_share_a_workspace(hk):
    """Captured calls of both kernels over 4 bits and of both over 16, on one workspace, replayed in any order: the bits of calls by themselves."""
    calls, size = [], 0
    for n, l in enumerate(([(1, 900), (1, 9000), (2, 70)], [(300, 1000), (1, 700), (65, 65)])):
        rng, g = np.random.default_rng(n), torch.Generator("cuda").manual_seed(n)
        pool, b, table, _, _ = _filled(hk, g, rng, l, 2, 128, torch.bfloat16)
        pages = [torch.empty(pool.n_pages, 2, PAGE, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in "kv"]
        pool16 = hk.PagedPool.make(*pages)
        q = torch.empty(b.n_tokens, 16, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        for p, bytes_of, attend in ((pool, hk.heatkv_paged4_workspace_bytes, hk.heatkv_paged4_attention),
                                    (pool16, hk.heatkv_paged_workspace_bytes, hk.heatkv_paged_attention)):
            need = bytes_of(p, b, 16)
            want, out = torch.zeros_like(q), torch.zeros_like(q)
            attend(p, b, q, want, None, torch.zeros(need, dtype=torch.uint8, device="cuda"))
            calls.append((attend, p, b, q, out, want, pages))
            size = max(size, need)
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    graphs = []
    for attend, p, b, q, out, _, _ in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            attend(p, b, q, out, None, ws)
        graphs.append(graph)
    for i in (0, 1, 2, 3, 3, 1, 0, 2, 0, 0, 3, 2, 1):
        out, want = calls[i][4:6]
        out.zero_()
        graphs[i].replay()
        assert torch.equal(out, want), i
    assert hk.heatkv_paged_status(ws) == 0


# ------------------------------------------------------------------------------------------------ rows between steps

def _rows_state(hk, lengths, width, free, seed, shared=()):
    """Lengths, table, ring and the rest of a cache; shared: (row, of row, pages) that a row has from another."""
    rng = np.random.default_rng(seed)
    lists = {row: (of, pages) for row, of, pages in shared}
    held = [-(-max(n, 0) // PAGE) - lists.get(i, (0, 0))[1] for i, n in enumerate(lengths)]
    n_pages = sum(held) + free + 3
    order = rng.permutation(n_pages)
    table, at = np.full((len(lengths), width), -1), 0
    for i, n in enumerate(lengths):
        of, pages = lists.get(i, (0, 0))
        table[i, :pages] = table[of, :pages]
        table[i, pages: pages + held[i]] = order[at: at + held[i]]
        at += held[i]
    fifo, head = [int(x) for x in order[at: at + free]], n_pages - 2      # the ring goes round its end
    ring = np.full(n_pages, -1)
    for j, page in enumerate(fifo):
        ring[(head + j) % n_pages] = page
    return table, fifo, ring, head, n_pages


def _rearranged(hk, call, lengths, table, ring, head, count, n_moves, ws=None):
    """Runs one of the two calls twice (it may be repeated): (lengths, table, from, to, state, ring)."""
    n, width = table.shape
    old = torch.full((n, width + 3), -7, dtype=torch.int32, device="cuda")
    new = torch.full((n, width + 5), -9, dtype=torch.int32, device="cuda")
    old[:, :width] = _i32(table)
    state, state_out, free, lens = _i32([head, count, 0, 0]), _i32([5] * 4), _i32(ring), _i32(lengths)
    out, moves = _i32([-3] * n), (_i32([-3] * n_moves), _i32([-3] * n_moves))
    if ws is None:
        ws = torch.zeros(hk.heatkv_paged_rows_workspace_bytes(n, width, len(ring)), dtype=torch.uint8, device="cuda")
    for _ in range(2):
        call(lens, old[:, :width], free, state, out, new[:, :width], state_out, *moves, ws)
    assert (new[:, width:] == -9).all() and lens.tolist() == list(lengths) and np.array_equal(old[:, :width].cpu().numpy(), table)
    return [x.cpu().numpy() for x in (out, new[:, :width], *moves, state_out, free)]


def _same(got, want, ring, head, count, last):
    """want: the oracle's (lengths, table, from, to, taken, refused, back)."""
    for g, w, what in zip(got, want, ("lengths", "table", "from", "to")):
        assert np.array_equal(g, w), what
    taken, refused, back = want[4:7]
    n_pages = len(ring)
    assert got[4].tolist() == [(head + taken) % n_pages, count - taken + len(back), refused, last]
    for j, page in enumerate(back):
        ring[(head + count + j) % n_pages] = page
    assert np.array_equal(got[5], ring)


FORKS = {
    "as_they_are": dict(lengths=[70, 0, 64, 5], parents=[0, 1, 2, 3]),
    "all_over": dict(lengths=[70, 0, 64, 5], parents=[-1, -1, 99, -7]),
    "one_to_many": dict(lengths=[200, 0, 0, 0, 0], parents=[0] * 5),
    "one_to_many_from_the_middle": dict(lengths=[0, 0, 200, 0, 0], parents=[2] * 5),
    "its_own_row_ends": dict(lengths=[0, 130, 0], parents=[1, -1, 1]),
    "whole_pages": dict(lengths=[128, 0, 64, 0], parents=[0, 0, 2, 2]),
    "permuted": dict(lengths=[10, 75, 128, 300], parents=[3, 2, 1, 0]),
    "beams": dict(lengths=[300, 300, 300, 300], parents=[1, 1, 0, 3], shared=[(1, 0, 4), (2, 0, 4), (3, 0, 3)]),
    "cut_back": dict(lengths=[300, 300, 70, 64], parents=[0, 1, 2, 3], keep=[130, 300, 0, 64], shared=[(1, 0, 4)]),
    "cut_into_a_shared_page": dict(lengths=[300, 300, 300], parents=[0, 1, 2], keep=[100, 100, 300], shared=[(1, 0, 4), (2, 0, 4)]),
    "cut_to_different_lengths": dict(lengths=[300, 0, 0, 0], parents=[0, 0, 0, 0], keep=[100, 110, 128, 65]),
    "negative": dict(lengths=[-5, 70, 80], parents=[0, 1, 1], keep=[9, -2, 70]),
    "too_few_pages": dict(lengths=[200, 0, 0, 0, 20], parents=[0, 0, 0, 0, 4], free=2),
    "no_free_page": dict(lengths=[30, 0, 300], parents=[0, 0, 2], free=0),
    "longer_than_the_table": dict(lengths=[10000, 0], parents=[0, 0], width=6, listed=384),
    "many": dict(lengths=[(i * 37) % 500 for i in range(4096)], parents=[i - i % 5 for i in range(4096)], free=4096),
}


@pytest.mark.parametrize("name", FORKS)
def test_fork(hk, name):
    c = FORKS[name]
    lengths, parents = c["lengths"], c["parents"]
    n = len(lengths)
    there = [min(x, c.get("listed", x)) for x in lengths]
    width = c.get("width") or max(max(-(-x // PAGE) for x in there), 1) + 2
    free = c.get("free", 2 * n)
    table, fifo, ring, head, n_pages = _rows_state(hk, there, width, free, len(name), c.get("shared", ()))
    keep = c.get("keep")
    want = P.fork(parents, keep or [10**6] * n, there, table, fifo)
    got = _rearranged(hk, lambda *a: hk.heatkv_paged_fork(_i32(parents), None if keep is None else _i32(keep), *a), lengths, table, ring, head,
                      len(fifo), n * PAGE)
    _same(got, want, ring, head, len(fifo), len(want[6]))


COMPACTS = {
    "nothing_leaves": dict(lengths=[100, 0, 64], part=1.0),
    "everything_leaves": dict(lengths=[100, 0, 64, 1], part=0.0),
    "some": dict(lengths=[1, 63, 64, 65, 500, 1000], part=0.5),
    "few_stay": dict(lengths=[700, 3000, 129], part=0.03),
    "few_leave": dict(lengths=[700, 3000, 129], part=0.999),
    "the_end_leaves": dict(lengths=[300, 128, 70], cut=100),
    "the_beginning_leaves": dict(lengths=[300, 128, 70], skip=65),
    "narrow": dict(lengths=[300, 128, 70], part=0.5, narrow=100),
    "too_few_pages": dict(lengths=[300, 1000, 128, 20], part=0.5, free=6),
    "no_free_page": dict(lengths=[300, 64, 128], part=0.5, free=0),
    "too_few_moves": dict(lengths=[300, 1000, 128, 20], part=0.5, n_moves=200),
    "shared": dict(lengths=[300, 300, 300], part=0.5, shared=[(1, 0, 4), (2, 0, 2)]),
    "long": dict(lengths=[50000, 3], part=0.3),
    "many": dict(lengths=[(i * 37) % 300 for i in range(4096)], part=0.6),
}


@pytest.mark.parametrize("kind", ["bool", "uint8"])
@pytest.mark.parametrize("name", COMPACTS)
def test_compact(hk, name, kind):
    c = COMPACTS[name]
    lengths, rng = c["lengths"], np.random.default_rng(len(name))
    n, most = len(lengths), max(lengths)
    stays = rng.random((n, most)) < c.get("part", 1.0)
    if "cut" in c:
        stays[:, c["cut"]:] = False
    stays[:, : c.get("skip", 0)] = False
    stays = stays[:, : c.get("narrow", most)]
    width = -(-most // PAGE) + 2
    free = c.get("free", sum(-(-x // PAGE) for x in lengths) + 2)
    table, fifo, ring, head, n_pages = _rows_state(hk, lengths, width, free, len(name), c.get("shared", ()))
    n_moves = c.get("n_moves", sum(lengths) + 5)
    *want, done = P.compact(stays, lengths, table, fifo, n_moves)
    wide = torch.zeros(n, stays.shape[1] + 3, dtype=torch.uint8, device="cuda")
    mask = wide[:, : stays.shape[1]]
    mask.copy_(torch.from_numpy(stays * 3 if kind == "uint8" else stays))
    if kind == "bool":
        mask = mask.bool()
    got = _rearranged(hk, lambda *a: hk.heatkv_paged_compact(mask, *a), lengths, table, ring, head, len(fifo), n_moves)
    _same(got, want, ring, head, len(fifo), done)


def test_rows_share_a_workspace(hk):
    """Forks and compactions of one batch after another on one workspace: no mark of one is left for the next."""
    ws = torch.zeros(hk.heatkv_paged_rows_workspace_bytes(60, 30, 5000), dtype=torch.uint8, device="cuda")
    for seed in range(6):
        rng = np.random.default_rng(seed)
        n = int(rng.integers(1, 60))
        lengths, free = [int(x) for x in rng.integers(0, 1000, n)], int(rng.integers(0, 1000))
        table, fifo, ring, head, n_pages = _rows_state(hk, lengths, 20, free, seed)
        if seed % 2:
            parents = [int(x) for x in rng.integers(-1, n, n)]
            want = P.fork(parents, [10**6] * n, lengths, table, fifo)
            got = _rearranged(hk, lambda *a: hk.heatkv_paged_fork(_i32(parents), None, *a), lengths, table, ring, head, free, n * PAGE, ws)
            _same(got, want, ring, head, free, len(want[6]))
        else:
            stays = rng.random((n, 1000)) < 0.5
            *want, done = P.compact(stays, lengths, table, fifo, sum(lengths) + 1)
            mask = torch.from_numpy(stays).cuda()
            got = _rearranged(hk, lambda *a: hk.heatkv_paged_compact(mask, *a), lengths, table, ring, head, free, sum(lengths) + 1, ws)
            _same(got, want, ring, head, free, done)


@pytest.mark.parametrize("n_pages", [16384, 16385, 70000])
def test_rows_of_large_pools(hk, n_pages):
    """Pools at the end of what shared memory has marks for, behind it, and of several chunks; forks and compactions in turn on one workspace."""
    ws = torch.zeros(hk.heatkv_paged_rows_workspace_bytes(9, 4000, n_pages), dtype=torch.uint8, device="cuda")
    for seed in range(4):
        rng = np.random.default_rng(seed)
        lengths = [int(x) for x in rng.integers(0, 64 * 3000, 5)] + [0, 1, 64, 0]
        free = n_pages - 3 - sum(-(-x // PAGE) for x in lengths)
        n_free = min(free, 9000)
        table, fifo, ring, head, total = _rows_state(hk, lengths, 3200, free, seed)
        assert total == n_pages
        fifo = fifo[:n_free]
        if seed % 2 == 0:
            parents = [int(x) for x in rng.integers(-1, 9, 9)]
            want = P.fork(parents, [10**7] * 9, lengths, table, fifo)
            got = _rearranged(hk, lambda *a: hk.heatkv_paged_fork(_i32(parents), None, *a), lengths, table, ring, head, n_free, 9 * PAGE, ws)
            _same(got, want, ring, head, n_free, len(want[6]))
        else:
            stays = rng.random((9, 64 * 3000)) < 0.7
            *want, done = P.compact(stays, lengths, table, fifo, sum(lengths))
            mask = torch.from_numpy(stays).cuda()
            got = _rearranged(hk, lambda *a: hk.heatkv_paged_compact(mask, *a), lengths, table, ring, head, n_free, sum(lengths), ws)
            _same(got, want, ring, head, n_free, done)


@pytest.mark.parametrize("n_pages", [50, 20000])
def test_rings_and_tables_that_contradict_each_other(hk, n_pages):
    """A full ring whose pages the table lists all the same: nothing outside of the buffers is written, for whatever the result is worth."""
    guard = 4096
    free = torch.full((n_pages + 2 * guard,), -5, dtype=torch.int32, device="cuda")
    ring = free[guard: guard + n_pages]
    ring.copy_(torch.arange(n_pages))
    table, lengths = torch.arange(n_pages, dtype=torch.int32, device="cuda")[None], _i32([n_pages * PAGE])
    ws = torch.zeros(hk.heatkv_paged_rows_workspace_bytes(1, n_pages, n_pages), dtype=torch.uint8, device="cuda")
    moves = [torch.zeros(n_pages * PAGE, dtype=torch.int32, device="cuda") for _ in range(2)]
    stays = torch.zeros(1, n_pages * PAGE, dtype=torch.bool, device="cuda")
    for call, args in ((hk.heatkv_paged_fork, (_i32([-1]), None)), (hk.heatkv_paged_compact, (stays,))):
        for state in ([n_pages - 1, n_pages], [-1, 2**31 - 1], [2**31 - 1, -7]):
            out, state_out = torch.zeros_like(table), _i32([0] * 4)
            call(*args, lengths, table, ring, _i32([*state, 0, 0]), _i32([0]), out, state_out, *(m[:PAGE] if args[-1] is None else m for m in moves), ws)
            torch.cuda.synchronize()
            assert (free[:guard] == -5).all() and (free[guard + n_pages:] == -5).all()
            assert (ring >= 0).all() and (ring < n_pages).all() and (out == -1).all()


@pytest.mark.parametrize("n_pages", [400, 20000])
def test_rows_captured_and_replayed(hk, n_pages):
    """A fork, its moves, a compaction and its moves as one graph, replayed over states of different lengths: what the calls give one by one."""
    n, width, moved = 9, 20, 9 * 20 * PAGE
    g = torch.Generator("cuda").manual_seed(n_pages)
    i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")      # noqa: E731
    blocks = _garbage(g, 400, 2, 64)
    pool, ws = hk.PagedPool4.make(blocks, 64, torch.bfloat16), torch.zeros(hk.heatkv_paged_rows_workspace_bytes(n, width, n_pages), dtype=torch.uint8, device="cuda")
    parents, stays, lengths, table, ring, state = i32(n), torch.zeros(n, 1000, dtype=torch.bool, device="cuda"), i32(n), i32(n, width), i32(n_pages), i32(4)
    made = [(i32(n), i32(n, width), i32(4), i32(m), i32(m)) for m in (n * PAGE, moved)]

    def step(ws):
        (l1, t1, s1, *m1), (l2, t2, s2, *m2) = made
        hk.heatkv_paged_fork(parents, None, lengths, table, ring, state, l1, t1, s1, *m1, ws)
        hk.heatkv_paged4_move(pool, *m1)
        hk.heatkv_paged_compact(stays, l1, t1, ring, s1, l2, t2, s2, *m2, ws)
        hk.heatkv_paged4_move(pool, *m2)

    graph = torch.cuda.CUDAGraph()
    first = blocks.clone()
    step(ws)
    with torch.cuda.graph(graph):
        step(ws)
    for seed in range(4):
        rng = np.random.default_rng(seed)
        lens = [int(x) for x in rng.integers(0, 900, n)]
        held = sum(-(-x // PAGE) for x in lens)
        pages, at = rng.permutation(400), 0
        for i, x in enumerate(lens):
            k = -(-x // PAGE)
            table[i] = -1
            table[i, :k] = _i32(pages[at: at + k])
            at += k
        ring[: 400 - held] = _i32(pages[held:])
        free = ring.clone()
        state.copy_(_i32([0, 400 - held, 0, 0]))
        lengths.copy_(_i32(lens))
        parents.copy_(_i32(rng.integers(-1, n, n)))
        stays.copy_(torch.from_numpy(rng.random((n, 1000)) < 0.6))
        got = []
        for run in (lambda: step(torch.zeros_like(ws)), graph.replay):
            ring.copy_(free)
            blocks.copy_(first)
            run()
            got.append([x.clone() for x in (*made[0], *made[1], ring, blocks)])
        for a, b in zip(*got):
            assert torch.equal(a, b)
        assert got[0][2][2] == 0 and got[0][7][2] == 0               # nobody lost tokens or was left as it was


# ------------------------------------------------------------------------------------------------ moves

def _moves(rng, n_pages, count):
    slots = rng.permutation(n_pages * PAGE)
    source, target = slots[:count].copy(), slots[count: 2 * count].copy()
    source[3], target[5] = -1, n_pages * PAGE              # nothing there
    return source, target


@pytest.mark.parametrize("dtype,d,Hkv,layout", [("bf16", 128, 8, "head"), ("fp16", 64, 3, "token"), ("fp16", 128, 1, "token")])
def test_move(hk, dtype, d, Hkv, layout):
    rng, g = np.random.default_rng(d), torch.Generator("cuda").manual_seed(d)
    n_pages, shape = 12, (12, Hkv, PAGE, d) if layout == "head" else (12, PAGE, Hkv, d + 8)
    k, v = (torch.empty(shape, dtype=DTYPES[dtype], device="cuda").normal_(generator=g) for _ in "kv")
    if layout == "token":
        k, v = (x[..., :d].transpose(1, 2) for x in (k, v))
    pool = hk.PagedPool.make(k, v)
    source, target = _moves(rng, n_pages, 300)
    want = [_np(x) for x in (k, v)]
    for x in want:
        for a, b in zip(source, target):
            if 0 <= a < n_pages * PAGE and 0 <= b < n_pages * PAGE:
                x[b // PAGE, :, b % PAGE] = x[a // PAGE, :, a % PAGE]
    hk.heatkv_paged_move(pool, _i32(source), _i32(target))
    for x, w in zip((k, v), want):
        assert np.array_equal(_np(x), w)


def test_move_with_summaries(hk):
    """A page whose last row is moved to gets the summary of its 64 keys, no other page any."""
    g, Hkv, d, n_pages = torch.Generator("cuda").manual_seed(2), 3, 64, 6
    k, v = (torch.empty(n_pages, Hkv, PAGE, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in "kv")
    code, scale = torch.full((n_pages, Hkv, d), 99, dtype=torch.int8, device="cuda"), torch.full((n_pages, Hkv), -1.0, device="cuda")
    pool = hk.PagedPool.make(k, v, code, scale)
    source, target = np.arange(10, 138), np.arange(3 * PAGE, 5 * PAGE)
    target[-1] = -1                                        # the second page's last row stays away
    hk.heatkv_paged_move(pool, _i32(source), _i32(target))
    for h in range(Hkv):
        c, s = P.summary(k[3, h].float().cpu().numpy())
        assert np.array_equal(code[3, h].cpu().numpy(), c) and scale[3, h].item() == s
    others = [0, 1, 2, 4, 5]
    assert (code[others] == 99).all() and (scale[others] == -1.0).all()


@pytest.mark.parametrize("d,Hkv", [(128, 5), (64, 8)])
def test_move_in_4_bits(hk, d, Hkv):
    rng, g, n_pages = np.random.default_rng(d), torch.Generator("cuda").manual_seed(d), 12
    blocks = _garbage(g, n_pages, Hkv, d)
    pool = hk.PagedPool4.make(blocks, d, torch.bfloat16)
    source, target = _moves(rng, n_pages, 300)
    want = P.unblock(blocks.cpu().numpy(), d)
    for pair in want:
        for x in pair:
            for a, b in zip(source, target):
                if 0 <= a < n_pages * PAGE and 0 <= b < n_pages * PAGE:
                    x[b // PAGE, :, b % PAGE] = x[a // PAGE, :, a % PAGE]
    hk.heatkv_paged4_move(pool, _i32(source), _i32(target))
    for got, w in zip(P.unblock(blocks.cpu().numpy(), d), want):
        assert np.array_equal(got[0], w[0]) and np.array_equal(got[1], w[1])


# ------------------------------------------------------------------------------------------------ all of it, as a server uses it

@pytest.mark.parametrize("bits,dtype,d", [(4, "bf16", 128), (4, "fp16", 64), (16, "bf16", 64)])
def test_cache_with_forks_and_compactions(hk, bits, dtype, d):
    """A prompt answered three ways beside another request, rows cut back into pages that they share, tokens taken out, rows that end; two layers.
    Every attention against the rows that a plain list has, every position, and in the end every page is free."""
    from paper_2605_14877_b200.paged import PagedCache
    layers, H, Hkv, rows, dt = 2, 6, 2, 4, DTYPES[dtype]
    g, rng = torch.Generator("cuda").manual_seed(bits + d), np.random.default_rng(bits + d)
    cache = PagedCache(layers, H, Hkv, d, n_pages=40, rows=rows, max_pages=12, dtype=dt, bits=bits)
    held = [[[] for _ in range(rows)] for _ in range(layers)]      # (k, v) of every token, [heads, d] each
    count = [0] * rows                                             # tokens that a row has had

    def kept(x):
        x = _np(x)
        return P.values(*P.quantise(x)) if bits == 4 else x

    def step(new):
        s = cache.begin(new)
        want = [count[i] + t for i, n in enumerate(new) for t in range(n)]
        assert s.positions.tolist() == want
        begin = np.concatenate([[0], np.cumsum(new)])
        for layer in range(layers):
            q, k, v = (torch.empty(sum(new), h, d, dtype=dt, device="cuda").normal_(generator=g) for h in (H, Hkv, Hkv))
            out, lse = torch.full_like(q, 7.0), torch.full((sum(new), H), 7.0, device="cuda")
            cache.attend(layer, s, q, k, v, out, lse)
            k, v = kept(k), kept(v)
            lens = []
            for i, n in enumerate(new):
                held[layer][i] += [(k[t], v[t]) for t in range(begin[i], begin[i + 1])]
                lens.append((n, len(held[layer][i])))
            # rows one behind another, as if in pages of their own
            pages = [-(-n // PAGE) for _, n in lens]
            table, at = np.full((rows, max(pages) + 1), -1), 0
            kv = np.full((2, sum(pages) + 1, Hkv, PAGE, d), np.nan)
            for i, p in enumerate(pages):
                table[i, :p] = np.arange(at, at + p)
                for t, pair in enumerate(held[layer][i]):
                    kv[:, at + t // PAGE, :, t % PAGE] = pair
                at += p
            _check(out, lse, q, kv, lens, table, begin, Hkv, True, 1 / math.sqrt(d), dtype)
        for i, n in enumerate(new):
            count[i] += n

    def fork(parents):
        cache.fork(parents)
        for layer in range(layers):
            held[layer] = [[] if p is None else list(held[layer][p]) for p in parents]
        count[:] = [0 if p is None else count[p] for p in parents]

    def keep(lengths):
        cache.keep(lengths)
        for i, n in enumerate(lengths):
            cut = len(held[0][i]) - n
            if cut > 0:
                count[i] = count[i] - cut if n else 0
            for layer in range(layers):
                del held[layer][i][n:]

    step([200, 0, 0, 70])
    fork([0, 0, 0, 3])
    step([1, 2, 3, 1])
    keep([1000, 150, 201, 64])                                     # row 1 into a page that it shares, row 2 to what was forked
    step([5, 60, 1, 1])
    stays = torch.from_numpy(rng.random((rows, 180)) < 0.6).cuda()
    cache.compact(stays)
    for layer in range(layers):
        for i in range(rows):
            held[layer][i] = [x for t, x in enumerate(held[layer][i]) if t >= 180 or stays[i, t]]
    assert cache.lengths.tolist() == [len(x) for x in held[0]] and cache.state.tolist()[2] == 0
    step([1, 1, 1, 1])
    fork([1, None, 1, 2])                                          # row 0 is over, rows move
    step([2, 0, 130, 1])
    keep([1000, 0, 0, 30])
    step([1, 40, 0, 1])
    assert cache.lengths.tolist() == [len(x) for x in held[0]]
    cache.check()
    keep([0, 0, 0, 0])
    assert cache.state.tolist()[1] == 40 and sorted(cache.free.tolist()) == list(range(40))


def test_cache_that_runs_out_of_pages_for_forks(hk):
    """Rows for which no page is left lose the tokens of the one that is not full, and say so; compaction then leaves a row as it is."""
    from paper_2605_14877_b200.paged import PagedCache
    cache = PagedCache(1, 2, 2, 64, n_pages=4, rows=3, max_pages=4, bits=4)
    q = torch.zeros(130, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache.attend(0, cache.begin([130, 0, 0]), q, q, q, torch.empty_like(q))
    cache.fork([0, 0, 0])
    assert cache.lengths.tolist() == [130, 130, 128] and cache.state.tolist()[1:3] == [0, 1]
    stays = torch.ones(3, 130, dtype=torch.bool, device="cuda")
    stays[:, 3] = False
    cache.compact(stays)
    assert cache.lengths.tolist() == [130, 130, 128] and cache.state.tolist()[2] == 3
    cache.keep([0, 0, 128])
    assert cache.lengths.tolist() == [0, 0, 128] and cache.state.tolist()[1] == 2
    cache.compact(stays)
    assert cache.lengths.tolist() == [0, 0, 127] and cache.state.tolist()[1:3] == [2, 0]
