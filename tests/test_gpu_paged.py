"""The paged cache for requests of any length against plain numpy (whole numbers and summaries bit for bit, attention in 64 bits).

Tolerances.  With u = 2^-8 (bf16, 8 significant bits) or 2^-11 (fp16, 11), the relative rounding of a 16-bit result: the output is rounded once (u |out|), the
probabilities once (u sum p |v|); a logit is a 32-bit sum of d products and one scaling, off by at most (d + 8) 2^-24 of sum |q k| scale,
which moves a probability by twice that and the logarithm of the sum by once that; exponentials and sums of 32 bits add 2^-18.  In fp16
a probability may be subnormal: at most 2^-25 of the largest each."""
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
    return x.detach().float().cpu().numpy()


# ------------------------------------------------------------------------------------------------ tables and slots

TABLES = {
    "one": dict(new=[1], past=[0]),
    "one_page_ends": dict(new=[1, 1, 1], past=[63, 64, 65]),
    "nothing_new": dict(new=[0, 5, 0], past=[100, 0, 0]),
    "prompts": dict(new=[1, 64, 65, 200, 1000, 63], past=[0, 0, 63, 7, 128, 1]),
    "negative": dict(new=[-3, 4], past=[5, -7]),
    "pool_too_small": dict(new=[100, 300, 10, 1, 200, 0], past=[0, 0, 54, 64, 0, 64], free=4),
    "row_too_short": dict(new=[100, 700, 64], past=[0, 0, 0], width=6),
    "no_free_page": dict(new=[1, 1, 1], past=[3, 64, 70], free=0),
    "places_to_spare": dict(new=[70, 3], past=[10, 10], spare=37),
    "many": dict(new=[1 + i % 3 for i in range(4096)], past=[(i * 37) % 300 for i in range(4096)]),
    "long": dict(new=[40000, 3], past=[25000, 64 * 900 - 1]),
}


def _tables_case(new, past, free=None, width=None, spare=0, seed=0):
    rng = np.random.default_rng(seed)
    had = [-(-max(p, 0) // PAGE) for p in past]
    width = width or max(-(-(max(n, 0) + max(p, 0)) // PAGE) for n, p in zip(new, past)) + 2
    wanted = sum(max(-(-(max(n, 0) + max(p, 0)) // PAGE) - h, 0) for n, p, h in zip(new, past, had))
    free = wanted + 3 if free is None else free
    n_pages = sum(had) + free + 2
    order = rng.permutation(n_pages)
    table = np.full((len(new), width), -1)
    at = 0
    for i, h in enumerate(had):
        table[i, :h] = order[at: at + h]
        at += h
    fifo = list(order[at: at + free])
    head = n_pages - 2                                     # the ring goes round its end
    ring = np.full(n_pages, -1)
    for j, page in enumerate(fifo):
        ring[(head + j) % n_pages] = page
    total = sum(max(n, 0) for n in new)
    return table, fifo, ring, head, n_pages, max(total + spare, 1)


@pytest.mark.parametrize("name", TABLES)
def test_tables(hk, name):
    c = TABLES[name]
    table, fifo, ring, head, n_pages, n_tokens = _tables_case(**c)
    want = P.tables(c["new"], c["past"], fifo, table, n_tokens)
    wide = torch.full((len(c["new"]), table.shape[1] + 5), -7, dtype=torch.int32, device="cuda")
    dev = wide[:, : table.shape[1]]
    dev.copy_(_i32(table))
    state, state_out = _i32([head, len(fifo), 0, 0]), _i32([9] * 4)
    n = len(c["new"])
    q_begin, kv, slots, pos = _i32([-5] * (n + 1)), _i32([-5] * n), _i32([-5] * n_tokens), _i32([-5] * n_tokens)
    free = _i32(ring)
    for positions in (pos, None):                          # twice: the call may be repeated
        hk.heatkv_paged_tables(_i32(c["new"]), _i32(c["past"]), free, state, state_out, dev, q_begin, kv, slots, positions)
    got = [x.cpu().numpy() for x in (dev, q_begin, kv, slots, pos)]
    for g, w, what in zip(got, want, ("table", "q_begin", "kv_len", "slots", "positions")):
        assert np.array_equal(g, w), what
    taken, refused = want[5:]
    assert state_out.tolist() == [(head + taken) % n_pages, len(fifo) - taken, refused, want[1][-1]]
    assert np.array_equal(free.cpu().numpy(), ring) and (wide[:, table.shape[1]:] == -7).all()


def test_release_gives_pages_back_in_order(hk):
    new, past = [1, 64, 65, 200, 40], [0, 0, 63, 7, 0]
    table, fifo, ring, head, n_pages, n_tokens = _tables_case(new, past)
    dev, state, mid, end = _i32(table), _i32([head, len(fifo), 0, 0]), _i32([0] * 4), _i32([0] * 4)
    n = len(new)
    q_begin, kv, slots, free = _i32([0] * (n + 1)), _i32([0] * n), _i32([0] * n_tokens), _i32(ring)
    hk.heatkv_paged_tables(_i32(new), _i32(past), free, state, mid, dev, q_begin, kv, slots)
    keep = [1, 0, 65, 64, 400]                             # all, none, some, exactly one page, more than there are
    hk.heatkv_paged_release(kv, _i32(keep), dev, free, mid, end)
    lens, rows = kv.tolist(), dev.cpu().numpy()
    back = [rows[i, j] for i in range(n) for j in range(-(-min(keep[i], lens[i]) // PAGE), -(-lens[i] // PAGE))]
    h, count = mid.tolist()[:2]
    got = free.cpu().numpy()
    assert [got[(h + count + j) % n_pages] for j in range(len(back))] == back
    assert end.tolist() == [h, count + len(back), 0, len(back)] and len(back) == 4
    # what was given back is handed out again, the oldest first
    again = P.tables([64 * (count + len(back))], [0], [got[(h + j) % n_pages] for j in range(count + len(back))], np.full((1, 99), -1), 6400)
    row, out = _i32(np.full((1, 99), -1)), _i32([0] * 4)
    hk.heatkv_paged_tables(_i32([64 * (count + len(back))]), _i32([0]), free, end, out, row, _i32([0, 0]), _i32([0]), _i32([0] * 6400))
    assert np.array_equal(row.cpu().numpy(), again[0]) and out.tolist()[1] == 0


# ------------------------------------------------------------------------------------------------ pools

def _pool(hk, g, n_pages, Hkv, d, dtype, layout="head", summaries=True, fill=math.nan):
    """A pool whose every value is `fill`; layout "head": [page][head][row][d], "token": [page][row][head][d]."""
    if layout == "head":
        k, v = (torch.full((n_pages, Hkv, PAGE, d), fill, dtype=dtype, device="cuda") for _ in "kv")
    else:
        k, v = (torch.full((n_pages, PAGE, Hkv, d + 8), fill, dtype=dtype, device="cuda")[..., :d].transpose(1, 2) for _ in "kv")
    code = torch.full((n_pages, Hkv, d), 99, dtype=torch.int8, device="cuda") if summaries else None
    scale = torch.full((n_pages, Hkv), -1.0, device="cuda") if summaries else None
    return hk.PagedPool.make(k, v, code, scale), k, v, code, scale


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
    assert at <= n_pages
    q_begin = np.concatenate([[0], np.cumsum([n for n, _ in lens])])
    b = hk.PagedBatch.make(_i32(q_begin), _i32([kv for _, kv in lens]), _i32(table), int(q_begin[-1]) + spare, max(max(n for n, _ in lens), 1))
    return b, table, q_begin


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,Hkv,layout", [(128, 8, "head"), (128, 1, "token"), (64, 5, "token"), (64, 16, "head")])
def test_store(hk, dtype, d, Hkv, layout):
    rng = np.random.default_rng(d + Hkv)
    g = torch.Generator("cuda").manual_seed(d + Hkv)
    dt = DTYPES[dtype]
    n_pages = 24
    pool, k, v, code, scale = _pool(hk, g, n_pages, Hkv, d, dt, layout, fill=0.0)
    k.normal_(generator=g), v.normal_(generator=g)
    # (past, new): a page that fills up with what was there, whole pages, a page's last row alone, nothing that fills up
    parts = [(10, 200), (0, 128), (63, 1), (64, 3), (5, 59)]
    order = list(rng.permutation(n_pages))
    slots, full = [], []
    for past, new in parts:
        pages = [order.pop() for _ in range(-(-(past + new) // PAGE))]
        slots += [pages[p // PAGE] * PAGE + p % PAGE for p in range(past, past + new)]
        full += [pages[p // PAGE] for p in range(past, past + new) if p % PAGE == PAGE - 1]
    at = 200                                               # behind the first request
    slots[at:at] = [-1, n_pages * PAGE, 2**31 - 1]         # tokens without a place
    T = len(slots)
    qkv = torch.empty(T, 3, Hkv, d, dtype=dt, device="cuda").normal_(generator=g)
    before = [_np(x) for x in (k, v)]
    hk.heatkv_paged_store(pool, qkv[:, 1], qkv[:, 2], _i32(slots))
    new = [_np(qkv[:, 1]), _np(qkv[:, 2])]
    for x, b, n in zip((k, v), before, new):
        for t, s in enumerate(slots):
            if 0 <= s < n_pages * PAGE:
                b[s // PAGE, :, s % PAGE] = n[t]
        assert np.array_equal(_np(x), b)
    assert len(full) == 7
    for page in range(n_pages):
        for h in range(Hkv):
            if page in full:
                c, s = P.summary(before[0][page, h])
                assert np.array_equal(code[page, h].cpu().numpy(), c) and scale[page, h].item() == s
            else:
                assert (code[page, h] == 99).all() and scale[page, h].item() == -1.0


def test_store_of_one_head_shared_and_of_zero_keys(hk):
    """K and V broadcast over the heads (stride 0), a page of zeros (scale 0, codes 0), and no summaries kept."""
    pool, k, v, code, scale = _pool(hk, None, 3, 4, 64, torch.bfloat16)
    x = torch.zeros(64, 1, 64, dtype=torch.bfloat16, device="cuda").expand(64, 4, 64)
    hk.heatkv_paged_store(pool, x, x, _i32(range(64, 128)))
    assert (k[1] == 0).all() and (code[1] == 0).all() and (scale[1] == 0).all() and k[0].isnan().all() and k[2].isnan().all()
    pool, k, v, _, _ = _pool(hk, None, 3, 4, 64, torch.bfloat16, summaries=False)
    hk.heatkv_paged_store(pool, x, x, _i32(range(64)))
    assert (v[0] == 0).all() and v[1].isnan().all()


# ------------------------------------------------------------------------------------------------ attention

def _filled(hk, g, rng, lens, Hkv, d, dt, layout="head", spare_pages=2, **more):
    """A pool whose requests' rows are random and everything else NaN."""
    n_pages = sum(-(-kv // PAGE) for _, kv in lens) + spare_pages
    pool, k, v, code, scale = _pool(hk, g, n_pages, Hkv, d, dt, layout)
    b, table, q_begin = _batch(hk, rng, lens, n_pages, **more)
    for i, (_, kv) in enumerate(lens):
        for pg in range(-(-kv // PAGE)):
            rows = min(PAGE, kv - pg * PAGE)
            for x in (k, v):
                x[table[i, pg], :, :rows] = torch.empty(Hkv, rows, d, dtype=dt, device="cuda").normal_(generator=g)
    return pool, b, table, q_begin, k, v, code, scale


def _check(out, lse, q, k, v, lens, table, q_begin, Hkv, causal, scale, dtype, chosen=None):
    G, d = q.shape[1] // Hkv, q.shape[2]
    u = 2.0**-8 if dtype == "bf16" else 2.0**-11
    out, q, k, v = (_np(x).astype(np.float64) for x in (out, q, k, v))
    lse = None if lse is None else lse.cpu().numpy().astype(np.float64)
    for i, (n, kv) in enumerate(lens):
        pages = table[i, : -(-kv // PAGE)]
        for h in range(Hkv):
            keys, values = k[pages, h].reshape(-1, d), v[pages, h].reshape(-1, d)
            rows = slice(q_begin[i], q_begin[i] + n)
            at = np.arange(kv - n, kv)
            j = np.arange(len(keys))
            seen = np.broadcast_to(j < kv, (n, len(keys)))
            if causal:
                seen = seen & (j <= at[:, None])
            if chosen is not None:
                seen = seen & np.repeat(chosen[i][h], PAGE, axis=1)
            for g in range(G):
                o, l, pv, reach = P.attention(q[rows, h * G + g], keys, values, seen, scale)
                off = (d + 8) * 2.0**-24 * reach + 2.0**-18
                big = np.abs(np.where(np.isfinite(values), values, 0.0)).max(initial=0.0)
                tol = u * np.abs(o) + (u + 2 * off)[:, None] * pv + (len(keys) * 2.0**-25 * big if dtype == "fp16" else 0.0) + 1e-30
                got = out[rows, h * G + g]
                assert np.isfinite(got).all()
                assert (np.abs(got - o) <= tol).all(), (i, h, g, float((np.abs(got - o) / tol).max()))
                if lse is not None:
                    gl = lse[rows, h * G + g]
                    assert np.array_equal(np.isinf(gl), np.isinf(l))
                    fin = np.isfinite(l)
                    assert (np.abs(gl[fin] - l[fin]) <= (off + 2.0**-22 * np.abs(l))[fin]).all(), (i, h, g)


LENS = {                                                   # (new tokens, tokens in all) per request
    "one_key": [(1, 1)],
    "one_of_each": [(1, 2), (1, 63), (1, 64), (1, 65), (1, 128), (1, 129)],
    "no_keys": [(1, 0), (1, 70), (0, 0), (2, 0), (0, 100)],
    "decode": [(1, 1000), (1, 17), (1, 3), (1, 517), (1, 64)],
    "long_one": [(1, 20011)],
    "drafts": [(5, 130), (1, 40), (3, 64), (5, 5), (4, 66)],
    "more_new_than_tokens": [(4, 2), (3, 0), (2, 65)],
    "short_prompts": [(1, 1), (33, 33), (64, 64), (65, 65), (127, 127)],
    "prompt": [(300, 300)],
    "chunk_behind": [(130, 700), (257, 260), (128, 128 * 3)],
    "mixed": [(1, 900), (200, 450), (1, 5), (70, 1000)],
}


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("H,Hkv,d,dtype", [(16, 16, 128, "bf16"), (32, 8, 128, "fp16"), (28, 4, 64, "bf16"), (5, 5, 64, "fp16"), (8, 1, 128, "bf16")])
@pytest.mark.parametrize("name", LENS)
def test_attention(hk, name, H, Hkv, d, dtype, causal):
    lens = LENS[name]
    rng = np.random.default_rng(len(name) + H)
    g = torch.Generator("cuda").manual_seed(len(name) + H)
    dt = DTYPES[dtype]
    layout = "token" if (H + len(name)) % 2 else "head"
    pool, b, table, q_begin, k, v, _, _ = _filled(hk, g, rng, lens, Hkv, d, dt, layout, spare=3)
    T = b.n_tokens
    q = torch.empty(T, H, d, dtype=dt, device="cuda").normal_(generator=g)
    out, lse = torch.full_like(q, 7.0), torch.full((T, H), 7.0, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, H), dtype=torch.uint8, device="cuda")
    hk.heatkv_paged_attention(pool, b, q, out, lse, ws, causal=causal)
    assert hk.heatkv_paged_status(ws) == 0
    _check(out, lse, q, k, v, lens, table, q_begin, Hkv, causal, 1 / math.sqrt(d), dtype)
    assert (out[q_begin[-1]:] == 7.0).all() and (lse[q_begin[-1]:] == 7.0).all()
    again = torch.zeros_like(out)
    hk.heatkv_paged_attention(pool, b, q, again, None, ws, causal=causal)
    assert torch.equal(again[: q_begin[-1]], out[: q_begin[-1]])      # and the same bits again, without the logarithms


@pytest.mark.parametrize("G", [1, 3, 16, 17, 32, 33, 64, 128])
def test_attention_any_group(hk, G):
    """Query heads per kv head, from one to 128."""
    lens = [(1, 200), (2, 64), (1, 1)]
    rng, g = np.random.default_rng(G), torch.Generator("cuda").manual_seed(G)
    pool, b, table, q_begin, k, v, _, _ = _filled(hk, g, rng, lens, 2, 128, torch.bfloat16)
    q = torch.empty(b.n_tokens, 2 * G, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out, lse = torch.zeros_like(q), torch.zeros(b.n_tokens, 2 * G, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, 2 * G), dtype=torch.uint8, device="cuda")
    hk.heatkv_paged_attention(pool, b, q, out, lse, ws, sm_scale=0.05)
    _check(out, lse, q, k, v, lens, table, q_begin, 2, True, 0.05, "bf16")


@pytest.mark.parametrize("max_new", [1, 4, 1000])
@pytest.mark.parametrize("name", ["decode", "drafts", "mixed"])
def test_attention_with_a_wrong_longest_request(hk, name, max_new):
    """max_new picks the kernel and nothing else."""
    lens = LENS[name]
    rng, g = np.random.default_rng(3), torch.Generator("cuda").manual_seed(3)
    pool, b, table, q_begin, k, v, _, _ = _filled(hk, g, rng, lens, 4, 128, torch.bfloat16)
    b.max_new = max_new
    q = torch.empty(b.n_tokens, 16, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out, lse = torch.zeros_like(q), torch.zeros(b.n_tokens, 16, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, 16), dtype=torch.uint8, device="cuda")
    hk.heatkv_paged_attention(pool, b, q, out, lse, ws)
    _check(out, lse, q, k, v, lens, table, q_begin, 4, True, 1 / math.sqrt(128), "bf16")


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("H,Hkv,d,dtype", [(16, 16, 128, "bf16"), (32, 8, 128, "fp16"), (28, 4, 64, "bf16"), (5, 5, 64, "fp16"), (132, 4, 128, "bf16")])
@pytest.mark.parametrize("name", ["one_key", "one_of_each", "no_keys", "drafts", "more_new_than_tokens", "short_prompts"])
def test_attention_of_small_calls_as_if_large(hk, name, H, Hkv, d, dtype, causal):
    """Few rows and short requests on the kernel that large calls take."""
    lens = LENS[name]
    rng, g = np.random.default_rng(len(name)), torch.Generator("cuda").manual_seed(len(name))
    pool, b, table, q_begin, k, v, _, _ = _filled(hk, g, rng, lens, Hkv, d, DTYPES[dtype], spare=2)
    b.max_new = 1 << 16
    q = torch.empty(b.n_tokens, H, d, dtype=DTYPES[dtype], device="cuda").normal_(generator=g)
    out, lse = torch.full_like(q, 7.0), torch.full((b.n_tokens, H), 7.0, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, H), dtype=torch.uint8, device="cuda")
    hk.heatkv_paged_attention(pool, b, q, out, lse, ws, causal=causal)
    assert hk.heatkv_paged_status(ws) == 0
    _check(out, lse, q, k, v, lens, table, q_begin, Hkv, causal, 1 / math.sqrt(d), dtype)
    assert (out[q_begin[-1]:] == 7.0).all()


@pytest.mark.parametrize("name", ["decode", "chunk_behind"])
def test_attention_strides_streams_and_shifted_maxima(hk, name):
    """q inside a QKV tensor, out with a gap between heads, another stream than the tensors', and logits whose maximum rises by
    hundreds along the keys (every reference moves) or sits on the first key."""
    lens = LENS[name]
    rng, g = np.random.default_rng(5), torch.Generator("cuda").manual_seed(5)
    for rise in (40.0, -40.0):
        pool, b, table, q_begin, k, v, _, _ = _filled(hk, g, rng, lens, 2, 64, torch.bfloat16)
        for i, (_, kv) in enumerate(lens):
            for pg in range(-(-kv // PAGE)):
                k[table[i, pg], :, :, 0] = rise * pg / max(kv // PAGE, 1)
        qkv = torch.empty(b.n_tokens, 8, 64, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        qkv[:, :, 0] = 16.0
        q = qkv[:, 2:6]
        wide = torch.full((b.n_tokens, 4, 80), 7.0, dtype=torch.bfloat16, device="cuda")
        out, lse = wide[..., :64], torch.zeros(b.n_tokens, 4, device="cuda")
        ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, 4), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        hk.heatkv_paged_attention(pool, b, q, out, lse, ws, stream=side)
        side.synchronize()
        _check(out, lse, q, k, v, lens, table, q_begin, 2, True, 0.125, "bf16")
        assert (wide[..., 64:] == 7.0).all()


def test_attention_of_a_pool_past_32_bits(hk):
    """Pages whose first element lies past 2^31 and, in bytes, past 2^32."""
    Hkv, d, n_pages = 8, 128, 33500
    k, v = (torch.empty(n_pages, Hkv, PAGE, d, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    g = torch.Generator("cuda").manual_seed(0)
    table = np.array([[n_pages - 1, 3, n_pages - 2], [n_pages - 7, 32768, -1]])
    lens = [(1, 180), (70, 100)]
    code = torch.zeros(n_pages, Hkv, d, dtype=torch.int8, device="cuda")
    pool = hk.PagedPool.make(k, v, code, torch.zeros(n_pages, Hkv, device="cuda"))
    b = hk.PagedBatch.make(_i32([0, 1, 71]), _i32([180, 100]), _i32(table), 71, 70)
    slots = [table[i, p // PAGE] * PAGE + p % PAGE for i, (_, kv) in enumerate(lens) for p in range(kv)]
    kv_new = torch.empty(2, len(slots), Hkv, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    hk.heatkv_paged_store(pool, kv_new[0], kv_new[1], _i32(slots))
    q = torch.empty(71, 16, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out, lse = torch.zeros_like(q), torch.zeros(71, 16, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, 16), dtype=torch.uint8, device="cuda")
    used = sorted(set(table[table >= 0].tolist()))
    small = {p: i for i, p in enumerate(used)}
    mapped = np.vectorize(lambda p: small.get(p, -1))(table)
    ks, vs = k[used], v[used]
    hk.heatkv_paged_attention(pool, b, q, out, lse, ws)
    _check(out, lse, q, ks, vs, lens, mapped, [0, 1, 71], Hkv, True, 1 / math.sqrt(d), "bf16")
    b.max_new = 1
    hk.heatkv_paged_attention(pool, b, q, out, lse, ws)
    _check(out, lse, q, ks, vs, lens, mapped, [0, 1, 71], Hkv, True, 1 / math.sqrt(d), "bf16")
    c, s = P.summary(_np(k[n_pages - 1, 2]))
    assert np.array_equal(code[n_pages - 1, 2].cpu().numpy(), c)


# ------------------------------------------------------------------------------------------------ page selection

def _summaries(k, code, scale, pages):
    for page in pages:
        for h in range(k.shape[1]):
            c, s = P.summary(_np(k[page, h]))
            code[page, h], scale[page, h] = torch.from_numpy(c).to(torch.int8), float(s)


@pytest.mark.parametrize("sink,local,n_select", [(0, 1, 1), (1, 2, 8), (2, 3, 5), (0, 1, 40)])
@pytest.mark.parametrize("H,Hkv,d,dtype", [(16, 16, 128, "bf16"), (14, 2, 64, "fp16"), (16, 1, 128, "fp16"), (8, 2, 128, "bf16")])
@pytest.mark.parametrize("name", ["decode", "drafts", "no_keys", "more_new_than_tokens", "chunk_behind"])
def test_select_and_sparse_attention(hk, name, H, Hkv, d, dtype, sink, local, n_select):
    lens = LENS[name]
    rng, g = np.random.default_rng(H + d), torch.Generator("cuda").manual_seed(H + d)
    dt = DTYPES[dtype]
    pool, b, table, q_begin, k, v, code, scale = _filled(hk, g, rng, lens, Hkv, d, dt, spare=2)
    for i, (_, kv) in enumerate(lens):
        _summaries(k, code, scale, table[i, : kv // PAGE])
    # ties: two pages of the longest request have the same summary, and one head's codes are all zero
    longest = max(range(len(lens)), key=lambda i: lens[i][1])
    if lens[longest][1] >= 4 * PAGE:
        a, c = table[longest, 1], table[longest, 3]
        code[a], scale[a] = code[c], scale[c]
    code[:, Hkv - 1] = 0
    T, G = b.n_tokens, H // Hkv
    q = torch.empty(T, H, d, dtype=dt, device="cuda").normal_(generator=g)
    sel = torch.full((T, Hkv, n_select), -9, dtype=torch.int32, device="cuda")
    hk.heatkv_paged_select(pool, b, q, sel, sink, local)
    got, qf, cn, sn = sel.cpu().numpy(), _np(q), code.cpu().numpy(), scale.cpu().numpy()
    chosen = []
    for i, (n, kv) in enumerate(lens):
        pages = table[i, : -(-kv // PAGE)]
        mask = np.zeros((Hkv, n, len(pages)), dtype=bool)
        for t in range(n):
            pos = kv - n + t
            for h in range(Hkv):
                want = P.select(qf[q_begin[i] + t, h * G:(h + 1) * G], cn[pages, h], sn[pages, h], pos, sink, local, n_select) if pos >= 0 else []
                assert got[q_begin[i] + t, h].tolist() == want + [-1] * (n_select - len(want)), (i, t, h)
                mask[h, t, want] = True
        chosen.append(mask)
    assert (got[q_begin[-1]:] == -1).all()
    out, lse = torch.full_like(q, 7.0), torch.full((T, H), 7.0, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, H), dtype=torch.uint8, device="cuda")
    hk.heatkv_paged_sparse_attention(pool, b, q, sel, out, lse, ws)
    assert hk.heatkv_paged_status(ws) == 0
    _check(out, lse, q, k, v, lens, table, q_begin, Hkv, True, 1 / math.sqrt(d), dtype, chosen)
    assert (out[q_begin[-1]:] == 7.0).all() and (lse[q_begin[-1]:] == 7.0).all()


@pytest.mark.parametrize("G", [1, 17, 33, 64])
def test_sparse_attention_any_group(hk, G):
    """Query heads per kv head from one to 64; every second page."""
    lens = [(1, 500), (3, 64), (1, 130)]
    rng, g = np.random.default_rng(G), torch.Generator("cuda").manual_seed(G)
    pool, b, table, q_begin, k, v, _, _ = _filled(hk, g, rng, lens, 2, 128, torch.bfloat16)
    q = torch.empty(b.n_tokens, 2 * G, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    sel = np.tile(np.arange(0, 8, 2), (b.n_tokens, 2, 1))
    chosen = [np.broadcast_to(np.arange(-(-kv // PAGE)) % 2 == 0, (2, n, -(-kv // PAGE))) for n, kv in lens]
    out, lse = torch.zeros_like(q), torch.zeros(b.n_tokens, 2 * G, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, 2 * G), dtype=torch.uint8, device="cuda")
    hk.heatkv_paged_sparse_attention(pool, b, q, _i32(sel), out, lse, ws)
    _check(out, lse, q, k, v, lens, table, q_begin, 2, True, 1 / math.sqrt(128), "bf16", chosen)


@pytest.mark.parametrize("G,d,dtype", [(1, 128, "bf16"), (2, 64, "fp16"), (3, 128, "fp16"), (8, 64, "bf16"), (40, 128, "bf16"), (64, 64, "bf16")])
@pytest.mark.parametrize("max_new", [1, 100])
def test_sparse_attention_of_chunks_over_random_lists(hk, G, d, dtype, max_new):
    """Lists of random lengths in random order with gaps, for chunks that end inside a tile; both kernels (max_new picks one)."""
    lens = [(90, 700), (1, 65), (0, 0), (67, 67), (40, 1000)]
    Hkv, n_select = 4, 32                                  # as many lists as it takes for them to be merged
    rng, g = np.random.default_rng(G), torch.Generator("cuda").manual_seed(G)
    dt = DTYPES[dtype]
    pool, b, table, q_begin, k, v, _, _ = _filled(hk, g, rng, lens, Hkv, d, dt, spare=2)
    b.max_new = max_new
    sel = np.full((b.n_tokens, Hkv, n_select), -1)
    chosen = []
    for i, (n, kv) in enumerate(lens):
        mask = np.zeros((Hkv, n, -(-kv // PAGE)), dtype=bool)
        for t in range(n):
            for h in range(Hkv):
                pages = rng.permutation((kv - n + t) // PAGE + 1)[: rng.integers(0, 7)]
                sel[q_begin[i] + t, h, rng.permutation(n_select)[: len(pages)]] = pages
                mask[h, t, pages] = True
        chosen.append(mask)
    q = torch.empty(b.n_tokens, Hkv * G, d, dtype=dt, device="cuda").normal_(generator=g)
    out, lse = torch.full_like(q, 7.0), torch.full((b.n_tokens, Hkv * G), 7.0, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, Hkv * G), dtype=torch.uint8, device="cuda")
    for _ in range(2):
        hk.heatkv_paged_sparse_attention(pool, b, q, _i32(sel), out, lse, ws)
    assert hk.heatkv_paged_status(ws) == 0
    _check(out, lse, q, k, v, lens, table, q_begin, Hkv, True, 1 / math.sqrt(d), dtype, chosen)
    assert (out[q_begin[-1]:] == 7.0).all() and (lse[q_begin[-1]:] == 7.0).all()


@pytest.mark.parametrize("n_select", [8, 12, 50, 200])
@pytest.mark.parametrize("tokens,codes", [(3, 1), (3, 127), (21, 1), (21, 127)])
def test_select_of_a_long_context(hk, tokens, codes, n_select):
    """1500 pages; scores of which many are equal (three codes) or hardly any, and of either sign."""
    n_pages, Hkv, d = 1500, 2, 64
    rng, g = np.random.default_rng(1), torch.Generator("cuda").manual_seed(1)
    pool, k, v, code, scale = _pool(hk, g, n_pages, Hkv, d, torch.bfloat16, fill=0.0)
    code.copy_(torch.randint(-codes, codes + 1, code.shape, generator=g, device="cuda"))
    scale.copy_(2.0 ** torch.randint(-2, 1, scale.shape, generator=g, device="cuda"))
    kv = n_pages * PAGE - 5
    b, table, _ = _batch(hk, rng, [(tokens, kv)], n_pages)
    q = torch.randint(-codes, codes + 1, (tokens, 4, d), generator=g, device="cuda").to(torch.bfloat16)
    q[2] = 0
    sel = torch.zeros(tokens, Hkv, n_select, dtype=torch.int32, device="cuda")
    hk.heatkv_paged_select(pool, b, q, sel, 3, 4)
    pages, cn, sn = table[0, :n_pages], code.cpu().numpy(), scale.cpu().numpy()
    for t in range(tokens):
        for h in range(Hkv):
            assert sel[t, h].tolist() == P.select(_np(q)[t, 2 * h: 2 * h + 2], cn[pages, h], sn[pages, h], kv - tokens + t, 3, 4, n_select)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("codes", [1, 127])
@pytest.mark.parametrize("requests", [3, 9, 18, 40, 100])
def test_select_of_many_requests(hk, requests, codes, d):
    """A token each, from so few that eight SMs share a token's pages to more than there are SMs; many equal scores or hardly any."""
    n_pages, Hkv, G = 300, 2, 3
    rng, g = np.random.default_rng(requests), torch.Generator("cuda").manual_seed(requests)
    pool, _, _, code, scale = _pool(hk, g, n_pages, Hkv, d, torch.bfloat16, fill=0.0)
    code.copy_(torch.randint(-codes, codes + 1, code.shape, generator=g, device="cuda"))
    scale.copy_(2.0 ** torch.randint(-2, 1, scale.shape, generator=g, device="cuda"))
    kv = [int(x) for x in rng.integers(1, n_pages * PAGE, requests)]
    kv[0], kv[-1] = n_pages * PAGE, 1
    table = _i32([rng.permutation(n_pages) for _ in range(requests)])                         # requests may share pages
    b = hk.PagedBatch.make(_i32(range(requests + 1)), _i32(kv), table, requests, 1)
    q = torch.randint(-codes, codes + 1, (requests, Hkv * G, d), generator=g, device="cuda").to(torch.bfloat16)
    sel = torch.zeros(requests, Hkv, 21, dtype=torch.int32, device="cuda")
    hk.heatkv_paged_select(pool, b, q, sel, 1, 2)
    cn, sn, tn, qn = code.cpu().numpy(), scale.cpu().numpy(), table.cpu().numpy(), _np(q)
    for t in range(requests):
        pages = tn[t, : -(-kv[t] // PAGE)]
        for h in range(Hkv):
            want = P.select(qn[t, G * h: G * h + G], cn[pages, h], sn[pages, h], kv[t] - 1, 1, 2, 21)
            assert sel[t, h].tolist() == want + [-1] * (21 - len(want)), (t, h)


def test_sparse_attention_over_lists_of_any_kind(hk):
    """Gaps in a list, entries past the token's page and past the table, an empty list, pages out of order."""
    lens = [(2, 500), (1, 64 * 6)]
    rng, g = np.random.default_rng(2), torch.Generator("cuda").manual_seed(2)
    pool, b, table, q_begin, k, v, _, _ = _filled(hk, g, rng, lens, 2, 128, torch.bfloat16)
    sel = np.full((3, 2, 5), -1)
    sel[0, 0] = [3, -1, 7, 0, 2**30]
    sel[0, 1] = [1, 2, -5, 8, 9]                           # page 8: past the token's own; 9: past the table
    sel[1, 0] = [7, 6, 5, 4, 3]
    sel[2] = [[5, -1, -1, -1, -1], [0, 1, 2, 3, 4]]
    chosen = [np.zeros((2, n, -(-kv // PAGE)), dtype=bool) for n, kv in lens]
    for t, (i, at) in enumerate([(0, 0), (0, 1), (1, 0)]):
        for h in range(2):
            for p in sel[t, h]:
                if 0 <= p < chosen[i].shape[2]:
                    chosen[i][h, at, p] = True
    q = torch.empty(3, 8, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out, lse = torch.full_like(q, 7.0), torch.full((3, 8), 7.0, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, 8), dtype=torch.uint8, device="cuda")
    hk.heatkv_paged_sparse_attention(pool, b, q, _i32(sel), out, lse, ws)
    _check(out, lse, q, k, v, lens, table, q_begin, 2, True, 1 / math.sqrt(128), "bf16", chosen)
    assert (out[1, 4:] == 0).all()


# ------------------------------------------------------------------------------------------------ all together

@pytest.mark.parametrize("pages", [0, 4])
def test_serving_loop(hk, pages):
    """Prompts of three requests, answers token by token, drafted tokens of which some are turned down, a request that ends and one that
    takes its place and its pages: every step of two layers against attention over the tokens that each request really has."""
    from paper_2605_14877_b200.paged import PagedCache
    H, Hkv, d, layers = 8, 2, 64, 2
    cache = PagedCache(layers, H, Hkv, d, n_pages=26, rows=3, max_pages=16, summaries=pages > 0)
    g = torch.Generator("cuda").manual_seed(4)
    kept = [[[np.zeros((0, Hkv, d))] * 2 for _ in range(layers)] for _ in range(3)]          # per request and layer: K, V rows
    # (new tokens, tokens kept afterwards (None: all))
    plan = [([300, 70, 0], None), ([1, 1, 0], None), ([1, 1, 640], None), ([4, 5, 1], (303, 73, 641)), ([1, 1, 1], None), ([0, 0, 1], (304, 0, 642)),
            ([1, 500, 1], None), ([1, 1, 1], None)]
    for new, keep in plan:
        step = cache.begin(new)
        lens = [len(kept[i][0][0]) for i in range(3)]
        begin = np.concatenate([[0], np.cumsum(new)])
        want_pos = np.concatenate([np.arange(lens[i], lens[i] + new[i]) for i in range(3)])
        assert np.array_equal(step.positions.cpu().numpy(), want_pos)
        assert cache.state.tolist()[2] == 0
        for layer in range(layers):
            T = sum(new)
            q = torch.empty(T, H, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
            kv = torch.empty(2, T, Hkv, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
            out, lse = torch.empty_like(q), torch.empty(T, H, device="cuda")
            cache.attend(layer, step, q, kv[0], kv[1], out, lse, pages=pages)
            for i in range(3):
                rows = slice(begin[i], begin[i + 1])
                for x in range(2):
                    kept[i][layer][x] = np.concatenate([kept[i][layer][x], _np(kv[x, rows])])
                K, V = kept[i][layer]
                n, total = new[i], len(K)
                at = np.arange(total - n, total)
                for h in range(H):
                    hk_ = h // (H // Hkv)
                    seen = np.arange(total) <= at[:, None]
                    if pages:
                        got = np.zeros_like(seen)
                        whole = [P.summary(K[p * PAGE:(p + 1) * PAGE, hk_].astype(np.float32)) for p in range(total // PAGE)] + [(np.zeros(d), 0.0)]
                        codes, scales = np.array([c for c, _ in whole]), np.array([s for _, s in whole], dtype=np.float32)
                        group = _np(q[rows, hk_ * 4: hk_ * 4 + 4])
                        for t in range(n):
                            for p in P.select(group[t], codes, scales, at[t], 1, 2, pages):
                                got[t, p * PAGE:(p + 1) * PAGE] = True
                        seen = seen & got
                    o, l, pv, reach = P.attention(_np(q[rows, h]).astype(np.float64), K[:, hk_], V[:, hk_], seen, 0.125)
                    off = (d + 8) * 2.0**-24 * reach + 2.0**-18
                    tol = 2.0**-8 * np.abs(o) + (2.0**-8 + 2 * off)[:, None] * pv + 1e-30
                    assert (np.abs(_np(out[rows, h]) - o) <= tol).all(), (new, layer, i, h)
                    assert (np.abs(lse[rows, h].cpu().numpy() - l) <= off + 2.0**-22 * np.abs(l)).all()
        if keep is not None:
            cache.keep(keep)
            for i in range(3):
                for layer in range(layers):
                    kept[i][layer] = [x[: keep[i]] for x in kept[i][layer]]
    assert hk.heatkv_paged_status(cache.workspace) == 0
    used = sum(-(-n // PAGE) for n in cache.lengths.tolist())
    assert cache.state.tolist()[1] == 26 - used
    cache.keep([0, 0, 0])
    assert cache.state.tolist()[1] == 26 and sorted(cache.free.tolist()) == list(range(26))


def test_a_host_tensor_is_refused(hk):
    pool = hk.PagedPool.make(*(torch.zeros(4, 2, 64, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    slots = _i32([0, 1, 2])
    for args in ((k.cpu(), k.cpu(), slots), (k, k, slots.cpu())):
        with pytest.raises(ValueError, match="not on the current CUDA device"):
            hk.heatkv_paged_store(pool, *args)
    with pytest.raises(ValueError, match="more than one device"):
        hk.PagedBatch.make(_i32([0, 3]), _i32([3]), _i32([[0]]).cpu(), 3, 3)
    hk.heatkv_paged_store(pool, k, k, slots)


# ------------------------------------------------------------------------------------------------ batches that begin behind token 0

@pytest.mark.parametrize("H,Hkv,d,dtype", [(16, 16, 128, "bf16"), (14, 2, 64, "fp16")])
@pytest.mark.parametrize("max_new", [1, 1000])
@pytest.mark.parametrize("ahead", [1, 5, 37])
@pytest.mark.parametrize("name", ["decode", "no_keys", "chunk_behind", "mixed"])
def test_batch_that_begins_behind_token_0(hk, name, ahead, max_new, H, Hkv, d, dtype):
    """q_begin[0] > 0 (the later requests of a larger batch): every form of selection and attention takes the requests' tokens and leaves those
    in front of them as they are."""
    lens = LENS[name]
    rng, g = np.random.default_rng(ahead), torch.Generator("cuda").manual_seed(ahead)
    dt, sink, local, n_select = DTYPES[dtype], 1, 2, 30
    pool, b0, table, q_begin, k, v, code, scale = _filled(hk, g, rng, lens, Hkv, d, dt, spare=2)
    for i, (_, kv) in enumerate(lens):
        _summaries(k, code, scale, table[i, : kv // PAGE])
    q_begin = q_begin + ahead
    T, G = b0.n_tokens + ahead, H // Hkv
    b = hk.PagedBatch.make(_i32(q_begin), *b0.tensors[1:], T, max_new)
    q = torch.empty(T, H, d, dtype=dt, device="cuda").normal_(generator=g)
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, H), dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((T, H), 7.0, device="cuda")
    hk.heatkv_paged_attention(pool, b, q, out, lse, ws)
    _check(out, lse, q, k, v, lens, table, q_begin, Hkv, True, 1 / math.sqrt(d), dtype)
    assert (out[:ahead] == 7.0).all() and (out[q_begin[-1]:] == 7.0).all()
    sel = torch.full((T, Hkv, n_select), -9, dtype=torch.int32, device="cuda")
    hk.heatkv_paged_select(pool, b, q, sel, sink, local)
    got, qf, cn, sn = sel.cpu().numpy(), _np(q), code.cpu().numpy(), scale.cpu().numpy()
    chosen = []
    for i, (n, kv) in enumerate(lens):
        pages = table[i, : -(-kv // PAGE)]
        mask = np.zeros((Hkv, n, len(pages)), dtype=bool)
        for t in range(n):
            for h in range(Hkv):
                want = P.select(qf[q_begin[i] + t, h * G:(h + 1) * G], cn[pages, h], sn[pages, h], kv - n + t, sink, local, n_select) if kv - n + t >= 0 else []
                assert got[q_begin[i] + t, h].tolist() == want + [-1] * (n_select - len(want)), (i, t, h)
                mask[h, t, want] = True
        chosen.append(mask)
    assert (got[:ahead] == -1).all() and (got[q_begin[-1]:] == -1).all()
    out.fill_(7.0), lse.fill_(7.0)
    hk.heatkv_paged_sparse_attention(pool, b, q, sel, out, lse, ws)
    assert hk.heatkv_paged_status(ws) == 0
    _check(out, lse, q, k, v, lens, table, q_begin, Hkv, True, 1 / math.sqrt(d), dtype, chosen)
    assert (out[:ahead] == 7.0).all() and (out[q_begin[-1]:] == 7.0).all() and (lse[:ahead] == 7.0).all()


# ------------------------------------------------------------------------------------------------ threads

@pytest.mark.parametrize("max_new", [1, 1 << 16])
def test_the_first_cuda_call_of_a_thread(hk, max_new):
    """A thread that has made no CUDA call of its own yet attends (by either kernel) as any other does."""
    import threading
    lens = [(2, 300), (1, 65)]
    rng, g = np.random.default_rng(11), torch.Generator("cuda").manual_seed(11)
    pool, b, table, q_begin, k, v, _, _ = _filled(hk, g, rng, lens, 2, 128, torch.bfloat16)
    b.max_new = max_new
    q = torch.empty(b.n_tokens, 4, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out, lse = torch.zeros_like(q), torch.zeros(b.n_tokens, 4, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, 4), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    raised = []

    def attend():
        try:
            hk.heatkv_paged_attention(pool, b, q, out, lse, ws)
        except Exception as e:                             # noqa: BLE001
            raised.append(e)
    thread = threading.Thread(target=attend)
    thread.start()
    thread.join()
    assert not raised, raised
    _check(out, lse, q, k, v, lens, table, q_begin, 2, True, 1 / math.sqrt(128), "bf16")


def _in_two_threads(calls, rounds):
    """calls[i]() again and again in thread i, all at once; what they raised."""
    import threading
    raised, start = [], threading.Barrier(len(calls))

    def loop(call):
        stream = torch.cuda.Stream()
        start.wait()
        try:
            for _ in range(rounds):
                call(stream)
        except Exception as e:                             # noqa: BLE001  (reported by the caller)
            raised.append(e)
        stream.synchronize()
    threads = [threading.Thread(target=loop, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    return raised


@pytest.mark.parametrize("what", ["tables", "attention", "select", "select_chunk"])
def test_calls_of_two_threads(hk, what):
    """Calls of different sizes from two threads, each with buffers and a stream of its own: every one is made, and gives what it gives alone."""
    g = torch.Generator("cuda").manual_seed(6)
    Hkv, d = 2, 128
    pool, *_ = _pool(hk, g, 8, Hkv, d, torch.bfloat16, fill=0.0)
    calls, results = [], []
    for n, width in ((4000, 6000), (3300, 3200)) if what == "tables" else ((600, 3000), (20, 2000)) if what == "select_chunk" else ((1000, 24000), (20, 9000)):
        if what == "tables":
            out = [_i32([0] * 4), torch.full((n, 4), -1, dtype=torch.int32, device="cuda"), _i32([0] * (n + 1)), _i32([0] * n), _i32([0] * n)]
            args = _i32([1] * n), _i32([0] * n), _i32(range(n)), _i32([0, n, 0, 0])
            calls.append(lambda s, a=args, o=out: hk.heatkv_paged_tables(*a, *o, stream=s))
            results.append(out)
            continue
        rows = 20 if what == "select_chunk" else 1
        kv = width * PAGE if what != "attention" else 8 * PAGE - 5
        table = _i32([list(range(8)) + [-1] * (width - 8)] * (n // rows)) if what != "attention" else _i32([list(range(8))] * n)
        b = hk.PagedBatch.make(_i32(range(0, n + 1, rows)), _i32([kv] * (n // rows)), table, n, rows)
        q = torch.empty(n, 4, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        if what == "attention":
            out = torch.zeros_like(q)
            ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, 4), dtype=torch.uint8, device="cuda")
            calls.append(lambda s, b=b, q=q, o=out, w=ws: hk.heatkv_paged_attention(pool, b, q, o, None, w, stream=s))
        else:
            out = torch.zeros(n, Hkv, 12, dtype=torch.int32, device="cuda")
            calls.append(lambda s, b=b, q=q, o=out: hk.heatkv_paged_select(pool, b, q, o, 1, 2, stream=s))
        results.append([out])
    alone = []
    torch.cuda.synchronize()
    for call, out in zip(calls, results):
        call(None)
        alone.append([x.clone() for x in out])
    torch.cuda.synchronize()
    raised = _in_two_threads(calls, 1500)
    assert not raised, raised
    for a, r in zip(alone, results):
        assert all(torch.equal(x, y) for x, y in zip(a, r))


# ------------------------------------------------------------------------------------------------ NaN and infinity in a query

@pytest.mark.parametrize("form", ["small", "large", "selected", "selected_chunk"])
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "bf16"), (64, "fp16")])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_query_that_is_no_number_shows(hk, form, d, dtype, bad):
    """A row whose query holds NaN or an infinity is NaN, its logarithm too: minus infinity would say that it saw no key.  Rows beside it and
    rows without keys are as ever."""
    lens = [(9, 700), (1, 65), (3, 0), (20, 20), (1, 5000)]
    Hkv, G, n_select = 2, 4, 96
    rng, g = np.random.default_rng(8), torch.Generator("cuda").manual_seed(8)
    dt = DTYPES[dtype]
    pool, b, table, q_begin, k, v, _, _ = _filled(hk, g, rng, lens, Hkv, d, dt)
    for x in k:                                            # (an infinity times keys of either sign is minus infinity for half of them)
        x[..., 0].abs_()
    T, H = b.n_tokens, Hkv * G
    q = torch.empty(T, H, d, dtype=dt, device="cuda").normal_(generator=g)
    clean = q.clone()
    hit = [(q_begin[0] + 4, 5), (q_begin[1], 0), (q_begin[2] + 1, 2), (q_begin[3], 7), (q_begin[3] + 19, 1), (q_begin[4], 3)]
    for t, h in hit:
        q[t, h, 0] = bad
    b.max_new = 1 << 16 if form in ("large", "selected_chunk") else 1
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, H), dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((T, H), 7.0, device="cuda")
    chosen = None
    if form in ("small", "large"):
        hk.heatkv_paged_attention(pool, b, q, out, lse, ws)
    else:
        n_select = 2048 // (2 * 32) if form == "selected_chunk" else n_select
        sel = np.tile(np.concatenate([np.arange(n_select - 1), [-1]]), (T, Hkv, 1))
        if form == "selected_chunk":                       # as many lists as it takes for them to be merged
            hk_rows = 24576 // (Hkv * n_select) + 1
            pad = max(hk_rows - T, 0)
            b = hk.PagedBatch.make(*b.tensors, T + pad, 1 << 16)
            q, sel = torch.cat([q, q.new_zeros(pad, H, d)]), np.concatenate([sel, np.full((pad, Hkv, n_select), -1)])
            clean = torch.cat([clean, clean.new_zeros(pad, H, d)])
            out, lse = torch.full_like(q, 7.0), torch.full((T + pad, H), 7.0, device="cuda")
            ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, H), dtype=torch.uint8, device="cuda")
        chosen = [np.broadcast_to(np.arange(-(-kv // PAGE)) < n_select - 1, (Hkv, n, -(-kv // PAGE))) for n, kv in lens]
        hk.heatkv_paged_sparse_attention(pool, b, q, _i32(sel), out, lse, ws)
    assert hk.heatkv_paged_status(ws) == 0
    for t, h in hit:
        if q_begin[2] <= t < q_begin[3]:                   # no keys
            assert (out[t, h] == 0).all() and lse[t, h].item() == -math.inf
        else:
            assert out[t, h].isnan().all() and lse[t, h].isnan(), (t, h, out[t, h, :4], lse[t, h])
        out[t, h], lse[t, h] = 0.0, 0.0                    # (the rest against 64 bits; these rows' queries see nothing there)
    for t, h in hit:
        clean[t, h] = 0
    rest = torch.ones(T, H, dtype=torch.bool, device="cuda")
    for t, h in hit:
        rest[t, h] = False
    # the rows beside them: the same bits as without the bad ones
    want, want_lse = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
    if chosen is None:
        hk.heatkv_paged_attention(pool, b, clean, want, want_lse, ws)
    else:
        hk.heatkv_paged_sparse_attention(pool, b, clean, _i32(sel), want, want_lse, ws)
    _check(want[:T], want_lse[:T], clean[:T], k, v, lens, table, q_begin, Hkv, True, 1 / math.sqrt(d), dtype, chosen)
    assert torch.equal(out[:T][rest], want[:T][rest]) and torch.equal(lse[:T][rest], want_lse[:T][rest])


@pytest.mark.parametrize("form", ["small", "large"])
@pytest.mark.parametrize("d", [64, 128])
def test_logits_of_minus_infinity(hk, form, d):
    """A row all of whose logits are minus infinity: no weight anywhere, zero and minus infinity, whichever kernel has it."""
    lens = [(3, 200), (1, 3000)]
    rng, g = np.random.default_rng(9), torch.Generator("cuda").manual_seed(9)
    pool, b, table, q_begin, k, v, _, _ = _filled(hk, g, rng, lens, 2, d, torch.bfloat16)
    k[..., 0] = 1.0
    b.max_new = 1 << 16 if form == "large" else 1
    q = torch.empty(4, 4, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    q[1, 2, 0] = q[3, 0, 0] = -math.inf
    out, lse = torch.full_like(q, 7.0), torch.full((4, 4), 7.0, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, 4), dtype=torch.uint8, device="cuda")
    hk.heatkv_paged_attention(pool, b, q, out, lse, ws)
    for t, h in ((1, 2), (3, 0)):
        assert (out[t, h] == 0).all() and lse[t, h].item() == -math.inf
    assert out.isfinite().all() and lse.isfinite().sum() == 14


@pytest.mark.parametrize("max_new", [1, 1 << 16])
@pytest.mark.parametrize("d", [64, 128])
def test_a_key_that_a_row_does_not_see_has_no_weight(hk, d, max_new):
    """Values near the type's largest behind a row's own position leave it as it is: their weight is zero,
    not merely small."""
    lens = [(150, 300), (70, 70)]
    rng, g = np.random.default_rng(10), torch.Generator("cuda").manual_seed(10)
    pool, b, table, q_begin, k, v, _, _ = _filled(hk, g, rng, lens, 2, d, torch.bfloat16)
    b.max_new = max_new
    for i, (n, kv) in enumerate(lens):                     # the last 40 tokens' values
        for p in range(kv - 40, kv):
            v[table[i, p // PAGE], :, p % PAGE] = 3e38
    q = torch.empty(b.n_tokens, 4, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out, lse = torch.zeros_like(q), torch.zeros(b.n_tokens, 4, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, 4), dtype=torch.uint8, device="cuda")
    hk.heatkv_paged_attention(pool, b, q, out, lse, ws)
    # the requests without their last 40 tokens
    short = [(n - 40, kv - 40) for n, kv in lens]
    begin = [q_begin[0], q_begin[1]]
    _check(out, lse, q, k, v, short, table, begin, 2, True, 1 / math.sqrt(d), "bf16")


# ------------------------------------------------------------------------------------------------ calls that give up

@pytest.mark.parametrize("G,max_new", [(4, 1), (64, 1), (4, 1 << 16)])
def test_calls_on_a_workspace_whose_status_is_set(hk, G, max_new):
    """After a wait has run out, calls on the workspace end at once whatever the kernels before have left in it; zeroed, it serves again."""
    lens = [(1, 3000), (3, 700), (1, 64 * 40)]
    Hkv, n_select = 2, 32
    rng, g = np.random.default_rng(12), torch.Generator("cuda").manual_seed(12)
    pool, b0, table, q_begin, k, v, _, _ = _filled(hk, g, rng, lens, Hkv, 128, torch.bfloat16)
    T = 5 if max_new == 1 else 400                         # (rows that are nobody's: as many lists as it takes for them to be merged)
    b = hk.PagedBatch.make(*b0.tensors, T, max_new)
    q = torch.empty(T, Hkv * G, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    sel = np.full((T, Hkv, n_select), -1)
    sel[:5] = np.arange(n_select)
    sel, chosen = _i32(sel), [np.broadcast_to(np.arange(-(-kv // PAGE)) < n_select, (Hkv, n, -(-kv // PAGE))) for n, kv in lens]
    out, lse = torch.full_like(q, 7.0), torch.full((T, Hkv * G), 7.0, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, Hkv * G), dtype=torch.uint8, device="cuda")
    words = ws.view(torch.int32)
    head = 64 + 8192                                       # status and counters; behind them what kernels hand to one another
    for entry in ([2**31 - 5, 20], [5, -2**31 + 7], [2**30, 40000], [3, 2**31 - 60000], [900, 300], None):
        words.zero_()
        if entry is None:
            words[head:] = torch.randint(-2**31, 2**31 - 1, (len(words) - head,), generator=g, device="cuda").int()
        else:
            words[head: head + 2 * (len(words[head:]) // 2)].view(-1, 2)[:] = _i32(entry)
        words[0] = 1
        hk.heatkv_paged_attention(pool, b, q, out, lse, ws)
        hk.heatkv_paged_sparse_attention(pool, b, q, sel, out, lse, ws)
        assert hk.heatkv_paged_status(ws) == -7
    words.zero_()
    out.fill_(7.0), lse.fill_(7.0)
    hk.heatkv_paged_attention(pool, b, q, out, lse, ws)
    _check(out, lse, q, k, v, lens, table, q_begin, Hkv, True, 1 / math.sqrt(128), "bf16")
    hk.heatkv_paged_sparse_attention(pool, b, q, sel, out, lse, ws)
    _check(out, lse, q, k, v, lens, table, q_begin, Hkv, True, 1 / math.sqrt(128), "bf16", chosen)
    assert hk.heatkv_paged_status(ws) == 0


def test_plan_of_a_call_whose_key_tiles_pass_32_bits(hk):
    """Half a million new tokens of 128 heads a group behind a million and a half: 3.8e9 key tiles a kv head.  The call is made on a workspace whose
    status is set, so that its plan is made and nothing else (the attention would take minutes); every SM's run of the plan is looked at."""
    n, kv, Hkv, G = 1 << 19, 1 << 21, 2, 128
    k, v = (torch.zeros(1, Hkv, PAGE, 64, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    pool = hk.PagedPool.make(k, v)
    b = hk.PagedBatch.make(_i32([0, n]), _i32([kv]), torch.full((1, kv // PAGE), -1, dtype=torch.int32, device="cuda"), n, n)
    q, out = (torch.zeros((n + Hkv * G) * 64, dtype=torch.bfloat16, device="cuda").as_strided((n, Hkv * G, 64), (64, 64, 1)) for _ in range(2))
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, Hkv * G), dtype=torch.uint8, device="cuda")
    words = ws.view(torch.int32)
    words[0] = 1
    hk.heatkv_paged_attention(pool, b, q, out, None, ws)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    runs = words[64 + 8192:][: sms * 10].view(sms, 10).cpu().numpy()             # behind the status and the counters
    # what the plan has to say: items of two tokens, a unit for each of their key tiles and one for their end
    upto = kv - n + 2 * (np.arange(n // 2, dtype=np.int64) + 1)
    tiles = -(-upto // 128)
    begin = np.concatenate([[0], np.cumsum(tiles + 1)])
    per_head = int(begin[-1])
    assert per_head > 2**31
    bound = [per_head * Hkv * c // sms for c in range(sms + 1)]
    for c in range(sms):
        seq, head, item, j0 = (int(x) for x in runs[c, :4])
        units = int(runs[c, 4:6].copy().view(np.int64)[0])
        y = head * per_head + int(begin[item]) + j0
        h, at = divmod(bound[c], per_head)
        i = int(np.searchsorted(begin, at, side="right")) - 1
        ends = at - int(begin[i]) == tiles[i]              # a run that would begin with an item's end begins with the next item
        assert (seq, y, units) == (0, bound[c] + ends, bound[c + 1] - bound[c] - ends), c
        assert 0 <= head < Hkv and 0 <= j0 < tiles[item]
        first = [x for x in range(sms) if bound[x] <= head * per_head + begin[item] < bound[x + 1]]
        assert [int(runs[c, 6])] == first


def test_cache_of_rows_that_are_refused(hk):
    """Rows that find no pages, or would outgrow their row of the table, sit a step out and say so; the others go on, and the tokens may come again."""
    from paper_2605_14877_b200.paged import PagedCache
    H, Hkv, d, rows = 4, 2, 64, 4
    cache = PagedCache(1, H, Hkv, d, n_pages=6, rows=rows, max_pages=5)
    g = torch.Generator("cuda").manual_seed(13)
    kept = [[np.zeros((0, Hkv, d))] * 2 for _ in range(rows)]

    def step_of(new, refused):
        step, before = cache.begin(new), [len(x[0]) for x in kept]
        T, begin = sum(new), np.concatenate([[0], np.cumsum(new)])
        served = [0 if i in refused else before[i] + new[i] for i in range(rows)]
        assert step.kv_len.tolist() == served and cache.state.tolist()[2] == len(refused)
        assert cache.lengths.tolist() == [before[i] if i in refused else served[i] for i in range(rows)]
        assert ((step.slots == -1).cpu().numpy() == np.isin(np.repeat(np.arange(rows), new), refused)).all()
        q = torch.empty(T, H, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        kv = torch.empty(2, T, Hkv, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        out, lse = torch.full_like(q, 7.0), torch.full((T, H), 7.0, device="cuda")
        cache.attend(0, step, q, kv[0], kv[1], out, lse)
        for i in range(rows):
            at = slice(begin[i], begin[i + 1])
            if i in refused:
                assert (out[at] == 0).all() and (lse[at] == -math.inf).all()
                continue
            kept[i] = [np.concatenate([x, _np(kv[j, at])]) for j, x in enumerate(kept[i])]
            K, V = kept[i]
            seen = np.arange(len(K)) <= np.arange(len(K) - new[i], len(K))[:, None]
            for h in range(H):
                o, l, pv, reach = P.attention(_np(q[at, h]).astype(np.float64), K[:, h // 2], V[:, h // 2], seen, 0.125)
                off = (d + 8) * 2.0**-24 * reach + 2.0**-18
                assert (np.abs(_np(out[at, h]) - o) <= 2.0**-8 * np.abs(o) + (2.0**-8 + 2 * off)[:, None] * pv + 1e-30).all()
                assert (np.abs(lse[at, h].cpu().numpy() - l) <= off + 2.0**-22 * np.abs(l)).all()

    step_of([60, 100, 0, 64], [])                          # 1 + 2 + 1 pages of 6
    step_of([3, 200, 65, 1], [1, 2, 3])                    # row 0 has room in its page; row 1 wants 3 pages of 2, and all behind it are refused
    step_of([300, 1, 65, 1], [0, 3])                       # row 0 would outgrow its row; row 1 has room, row 2 takes the last two pages
    cache.keep([63, 0, 65, 64])
    kept[1] = [x[:0] for x in kept[1]]
    step_of([1, 70, 1, 1], [3])                            # row 1 takes the two pages that came back
    assert cache.state.tolist()[1] == 0
    cache.keep([0, 0, 0, 0])
    assert sorted(cache.free.tolist()) == list(range(6)) and cache.state.tolist()[1] == 6


def test_a_wait_that_runs_out(hk):
    """The paged kernels' own bounded waits, on a barrier that nothing signals: they give up, the status says so until the workspace is zeroed, and
    a cache's check raises once and leaves a cache that serves, also where its workspace grew in between."""
    from paper_2605_14877_b200.paged import PagedCache
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    assert hk.heatkv_paged_status(ws) == 0
    assert hk.heatkv_paged_selftest_wait_expiry(ws) == -7 and hk.heatkv_paged_status(ws) == -7
    assert (ws[4:] == 0).all()
    assert hk.heatkv_paged_selftest_wait_expiry(ws) == -7      # (the first code stays)
    ws.zero_()
    assert hk.heatkv_paged_status(ws) == 0

    H, Hkv, d = 4, 2, 64
    cache = PagedCache(1, H, Hkv, d, n_pages=210, rows=2, max_pages=200)
    cache.check()                                              # nothing has run yet
    g = torch.Generator("cuda").manual_seed(14)
    rows = lambda n, heads: torch.empty(n, heads, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)      # noqa: E731
    step = cache.begin([1, 1])
    q, k, v = rows(2, H), rows(2, Hkv), rows(2, Hkv)
    cache.attend(0, step, q, k, v, torch.empty_like(q))
    cache.check()
    for again in range(2):
        assert hk.heatkv_paged_selftest_wait_expiry(cache.workspace) == -7
        size = cache.workspace.numel()
        step = cache.begin([6000, 1 + again])                  # (its workspace is larger the first time)
        assert again == 1 or cache.workspace.numel() > size
        q, k, v = rows(6001 + again, H), rows(6001 + again, Hkv), rows(6001 + again, Hkv)
        out = torch.full_like(q, 7.0)
        cache.attend(0, step, q, k, v, out)
        with pytest.raises(hk.HeatKVError, match="-7"):
            cache.check()
        cache.check()
        cache.attend(0, step, q, k, v, out)
        cache.check()
        want = torch.zeros_like(out)
        pool = cache.pools[0]
        hk.heatkv_paged_attention(pool, step.batch, q, want, None,
                                  torch.zeros(hk.heatkv_paged_workspace_bytes(pool, step.batch, H), dtype=torch.uint8, device="cuda"))
        assert torch.equal(out, want) and (out != 7.0).any(-1).all()


# ------------------------------------------------------------------------------------------------ many requests

def _many(hk, seed, new, kv, Hkv, d, dt):
    """A pool of requests' pages in random order, NaN past every request's last key; everything by whole tensors."""
    g, rng = torch.Generator("cuda").manual_seed(seed), np.random.default_rng(seed)
    held = -(-np.asarray(kv) // PAGE)
    n_pages, width = int(held.sum()) + 2, int(held.max()) + 1
    table = np.full((len(kv), width), -1)
    row, col = np.repeat(np.arange(len(kv)), held), np.concatenate([np.arange(h) for h in held])
    table[row, col] = rng.permutation(n_pages)[: len(row)]
    pool, k, v, code, scale = _pool(hk, g, n_pages, Hkv, d, dt)
    empty = torch.ones(n_pages, PAGE, dtype=torch.bool, device="cuda")
    pages = torch.tensor(table[row, col], device="cuda")
    left = torch.tensor(np.asarray(kv)[row] - col * PAGE, device="cuda")
    empty[pages] = torch.arange(PAGE, device="cuda") >= left[:, None]
    for x in (k, v):
        x.normal_(generator=g)
        x.masked_fill_(empty[:, None, :, None], math.nan)
    q_begin = np.concatenate([[0], np.cumsum(new)])
    b = hk.PagedBatch.make(_i32(q_begin), _i32(kv), _i32(table), int(q_begin[-1]), int(max(new)))
    return pool, b, k, v, code, scale, g


def _check_many(out, lse, q, k, v, b, dtype, sel=None):
    """_check by whole tensors on the device, causal, 1 / sqrt(d): every row of every request against 64 bits."""
    u = 2.0**-8 if dtype == "bf16" else 2.0**-11
    q_begin, kv, table = (x.long() for x in b.tensors)
    T, H, d = q.shape
    Hkv = k.shape[1]
    G, scale, new = H // Hkv, 1 / math.sqrt(d), q_begin[1:] - q_begin[:-1]
    for lo in range(0, len(kv), 64):
        ids = slice(lo, min(lo + 64, len(kv)))
        n, most, pages = new[ids], max(int(new[ids].max()), 1), max(-(-int(kv[ids].max()) // PAGE), 1)
        t = torch.arange(most, device="cuda")
        at = (q_begin[:-1][ids, None] + t).clamp(max=T - 1)
        keys, values = (x[table[ids, :pages].clamp(min=0)].transpose(1, 2).flatten(2, 3).double().nan_to_num() for x in (k, v))     # [r, Hkv, keys, d]
        qq = q[at].double().view(len(n), most, Hkv, G, d)
        j = torch.arange(pages * PAGE, device="cuda")
        pos = (kv[ids] - n)[:, None] + t                                         # [r, t]
        seen = ((j < kv[ids, None])[:, None] & (j <= pos[..., None]))[:, None, None]   # [r, 1, 1, t, keys]
        if sel is not None:
            took = torch.zeros(len(n), most, Hkv, pages + 1, dtype=torch.bool, device="cuda")
            place = sel[at].long()
            took.scatter_(3, torch.where((place < 0) | (place >= pages), pages, place), True)
            seen = seen & took[..., :pages].repeat_interleave(PAGE, -1).permute(0, 2, 1, 3)[:, :, None]
        logits = torch.einsum("rthgd,rhkd->rhgtk", qq, keys).mul_(scale).masked_fill_(~seen, -math.inf)
        want_lse = torch.logsumexp(logits, -1)
        p = torch.exp(logits - want_lse.clamp(min=-1e300)[..., None])
        o, pv = torch.einsum("rhgtk,rhkd->rthgd", p, values), torch.einsum("rhgtk,rhkd->rthgd", p, values.abs())
        reach = (torch.einsum("rthgd,rhkd->rhgtk", qq.abs(), keys.abs()) * scale * seen).amax(-1).permute(0, 3, 1, 2)
        want_lse = want_lse.permute(0, 3, 1, 2)
        off = (d + 8) * 2.0**-24 * reach + 2.0**-18
        small = pages * PAGE * 2.0**-25 * values.abs().max() if dtype == "fp16" else 0.0
        tol = u * o.abs() + (u + 2 * off)[..., None] * pv + small + 1e-30
        real = t < n[:, None]
        got, got_lse = out[at].double().view_as(o), lse[at].double().view_as(want_lse)
        assert got[real].isfinite().all()
        assert ((got - o).abs() <= tol)[real].all(), lo
        assert torch.equal(got_lse.isinf()[real], want_lse.isinf()[real])
        fine = (got_lse - want_lse).abs() <= off + 2.0**-22 * want_lse.abs()
        assert (fine | want_lse.isinf())[real].all(), lo


MANY = {
    # more requests than threads that plan, most short, a few long, some without keys or new tokens
    "few_tokens": dict(n=4096, new=(0, 3), H=8, Hkv=2, d=64, dtype="bf16"),
    "wide_group": dict(n=1500, new=(1, 4), H=48, Hkv=3, d=128, dtype="fp16"),
    # more items than the plan keeps in shared memory
    "many_items": dict(n=4096, new=(6, 8), H=128, Hkv=1, d=64, dtype="bf16"),
}


def _many_lens(c, seed):
    rng = np.random.default_rng(seed)
    new = rng.integers(c["new"][0], c["new"][1] + 1, c["n"])
    kv = new + rng.integers(0, 150, c["n"])
    kv[:: 97] = 1200 + rng.integers(0, 400, len(kv[:: 97]))
    kv[5:: 301] = 0
    kv[7:: 301] = 1                                        # (fewer than the new tokens)
    return new, kv


@pytest.mark.parametrize("max_new", [1, 1 << 16])
@pytest.mark.parametrize("name", MANY)
def test_attention_of_many_requests(hk, name, max_new):
    c = MANY[name]
    new, kv = _many_lens(c, 21)
    pool, b, k, v, _, _, g = _many(hk, 21, new, kv, c["Hkv"], c["d"], DTYPES[c["dtype"]])
    b.max_new = max_new
    q = torch.empty(b.n_tokens, c["H"], c["d"], dtype=DTYPES[c["dtype"]], device="cuda").normal_(generator=g)
    out, lse = torch.full_like(q, math.nan), torch.full((b.n_tokens, c["H"]), math.nan, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, c["H"]), dtype=torch.uint8, device="cuda")
    hk.heatkv_paged_attention(pool, b, q, out, lse, ws)
    assert hk.heatkv_paged_status(ws) == 0
    _check_many(out, lse, q, k, v, b, c["dtype"])


@pytest.mark.parametrize("max_new", [1, 1 << 16])
@pytest.mark.parametrize("Hkv,G,d", [(4, 2, 64), (8, 1, 128), (2, 16, 128)])
def test_sparse_attention_of_many_requests(hk, Hkv, G, d, max_new):
    """As many lists (4096 requests, 2 or more kv heads) as their sums do not fit shared memory for, with gaps and in any order; both kernels."""
    new, kv = _many_lens(dict(n=4096, new=(0, 3)), 22)
    pool, b, k, v, _, _, g = _many(hk, 22, new, kv, Hkv, d, torch.bfloat16)
    b.max_new = max_new
    T, H, n_select = b.n_tokens, Hkv * G, 9
    q = torch.empty(T, H, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    order = torch.rand(T, Hkv, 26, generator=g, device="cuda").argsort(-1)[..., :n_select]      # distinct pages, some past the request's last
    sel = torch.where(torch.rand(T, Hkv, n_select, generator=g, device="cuda") < 0.2, -1, order).int().contiguous()
    out, lse = torch.full_like(q, math.nan), torch.full((T, H), math.nan, device="cuda")
    ws = torch.zeros(hk.heatkv_paged_workspace_bytes(pool, b, H), dtype=torch.uint8, device="cuda")
    hk.heatkv_paged_sparse_attention(pool, b, q, sel, out, lse, ws)
    assert hk.heatkv_paged_status(ws) == 0
    _check_many(out, lse, q, k, v, b, "bf16", sel)


@pytest.mark.parametrize("H,Hkv,d,dtype", [(14, 2, 64, "fp16"), (16, 4, 128, "bf16")])
def test_select_of_single_tokens_between_chunks(hk, H, Hkv, d, dtype):
    """Chunks and single tokens in one batch, more requests than 16 tokens have: both forms of selection give the definition's pages."""
    new = np.array([1, 40, 1, 1, 0, 1, 17, 1, 1, 1, 2, 0, 0, 1, 1, 16, 1] + [1] * 40 + [33])
    rng = np.random.default_rng(23)
    kv = new + rng.integers(0, 3000, len(new))
    kv[[3, 6]] = 0, 5                                      # no keys, and fewer than the new tokens
    pool, b, k, v, code, scale, g = _many(hk, 23, new, kv, Hkv, d, DTYPES[dtype])
    code.copy_(torch.randint(-127, 128, code.shape, generator=g, device="cuda"))
    scale.uniform_(0.5, 2.0, generator=g)
    q = torch.empty(b.n_tokens, H, d, dtype=DTYPES[dtype], device="cuda").normal_(generator=g)
    q_begin, _, table = (x.cpu().numpy() for x in b.tensors)
    qf, cn, sn, G, n_select = _np(q), code.cpu().numpy(), scale.cpu().numpy(), H // Hkv, 12
    for max_new in (1, 40):
        b.max_new = max_new
        sel = torch.full((b.n_tokens, Hkv, n_select), -9, dtype=torch.int32, device="cuda")
        hk.heatkv_paged_select(pool, b, q, sel, 2, 3)
        got = sel.cpu().numpy()
        for i, n in enumerate(new):
            pages = table[i, : -(-kv[i] // PAGE)]
            for t in range(n):
                at = kv[i] - n + t
                for h in range(Hkv):
                    want = P.select(qf[q_begin[i] + t, h * G:(h + 1) * G], cn[pages, h], sn[pages, h], at, 2, 3, n_select) if at >= 0 else []
                    assert got[q_begin[i] + t, h].tolist() == want + [-1] * (n_select - len(want)), (max_new, i, t, h)


def test_one_workspace_for_calls_of_all_kinds(hk):
    """A workspace of the largest batch serves smaller ones of either kernel in any order, with the bits that one of its own gives."""
    H, Hkv, d = 16, 4, 128
    cases = []
    for seed, (n, new, more) in enumerate(((40, (30, 90), 3000), (7, (1, 1), 9000), (300, (1, 4), 500), (3, (200, 300), 100), (60, (1, 1), 4000))):
        rng = np.random.default_rng(seed)
        lens = rng.integers(new[0], new[1] + 1, n)
        pool, b, k, v, _, _, g = _many(hk, seed, lens, lens + rng.integers(0, more, n), Hkv, d, torch.bfloat16)
        q = torch.empty(b.n_tokens, H, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        sel = torch.rand(b.n_tokens, Hkv, 47, generator=g, device="cuda").argsort(-1)[..., :32].int().contiguous()
        cases.append((pool, b, q, sel, hk.heatkv_paged_workspace_bytes(pool, b, H)))
    ws = torch.zeros(max(c[-1] for c in cases), dtype=torch.uint8, device="cuda")
    order = [0, 1, 2, 3, 4, 1, 0, 4, 3, 2, 0]
    for i in order:
        pool, b, q, sel, size = cases[i]
        own = torch.zeros(size, dtype=torch.uint8, device="cuda")
        got, want = ([torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")] for _ in range(2))
        for call in (lambda o, w: hk.heatkv_paged_attention(pool, b, q, *o, w), lambda o, w: hk.heatkv_paged_sparse_attention(pool, b, q, sel, *o, w)):
            call(got, ws), call(want, own)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and (want[1] != 7.0).all(), i
    assert hk.heatkv_paged_status(ws) == 0


def _check_select(pool_codes, b, q, lens, Hkv, sel, sink, local, tokens=None):
    """Every token's list (or those of `tokens`) against the definition."""
    code, scale = (x.cpu().numpy() for x in pool_codes)
    (q_begin, _, table), qf, got, G, n_select = (x.cpu().numpy() for x in b.tensors), _np(q), sel.cpu().numpy(), q.shape[1] // Hkv, sel.shape[2]
    for i, (n, kv) in enumerate(lens):
        pages = table[i, : -(-kv // PAGE)]
        for t in range(n):
            if tokens is not None and q_begin[i] + t not in tokens:
                continue
            for h in range(Hkv):
                at = kv - n + t
                want = P.select(qf[q_begin[i] + t, h * G:(h + 1) * G], code[pages, h], scale[pages, h], at, sink, local, n_select) if at >= 0 else []
                assert got[q_begin[i] + t, h].tolist() == want + [-1] * (n_select - len(want)), (i, t, h)


def _select_batch(hk, seed, lens, Hkv, G, d, codes=127):
    pool, b, _, _, code, scale, g = _many(hk, seed, [n for n, _ in lens], [kv for _, kv in lens], Hkv, d, torch.bfloat16)
    code.copy_(torch.randint(-codes, codes + 1, code.shape, generator=g, device="cuda"))
    scale.copy_(2.0 ** torch.randint(-2, 1, scale.shape, generator=g, device="cuda"))
    q = torch.randint(-codes, codes + 1, (b.n_tokens, Hkv * G, d), generator=g, device="cuda").to(torch.bfloat16)
    return pool, b, q, (code, scale)


@pytest.mark.parametrize("n_select", [8, 40, 100, 200])
@pytest.mark.parametrize("codes", [1, 127])
def test_select_of_a_long_context_by_many_tokens(hk, codes, n_select):
    """1500 pages chosen from by as many tokens as it takes for 16 of them to share a CTA; many equal scores or hardly any."""
    lens = [(333, 1500 * PAGE - 5)]
    pool, b, q, summaries = _select_batch(hk, 31, lens, 2, 2, 64, codes)
    q[2] = 0
    sel = torch.zeros(333, 2, n_select, dtype=torch.int32, device="cuda")
    hk.heatkv_paged_select(pool, b, q, sel, 3, 4)
    _check_select(summaries, b, q, lens, 2, sel, 3, 4, set(range(0, 333, 4)) | {2, 331, 332})


def test_select_of_a_chunk_beside_as_many_single_tokens_as_share_a_cta(hk):
    """A chunk long enough that 16 tokens share a CTA whosever they are, single tokens in front of it and behind it."""
    lens = [(1, 500 + 37 * i) for i in range(20)] + [(0, 77), (600, 3000), (1, 0), (2, 1)] + [(1, 64 * i + 1) for i in range(37)] + [(3, 900)]
    pool, b, q, summaries = _select_batch(hk, 32, lens, 16, 1, 64)
    sel = torch.zeros(b.n_tokens, 16, 9, dtype=torch.int32, device="cuda")
    hk.heatkv_paged_select(pool, b, q, sel, 1, 2)
    _check_select(summaries, b, q, lens, 16, sel, 1, 2, set(range(0, 30)) | set(range(30, 600, 50)) | set(range(600, b.n_tokens)))


def test_select_of_a_chunk_beside_single_tokens_takes_no_longer_than_both(hk):
    """One request of 8 new tokens among 64 of one: all of them had been sent through the form in which 16 tokens share a CTA, which takes a request
    after another (108 us where a token a CTA takes 11).  Four times the single tokens' own time is far above any noise."""
    times = []
    for lens in ([(1, 20000)] * 64, [(8, 20000)] + [(1, 20000)] * 64):
        pool, b, q, _ = _select_batch(hk, 33, lens, 8, 4, 128)
        sel = torch.zeros(b.n_tokens, 8, 16, dtype=torch.int32, device="cuda")
        for _ in range(3):
            hk.heatkv_paged_select(pool, b, q, sel, 1, 2)
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        best = math.inf
        for _ in range(5):
            begin.record()
            for _ in range(30):
                hk.heatkv_paged_select(pool, b, q, sel, 1, 2)
            end.record()
            torch.cuda.synchronize()
            best = min(best, begin.elapsed_time(end))
        times.append(best)
    assert times[1] < 4 * times[0], times
