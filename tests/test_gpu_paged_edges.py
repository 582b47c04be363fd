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


# ------------------------------------------------------------------------------------------------ kernels

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,n_seq,G", [(1, 250, 2), (1, 160, 12), (70, 19, 2)])
def test_one_heavy_key_and_very_many_light_ones(hk, new, n_seq, G, d, dtype):
    """A key that holds most of the weight and 262 143 whose weights are 2^-25.5 of its: together half a percent of the output.  (All of a request's pages but the
    first are the same one, and there are so many requests that most are no two warps' or CTAs' work.)

    Weights are rounded to 16 bits, in fp16 to half of 2^-24 at least where they are subnormal.  They are held against a reference that the heaviest key
    is 2^7 above, or more, so that is 2^-32 of the whole for each of them; beyond that the roundings of weights and output, u each, and the 32-bit
    logits and exponentials as elsewhere, which move a weight by 2 ((d + 8) 2^-24 |q k| scale + 2^-18).  Sums of 32 bits, each rounded to 2^-24 of what is
    there already: a page's 64 weights and its products with values are added up first, at the coarsest, so there are a page's eight additions
    a thread and 4 096 to the sum, and of products four (of sixteen keys) a page, whose additions are off by 2^-23."""
    pages, Hkv, u = 4096, 8, 2.0**-8 if dtype == "bf16" else 2.0**-11
    blocks = torch.zeros(2, Hkv, hk.PagedPool4.block_bytes(d), dtype=torch.uint8, device="cuda")
    pool = hk.PagedPool4.make(blocks, d, DTYPES[dtype])
    k, v = torch.zeros(2 * PAGE, Hkv, d, dtype=DTYPES[dtype], device="cuda"), torch.ones(2 * PAGE, Hkv, d, dtype=DTYPES[dtype], device="cuda")
    k[0, :, 0], v[0] = 7.0, 0.0
    hk.heatkv_paged4_store(pool, k, v, _i32(range(2 * PAGE)))
    table = torch.ones(n_seq, pages, dtype=torch.int32, device="cuda")
    table[:, 0] = 0
    b = hk.PagedBatch.make(_i32(np.arange(n_seq + 1) * new), _i32([pages * PAGE] * n_seq), table, n_seq * new, new)
    q = torch.zeros(n_seq * new, Hkv * G, d, dtype=DTYPES[dtype], device="cuda")
    q[:, :, 0] = 1.0
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    ws = torch.zeros(hk.heatkv_paged4_workspace_bytes(pool, b, Hkv * G), dtype=torch.uint8, device="cuda")
    scale = float(np.float32(25.5 * math.log(2) / 7))
    hk.heatkv_paged4_attention(pool, b, q, out, lse, ws, causal=False, sm_scale=scale)
    assert hk.heatkv_paged_status(ws) == 0
    light, value = (pages * PAGE - 1) * math.exp(-7 * scale), float(P.values(*P.quantise(np.ones((1, 16))))[0, 0])
    want, off = value * light / (1 + light), (d + 8) * 2.0**-24 * 7 * scale + 2.0**-18
    sums, products = (pages + 128) * 2.0**-24, 4 * pages * 2.0**-23
    tol = (2 * u + 2 * off + sums + products) * want + pages * PAGE * 2.0**-32 * value
    worst = (float((out.double() - want).abs().max()), float((lse.double() - (7 * scale + math.log1p(light))).abs().max()))
    assert worst[0] <= tol < want / 40, (worst, tol, want)
    assert worst[1] <= off + sums + 2.0**-22 * 20, (worst, off + sums)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("exp", [0, -5, 9])
def test_codes_of_ties_and_of_their_neighbours(hk, dtype, exp):
    """For every scale of four bits and every pair of codes: the number in the middle of them, and the two 16-bit numbers on either side of it."""
    kind = {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    groups = []
    for power in (-4, -1, 0, 2) if dtype == "fp16" else (-6, -4, 0, 5):
        for m in range(8, 16):
            s = m * 2.0 ** (power - 3 + exp)
            ties = torch.tensor([(c + 0.5) * s for c in range(7)], dtype=torch.float64).to(kind)
            assert torch.equal(ties.double(), torch.tensor([(c + 0.5) * s for c in range(7)], dtype=torch.float64))
            near = torch.stack([(ties.view(torch.int16) + by).view(kind) for by in (-2, -1, 0, 1, 2)], 1).flatten()[:34]    # (6.5 s and two steps: below 7 s)
            for x in (near, -near):
                x = torch.cat([x, torch.zeros(-len(x) % 15, dtype=kind)]).view(-1, 15)
                groups.append(torch.cat([torch.full((len(x), 1), 7 * s, dtype=torch.float64).to(kind), x], 1))
    x = torch.cat(groups)
    x = torch.cat([x, torch.zeros(-len(x) % 4, 16, dtype=kind)]).view(-1, 1, 64).cuda()
    n_pages = -(-len(x) // PAGE)
    blocks = torch.zeros(n_pages, 1, hk.PagedPool4.block_bytes(64), dtype=torch.uint8, device="cuda")
    hk.heatkv_paged4_store(hk.PagedPool4.make(blocks, 64, kind, exp, exp), x, x.flip(2).contiguous(), _i32(range(len(x))))
    for got, rows in zip(P.unblock(blocks.cpu().numpy(), 64), (x, x.flip(2))):
        for g, want in zip(got, P.quantise(_np(rows), exp)):
            assert np.array_equal(g[:, 0].reshape(-1, g.shape[-1])[: len(x)], want[:, 0])


@pytest.mark.parametrize("lens,H,Hkv", [
    ([(12, 10000)] * 8, 32, 8), ([(12, 10000)] * 7, 32, 8),                               # three tiles, either side of what the warp-level kernel takes
    ([(6, 5000)] + [(1, 40 + 61 * i) for i in range(23)], 28, 4), ([(6, 5000)] * 40, 28, 4),
    ([(200, 700)] + [(1, 30 + 7 * i) for i in range(60)], 8, 8), ([(900, 2000)] + [(1, 30 + 7 * i) for i in range(60)], 8, 8),
    ([(33, 33)], 1, 1), ([(33, 33), (0, 64), (1, 0)], 2, 2), ([(2, 900)] * 3, 96, 2)])
def test_attention_on_either_side_of_the_kernels_border(hk, lens, H, Hkv):
    """Drafts, chunks among single tokens and small prompts, where the choice of kernel changes."""
    from test_gpu_paged4 import _attend, _filled
    rng, g = np.random.default_rng(len(lens)), torch.Generator("cuda").manual_seed(H)
    pool, b, table, q_begin, kv = _filled(hk, g, rng, lens, Hkv, 64, torch.float16)
    q = torch.empty(b.n_tokens, H, 64, dtype=torch.float16, device="cuda").normal_(generator=g)
    _attend(hk, pool, b, q, lens, table, q_begin, kv, Hkv, dtype="fp16")


@pytest.mark.parametrize("lens", [[(1, 64 * 1248)], [(1, 64 * 1249)], [(1, 64 * 40 + 1)] + [(1, 100 + 67 * i) for i in range(28)],
                                  [(1, 64 * 40 + 1)] + [(1, 100 + 67 * i) for i in range(29)]])
def test_attention_on_either_side_of_the_borders_of_warps(hk, lens):
    """One row tile, eight kv heads of 128 columns, where the number of warps changes."""
    from test_gpu_paged4 import _attend, _filled
    rng, g = np.random.default_rng(len(lens)), torch.Generator("cuda").manual_seed(len(lens))
    pool, b, table, q_begin, kv = _filled(hk, g, rng, lens, 8, 128, torch.bfloat16)
    q = torch.empty(b.n_tokens, 16, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    _attend(hk, pool, b, q, lens, table, q_begin, kv, 8)


@pytest.mark.parametrize("n,width,pages", [(112, 9, 0), (114, 9, 0), (132, 9, 4000), (133, 9, 4000), (197, 9, 16384), (198, 9, 16384), (16, 750, 4000), (16, 751, 4000),
                                           (64, 512, 4000), (64, 513, 4000)])
def test_rows_on_either_side_of_what_one_cta_sees_to(hk, n, width, pages):
    """Forks and compactions where other launches take over: as many rows and entries as one CTA takes, and more (pages 0: as many as there have to be)."""
    from test_gpu_paged4 import _rearranged, _rows_state, _same
    ws = None
    for seed in range(3):
        rng = np.random.default_rng(seed)
        lengths = [int(x) for x in rng.integers(0, 200, n)]
        held = sum(-(-x // PAGE) for x in lengths)
        table, fifo, ring, head, n_pages = _rows_state(hk, lengths, width, max(pages - held - 3, 90), seed)
        assert n_pages == pages or pages == 0
        if ws is None:
            ws = torch.zeros(hk.heatkv_paged_rows_workspace_bytes(n, width, 16384), dtype=torch.uint8, device="cuda")
        fifo = fifo[:90]
        parents, keep = [int(x) for x in rng.integers(-1, n, n)], [int(x) for x in rng.integers(0, 250, n)]
        want = P.fork(parents, keep, lengths, table, fifo)
        got = _rearranged(hk, lambda *a: hk.heatkv_paged_fork(_i32(parents), _i32(keep), *a), lengths, table, ring.copy(), head, 90, n * PAGE, ws)
        _same(got, want, ring.copy(), head, 90, len(want[6]))
        stays = rng.random((n, 200)) < 0.8
        *want, done = P.compact(stays, lengths, table, fifo, sum(lengths))
        mask = torch.from_numpy(stays).cuda()
        got = _rearranged(hk, lambda *a: hk.heatkv_paged_compact(mask, *a), lengths, table, ring.copy(), head, 90, sum(lengths), ws)
        _same(got, want, ring.copy(), head, 90, done)
