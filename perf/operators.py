"""Operators of the paged cache for requests of any length, and what they compute in plain form.

Four operators.  `tables`: block tables and slot maps of a step's requests, from their lengths.  `store`: the new tokens' K/V
rows go to their slots, and pages that fill up get the summary that page selection reads.  `attend`: attention of every
request's new tokens (one, a few drafted ones, a chunk of a prompt, a whole scale of an image) over its pages.  `sparse`: the
pages that a cheap score selects for each query, and attention over those.

The lengths of a case's requests belong to the case; every value comes from the seed.
"""
from __future__ import annotations

import functools
import math
import random

import numpy as np
import torch

own = False

PAGE = 64                                             # tokens of a page
CODE_STEP = float(np.float32(1.0) / np.float32(127.0))   # page and query summaries: codes of 8 bits, scale = largest magnitude / 127
MAX_FLOPS = 8e11                                      # what drawn cases stay within: the largest listed ones
MAX_BYTES = 3.2e9


def _case(name, op, req, new, past, H=16, Hkv=16, d=128, dtype="bf16", **more):
    """req requests of new[0]..new[1] new tokens after past[0]..past[1] cached ones (spread over the logarithm)."""
    return dict(name=name, op=op, req=req, new_lo=new[0], new_hi=new[1], past_lo=past[0], past_hi=past[1], H=H, Hkv=Hkv, d=d,
                dtype=dtype, **more)


def listed():
    return [
        # A decode step of a small batch: nothing but latency.
        _case("tables_decode", "tables", 24, (1, 1), (1, 9000)),
        # A batch of prompts is admitted, a few of them behind a cached prefix.
        _case("tables_prompts", "tables", 300, (7, 4000), (0, 2000)),
        # A decode step's rows, one per request: latency again.
        _case("store_decode", "store", 64, (1, 1), (30, 1500), H=32, Hkv=8),
        # The rows of a batch of prompts.
        _case("store_prompts", "store", 12, (300, 4096), (0, 700)),
        # One request, a short answer to a short prompt: the smallest attention.
        _case("attend_one", "attend", 1, (1, 1), (129, 129), causal=True),
        # Decode of a serving batch with shared heads: every cached byte is read once.
        _case("attend_decode", "attend", 64, (1, 1), (300, 12000), H=32, Hkv=8, causal=True),
        # Drafted tokens to be verified, seven query heads to a kv head.
        _case("attend_drafts", "attend", 24, (1, 6), (40, 8000), H=28, Hkv=4, dtype="fp16", causal=True),
        # Prompts of the larger model's 32 heads, some behind a cached prefix.
        _case("attend_prompts", "attend", 3, (2100, 4096), (1, 2500), H=32, Hkv=32, causal=True),
        # Decode beside one chunk of a long prompt, 40 heads of 64.
        _case("attend_mixed", "attend", 32, (1, 1), (64, 5000), H=40, Hkv=8, d=64, causal=True, chunk=1500, chunk_past=20000),
        # One request with a long context: 32 of 2000 pages.
        _case("sparse_long", "sparse", 1, (1, 1), (131000, 131000), H=32, Hkv=8, pages=32, sink=1, local=2),
        # Decode of a batch, no shared heads.
        _case("sparse_decode", "sparse", 32, (1, 1), (9000, 40000), dtype="fp16", pages=24, sink=1, local=2),
        # A chunk of a long prompt: every query has pages of its own.
        _case("sparse_chunk", "sparse", 1, (2001, 2001), (30000, 30000), H=32, Hkv=4, pages=16, sink=1, local=2),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    while True:
        op = rng.choice(("tables", "store", "attend", "attend", "attend", "sparse", "sparse"))
        Hkv = rng.choice((1, 2, 4, 5, 8, 16, 28))
        H = Hkv * rng.choice((1, 1, 2, 4, 5, 7, 8)) if Hkv < 28 else 28
        if H > 64:
            continue
        c = dict(op=op, H=H, Hkv=Hkv, d=rng.choice((64, 128, 128)), dtype=rng.choice(("bf16", "bf16", "fp16")))
        kind = rng.choice(("one", "drafts", "chunk"))
        if op == "tables":
            c.update(req=_log_int(rng, 1, 2000), past_lo=rng.choice((0, 1)), past_hi=_log_int(rng, 10, 20000))
            top = _log_int(rng, 1, max(1, 400000 // c["req"]))
        else:
            c.update(req=_log_int(rng, 1, 200 if kind != "chunk" else 8), past_lo=_log_int(rng, 1, 500))
            c["past_hi"] = c["past_lo"] + _log_int(rng, 1, 40000)
            top = {"one": 1, "drafts": rng.randint(2, 9), "chunk": _log_int(rng, 10, 4500)}[kind]
        c.update(new_lo=max(1, top // rng.choice((1, 1, 4))), new_hi=top)
        if op == "attend":
            c["causal"] = kind != "chunk" or rng.random() < 0.7
        if op == "sparse":
            c.update(pages=_log_int(rng, 4, 64), sink=rng.randint(0, 1), local=rng.randint(1, 3))
        new, past = _lengths(c)
        w, rows = work(c), len(new) * max(new)
        longest = max(n + p for n, p in zip(new, past))
        # what a state and the plain form hold
        pool = sum(n + p + PAGE for n, p in zip(new, past)) * c["Hkv"] * c["d"] * 4.0
        plain = 0.0
        if op == "attend":
            plain = 4.0 * len(new) * (longest * c["Hkv"] * c["d"] * 2 + max(new) * c["H"] * longest * 3)
        if op == "sparse":
            plain = 8.0 * rows * c["Hkv"] * (c["pages"] * PAGE * c["d"] + longest / PAGE * 2)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES and pool <= 6e9 and plain <= 3e10 and rows * c["H"] * c["d"] <= 3e8:
            return c


def _lengths(case):
    """New and cached tokens of every request: the batch's shape, the same for every seed."""
    rng = random.Random(f"{case['req']} {case['new_lo']} {case['new_hi']} {case['past_lo']} {case['past_hi']}")

    def spread(lo, hi):
        return lo + _log_int(rng, 1, hi - lo + 1) - 1

    new = [spread(case["new_lo"], case["new_hi"]) for _ in range(case["req"])]
    past = [spread(case["past_lo"], case["past_hi"]) for _ in range(case["req"])]
    if case.get("chunk"):
        at = case["req"] // 2
        new[at], past[at] = case["chunk"], case["chunk_past"]
    return new, past


def _pages(tokens):
    return -(-tokens // PAGE)


def work(case):
    new, past = _lengths(case)
    T, d, H, Hkv = sum(new), case["d"], case["H"], case["Hkv"]
    rows = 2.0 * d                                    # bytes of a row of one head
    if case["op"] == "tables":
        fresh = sum(_pages(n + p) - _pages(p) for n, p in zip(new, past))
        return {"bytes": 16.0 * len(new) + 8.0 * fresh + 8.0 * T, "flops": 0.0}
    if case["op"] == "store":
        return {"bytes": 4.0 * T * Hkv * rows + 4.0 * T, "flops": 0.0}
    if case["op"] == "attend":
        if case["causal"]:
            pairs = sum(n * p + n * (n + 1) // 2 for n, p in zip(new, past))
        else:
            pairs = sum(n * (n + p) for n, p in zip(new, past))
        cached = sum(n + p for n, p in zip(new, past))
        return {"bytes": 2.0 * cached * Hkv * rows + 2.0 * T * H * rows + 4.0 * T * H, "flops": 4.0 * d * H * pairs}
    pages = [_pages(n + p) for n, p in zip(new, past)]
    taken = sum(min(c, n * case["pages"]) for c, n in zip(pages, new))      # of one head; no page is read twice
    read = sum(n * min(c, case["pages"]) for c, n in zip(pages, new)) * PAGE
    return {"bytes": sum(pages) * Hkv * (d + 4.0) + 2.0 * taken * PAGE * Hkv * rows + T * (2.0 * H * rows + 4.0 * H + 4.0 * Hkv * case["pages"]),
            "flops": 4.0 * d * H * read + 2.0 * d * Hkv * sum(n * c for n, c in zip(new, pages))}


# ------------------------------------------------------------------------------------------------ inputs

def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    new, past = _lengths(case)
    n, T, H, Hkv, d = len(new), sum(new), case["H"], case["Hkv"], case["d"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float16
    g = torch.Generator("cuda").manual_seed(seed)
    total = [a + b for a, b in zip(new, past)]
    held = [_pages(t) for t in (past if case["op"] == "tables" else total)]
    width = max(_pages(t) for t in total) + 3
    n_pages = sum(_pages(t) for t in total) + 5
    order = torch.randperm(n_pages, generator=g, device="cuda").int()     # which page is whose
    first = np.concatenate([[0], np.cumsum(held)])
    table = torch.full((n, width), -1, dtype=torch.int32)
    row, col = np.repeat(np.arange(n), held), np.concatenate([np.arange(h) for h in held])
    table[row, col] = order[: first[-1]].cpu()
    s = dict(case=case, table=table.cuda(), new=_ints(new), past=_ints(past), T=T, pages_per_row=width,
             q_begin=_ints([0] + list(np.cumsum(new))), kv_len=_ints(total), max_new=max(new), max_kv=max(total))
    if case["op"] == "tables":
        # the free pages, as a ring whose oldest entry is somewhere in the middle
        free = n_pages - int(first[-1])
        head = int(np.random.default_rng(seed).integers(n_pages))
        ring = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
        ring[(head + torch.arange(free, device="cuda")) % n_pages] = order[first[-1]:]
        s.update(ring=ring, state=_ints([head, free, 0, 0]), new_state=_ints([0] * 4), new_begin=_ints([0] * (n + 1)),
                 new_kv=_ints([0] * n), slots=torch.zeros(T, dtype=torch.int32, device="cuda"),
                 positions=torch.zeros(T, dtype=torch.int32, device="cuda"))
        return s
    rand = lambda *shape: torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)    # noqa: E731
    s["k"], s["v"] = rand(n_pages, Hkv, PAGE, d), rand(n_pages, Hkv, PAGE, d)
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), s["new"].long(), output_size=T)
    pos = s["past"][seq] + torch.arange(T, device="cuda") - s["q_begin"][seq]
    s["code"] = torch.zeros(n_pages, Hkv, d, dtype=torch.int8, device="cuda")
    s["scale"] = torch.zeros(n_pages, Hkv, dtype=torch.float32, device="cuda")
    if case["op"] == "store":
        s["slots"] = (s["table"][seq, pos // PAGE] * PAGE + pos % PAGE).int()
        qkv = rand(T, 3, Hkv, d)                      # K and V where a model's projection leaves them
        s["k_new"], s["v_new"] = qkv[:, 1], qkv[:, 2]
        return s
    s["q"] = rand(T, H, d)
    s["out"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros(T, H, dtype=torch.float32, device="cuda")
    # requests of one new token, and the others: (their numbers, their largest number of new tokens, of tokens)
    kinds = [[i for i in range(n) if new[i] == 1], [i for i in range(n) if new[i] > 1]]
    s["groups"] = [(torch.tensor(ids, device="cuda"), max(new[i] for i in ids), max(total[i] for i in ids)) for ids in kinds if ids]
    if case["op"] == "sparse":
        # What a text is about changes every few hundred tokens and comes back: keys of one subject lie together, and the queries
        # of neighbouring tokens look for the same few.
        subjects = torch.empty(24, Hkv, d, device="cuda").normal_(generator=g)
        of_page = torch.randint(24, (n, width // 5 + 1), generator=g, device="cuda").repeat_interleave(5, 1)[:, :width]
        known = s["table"] >= 0
        s["k"][s["table"][known].long()] += subjects[of_page[known]][:, :, None].to(dtype)
        looks = torch.randint(24, (T // 40 + 2,), generator=g, device="cuda").repeat_interleave(40)[:T]
        s["q"] += 0.7 * subjects[looks].repeat_interleave(H // Hkv, 1).to(dtype)
        _summarise(s, torch.arange(n_pages, device="cuda"))
        s["sel"] = torch.zeros(T, Hkv, case["pages"], dtype=torch.int32, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _codes(x):
    """x [.., d] in 32 bits -> (8-bit codes as numbers, scale)."""
    scale = x.abs().amax(-1, keepdim=True) * CODE_STEP
    return torch.where(scale > 0, torch.round(x / scale).clamp(-127, 127), 0.0), scale


def _summarise(s, pages):
    """The mean key of whole pages, summed as a tree: rows i and i + 32, then i and i + 16, and so on."""
    m = s["k"][pages].float()
    m = m[:, :, :32] + m[:, :, 32:]
    m = m[:, :, :16] + m[:, :, 16:]
    m = m[:, :, :8] + m[:, :, 8:]
    m = m[:, :, :4] + m[:, :, 4:]
    m = m[:, :, :2] + m[:, :, 2:]
    code, scale = _codes((m[:, :, 0] + m[:, :, 1]) * (1.0 / PAGE))
    s["code"][pages], s["scale"][pages] = code.to(torch.int8), scale[..., 0]


def _tables(s):
    new, past, table, n_pages = s["new"].long(), s["past"].long(), s["table"], s["ring"].shape[0]
    had, has = (past + PAGE - 1) // PAGE, (past + new + PAGE - 1) // PAGE
    fits = has <= table.shape[1]
    need = torch.where(fits, has - had, 0)
    upto = need.cumsum(0)
    served = fits & ((need == 0) | (upto <= s["state"][1]))
    col = torch.arange(table.shape[1], device="cuda")
    fresh = served[:, None] & (col >= had[:, None]) & (col < has[:, None])
    rank = (upto - need)[:, None] + col - had[:, None]
    table = torch.where(fresh, s["ring"][(s["state"][0] + rank.clamp(min=0)) % n_pages], table)
    begin = torch.cat([new.new_zeros(1), new.cumsum(0)])
    seq = torch.repeat_interleave(torch.arange(len(new), device="cuda"), new, output_size=s["T"])
    pos = past[seq] + torch.arange(s["T"], device="cuda") - begin[seq]
    slots = torch.where(served[seq], table[seq, (pos // PAGE).clamp(max=table.shape[1] - 1)] * PAGE + pos % PAGE, -1)
    took = torch.where(served, need, 0).sum()
    state = torch.stack([(s["state"][0] + took) % n_pages, s["state"][1] - took, (~served).sum(), begin[-1]])
    return {"table": table, "begin": begin.int(), "kv": torch.where(served, past + new, 0).int(), "slots": slots.int(),
            "positions": pos.int(), "state": state.int()}


def _store(s):
    slots = s["slots"].long()
    page, row = slots // PAGE, slots % PAGE
    s["k"][page, :, row], s["v"][page, :, row] = s["k_new"], s["v_new"]
    _summarise(s, page[row == PAGE - 1])


def _softmax(scores, mask, v):
    """scores [.., rows, keys], mask that broadcasts to it, v [.., keys, d]: (weighted sum, logarithm of the sum)."""
    scores = scores.masked_fill(~mask, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    return (p @ v) / total.clamp(min=1e-37), (top + torch.log(total))[..., 0]


def _of_group(s, x, ids, most):
    """The tokens' rows of some requests, [request, most, ..], and where each belongs (T: nowhere)."""
    local = torch.arange(most, device="cuda")
    at = s["q_begin"][ids][:, None] + local
    return x[at.clamp(max=s["T"] - 1)], torch.where(local < s["new"][ids][:, None], at, s["T"]).long()


def _attend_group(s, group, out, lse):
    ids, most, longest = group
    case = s["case"]
    Hkv, d = case["Hkv"], case["d"]
    G = case["H"] // Hkv
    q, at = _of_group(s, s["q"], ids, most)
    n, pages = len(ids), _pages(longest)
    place = s["table"][ids, :pages].clamp(min=0).long()
    k, v = (s[x][place].transpose(1, 2).reshape(n, Hkv, pages * PAGE, d).float() for x in "kv")
    q = q.float().view(n, most, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(n, Hkv, G * most, d)
    key = torch.arange(pages * PAGE, device="cuda")
    seen = (key < s["kv_len"][ids][:, None])[:, None]                              # [n, 1, keys]
    v = v.masked_fill(~seen[..., None], 0.0)
    if case["causal"]:
        seen = seen & (key <= (s["past"][ids][:, None] + torch.arange(most, device="cuda"))[..., None])
    o, l = _softmax((q @ k.transpose(2, 3) / math.sqrt(d)).view(n, Hkv, G, most, -1), seen[:, None, None], v[:, :, None])
    out[at] = o.permute(0, 3, 1, 2, 4).reshape(n, most, Hkv * G, d)
    lse[at] = l.permute(0, 3, 1, 2).reshape(n, most, Hkv * G)


def _attend(s):
    out = torch.zeros(s["T"] + 1, *s["q"].shape[1:], device="cuda")
    lse = torch.zeros(s["T"] + 1, s["q"].shape[1], device="cuda")
    _attend_group(s, s["groups"][0], out, lse)
    if len(s["groups"]) > 1:
        _attend_group(s, s["groups"][1], out, lse)
    return {"out": out[:-1].to(s["q"].dtype), "lse": lse[:-1]}


def _sparse(s):
    case = s["case"]
    T, Hkv, d, n_sel = s["T"], case["Hkv"], case["d"], case["pages"]
    G, n, most, width = case["H"] // Hkv, len(s["new"]), s["max_new"], _pages(s["max_kv"])
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), s["new"].long(), output_size=T)
    pos = s["past"][seq] + torch.arange(T, device="cuda") - s["q_begin"][seq]
    # the score: codes of the group's summed queries times codes of the pages' mean keys, whole numbers below 2^24
    q = s["q"].float().view(T, Hkv, G, d)
    wanted, _ = _codes(functools.reduce(torch.add, q.unbind(2)))
    wanted, at = _of_group(s, wanted, torch.arange(n, device="cuda"), most)         # [n, most, Hkv, d]
    place = s["table"][:, :width].clamp(min=0).long()
    score = torch.einsum("nthd,nphd->nthp", wanted, s["code"][place].float()) * s["scale"][place].transpose(1, 2)[:, None]
    score = torch.empty(T + 1, Hkv, width, device="cuda").index_put_((at,), score)[:T]
    page, last = torch.arange(width, device="cuda"), (pos // PAGE)[:, None, None]
    forced = (page < case["sink"]) | (page > last - case["local"])
    score = score.masked_fill(forced, math.inf).masked_fill(page > last, -math.inf)
    best = torch.sort(score, descending=True, stable=True)[1][..., :n_sel]
    best = torch.nn.functional.pad(best, (0, n_sel - best.shape[-1]), value=width)
    best = torch.sort(torch.where(best > last, width, best))[0]
    taken = best < width
    # attention over them
    place = place[seq[:, None, None], best.clamp(max=width - 1)]
    head = torch.arange(Hkv, device="cuda")[:, None]
    k, v = (s[x][place, head].reshape(T, Hkv, n_sel * PAGE, d).float() for x in "kv")
    key = (best[..., None] * PAGE + torch.arange(PAGE, device="cuda"))
    seen = (taken[..., None] & (key <= pos[:, None, None, None])).view(T, Hkv, n_sel * PAGE)
    v = v.masked_fill(~seen[..., None], 0.0)
    o, l = _softmax(q @ k.transpose(2, 3) / math.sqrt(d), seen[:, :, None], v)
    return {"sel": torch.where(taken, best, -1).int(), "out": o.reshape(T, -1, d).to(s["q"].dtype), "lse": l.reshape(T, -1)}


# ------------------------------------------------------------------------------------------------ one pass

def _framework(s):
    """The handles that a program keeps beside its buffers: made on the first pass on a state."""
    import paper_2605_14877_b200 as hk
    if "pool" not in s and "k" in s:
        s["pool"] = hk.PagedPool.make(s["k"], s["v"], s["code"], s["scale"])
        if "q" in s:
            s["batch"] = hk.PagedBatch.make(s["q_begin"], s["kv_len"], s["table"], s["T"], s["max_new"])
            size = hk.heatkv_paged_workspace_bytes(s["pool"], s["batch"], s["case"]["H"])
            s["workspace"] = torch.zeros(size, dtype=torch.uint8, device="cuda")
    return hk


def run(s):
    op = s["case"]["op"]
    if own:
        hk = _framework(s)
        if op == "tables":
            hk.heatkv_paged_tables(s["new"], s["past"], s["ring"], s["state"], s["new_state"], s["table"], s["new_begin"], s["new_kv"],
                                   s["slots"], s["positions"])
            return {"table": s["table"], "begin": s["new_begin"], "kv": s["new_kv"], "slots": s["slots"], "positions": s["positions"],
                    "state": s["new_state"]}
        if op == "store":
            hk.heatkv_paged_store(s["pool"], s["k_new"], s["v_new"], s["slots"])
        if op == "attend":
            hk.heatkv_paged_attention(s["pool"], s["batch"], s["q"], s["out"], s["lse"], s["workspace"], causal=s["case"]["causal"])
            return {"out": s["out"], "lse": s["lse"]}
        if op == "sparse":
            hk.heatkv_paged_select(s["pool"], s["batch"], s["q"], s["sel"], s["case"]["sink"], s["case"]["local"])
            hk.heatkv_paged_sparse_attention(s["pool"], s["batch"], s["q"], s["sel"], s["out"], s["lse"], s["workspace"])
            return {"sel": s["sel"], "out": s["out"], "lse": s["lse"]}
    elif op == "tables":
        return _tables(s)
    elif op == "store":
        _store(s)
    else:
        return _attend(s) if op == "attend" else _sparse(s)
    # what the codes stand for
    return {"k": s["k"], "v": s["v"], "summary": s["code"] * s["scale"][..., None]}


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    if case["op"] == "tables":
        return None                                    # whole numbers only
    s = prepare(case, seed)
    new, past = _lengths(case)
    T, H, Hkv, d = s["T"], case["H"], case["Hkv"], case["d"]
    G, table = H // Hkv, s["table"].cpu().numpy()
    begin = np.concatenate([[0], np.cumsum(new)])
    if case["op"] == "store":
        k, v, mean = s["k"].double(), s["v"].double(), (s["code"].double() * s["scale"].double()[..., None])
        for i in range(len(new)):
            at = np.arange(past[i], past[i] + new[i])
            page, rows = torch.from_numpy(table[i][at // PAGE]).cuda().long(), slice(int(begin[i]), int(begin[i + 1]))
            k[page, :, torch.from_numpy(at % PAGE).cuda()] = s["k_new"][rows].double()
            v[page, :, torch.from_numpy(at % PAGE).cuda()] = s["v_new"][rows].double()
            full = torch.from_numpy(table[i][at[at % PAGE == PAGE - 1] // PAGE]).cuda().long()
            mean[full] = k[full].mean(2)               # the mean itself, which the 8-bit codes are near
        return {"k": k, "v": v, "summary": mean}
    if 8.0 * Hkv * d * max(n * G * 2 if case["op"] == "attend" else n * case["pages"] * PAGE for n in new) > 4e10:
        return None
    out = torch.zeros(T, H, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(T, H, dtype=torch.float64, device="cuda")
    for i in range(len(new)):
        kv = past[i] + new[i]
        pages = torch.from_numpy(table[i][: _pages(kv)]).cuda().long()
        q = s["q"][int(begin[i]): int(begin[i + 1])].view(new[i], Hkv, G, d)
        at = torch.arange(past[i], kv, device="cuda")
        for h in range(Hkv):
            # a few query rows at a time: the logits of a chunk against every key
            step = max(1, int(2e8) // (G * len(pages) * PAGE))
            keys, values = (s[x][pages, h].reshape(-1, d).double() for x in "kv")
            if case["op"] == "sparse":
                chosen = _chosen(q[:, h].float(), s["code"][pages, h], s["scale"][pages, h], at, case)
            for lo in range(0, new[i], step):
                rows = slice(lo, min(new[i], lo + step))
                logits = torch.einsum("tgd,kd->tgk", q[rows, h].double(), keys) / math.sqrt(d)
                j = torch.arange(keys.shape[0], device="cuda")
                hidden = j[None] >= kv
                if case["op"] == "sparse" or case["causal"]:
                    hidden = hidden | (j[None] > at[rows, None])
                if case["op"] == "sparse":
                    hidden = hidden | ~chosen[rows].repeat_interleave(PAGE, 1)
                logits.masked_fill_(hidden[:, None], -math.inf)
                total = torch.logsumexp(logits, -1)
                t = slice(int(begin[i]) + rows.start, int(begin[i]) + rows.stop)
                lse[t, h * G:(h + 1) * G] = total
                out[t, h * G:(h + 1) * G] = torch.exp(logits - total[..., None]) @ values
    return {"sel": None, "out": out, "lse": lse} if case["op"] == "sparse" else {"out": out, "lse": lse}


def _chosen(q, code, scale, at, case):
    """Which pages each query takes, [t, pages]: the definition's 32-bit steps on the host, the dot product in whole numbers."""
    q, code, scale = q.cpu().numpy(), code.cpu().numpy().astype(np.int64), scale.cpu().numpy()
    wanted = q[:, 0]
    for g in range(1, q.shape[1]):
        wanted = wanted + q[:, g]
    step = np.abs(wanted).max(1, keepdims=True) * np.float32(CODE_STEP)
    wanted = np.where(step > 0, np.clip(np.rint(wanted / np.where(step > 0, step, np.float32(1))), -127, 127), 0).astype(np.int64)
    score = (wanted.astype(np.float64) @ code.T.astype(np.float64)).astype(np.float32) * scale
    last = at.cpu().numpy()[:, None] // PAGE
    page = np.arange(len(code))[None]
    score = np.where((page < case["sink"]) | (page > last - case["local"]), np.inf, score)
    score = np.where(page > last, -np.inf, score)
    best = np.argsort(-score, axis=1, kind="stable")[:, : case["pages"]]
    taken = np.zeros(score.shape, dtype=bool)
    np.put_along_axis(taken, best, True, 1)
    return torch.from_numpy(taken & (page <= last)).cuda()
