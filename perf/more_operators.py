"""More operators of the paged cache: a cache held in 4 bits with the attention that reads it, and what happens to requests' pages between steps.

Four operators.  `store4`: new tokens' K/V rows go to their slots as 4-bit codes with a scale for every 16 columns, and come back as the rows that
attention will see.  `attend4`: attention of every request's new tokens (one, a few drafted ones, a chunk of a prompt) over such a cache.  `fork`: rows
of the block table go on as copies of others (beams, several answers to one prompt), are cut back or end; whole pages are shared, a page that is
not full is copied, and pages that no row lists any longer become free.  `compact`: the tokens that a mask drops leave the cache, the others move
together.

The lengths of a case's requests belong to the case; every value comes from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

PAGE = 64                                             # tokens of a page
GROUP = 16                                            # columns that share a scale
MAX_FLOPS = 4e11                                      # what drawn cases stay within: the largest listed ones
MAX_BYTES = 6e8
# the eight columns of a 4-byte word, by the place of their 4 bits
NIBBLE_OF_COLUMN = (0, 4, 1, 5, 2, 6, 3, 7)


def _case(name, op, req, length, H=16, Hkv=16, d=128, dtype="bf16", **more):
    """req requests of length[0]..length[1] cached tokens (spread over the logarithm)."""
    return dict(name=name, op=op, req=req, past_lo=length[0], past_hi=length[1], H=H, Hkv=Hkv, d=d, dtype=dtype, **more)


def listed():
    return [
        # A decode step's rows, one per request: latency.
        _case("store4_decode", "store4", 64, (30, 1500), H=32, Hkv=8, new_lo=1, new_hi=1),
        # The rows of a batch of prompts, some behind a cached prefix.
        _case("store4_prompts", "store4", 12, (1, 700), new_lo=300, new_hi=4096),
        # One request, a short answer to a short prompt: the smallest attention.
        _case("attend4_one", "attend4", 1, (200, 200), new_lo=1, new_hi=1, causal=True),
        # Decode of a serving batch with shared heads: every cached byte is read once.
        _case("attend4_decode", "attend4", 64, (300, 12000), H=32, Hkv=8, new_lo=1, new_hi=1, causal=True),
        # One request with a long context.
        _case("attend4_long", "attend4", 1, (131000, 131000), H=40, Hkv=8, new_lo=1, new_hi=1, causal=True),
        # Drafted tokens to be verified, seven query heads to a kv head.
        _case("attend4_drafts", "attend4", 24, (40, 8000), H=28, Hkv=4, dtype="fp16", new_lo=1, new_hi=6, causal=True),
        # Chunks of long prompts, heads of 64 as in the small model.
        _case("attend4_chunk", "attend4", 3, (900, 20000), H=40, Hkv=8, d=64, new_lo=500, new_hi=1500, causal=True),
        # A beam search's step: four beams for each of eight requests, of which some go on twice and some end.
        _case("fork_beams", "fork", 32, (100, 2500), H=32, Hkv=8, bits=16, ways=4),
        # A long prompt is answered 96 times over, of a cache in 4 bits.
        _case("fork_samples", "fork", 97, (9001, 9001), H=32, Hkv=8, bits=4, ways=97),
        # Three tenths of a long request's tokens stay.
        _case("compact_long", "compact", 1, (100000, 100000), H=32, Hkv=8, bits=16, part=0.3),
        # A batch whose requests are each cut to half, fp16 and heads of 64.
        _case("compact_batch", "compact", 40, (50, 9000), d=64, dtype="fp16", bits=16, part=0.5),
        # The same of a cache in 4 bits.
        _case("compact4_batch", "compact", 24, (2000, 16000), H=32, Hkv=8, bits=4, part=0.4),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    while True:
        op = rng.choice(("store4", "attend4", "attend4", "attend4", "fork", "compact"))
        Hkv = rng.choice((1, 2, 4, 5, 8, 16, 28))
        H = Hkv * rng.choice((1, 1, 2, 4, 5, 7, 8)) if Hkv < 28 else 28
        if H > 64:
            continue
        c = dict(op=op, H=H, Hkv=Hkv, d=rng.choice((64, 128, 128)), dtype=rng.choice(("bf16", "bf16", "fp16")))
        kind = rng.choice(("one", "drafts", "chunk"))
        c.update(req=_log_int(rng, 1, 200 if kind != "chunk" else 8), past_lo=_log_int(rng, 1, 500))
        c["past_hi"] = c["past_lo"] + _log_int(rng, 1, 40000)
        if op in ("store4", "attend4"):
            top = {"one": 1, "drafts": rng.randint(2, 9), "chunk": _log_int(rng, 10, 4500)}[kind]
            c.update(new_lo=max(1, top // rng.choice((1, 1, 4))), new_hi=top)
        if op == "attend4":
            c["causal"] = kind != "chunk" or rng.random() < 0.7
        if op in ("fork", "compact"):
            c["bits"] = rng.choice((4, 16))
        if op == "fork":
            c["ways"] = rng.choice((2, 4, 8, c["req"]))
        if op == "compact":
            c["part"] = round(rng.uniform(0.1, 0.9), 2)
        new, past = _lengths(c)
        w, rows = work(c), len(new) * max(new)
        longest = max(n + p for n, p in zip(new, past))
        # what a state and the plain form hold
        pool = sum(n + p + PAGE for n, p in zip(new, past)) * c["Hkv"] * c["d"] * (4.0 if c.get("bits") == 16 else 1.2)
        plain = 0.0
        if op == "attend4":
            plain = 4.0 * len(new) * (longest * c["Hkv"] * c["d"] * 5 + max(new) * c["H"] * longest * 3)
        if op == "compact":
            plain = 8.0 * len(new) * longest
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES and pool <= 3e9 and plain <= 3e10 and rows * c["H"] * c["d"] <= 3e8:
            return c


def _lengths(case):
    """New and cached tokens of every request: the batch's shape, the same for every seed."""
    rng = random.Random(f"{case['req']} {case.get('new_lo', 0)} {case.get('new_hi', 0)} {case['past_lo']} {case['past_hi']}")

    def spread(lo, hi):
        return lo + _log_int(rng, 1, hi - lo + 1) - 1

    new = [spread(case["new_lo"], case["new_hi"]) if "new_lo" in case else 0 for _ in range(case["req"])]
    past = [spread(case["past_lo"], case["past_hi"]) for _ in range(case["req"])]
    if case["op"] == "fork":                          # rows of a family begin as copies of its first
        for i in range(case["req"]):
            past[i] = past[i - i % case["ways"]]
    return new, past


def _parents(case):
    """Which row each row goes on from (-1: it ends), and the most tokens that it keeps."""
    _, past = _lengths(case)
    rng = random.Random(f"parents {case['req']} {case['ways']}")
    parents, keep = [], []
    for i in range(case["req"]):
        first = i - i % case["ways"]
        size = min(case["ways"], case["req"] - first)
        if case["ways"] >= case["req"]:               # one request answered many times: all rows but the first are free
            parents.append(0)
        else:                                         # beams: the better ones go on more than once, now and then a request is over
            parents.append(-1 if (first // case["ways"]) % 7 == 5 else first + min(rng.randrange(size), rng.randrange(size)))
        keep.append(past[max(parents[i], 0)] - (rng.randrange(1, 9) if rng.random() < 0.2 else 0))
    return parents, [max(k, 0) for k in keep]


def _dropped(case):
    """(First page with a token that goes, tokens that stay from it on) of every request: a program that drops tokens to a budget knows these."""
    _, past = _lengths(case)
    out = []
    for n in past:
        stay = [_stays(j, n, case["part"]) for j in range(n)] if n <= 4096 else None
        if stay is None:
            period = 997                              # (`_stays` repeats itself between the ends)
            one = [_stays(j + 100 * period, 1 << 30, case["part"]) for j in range(period)]
            stay = [_stays(j, n, case["part"]) if j < 2 * period or j >= n - 2 * period else one[j % period] for j in range(n)]
        first = next((j for j in range(n) if not stay[j]), None)
        out.append((None, 0) if first is None else (first // PAGE, sum(stay[first // PAGE * PAGE:])))
    return out


def _stays(j, n, part):
    """The first four tokens and the last thirty-two stay, of the others about `part`."""
    return j < 4 or j >= n - 32 or (j % 997 * 619) % 997 < part * 997


def _pages(tokens):
    return -(-tokens // PAGE)


def work(case):
    new, past = _lengths(case)
    T, d, H, Hkv = sum(new), case["d"], case["H"], case["Hkv"]
    row, row4 = 2.0 * d, d * 9 / 16                   # bytes of a row of one head, in 16 and in 4 bits
    if case["op"] == "store4":                        # both ways
        return {"bytes": 2 * T * Hkv * 2 * (row + row4) + 8.0 * T, "flops": 0.0}
    if case["op"] == "attend4":
        if case["causal"]:
            pairs = sum(n * p + n * (n + 1) // 2 for n, p in zip(new, past))
        else:
            pairs = sum(n * (n + p) for n, p in zip(new, past))
        cached = sum(n + p for n, p in zip(new, past))
        return {"bytes": 2.0 * cached * Hkv * row4 + 2.0 * T * H * row + 4.0 * T * H, "flops": 4.0 * d * H * pairs}
    entries = sum(_pages(p) for p in past)
    if case["op"] == "fork":
        parents, keep = _parents(case)
        # a page that is not full stays with one of the rows that go on from it
        last = [(p, k // PAGE) for p, k in zip(parents, keep) if p >= 0 and k % PAGE]
        moved = sum(k % PAGE for p, k in zip(parents, keep) if p >= 0) * (1 - len(set(last)) / max(len(last), 1))
        table = 8.0 * entries
    else:
        moved = sum(m for _, m in _dropped(case))
        table = 4.0 * entries + sum(past) + 8.0 * moved
    each = row if case["bits"] == 16 else row4
    back = 0.0 if case["bits"] == 16 else 2.0 * moved * Hkv * (row + row4)
    return {"bytes": table + 2.0 * moved * Hkv * 2 * each + back, "flops": 0.0}


# ------------------------------------------------------------------------------------------------ inputs

def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    new, past = _lengths(case)
    n, T, H, Hkv, d = len(new), sum(new), case["H"], case["Hkv"], case["d"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float16
    g = torch.Generator("cuda").manual_seed(seed)
    total = [a + b for a, b in zip(new, past)]
    width = max(_pages(t) for t in total) + 3
    held = [_pages(t) for t in total]
    if case["op"] == "fork":
        one = case["ways"] >= case["req"]             # only the first row is there yet
        held = [0 if one and i else _pages(past[i]) for i in range(n)]
        shared = [_pages(past[i]) - 1 if not one and i % case["ways"] else 0 for i in range(n)]    # pages that a row has from its family's first
        held = [h - s for h, s in zip(held, shared)]
    spare = {"fork": n + 9, "compact": sum(held) + 9}.get(case["op"], 5)
    n_pages = sum(held) + spare
    order = torch.randperm(n_pages - 1, generator=g, device="cuda").int()          # which page is whose (the last one is nobody's)
    table = torch.full((n, width), -1, dtype=torch.int32)
    at, pages = 0, order.cpu()
    for i in range(n):
        skip = 0
        if case["op"] == "fork" and shared[i]:
            skip = shared[i]
            table[i, :skip] = table[i - i % case["ways"], :skip]
        table[i, skip: skip + held[i]] = pages[at: at + held[i]]
        at += held[i]
    s = dict(case=case, table=table.cuda(), n_pages=n_pages, dtype=dtype)
    rand = lambda *shape: torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)    # noqa: E731
    if case["op"] in ("store4", "attend4"):
        s.update(new=_ints(new), past=_ints(past), T=T, q_begin=_ints([0] + torch.tensor(new).cumsum(0).tolist()), kv_len=_ints(total),
                 max_new=max(new), max_kv=max(total))
        s["blocks"] = torch.zeros(n_pages, Hkv, PAGE * (d + d // 8), dtype=torch.uint8, device="cuda")
    if case["op"] == "store4":
        seq = torch.repeat_interleave(torch.arange(n, device="cuda"), s["new"].long(), output_size=T)
        pos = s["past"][seq] + torch.arange(T, device="cuda") - s["q_begin"][seq]
        s["slots"] = (s["table"][seq, pos // PAGE] * PAGE + pos % PAGE).int()
        qkv = rand(T, 3, Hkv, d)                      # K and V where a model's projection leaves them
        qkv[:, 1] *= _channels(g, Hkv, d).to(dtype)
        s["k_new"], s["v_new"] = qkv[:, 1], qkv[:, 2]
        s["k_back"], s["v_back"] = torch.zeros(T, Hkv, d, dtype=dtype, device="cuda"), torch.zeros(T, Hkv, d, dtype=dtype, device="cuda")
        return s
    if case["op"] == "attend4":
        size = _channels(g, Hkv, d)[:, None]
        step = max(1, int(3e7) // (Hkv * PAGE * d))
        for lo in range(0, n_pages, step):
            count = min(step, n_pages - lo)
            k, v = (torch.empty(count, Hkv, PAGE, d, device="cuda").normal_(generator=g) for _ in "kv")
            _put(s["blocks"][lo: lo + count], slice(None), slice(None), _quantise((k * size).to(dtype)), _quantise(v.to(dtype)), d)
        s["q"] = (rand(T, H, d).float() / size.squeeze(1).repeat_interleave(H // Hkv, 0) * 1.5).to(dtype)
        s["out"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros(T, H, dtype=torch.float32, device="cuda")
        # requests of one new token, and the others: (their numbers, their largest number of new tokens, of tokens)
        kinds = [[i for i in range(n) if new[i] == 1], [i for i in range(n) if new[i] > 1]]
        s["groups"] = [(torch.tensor(ids, device="cuda"), max(new[i] for i in ids), max(total[i] for i in ids)) for ids in kinds if ids]
        return s
    # the free pages, as a ring whose oldest entry is somewhere in the middle
    free, head = n_pages - 1 - at, int(torch.randint(n_pages, (1,), generator=g, device="cuda"))
    ring = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    ring[(head + torch.arange(free, device="cuda")) % n_pages] = order[at:]
    s.update(ring=ring, state=_ints([head, free, 0, 0]), new_state=_ints([0] * 4), lengths=_ints(past), new_lengths=_ints([0] * n),
             new_table=torch.zeros_like(s["table"]))
    if case["op"] == "fork":
        parents, keep = _parents(case)
        if one:
            s["lengths"][1:] = 0
        s.update(parents=_ints(parents), keep=_ints(keep))
        n_moves = n * PAGE
    else:
        j, lengths = torch.arange(width * PAGE, device="cuda"), s["lengths"][:, None]
        s["stays"] = (j < 4) | (j >= lengths - 32) | ((j % 997 * 619) % 997 < case["part"] * 997)
        n_moves = max(sum(m for _, m in _dropped(case)), 1)
    s["moves"] = (_ints([0] * n_moves), _ints([0] * n_moves))
    if case["bits"] == 16:
        s["k"], s["v"] = rand(n_pages, Hkv, PAGE, d), rand(n_pages, Hkv, PAGE, d)
        return s
    s["blocks"] = torch.randint(0, 256, (n_pages, Hkv, PAGE * (d + d // 8)), dtype=torch.uint8, generator=g, device="cuda")
    scales = s["blocks"][:, :, PAGE * d:]
    scales.remainder_(48).add_(24)                    # of values between 1/32 and 7 or so
    s["k_back"], s["v_back"] = (torch.zeros(n_moves, Hkv, d, dtype=dtype, device="cuda") for _ in "kv")
    return s


def _channels(g, Hkv, d):
    """The sizes of keys' columns: most about one, a few several times that, as models have them."""
    size = torch.empty(Hkv, d, device="cuda").uniform_(0.5, 1.5, generator=g)
    return size * (1 + 5 * (torch.empty(Hkv, d, device="cuda").uniform_(generator=g) > 0.95))


# ------------------------------------------------------------------------------------------------ plain forms

def _quantise(x):
    """x [.., d] -> (codes + 8 as whole numbers [.., d], scales as bytes [.., d / 16])."""
    x = x.float().unflatten(-1, (-1, GROUP))
    scale = (x.abs().amax(-1) * (1.0 / 7.0)).clamp(max=448.0).to(torch.float8_e4m3fn)
    s = scale.float()[..., None]
    code = torch.where(s > 0, torch.round(x / s).clamp(-7, 7), 0.0)
    return (code + 8).to(torch.uint8).flatten(-2), scale.view(torch.uint8)


def _put(blocks, head, row, k, v, d):
    """Codes and scales of K and V to places [page, head, row] of blocks [pages, heads, bytes]."""
    codes, scales = _parts(blocks, d)
    for i, (code, scale) in enumerate((k, v)):
        code = code.unflatten(-1, (-1, 4, 2))         # words of (even, odd) pairs
        byte = code[..., 0::2, :] | code[..., 1::2, :] << 4                        # [.., word, half, even or odd]
        codes[i][:, head, row] = byte.transpose(-1, -2).flatten(-3)
        scales[i][:, head, row] = scale


def _parts(blocks, d):
    """The codes [pages, heads, 64, d / 2] and scales [pages, heads, 64, d / 16] of K and of V."""
    def part(at, each):
        return blocks[:, :, PAGE * at: PAGE * (at + each)].unflatten(-1, (PAGE, each))

    return (part(0, d // 2), part(d // 2, d // 2)), (part(d, d // GROUP), part(d + d // GROUP, d // GROUP))


def _values(code, scale):
    """Bytes [.., d / 2] and [.., d / 16] -> the values [.., d] that they stand for, in 32 bits."""
    word = code.unflatten(-1, (-1, 2, 2))             # [.., word, even or odd, half]
    nibble = torch.stack([word & 15, word >> 4], -1)  # [.., word, even or odd, half, low or high]
    number = nibble.permute(*range(nibble.dim() - 3), -2, -1, -3).flatten(-4).float() - 8
    return (number.unflatten(-1, (-1, GROUP)) * scale.view(torch.float8_e4m3fn).float()[..., None]).flatten(-2)


def _rows4(s, slots):
    """The rows of some slots, as 16-bit numbers (slots below 0: zeros)."""
    page, row = slots.clamp(min=0).long() // PAGE, slots.clamp(min=0).long() % PAGE
    codes, scales = _parts(s["blocks"], s["case"]["d"])
    return [torch.where((slots >= 0)[:, None, None], _values(c[page, :, row], x[page, :, row]), 0.0).to(s["dtype"]) for c, x in zip(codes, scales)]


def _store4(s):
    d, slots = s["case"]["d"], s["slots"].long()
    codes, scales = _parts(s["blocks"], d)
    for i, x in enumerate((s["k_new"], s["v_new"])):
        code, scale = _quantise(x)
        code = code.unflatten(-1, (-1, 4, 2))
        codes[i][slots // PAGE, :, slots % PAGE] = (code[..., 0::2, :] | code[..., 1::2, :] << 4).transpose(-1, -2).flatten(-3)
        scales[i][slots // PAGE, :, slots % PAGE] = scale
    k, v = _rows4(s, s["slots"])
    return {"k": k, "v": v}


def _softmax(scores, mask, v):
    """scores [.., rows, keys], mask that broadcasts to it, v [.., keys, d]: (weighted sum, logarithm of the sum)."""
    scores = scores.masked_fill(~mask, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    return (p @ v) / total.clamp(min=1e-37), (top + torch.log(total))[..., 0]


def _attend_group(s, group, out, lse):
    ids, most, longest = group
    case = s["case"]
    Hkv, d = case["Hkv"], case["d"]
    G = case["H"] // Hkv
    local = torch.arange(most, device="cuda")
    at = s["q_begin"][ids][:, None] + local
    q, at = s["q"][at.clamp(max=s["T"] - 1)], torch.where(local < s["new"][ids][:, None], at, s["T"]).long()
    n, pages = len(ids), _pages(longest)
    place = s["table"][ids, :pages].clamp(min=0).long()
    codes, scales = _parts(s["blocks"][place].flatten(0, 1), d)
    k, v = (_values(c, x).unflatten(0, (n, pages)).transpose(1, 2).reshape(n, Hkv, pages * PAGE, d) for c, x in zip(codes, scales))
    q = q.float().view(n, most, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(n, Hkv, G * most, d)
    key = torch.arange(pages * PAGE, device="cuda")
    seen = (key < s["kv_len"][ids][:, None])[:, None]                              # [n, 1, keys]
    v = v.masked_fill(~seen[..., None], 0.0)
    if case["causal"]:
        seen = seen & (key <= (s["past"][ids][:, None] + local)[..., None])
    o, l = _softmax((q @ k.transpose(2, 3) / math.sqrt(d)).view(n, Hkv, G, most, -1), seen[:, None, None], v[:, :, None])
    out[at] = o.permute(0, 3, 1, 2, 4).reshape(n, most, Hkv * G, d)
    lse[at] = l.permute(0, 3, 1, 2).reshape(n, most, Hkv * G)


def _attend4(s):
    out = torch.zeros(s["T"] + 1, *s["q"].shape[1:], device="cuda")
    lse = torch.zeros(s["T"] + 1, s["q"].shape[1], device="cuda")
    for group in s["groups"]:
        _attend_group(s, group, out, lse)
    return {"out": out[:-1].to(s["dtype"]), "lse": lse[:-1]}


def _freed(s, listed):
    """Pages of the old table that `listed` (a truth value for every page and one more) no longer has go to the ring's end, in page order."""
    n_pages, col = s["n_pages"], torch.arange(s["table"].shape[1], device="cuda")
    had = torch.zeros(n_pages + 1, dtype=torch.bool, device="cuda")
    had[torch.where(col < (s["lengths"][:, None] + PAGE - 1) // PAGE, s["table"], n_pages).long()] = True
    gone = (had & ~listed)[:-1]
    place = (s["state"][0] + s["state"][1] + gone.cumsum(0) - 1) % n_pages
    ring = torch.cat([s["ring"], s["ring"][:1]])
    ring[torch.where(gone, place, n_pages)] = torch.arange(n_pages, dtype=torch.int32, device="cuda")
    s["ring"].copy_(ring[:-1])
    return gone.sum()


def _fork(s):
    table, n_pages, n = s["table"], s["n_pages"], len(s["parents"])
    width, rows, col = table.shape[1], torch.arange(n, device="cuda"), torch.arange(table.shape[1], device="cuda")
    parents = s["parents"].long()
    length = torch.where(parents >= 0, torch.minimum(s["lengths"][parents.clamp(min=0)], s["keep"]), 0).long()
    whole, rest = length // PAGE, length % PAGE
    table = table[parents.clamp(min=0)].long()
    full = torch.zeros(n_pages + 1, dtype=torch.bool, device="cuda")
    full[torch.where(col < whole[:, None], table, n_pages)] = True
    listed = full.clone()
    last = torch.where(rest > 0, table.gather(1, whole.clamp(max=width - 1)[:, None])[:, 0], n_pages)
    listed[last] = True
    # a page that is not full is its own row's, else the lowest row's, unless another row has it whole
    rank = torch.where(parents == rows, rows, rows + n)
    keeper = torch.full((n_pages + 1,), 2 * n, device="cuda").scatter_reduce(0, last, rank, "amin")
    wants = (rest > 0) & (full[last] | (keeper[last] != rank))
    place = wants.cumsum(0) - 1
    served = wants & (place < s["state"][1])
    fresh = s["ring"][(s["state"][0] + place.clamp(min=0)) % n_pages].long()
    length = torch.where(wants & ~served, whole * PAGE, length)
    table = torch.where(served[:, None] & (col == whole[:, None]), fresh[:, None], table)
    table = torch.where(col < ((length + PAGE - 1) // PAGE)[:, None], table, -1)
    r = torch.arange(PAGE, device="cuda")
    moved = served[:, None] & (r < rest[:, None])
    source, target = (torch.where(moved, x[:, None] * PAGE + r, -1).flatten().int() for x in (last, fresh))
    gone, took = _freed(s, listed), served.sum()
    state = torch.stack([(s["state"][0] + took) % n_pages, s["state"][1] - took + gone, (wants & ~served).sum(), gone])
    return {"table": table.int(), "lengths": length.int(), "state": state.int(), "ring": s["ring"], "from": source, "to": target}


def _compact(s):
    table, n_pages, count = s["table"].long(), s["n_pages"], len(s["moves"][0])
    n, width = table.shape
    col, token = torch.arange(width, device="cuda"), torch.arange(width * PAGE, device="cuda")
    length = s["lengths"].long()
    there = token < length[:, None]
    stays, goes = there & s["stays"], there & ~s["stays"]
    first = torch.where(goes.any(1), goes.int().argmax(1) // PAGE, width)          # the first page that something leaves
    moves = stays & (token >= first[:, None] * PAGE)
    m = moves.sum(1)
    need = (m + PAGE - 1) // PAGE
    upto, moved_upto = need.cumsum(0), m.cumsum(0)
    served = goes.any(1) & ((need == 0) | ((upto <= s["state"][1]) & (moved_upto <= count)))
    moves = moves & served[:, None]
    new_length = torch.where(served, first * PAGE + m, length)
    rank = (upto - need)[:, None] + col - first[:, None]
    fresh = served[:, None] & (col >= first[:, None]) & (col < (first + need)[:, None])
    new_table = torch.where(fresh, s["ring"][(s["state"][0] + rank.clamp(min=0)) % n_pages].long(), table)
    new_table = torch.where(col < ((new_length + PAGE - 1) // PAGE)[:, None], new_table, -1)
    # the moves, request by request
    place = torch.where(moves, moves.flatten().cumsum(0).view_as(moves) - 1, count)
    to = first[:, None] * PAGE + moves.cumsum(1) - 1
    source = torch.full((count + 1,), -1, device="cuda")
    target = source.clone()
    source[place] = table.repeat_interleave(PAGE, 1) * PAGE + token % PAGE
    target[place] = new_table.gather(1, (to // PAGE).clamp(0, width - 1)) * PAGE + to % PAGE
    listed = torch.zeros(n_pages + 1, dtype=torch.bool, device="cuda")
    listed[torch.where((col < ((new_length + PAGE - 1) // PAGE)[:, None]) & ~fresh, table, n_pages)] = True
    gone, took = _freed(s, listed), torch.where(served, need, 0).sum()
    state = torch.stack([(s["state"][0] + took) % n_pages, s["state"][1] - took + gone, ((need > 0) & ~served).sum(), moves.sum()])
    return {"table": new_table.int(), "lengths": new_length.int(), "state": state.int(), "ring": s["ring"], "from": source[:-1].int(), "to": target[:-1].int()}


def _move(s, source, target):
    spare = (s["n_pages"] - 1) * PAGE                 # what is nobody's stays where it is
    a, b = (torch.where(source >= 0, x, spare).long() for x in (source, target))
    if s["case"]["bits"] == 16:
        for x in (s["k"], s["v"]):
            x[b // PAGE, :, b % PAGE] = x[a // PAGE, :, a % PAGE]
        return {"k": s["k"], "v": s["v"]}
    codes, scales = _parts(s["blocks"], s["case"]["d"])
    for x in codes + scales:
        x[b // PAGE, :, b % PAGE] = x[a // PAGE, :, a % PAGE]
    k, v = _rows4(s, target)
    return {"k": k, "v": v}


# ------------------------------------------------------------------------------------------------ one pass

def _framework(s):
    """The handles that a program keeps beside its buffers: made on the first pass on a state."""
    import paper_2605_14877_b200 as hk
    if "pool" not in s:
        case, zeros = s["case"], lambda size: torch.zeros(size, dtype=torch.uint8, device="cuda")     # noqa: E731
        s["pool"] = hk.PagedPool4.make(s["blocks"], case["d"], s["dtype"]) if "blocks" in s else hk.PagedPool.make(s["k"], s["v"])
        if case["op"] == "attend4":
            s["batch"] = hk.PagedBatch.make(s["q_begin"], s["kv_len"], s["table"], s["T"], s["max_new"])
            s["workspace"] = zeros(hk.heatkv_paged4_workspace_bytes(s["pool"], s["batch"], case["H"]))
        if case["op"] in ("fork", "compact"):
            s["workspace"] = zeros(hk.heatkv_paged_rows_workspace_bytes(*s["table"].shape, s["n_pages"]))
    return hk


def run(s):
    op = s["case"]["op"]
    if not own:
        if op in ("store4", "attend4"):
            return _store4(s) if op == "store4" else _attend4(s)
        out = _fork(s) if op == "fork" else _compact(s)
        return {**out, **_move(s, out["from"], out["to"])}
    hk = _framework(s)
    if op == "store4":
        hk.heatkv_paged4_store(s["pool"], s["k_new"], s["v_new"], s["slots"])
        hk.heatkv_paged4_load(s["pool"], s["slots"], s["k_back"], s["v_back"])
        return {"k": s["k_back"], "v": s["v_back"]}
    if op == "attend4":
        hk.heatkv_paged4_attention(s["pool"], s["batch"], s["q"], s["out"], s["lse"], s["workspace"], causal=s["case"]["causal"])
        return {"out": s["out"], "lse": s["lse"]}
    rows = (s["lengths"], s["table"], s["ring"], s["state"], s["new_lengths"], s["new_table"], s["new_state"], *s["moves"], s["workspace"])
    if op == "fork":
        hk.heatkv_paged_fork(s["parents"], s["keep"], *rows)
    else:
        hk.heatkv_paged_compact(s["stays"], *rows)
    out = {"table": s["new_table"], "lengths": s["new_lengths"], "state": s["new_state"], "ring": s["ring"], "from": s["moves"][0], "to": s["moves"][1]}
    if s["case"]["bits"] == 16:
        hk.heatkv_paged_move(s["pool"], *s["moves"])
        return {**out, "k": s["k"], "v": s["v"]}
    hk.heatkv_paged4_move(s["pool"], *s["moves"])
    hk.heatkv_paged4_load(s["pool"], s["moves"][1], s["k_back"], s["v_back"])
    return {**out, "k": s["k_back"], "v": s["v_back"]}


# ------------------------------------------------------------------------------------------------ in 64 bits

def _exact_rows(block, d):
    """The 64 rows of K and of V of one page and head or of many, block [.., bytes], by the format's definition."""
    out = []
    for part in range(2):
        code = block[..., part * PAGE * d // 2: (part + 1) * PAGE * d // 2].reshape(*block.shape[:-1], PAGE, d // 8, 4).long()
        word = code[..., 0] + code[..., 1] * 256 + code[..., 2] * 65536 + code[..., 3] * 16777216
        number = torch.stack([(word // 16 ** i) % 16 - 8 for i in NIBBLE_OF_COLUMN], -1).flatten(-2).double()
        at = PAGE * d + part * PAGE * d // GROUP
        byte = block[..., at: at + PAGE * d // GROUP].reshape(*block.shape[:-1], PAGE, d // GROUP).long()
        power, rest = byte // 8, byte % 8
        powers = torch.tensor([2.0 ** (k - 10) for k in range(32)], dtype=torch.float64, device=block.device)
        scale = torch.where(power > 0, (8 + rest).double() * powers[power], rest.double() / 512)
        out.append(number * scale.repeat_interleave(GROUP, -1))
    return out


def _exact_codes(x):
    """What a row's 4-bit form stands for: the scale by the e4m3 numbers' definition, codes to the nearest, ties to even."""
    x = x.double().unflatten(-1, (-1, GROUP))
    want = (x.abs().amax(-1).float() * torch.tensor(1.0 / 7.0, dtype=torch.float32, device=x.device)).double().clamp(max=448.0)
    powers = torch.tensor([2.0 ** k for k in range(-6, 9)], dtype=torch.float64, device=x.device)
    step = powers[(torch.searchsorted(powers, want.contiguous(), right=True) - 1).clamp(min=0)] / 8
    scale = (torch.round(want / step) * step)[..., None]
    return torch.where(scale > 0, torch.round(x / scale.clamp(min=1e-30)).clamp(-7, 7) * scale, 0.0).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    new, past = _lengths(case)
    T, H, Hkv, d = sum(new), case["H"], case["Hkv"], case["d"]
    if case["op"] == "store4":
        return {"k": _exact_codes(s["k_new"]), "v": _exact_codes(s["v_new"])}
    if case["op"] in ("fork", "compact"):
        return _exact_moves(s)
    G, table = H // Hkv, s["table"].cpu()
    if 8.0 * Hkv * d * max(n * G * 2 for n in new) > 4e10:
        return None
    out = torch.zeros(T, H, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(T, H, dtype=torch.float64, device="cuda")
    begin = 0
    for i in range(len(new)):
        kv = past[i] + new[i]
        pages = table[i, : _pages(kv)].cuda().long()
        at = torch.arange(past[i], kv, device="cuda")
        for h in range(Hkv):
            # a few query rows at a time: the logits of a chunk against every key
            step = max(1, int(2e8) // (G * len(pages) * PAGE))
            keys, values = (x.reshape(-1, d) for x in _exact_rows(s["blocks"][pages, h], d))
            for lo in range(0, new[i], step):
                rows = slice(begin + lo, begin + min(new[i], lo + step))
                q = s["q"][rows, h * G: (h + 1) * G].double()
                logits = torch.einsum("tgd,kd->tgk", q, keys) / math.sqrt(d)
                j = torch.arange(keys.shape[0], device="cuda")
                hidden = (j >= kv)[None]
                if case["causal"]:
                    hidden = hidden | (j[None] > at[lo: lo + len(q), None])
                logits.masked_fill_(hidden[:, None], -math.inf)
                total = torch.logsumexp(logits, -1)
                lse[rows, h * G: (h + 1) * G] = total
                out[rows, h * G: (h + 1) * G] = torch.exp(logits - total[..., None]) @ values
        begin += new[i]
    return {"out": out, "lse": lse}


def _exact_moves(s):
    """Where rows lie afterwards, by a walk over the requests; whole numbers are left to the comparison with the plain form."""
    case, table, ring = s["case"], s["table"].tolist(), s["ring"].tolist()
    head, n_pages, width = int(s["state"][0]), s["n_pages"], s["table"].shape[1]
    lengths, pairs, taken = s["lengths"].tolist(), [], 0
    if case["op"] == "fork":
        parents, keep = s["parents"].tolist(), s["keep"].tolist()
        cut = [min(lengths[p], k) if p >= 0 else 0 for p, k in zip(parents, keep)]
        whole = {table[p][j] for p, c in zip(parents, cut) for j in range(c // PAGE)}
        mine = {}
        for i in sorted(range(len(parents)), key=lambda i: (parents[i] != i, i)):
            if cut[i] % PAGE:
                mine.setdefault(table[parents[i]][cut[i] // PAGE], i)
        slots = [[-1, -1]] * (len(parents) * PAGE)
        for i, (p, c) in enumerate(zip(parents, cut)):
            if c % PAGE and (table[p][c // PAGE] in whole or mine[table[p][c // PAGE]] != i):
                a, b = table[p][c // PAGE], ring[(head + taken) % n_pages]
                taken += 1
                for r in range(c % PAGE):
                    slots[i * PAGE + r] = [a * PAGE + r, b * PAGE + r]
        pairs = slots
    else:
        stays = s["stays"].cpu().numpy()
        for i, n in enumerate(lengths):
            gone = [j for j in range(n) if not stays[i][j]] if n < 1000 else (~stays[i][:n]).nonzero()[0].tolist()
            if not gone:
                continue
            first = gone[0] // PAGE * PAGE
            staying = [j for j in range(first, n) if stays[i][j]]
            for k, j in enumerate(staying):
                pairs.append([table[i][j // PAGE] * PAGE + j % PAGE, ring[(head + taken + k // PAGE) % n_pages] * PAGE + k % PAGE])
            taken += -(-len(staying) // PAGE)
        pairs += [[-1, -1]] * (len(s["moves"][0]) - len(pairs))
    none = {"table": None, "lengths": None, "state": None, "ring": None, "from": None, "to": None}
    pairs = torch.tensor(pairs, device="cuda")
    there = pairs[:, 0] >= 0
    a, b = pairs[there].unbind(1)
    if case["bits"] == 16:
        k, v = s["k"].double(), s["v"].double()
        for x in (k, v):
            x[b // PAGE, :, b % PAGE] = x[a // PAGE, :, a % PAGE]
        return {**none, "k": k, "v": v}
    out = [torch.zeros(len(pairs), case["Hkv"], case["d"], dtype=torch.float64, device="cuda") for _ in "kv"]
    where = there.nonzero()[:, 0]
    step = max(1, int(2e7) // (case["Hkv"] * PAGE * case["d"]))
    for lo in range(0, len(a), step):                 # (a page of each, and of it one row)
        rows = torch.arange(len(a[lo: lo + step]), device="cuda")
        for x, page in zip(out, _exact_rows(s["blocks"][a[lo: lo + step] // PAGE], case["d"])):
            x[where[lo: lo + step]] = page[rows, :, a[lo: lo + step] % PAGE]
    return {**none, "k": out[0], "v": out[1]}
